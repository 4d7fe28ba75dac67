"""Cases and plain forms of the operators around the INT8 KV cache.

  rotate   norm and position rotation of the heads' queries and keys (slim_norm_rope)
  append   the same, the keys and values going into the INT8 cache in that pass (slim_norm_rope_append)
  shared   decode attention of a batch whose sequences share a long prefix (slim_attn_decode_shared)
  weights  decode attention that also accumulates every cached token's attention weight (slim_attn_decode_weights)
  evict    eviction from the cache by accumulated weight (slim_kv_evict)

`own` False: elementary torch operations.  `own` True: the calls a user makes of the library.
"""
import math

import torch

own = False

D = 128          # head dimension
PAGE = 128       # token positions per page
EPS = 1e-6


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a batch of 16, 32 query and 32 kv heads: the new tokens' projections, latency counts
        {"name": "rotate_step_b16_32x32", "op": "rotate", "tokens": 16, "hq": 32, "hkv": 32, "rotary": 128, "axes": 1, "inter": False,
         "norm": True, "theta": 10000.0, "far": 2048},
        # a prompt of 8192 tokens in the same layer, queries and keys read out of the fused projection's rows
        {"name": "rotate_prompt_8192_32x32", "op": "rotate", "tokens": 8192, "hq": 32, "hkv": 32, "rotary": 128, "axes": 1, "inter": False,
         "norm": True, "theta": 10000.0, "far": 8192},
        # sixteen prompts of 256 to 4096 tokens, 64 query heads on 8 kv heads, positions with three axes (images in the prompts)
        {"name": "append_ragged_b16_64x8", "op": "append", "batch": 16, "lo": 256, "hi": 4096, "hq": 64, "hkv": 8, "rotary": 128, "axes": 3,
         "inter": False, "norm": True, "theta": 1000000.0, "lens": 1},
        # one long prompt, 32 query heads on 2 kv heads, half of every head rotated in adjacent pairs, no norms
        {"name": "append_16384_32x2", "op": "append", "batch": 1, "lo": 16384, "hi": 16384, "hq": 32, "hkv": 2, "rotary": 64, "axes": 1,
         "inter": True, "norm": False, "theta": 500000.0, "lens": 2},
        # sixteen conversations behind one system prompt of 2048 tokens, one query head per kv head
        {"name": "shared_b16_32x32_2048", "op": "shared", "groups": 1, "batch": 16, "prefix": 2048, "lo": 1, "hi": 256, "hq": 32, "hkv": 32, "lens": 3},
        # a batch of 32 questions about one document of 8192 tokens, 64 query heads on 8 kv heads
        {"name": "shared_b32_64x8_8192", "op": "shared", "groups": 1, "batch": 32, "prefix": 8192, "lo": 64, "hi": 1024, "hq": 64, "hkv": 8, "lens": 4},
        # four documents of 16384 tokens, sixteen samples each, 32 query heads on 2 kv heads
        {"name": "shared_4xb16_32x2_16384", "op": "shared", "groups": 4, "batch": 64, "prefix": 16384, "lo": 1, "hi": 2048, "hq": 32, "hkv": 2, "lens": 5},
        # a short single sequence: the smallest decode step, latency counts
        {"name": "weights_b1_32x32_272", "op": "weights", "batch": 1, "lo": 272, "hi": 272, "hq": 32, "hkv": 32, "lens": 6},
        # the ragged batch of the grouped-query decode workload
        {"name": "weights_b32_64x8_4096", "op": "weights", "batch": 32, "lo": 1024, "hi": 4096, "hq": 64, "hkv": 8, "lens": 7},
        # every step of a batch of 16 drops one token of a full budget of 2048
        {"name": "evict_one_b16_32x32_2049", "op": "evict", "batch": 16, "lo": 2049, "hi": 2049, "hq": 32, "hkv": 32, "budget": 2048, "sink": 4,
         "recent": 256, "lens": 8},
        # a ragged batch of up to 4096 tokens cut back to 1024 at once
        {"name": "evict_b32_64x8_4096_to_1024", "op": "evict", "batch": 32, "lo": 1024, "hi": 4096, "hq": 64, "hkv": 8, "budget": 1024, "sink": 4,
         "recent": 256, "lens": 9},
        # one long sequence of 32768 tokens on 2 kv heads cut back to a quarter
        {"name": "evict_b1_32x2_32768_to_8192", "op": "evict", "batch": 1, "lo": 32768, "hi": 32768, "hq": 32, "hkv": 2, "budget": 8192, "sink": 16,
         "recent": 1024, "lens": 10},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng, most_group=16):
    """Query and kv heads."""
    hkv = rng.choice([1, 2, 4, 5, 8, 16, 32])
    group = rng.choice([g for g in (1, 2, 3, 4, 7, 8, 16) if g <= most_group and g * hkv <= 64])
    return group * hkv, hkv


def draw(rng):
    op = rng.choice(["rotate", "append", "shared", "weights", "evict"])
    hq, hkv = _heads(rng)
    lens = rng.randrange(1 << 20)
    rope = {"rotary": rng.choice([32, 64, 96, 128, 128]), "axes": rng.choice([1, 1, 2, 3]), "inter": rng.random() < 0.4, "norm": rng.random() < 0.7,
            "theta": rng.choice([10000.0, 500000.0, 1000000.0])}
    if op == "rotate":
        tokens = _spread(rng, 1, min(16384, 1400000 // (hq + hkv)))
        return {"op": op, "tokens": tokens, "hq": hq, "hkv": hkv, "far": _spread(rng, tokens, 1 << 20), **rope}
    if op == "append":
        batch = _spread(rng, 1, 32)
        hi = _spread(rng, 1, min(16384, 1800000 // (hq + hkv) // batch))
        return {"op": op, "batch": batch, "lo": max(1, hi // rng.choice([1, 4, 16])), "hi": hi, "hq": hq, "hkv": hkv, "lens": lens, **rope}
    rows = 1800000 // hkv   # token rows of the batch and kv head that a drawn case may attend over
    if op == "shared":
        groups = rng.choice([1, 1, 2, 4])
        batch = groups * _spread(rng, 2, 64 // groups)
        total = min(20480, rows // batch)
        hi = _spread(rng, 1, max(1, min(2048, total // 3)))
        prefix = max(1, _spread(rng, 128, max(128, total - hi)) // PAGE) * PAGE
        return {"op": op, "groups": groups, "batch": batch, "prefix": prefix, "lo": max(1, hi // rng.choice([1, 4, 16])), "hi": hi, "hq": hq, "hkv": hkv, "lens": lens}
    batch = _spread(rng, 1, 64)
    hi = _spread(rng, 3, min(32768, rows // batch))
    lo = max(2, hi // rng.choice([1, 2, 4]))
    if op == "weights":
        return {"op": op, "batch": batch, "lo": lo, "hi": hi, "hq": hq, "hkv": hkv, "lens": lens}
    budget = max(1, min(hi - 1, rng.choice([hi - 1, hi - rng.randrange(1, hi), hi // 2, hi // 4])))
    sink = min(budget // 4, rng.choice([0, 1, 4]))
    return {"op": op, "batch": batch, "lo": lo, "hi": hi, "hq": hq, "hkv": hkv, "budget": budget, "sink": sink,
            "recent": rng.randrange(0, max(1, (budget - sink) // 2)), "lens": lens}


def _lengths(case):
    """The batch's lengths: they belong to the case, not to the inputs' seed."""
    g = torch.Generator().manual_seed(240707304 + case["lens"])
    return torch.randint(case["lo"], case["hi"] + 1, (case["batch"],), generator=g).tolist()


def work(case):
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    row = 2 * D + 8                                      # a cached token and kv head: two rows of codes and their scales
    if op == "rotate":
        n = case["tokens"]
        return {"bytes": n * ((hq + hkv) * 2 * D * 2 + 4 * case["axes"]), "flops": n * (hq + hkv) * D * 8}
    if op == "append":
        n = sum(_lengths(case))
        return {"bytes": n * ((2 * hq + 2 * hkv) * D * 2 + hkv * row + 4 * case["axes"]), "flops": n * (hq + 2 * hkv) * D * 8}
    lens = _lengths(case)
    b = case["batch"]
    if op == "shared":
        rows = case["groups"] * case["prefix"] + sum(lens)
        return {"bytes": rows * hkv * row + b * hq * D * 4, "flops": 4 * D * hq * (b * case["prefix"] + sum(lens))}
    if op == "weights":
        return {"bytes": sum(lens) * hkv * (row + 8) + b * hq * D * 4, "flops": 4 * D * hq * sum(lens)}
    moved = sum(case["budget"] * (n - case["budget"]) / n for n in lens if n > case["budget"])
    kept = sum(min(n, case["budget"]) for n in lens)
    return {"bytes": hkv * (4 * sum(lens) + 4 * kept + 8 * kept + 2 * row * moved), "flops": hkv * sum(lens)}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pool(g, pages, hkv):
    """A cache pool in use: normal rows with four large channels per head, K and V, as INT8 codes and their scales."""
    x = _randn(g, pages * hkv * 2, PAGE, D).view(pages, hkv, 2, PAGE, D)
    big = torch.rand((hkv, 2, 1, D), generator=g, device="cuda").argsort(-1) < 4
    x *= torch.where(big, 8.0, 1.0)
    amax = x.abs().amax(-1, keepdim=True)
    codes = (x * (127.0 / amax)).round_().clamp_(-127, 127).to(torch.int8)
    return codes, (amax / 127.0).squeeze(-1).contiguous()


def _handle(state, b, hkv, pages_per_seq):
    """The library's cache over the state's pool; the state's codes and scales become that cache's own."""
    from paper_2407_07304_b200 import binding as slim
    codes, scales = state["codes"], state["scales"]
    cache = slim.SlimCache(b, hkv, pages_per_seq, block_table=state["table"], num_pages=codes.shape[0])
    cache.codes.copy_(codes.reshape(-1))
    cache.scales.copy_(scales.reshape(-1))
    state.update(slim=slim, cache=cache, codes=cache.codes_view(), scales=cache.scales_view())


def _prepare_rope(case, g, state, tokens):
    hq, hkv, half = case["hq"], case["hkv"], case["rotary"] // 2
    # the fused projection's rows [query heads | key heads | value heads]
    rows = (_randn(g, tokens, hq + 2 * hkv, D) * (0.5 + 1.5 * torch.rand((hq + 2 * hkv, D), generator=g, device="cuda"))).to(torch.bfloat16)
    state["q"], state["k"], state["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    state["inv_freq"] = torch.pow(torch.tensor(case["theta"], dtype=torch.float64, device="cuda"),
                                  -torch.arange(half, dtype=torch.float64, device="cuda") / half)
    state["axis"] = (torch.arange(half, device="cuda") * case["axes"] // half).to(torch.uint8)
    state["qw"] = (1.0 + 0.2 * _randn(g, D)).to(torch.bfloat16) if case["norm"] else None
    state["kw"] = (1.0 + 0.2 * _randn(g, D)).to(torch.bfloat16) if case["norm"] else None
    if own:
        from paper_2407_07304_b200 import binding as slim
        state["slim"] = slim
        state["rope"] = slim.NormRope(state["inv_freq"], q_weight=state["qw"], k_weight=state["kw"], eps=EPS, axis=state["axis"],
                                      n_axes=case["axes"], interleaved=case["inter"])
        state["q_out"] = torch.empty((tokens, hq, D), dtype=torch.bfloat16, device="cuda")
        state["k_out"] = torch.empty((tokens, hkv, D), dtype=torch.bfloat16, device="cuda")


def prepare(case, seed):
    g, op, hq, hkv = _gen(seed), case["op"], case["hq"], case["hkv"]
    state = {"op": op, "case": case}
    if op == "rotate":
        n = case["tokens"]
        _prepare_rope(case, g, state, n)
        first = torch.randint(0, max(1, case["far"] - n + 1), (case["axes"], 1), generator=g, device="cuda")
        state["pos"] = (first + torch.arange(n, device="cuda")).to(torch.int32)
        return state
    lens = _lengths(case)
    b = case["batch"]
    if op == "append":
        n = sum(lens)
        _prepare_rope(case, g, state, n)
        mp = (max(lens) + PAGE - 1) // PAGE
        cu = [0]
        for x in lens:
            cu.append(cu[-1] + x)
        state["cu"], state["start"] = _i32(cu), _i32([0] * b)
        # text positions on the first axis, rows and columns of image patches on the others
        seq = torch.repeat_interleave(torch.arange(b, device="cuda"), _i32(lens).long())
        t = torch.arange(n, device="cuda") - state["cu"][:-1].long()[seq]
        side = torch.randint(16, 64, (b,), generator=g, device="cuda")[seq]
        state["pos"] = torch.stack([t, t // side, t % side][:case["axes"]]).to(torch.int32)
        pages = b * mp
        state["table"] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(b, mp)
        state["codes"] = torch.zeros((pages, hkv, 2, PAGE, D), dtype=torch.int8, device="cuda")
        state["scales"] = torch.zeros((pages, hkv, 2, PAGE), device="cuda")
        state["seq"], state["slot"] = seq, t
        if own:
            _handle(state, b, hkv, mp)
        return state
    if op == "shared":
        per, pre = b // case["groups"], case["prefix"] // PAGE
        tail = (max(lens) + PAGE - 1) // PAGE
        pages = case["groups"] * pre + b * tail
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        state["table"] = torch.cat([order[:case["groups"] * pre].view(case["groups"], pre).repeat_interleave(per, 0),
                                    order[case["groups"] * pre:].view(b, tail)], 1).contiguous()
        state["lens"] = _i32([case["prefix"] + x for x in lens])
        state["shared"] = _i32([case["prefix"]] * b)
        state["cu_group"] = _i32([per * i for i in range(case["groups"] + 1)])
        mp = pre + tail
    else:
        mp = (max(lens) + PAGE - 1) // PAGE
        pages = b * mp
        state["table"] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(b, mp)
        state["lens"] = _i32(lens)
    state["codes"], state["scales"] = _pool(g, pages, hkv)
    if op != "evict":
        state["q"] = _randn(g, b, hq, D).to(torch.bfloat16)
        state["scale"] = D ** -0.5
    if op in ("weights", "evict"):
        # weights that earlier steps left: some tokens many times the others', a fifth of them never attended, some equal
        m = mp * PAGE
        w = torch.exp(2.0 * _randn(g, b, hkv, m))
        w = torch.where(w < 1.0, torch.floor(w * 16.0) / 16.0, w)
        state["w"] = torch.where(torch.rand((b, hkv, m), generator=g, device="cuda") < 0.2, torch.zeros_like(w), w)
        state["w_out"] = torch.zeros_like(w)
    if op == "weights":
        state["weighed"] = state["lens"] - 1
    if op == "evict":
        # an earlier eviction left its budget of tokens in no order, the later ones follow in order
        placed = torch.clamp(state["lens"] - 1, max=case["budget"])
        before = 2 * m
        state["placed"], state["seen"] = placed, before + state["lens"] - placed
        state["pos"] = torch.rand((b, hkv, before), generator=g, device="cuda").argsort(-1)[..., :m].to(torch.int32).contiguous()
        state["pos_out"] = torch.zeros_like(state["pos"])
    if own:
        _handle(state, b, hkv, mp)
        slim = state["slim"]
        if op == "shared":
            state["ws"] = slim.shared_workspace(b, hq, hkv, case["groups"], per, case["prefix"], max(lens))
            state["out"] = torch.empty_like(state["q"])
        elif op == "weights":
            state["ws"] = slim.weights_workspace(b, hq, hkv, max(lens))
            state["out"] = torch.empty_like(state["q"])
        else:
            state["ws"] = slim.evict_workspace(b, hkv, max(lens), case["budget"])
    state["longest"] = max(lens)
    return state


# ---------------------------------------------------------------------------------------------- one pass
def _held(codes, scales):
    """The values that codes and scales stand for, in the working type."""
    return torch.mul(codes, scales.unsqueeze(-1), out=torch.empty(codes.shape, dtype=torch.bfloat16, device=codes.device))


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    slim, op, case = s["slim"], s["op"], s["case"]
    if op == "rotate":
        slim.slim_norm_rope(s["rope"], s["q"], s["q_out"], s["k"], s["k_out"], s["pos"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        slim.slim_norm_rope_append(s["cache"], s["rope"], s["q"], s["q_out"], s["k"], s["v"], s["pos"], s["cu"], s["start"], case["batch"])
        return {"q": s["q_out"], "held": _held(s["codes"], s["scales"]), "scales": s["scales"]}
    if op == "shared":
        slim.slim_attn_decode_shared(s["cache"], s["q"], s["out"], s["cu_group"], s["shared"], s["lens"], case["groups"], case["batch"],
                                     case["batch"] // case["groups"], case["prefix"], s["longest"], case["hq"], s["scale"], s["ws"])
        return {"out": s["out"]}
    if op == "weights":
        slim.slim_attn_decode_weights(s["cache"], s["q"], s["out"], s["w"], s["w_out"], s["weighed"], s["lens"], case["batch"], s["longest"],
                                      case["hq"], s["scale"], 1.0, s["ws"])
        return {"out": s["out"], "weights": s["w_out"]}
    slim.slim_kv_evict(s["cache"], s["w"], s["w_out"], s["pos"], s["pos_out"], s["lens"], s["placed"], s["seen"], case["batch"], s["longest"],
                       case["budget"], case["sink"], case["recent"], s["ws"])
    return {"codes": s["codes"], "scales": s["scales"], "weights": s["w_out"], "pos": s["pos_out"]}


def _rotated(x, weight, cos, sin, inter):
    """fp32 heads [tokens, heads, 128]: norm (with a weight), then the rotation of the first 2 * half dimensions."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    half = cos.shape[-1]
    c, s, turn = cos[:, None], sin[:, None], x[..., :2 * half]
    if inter:
        a, b = turn[..., 0::2], turn[..., 1::2]
        y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = turn[..., :half], turn[..., half:]
        y = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([y, x[..., 2 * half:]], -1)


def _quantised(x):
    """fp32 rows [..., 128] -> codes and scales."""
    amax = x.abs().amax(-1, keepdim=True)
    codes = torch.where(amax > 0, x * 127.0 / amax, torch.zeros_like(x)).round().clamp(-127, 127)
    return codes.to(torch.int8), (amax / 127.0).squeeze(-1)


def _run_plain(s):
    op, case = s["op"], s["case"]
    if op in ("rotate", "append"):
        angle = s["pos"].double()[s["axis"].long()].transpose(0, 1) * s["inv_freq"]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        q = _rotated(s["q"], s["qw"], cos, sin, case["inter"]).to(torch.bfloat16)
        k = _rotated(s["k"], s["kw"], cos, sin, case["inter"])
        if op == "rotate":
            return {"q": q, "k": k.to(torch.bfloat16)}
        codes, scales = _quantised(torch.stack([k, s["v"].float()], 2))          # [tokens, hkv, 2, 128]
        page = s["table"][s["seq"], s["slot"] // PAGE].long()
        s["codes"][page, :, :, s["slot"] % PAGE] = codes
        s["scales"][page, :, :, s["slot"] % PAGE] = scales
        return {"q": q, "held": _held(s["codes"], s["scales"]), "scales": s["scales"]}
    if op in ("shared", "weights"):
        b, hq, hkv, t = case["batch"], case["hq"], case["hkv"], s["table"].shape[1] * PAGE
        rows = s["codes"][s["table"].long()].float() * s["scales"][s["table"].long()].unsqueeze(-1)     # [b, pages, hkv, 2, 128, 128]
        k, v = rows.permute(3, 0, 2, 1, 4, 5).reshape(2, b, hkv, t, D)
        del rows
        seen = (torch.arange(t, device="cuda") < s["lens"][:, None])[:, None, None]
        score = torch.matmul(s["q"].float().view(b, hkv, hq // hkv, D), k.transpose(-1, -2)) * s["scale"]
        score = torch.where(seen, score, torch.full_like(score, -math.inf))
        p = torch.exp(score - score.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        out = torch.matmul(p, v).view(b, hq, D).to(torch.bfloat16)
        if op == "shared":
            return {"out": out}
        weighed = (torch.arange(t, device="cuda") < s["weighed"][:, None])[:, None]
        w = torch.where(weighed, s["w"], torch.zeros_like(s["w"])) + p.sum(2)
        return {"out": out, "weights": torch.where(seen[:, 0], w, s["w_out"])}
    # ---- eviction: rank the slots (protected ones first, then by weight, equal ones by slot), keep the budget's best;
    #      the kept tokens behind the budget fill the freed slots before it, both in ascending order
    b, hkv, m = s["w"].shape
    budget = case["budget"]
    slot = torch.arange(m, device="cuda").expand(b, hkv, m)
    n = s["lens"][:, None, None]
    pos = torch.where(slot < s["placed"][:, None, None], s["pos"], (s["seen"] - s["lens"])[:, None, None] + slot)
    safe = (pos < case["sink"]) | (pos >= s["seen"][:, None, None] - case["recent"])
    rank = torch.where(slot < n, safe.to(torch.int32) + 1, 0)
    by_weight = s["w"].sort(dim=-1, descending=True, stable=True).indices
    order = by_weight.gather(-1, rank.gather(-1, by_weight).sort(dim=-1, descending=True, stable=True).indices)
    keep = torch.zeros_like(slot, dtype=torch.bool).scatter(-1, order[..., :budget], True) & (slot < n)
    hole = ~keep & (slot < torch.clamp(n, max=budget))
    move = keep & (slot >= budget)
    source = torch.where(move, slot, m).sort(-1).values                          # the movers, ascending, then m
    source = torch.where(hole, source.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), slot)[..., :min(budget, m)]
    stays = source.new_tensor(0) + (slot < torch.clamp(n, max=budget))[..., :min(budget, m)]
    head = torch.arange(hkv, device="cuda")[None, :, None]
    seq = torch.arange(b, device="cuda")[:, None, None]
    to = slot[..., :min(budget, m)]
    page_to, page_from = (s["table"][seq, x // PAGE].long() for x in (to, source))
    s["codes"][page_to, head, :, to % PAGE] = s["codes"][page_from, head, :, source % PAGE]
    s["scales"][page_to, head, :, to % PAGE] = s["scales"][page_from, head, :, source % PAGE]
    w, pos_out = s["w_out"].clone(), s["pos_out"].clone()
    w[..., :min(budget, m)] = torch.where(stays > 0, s["w"].gather(-1, source), w[..., :min(budget, m)])
    pos_out[..., :min(budget, m)] = torch.where(stays > 0, pos.gather(-1, source).to(torch.int32), pos_out[..., :min(budget, m)])
    return {"codes": s["codes"], "scales": s["scales"], "weights": w, "pos": pos_out}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    op = case["op"]
    if op == "evict":
        return None                     # everything it returns is chosen and moved, nothing is computed
    with torch.no_grad():
        s = _without_handle(case, seed)
        if op in ("rotate", "append"):
            return _exact_rope(case, s)
        return _exact_decode(case, s)


def _without_handle(case, seed):
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_rope(case, s):
    half = case["rotary"] // 2
    n = s["q"].shape[0]
    first = [2 * i if case["inter"] else i for i in range(half)]
    second = [2 * i + 1 if case["inter"] else i + half for i in range(half)]

    def turned(x, w):
        x = x.to(torch.float64)
        if w is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * w.to(torch.float64)
        y = x.clone()
        for i in range(half):
            a = s["pos"][int(s["axis"][i])].to(torch.float64) * s["inv_freq"][i]
            u, v = x[:, :, first[i]], x[:, :, second[i]]
            y[:, :, first[i]] = u * a.cos()[:, None] - v * a.sin()[:, None]
            y[:, :, second[i]] = v * a.cos()[:, None] + u * a.sin()[:, None]
        return y

    q = turned(s["q"], s["qw"])
    k = turned(s["k"], s["kw"])
    if case["op"] == "rotate":
        return {"q": q, "k": k}
    held = torch.zeros(s["codes"].shape, dtype=torch.float64, device="cuda")
    scales = torch.zeros(s["scales"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for b, length in enumerate(_lengths(case)):
        for j in range(0, length, PAGE):
            rows, page = min(PAGE, length - j), int(s["table"][b, j // PAGE])
            for kv, x in enumerate((k, s["v"])):
                y = x[at + j:at + j + rows].to(torch.float64).transpose(0, 1)    # [hkv, rows, 128]
                top = y.abs().max(-1, keepdim=True).values
                code = torch.where(top > 0, torch.round(127.0 * y / top), 0.0)
                held[page, :, kv, :rows] = code * (top / 127.0)
                scales[page, :, kv, :rows] = (top / 127.0).squeeze(-1)
        at += length
    assert at == n
    return {"q": q, "held": held, "scales": scales}


def _exact_decode(case, s):
    hq, hkv = case["hq"], case["hkv"]
    group = hq // hkv
    outs, weights = [], s["w_out"].double() if case["op"] == "weights" else None
    for b in range(case["batch"]):
        n = int(s["lens"][b])
        pages = s["table"][b, :(n + PAGE - 1) // PAGE].long()
        c = s["codes"][pages].to(torch.float64) * s["scales"][pages].to(torch.float64)[..., None]
        k = torch.cat([c[i, :, 0] for i in range(c.shape[0])], 1)[:, :n]
        v = torch.cat([c[i, :, 1] for i in range(c.shape[0])], 1)[:, :n]
        q = s["q"][b].to(torch.float64)
        rows = []
        for h in range(hkv):
            z = q[h * group:(h + 1) * group] @ k[h].T / math.sqrt(D)
            p = torch.softmax(z, -1)
            rows.append(p @ v[h])
            if weights is not None:
                weights[b, h, :n] = p.sum(0)
                weights[b, h, :int(s["weighed"][b])] += s["w"][b, h, :int(s["weighed"][b])].double()
        outs.append(torch.cat(rows))
    out = torch.stack(outs)
    return {"out": out} if weights is None else {"out": out, "weights": weights}
