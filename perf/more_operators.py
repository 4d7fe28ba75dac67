"""Cases and plain forms of the operators around the 4-bit KV cache and of the page tables of a cache.

  append4   quantising keys and values into the 4-bit cache, and reading the same rows back (slim_kv4_append, slim_kv4_read)
  decode4   decode attention over the 4-bit cache, with "step" the new tokens going into it in the same call (slim_attn4_decode)
  prefill4  causal attention of new rows over the 4-bit cache that holds them (slim_attn4_prefill)
  fork      the page table's rows continue by parent, then every row gets room for its next tokens (slim_pages_fork, slim_pages_grow)
  compact   finished sequences leave the page table, then the pages in use move together (slim_pages_fork, slim_pages_compact)

`own` False: elementary torch operations.  `own` True: the calls a user makes of the library.
"""
import math

import torch

own = False

D = 128          # head dimension
PAGE = 128       # token positions per page


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the new tokens of one decode step of a batch of 16, 32 kv heads: latency counts
        {"name": "append4_step_b16_hkv32", "op": "append4", "batch": 16, "lo": 1, "hi": 1, "hkv": 32, "start": 2048, "lens": 1},
        # sixteen prompts of 256 to 4096 tokens, 8 kv heads
        {"name": "append4_ragged_b16_hkv8", "op": "append4", "batch": 16, "lo": 256, "hi": 4096, "hkv": 8, "start": 0, "lens": 2},
        # a short single sequence: the smallest decode step, latency counts
        {"name": "decode4_b1_32x32_272", "op": "decode4", "batch": 1, "lo": 272, "hi": 272, "hq": 32, "hkv": 32, "step": False, "lens": 3},
        # a batch of 16 in lockstep, one query head per kv head, the new tokens appended in the call
        {"name": "decode4_step_b16_32x32_2049", "op": "decode4", "batch": 16, "lo": 2049, "hi": 2049, "hq": 32, "hkv": 32, "step": True, "lens": 4},
        # a ragged batch of 32, 64 query heads on 8 kv heads
        {"name": "decode4_b32_64x8_4096", "op": "decode4", "batch": 32, "lo": 1024, "hi": 4096, "hq": 64, "hkv": 8, "step": False, "lens": 5},
        # one long sequence, 32 query heads on 2 kv heads: few rows, the key axis is what can be split
        {"name": "decode4_b1_32x2_32768", "op": "decode4", "batch": 1, "lo": 32768, "hi": 32768, "hq": 32, "hkv": 2, "step": False, "lens": 6},
        # pieces of 256 to 512 rows of four long prompts, each behind what came before, 64 query heads on 8 kv heads
        {"name": "prefill4_pieces_b4_64x8_512_behind_4000", "op": "prefill4", "batch": 4, "lo": 256, "hi": 512, "before": 4000, "hq": 64, "hkv": 8, "lens": 7},
        # a whole prompt of 8192 tokens
        {"name": "prefill4_8192_32x32", "op": "prefill4", "batch": 1, "lo": 8192, "hi": 8192, "before": 0, "hq": 32, "hkv": 32, "lens": 8},
        # a step of a beam search: four prompts with four beams each, some beams continued twice, others dropped; two INT8 layers
        {"name": "fork_beams_4x4_300_int8", "op": "fork", "batch": 16, "per": 4, "out": 16, "lo": 260, "hi": 340, "hkv": 8, "bits": 8, "layers": 2, "room": 1, "lens": 9},
        # a long prompt of every one of four requests sampled 64 times, sixteen 4-bit layers
        {"name": "fork_samples_4x64_8000_int4", "op": "fork", "batch": 4, "per": 1, "out": 256, "lo": 7900, "hi": 8100, "hkv": 8, "bits": 4, "layers": 16, "room": 128, "lens": 10},
        # a small batch of which a third has ended, one layer
        {"name": "compact_b16_1000_int4", "op": "compact", "batch": 16, "lo": 500, "hi": 1500, "hkv": 8, "bits": 4, "layers": 1, "drop": 3, "lens": 11},
        # a large batch of which half has ended, eight INT8 layers
        {"name": "compact_b128_2000_int8", "op": "compact", "batch": 128, "lo": 1000, "hi": 2900, "hkv": 8, "bits": 8, "layers": 8, "drop": 2, "lens": 12},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    """Query and kv heads."""
    hkv = rng.choice([1, 2, 4, 5, 8, 16, 32])
    return rng.choice([g for g in (1, 2, 3, 4, 7, 8, 16) if g * hkv <= 64]) * hkv, hkv


def draw(rng):
    op = rng.choice(["append4", "decode4", "decode4", "prefill4", "fork", "compact"])
    hq, hkv = _heads(rng)
    lens = rng.randrange(1 << 20)
    if op == "append4":
        batch = _spread(rng, 1, 32)
        hi = _spread(rng, 1, min(16384, 300000 // hkv // batch))
        return {"op": op, "batch": batch, "lo": max(1, hi // rng.choice([1, 4, 16])), "hi": hi, "hkv": hkv, "start": rng.choice([0, rng.randrange(1, 1000)]),
                "lens": lens}
    if op == "decode4":
        batch = _spread(rng, 1, 64)
        hi = _spread(rng, 1, min(65536, 1000000 // hkv // batch))
        return {"op": op, "batch": batch, "lo": max(1, hi // rng.choice([1, 2, 16])), "hi": hi, "hq": hq, "hkv": hkv, "step": rng.random() < 0.5, "lens": lens}
    if op == "prefill4":
        batch = _spread(rng, 1, 8)
        hi = _spread(rng, 1, 4096 // batch)
        return {"op": op, "batch": batch, "lo": max(1, hi // rng.choice([1, 2, 8])), "hi": hi, "before": rng.choice([0, _spread(rng, 1, 8192 // batch)]),
                "hq": hq, "hkv": hkv, "lens": lens}
    hkv, bits, layers = rng.choice([2, 5, 8]), rng.choice([4, 8]), rng.choice([1, 2, 7])
    if op == "fork":
        per, batch = rng.choice([(1, _spread(rng, 1, 8)), (4, 4 * _spread(rng, 1, 8))])
        hi = _spread(rng, 1, 4096)
        return {"op": op, "batch": batch, "per": per, "out": _spread(rng, 1, 96), "lo": max(1, hi // rng.choice([1, 2, 16])), "hi": hi, "hkv": hkv, "bits": bits,
                "layers": layers, "room": _spread(rng, 1, 512), "lens": lens}
    batch = _spread(rng, 2, 128)
    hi = _spread(rng, 1, 2048)
    return {"op": op, "batch": batch, "lo": max(1, hi // rng.choice([1, 2, 16])), "hi": hi, "hkv": hkv, "bits": bits, "layers": layers, "drop": rng.choice([2, 3, 8]),
            "lens": lens}


def _lengths(case):
    """The batch's lengths: they belong to the case, not to the inputs' seed."""
    g = torch.Generator().manual_seed(407304 + case["lens"])
    lens = torch.randint(case["lo"], case["hi"] + 1, (case["batch"],), generator=g).tolist()
    return [lens[i - i % case.get("per", 1)] for i in range(len(lens))]        # the beams of a request are of one length


def _pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def _parents(case):
    """Which old row every new row continues (-1: an empty row): they belong to the case too."""
    g = torch.Generator().manual_seed(30407 + case["lens"])
    n = case["batch"]
    if case["op"] == "compact":
        ended = torch.randperm(n, generator=g)[:max(1, n // case["drop"])]
        keep = torch.arange(n)
        keep[ended] = -1
        return keep.tolist()
    if case["per"] == 1:
        return [i * n // case["out"] for i in range(case["out"])]         # samples of a request side by side
    first = torch.arange(case["out"]) * (n // case["per"]) // case["out"] * case["per"]   # a beam continues a beam of its own request
    return (first + torch.randint(0, case["per"], (case["out"],), generator=g)).tolist()


def _moves(case):
    """Pages that compacting moves: used ones beyond as many as are used.  The pool of `compact` is filled at random, so that is what is to be expected."""
    lens, keep = _lengths(case), _parents(case)
    used = sum(_pages(n) for n, k in zip(lens, keep) if k >= 0)
    pool = sum(_pages(n) for n in lens)
    return used * (pool - used) / max(1, pool)


def work(case):
    op, hkv = case["op"], case["hkv"]
    row = D // 2 + 4                                     # a cached row: 128 codes of 4 bits, scale and offset
    if op == "append4":
        n = sum(_lengths(case)) * hkv * 2
        return {"bytes": n * (2 * D + 2 * row + 2 * D), "flops": n * D * 6}
    if op == "decode4":
        lens = _lengths(case)
        new = case["batch"] * hkv * 2 * (2 * D + row) if case["step"] else 0
        return {"bytes": sum(lens) * hkv * 2 * row + 2 * case["batch"] * case["hq"] * D * 2 + new, "flops": 4 * D * case["hq"] * sum(lens)}
    if op == "prefill4":
        lens = _lengths(case)
        seen = sum(n * case["before"] + n * (n + 1) // 2 for n in lens)
        return {"bytes": sum(n + case["before"] for n in lens) * hkv * 2 * row + 2 * sum(lens) * case["hq"] * D * 2, "flops": 4 * D * case["hq"] * seen}
    row = hkv * 2 * (D * case["bits"] // 8 + 4) * case["layers"]      # a token in every layer
    table = 4 * case["batch"] * _pages(case["hi"])
    if op == "fork":
        lens, parents = _lengths(case), _parents(case)
        copies = [lens[p] % PAGE for i, p in enumerate(parents) if p in parents[:i]]
        return {"bytes": 2 * sum(copies) * row + table + 4 * case["out"] * _pages(case["hi"] + case["room"]), "flops": 0}
    return {"bytes": 2 * _moves(case) * PAGE * row + 2 * table, "flops": 0}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rows(g, *shape):
    """Keys or values [..., heads, 128] as projections leave them: normal, four large channels per head, an offset of their own per channel."""
    heads = shape[-1]
    big = torch.rand((heads, D), generator=g, device="cuda").argsort(-1) < 4
    return (_randn(g, *shape, D) * torch.where(big, 6.0, 1.0) + 0.5 * _randn(g, heads, D)).to(torch.bfloat16)


def _pool(g, pages, hkv):
    """A 4-bit cache pool in use: codes and (scale, offset) pairs."""
    x = _rows(g, pages, 2, PAGE, hkv).permute(0, 3, 1, 2, 4)
    codes, scale, offset = _quantised(x.float())
    return codes.contiguous(), torch.stack([scale, offset], -1).contiguous()


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _handle(state, b, hkv, stride):
    """The library's cache over the state's pool; the state's codes and scales become that cache's own."""
    from paper_2407_07304_b200 import binding as slim
    cache = slim.SlimCache4(b, hkv, stride, block_table=state["table"], num_pages=state["codes"].shape[0])
    cache.codes_view().copy_(state["codes"])
    cache.scales_view().copy_(state["scales"])
    state.update(slim=slim, cache=cache, codes=cache.codes_view(), scales=cache.scales_view())


def prepare(case, seed):
    g, op, hkv, b = _gen(seed), case["op"], case["hkv"], case["batch"]
    lens = _lengths(case)
    state = {"op": op, "case": case, "lens_host": lens, "longest": max(lens)}
    if op in ("fork", "compact"):
        return _prepare_pages(case, g, state, lens)
    if op == "append4":
        start = torch.randint(0, case["start"] + 1, (b,), generator=g, device="cuda").to(torch.int32)
        stride = _pages(case["start"] + max(lens))
        n, cu = sum(lens), _cu(lens)
        state["cu"], state["start"] = _i32(cu), start
        seq = torch.repeat_interleave(torch.arange(b, device="cuda"), _i32(lens).long())
        state["seq"], state["slot"] = seq, start[seq].long() + torch.arange(n, device="cuda") - state["cu"][:-1].long()[seq]
        state["k"], state["v"] = _rows(g, n, hkv), _rows(g, n, hkv)
        state["k_held"], state["v_held"] = torch.zeros_like(state["k"]), torch.zeros_like(state["v"])
        pages = b * stride
        state["codes"] = torch.zeros((pages, hkv, 2, PAGE, D // 2), dtype=torch.uint8, device="cuda")
        state["scales"] = torch.zeros((pages, hkv, 2, PAGE, 2), dtype=torch.bfloat16, device="cuda")
    else:
        before = case.get("before", 0)
        stride = _pages(before + max(lens))
        pages = b * stride
        state["codes"], state["scales"] = _pool(g, pages, hkv)
        state["lens"] = _i32([before + n for n in lens])
        rows = b if op == "decode4" else sum(lens)
        state["q"] = _randn(g, rows, case["hq"], D).to(torch.bfloat16)
        state["scale"] = D ** -0.5
        if op == "prefill4":
            state["cu_host"] = _cu(lens)
            state["cu"] = _i32(state["cu_host"])
        elif case["step"]:
            state["k"], state["v"] = _rows(g, b, hkv), _rows(g, b, hkv)
            state["k_held"], state["v_held"] = torch.zeros_like(state["k"]), torch.zeros_like(state["v"])
            state["cu"], state["start"] = _i32(list(range(b + 1))), state["lens"] - 1
            state["seq"], state["slot"] = torch.arange(b, device="cuda"), state["start"].long()
    state["table"] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(b, stride)
    if own:
        _handle(state, b, hkv, stride)
        if op != "append4":
            state["out"] = torch.empty_like(state["q"])
        if op == "decode4":
            state["ws"] = state["slim"].decode4_workspace(b, case["hq"], hkv, max(lens))
        if op == "prefill4":
            state["ws"] = state["slim"].workspace(state["slim"].PHASE_PREFILL, b, case["hq"], hkv, max(lens), stride * PAGE)
    return state


def _prepare_pages(case, g, state, lens):
    b, hkv, bits = case["batch"], case["hkv"], case["bits"]
    parents = _parents(case)
    n_out = len(parents)
    room = case.get("room", 0)
    stride = _pages(case["hi"] + room)
    held = [_pages(n) for n in lens]
    per = case.get("per", 1)
    # the beams of a request share all pages but the last one
    own_pages = sum(held) if per == 1 else sum(h - 1 if i % per == 0 else 0 for i, h in enumerate(held)) + b
    extra = 0 if case["op"] == "compact" else sum(1 + _pages(lens[p] + room) - lens[p] // PAGE for p in parents)
    pages = own_pages + extra + 3
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table, at = [[-1] * stride for _ in range(b)], 0
    refs = [0] * pages
    for i in range(b):
        for j in range(held[i]):
            if per > 1 and i % per and j < held[i] - 1:
                table[i][j] = table[i - i % per][j]
            else:
                table[i][j] = order[at]
                at += 1
            refs[table[i][j]] += 1
    state["table"], state["refs"], state["held"], state["kv_len"] = _i32(table), _i32(refs), _i32(held), _i32(lens)
    state["parent"], state["room"] = _i32(parents), room
    state["table_out"] = torch.full((n_out, stride), -1, dtype=torch.int32, device="cuda")
    state["refs_out"], state["held_out"] = torch.zeros_like(state["refs"]), torch.zeros(n_out, dtype=torch.int32, device="cuda")
    state["len_out"] = torch.zeros(n_out, dtype=torch.int32, device="cuda")
    state["layers"] = []
    for _ in range(case["layers"]):
        codes = torch.randint(0, 256, (pages, hkv, 2, PAGE, D * bits // 8), generator=g, device="cuda", dtype=torch.uint8)
        scales = torch.randint(0, 1 << 30, (pages, hkv, 2, PAGE), generator=g, device="cuda", dtype=torch.int32)
        state["layers"].append([codes, scales])
    if own:
        from paper_2407_07304_b200 import binding as slim
        state["slim"] = slim
        kind = slim.SlimCache if bits == 8 else slim.SlimCache4
        state["caches"] = []
        for layer in state["layers"]:
            cache = kind(b, hkv, stride, block_table=state["table"], num_pages=pages)
            cache.codes.view(torch.uint8).copy_(layer[0].reshape(-1))
            cache.scales.view(torch.int32).copy_(layer[1].reshape(-1))
            layer[0] = cache.codes.view(torch.uint8).view(layer[0].shape)
            layer[1] = cache.scales.view(torch.int32).view(layer[1].shape)
            state["caches"].append(cache)
        state["from"] = slim.SlimPages(state["refs"], state["table"], state["held"])
        state["to"] = slim.SlimPages(state["refs_out"], state["table_out"], state["held_out"])
        state["ws"] = slim.pages_workspace(pages, max(b, n_out))
        state["plan"] = slim.PageLayers(state["caches"])
        state["result"] = torch.zeros(2, dtype=torch.int32, device="cuda")
        state["result2"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    return state


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    slim, op, case = s["slim"], s["op"], s["case"]
    b = case["batch"]
    if op == "append4":
        slim.slim_kv4_append(s["cache"], s["k"], s["v"], s["cu"], s["start"], b, s["longest"])
        slim.slim_kv4_read(s["cache"], s["k_held"], s["v_held"], s["cu"], s["start"], b, s["longest"])
        return {"k": s["k_held"], "v": s["v_held"], "scales": s["scales"]}
    if op == "decode4":
        slim.slim_attn4_decode(s["cache"], s["q"], s["out"], s["lens"], b, s["longest"], case["hq"], s["scale"], s["ws"],
                               k_new=s.get("k"), v_new=s.get("v"))
        if not case["step"]:
            return {"out": s["out"]}
        slim.slim_kv4_read(s["cache"], s["k_held"], s["v_held"], s["cu"], s["start"], b, 1)
        return {"out": s["out"], "k": s["k_held"], "v": s["v_held"], "scales": s["scales"]}
    if op == "prefill4":
        slim.slim_attn4_prefill(s["cache"], s["q"], s["out"], s["cu"], s["lens"], b, s["longest"], case["before"] + s["longest"], case["hq"],
                                s["scale"], s["ws"])
        return {"out": s["out"]}
    if op == "fork":
        slim.slim_pages_fork(s["plan"], s["from"], s["to"], s["parent"], s["kv_len"], s["len_out"], s["result"], s["ws"])
        slim.slim_pages_grow(s["to"], s["len_out"], s["room"], s["result2"], s["ws"])
        return _pages_out(s, s["refs_out"], s["table_out"], s["held_out"], s["len_out"], s["result"], s["result2"])
    slim.slim_pages_fork(None, s["from"], s["to"], s["parent"], s["kv_len"], s["len_out"], s["result"], s["ws"])
    slim.slim_pages_compact(s["plan"], s["to"], s["to"], s["result2"], s["ws"])
    return _pages_out(s, s["refs_out"], s["table_out"], s["held_out"], s["len_out"], s["result"], s["result2"])


def _pages_out(s, refs, table, held, kv_len, result, result2):
    out = {"refs": refs, "table": table, "held": held, "len": kv_len, "result": result, "result2": result2}
    for i, (codes, scales) in enumerate(s["layers"]):
        out[f"codes{i}"], out[f"scales{i}"] = codes, scales
    return out


def _quantised(x):
    """fp32 rows [..., 128] -> packed codes [..., 64], scale and offset (bf16)."""
    low, high = x.amin(-1), x.amax(-1)
    scale = ((high - low) / torch.full_like(low, 15.0)).to(torch.bfloat16)      # (by a number it would be a product with 1 / 15)
    step = scale.float().unsqueeze(-1)
    u = torch.where(step > 0, ((x - low.unsqueeze(-1)) / step).round().clamp(0, 15), torch.zeros_like(x)).to(torch.uint8)
    return u[..., :D // 2] | (u[..., D // 2:] << 4), scale, low.to(torch.bfloat16)


def _values(codes, scales):
    """The fp32 values that codes [..., 64] and their (scale, offset) stand for."""
    u = torch.cat([codes & 15, codes >> 4], -1).float()
    return u * scales[..., 0:1].float() + scales[..., 1:2].float()


def _append_plain(s):
    codes, scale, offset = _quantised(torch.stack([s["k"], s["v"]], 2).float())              # [tokens, hkv, 2, ...]
    page = s["table"][s["seq"], s["slot"] // PAGE].long()
    s["codes"][page, :, :, s["slot"] % PAGE] = codes
    s["scales"][page, :, :, s["slot"] % PAGE] = torch.stack([scale, offset], -1)
    held = _values(s["codes"][page, :, :, s["slot"] % PAGE], s["scales"][page, :, :, s["slot"] % PAGE]).to(torch.bfloat16)
    return {"k": held[:, :, 0].contiguous(), "v": held[:, :, 1].contiguous(), "scales": s["scales"]}


def _run_plain(s):
    op, case = s["op"], s["case"]
    if op == "append4":
        return _append_plain(s)
    if op in ("fork", "compact"):
        return _pages_plain(s, case)
    b, hq, hkv = case["batch"], case["hq"], case["hkv"]
    if op == "decode4":
        held = _append_plain(s) if case["step"] else {}
        t = s["table"].shape[1] * PAGE
        rows = _values(s["codes"][s["table"].long()], s["scales"][s["table"].long()])         # [b, pages, hkv, 2, 128, 128]
        k, v = rows.permute(3, 0, 2, 1, 4, 5).reshape(2, b, hkv, t, D)
        del rows
        seen = (torch.arange(t, device="cuda") < s["lens"][:, None])[:, None, None]
        score = torch.matmul(s["q"].float().view(b, hkv, hq // hkv, D), k.transpose(-1, -2)) * s["scale"]
        score = torch.where(seen, score, torch.full_like(score, -math.inf))
        p = torch.exp(score - score.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        return {"out": torch.matmul(p, v).view(b, hq, D).to(torch.bfloat16), **held}
    out, group = torch.empty_like(s["q"]), hq // hkv
    for i in range(b):
        at, n = s["cu_host"][i], s["lens_host"][i]
        total = case["before"] + n
        pages = s["table"][i, :_pages(total)].long()
        k, v = _values(s["codes"][pages], s["scales"][pages]).permute(2, 1, 0, 3, 4).reshape(2, hkv, -1, D)[:, :, :total]
        hidden = torch.arange(total, device="cuda") > case["before"] + torch.arange(n, device="cuda")[:, None]
        for h in range(hkv):
            q = s["q"][at:at + n, h * group:(h + 1) * group].float().transpose(0, 1)
            score = torch.matmul(q, k[h].T) * s["scale"]
            score.masked_fill_(hidden, -math.inf)
            p = torch.exp(score - score.amax(-1, keepdim=True))
            p = p / p.sum(-1, keepdim=True)
            out[at:at + n, h * group:(h + 1) * group] = torch.matmul(p, v[h]).transpose(0, 1).to(torch.bfloat16)
    return {"out": out}


def _free_pages(refs):
    """Page ids, the free ones first, in ascending order."""
    return torch.sort((refs != 0).to(torch.int32), stable=True).indices


def _pages_plain(s, case):
    table, refs, held, parent = s["table"].long(), s["refs"], s["held"].long(), s["parent"].long()
    n_in, stride = table.shape
    n_out = len(parent)
    slot = torch.arange(stride, device="cuda")
    # ---- rows continued: the first child takes the row over, the others share its whole pages
    alive = parent >= 0
    by = parent.clamp(min=0)
    order = torch.arange(n_out, device="cuda")
    first = torch.full((n_in,), n_out, device="cuda").scatter_reduce(0, by, torch.where(alive, order, n_out), "amin")
    heir = alive & (first[by] == order)
    kv_len = torch.where(alive, s["kv_len"].long()[by], -1)                      # -1: an empty row
    whole, part = kv_len.clamp(min=0) // PAGE, kv_len.clamp(min=0) % PAGE
    copied = alive & ~heir & (part > 0)
    new_held = torch.where(heir, held[by], torch.where(alive, whole, 0))
    new = torch.where(slot < new_held[:, None], table[by], -1)

    def counted(rows, sign, into):
        inside = rows >= 0
        return into + sign * torch.zeros_like(into).scatter_add(0, rows.clamp(min=0).flatten(), inside.flatten().to(into.dtype))

    count = counted(new, 1, counted(torch.where(slot < held[:, None], table, -1), -1, refs))
    fresh = _free_pages(count)[(copied.cumsum(0) - 1).clamp(min=0)]
    free = (count == 0).sum() - copied.sum()
    new = torch.where(copied[:, None] & (slot == whole[:, None]), fresh[:, None], new)
    count = counted(torch.where(copied, fresh, -1), 1, count)
    new_held = new_held + copied
    result = torch.stack([torch.zeros_like(free), free]).to(torch.int32)
    which = copied.nonzero().flatten()
    if len(which):
        source, target, rows = table[by[which], whole[which]], fresh[which], part[which]
        inside = (torch.arange(PAGE, device="cuda") < rows[:, None])[:, None, None]
        for codes, scales in s["layers"] if case["op"] == "fork" else []:
            codes[target] = torch.where(inside[..., None], codes[source], codes[target])
            scales[target] = torch.where(inside, scales[source], scales[target])
    if case["op"] == "fork":
        # ---- room for the next tokens: missing pages by row, then by place
        want = torch.maximum(new_held, torch.where(alive, (kv_len + s["room"] + PAGE - 1) // PAGE, 0))
        missing = (slot >= new_held[:, None]) & (slot < want[:, None])
        at = (missing.flatten().cumsum(0) - 1).clamp(min=0).view_as(new)
        ids = _free_pages(count)
        free = (count == 0).sum() - missing.sum()
        new = torch.where(missing, ids[at.clamp(max=len(ids) - 1)], new)
        count = counted(torch.where(missing, new, -1), 1, count)
        new_held = want
        result2 = torch.stack([torch.zeros_like(free), free]).to(torch.int32)
    else:
        # ---- used pages beyond as many as are used fill the free ones before that, both in ascending order
        used = count > 0
        n_used = used.sum()
        page = torch.arange(len(count), device="cuda")
        mover, hole = used & (page >= n_used), ~used & (page < n_used)
        holes = torch.sort((~hole).to(torch.int32), stable=True).indices
        to = torch.where(mover, holes[(mover.cumsum(0) - 1).clamp(min=0)], page)
        source = mover.nonzero().flatten()
        for codes, scales in s["layers"]:
            codes[to[source]] = codes[source]
            scales[to[source]] = scales[source]
        count = torch.where(mover, 0, count).scatter_add(0, torch.where(mover, to, page), torch.where(mover, count, 0))
        new = torch.where(new >= 0, to[new.clamp(min=0)], -1)
        result2 = torch.stack([n_used, mover.sum()]).to(torch.int32)
    i32 = [x.to(torch.int32) for x in (count, new, new_held, kv_len)]
    return _pages_out(s, *i32, result, result2)


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None                     # everything they return is chosen and moved, nothing is computed
    with torch.no_grad():
        s = _without_handle(case, seed)
        if case["op"] == "append4":
            return _exact_append(s)
        return _exact_attention(case, s)


def _without_handle(case, seed):
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_append(s):
    scales = s["scales"].double()
    out = {}
    for kv, name in enumerate(("k", "v")):
        x = s[name].to(torch.float64)
        low, high = x.min(-1).values, x.max(-1).values
        step = ((high - low) / 15).to(torch.bfloat16).to(torch.float64)
        code = torch.nan_to_num(torch.round((x - low[..., None]) / step[..., None]), nan=0.0).clamp(0, 15)
        out[name] = low[..., None] + code * step[..., None]
        for i in range(x.shape[1]):
            page = s["table"][s["seq"], torch.div(s["slot"], PAGE, rounding_mode="floor")].long()
            scales[page, i, kv, s["slot"].remainder(PAGE)] = torch.stack([step[:, i], low[:, i]], -1)
    return {**out, "scales": scales}


def _exact_attention(case, s):
    hq, hkv = case["hq"], case["hkv"]
    group, step = hq // hkv, case.get("step", False)
    held = _exact_append(s) if step else {}
    outs = []
    for i in range(case["batch"]):
        n = int(s["lens"][i])
        pages = s["table"][i, :(n + PAGE - 1) // PAGE].long()
        c = s["codes"][pages]
        u = torch.empty((*c.shape[:-1], D), dtype=torch.float64, device="cuda")
        u[..., :D // 2], u[..., D // 2:] = c.bitwise_and(15), c.bitwise_right_shift(4)
        scale, offset = (s["scales"][pages].double()[..., x, None] for x in (0, 1))
        x = offset + scale * u
        rows = s["q"][i:i + 1] if case["op"] == "decode4" else s["q"][s["cu_host"][i]:s["cu_host"][i + 1]]
        part = torch.empty(rows.shape, dtype=torch.float64, device="cuda")
        for h in range(hkv):
            k = x[:, h, 0].reshape(-1, D)[:n].clone()
            v = x[:, h, 1].reshape(-1, D)[:n].clone()
            if step:
                k[n - 1], v[n - 1] = held["k"][i, h], held["v"][i, h]
            ahead = torch.ones((len(rows), n), dtype=torch.bool, device="cuda").triu(n - len(rows) + 1)
            for j in range(h * group, (h + 1) * group):
                z = rows[:, j].double() @ k.T / math.sqrt(D)
                part[:, j] = torch.softmax(z.masked_fill(ahead, -math.inf), -1) @ v
        outs.append(part)
    return {"out": torch.cat(outs), **held}
