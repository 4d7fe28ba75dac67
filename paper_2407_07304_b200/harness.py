"""Drives a workload through the library on one GPU: buffers, call order, gathering results.

Plumbing only (uploads, index tensors, the append -> prefill -> append -> decode call
sequence of a workload); all arithmetic happens inside the library calls.
"""
import torch

from . import binding as slim
from .workloads import PAGE_TOKENS, Workload


class LayerRun:
    """One attention layer's cache and device copies of a workload's tensors."""

    def __init__(self, w: Workload, device="cuda", block_table=None, num_pages=None):
        self.w = w
        self.device = torch.device(device)
        self.cache = slim.SlimCache(w.B, w.Hkv, w.pages_per_seq(), device=device, block_table=block_table,
                                    num_pages=num_pages)
        self.k = [t.to(device) for t in w.k]
        self.v = [t.to(device) for t in w.v]
        self.pos = [0] * w.B          # tokens in the cache per sequence
        self.max_total = max(w.total_len(b) for b in range(w.B))
        self.ws_decode = slim.workspace(slim.PHASE_DECODE, w.B, w.Hq, w.Hkv, 1, self.max_total, device=device)
        self.ws_prefill = slim.workspace(slim.PHASE_PREFILL, w.B, w.Hq, w.Hkv, max(w.prefill_len + [1]),
                                         self.max_total, device=device)

    def _i32(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.device)

    # ------------------------------------------------------------------ append
    def append(self, counts):
        """Append the next counts[b] rows of sequence b's K/V to the cache."""
        w = self.w
        ks = [self.k[b][self.pos[b]:self.pos[b] + counts[b]] for b in range(w.B)]
        vs = [self.v[b][self.pos[b]:self.pos[b] + counts[b]] for b in range(w.B)]
        k_new = torch.cat(ks).contiguous()
        v_new = torch.cat(vs).contiguous()
        cu = [0]
        for c in counts:
            cu.append(cu[-1] + c)
        slim.slim_kv_append(self.cache, k_new, v_new, self._i32(cu), self._i32(self.pos), w.B, max(counts))
        for b in range(w.B):
            self.pos[b] += counts[b]

    # ------------------------------------------------------------------ attention
    def prefill(self, q_list, two_pass=False, full_row=False):
        """Causal attention of q_list[b] (bf16 [n_b, Hq, 128], the last n_b cached positions);
        two_pass selects slim_attn_prefill_two_pass (maxima first, then P.V, no corrections), full_row
        slim_attn_prefill_full_row (the whole score row on chip; caches of at most 256 tokens)."""
        w = self.w
        lens = [int(q.shape[0]) for q in q_list]
        q = torch.cat([t.to(self.device) for t in q_list]).contiguous()
        out = torch.empty_like(q)
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        fn = slim.slim_attn_prefill_full_row if full_row else (slim.slim_attn_prefill_two_pass if two_pass else slim.slim_attn_prefill)
        fn(self.cache, q, out, self._i32(cu), self._i32(self.pos), w.B, max(lens), max(self.pos), w.Hq, w.sm_scale,
           self.ws_prefill)
        return [out[cu[b]:cu[b + 1]] for b in range(w.B)]

    def prefill_step(self, counts, q_list):
        """Append the next counts[b] rows of sequence b and attend q_list[b] (one query row per new token) over the
        lengthened cache, in one library call."""
        w = self.w
        k_new = torch.cat([self.k[b][self.pos[b]:self.pos[b] + counts[b]] for b in range(w.B)]).contiguous()
        v_new = torch.cat([self.v[b][self.pos[b]:self.pos[b] + counts[b]] for b in range(w.B)]).contiguous()
        q = torch.cat([t.to(self.device) for t in q_list]).contiguous()
        out = torch.empty_like(q)
        cu = [0]
        for c in counts:
            cu.append(cu[-1] + c)
        for b in range(w.B):
            self.pos[b] += counts[b]
        slim.slim_prefill_step(self.cache, q, k_new, v_new, out, self._i32(cu), self._i32(self.pos), w.B, max(counts),
                               max(self.pos), w.Hq, w.sm_scale, self.ws_prefill)
        return [out[cu[b]:cu[b + 1]] for b in range(w.B)]

    def decode(self, q):
        """One query token per sequence (bf16 [B, Hq, 128]) against the whole cache."""
        w = self.w
        q = q.to(self.device).contiguous()
        out = torch.empty_like(q)
        slim.slim_attn_decode(self.cache, q, out, self._i32(self.pos), w.B, max(self.pos), w.Hq, w.sm_scale,
                              self.ws_decode)
        return out

    def decode_step(self, q):
        """Append the next token of every sequence and attend over the lengthened cache in one library call."""
        w = self.w
        k_new = torch.stack([self.k[b][self.pos[b]] for b in range(w.B)]).contiguous()
        v_new = torch.stack([self.v[b][self.pos[b]] for b in range(w.B)]).contiguous()
        for b in range(w.B):
            self.pos[b] += 1
        q = q.to(self.device).contiguous()
        out = torch.empty_like(q)
        slim.slim_decode_step(self.cache, q, k_new, v_new, out, self._i32(self.pos), w.B, max(self.pos), w.Hq,
                              w.sm_scale, self.ws_decode)
        return out

    # ------------------------------------------------------------------ read-back
    def gather_cache(self, b):
        """Sequence b's cached rows in position order:
        (k_codes, k_scales, v_codes, v_scales) as CPU tensors [T, Hkv, 128] int8 / [T, Hkv] fp32."""
        T = self.pos[b]
        n_pages = (T + PAGE_TOKENS - 1) // PAGE_TOKENS
        pages = self.cache.block_table[b, :n_pages].long()
        codes = self.cache.codes_view()[pages]      # [n_pages, Hkv, 2, 128, 128]
        scales = self.cache.scales_view()[pages]    # [n_pages, Hkv, 2, 128]
        codes = codes.permute(2, 0, 3, 1, 4).reshape(2, n_pages * PAGE_TOKENS, self.w.Hkv, 128)[:, :T]
        scales = scales.permute(2, 0, 3, 1).reshape(2, n_pages * PAGE_TOKENS, self.w.Hkv)[:, :T]
        codes, scales = codes.cpu(), scales.cpu()
        return codes[0], scales[0], codes[1], scales[1]


class RotatedRun:
    """One attention layer of a serving loop on a cache of bounded size: projections in, attention out.

    The queries and keys of every token are normed, rotated by position and the keys and values quantised into the cache
    in one call; every decode step accumulates the tokens' attention weights; evict() cuts each sequence back to `budget`
    tokens by those weights (the first n_sink and the last n_recent always stay).  Slots stop telling positions then, so
    positions are counted here (`seen`) and kept per slot (`positions`)."""

    def __init__(self, B, Hq, Hkv, max_tokens, inv_freq, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, budget=None, n_sink=4,
                 n_recent=32, decay=1.0, device="cuda"):
        self.B, self.Hq, self.Hkv, self.device = B, Hq, Hkv, torch.device(device)
        self.pages = (max_tokens + PAGE_TOKENS - 1) // PAGE_TOKENS
        self.max_tokens = self.pages * PAGE_TOKENS
        self.budget, self.n_sink, self.n_recent, self.decay = budget, n_sink, n_recent, decay
        self.sm_scale = slim.HEAD_DIM ** -0.5
        self.cache = slim.SlimCache(B, Hkv, self.pages, device=device)
        on = lambda t: None if t is None else t.to(self.device)  # noqa: E731
        self.rope = slim.NormRope(on(inv_freq), on(q_weight), on(k_weight), eps, interleaved=interleaved)
        self.weights = torch.zeros((B, Hkv, self.max_tokens), dtype=torch.float32, device=device)
        self.positions = torch.zeros((B, Hkv, self.max_tokens), dtype=torch.int32, device=device)
        self.lens, self.seen, self.placed = [0] * B, [0] * B, [0] * B
        self.weighed = [0] * B        # tokens that the weights cover
        self.ws_prefill = slim.workspace(slim.PHASE_PREFILL, B, Hq, Hkv, self.max_tokens, self.max_tokens, device=device)
        self.ws_decode = slim.weights_workspace(B, Hq, Hkv, self.max_tokens, device=device)
        self.ws_evict = None if budget is None else slim.evict_workspace(B, Hkv, self.max_tokens, budget, device=device)
        self.q_last = None            # the last call's normed and rotated queries

    def _i32(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.device)

    def _append(self, qkv, counts):
        """qkv bf16 [tokens, Hq + 2 Hkv, 128]: the next counts[b] tokens of every sequence, as the fused projection leaves them."""
        if len(counts) != self.B or min(counts) < 0:
            raise ValueError("one count of new tokens per sequence")
        if any(n + c > self.max_tokens for n, c in zip(self.lens, counts)):
            raise ValueError("the cache is full: evict first")
        q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]
        cu = [0]
        for c in counts:
            cu.append(cu[-1] + c)
        positions = self._i32([s + t for s, c in zip(self.seen, counts) for t in range(c)]).view(1, -1)
        self.q_last = torch.empty((qkv.shape[0], self.Hq, slim.HEAD_DIM), dtype=torch.bfloat16, device=self.device)
        slim.slim_norm_rope_append(self.cache, self.rope, q, self.q_last, k, v, positions, self._i32(cu), self._i32(self.lens), self.B)
        self.lens = [n + c for n, c in zip(self.lens, counts)]
        self.seen = [n + c for n, c in zip(self.seen, counts)]
        return cu

    def prompt(self, qkv, counts):
        """Causal attention of the next counts[b] tokens of every sequence; per sequence bf16 [counts[b], Hq, 128]."""
        cu = self._append(qkv, counts)
        out = torch.empty_like(self.q_last)
        slim.slim_attn_prefill(self.cache, self.q_last, out, self._i32(cu), self._i32(self.lens), self.B, max(counts), max(self.lens), self.Hq,
                               self.sm_scale, self.ws_prefill)
        return [out[cu[b]:cu[b + 1]] for b in range(self.B)]

    def step(self, qkv):
        """One new token per sequence (bf16 [B, Hq + 2 Hkv, 128]): appended, attended, every cached token's weight accumulated."""
        self._append(qkv, [1] * self.B)
        out = torch.empty_like(self.q_last)
        slim.slim_attn_decode_weights(self.cache, self.q_last, out, self.weights, self.weights, self._i32(self.weighed), self._i32(self.lens), self.B,
                                      max(self.lens), self.Hq, self.sm_scale, self.decay, self.ws_decode)
        self.weighed = list(self.lens)
        return out

    def evict(self):
        """Cuts every sequence back to the budget.  The weights must cover every cached token: call it after a step."""
        if self.budget is None or self.weighed != self.lens:
            raise ValueError("no budget, or tokens that no step has weighed")
        slim.slim_kv_evict(self.cache, self.weights, self.weights, self.positions, self.positions, self._i32(self.lens), self._i32(self.placed),
                           self._i32(self.seen), self.B, max(self.lens), self.budget, self.n_sink, self.n_recent, self.ws_evict)
        self.lens = [min(n, self.budget) for n in self.lens]
        self.weighed, self.placed = list(self.lens), list(self.lens)


class SampledRun:
    """The attention layers of a batch whose sequences fork and end, on caches of 4 bits (or 8) that share one pool of pages.

    A step is advance() (room for the new tokens), then prompt() or step() for every layer; fork() lets rows continue, share
    or end by parent, compact() moves the pages in use together.  Lengths are kept on the device and, for the launches'
    bounds, here.  A pool without enough pages is a MemoryError, and nothing has changed then.  step() writes one token
    into every row that is not empty: a finished row has to end (a fork in which nobody continues it) before."""

    def __init__(self, n_layers, Hq, Hkv, num_pages, rows, max_tokens, bits=4, device="cuda"):
        if bits not in (4, 8):
            raise ValueError("caches hold 4 or 8 bits")
        self.Hq, self.Hkv, self.rows, self.bits, self.device = Hq, Hkv, rows, bits, torch.device(device)
        stride = (max_tokens + PAGE_TOKENS - 1) // PAGE_TOKENS
        self.max_tokens, self.sm_scale = stride * PAGE_TOKENS, slim.HEAD_DIM ** -0.5
        kind = slim.SlimCache4 if bits == 4 else slim.SlimCache
        self.caches = [kind(rows, Hkv, stride, device=device, num_pages=num_pages) for _ in range(n_layers)]
        self.layers = slim.PageLayers(self.caches)
        self.pages = slim.SlimPages.empty(num_pages, rows, stride, device)
        # the other tables: a fork goes from one set to the other (the page counters are kept in place)
        self.other = slim.SlimPages(self.pages.refs, self.pages.table.clone(), self.pages.held.clone())
        self.lens = [-1] * rows      # -1: the row is empty
        self.counts = [0] * rows     # new tokens of every row, as the last advance() announced them
        self.kv_len, self.len_other = self._i32(self.lens), self._i32(self.lens)
        self.result = self._i32([0, 0])
        self.ws_pages = slim.pages_workspace(num_pages, rows, device)
        self.ws_prefill = slim.workspace(slim.PHASE_PREFILL, rows, Hq, Hkv, self.max_tokens, self.max_tokens, device=device)
        self.ws_decode = slim.decode4_workspace(rows, Hq, Hkv, self.max_tokens, device) if bits == 4 else \
            slim.workspace(slim.PHASE_DECODE, rows, Hq, Hkv, 1, self.max_tokens, device=device)
        self._use_tables()

    def _i32(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.device)

    def _use_tables(self):
        for cache in self.caches:
            cache.set_block_table(self.pages.table)

    def _enough(self):
        missing = int(self.result[0])
        if missing:
            raise MemoryError(f"{missing} pages are missing")

    def advance(self, counts):
        """The next counts[row] tokens of every row; a row that gets its first ones starts a sequence."""
        if len(counts) != self.rows or min(counts) < 0:
            raise ValueError("one count of new tokens per row")
        lens = [max(n, 0) + c if c else n for n, c in zip(self.lens, counts)]
        if max(lens) > self.max_tokens:
            raise ValueError("a row is full")
        kv_len = self._i32(lens)
        slim.slim_pages_grow(self.pages, kv_len, 0, self.result, self.ws_pages)
        self._enough()
        self.counts, self.lens, self.kv_len = list(counts), lens, kv_len

    @staticmethod
    def _rows_are(n, *tensors):
        if any(len(t) != n for t in tensors):
            raise ValueError(f"{n} rows of queries, keys and values are needed")

    def prompt(self, layer, q, k, v):
        """Layer `layer` of the tokens that advance() announced, all rows' one after the other (q bf16 [tokens, Hq, 128], k and v [tokens, Hkv, 128])."""
        cu = [0]
        for c in self.counts:
            cu.append(cu[-1] + c)
        self._rows_are(cu[-1], q, k, v)
        out = torch.empty_like(q)
        if cu[-1] == 0:
            return out
        fn = slim.slim_prefill4_step if self.bits == 4 else slim.slim_prefill_step
        fn(self.caches[layer], q, k, v, out, self._i32(cu), self.kv_len, self.rows, max(self.counts), max(self.lens), self.Hq, self.sm_scale, self.ws_prefill)
        return out

    def step(self, layer, q, k, v):
        """Layer `layer` of one new token in every row that is not empty (q bf16 [rows, Hq, 128], k and v [rows, Hkv, 128]); empty rows give zeros."""
        self._rows_are(self.rows, q, k, v)
        # (the token goes to a row's last position: without room of its own it would take the place of one that is there,
        # which at the end of a page is one that forked rows share)
        if any(c != (1 if n >= 0 else 0) for n, c in zip(self.lens, self.counts)):
            raise ValueError("advance() has to announce one token for every row that is not empty")
        if max(self.lens) < 0:
            return torch.zeros_like(q)
        out = torch.empty_like(q)
        if self.bits == 4:
            slim.slim_attn4_decode(self.caches[layer], q, out, self.kv_len, self.rows, max(self.lens), self.Hq, self.sm_scale, self.ws_decode, k_new=k, v_new=v)
        else:
            slim.slim_decode_step(self.caches[layer], q, k, v, out, self.kv_len, self.rows, max(self.lens), self.Hq, self.sm_scale, self.ws_decode)
        return out

    def fork(self, parents):
        """Row i continues row parents[i]; -1 leaves it empty.  Rows that nobody continues are freed.  Ends the step: advance() comes next."""
        if len(parents) != self.rows or not all(-1 <= p < self.rows for p in parents):
            raise ValueError("one parent per row, -1 for none")
        slim.slim_pages_fork(self.layers, self.pages, self.other, self._i32(parents), self.kv_len, self.len_other, self.result, self.ws_pages)
        self._enough()
        self.pages, self.other = self.other, self.pages
        self.kv_len, self.len_other = self.len_other, self.kv_len
        self._forked(parents)
        self._use_tables()

    def _forked(self, parents):
        self.lens = [self.lens[p] if p >= 0 else -1 for p in parents]
        self.counts = [0] * self.rows

    def compact(self):
        """Moves the pages in use together; returns how many there are.  (Pages kept beside the rows: slim.pages_moved on ws_pages.)"""
        slim.slim_pages_compact(self.layers, self.pages, self.pages, self.result, self.ws_pages)
        return int(self.result[0])


def run_workload(w: Workload, device="cuda", decode_steps=None, block_table=None, num_pages=None, one_call_step=False):
    """The workload's full call sequence.  Returns (LayerRun, prefill outputs per sequence or None,
    {decode step: output [B, Hq, 128]}); decode_steps limits which steps' outputs are kept.  With one_call_step
    every decode step is one slim_decode_step call instead of slim_kv_append followed by slim_attn_decode."""
    run = LayerRun(w, device=device, block_table=block_table, num_pages=num_pages)
    out_prefill = None
    if any(n > 0 for n in w.prefill_len):
        run.append(w.prefill_len)
        out_prefill = run.prefill(w.q_prefill)
    if any(n > 0 for n in w.bulk_len):
        run.append(w.bulk_len)
    outs = {}
    for s in range(w.decode_steps):
        if one_call_step:
            o = run.decode_step(w.q_decode[s])
        else:
            run.append([1] * w.B)
            o = run.decode(w.q_decode[s])
        if decode_steps is None or s in decode_steps:
            outs[s] = o
    torch.cuda.synchronize()
    return run, out_prefill, outs
