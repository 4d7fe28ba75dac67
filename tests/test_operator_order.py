"""The shared-prefix call right behind the kernels that write what it reads, with nothing of the host in between."""
import pytest
import torch

from test_operators import D, PAGE, fill, gen, i32, rope_inputs, shared_setup

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2407_07304_b200 import binding
    return binding


@pytest.mark.parametrize("hq,hkv,batch", [(16, 2, 16), (4, 4, 30)])
def test_decode_shared_sees_what_the_stream_wrote_before_it(hq, hkv, batch):
    """Queries by slim_norm_rope, keys and values of the tails by slim_norm_rope_append (both launched so that the next kernel may
    start early), lengths and prefix by copies: the call's tails start beside the prefix kernel, and must see all of it.
    Every round writes other values into the same arrays; the results are those of rounds with a synchronisation after every
    kernel."""
    slim = _slim()
    pre, rounds = 5 * PAGE, 24
    cache, B, cu = shared_setup(batch, [(5, batch)], hq, hkv, 3)
    codes, scales = cache.codes.clone(), cache.scales.clone()
    rows, inv, _, _, w = rope_inputs(batch, rounds * B, hq, hkv, 128, 1, True)
    rows = rows.view(rounds, B, hq + 2 * hkv, D)
    nr = slim.NormRope(inv, w[0], w[1])
    ones, groups, shared = i32(list(range(B + 1))), i32(cu), i32([pre] * B)
    every = torch.randint(1, 380, (rounds, B), generator=gen(1)).to(torch.int32).cuda() + pre
    ws = slim.shared_workspace(B, hq, hkv, 1, B, pre, 380)

    def run(wait):
        cache.codes.copy_(codes)
        cache.scales.copy_(scales)
        lens, start = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        q = torch.zeros((B, hq, D), dtype=torch.bfloat16, device="cuda")
        outs = torch.zeros((rounds, B, hq, D), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        for r in range(rounds):
            lens.copy_(every[r])
            wait()
            torch.sub(lens, 1, out=start)
            wait()
            x = rows[r]
            slim.slim_norm_rope_append(cache, nr, x[:, :hq], q, x[:, hq:hq + hkv], x[:, hq + hkv:], None, ones, start, B)
            wait()
            slim.slim_attn_decode_shared(cache, q, outs[r], groups, shared, lens, 1, B, B, pre, 380, hq, D ** -0.5, ws)
            wait()
        torch.cuda.synchronize()
        assert slim.slim_read_status(ws) == slim.SLIM_OK and not ws[:slim.WORKSPACE_HEADER_BYTES].any()
        return outs

    slow = run(torch.cuda.synchronize)
    for _ in range(4):
        assert torch.equal(run(lambda: None), slow)
