"""Head counts whose rows per token pass 32 bits.  No GPU: the host's checks answer."""
import pytest

from test_operator_refusals import UNSUPPORTED, cache, call_append, call_norm_rope

MANY = (1 << 31) - 1


@pytest.mark.parametrize("kw", [dict(hq=MANY, hkv=2), dict(hq=2, hkv=MANY), dict(hq=MANY, hkv=MANY), dict(hq=1 << 30, hkv=1 << 30)])
def test_norm_rope_refuses_rows_beyond_32_bits(kw):
    assert call_norm_rope(n=1, qs=MANY * 128 + 128, ks=MANY * 128 + 128, **kw) == UNSUPPORTED


@pytest.mark.parametrize("hq,hkv,n", [(MANY, 1, 1), (0, 1 << 30, 1), (4, 1 << 30, 3), (MANY - 1, 2, 1), (64, 8, 1 << 25)])
def test_norm_rope_append_refuses_rows_beyond_32_bits(hq, hkv, n):
    assert call_append(c=cache(num_kv_heads=hkv), hq=hq, n=n, qs=MANY * 128 + 128, ks=MANY * 128 + 128, vs=MANY * 128 + 128) == UNSUPPORTED
