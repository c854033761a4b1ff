"""Calls of more workgroups than HIP launches (2^32 threads of 256) are refused before any launch.  No GPU."""
import pytest

import paper_2505_18698_amd as ma
from test_sequences_abi import _packed, _packed_bwd, _paged, _write

MANY = 1 << 24
FAR = [(i + 1) << 42 for i in range(11)]  # far enough apart for these sizes
PACKED = dict(zip(("q", "k", "v", "out", "lse", "cu", "dout", "dq", "dk", "dv"), FAR))


@pytest.mark.parametrize("sizes", [dict(B=MANY // 2), dict(B=MANY, Hkv=1, Hq=1, ldq=64), dict(total=1 << 30, Hq=8, Hkv=8, ldk=512, ldv=512)])
def test_packed(sizes):
    for call, more in ((_packed, 6), (_packed_bwd, 10)):
        names = list(PACKED)[:more]
        assert call(**{n: PACKED[n] for n in names}, **sizes) == ma.MA_EUNSUPPORTED, ma.monarch_attn_last_error()
        assert "grid" in ma.monarch_attn_last_error()


@pytest.mark.parametrize("sizes", [dict(B=MANY // 2), dict(B=MANY, total=MANY)])
def test_paged(sizes):
    at = dict(zip(("q", "k", "v", "out", "lse", "cu", "kv", "table"), FAR))
    assert _paged(**at, **sizes) == ma.MA_EUNSUPPORTED and "grid" in ma.monarch_attn_last_error()


def test_write():
    at = dict(zip(("k", "v", "kp", "vp", "slots"), FAR))
    assert _write(**at, rows=MANY, Hkv=128, ldk=8192, ldv=8192) == ma.MA_EUNSUPPORTED and "grid" in ma.monarch_attn_last_error()
