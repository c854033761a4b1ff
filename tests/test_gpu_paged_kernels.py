"""Every kernel of the attention over pages: each type and tile width, with few
and with many rows a sequence, in one launch and split over the keys."""
import pytest
import torch

from sequence_reference import DTYPES, starts
from test_gpu_paged import _attend, _cache, _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def _launches(ma, call):
    ma.monarch_attn_timing_enable(True)
    try:
        call()
        return [kind for kind, _ in ma.monarch_attn_timing_read()]
    finally:
        ma.monarch_attn_timing_enable(False)


# A call is split where the keys of a row of the table take more than 128 KB: from 256 (fp32, 128 columns) to 1024 keys.
ROWS = {"few": ([1, 2, 1, 1], [0, 130, 199, 64]), "many": ([40, 3, 70], [100, 0, 129])}


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 64), (8, 2, 96), (6, 2, 80), (4, 1, 128), (3, 3, 104)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_each_kernel(ma, dtype, Hq, Hkv, d, rows, split):
    print(dtype, Hq, Hkv, d, rows, split, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(81)
    new, past = ROWS[rows]
    if split:
        past = [past[0], past[1] + 1700, *past[2:]]
    seqs, kp, vp, table, kv = _cache(new, past, Hkv, d, 16, dtype, gen)
    cu = starts(new, "cuda", 1)
    q = torch.randn(sum(new) + 2, Hq, d, generator=gen, device="cuda").to(DTYPES[dtype])
    got = []
    launches = _launches(ma, lambda: got.extend(_attend(ma, q, kp, vp, cu, kv, table)))
    assert ("seq_join" in launches) == split
    _check(*got, q, cu, seqs, past)
    for _ in range(3):
        again = _attend(ma, q, kp, vp, cu, kv, table)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
