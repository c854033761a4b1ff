"""Every kernel of the attention over pages: each type and tile width, with few
and with many rows a sequence, in one launch and split over the keys."""
import pytest
import torch

from sequence_reference import DTYPES, attention, starts, worst
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


def test_workspace_of_a_split_call(ma):
    """900 requests on 8 key heads: two segments of 32 rows a workgroup (17 MB), not one a request more (133 MB)."""
    gen = torch.Generator(device="cuda").manual_seed(82)
    seqs, kp, vp, table, kv = _cache([1] * 900, [1000 if i % 300 == 0 else i % 40 for i in range(900)], 8, 128, 16, "bf16", gen)
    q = torch.randn(900, 32, 128, generator=gen, device="cuda").bfloat16()
    cu = starts([1] * 900, "cuda")
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    ma.monarch_attn_release_workspace()
    free = torch.cuda.mem_get_info()[0]
    ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table)
    torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] < 40 << 20
    for i in (0, 1, 39, 300, 623, 899):
        assert worst(out[i : i + 1], *attention(q[i : i + 1], *seqs[i], True, len(seqs[i][0]) - 1)["out"]) <= 1.0, i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_context_among_many_short_ones(ma, dtype):
    """However many single tokens there are, the work is shared evenly."""
    gen = torch.Generator(device="cuda").manual_seed(83)
    past = [9000 if i == 700 else i % 50 for i in range(1200)]
    seqs, kp, vp, table, kv = _cache([1] * 1200, past, 8, 64, 16, dtype, gen)
    q = torch.randn(1200, 16, 64, generator=gen, device="cuda").to(DTYPES[dtype])
    got = []
    launches = _launches(ma, lambda: got.extend(_attend(ma, q, kp, vp, starts([1] * 1200, "cuda"), kv, table)))
    assert "seq_join" in launches
    for i in (0, 1, 49, 699, 700, 701, 1199):
        ref = attention(q[i : i + 1], *seqs[i], True, past[i])
        assert worst(got[0][i : i + 1], *ref["out"]) <= 1.0 and worst(got[1][:, i : i + 1], *ref["lse"]) <= 1.0, i


def test_two_streams_at_once_over_shared_pages(ma):
    """Split calls on two streams, whose requests share pages of a common prefix: each the bits of a call alone."""
    gen = torch.Generator(device="cuda").manual_seed(84)
    _, kp, vp, table, kv = _cache([1, 1, 1, 40], [3000, 2000, 900, 1700], 2, 64, 16, "bf16", gen)
    table[1:, :50] = table[0, :50]  # 800 tokens
    cu = starts([1, 1, 1, 40], "cuda")
    qs = [torch.randn(43, 8, 64, generator=gen, device="cuda").bfloat16() for _ in range(2)]
    want = [_attend(ma, q, kp, vp, cu, kv, table) for q in qs]
    got = [(torch.empty_like(o), torch.empty_like(x)) for o, x in want]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for q, (out, lse), s in zip(qs, got, streams):
            ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table, True, lse, stream=s)
    torch.cuda.synchronize()
    for (o, x), (out, lse) in zip(want, got):
        assert torch.equal(o, out) and torch.equal(x, lse)
    for row, i in ((0, 0), (1, 1), (2, 2)):
        n = int(kv[i])
        pos = torch.arange(n, device="cuda")
        k, v = (t[table[i, pos // 16].long(), :, pos % 16] for t in (kp, vp))
        assert worst(want[0][0][row : row + 1], *attention(qs[0][row : row + 1], k, v, True, n - 1)["out"]) <= 1.0, i
