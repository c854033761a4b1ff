"""Keys of weight zero in a split call: scores of -inf that a row sees."""
import math

import pytest
import torch

from sequence_reference import DTYPES, attention, starts, worst
from test_gpu_paged import _attend, _cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def _with_scores_of_minus_infinity(new, past, d, dtype, where, seed):
    """A cache in which the keys `where` of every sequence have the score -inf for every row, and its queries."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    seqs, kp, vp, table, kv = _cache(new, past, 2, d, 16, dtype, gen)
    q = torch.randn(sum(new), 4, d, generator=gen, device="cuda")
    q[..., 0] = 1.0
    for (k, _), row in zip(seqs, table.tolist()):
        for t in range(*where.indices(len(k))):
            kp[row[t // 16], :, t % 16, 0] = -math.inf
    return seqs, kp, vp, table, kv, q.to(DTYPES[dtype])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,past", [([1], [2999]), ([2, 1], [2800, 3100]), ([60], [2940])])
def test_a_long_run_of_keys_has_no_weight(ma, new, past, d, dtype):
    """Whole parts of the split have no weight: the row is that of the other keys."""
    print(new, past, d, dtype, flush=True)
    seqs, kp, vp, table, kv, q = _with_scores_of_minus_infinity(new, past, d, dtype, slice(300, 2700), 91)
    out, lse = _attend(ma, q, kp, vp, starts(new, "cuda"), kv, table)
    at = 0
    for n, p, (k, v) in zip(new, past, seqs):
        keep = torch.ones(len(k), dtype=torch.bool, device="cuda")
        keep[300:2700] = False
        ref = attention(q[at : at + n], k[keep], v[keep], True, p - 2400)
        assert worst(out[at : at + n], *ref["out"]) <= 1.0 and worst(lse[:, at : at + n], *ref["lse"]) <= 1.0
        at += n


@pytest.mark.parametrize("keys", [200, 3000])  # in one launch, and split
@pytest.mark.parametrize("rows", [1, 60])
def test_no_key_has_a_weight(ma, keys, rows):
    """All scores of a row -inf: exp(s - lse) is no number, and neither is the row, however the call runs."""
    seqs, kp, vp, table, kv, q = _with_scores_of_minus_infinity([rows], [keys - rows], 64, "bf16", slice(0, None), 92)
    out, lse = _attend(ma, q, kp, vp, starts([rows], "cuda"), kv, table)
    assert bool(torch.isnan(out).all()) and bool((lse == -math.inf).all())
