"""fp16: weights and gradients far below the largest one."""
import math

import pytest
import torch

from sequence_reference import attention, starts, worst
from test_gpu_sequences import _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


@pytest.mark.parametrize("causal", [True, False])
def test_many_small_weights_beside_a_large_one(ma, causal):
    """The first key has the weight 1, and each of the n = 2^17 - 1 others 2^-25.1, less than half of fp16's smallest
    number: together they are 0.36 % of the row.

    With |V| = 1 and A the sum of the weights, 1, the row may be off by 2^-11 for its own rounding, 2^-11 for the
    weights', and the fp32 sums: the products add 16 keys at a time, n / 16 roundings of 2^-24, the weights' sum fewer,
    and a score's 68 roundings of 2^-24 |s| shift its weight (17.4 = 25.1 ln 2)."""
    n, d, rows = 1 << 17, 64, slice(-8, None)
    q, k, v = (torch.zeros(n, 1, d, device="cuda") for _ in range(3))
    q[..., 0], k[0, 0, 0] = 16.0, 25.1 * math.log(2.0) / 2  # s q.k = 2 k
    v[:] = torch.where(torch.arange(d, device="cuda") % 3 == 0, -1.0, 1.0)
    q, k, v = q.half(), k.half(), v.half()
    out, lse = torch.zeros_like(q), torch.zeros(1, n, device="cuda")
    ma.monarch_attn_exact_packed_fwd(q, k, v, out, starts([n], "cuda"), causal, lse)
    torch.cuda.synchronize()
    ref = attention(q[rows], k, v, causal, n - 8)
    bound = 2 * 2.0 ** -11 + (n / 16 + 68 * 17.5) * 2.0 ** -24
    assert float((out[rows].double() - ref["out"][0]).abs().max()) <= bound < 0.0017
    assert worst(lse[:, rows], *ref["lse"]) <= 1.0


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("small", [0, 1])
def test_gradients_of_sequences_of_different_scales(ma, small, causal):
    """One sequence's upstream gradient is 2^23 times the other's: each gradient is as exact as alone, and its bits do
    not depend on the other sequence."""
    q, k, v, dout, cu = _inputs([500, 450], 4, 2, 64, "f16", 51, spare=0, first=0)
    seqs = slice(0, 500), slice(500, 950)
    x = dout.clone()
    x[seqs[small]] *= 2.0 ** -10
    alone = _run(ma, q, k, v, x, cu, causal)
    x[seqs[1 - small]] *= 2.0 ** 12
    r = _run(ma, q, k, v, x, cu, causal)
    for i, rows in enumerate(seqs):
        ref = attention(q[rows], k[rows], v[rows], causal, 0, x[rows])
        for name in ("dq", "dk", "dv"):
            assert worst(r[name][rows], *ref[name]) <= 1.0, (i, name)
            assert i != small or torch.equal(r[name][rows], alone[name][rows]), name


def test_gradients_of_rows_of_different_scales(ma):
    """Rows of one sequence whose upstream gradients differ by 2^24: dQ is exact row by row.  (dK and dV sum over the
    rows, relative to the largest.)"""
    q, k, v, dout, cu = _inputs([700], 2, 1, 96, "f16", 52, spare=0, first=0)
    x = dout.clone()
    x[::2] *= 2.0 ** 12
    x[1::2] *= 2.0 ** -12
    assert worst(_run(ma, q, k, v, x, cu, True)["dq"], *attention(q, k, v, True, 0, x)["dq"]) <= 1.0
