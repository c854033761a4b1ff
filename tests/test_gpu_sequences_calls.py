"""How calls of packed sequences run."""
import math

import pytest
import torch

from test_gpu_paged_kernels import _launches
from test_gpu_sequences import _check, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,Hq,Hkv,d,join", [
    ([10] * 64, 4, 4, 64, False),  # no walk over the call's rows has the tiles of two pieces
    ([64, 700, 0, 1, 600, 100], 2, 2, 64, True),  # walks of 1 to 11 tiles
    ([1, 40, 1400, 90, 3, 2, 500], 6, 2, 96, True),  # 3 to 66
    ([33] * 30, 8, 1, 128, True),  # 8 each
    ([129, 31, 1], 32, 1, 40, True)])
def test_pieces_of_the_gradient(ma, lens, Hq, Hkv, d, join, causal, dtype):
    """Walks of all lengths, cut into pieces, whose sums a further launch adds up."""
    x = _inputs(lens, Hq, Hkv, d, dtype, 61)
    r = {}
    assert ("seq_bwd_join" in _launches(ma, lambda: r.update(_run(ma, *x, causal)))) == join
    _check(r, *x, causal)
    again = _run(ma, *x, causal)
    assert all(torch.equal(r[n], again[n]) for n in r)


def test_rows_far_apart_are_copied(ma):
    """The torch op takes rows further apart than the kernels do."""
    q, k, v, dout, cu = _inputs([30, 9], 4, 2, 64, "bf16", 62, spare=0, first=0)
    want = _run(ma, q, k, v, dout, cu, True)
    buf = torch.zeros(39, (1 << 20) + 8, device="cuda", dtype=torch.bfloat16)
    leaves = []
    for i, t in enumerate((q, k, v)):
        far = buf[:, 256 * i : 256 * i + t.shape[1] * 64].unflatten(1, (-1, 64))
        leaves.append(far.copy_(t).detach().requires_grad_())
    out = ma.exact_attention_packed(*leaves, cu)
    assert torch.equal(out, want["out"])
    for g, n in zip(torch.autograd.grad(out, leaves, dout), ("dq", "dk", "dv")):
        assert torch.equal(g, want[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_without_a_mask(ma, bad, dtype):
    """Every weight is positive, so the column of the sequence becomes the value; nothing else changes."""
    q, k, v, _, cu = _inputs([40, 130, 9], 4, 2, 64, dtype, 63, spare=0, first=0)
    clean = _run(ma, q, k, v, None, cu, False)["out"]
    for at, rows in ((10, slice(0, 40)), (45, slice(40, 170)), (168, slice(40, 170)), (175, slice(170, 179))):
        keep = v[at].clone()
        v[at, 1, 5] = bad
        out = _run(ma, q, k, v, None, cu, False)["out"]
        want = clean.clone()
        want[rows, 2:, 5] = bad
        assert torch.equal(out, want) if not math.isnan(bad) else torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0)), at
        v[at] = keep
