"""How calls of packed sequences run."""
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
