"""Refusals of cross attention, at the C ABI (before any HIP call) and in the binding (by name, before the library).  No GPU."""
import pytest
import torch

import paper_2505_18698_amd as ma

A = [(i + 1) << 42 for i in range(13)]  # aligned addresses far apart that are never dereferenced
HUGE = 1 << 62
INVALID, UNSUPPORTED = ma.MA_EINVAL, ma.MA_EUNSUPPORTED
SIZES = dict(B=2, total=100, total_k=300, Hq=8, Hkv=2, d=64, ldq=512, ldk=128, ldv=256, clear=0, dtype=1, stream=None)


def _fwd(**x):
    a = dict(q=A[0], k=A[1], v=A[2], out=A[3], lse=A[4], rest=A[5], cu_q=A[6], cu_k=A[7], k_lens=A[8]) | SIZES
    a.update(x)
    return ma.LIB.monarch_attn_exact_cross_fwd(*a.values())


def _bwd(**x):
    a = dict(q=A[0], k=A[1], v=A[2], out=A[3], lse=A[4], rest=A[5], dout=A[9], dq=A[10], dk=A[11], dv=A[12], cu_q=A[6], cu_k=A[7],
             k_lens=A[8]) | SIZES
    a.update(x)
    return ma.LIB.monarch_attn_exact_cross_bwd(*a.values())


BOTH = [(dict(dtype=3), INVALID), (dict(B=-1), INVALID), (dict(total=-1), INVALID), (dict(total_k=-1), INVALID), (dict(Hq=0), INVALID),
        (dict(Hkv=0), INVALID), (dict(Hkv=3), INVALID), (dict(d=0), INVALID), (dict(d=60), UNSUPPORTED), (dict(d=136), UNSUPPORTED),
        (dict(d=6, dtype=0), UNSUPPORTED), (dict(Hq=1 << 21, Hkv=1), UNSUPPORTED), (dict(Hq=HUGE, Hkv=2), UNSUPPORTED),
        (dict(total=1 << 31), UNSUPPORTED), (dict(total=HUGE), UNSUPPORTED), (dict(total=1 << 30), UNSUPPORTED),
        (dict(total_k=1 << 31), UNSUPPORTED), (dict(total_k=HUGE), UNSUPPORTED), (dict(B=1 << 31), UNSUPPORTED), (dict(B=HUGE), UNSUPPORTED),
        (dict(ldq=504), INVALID), (dict(ldq=516), INVALID), (dict(ldq=1 << 21), UNSUPPORTED), (dict(ldk=120), INVALID), (dict(ldv=130), INVALID),
        (dict(ldk=1 << 21), UNSUPPORTED), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
        (dict(cu_q=None), INVALID), (dict(cu_k=None), INVALID), (dict(q=A[0] + 8), INVALID), (dict(k=A[1] + 2), INVALID),
        (dict(out=A[3] + 2), INVALID), (dict(cu_q=A[6] + 2), INVALID), (dict(cu_k=A[7] + 1), INVALID), (dict(k_lens=A[8] + 2), INVALID),
        (dict(rest=A[5] + 2), INVALID), (dict(rest=A[5], dtype=0), INVALID), (dict(B=1 << 24), UNSUPPORTED)]


@pytest.mark.parametrize("change,code", BOTH + [
    (dict(lse=A[4] + 1), INVALID), (dict(out=A[0]), INVALID), (dict(out=A[1]), INVALID), (dict(out=A[2] + 299 * 512 + 240), INVALID),
    (dict(lse=A[3] + 64), INVALID), (dict(lse=A[6]), INVALID), (dict(rest=A[3]), INVALID), (dict(out=A[7]), INVALID), (dict(out=A[8]), INVALID)])
def test_forward(change, code):
    assert _fwd(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", BOTH + [
    (dict(lse=None), INVALID), (dict(dout=None), INVALID), (dict(dq=None), INVALID), (dict(dk=None), INVALID), (dict(dv=A[12] + 8), INVALID),
    (dict(dq=A[0]), INVALID), (dict(dk=A[12]), INVALID), (dict(dv=A[3]), INVALID), (dict(dq=A[9]), INVALID), (dict(dk=A[4]), INVALID),
    (dict(dv=A[8]), INVALID), (dict(rest=A[10]), INVALID)])
def test_gradient(change, code):
    assert _bwd(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


def test_calls_with_nothing_to_compute():
    nothing = dict(q=None, k=None, v=None, out=None, lse=None, rest=None, cu_q=None, cu_k=None, k_lens=None)
    for empty in (dict(B=0), dict(total=0)):
        assert _fwd(**nothing, **empty) == ma.MA_OK
    for empty in (dict(B=0), dict(total=0, total_k=0)):
        assert _bwd(**nothing, dout=None, dq=None, dk=None, dv=None, **empty) == ma.MA_OK
    # gradients of keys without queries are zero, rows of no sequence are cleared: the pointers are needed
    assert _bwd(**nothing, dout=None, total=0) == INVALID
    assert _fwd(**nothing, B=0, clear=1) == _bwd(**nothing, dout=None, B=0, clear=1) == INVALID


def _tensors():
    q = torch.zeros(6, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(9, 2, 64, dtype=torch.bfloat16)
    return q, k, torch.tensor([0, 6], dtype=torch.int32)


def test_binding_names_what_it_refuses():
    q, k, cu = _tensors()
    with pytest.raises(TypeError, match="q must be a device tensor"):
        ma.monarch_attn_exact_cross_fwd(q, k, k, torch.zeros_like(q), cu, cu)
    with pytest.raises(TypeError, match="q must be a device tensor"):
        ma.monarch_attn_exact_cross_fwd(None, k, k, None, cu, cu)
    with pytest.raises(TypeError, match="q must be a device tensor"):
        ma.exact_cross_attention(q, k, k, cu, cu)


class _Device(torch.Tensor):
    """A CPU tensor that says it is on a device: the checks before the library see nothing else."""

    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def _on_device(*tensors):
    return [t.as_subclass(_Device) for t in tensors]


@pytest.mark.parametrize("change,message", [
    (dict(k=torch.zeros(9, 2, 32, dtype=torch.bfloat16)), "head dimension of q"), (dict(v=torch.zeros(8, 2, 64, dtype=torch.bfloat16)), "head dimension of q"),
    (dict(k=torch.zeros(9, 2, 64)), "k must match q in dtype"), (dict(k=torch.zeros(9, 128, dtype=torch.bfloat16)), "k must be a .rows, heads, d. tensor"),
    (dict(cu_q=torch.zeros(2, dtype=torch.int64)), "cu_q must be a contiguous torch.int32"), (dict(cu_k=torch.zeros(3, dtype=torch.int32)), "cu_k must be"),
    (dict(cu_q=torch.zeros(0, dtype=torch.int32)), "cu_q must be an int32 tensor"), (dict(k_lens=torch.zeros(2, dtype=torch.int32)), "k_lens must be"),
    (dict(k_lens=torch.zeros(1)), "k_lens must be"), (dict(out=torch.zeros(6, 4, 64)), "out must be"), (dict(out=torch.zeros(6, 64, 4, dtype=torch.bfloat16)), "out must be"),
    (dict(lse=torch.zeros(6, 4)), "lse must be"), (dict(rest=torch.zeros(6, 4, 64)), "rest must be")])
def test_binding_checks_shapes(change, message):
    q, k, cu = _tensors()
    a = dict(q=q, k=k, v=k.clone(), out=torch.zeros_like(q), cu_q=cu, cu_k=cu.clone(), k_lens=None) | change
    a = {n: t if t is None else _on_device(t)[0] for n, t in a.items()}
    with pytest.raises(ValueError, match=message):
        ma.monarch_attn_exact_cross_fwd(**a)
