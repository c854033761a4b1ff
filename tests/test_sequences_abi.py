"""Refusals of the exact attention over sequences and of the paged cache, at the C
ABI (before any HIP call) and in the binding (by name, before the library).  No GPU."""
import pytest
import torch

import paper_2505_18698_amd as ma

A = [(i + 1) << 32 for i in range(11)]  # aligned addresses 4 GB apart that are never dereferenced
HUGE = 1 << 62


def _packed(**x):
    a = dict(q=A[0], k=A[1], v=A[2], out=A[3], lse=A[4], rest=None, cu=A[5], B=2, total=100, Hq=8, Hkv=2, d=64, ldq=512, ldk=128,
             ldv=128, causal=1, clear=0, dtype=1, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_exact_packed_fwd(*a.values())


def _packed_bwd(**x):
    a = dict(q=A[0], k=A[1], v=A[2], out=A[3], lse=A[4], rest=None, dout=A[6], dq=A[7], dk=A[8], dv=A[9], cu=A[5], B=2, total=100,
             Hq=8, Hkv=2, d=64, ldq=512, ldk=128, ldv=128, causal=1, clear=0, dtype=1, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_exact_packed_bwd(*a.values())


def _paged(**x):
    a = dict(q=A[0], k=A[1], v=A[2], out=A[3], lse=A[4], cu=A[5], kv=A[6], table=A[7], B=2, total=100, Hq=8, Hkv=2, d=64, ldq=512,
             pages=50, page=16, blocks=10, causal=1, dtype=1, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_exact_paged_fwd(*a.values())


def _plan(**x):
    a = dict(past=A[0], fresh=A[1], ring=A[2], free=A[3], table=A[4], cu=A[5], kv=A[6], slots=A[7], left=A[8], status=A[9], B=4,
             ring_len=100, blocks=10, page=16, capacity=64, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_paged_plan(*a.values())


def _write(**x):
    a = dict(k=A[0], v=A[1], kp=A[2], vp=A[3], slots=A[4], rows=64, Hkv=2, d=64, ldk=128, ldv=128, pages=50, page=16, dtype=1,
             stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_paged_write(*a.values())


INVALID, UNSUPPORTED = ma.MA_EINVAL, ma.MA_EUNSUPPORTED
HEADS = [(dict(dtype=3), INVALID), (dict(B=-1), INVALID), (dict(total=-1), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID),
         (dict(Hkv=3), INVALID), (dict(d=0), INVALID), (dict(d=60), UNSUPPORTED), (dict(d=136), UNSUPPORTED),
         (dict(d=6, dtype=0), UNSUPPORTED), (dict(Hq=1 << 21, Hkv=1), UNSUPPORTED), (dict(Hq=HUGE, Hkv=2), UNSUPPORTED),
         (dict(total=1 << 31), UNSUPPORTED), (dict(total=HUGE), UNSUPPORTED), (dict(B=1 << 31), UNSUPPORTED), (dict(B=HUGE), UNSUPPORTED),
         (dict(total=1 << 30), UNSUPPORTED), (dict(ldq=504), INVALID), (dict(ldq=516), INVALID), (dict(ldq=1 << 21), UNSUPPORTED),
         (dict(ldq=-512), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(cu=None), INVALID),
         (dict(q=A[0] + 8), INVALID), (dict(out=A[3] + 2), INVALID), (dict(cu=A[5] + 2), INVALID), (dict(lse=A[4] + 1), INVALID),
         (dict(out=A[0]), INVALID), (dict(out=A[0] + 2 * 512 * 99 + 1008), INVALID), (dict(lse=A[3] + 64), INVALID),
         (dict(lse=A[5]), INVALID)]
KV = [(dict(ldk=120), INVALID), (dict(ldv=130), INVALID), (dict(ldk=1 << 21), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=A[2] + 4), INVALID),
      (dict(rest=A[6] + 2), INVALID), (dict(rest=A[6], dtype=0), INVALID)]


@pytest.mark.parametrize("change,code", HEADS + KV + [(dict(rest=A[3]), INVALID), (dict(out=A[2]), INVALID)])
def test_packed_forward(change, code):
    assert _packed(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", [c for c in HEADS if c[0].keys() & {"out", "lse"} == set()] + KV + [
    (dict(out=None), INVALID), (dict(lse=None), INVALID), (dict(dout=None), INVALID), (dict(dq=None), INVALID), (dict(dk=A[8] + 2), INVALID),
    (dict(dq=A[0]), INVALID), (dict(dk=A[9]), INVALID), (dict(dv=A[3]), INVALID), (dict(dq=A[6]), INVALID), (dict(dk=A[4]), INVALID),
    (dict(dv=A[5]), INVALID), (dict(rest=A[7]), INVALID)])
def test_packed_gradient(change, code):
    assert _packed_bwd(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


PAGES = [(dict(page=0), UNSUPPORTED), (dict(page=4), UNSUPPORTED), (dict(page=24), UNSUPPORTED), (dict(page=8192), UNSUPPORTED),
         (dict(page=-16), UNSUPPORTED)]


@pytest.mark.parametrize("change,code", HEADS + PAGES + [
    (dict(pages=-1), INVALID), (dict(pages=HUGE), INVALID), (dict(blocks=-1), INVALID), (dict(blocks=HUGE), INVALID), (dict(k=None), INVALID),
    (dict(v=A[2] + 8), INVALID), (dict(kv=None), INVALID), (dict(kv=A[6] + 2), INVALID), (dict(table=None), INVALID),
    (dict(table=A[7] + 1), INVALID), (dict(out=A[1]), INVALID), (dict(out=A[7]), INVALID), (dict(lse=A[6]), INVALID)])
def test_paged_attention(change, code):
    assert _paged(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", PAGES + [
    (dict(B=-1), INVALID), (dict(ring_len=-1), INVALID), (dict(blocks=-1), INVALID), (dict(capacity=-1), INVALID), (dict(B=8193), UNSUPPORTED),
    (dict(capacity=1 << 31), UNSUPPORTED), (dict(blocks=1 << 31), UNSUPPORTED), (dict(ring_len=1 << 31), UNSUPPORTED)]
    + [({n: None}, INVALID) for n in ("past", "fresh", "ring", "free", "table", "cu", "kv", "slots", "left", "status")]
    + [({n: (1 << 20) + 2}, INVALID) for n in ("past", "fresh", "ring", "free", "table", "cu", "kv", "left", "status")]
    + [(dict(slots=A[7] + 4), INVALID), (dict(left=A[3]), INVALID), (dict(cu=A[0]), INVALID), (dict(kv=A[1]), INVALID),
       (dict(table=A[2]), INVALID), (dict(status=A[8]), INVALID), (dict(kv=A[5] + 4), INVALID)])
def test_plan(change, code):
    assert _plan(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", PAGES + [
    (dict(dtype=9), INVALID), (dict(rows=-1), INVALID), (dict(Hkv=0), INVALID), (dict(d=20), UNSUPPORTED), (dict(ldk=64), INVALID),
    (dict(ldv=132), INVALID), (dict(pages=-2), INVALID), (dict(rows=HUGE), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=A[1] + 2), INVALID),
    (dict(kp=None), INVALID), (dict(vp=A[3] + 8), INVALID), (dict(slots=None), INVALID), (dict(slots=A[4] + 4), INVALID),
    (dict(kp=A[0]), INVALID), (dict(vp=A[2]), INVALID), (dict(kp=A[4]), INVALID)])
def test_write(change, code):
    assert _write(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


def test_calls_with_nothing_to_compute():
    nothing = dict(q=None, k=None, v=None, out=None, lse=None, cu=None)
    for empty in (dict(B=0), dict(total=0)):
        assert _packed(**nothing, **empty) == ma.MA_OK
        assert _packed_bwd(**nothing, dout=None, dq=None, dk=None, dv=None, **empty) == ma.MA_OK
        if "B" in empty:  # rows of no sequence are cleared all the same: the pointers are needed
            assert _packed(**nothing, **empty, clear=1) == _packed_bwd(**nothing, dout=None, **empty, clear=1) == ma.MA_EINVAL
        assert _paged(**nothing, kv=None, table=None, **empty) == ma.MA_OK
    assert _write(rows=0, k=None, v=None, kp=None, vp=None, slots=None) == ma.MA_OK
    assert _write(pages=0, k=None, v=None, kp=None, vp=None, slots=None) == ma.MA_OK


def test_status_bits_match_the_header():
    import os
    import re

    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "monarch_attn.h")).read()
    for name in ("NO_PAGES", "TABLE_FULL", "BAD_LENGTH", "NO_SLOTS"):
        assert int(re.search(rf"#define MA_PLAN_{name} (\d+)", text).group(1)) == getattr(ma, f"PLAN_{name}")
    assert int(re.search(r"#define MONARCH_ATTN_PLAN_MAX_B (\d+)", text).group(1)) == ma.PLAN_MAX_B


# ---- the binding (host tensors that say they are device tensors; the library is replaced) ----

class _Tensor(torch.Tensor):
    is_cuda = True


class _Library:
    def __getattr__(self, name):
        def reached(*args):
            raise AssertionError(f"{name} reached")

        return reached


def _t(*shape, dtype=torch.bfloat16, device="cpu"):
    return torch.zeros(shape, dtype=dtype, device=device).as_subclass(_Tensor)


@pytest.fixture
def no_library(monkeypatch):
    from paper_2505_18698_amd import _binding

    monkeypatch.setattr(_binding, "LIB", _Library())
    monkeypatch.setattr(_binding._torch(), "current_device", lambda: None)
    monkeypatch.setattr(_binding._torch(), "current_stream", lambda index: 0)


I32, I64, F32 = torch.int32, torch.int64, torch.float32
CALLS = {
    "packed_fwd": (lambda **t: ma.monarch_attn_exact_packed_fwd(**t), dict(
        q=_t(10, 4, 8), k=_t(10, 2, 8), v=_t(10, 2, 8), out=_t(10, 4, 8), cu_seqlens=_t(3, dtype=I32), lse=_t(4, 10, dtype=F32),
        rest=_t(10, 4, 8))),
    "packed_bwd": (lambda **t: ma.monarch_attn_exact_packed_bwd(**t), dict(
        q=_t(10, 4, 8), k=_t(10, 2, 8), v=_t(10, 2, 8), out=_t(10, 4, 8), lse=_t(4, 10, dtype=F32), dout=_t(10, 4, 8), dq=_t(10, 4, 8),
        dk=_t(10, 2, 8), dv=_t(10, 2, 8), cu_seqlens=_t(3, dtype=I32), rest=_t(10, 4, 8))),
    "paged_fwd": (lambda **t: ma.monarch_attn_exact_paged_fwd(**t), dict(
        q=_t(10, 4, 8), k_pages=_t(6, 2, 16, 8), v_pages=_t(6, 2, 16, 8), out=_t(10, 4, 8), cu_seqlens=_t(3, dtype=I32),
        kv_lens=_t(2, dtype=I32), block_table=_t(2, 5, dtype=I32), lse=_t(4, 10, dtype=F32))),
    "plan": (lambda **t: ma.monarch_attn_paged_plan(**t, page=16), dict(
        past=_t(2, dtype=I32), fresh=_t(2, dtype=I32), ring=_t(9, dtype=I32), free_in=_t(2, dtype=I32), block_table=_t(2, 5, dtype=I32),
        cu_seqlens=_t(3, dtype=I32), kv_lens=_t(2, dtype=I32), slots=_t(10, dtype=I64), free_out=_t(2, dtype=I32), status=_t(1, dtype=I32))),
    "write": (lambda **t: ma.monarch_attn_paged_write(**t), dict(
        k=_t(10, 2, 8), v=_t(10, 2, 8), k_pages=_t(6, 2, 16, 8), v_pages=_t(6, 2, 16, 8), slots=_t(10, dtype=I64))),
}


@pytest.mark.parametrize("name", CALLS)
def test_matching_tensors_reach_the_library(no_library, name):
    call, tensors = CALLS[name]
    with pytest.raises(AssertionError, match="reached"):
        call(**tensors)


@pytest.mark.parametrize("fault", ["none", "host", "dtype", "more", "flat", "strided", "device"])
@pytest.mark.parametrize("name", CALLS)
def test_each_tensor_is_checked(no_library, name, fault):
    call, tensors = CALLS[name]
    free = {"plan": ("ring", "slots", "block_table"), "paged_fwd": ("block_table",)}  # of any length
    for arg, t in tensors.items():
        if fault == "none" and arg in ("lse", "rest") and name != "packed_bwd" or fault == "none" and arg == "rest":
            continue  # optional
        if fault == "more" and arg in free.get(name, ()) or fault == "strided" and t.numel() == 1 or arg == "cu_seqlens" and name.startswith("packed") and fault == "more":
            continue
        bad = {"none": lambda: None, "host": lambda: torch.zeros(t.shape, dtype=t.dtype, device="meta"),
               "dtype": lambda: _t(*t.shape, dtype=torch.float64), "more": lambda: _t(*t.shape[:-1], t.shape[-1] + 1, dtype=t.dtype),
               "flat": lambda: _t(t.numel(), 1, 1, 1, 1, dtype=t.dtype), "device": lambda: _t(*t.shape, dtype=t.dtype, device="meta"),
               "strided": lambda: torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype).as_subclass(_Tensor)[..., ::2]}[fault]()
        with pytest.raises((TypeError, ValueError)):
            call(**{**tensors, arg: bad})


def test_rows_may_be_strided(no_library):
    call, tensors = CALLS["packed_fwd"]
    joint = _t(10, 64)
    q, k, v = (x.unflatten(1, (-1, 8)) for x in joint.split((32, 16, 16), 1))
    with pytest.raises(AssertionError, match="reached"):
        call(**{**tensors, "q": q, "k": k, "v": v})
    with pytest.raises(ValueError, match="k must be"):  # heads that are not adjacent
        call(**{**tensors, "k": _t(2, 10, 8).transpose(0, 1)})
    with pytest.raises(ValueError, match="out must be"):
        call(**{**tensors, "out": q})


def test_heads_wider_than_their_tiles_are_refused():
    """Offsets within a tile count heads of the tile's width: 32768 heads of 32 columns take 2^21."""
    assert _paged(Hq=1 << 15, Hkv=1, d=32, ldq=1 << 20) == UNSUPPORTED
    assert "rounded up" in ma.monarch_attn_last_error()
