"""Refusals of the rotation, the append, the selection of beams and the cache's reordering, at the C ABI (before any HIP
call) and in the binding (by name, before the library).  No GPU."""
import pytest
import torch

import paper_2505_18698_amd as ma
from test_cross_abi import _on_device

A = [(i + 1) << 42 for i in range(11)]  # aligned addresses far apart that are never dereferenced
HUGE = 1 << 62
INVALID, UNSUPPORTED = ma.MA_EINVAL, ma.MA_EUNSUPPORTED


def _rotate(**x):
    a = dict(q=A[0], k=A[1], q_out=A[2], k_out=A[3], freq=A[4], cu=A[5], kv=A[6], B=2, total=100, Hq=8, Hk=2, d=64, rot=64, ldq=512,
             ldk=128, interleaved=0, inverse=0, clear=0, dtype=1, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_rotate(*a.values())


def _append(**x):
    a = dict(q=A[0], k=A[1], v=A[2], q_out=A[3], kp=A[4], vp=A[5], freq=A[6], cu=A[7], kv=A[8], slots=A[9], B=2, total=100, Hq=8, Hkv=2,
             d=64, rot=64, ldq=512, ldk=128, ldv=256, pages=50, page=16, interleaved=0, dtype=1, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_paged_append(*a.values())


def _select(**x):
    a = dict(logits=A[0], scores=A[1], done=A[2], out=A[3], tokens=A[4], parents=A[5], done_out=A[6], B=2, K=4, V=1000, M=8, ld=1000, eos=2,
             dtype=1, stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_beam_select(*a.values())


def _reorder(**x):
    a = dict(kp=A[0], vp=A[1], table=A[2], parents=A[3], lens=A[4], B=2, K=4, Hkv=2, d=64, pages=50, page=16, blocks=10, move=1, dtype=1,
             stream=None)
    a.update(x)
    return ma.LIB.monarch_attn_paged_reorder(*a.values())


ROTATION = [(dict(dtype=3), INVALID), (dict(B=-1), INVALID), (dict(total=-1), INVALID), (dict(Hq=0), INVALID), (dict(d=0), INVALID),
            (dict(d=60, rot=56), UNSUPPORTED), (dict(d=136), UNSUPPORTED), (dict(Hq=HUGE), UNSUPPORTED), (dict(total=1 << 31), UNSUPPORTED),
            (dict(total=HUGE), UNSUPPORTED), (dict(B=HUGE), UNSUPPORTED), (dict(rot=0), INVALID), (dict(rot=-8), INVALID), (dict(rot=72), INVALID),
            (dict(rot=7), INVALID), (dict(rot=12), UNSUPPORTED), (dict(rot=4), UNSUPPORTED), (dict(ldq=504), INVALID), (dict(ldq=516), INVALID),
            (dict(ldq=1 << 21), UNSUPPORTED), (dict(ldk=120), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(q_out=None), INVALID),
            (dict(freq=None), INVALID), (dict(cu=None), INVALID), (dict(q=A[0] + 8), INVALID), (dict(k=A[1] + 2), INVALID), (dict(q_out=A[0]), INVALID)]


@pytest.mark.parametrize("change,code", ROTATION + [
    (dict(Hk=-1), INVALID), (dict(Hk=HUGE), UNSUPPORTED), (dict(k_out=None), INVALID), (dict(k_out=A[3] + 4), INVALID), (dict(k_out=A[1]), INVALID),
    (dict(q_out=A[3]), INVALID), (dict(q_out=A[4]), INVALID), (dict(k_out=A[5]), INVALID), (dict(k_out=A[6]), INVALID), (dict(freq=A[4] + 2), INVALID),
    (dict(cu=A[5] + 1), INVALID), (dict(kv=A[6] + 2), INVALID)])
def test_rotate(change, code):
    assert _rotate(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", ROTATION + [
    (dict(Hkv=0), INVALID), (dict(Hkv=-1), INVALID), (dict(ldv=130), INVALID), (dict(ldv=64), INVALID), (dict(page=0), UNSUPPORTED),
    (dict(page=24), UNSUPPORTED), (dict(page=8192), UNSUPPORTED), (dict(pages=-1), INVALID), (dict(pages=HUGE), INVALID), (dict(v=None), INVALID),
    (dict(kp=None), INVALID), (dict(vp=A[5] + 8), INVALID), (dict(kv=None), INVALID), (dict(slots=None), INVALID), (dict(slots=A[9] + 4), INVALID),
    (dict(kp=A[5]), INVALID), (dict(vp=A[2]), INVALID), (dict(q_out=A[9]), INVALID), (dict(kp=A[8]), INVALID)])
def test_append(change, code):
    assert _append(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-1), INVALID), (dict(B=-1), INVALID), (dict(K=0), INVALID), (dict(V=0), INVALID), (dict(M=0), INVALID), (dict(K=33), UNSUPPORTED),
    (dict(M=33), UNSUPPORTED), (dict(V=524289, ld=524289), UNSUPPORTED), (dict(V=HUGE, ld=HUGE), UNSUPPORTED), (dict(K=1, V=7, M=8), INVALID),
    (dict(ld=999), INVALID), (dict(ld=HUGE), UNSUPPORTED), (dict(B=HUGE), UNSUPPORTED), (dict(B=1 << 30), UNSUPPORTED), (dict(eos=-1), INVALID),
    (dict(eos=1000), INVALID), (dict(eos=-1, done=None), INVALID), (dict(eos=-1, done_out=None), INVALID), (dict(logits=None), INVALID),
    (dict(logits=A[0] + 1), INVALID), (dict(logits=A[0] + 2, dtype=0), INVALID), (dict(scores=None), INVALID), (dict(scores=A[1] + 2), INVALID),
    (dict(out=None), INVALID), (dict(tokens=None), INVALID), (dict(parents=A[5] + 1), INVALID), (dict(out=A[1]), INVALID), (dict(tokens=A[3]), INVALID),
    (dict(parents=A[0]), INVALID), (dict(done_out=A[2]), INVALID), (dict(done_out=A[3]), INVALID)])
def test_select(change, code):
    assert _select(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


@pytest.mark.parametrize("change,code", [
    (dict(dtype=5), INVALID), (dict(B=-1), INVALID), (dict(K=0), INVALID), (dict(K=33), UNSUPPORTED), (dict(B=65536), UNSUPPORTED), (dict(B=HUGE), UNSUPPORTED),
    (dict(Hkv=0), INVALID), (dict(Hkv=HUGE), UNSUPPORTED), (dict(d=60), UNSUPPORTED), (dict(page=12), UNSUPPORTED), (dict(pages=-1), INVALID),
    (dict(blocks=-1), INVALID), (dict(blocks=HUGE), INVALID), (dict(kp=None), INVALID), (dict(vp=A[1] + 8), INVALID), (dict(table=None), INVALID),
    (dict(parents=None), INVALID), (dict(lens=A[4] + 2), INVALID), (dict(kp=A[1]), INVALID), (dict(table=A[0]), INVALID), (dict(table=A[3]), INVALID),
    (dict(vp=A[4]), INVALID)])
def test_reorder(change, code):
    assert _reorder(**change) == code, ma.monarch_attn_last_error()
    assert ma.monarch_attn_last_error() != ""


def test_calls_with_nothing_to_compute():
    nothing = dict.fromkeys(("q", "k", "q_out", "k_out", "freq", "cu", "kv"))
    assert _rotate(**nothing, B=0) == _rotate(**nothing, total=0) == ma.MA_OK
    assert _rotate(**nothing, B=0, clear=1) == INVALID
    more = dict.fromkeys(("q", "k", "v", "q_out", "kp", "vp", "freq", "cu", "kv", "slots"))
    assert _append(**more, B=0) == _append(**more, total=0) == ma.MA_OK
    assert _select(B=0, **dict.fromkeys(("logits", "scores", "done", "out", "tokens", "parents", "done_out"))) == ma.MA_OK
    table = dict.fromkeys(("kp", "vp", "table", "parents", "lens"))
    assert _reorder(**table, B=0) == _reorder(**table, K=1) == _reorder(**table, blocks=0) == ma.MA_OK


def _tensors(**change):
    x = dict(q=torch.zeros(6, 4, 64), k=torch.zeros(6, 2, 64), v=torch.zeros(6, 2, 64), q_out=torch.zeros(6, 4, 64), k_out=torch.zeros(6, 2, 64),
             k_pages=torch.zeros(3, 2, 8, 64), v_pages=torch.zeros(3, 2, 8, 64), inv_freq=torch.zeros(32), cu_seqlens=torch.zeros(3, dtype=torch.int32),
             kv_lens=torch.zeros(2, dtype=torch.int32), slots=torch.zeros(6, dtype=torch.int64))
    x.update(change)
    return {n: t if t is None else _on_device(t)[0] for n, t in x.items()}


@pytest.mark.parametrize("change,error,message", [
    (dict(k=torch.zeros(5, 2, 64)), ValueError, "k must have the rows"), (dict(k=torch.zeros(6, 2, 64, dtype=torch.bfloat16)), ValueError, "k must match q"),
    (dict(q=torch.zeros(6, 256)), ValueError, "q must be a .rows"), (dict(inv_freq=torch.zeros(32, dtype=torch.float64)), ValueError, "inv_freq must be"),
    (dict(inv_freq=torch.zeros(4, 8)), ValueError, "inv_freq must be"), (dict(cu_seqlens=torch.zeros(3)), ValueError, "cu_seqlens must be"),
    (dict(cu_seqlens=torch.zeros(0, dtype=torch.int32)), ValueError, "cu_seqlens must be"), (dict(kv_lens=torch.zeros(3, dtype=torch.int32)), ValueError, "kv_lens must be"),
    (dict(q_out=torch.zeros(6, 64, 4)), ValueError, "q_out must be")])
def test_binding_of_the_rotation(change, error, message):
    x = _tensors(**change)
    with pytest.raises(error, match=message):
        ma.monarch_attn_paged_append(**{n: t for n, t in x.items() if n != "k_out"})
    with pytest.raises(error, match=message):
        ma.monarch_attn_rotate(**{n: x[n] for n in ("q", "k", "q_out", "k_out", "inv_freq", "cu_seqlens", "kv_lens")})


@pytest.mark.parametrize("change,error,message", [
    (dict(k=None), TypeError, "k must be"), (dict(v=torch.zeros(6, 3, 64)), ValueError, "v must match k"), (dict(v=None), TypeError, "v must be a device"),
    (dict(kv_lens=None), TypeError, "kv_lens must be"), (dict(slots=torch.zeros(6, dtype=torch.int32)), ValueError, "slots must be"),
    (dict(k_pages=torch.zeros(3, 1, 8, 64)), ValueError, "k_pages must match k"), (dict(v_pages=torch.zeros(2, 2, 8, 64)), ValueError, "v_pages must be")])
def test_binding_of_the_append(change, error, message):
    with pytest.raises(error, match=message):
        ma.monarch_attn_paged_append(**{n: t for n, t in _tensors(**change).items() if n != "k_out"})


def test_binding_refuses_host_tensors():
    q = torch.zeros(6, 4, 64)
    ints = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError, match="q must be a device tensor"):
        ma.monarch_attn_rotate(q, None, q, None, torch.zeros(32), ints)
    with pytest.raises(TypeError, match="q must be a device tensor"):
        ma.rotate_packed(q, q, torch.zeros(32), ints)
    with pytest.raises(TypeError, match="logits must be a device tensor"):
        ma.monarch_attn_beam_select(torch.zeros(2, 3, 9), torch.zeros(2, 3), q, ints, ints)
    with pytest.raises(TypeError, match="parents must be a device tensor"):
        ma.monarch_attn_paged_reorder(torch.zeros(3, 2, 8, 64), torch.zeros(3, 2, 8, 64), ints.view(3, 1), ints.view(1, 3), ints)


def _selection(**change):
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    x = dict(logits=torch.zeros(2, 3, 9), scores=torch.zeros(2, 3), scores_out=torch.zeros(2, 4), tokens=ints(2, 4), parents=ints(2, 4),
             done=torch.zeros(2, 3, dtype=torch.bool), done_out=torch.zeros(2, 4, dtype=torch.bool))
    x.update(change)
    return {n: t if t is None else _on_device(t)[0] for n, t in x.items()}


@pytest.mark.parametrize("change,message", [
    (dict(logits=torch.zeros(6, 9)), "logits must have 3"), (dict(logits=torch.zeros(2, 9, 3).transpose(1, 2)), "logits must be a .B, K, V. tensor of rows"),
    (dict(logits=torch.zeros(3, 2, 9).transpose(0, 1)), "logits must be a .B, K, V. tensor of rows"), (dict(tokens=torch.zeros(8, dtype=torch.int32)), "tokens must have 2"),
    (dict(tokens=torch.zeros(2, 4, dtype=torch.int64)), "tokens must be"), (dict(scores=torch.zeros(2, 4)), "scores must be"),
    (dict(scores=torch.zeros(2, 3, dtype=torch.float64)), "scores must be"), (dict(scores_out=torch.zeros(2, 3)), "scores_out must be"),
    (dict(parents=torch.zeros(2, 3, dtype=torch.int32)), "parents must be"), (dict(done=torch.zeros(2, 3)), "done must be"),
    (dict(done_out=torch.zeros(2, 3, dtype=torch.bool)), "done_out must be")])
def test_binding_of_the_selection(change, message):
    with pytest.raises(ValueError, match=message):
        ma.monarch_attn_beam_select(**_selection(**change), eos=1)


@pytest.mark.parametrize("eos", [1 << 32, (1 << 32) + 1, -(1 << 32) + 1, 1 << 31, 1 << 64])
def test_eos_beyond_32_bits(eos):
    """No token, also where its lower bits are one."""
    with pytest.raises(ValueError, match="eos must be a token"):
        ma.monarch_attn_beam_select(**_selection(), eos=eos)


@pytest.mark.parametrize("change,message", [
    (dict(parents=torch.zeros(6, dtype=torch.int32)), "parents must have 2"), (dict(parents=torch.zeros(2, 3)), "parents must be"),
    (dict(block_table=torch.zeros(5, 4, dtype=torch.int32)), "block_table must be"), (dict(lens=torch.zeros(2, dtype=torch.int32)), "lens must be"),
    (dict(v_pages=torch.zeros(3, 2, 8, 32)), "v_pages must be"), (dict(k_pages=torch.zeros(3, 8, 64)), "k_pages must have 4")])
def test_binding_of_the_reordering(change, message):
    x = dict(k_pages=torch.zeros(3, 2, 8, 64), v_pages=torch.zeros(3, 2, 8, 64), block_table=torch.zeros(6, 4, dtype=torch.int32),
             parents=torch.zeros(2, 3, dtype=torch.int32), lens=torch.zeros(6, dtype=torch.int32)) | change
    with pytest.raises(ValueError, match=message):
        ma.monarch_attn_paged_reorder(**{n: _on_device(t)[0] for n, t in x.items()})


@pytest.mark.parametrize("call", ["append", "selection", "reordering"])
def test_what_is_no_stream(call):
    """What is wrong with the stream is not said of the tensors."""
    with pytest.raises(AttributeError, match="cuda_stream"):
        if call == "append":
            ma.monarch_attn_paged_append(**{n: t for n, t in _tensors().items() if n != "k_out"}, stream="s")
        elif call == "selection":
            ma.monarch_attn_beam_select(**_selection(), eos=1, stream="s")
        else:
            x = dict(k_pages=torch.zeros(3, 2, 8, 64), v_pages=torch.zeros(3, 2, 8, 64), block_table=torch.zeros(6, 4, dtype=torch.int32),
                     parents=torch.zeros(2, 3, dtype=torch.int32), lens=torch.zeros(6, dtype=torch.int32))
            ma.monarch_attn_paged_reorder(**{n: _on_device(t)[0] for n, t in x.items()}, stream="s")
