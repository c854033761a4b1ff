"""Exact attention over packed sequences (monarch_attn_exact_packed_fwd, _bwd,
exact_attention_packed) against 64 bits, element by element within the bounds of
sequence_reference.py."""
import math

import pytest
import torch

from sequence_reference import DTYPES, attention, starts, worst

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def _inputs(lens, Hq, Hkv, d, dtype, seed, spare=3, first=2, scale=1.0):
    """q, k, v as parts of one tensor, dout and the row starts; `first` rows before the sequences, `spare` behind."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    total = first + sum(lens) + spare
    joint = torch.randn(total, (Hq + 2 * Hkv) * d, generator=gen, device="cuda")
    joint[:, : (Hq + Hkv) * d] *= scale
    q, k, v = (x.unflatten(1, (-1, d)) for x in joint.to(DTYPES[dtype]).split((Hq * d, Hkv * d, Hkv * d), 1))
    dout = torch.randn(total, Hq, d, generator=gen, device="cuda").to(DTYPES[dtype])
    return q, k, v, dout, starts(lens, "cuda", first)


def _run(ma, q, k, v, dout, cu, causal, rest=True):
    """All results, in tensors that held 7 before."""
    total, Hq, d = q.shape
    like = lambda h: torch.full((total, h, d), 7.0, device="cuda", dtype=q.dtype)  # noqa: E731
    r = {"out": like(Hq), "lse": torch.full((Hq, total), 7.0, device="cuda")}
    more = like(Hq) if rest and q.dtype != torch.float32 else None
    ma.monarch_attn_exact_packed_fwd(q, k, v, r["out"], cu, causal, r["lse"], more)
    if dout is not None:
        r |= {"dq": like(Hq), "dk": like(k.shape[1]), "dv": like(k.shape[1])}
        ma.monarch_attn_exact_packed_bwd(q, k, v, r["out"], r["lse"], dout, r["dq"], r["dk"], r["dv"], cu, causal, more)
    torch.cuda.synchronize()
    return r


def _check(r, q, k, v, dout, cu, causal):
    at = cu.tolist()
    rows = lambda x, name: x.transpose(0, 1) if name == "lse" else x  # noqa: E731
    for name, x in r.items():
        assert bool((rows(x, name)[: at[0]] == 7).all()) and bool((rows(x, name)[at[-1]:] == 7).all()), f"{name}: rows of no sequence"
    for a, z in zip(at[:-1], at[1:]):
        if a == z:
            continue
        ref = attention(q[a:z], k[a:z], v[a:z], causal, 0, None if dout is None else dout[a:z])
        for name, (want, bound) in ref.items():
            if name in r:
                got = r[name][:, a:z] if name == "lse" else r[name][a:z]
                off = worst(got, want, bound)
                assert off <= 1.0, f"{name} of rows {a}..{z}: {off:.3g} of what rounding allows"


SHAPES = [
    # lengths, Hq, Hkv, d
    ([1], 1, 1, 8),
    ([5, 0, 1, 64], 2, 2, 64),
    ([127, 128, 129], 3, 1, 64),
    ([300, 0, 0, 33, 2], 4, 2, 128),
    ([63, 65, 200], 5, 1, 40),
    ([31, 32, 33, 1], 12, 3, 96),
    ([257], 8, 8, 72),
    ([700], 2, 1, 128),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens,Hq,Hkv,d", SHAPES)
def test_forward_and_gradient(ma, lens, Hq, Hkv, d, dtype, causal):
    print(lens, Hq, Hkv, d, dtype, causal, flush=True)
    x = _inputs(lens, Hq, Hkv, d, dtype, 1)
    _check(_run(ma, *x, causal), *x, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_rest(ma, dtype):
    """The gradient from out and lse alone."""
    x = _inputs([200, 17, 3], 4, 2, 64, dtype, 2)
    _check(_run(ma, *x, True, rest=False), *x, True)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_long_sequence(ma, dtype):
    x = _inputs([3001, 100], 4, 1, 64, dtype, 3)
    _check(_run(ma, *x, True), *x, True)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_large_scores(ma, dtype):
    """Scores of several hundred: weights of one key, rescaled many times as the maximum grows."""
    q, k, v, dout, cu = _inputs([400], 2, 2, 64, dtype, 4, scale=6.0)
    _check(_run(ma, q, k, v, None, cu, True), q, k, v, None, cu, True)


def test_many_sequences(ma):
    """More sequences than one step of the search takes (64), and than two (4096), most of them short or empty."""
    gen = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 4, (5000,), generator=gen).tolist()
    lens[17], lens[4700] = 300, 200
    x = _inputs(lens, 2, 1, 32, "bf16", 5)
    r = _run(ma, *x, True)
    at = x[4].tolist()
    for i in [0, 16, 17, 18, 63, 64, 65, 2500, 4095, 4096, 4700, 4999]:
        a, z = at[i], at[i + 1]
        if a == z:
            continue
        for name, (want, bound) in attention(*(t[a:z] for t in x[:3]), True, 0, x[3][a:z]).items():
            assert worst(r[name][:, a:z] if name == "lse" else r[name][a:z], want, bound) <= 1.0, (i, name)
    assert all(bool(torch.isfinite(t).all()) for t in r.values())
    single = [a for a, z in zip(at[:-1], at[1:]) if z == a + 1]  # one key: its value, and no gradient to q and k
    assert bool((r["out"][single] == x[2][single].expand(-1, 2, -1)).all())
    assert bool((r["dq"][single] == 0).all()) and bool((r["dk"][single] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_keys_that_are_not_seen_have_no_effect(ma, bad, dtype):
    """Values and keys that are not finite reach the rows that see them, no earlier row and no other sequence."""
    q, k, v, _, cu = _inputs([150, 90, 40], 4, 2, 64, dtype, 6, first=0)
    clean = _run(ma, q, k, v, None, cu, True)
    at = 150 + 37
    for which in (k, v):
        keep = which[at].clone()
        which[at, 1] = bad
        r = _run(ma, q, k, v, None, cu, True)
        hit = slice(at, 240)
        for h in range(4):
            rows = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
            if h >= 2:
                rows[hit] = False
                o = r["out"][hit, h].float()
                if which is v:  # every weight is positive here
                    assert bool(torch.isnan(o).all()) if math.isnan(bad) else bool((o == bad).all())
            assert torch.equal(r["out"][rows, h], clean["out"][rows, h])
        which[at] = keep


def test_both_infinities_in_a_column(ma):
    q, k, v, _, cu = _inputs([64], 1, 1, 64, "bf16", 7, first=0)
    v[10, 0, 3], v[20, 0, 3], v[20, 0, 4] = math.inf, -math.inf, -math.inf
    o = _run(ma, q, k, v, None, cu, True)["out"][:64, 0].float()
    assert bool(torch.isfinite(o[:10]).all()) and bool((o[10:20, 3] == math.inf).all()) and bool(torch.isnan(o[20:, 3]).all())
    assert bool(torch.isfinite(o[:20, 4]).all()) and bool((o[20:, 4] == -math.inf).all())
    assert bool(torch.isfinite(o[:, :3]).all()) and bool(torch.isfinite(o[:, 5:]).all())


def test_gradient_of_other_sequences_stays_finite(ma):
    q, k, v, dout, cu = _inputs([70, 200, 40], 2, 1, 64, "bf16", 8, first=0)
    clean = _run(ma, q, k, v, dout, cu, True)
    for t in (q, k, v, dout):
        t[70:270] = math.nan
    r = _run(ma, q, k, v, dout, cu, True)
    for name in ("dq", "dk", "dv", "out"):
        for rows in (slice(0, 70), slice(270, 310)):
            assert torch.equal(r[name][rows], clean[name][rows]), name


@pytest.mark.parametrize("scale", [1e-6, 1.0, 3e3])
def test_fp16_gradients_of_any_scale(ma, scale):
    """dS of fp16 is formed relative to the largest norms: an upstream gradient times 2^k gives gradients times 2^k
    to the same relative accuracy, as long as they are normal numbers."""
    k2 = 2.0 ** round(math.log2(scale))
    q, k, v, dout, cu = _inputs([500, 40], 2, 1, 64, "f16", 9)
    dout = dout * 2.0 ** -6  # of sizes that both scalings hold
    v.copy_((v.float() / k2).clamp(-6e4, 6e4).half())  # dP keeps its size in fp32 whatever the scale
    x = (q, k, v, (dout.float() * min(k2, 1.0)).half())
    _check(_run(ma, *x, cu, True), *x, cu, True)


def test_same_bits_again(ma):
    x = _inputs([777, 130], 4, 2, 128, "bf16", 10)
    a, b = _run(ma, *x, True), _run(ma, *x, True)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("causal", [True, False])
def test_gradient_against_differences(ma, causal):
    """<grad, direction> against central differences of the kernel's own fp32 forward.  The difference of step h has
    an error of h^2 from the third derivative and 2^-24 |f| / h from rounding: 1e-3 relative covers both at h = 2^-7."""
    q, k, v, dout, cu = _inputs([60, 9], 2, 1, 32, "f32", 11, spare=0, first=0)
    q, k, v = (t.contiguous() for t in (q, k, v))
    r = _run(ma, q, k, v, dout, cu, causal)
    f = lambda *t: float((_run(ma, *t, None, cu, causal)["out"].double() * dout.double()).sum())  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(12)
    for i, name in enumerate(("dq", "dk", "dv")):
        step = torch.randn((q, k, v)[i].shape, generator=gen, device="cuda")
        want = float((r[name].double() * step.double()).sum())
        up, down = ([t + sign * 2.0 ** -7 * step if j == i else t for j, t in enumerate((q, k, v))] for sign in (1, -1))
        got = (f(*up) - f(*down)) * 2.0 ** 6
        size = float((r[name].double().abs() * step.double().abs()).sum())
        assert abs(got - want) <= 1e-3 * size, (name, got, want, size)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_autograd(ma, dtype):
    """The differentiable op on parts of a joint projection and on a transposed view; rows of no sequence are zero."""
    q, k, v, dout, cu = _inputs([90, 0, 61], 4, 2, 64, dtype, 13)
    joint = torch.cat([t.flatten(1) for t in (q, k, v)], 1).requires_grad_()
    parts = [t.unflatten(1, (-1, 64)) for t in joint.split((256, 128, 128), 1)]
    out = ma.exact_attention_packed(*parts, cu, causal=True)
    (grad,) = torch.autograd.grad(out, joint, dout)
    got = dict(zip(("dq", "dk", "dv"), (t.unflatten(1, (-1, 64)) for t in grad.split((256, 128, 128), 1))), out=out.detach())
    for rows in (slice(0, 2), slice(153, 156)):
        assert all(bool((t[rows] == 0).all()) for t in got.values())
    for a, z in ((2, 92), (92, 153)):
        for name, (want, bound) in attention(*(t[a:z] for t in (q, k, v)), True, 0, dout[a:z]).items():
            if name != "lse":
                assert worst(got[name][a:z], want, bound) <= 1.0, name
    heads_first = [t.detach().transpose(0, 1).contiguous().transpose(0, 1).requires_grad_() for t in parts]
    again = ma.exact_attention_packed(*heads_first, cu)
    assert torch.equal(again, out)
    for x, name in zip(torch.autograd.grad(again, heads_first, dout.transpose(0, 1).contiguous().transpose(0, 1)), ("dq", "dk", "dv")):
        assert torch.equal(x, got[name])


def test_clear(ma):
    """Rows of no sequence are written as zero on request, without a sequence all rows."""
    q, k, v, dout, cu = _inputs([40, 0, 9], 4, 2, 64, "bf16", 21, spare=700, first=300)
    for at in (cu, cu[3:].contiguous()):
        out, lse = torch.full_like(dout, 7.0), torch.zeros(4, dout.shape[0], device="cuda")
        grads = [torch.full(t.shape, 7.0, device="cuda", dtype=t.dtype) for t in (q, k, v)]
        ma.monarch_attn_exact_packed_fwd(q, k, v, out, at, True, lse, clear=True)
        ma.monarch_attn_exact_packed_bwd(q, k, v, out, lse, dout, *grads, at, True, clear=True)
        torch.cuda.synchronize()
        real = torch.zeros(dout.shape[0], dtype=torch.bool, device="cuda")
        real[300:349] = at is cu
        assert all(bool((t[~real] == 0).all()) and bool((t[real] != 0).any() == (at is cu)) for t in (out, *grads))


def test_empty_calls(ma):
    for lens, rows in (([], 0), ([], 5), ([0, 0, 0], 5)):
        q = torch.randn(rows, 4, 64, device="cuda").bfloat16()
        cu = starts(lens, "cuda")
        out = torch.full_like(q, 7.0)
        ma.monarch_attn_exact_packed_fwd(q, q, q, out, cu)
        grads = [torch.full_like(q, 7.0) for _ in range(3)]
        lse = torch.zeros(4, rows, device="cuda")
        ma.monarch_attn_exact_packed_bwd(q, q, q, out, lse, out.clone(), *grads, cu)
        torch.cuda.synchronize()
        assert all(bool((t == 7).all()) for t in (out, *grads))


def test_row_starts_out_of_range(ma):
    """Row starts are clamped to the tensor: whatever they hold, nothing outside is read or written."""
    q, k, v, _, _ = _inputs([100], 2, 1, 64, "bf16", 14, spare=0, first=0)
    for at in ([0, 60, 1 << 30], [-5, 60, 100], [0, 100, 40, 100]):
        cu = torch.tensor(at, device="cuda", dtype=torch.int32)
        out = torch.full((300, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16)
        ma.monarch_attn_exact_packed_fwd(q, k, v, out[100:200], cu)
        torch.cuda.synchronize()
        assert bool((out[:100] == 7).all()) and bool((out[200:] == 7).all())
        ref = attention(q[:60], k[:60], v[:60], True)["out"]
        if at[1] == 60:
            assert worst(out[100:160], *ref) <= 1.0


def test_offsets_past_32_bits(ma):
    """Rows so far apart that their offsets pass 2^31 elements."""
    ld, rows = 1 << 20, 2300
    buf = torch.empty(rows, ld, device="cuda", dtype=torch.bfloat16)  # 4.8 GB
    q, k, v = (buf[:, i * 128 : (i + 1) * 128].unflatten(1, (2, 64)) for i in range(3))
    dense = _inputs([2300], 2, 2, 64, "bf16", 15, spare=0, first=0)
    for x, y in zip((q, k, v), dense):
        x.copy_(y)
    far, near = _run(ma, q, k, v, dense[3], dense[4], True), _run(ma, *dense, True)
    assert all(torch.equal(far[n], near[n]) for n in far)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_captured_forward_and_gradient(ma, dtype):
    """Captured calls replayed with other inputs between, each replay equal to eager calls on another stream."""
    x = _inputs([200, 77], 4, 2, 64, dtype, 16)
    q, k, v, dout, cu = x
    eager = _run(ma, *x, True)
    s = torch.cuda.Stream()
    r = {n: torch.empty_like(t) for n, t in eager.items()}
    rest = torch.empty_like(q)

    def calls():
        ma.monarch_attn_exact_packed_fwd(q, k, v, r["out"], cu, True, r["lse"], rest)
        ma.monarch_attn_exact_packed_bwd(q, k, v, r["out"], r["lse"], dout, r["dq"], r["dk"], r["dv"], cu, True, rest)

    with torch.cuda.stream(s):
        calls()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls()
    for i in range(4):
        y = _inputs([200, 77], 4, 2, 64, dtype, 17 + i)
        for dst, src in zip(x[:4], y[:4]):
            dst.copy_(src)
        cu.copy_(starts([120 + i, 50], "cuda", 2))
        for t in r.values():
            t.fill_(7.0)
        want = _run(ma, *x, True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in r.items():
            assert torch.equal(t, want[n]), (i, n)


def test_two_streams_at_once(ma):
    x, y = _inputs([900], 4, 2, 64, "bf16", 18), _inputs([300, 400], 4, 2, 64, "bf16", 19)
    want = [_run(ma, *x, True), _run(ma, *y, True)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [{n: torch.full_like(t, 7.0) for n, t in w.items()} for w in want]
    rests = [torch.empty_like(t[0].contiguous()) for t in (x, y)]
    torch.cuda.synchronize()
    for _ in range(5):
        for z, r, rest, s in zip((x, y), got, rests, streams):
            q, k, v, dout, cu = z
            ma.monarch_attn_exact_packed_fwd(q, k, v, r["out"], cu, True, r["lse"], rest, stream=s)
            ma.monarch_attn_exact_packed_bwd(q, k, v, r["out"], r["lse"], dout, r["dq"], r["dk"], r["dv"], cu, True, rest, stream=s)
    torch.cuda.synchronize()
    for w, r in zip(want, got):
        assert all(torch.equal(w[n], r[n]) for n in w)


def test_autograd_of_other_layouts(ma):
    """Leaves and upstream gradients that are not as the kernels need them: off 16 bytes, expanded, heads not adjacent."""
    lens, Hq, Hkv, d = [70, 3], 4, 2, 64
    q, k, v, dout, cu = _inputs(lens, Hq, Hkv, d, "bf16", 41, spare=0, first=0)
    want = _run(ma, q, k, v, dout, cu, True)

    def odd(t):  # contiguous, 2 bytes behind an aligned address
        flat = torch.empty(t.numel() + 1, device="cuda", dtype=t.dtype)[1:].view(t.shape)
        return flat.copy_(t)

    leaves = [odd(q).requires_grad_(), k.transpose(0, 1).contiguous().transpose(0, 1).requires_grad_(), odd(v).requires_grad_()]
    out = ma.exact_attention_packed(*leaves, cu)
    assert torch.equal(out, want["out"])
    for g, n in zip(torch.autograd.grad(out, leaves, odd(dout), retain_graph=True), ("dq", "dk", "dv")):
        assert torch.equal(g, want[n]), n
    ones = torch.autograd.grad(out.sum(), leaves, retain_graph=True)  # an upstream gradient with strides of zero
    for g, h in zip(ones, torch.autograd.grad(out, leaves, torch.ones_like(out))):
        assert torch.equal(g, h)


def test_gradient_of_the_gradient_is_refused(ma):
    q, k, v, _, cu = _inputs([20], 2, 2, 64, "f32", 42, spare=0, first=0)
    q = q.detach().requires_grad_()
    (g,) = torch.autograd.grad(ma.exact_attention_packed(q, k, v, cu).square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), q)


def test_captured_autograd(ma):
    """Forward and backward of the torch op in one graph, replayed with other inputs, against eager passes."""
    x = _inputs([130, 66], 4, 2, 64, "bf16", 43, spare=0, first=0)
    leaves, dout, cu = [t.detach().clone().requires_grad_() for t in x[:3]], x[3], x[4]
    s = torch.cuda.Stream()

    def once():
        out = ma.exact_attention_packed(*leaves, cu)
        return (out.detach(), *torch.autograd.grad(out, leaves, dout))

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        once()  # (its autograd graph is gone before the capture)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = once()
    for i in range(4):
        y = _inputs([130, 66], 4, 2, 64, "bf16", 44 + i, spare=0, first=0)
        with torch.no_grad():
            for dst, src in zip(leaves, y[:3]):
                dst.copy_(src)
        dout.copy_(y[3])
        want = _run(ma, *y, True)
        graph.replay()
        torch.cuda.synchronize()
        for t, n in zip(got, ("out", "dq", "dk", "dv")):
            assert torch.equal(t, want[n]), (i, n)


def test_decreasing_row_starts(ma):
    """Sequences whose ranges overlap: nothing outside the tensors is read or written, in the gradient too."""
    q, k, v, dout, _ = _inputs([300], 4, 2, 64, "bf16", 45, spare=0, first=0)
    cu = torch.tensor([0, 300, 0, 300, 0, 300, 100, 250], device="cuda", dtype=torch.int32)
    around = {n: torch.full((900, h, 64), 7.0, device="cuda", dtype=torch.bfloat16) for n, h in (("out", 4), ("dq", 4), ("dk", 2), ("dv", 2))}
    mid = {n: t[300:600] for n, t in around.items()}
    lse = torch.zeros(4, 300, device="cuda")
    ma.monarch_attn_exact_packed_fwd(q, k, v, mid["out"], cu, True, lse)
    ma.monarch_attn_exact_packed_bwd(q, k, v, mid["out"], lse, dout, mid["dq"], mid["dk"], mid["dv"], cu)
    torch.cuda.synchronize()
    for t in around.values():
        assert bool((t[:300] == 7).all()) and bool((t[600:] == 7).all())
