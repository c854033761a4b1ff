"""Rotation of queries and keys (monarch_attn_rotate, rotate_packed) and the same on the way into the
paged cache (monarch_attn_paged_append) against 64 bits.

An output is a sum of two products of a value with a sine or cosine, and is rounded once.  With u half a
step of the type and r = |a| + |b| of its pair: u |y| for the rounding, and fp32 inside: two products and
a sum (3 2^-24 r), the sine and cosine (two steps of 2^-24, r each), the fraction of a turn rounded to fp32 (2^-25 of half
a turn, pi 2^-25 r) and formed in 64 bits (t f 2^-52 r).  8 2^-24 r + t f 2^-52 r covers them."""
import math

import pytest
import torch

from sequence_reference import DTYPES, starts, worst

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def _freq(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def _reference(x, pos, freq, interleaved, sign=1.0):
    """(value, bound) of x [n, H, d] turned at positions pos [n], pair by pair as complex numbers in 64 bits."""
    u, n = torch.finfo(x.dtype).eps / 2, freq.shape[0]
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    angle = pos.double()[:, None, None] * freq.double()
    turn = torch.polar(torch.ones_like(angle), sign * angle)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    r = (y[..., a].abs() + y[..., b].abs()) * (8 * 2.0 ** -24 + angle.abs() * 2.0 ** -52)
    z = torch.complex(y[..., a], y[..., b]) * turn
    y[..., a], y[..., b], size[..., a], size[..., b] = z.real, z.imag, r, r
    size[..., : 2 * n] += u * y[..., : 2 * n].abs() + torch.finfo(x.dtype).smallest_normal * u
    return y, size


def _joint(gen, total, heads, d, dt):
    x = torch.randn(total, sum(heads) * d, generator=gen, device="cuda").to(dt)
    return [t.unflatten(1, (-1, d)) for t in x.split([h * d for h in heads], 1)]


SHAPES = [
    # lengths, Hq, Hk, d, rot
    ([1], 1, 1, 8, 8),
    ([3, 0, 70], 4, 2, 64, 64),
    ([1] * 130, 8, 2, 128, 128),
    ([200, 1, 5], 3, 1, 72, 72),
    ([65], 5, 5, 40, 8),
    ([33, 2], 2, 1, 96, 48),
    ([600, 700], 1, 1, 128, 24),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens,Hq,Hk,d,rot", SHAPES)
def test_rotate(ma, lens, Hq, Hk, d, rot, dtype, interleaved):
    print(lens, Hq, Hk, d, rot, dtype, interleaved, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    first, spare = 2, 3
    q, k = _joint(gen, first + sum(lens) + spare, (Hq, Hk), d, DTYPES[dtype])
    cu, freq = starts(lens, "cuda", first), _freq(rot)
    past = torch.arange(len(lens), device="cuda", dtype=torch.int32) * 37
    kv = past + cu[1:] - cu[:-1]
    for kv_lens, inverse, clear in ((None, False, False), (kv, True, True)):
        out = [torch.full(t.shape, 7.0, device="cuda", dtype=t.dtype) for t in (q, k)]
        got = ma.monarch_attn_rotate(q, k, *out, freq, cu, kv_lens, interleaved=interleaved, inverse=inverse, clear=clear)
        torch.cuda.synchronize()
        assert got[0] is out[0] and got[1] is out[1]
        pos = torch.cat([torch.arange(n, device="cuda") + (0 if kv_lens is None else int(past[i])) for i, n in enumerate(lens)])
        for x, y in zip((q, k), out):
            rows = slice(first, first + sum(lens))
            assert worst(y[rows], *_reference(x[rows], pos, freq, interleaved, -1.0 if inverse else 1.0)) <= 1.0
            outside = 0 if clear else 7
            assert bool((y[:first] == outside).all()) and bool((y[first + sum(lens):] == outside).all())
            assert torch.equal(y[rows, :, rot:], x[rows, :, rot:])


def test_without_keys(ma):
    gen = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(9, 3, 64, generator=gen, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    assert ma.monarch_attn_rotate(q, None, out, None, _freq(64), starts([9], "cuda"))[1] is None
    assert worst(out, *_reference(q, torch.arange(9, device="cuda"), _freq(64), False)) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(ma, dtype):
    """Positions up to the last 31-bit one, frequencies of a radian a token and more; and before the first token."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    ends = [1, 5, 70000, 1 << 20, (1 << 30) + 12345, (1 << 31) - 1]
    lens = [4] * len(ends)
    q, k = _joint(gen, sum(lens), (2, 1), 64, DTYPES[dtype])
    freq = torch.cat((_freq(48), torch.tensor([1.0, 3.1415927, 100.0, 0.0, -1.0, 1e-30, 2.5, 0.1], device="cuda")))
    cu, kv = starts(lens, "cuda"), torch.tensor(ends, dtype=torch.int32, device="cuda")
    out = [torch.zeros(t.shape, device="cuda", dtype=t.dtype) for t in (q, k)]
    ma.monarch_attn_rotate(q, k, *out, freq, cu, kv)
    pos = (kv.long()[:, None] - 4 + torch.arange(4, device="cuda")).flatten()
    assert int(pos.min()) == -3
    for x, y in zip((q, k), out):
        assert worst(y, *_reference(x, pos, freq, False)) <= 1.0


def test_values_that_are_not_finite_stay_in_their_pair(ma):
    q = torch.randn(70, 2, 64, device="cuda")
    clean = torch.zeros_like(q)
    freq, cu = _freq(32), starts([70], "cuda")
    ma.monarch_attn_rotate(q, None, clean, None, freq, cu)
    bad = q.clone()
    bad[33, 1, 5], bad[40, 0, 60] = math.nan, math.inf
    out = torch.zeros_like(q)
    ma.monarch_attn_rotate(bad, None, out, None, freq, cu)
    assert bool(torch.isnan(out[33, 1, [5, 21]]).all()) and float(out[40, 0, 60]) == math.inf
    out[33, 1, [5, 21]], out[40, 0, 60] = clean[33, 1, [5, 21]], clean[40, 0, 60]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_autograd(ma, dtype, interleaved):
    """Output and gradient of the differentiable op, on parts of a projection and on transposed views."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    lens, first = [50, 0, 31], 2
    joint = torch.randn(first + 81 + 4, 6 * 64, generator=gen, device="cuda").to(DTYPES[dtype]).requires_grad_()
    cu, freq = starts(lens, "cuda", first), _freq(48)
    q, k = (t.unflatten(1, (-1, 64)) for t in joint.split((256, 128), 1))
    grads = [torch.randn(t.shape, generator=gen, device="cuda").to(t.dtype) for t in (q, k)]
    out = ma.rotate_packed(q, k, freq, cu, interleaved=interleaved)
    (g,) = torch.autograd.grad(out, joint, grads)
    back = [t.unflatten(1, (-1, 64)) for t in g.split((256, 128), 1)]
    pos = torch.cat([torch.arange(n, device="cuda") for n in lens])
    rows = slice(first, first + 81)
    for x, y, sign in ((q, out[0], 1), (k, out[1], 1), (grads[0], back[0], -1), (grads[1], back[1], -1)):
        assert worst(y[rows].detach(), *_reference(x[rows].detach(), pos, freq, interleaved, float(sign))) <= 1.0
        assert bool((y[:first] == 0).all()) and bool((y[first + 81:] == 0).all())
    views = [t.detach().transpose(0, 1).contiguous().transpose(0, 1).requires_grad_() for t in (q, k)]
    again = ma.rotate_packed(*views, freq, cu, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(again, out))
    (only,) = torch.autograd.grad(again[0], views[:1], grads[0].transpose(0, 1).contiguous().transpose(0, 1))  # k's part unused
    assert torch.equal(only, back[0])


def test_gradient_against_differences(ma):
    """The op is linear: central differences of any step give the gradient but for rounding, 2^-20 of the sizes."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k = (torch.randn(40, h, 32, generator=gen, device="cuda", requires_grad=True) for h in (2, 1))
    cu, freq = starts([25, 15], "cuda"), _freq(32)
    g = [torch.randn(t.shape, generator=gen, device="cuda") for t in (q, k)]
    grads = torch.autograd.grad(ma.rotate_packed(q, k, freq, cu), (q, k), g)
    f = lambda q, k: sum(float((y.double() * w.double()).sum()) for y, w in zip(ma.rotate_packed(q, k, freq, cu), g))  # noqa: E731
    for i, t in enumerate((q, k)):
        step = torch.randn(t.shape, generator=gen, device="cuda")
        up, down = ([x.detach() + s * step if j == i else x.detach() for j, x in enumerate((q, k))] for s in (1, -1))
        want = float((grads[i].double() * step.double()).sum())
        size = float((grads[i].double().abs() * step.double().abs()).sum()) + float(sum(t.abs().sum() for t in g))
        assert abs((f(*up) - f(*down)) / 2 - want) <= 2.0 ** -20 * size


def _cache(gen, lens, past, Hkv, d, page, dt):
    """Pages (random values), slots of the new rows and what maps them."""
    have = [-(-(p + n) // page) for p, n in zip(past, lens)]
    ids = torch.randperm(sum(have) + 3, generator=gen, device="cuda").tolist()
    slots, at = [], 0
    for p, n, h in zip(past, lens, have):
        slots += [ids[at + t // page] * page + t % page for t in range(p, p + n)]
        at += h
    pages = [torch.randn(len(ids), Hkv, page, d, generator=gen, device="cuda").to(dt) for _ in range(2)]
    return pages, slots


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens,past,Hq,Hkv,d,rot,page", [
    ([1], [0], 1, 1, 8, 8, 8), ([1] * 70, list(range(70)), 4, 2, 64, 64, 16), ([5, 0, 40, 1], [7, 9, 0, 100], 8, 2, 128, 96, 32),
    ([33, 300], [3, 2], 3, 3, 72, 24, 64), ([700, 900], [0, 1], 2, 1, 32, 32, 8)])
def test_append(ma, lens, past, Hq, Hkv, d, rot, page, dtype, interleaved):
    print(lens[:4], past[:4], Hq, Hkv, d, rot, page, dtype, interleaved, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(6)
    first, spare, n = 0, 5, sum(lens)
    dt = DTYPES[dtype]
    q, k, v = _joint(gen, n + spare, (Hq, Hkv, Hkv), d, dt)
    pages, slots = _cache(gen, lens, past, Hkv, d, page, dt)
    old = [t.clone() for t in pages]
    slots += [-1] * spare
    dropped = n // 2
    slots[dropped] = -1 if n % 2 else pages[0].shape[0] * page  # no slot, or one outside the cache
    cu, freq = starts(lens, "cuda"), _freq(rot)
    kv = torch.tensor([p + m for p, m in zip(past, lens)], dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, 7.0, device="cuda", dtype=dt)
    ma.monarch_attn_paged_append(q, k, v, out, *pages, freq, cu, kv, torch.tensor(slots, device="cuda"), interleaved=interleaved)
    torch.cuda.synchronize()
    pos = torch.cat([torch.arange(p, p + m, device="cuda") for p, m in zip(past, lens)])
    assert worst(out[:n], *_reference(q[:n], pos, freq, interleaved)) <= 1.0 and bool((out[n:] == 7).all())
    keep = [i for i in range(n) if i != dropped]
    at = torch.tensor([slots[i] for i in keep], dtype=torch.int64, device="cuda")
    flat = [t.transpose(1, 2).flatten(0, 1) for t in pages]
    if keep:
        assert worst(flat[0][at], *[t[keep] for t in _reference(k[:n], pos, freq, interleaved)]) <= 1.0
        assert torch.equal(flat[1][at], v[keep])
    rest = torch.ones(flat[0].shape[0], dtype=torch.bool, device="cuda")
    rest[at] = False
    for t, o in zip(flat, old):
        assert torch.equal(t[rest], o.transpose(1, 2).flatten(0, 1)[rest])


def test_append_is_rotate_and_write(ma):
    gen = torch.Generator(device="cuda").manual_seed(7)
    lens, past, page = [3, 90, 1], [5, 0, 64], 16
    q, k, v = _joint(gen, 94, (4, 2, 2), 64, torch.bfloat16)
    pages, slots = _cache(gen, lens, past, 2, 64, page, torch.bfloat16)
    other = [t.clone() for t in pages]
    slots = torch.tensor(slots, device="cuda")
    cu, freq, kv = starts(lens, "cuda"), _freq(64), torch.tensor([8, 90, 65], dtype=torch.int32, device="cuda")
    out, q_out, k_out = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k)
    ma.monarch_attn_paged_append(q, k, v, out, *pages, freq, cu, kv, slots)
    ma.monarch_attn_rotate(q, k, q_out, k_out, freq, cu, kv)
    ma.monarch_attn_paged_write(k_out, v, *other, slots)
    assert torch.equal(out, q_out) and all(torch.equal(a, b) for a, b in zip(pages, other))


def test_many_sequences(ma):
    """More sequences than one step of the search takes, empty ones among them, and none."""
    gen = torch.Generator().manual_seed(8)
    lens = torch.randint(0, 3, (5000,), generator=gen).tolist()
    q = torch.randn(sum(lens) + 4, 1, 8, device="cuda")
    out = torch.zeros_like(q)
    freq, cu = torch.ones(4, device="cuda"), starts(lens, "cuda")
    ma.monarch_attn_rotate(q, None, out, None, freq, cu)
    pos = torch.cat([torch.arange(n) for n in lens]).cuda()
    n = sum(lens)
    assert worst(out[:n], *_reference(q[:n], pos, freq, False)) <= 1.0 and bool((out[n:] == 0).all())
    out.fill_(7.0)
    ma.monarch_attn_rotate(q, None, out, None, freq, starts([], "cuda"))
    assert bool((out == 7).all())
    ma.monarch_attn_rotate(q, None, out, None, freq, starts([], "cuda"), clear=True)
    assert bool((out == 0).all())


def test_captured(ma):
    """A rotation with its gradient, and an append, in a graph: replayed with other positions and values."""
    s = torch.cuda.Stream()
    gen = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = (t.contiguous() for t in _joint(gen, 6, (4, 2, 2), 64, torch.bfloat16))
    leaves = [q.clone().requires_grad_(), k.clone().requires_grad_()]
    cu, freq, kv = starts([1] * 6, "cuda"), _freq(64), torch.arange(6, dtype=torch.int32, device="cuda") + 20
    pages = [torch.zeros(8, 2, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    slots, out = torch.arange(6, device="cuda") * 17, torch.zeros_like(q)

    def step(leaves, out, pages):
        ma.monarch_attn_paged_append(q, k, v, out, *pages, freq, cu, kv, slots)
        y = ma.rotate_packed(*leaves, freq, cu)
        return (*y, *torch.autograd.grad(y, leaves, (q, k)))

    with torch.cuda.stream(s):
        step(leaves, out, pages)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        captured = step(leaves, out, pages)
    for i in range(3):
        with torch.no_grad():
            kv.add_(1000)
            slots.add_(1)
            q.mul_(-1.5)
            leaves[0].mul_(0.5)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        other = [t.clone().zero_() if i == 0 else t for t in pages] if i == 0 else other
        fresh = torch.zeros_like(out)
        want = step([t.detach().clone().requires_grad_() for t in leaves], fresh, other)
        torch.cuda.synchronize()
        assert torch.equal(out, fresh) and all(torch.equal(a, b) for a, b in zip(captured, want))
        for a, b in zip(pages, other):
            at = slots
            assert torch.equal(a.transpose(1, 2).flatten(0, 1)[at], b.transpose(1, 2).flatten(0, 1)[at])
