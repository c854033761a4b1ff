"""Cross attention (monarch_attn_exact_cross_fwd, _bwd, exact_cross_attention) against 64 bits,
element by element within the bounds of sequence_reference.py."""
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


class Case:
    """q, k, v (k and v parts of one tensor), dout and row starts; `first` rows before the sequences, `spare` behind.
    width: the keys lie in a padded batch of so many rows each."""

    def __init__(self, lens, keys, Hq, Hkv, d, dtype, seed, first=2, spare=3, width=None, scale=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dt = DTYPES[dtype]
        self.lens, self.keys = lens, keys
        self.cu = starts(lens, "cuda", first)
        self.cu_k = starts([width] * len(keys) if width else keys, "cuda", first)
        self.k_lens = torch.tensor(keys, dtype=torch.int32, device="cuda") if width else None
        total, total_k = (int(c[-1]) + spare for c in (self.cu, self.cu_k))
        self.q = (torch.randn(total, Hq, d, generator=gen, device="cuda") * scale).to(dt)
        joint = torch.randn(total_k, 2 * Hkv * d, generator=gen, device="cuda")
        joint[:, : Hkv * d] *= scale
        self.k, self.v = (x.unflatten(1, (Hkv, d)) for x in joint.to(dt).split(Hkv * d, 1))
        self.dout = torch.randn(total, Hq, d, generator=gen, device="cuda").to(dt)

    def run(self, ma, grads=True, rest=True, clear=False):
        """All results, in tensors that held 7 before."""
        q, k, v = self.q, self.k, self.v
        full = lambda t: torch.full(t.shape, 7.0, device="cuda", dtype=t.dtype)  # noqa: E731
        r = {"out": full(q), "lse": torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")}
        more = full(q) if rest and q.dtype != torch.float32 else None
        ma.monarch_attn_exact_cross_fwd(q, k, v, r["out"], self.cu, self.cu_k, self.k_lens, r["lse"], more, clear)
        if grads:
            r |= {"dq": full(q), "dk": full(k), "dv": full(v)}
            ma.monarch_attn_exact_cross_bwd(q, k, v, r["out"], r["lse"], self.dout, r["dq"], r["dk"], r["dv"], self.cu, self.cu_k,
                                            self.k_lens, more, clear)
        torch.cuda.synchronize()
        return r

    def check(self, r, clear=False, only=None):
        at, at_k = self.cu.tolist(), self.cu_k.tolist()
        for name, x in r.items():
            rows = x.transpose(0, 1) if name == "lse" else x
            a, z = (at_k if name in ("dk", "dv") else at)[:: len(at) - 1]
            outside = 0 if clear and name != "lse" else 7
            assert bool((rows[:a] == outside).all()) and bool((rows[z:] == outside).all()), f"{name}: rows of no sequence"
        for i, (n, L) in enumerate(zip(self.lens, self.keys)):
            if only is not None and i not in only:
                continue
            rows, keys = slice(at[i], at[i] + n), slice(at_k[i], at_k[i] + L)
            ref = attention(self.q[rows], self.k[keys], self.v[keys], False, 0, self.dout[rows] if "dq" in r else None)
            for name, (want, bound) in ref.items():
                if name not in r or 0 in want.shape:
                    continue
                got = r[name][:, rows] if name == "lse" else r[name][keys if name in ("dk", "dv") else rows]
                off = worst(got, want, bound)
                assert off <= 1.0, f"{name} of sequence {i}, {n} rows over {L} keys: {off:.3g} of what rounding allows"
            for name in ("dk", "dv"):
                if name in r:
                    assert bool((r[name][at_k[i] + L: at_k[i + 1]] == 0).all()), f"{name}: padding of sequence {i}"


SHAPES = [
    # rows, keys, Hq, Hkv, d
    ([1], [1], 1, 1, 8),
    ([5, 0, 1, 64, 3], [3, 7, 0, 1, 130], 2, 2, 64),
    ([127, 128, 129], [65, 64, 63], 3, 1, 64),
    ([300, 33, 2], [31, 500, 128], 4, 2, 128),
    ([63, 200], [1, 1000], 5, 1, 40),
    ([1, 31, 32, 33], [300, 2, 0, 96], 12, 3, 96),
    ([4, 4, 4], [700, 64, 1], 8, 8, 72),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("lens,keys,Hq,Hkv,d", SHAPES)
def test_forward_and_gradient(ma, lens, keys, Hq, Hkv, d, dtype, padded):
    print(lens, keys, Hq, Hkv, d, dtype, padded, flush=True)
    x = Case(lens, keys, Hq, Hkv, d, dtype, 1, width=max(keys) + 70 if padded else None)
    x.check(x.run(ma))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_rest(ma, dtype):
    x = Case([200, 17, 3], [40, 300, 90], 4, 2, 64, dtype, 2)
    x.check(x.run(ma, rest=False))


# few rows over long keys are split over the keys, and so are many where there are few of them
LONG = [
    ([4], [9000], 2, 2, 64),
    ([4, 4, 1, 0, 8], [3000, 17, 8000, 50, 1], 4, 4, 64),
    ([3, 2], [4097, 5000], 8, 2, 128),
    ([300], [5001], 2, 1, 128),
    ([150, 7], [2500, 4100], 3, 3, 80),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens,keys,Hq,Hkv,d", LONG)
def test_long_keys(ma, lens, keys, Hq, Hkv, d, dtype):
    print(lens, keys, Hq, Hkv, d, dtype, flush=True)
    x = Case(lens, keys, Hq, Hkv, d, dtype, 3)
    x.check(x.run(ma))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(ma, dtype):
    """Scores of several hundred: weights of one key, rescaled many times as the maximum grows."""
    for lens, keys in (([100], [400]), ([4], [6000])):
        x = Case(lens, keys, 2, 2, 64, dtype, 4, scale=6.0)
        x.check(x.run(ma, grads=False))


def test_weights_of_wide_heads_in_fp32(ma):
    """dK and dV of 16 rows over 700 keys of 128 columns, as a whole: a weight exp(s - lse) carries the roundings of lse (two,
    near 7 and near 10 in log2 units), of its product with sqrt(128) / log2 e (near 80, two) and of the difference (near
    80), of the scale (relative to 7), and of the scores' sums, half a step each at most: root mean squares of 2e-7 to 4e-7 in
    units of the weight, 8e-7 together, 1.2e-6 with half as much again.  (A sum that starts near 80 and rounds there 64 times is
    off by 2e-6.)"""
    x = Case([16], [700], 3, 3, 128, "f32", 31)
    r = x.run(ma)
    q, k, v, g = (t.double().transpose(0, 1) for t in (x.q[2:18], x.k[2:702], x.v[2:702], x.dout[2:18]))
    w = (q @ k.transpose(1, 2).contiguous() / math.sqrt(128)).softmax(-1)
    ds = w * (g @ v.transpose(1, 2).contiguous() - (g * (w @ v)).sum(-1, keepdim=True)) / math.sqrt(128)
    for name, want in (("dk", ds.transpose(1, 2).contiguous() @ q), ("dv", w.transpose(1, 2).contiguous() @ g)):
        off = (r[name][2:702].double().transpose(0, 1) - want).norm() / want.norm()
        assert off <= 1.2e-6, (name, off)


def test_many_sequences(ma):
    """More sequences than one step of the searches takes, most of them short or empty on either side."""
    gen = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 4, (5000,), generator=gen).tolist()
    keys = torch.randint(0, 5, (5000,), generator=gen).tolist()
    lens[17], keys[17], lens[4700], keys[4700], lens[100], keys[100] = 300, 2, 2, 900, 5, 0
    x = Case(lens, keys, 2, 1, 32, "bf16", 5)
    r = x.run(ma)
    x.check(r, only=[0, 16, 17, 18, 63, 64, 65, 100, 2500, 4095, 4096, 4700, 4999])
    assert all(bool(torch.isfinite(t[x.cu[0]: x.cu[-1]]).all()) for t in (r["out"], r["dq"]))
    assert all(bool(torch.isfinite(t[x.cu_k[0]: x.cu_k[-1]]).all()) for t in (r["dk"], r["dv"]))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_what_is_not_a_key_has_no_effect(ma, dtype):
    """Padding, rows of no sequence and other sequences may hold anything."""
    x = Case([40, 3, 70], [33, 4000, 100], 4, 2, 64, dtype, 6, width=4100)
    clean = x.run(ma)
    at, at_k = x.cu.tolist(), x.cu_k.tolist()
    real = torch.zeros(x.k.shape[0], dtype=torch.bool, device="cuda")
    for i in (0, 2):
        real[at_k[i]: at_k[i] + x.keys[i]] = True
    for t in (x.k, x.v):
        t[~real] = math.nan
    for t in (x.q, x.dout):
        t[: at[0]] = math.nan
        t[at[1]: at[2]] = math.inf
        t[at[3]:] = math.nan
    r = x.run(ma)
    for i in (0, 2):
        rows, keys = slice(at[i], at[i + 1]), slice(at_k[i], at_k[i + 1])
        for name in r:
            pick = (lambda t: t[:, rows]) if name == "lse" else (lambda t: t[keys if name in ("dk", "dv") else rows])  # noqa: B023
            assert torch.equal(pick(r[name]), pick(clean[name])), (name, i)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("keys", [90, 5000])
def test_values_that_are_not_finite(ma, bad, keys):
    """Every row has a positive weight of every key here: its column of V reaches all rows as it is, others none."""
    x = Case([6], [keys], 2, 2, 64, "bf16", 7, first=0)
    clean = x.run(ma, grads=False)["out"]
    x.v[keys - 3, 1, 5] = bad
    for rest in (True, False):
        out = x.run(ma, grads=False, rest=rest)["out"]
        hit = out[:6, 1, 5].float()
        assert bool(torch.isnan(hit).all()) if math.isnan(bad) else bool((hit == bad).all())
        out[:6, 1, 5] = clean[:6, 1, 5]
        assert worst(out[:6], clean[:6].double(), clean[:6].double().abs() * 2.0 ** -7 + 2.0 ** -7) <= 1.0


def test_scores_of_minus_infinity(ma):
    """A row all of whose scores are -infinity is 0 / 0; keys of such a score beside others have no weight."""
    for keys in (50, 6000):
        x = Case([3], [keys], 1, 1, 64, "f32", 8, first=0, spare=0)
        x.q[:] = 1.0
        x.k[10:] = -math.inf
        r = x.run(ma, grads=False)
        want = attention(x.q, x.k[:10], x.v[:10], False)
        assert all(worst(r[n], *want[n]) <= 1.0 for n in ("out", "lse"))
        x.k[:10] = -math.inf
        r = x.run(ma, grads=False)
        assert bool(torch.isnan(r["out"]).all()) and bool((r["lse"] == -math.inf).all())


def test_clear(ma):
    x = Case([40, 0, 9], [100, 3, 0], 4, 2, 64, "bf16", 21, spare=700, first=300)
    x.check(x.run(ma, clear=True), clear=True)
    y = Case([], [], 4, 2, 64, "bf16", 22, spare=50)  # without a sequence all rows
    r = y.run(ma, clear=True)
    assert all(bool((r[n] == 0).all()) for n in ("out", "dq", "dk", "dv"))
    assert all(bool((t == 7).all()) for t in y.run(ma).values())


def test_one_side_empty(ma):
    """No rows at all: zero gradients of k and v.  No keys at all: zero rows, and null pointers in their place."""
    x = Case([0, 0], [50, 9], 2, 2, 64, "f16", 23, first=0, spare=0)
    r = x.run(ma)
    assert x.q.shape[0] == 0 and bool((r["dk"] == 0).all()) and bool((r["dv"] == 0).all())
    x = Case([5, 70], [0, 0], 2, 2, 64, "bf16", 24, first=0, spare=0)
    r = x.run(ma)
    assert x.k.shape[0] == 0 and bool((r["out"] == 0).all()) and bool((r["dq"] == 0).all()) and bool((r["lse"] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_long_walks_of_an_empty_side(ma, dtype):
    """Many rows over no keys at all, no rows at all over many keys: the walks are long, but there is nothing to cut."""
    for lens, Hq, Hkv in (([300], 2, 2), ([512], 4, 1), ([600, 0, 2000], 4, 2), ([5000], 1, 1)):
        print(lens, Hq, Hkv, dtype, flush=True)
        x = Case(lens, [0] * len(lens), Hq, Hkv, 64, dtype, 26, first=0, spare=0)
        r = x.run(ma)
        assert x.k.shape[0] == 0 and bool((r["out"] == 0).all()) and bool((r["dq"] == 0).all()) and bool((r["lse"] == -math.inf).all())
        q, k, v = (t.detach().clone().requires_grad_() for t in (x.q, x.k, x.v))
        ma.exact_cross_attention(q, k, v, x.cu, x.cu_k).backward(x.dout)
        torch.cuda.synchronize()
        assert bool((q.grad == 0).all()) and k.grad.shape == x.k.shape and v.grad.shape == x.v.shape
    for keys in ([5000], [20000, 0, 900]):
        print(keys, dtype, flush=True)
        x = Case([0] * len(keys), keys, 2, 1, 64, dtype, 27, first=0, spare=0)
        r = x.run(ma)
        assert x.q.shape[0] == 0 and bool((r["dk"] == 0).all()) and bool((r["dv"] == 0).all())
    for rows, keys in ((3000, 0), (0, 3000)):  # no sequence: all rows cleared
        q, k = (torch.ones(n, 4, 64, device="cuda", dtype=DTYPES[dtype]) for n in (rows, keys))
        lse, cu = torch.zeros(4, rows, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        dq, dk, dv = q.clone(), k.clone(), k.clone()
        ma.monarch_attn_exact_cross_bwd(q, k, k, q, lse, q, dq, dk, dv, cu, cu, clear=True)
        torch.cuda.synchronize()
        assert bool((dq == 0).all()) and bool((dk == 0).all()) and bool((dv == 0).all())


def test_row_starts_out_of_range(ma):
    """Starts beyond the tensors are clamped: the sequences that are whole are right.  Starts that decrease, which the
    interface excludes, lead to no access out of range, and leave the forward pass of the others right."""
    x = Case([20, 30], [40, 50], 2, 1, 64, "bf16", 25, first=0, spare=0)
    cu, cu_k = x.cu, x.cu_k
    for end in (1 << 30, -5):
        more = torch.tensor([1 << 30, end], dtype=torch.int32, device="cuda")
        x.cu, x.cu_k = torch.cat((cu, more)), torch.cat((cu_k, more))
        r = x.run(ma)
        x.cu, x.cu_k = cu, cu_k
        x.check(r if end > 0 else {n: r[n] for n in ("out", "lse")})


def test_same_bits_again(ma):
    for lens, keys in (([77, 130], [500, 60]), ([4, 2], [3000, 5000])):
        x = Case(lens, keys, 4, 2, 128, "bf16", 10)
        a, b = x.run(ma), x.run(ma)
        assert all(torch.equal(a[n], b[n]) for n in a)


def test_gradient_against_differences(ma):
    """<grad, direction> against central differences of the kernel's own fp32 forward.  The difference of step h has
    an error of h^2 from the third derivative and 2^-24 |f| / h from rounding: 1e-3 relative covers both at h = 2^-7."""
    x = Case([60, 9], [33, 120], 2, 1, 32, "f32", 11, spare=0, first=0)
    x.k, x.v = x.k.contiguous(), x.v.contiguous()
    r = x.run(ma)
    gen = torch.Generator(device="cuda").manual_seed(12)

    def f(which, t):
        keep = getattr(x, which)
        setattr(x, which, t)
        value = float((x.run(ma, grads=False)["out"].double() * x.dout.double()).sum())
        setattr(x, which, keep)
        return value

    for which in ("q", "k", "v"):
        t, grad = getattr(x, which), r["d" + which]
        step = torch.randn(t.shape, generator=gen, device="cuda")
        want = float((grad.double() * step.double()).sum())
        got = (f(which, t + 2.0 ** -7 * step) - f(which, t - 2.0 ** -7 * step)) * 2.0 ** 6
        size = float((grad.double().abs() * step.double().abs()).sum())
        assert abs(got - want) <= 1e-3 * size, (which, got, want, size)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("padded", [False, True])
def test_autograd(ma, dtype, padded):
    """The differentiable op on parts of a joint projection and on transposed views."""
    x = Case([90, 0, 61], [30, 200, 7], 4, 2, 64, dtype, 13, width=210 if padded else None)
    joint = torch.cat((x.k.flatten(1), x.v.flatten(1)), 1).requires_grad_()
    q = x.q.clone().requires_grad_()
    parts = [t.unflatten(1, (-1, 64)) for t in joint.split((128, 128), 1)]
    out = ma.exact_cross_attention(q, *parts, x.cu, x.cu_k, x.k_lens)
    dq, dkv = torch.autograd.grad(out, (q, joint), x.dout)
    dk, dv = (t.unflatten(1, (-1, 64)) for t in dkv.split((128, 128), 1))
    r = {"out": out.detach(), "dq": dq, "dk": dk, "dv": dv}
    x.check(r, clear=True)
    views = [t.detach().transpose(0, 1).contiguous().transpose(0, 1).requires_grad_() for t in (q, *parts)]
    again = ma.exact_cross_attention(*views, x.cu, x.cu_k, x.k_lens)
    assert torch.equal(again, out)
    for t, name in zip(torch.autograd.grad(again, views, x.dout.transpose(0, 1).contiguous().transpose(0, 1)), ("dq", "dk", "dv")):
        assert torch.equal(t, r[name])


def test_captured_step_and_pass(ma):
    """A decoding step and a training pass, captured, with other lengths and inputs at every replay."""
    s = torch.cuda.Stream()
    x = Case([4, 4, 4], [3000, 10, 700], 4, 4, 64, "bf16", 30, width=3500)
    y = Case([50, 90], [300, 40], 4, 2, 64, "bf16", 31)
    leaves = [t.detach().clone().requires_grad_() for t in (y.q, y.k, y.v)]
    out = torch.zeros_like(x.q)

    def step():
        ma.monarch_attn_exact_cross_fwd(x.q, x.k, x.v, out, x.cu, x.cu_k, x.k_lens)
        o = ma.exact_cross_attention(*leaves, y.cu, y.cu_k)
        return (o, *torch.autograd.grad(o, leaves, y.dout))

    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        captured = step()
    for i in range(4):
        with torch.no_grad():
            x.q.mul_(-1.0)
            x.k_lens.copy_(torch.tensor([3500 - 900 * i, i, 700], dtype=torch.int32))
            leaves[0].mul_(-0.5)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.detach().clone() for t in (out, *captured)]
        fresh = torch.zeros_like(out)
        ma.monarch_attn_exact_cross_fwd(x.q, x.k, x.v, fresh, x.cu, x.cu_k, x.k_lens)
        mine = [t.detach().clone().requires_grad_() for t in leaves]
        o = ma.exact_cross_attention(*mine, y.cu, y.cu_k)
        want = (fresh, o.detach(), *torch.autograd.grad(o, mine, y.dout))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_two_streams_at_once(ma):
    x = [Case([4, 2], [5000, 900], 4, 4, 64, "bf16", 40 + i) for i in range(2)]
    want = [c.run(ma, grads=True) for c in x]
    streams = [torch.cuda.Stream() for _ in x]
    got = []
    torch.cuda.synchronize()
    for _ in range(5):
        got.clear()
        for c, s in zip(x, streams):
            with torch.cuda.stream(s):
                r = {"out": torch.full_like(c.q, 7.0), "lse": torch.full((4, c.q.shape[0]), 7.0, device="cuda")}
                rest = torch.full_like(c.q, 7.0)
                ma.monarch_attn_exact_cross_fwd(c.q, c.k, c.v, r["out"], c.cu, c.cu_k, None, r["lse"], rest)
                r |= {"dq": torch.full_like(c.q, 7.0), "dk": torch.full(c.k.shape, 7.0, device="cuda", dtype=c.k.dtype),
                      "dv": torch.full(c.k.shape, 7.0, device="cuda", dtype=c.k.dtype)}
                ma.monarch_attn_exact_cross_bwd(c.q, c.k, c.v, r["out"], r["lse"], c.dout, r["dq"], r["dk"], r["dv"], c.cu, c.cu_k, None, rest)
                got.append(r)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(a[n], b[n]) for n in b)
