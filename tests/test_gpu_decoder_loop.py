"""The decoder's operators as they are used together: beam search of a small encoder-decoder whose encoder runs
MonarchAttention, against the same decoder in 64 bits on every beam's whole history; the same operators captured into a
graph against eager ones; and a training pass through rotation, packed self attention and cross attention."""
import math

import pytest
import torch

from sequence_reference import starts
from test_gpu_beam import _check

pytestmark = pytest.mark.gpu
B, K, V, H, HKV, D, PAGE, LAYERS, ENC, EOS = 2, 3, 50, 4, 2, 32, 8, 2, 24, 1


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def _weights():
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = lambda *shape: torch.randn(*shape, generator=gen, device="cuda") / math.sqrt(shape[0])  # noqa: E731
    width = H * D
    layers = [{"qkv": w(width, (H + 2 * HKV) * D), "o": w(width, width), "cq": w(width, width), "ckv": w(width, 2 * HKV * D), "co": w(width, width)}
              for _ in range(LAYERS)]
    return {"emb": torch.randn(V, width, generator=gen, device="cuda"), "out": 3 * w(width, V), "layers": layers, "enc": w(width, 3 * width)}


def _encode(ma, w, lens):
    """States [B, ENC, H D] of a padded batch, by MonarchAttention."""
    x = torch.randn(B, ENC, H * D, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    q, k, v = ((x @ w["enc"]).view(B, ENC, 3, H, D).permute(2, 0, 3, 1, 4).contiguous())
    out = ma.monarch_attn_fwd_varlen(q, k, v, torch.empty_like(q), lens, m=4, b=6, T=2)
    return out.transpose(1, 2).flatten(2)


def _freq():
    return (100.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()


def _reference(w, states, lens, tokens):
    """Logits [V] after `tokens` for one request: the whole decoder in 64 bits."""
    d64 = lambda t: t.double()  # noqa: E731
    states = d64(states)[: int(lens)]
    h, n = d64(w["emb"])[tokens], len(tokens)
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * d64(_freq())
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turn(x):
        a, b = x[..., : D // 2], x[..., D // 2:]
        return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)

    def attend(q, k, v, causal):
        k, v = (t.repeat_interleave(H // HKV, 1) for t in (k, v))
        s = torch.stack([q[:, i] @ k[:, i].T for i in range(H)]) / math.sqrt(D)
        if causal:
            s = s.masked_fill(~torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), -math.inf)
        p = s.softmax(-1)
        return torch.stack([p[i] @ v[:, i] for i in range(H)], 1).flatten(1)

    for layer in w["layers"]:
        q, k, v = (t.unflatten(1, (-1, D)) for t in (h @ d64(layer["qkv"])).split((H * D, HKV * D, HKV * D), 1))
        h = h + attend(turn(q), turn(k), v, True) @ d64(layer["o"])
        k, v = (t.unflatten(1, (-1, D)) for t in (states @ d64(layer["ckv"])).split(HKV * D, 1))
        h = h + attend((h @ d64(layer["cq"])).unflatten(1, (-1, D)), k, v, False) @ d64(layer["co"])
    return h[-1] @ d64(w["out"])


def _ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


class _Serving:
    """What a program keeps from step to step."""

    def __init__(self, pages, blocks, dtype=torch.float32):
        gen = torch.Generator().manual_seed(3)
        rows = B * K
        self.ring, self.free, self.left = torch.randperm(pages, generator=gen).int().cuda(), torch.tensor([0, pages], dtype=torch.int32, device="cuda"), _ints(2)
        self.table, self.past, self.kv, self.cu = torch.full((rows, blocks), -1, dtype=torch.int32, device="cuda"), _ints(rows), _ints(rows), _ints(rows + 1)
        self.slots, self.status, self.fresh = torch.zeros(rows, dtype=torch.int64, device="cuda"), _ints(1), torch.ones(rows, dtype=torch.int32, device="cuda")
        self.caches = [[torch.full((pages, HKV, PAGE, D), math.nan, device="cuda", dtype=dtype) for _ in range(2)] for _ in range(LAYERS)]
        self.scores = torch.tensor([[0.0] + [-math.inf] * (K - 1)] * B, device="cuda")
        self.done = torch.zeros(B, K, dtype=torch.bool, device="cuda")
        self.out, self.tokens, self.parents, self.ended = torch.zeros(B, K, device="cuda"), _ints(B, K), _ints(B, K), torch.zeros_like(self.done)
        self.cu_q = torch.arange(0, rows + 1, K, dtype=torch.int32, device="cuda")
        self.cu_k = torch.arange(0, B * ENC + 1, ENC, dtype=torch.int32, device="cuda")

    def plan(self, ma):
        ma.monarch_attn_paged_plan(self.past, self.fresh, self.ring, self.free, self.table, self.cu, self.kv, self.slots, self.left, self.status, PAGE)

    def self_attention(self, ma, layer, joint, freq):
        q, k, v = (t.unflatten(1, (-1, D)) for t in joint.split((H * D, HKV * D, HKV * D), 1))
        turned, out = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(q.shape, device="cuda", dtype=q.dtype)
        ma.monarch_attn_paged_append(q, k, v, turned, *self.caches[layer], freq, self.cu, self.kv, self.slots)
        return ma.monarch_attn_exact_paged_fwd(turned, *self.caches[layer], out, self.cu, self.kv, self.table)[0].flatten(1)

    def cross_attention(self, ma, q, kv, lens):
        k, v = (t.unflatten(1, (-1, D)) for t in kv.split(HKV * D, 1))
        out = torch.empty(B * K, H, D, device="cuda", dtype=q.dtype)
        return ma.monarch_attn_exact_cross_fwd(q.unflatten(1, (-1, D)), k, v, out, self.cu_q, self.cu_k, lens)[0].flatten(1)

    def choose(self, ma, logits):
        ma.monarch_attn_beam_select(logits.view(B, K, V), self.scores, self.out, self.tokens, self.parents, done=self.done, done_out=self.ended, eos=EOS)
        for i, cache in enumerate(self.caches):
            ma.monarch_attn_paged_reorder(*cache, self.table, self.parents, self.kv, move_table=i == 0)
        for to, new in ((self.scores, self.out), (self.done, self.ended), (self.past, self.kv), (self.free, self.left)):
            to.copy_(new)


def test_beam_search(ma):
    """20 steps over three pages a beam.  An output of the decoder is a chain of about ten sums of at most 128 products,
    each off by no more than 2^7 2^-24 of its terms, and of two layers of residuals: 2^-12 of the largest logit."""
    w, lens = _weights(), torch.tensor([ENC, 13], dtype=torch.int32, device="cuda")
    states = _encode(ma, w, lens)
    kvs = [states.flatten(0, 1) @ layer["ckv"] for layer in w["layers"]]
    kvs[0][ENC + 13:] = math.nan  # padding is not read
    s = _Serving(pages=60, blocks=4)
    history, tokens = [[[0] for _ in range(K)] for _ in range(B)], _ints(B * K)
    for step in range(20):
        s.plan(ma)
        h = w["emb"][tokens.long()]
        for i, layer in enumerate(w["layers"]):
            h = h + s.self_attention(ma, i, h @ layer["qkv"], _freq()) @ layer["o"]
            h = h + s.cross_attention(ma, h @ layer["cq"], kvs[i], lens) @ layer["co"]
        logits = h @ w["out"]
        for b in range(B):
            for k in range(K):
                if not math.isinf(float(s.scores[b, k])):
                    want = _reference(w, states[b], lens[b], history[b][k])
                    off = float((logits[b * K + k].double() - want).abs().max() / want.abs().max())
                    assert off <= 2.0 ** -12, (step, b, k, off)
        scores, done = s.scores.clone(), s.done.clone()
        s.choose(ma, logits)
        _check((s.out, s.tokens, s.parents, s.ended), logits.view(B, K, V), scores, K, done, EOS)
        tokens = s.tokens.flatten()
        history = [[history[b][int(s.parents[b, k])] + [int(s.tokens[b, k])] for k in range(K)] for b in range(B)]
        assert int(s.status) == 0
    assert s.past.tolist() == [20] * (B * K)
    assert len(set(s.table[:, 2].tolist())) == B * K  # the started page is a beam's own


def test_captured_steps(ma):
    """A step of all operators in one graph, replayed for 20 tokens over new projections and logits, against eager steps."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    lens = torch.tensor([17, ENC], dtype=torch.int32, device="cuda")
    joint = torch.zeros(LAYERS, B * K, (H + 2 * HKV) * D, device="cuda", dtype=torch.bfloat16)
    cq, kv = torch.zeros(B * K, H * D, device="cuda", dtype=torch.bfloat16), torch.randn(B * ENC, 2 * HKV * D, generator=gen, device="cuda").bfloat16()
    logits, freq = torch.zeros(B * K, V, device="cuda", dtype=torch.bfloat16), _freq()

    def step(s):
        s.plan(ma)
        outs = [s.self_attention(ma, i, joint[i], freq) for i in range(LAYERS)] + [s.cross_attention(ma, cq, kv, lens)]
        s.choose(ma, logits)
        return outs

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(_Serving(60, 4, torch.bfloat16))  # sizes the stream's workspace
    torch.cuda.synchronize()
    one, other = _Serving(60, 4, torch.bfloat16), _Serving(60, 4, torch.bfloat16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        captured = step(one)
    for i in range(20):
        for t in (joint, cq, logits):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda") * 2)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = step(other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), i
        for name in ("table", "past", "scores", "done", "tokens", "parents", "free", "status"):
            assert torch.equal(getattr(one, name), getattr(other, name)), (i, name)
    assert one.past.tolist() == [20] * (B * K) and int(one.status) == 0


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2.0 ** -14), (torch.bfloat16, 2.0 ** -4)])
def test_training_pass(ma, dtype, tol):
    """Gradients of a layer of rotation, causal self attention and cross attention against autograd in 64 bits: eight
    roundings of half a step (2^-8 in bf16) one after another; in fp32 sums of at most 2^7 terms, 2^-17 each."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    lens, keys = [37, 5, 60], [20, 33, 1]
    cu, cu_k, freq = starts(lens, "cuda"), starts(keys, "cuda"), _freq()
    leaves = [torch.randn(n, h, D, generator=gen, device="cuda").to(dtype).requires_grad_()
              for n, h in ((sum(lens), H), (sum(lens), HKV), (sum(lens), HKV), (sum(keys), HKV), (sum(keys), HKV))]
    dout = torch.randn(sum(lens), H, D, generator=gen, device="cuda").to(dtype)

    def ours(q, k, v, ck, cv):
        q, k = ma.rotate_packed(q, k, freq, cu)
        return ma.exact_cross_attention(ma.exact_attention_packed(q, k, v, cu), ck, cv, cu, cu_k)

    def plain(q, k, v, ck, cv):
        outs = []
        for a, n, b, m in zip(cu.tolist(), lens, cu_k.tolist(), keys):
            angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None, None] * freq.double()

            def turn(x):
                x, y = x[a:a + n, :, : D // 2], x[a:a + n, :, D // 2:]  # noqa: B023
                return torch.cat((x * angle.cos() - y * angle.sin(), x * angle.sin() + y * angle.cos()), -1)  # noqa: B023

            def attend(q, k, v, causal):
                k, v = (t.repeat_interleave(H // HKV, 1) for t in (k, v))
                s = torch.stack([q[:, i] @ k[:, i].T for i in range(H)]) / math.sqrt(D)
                if causal:
                    s = s.masked_fill(~torch.ones_like(s[0], dtype=torch.bool).tril(), -math.inf)
                return torch.stack([s[i].softmax(-1) @ v[:, i] for i in range(H)], 1)

            outs.append(attend(attend(turn(q), turn(k), v[a:a + n], True), ck[b:b + m], cv[b:b + m], False))
        return torch.cat(outs)

    got = ours(*leaves)
    doubles = [t.detach().double().requires_grad_() for t in leaves]
    want = plain(*doubles)
    for name, a, b in zip("out q k v ck cv".split(), (got, *torch.autograd.grad(got, leaves, dout)), (want, *torch.autograd.grad(want, doubles, dout.double()))):
        off = float((a.detach().double() - b.detach()).norm() / b.detach().norm())
        assert off <= tol, (name, off)


def test_second_derivatives_are_refused(ma):
    cu, freq = starts([9], "cuda"), _freq()
    q, k, v = (torch.randn(9, h, D, device="cuda", requires_grad=True) for h in (H, HKV, HKV))
    for out, leaves in ((ma.rotate_packed(q, k, freq, cu)[0], (q,)), (ma.exact_cross_attention(q, k, v, cu, cu), (q, k, v))):
        plain = torch.autograd.grad(out.sum(), leaves, retain_graph=True)
        kept = torch.autograd.grad(out.sum(), leaves, create_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(plain, kept))
        with pytest.raises(RuntimeError, match="once_differentiable|does not require grad"):
            kept[0].sum().backward()
