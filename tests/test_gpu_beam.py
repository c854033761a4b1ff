"""Selection of beams (monarch_attn_beam_select) and the paged cache in their order
(monarch_attn_paged_reorder) against plain implementations in 64 bits.

A value is formed in 64 bits but for the sum of exponentials: a tree of fp32 sums (32 elements a thread, 6 and 4 steps:
45 2^-24), exponentials of 2^-23 whose argument, at most log2 V on average over the weights, is off by 2^-24 of itself
(20 2^-24).  So 2^-17 bounds its error; where the values of two beams' candidates are that close either may come first.  Within a
beam the order is exact: by the logit, then by the token."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CLOSE = 2.0 ** -17


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def _select(ma, logits, scores, M, done=None, eos=-1):
    B = logits.shape[0]
    out = torch.full((B, M), 7.0, device="cuda")
    tokens, parents = (torch.full((B, M), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    ended = None if done is None else torch.zeros(B, M, dtype=torch.bool, device="cuda")
    got = ma.monarch_attn_beam_select(logits, scores, out, tokens, parents, done=done, done_out=ended, eos=eos)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is tokens and got[2] is parents
    return out, tokens, parents, ended


def _candidates(logits, scores, done, eos):
    """[B, K, V] in 64 bits."""
    x = logits.double()
    cand = scores.double()[..., None] + torch.log_softmax(x, -1)
    if done is not None:
        only = torch.full_like(cand, -math.inf)
        only[..., eos] = scores.double()
        cand = torch.where(done[..., None], only, cand)
    return torch.where(torch.isnan(cand), -math.inf, cand)


def _check(got, logits, scores, M, done=None, eos=-1):
    out, tokens, parents, ended = got
    B, K, V = logits.shape
    cand = _candidates(logits, scores, done, eos)
    want = cand.flatten(1).sort(dim=1, descending=True, stable=True)
    at = parents.long() * V + tokens.long()
    assert bool(((parents >= 0) & (parents < K) & (tokens >= 0) & (tokens < V)).all())
    mine = cand.flatten(1).gather(1, at)
    best = want.values[:, :M]
    finite = torch.isfinite(best)
    assert torch.equal(torch.isfinite(mine), finite)
    near = lambda a, b, tol: bool((torch.where(finite, a - b, 0.0).abs() <= tol).all())  # noqa: E731
    assert near(mine, best, 2 * CLOSE)
    assert near(out.double(), mine, CLOSE + torch.where(finite, mine, 0.0).abs() * 2.0 ** -24)
    assert bool((out[~finite] == best[~finite]).all())
    # candidates that are not finite come in the order of their place
    assert torch.equal(at[~finite], want.indices[:, :M][~finite])
    for b in range(B):
        assert len(set(at[b].tolist())) == M
        for k in range(K):
            mine_k = [t for t, p, f in zip(tokens[b].tolist(), parents[b].tolist(), finite[b].tolist()) if p == k and f]
            if done is not None and bool(done[b, k]):
                assert mine_k in ([], [eos])
            else:  # the first ones of the beam, in its order
                assert mine_k == logits[b, k].double().sort(descending=True, stable=True).indices[: len(mine_k)].tolist()
    if ended is not None:
        assert torch.equal(ended, done.gather(1, parents.long()) | (tokens == eos))
    return at, want.indices[:, :M]


SHAPES = [
    # B, K, V, M
    (1, 1, 1, 1), (1, 4, 7, 8), (3, 1, 33, 32), (2, 32, 100, 32), (1, 3, 257, 6), (5, 4, 8191, 8), (2, 2, 8192, 4), (2, 5, 8193, 10),
    (1, 4, 32000, 8), (3, 8, 50001, 16), (1, 16, 200003, 32), (1, 32, 524288, 32), (40, 2, 1000, 4),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,K,V,M", SHAPES)
def test_select(ma, B, K, V, M, dtype):
    print(B, K, V, M, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = (torch.randn(B, K, V, generator=gen, device="cuda") * 3).to(DTYPES[dtype])
    scores = -torch.rand(B, K, generator=gen, device="cuda").cumsum(1) * 2
    _check(_select(ma, logits, scores, M), logits, scores, M)
    if V > 2:
        done = torch.rand(B, K, generator=gen, device="cuda") < 0.4
        logits = logits.masked_fill(torch.rand(B, K, V, generator=gen, device="cuda") < 0.3, -math.inf)
        _check(_select(ma, logits, scores, M, done, 2), logits, scores, M, done, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_at_any_address(ma, dtype):
    """Rows that start anywhere in 16 bytes, with other values between them."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    whole = (torch.randn(2, 3, 9001, generator=gen, device="cuda") * 3 + 50).to(DTYPES[dtype])
    for a, z in ((0, 9001), (1, 9000), (2, 8999), (3, 8000), (5, 300), (7, 8)):
        x = whole[:, :, a:z]
        x.sub_(50)
        scores = -torch.rand(2, 3, generator=gen, device="cuda")
        M = min(6, 3 * (z - a))
        _check(_select(ma, x, scores, M), x, scores, M)
        x.add_(50)
    one = whole[1:, 2:, 4:4004]
    _check(_select(ma, one, scores[:1, :1], 5), one, scores[:1, :1], 5)
    each = whole[:, 1:2]
    _check(_select(ma, each, scores[:, :1].contiguous(), 5), each, scores[:, :1], 5)


def test_ties(ma):
    """All logits alike, whole rows alike, -0 beside 0: the lowest (beam, token) first, exactly."""
    for V in (5, 40, 20000):
        scores = torch.zeros(2, 4, device="cuda")
        for dtype in DTYPES.values():
            x = torch.zeros(2, 4, V, device="cuda", dtype=dtype)
            x[:, :, 1::2] = -0.0
            got = _select(ma, x, scores, 4)
            at, want = _check(got, x, scores, 4)
            assert torch.equal(at, want) and at.tolist() == [[0, 1, 2, 3]] * 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randint(-3, 4, (2, 1, 30000), generator=gen, device="cuda").float().expand(2, 4, 30000).contiguous()
    at, want = _check(_select(ma, x, scores, 32), x, scores, 32)
    assert torch.equal(at, want)  # equal rows: 3 appears thousands of times in beam 0
    x = torch.full((1, 2, 30000), -1.0, device="cuda")
    x[0, :, [5, 8000, 17000, 29999]] = 4.0  # the same four in both beams
    at, want = _check(_select(ma, x, torch.zeros(1, 2, device="cuda"), 7), x, torch.zeros(1, 2, device="cuda"), 7)
    assert torch.equal(at, want)


@pytest.mark.parametrize("M", [1, 7, 32])
def test_concentrated(ma, M):
    """The largest in one thread's elements, in order up or down, and far apart."""
    scores = torch.zeros(1, 2, device="cuda")
    for x in (torch.arange(40000.0), -torch.arange(40000.0), torch.arange(40000.0).view(5, 8000).T.reshape(-1), torch.arange(40000.0).remainder(256.0)):
        x = (x / 2048).cuda().expand(1, 2, 40000).contiguous()
        at, want = _check(_select(ma, x, scores, M), x, scores, M)
        assert torch.equal(at, want)


@pytest.mark.parametrize("kind", ["random", "up", "down", "equal", "few allowed", "last only"])
def test_many_rows(ma, kind):
    """Rows of several chunks a workgroup: later chunks against the best so far."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    B, K, V, M = 64, 8, 39999, 32
    step = torch.arange(float(V), device="cuda") / 4096
    x = {"random": lambda: torch.randn(B, K, V, generator=gen, device="cuda"), "up": lambda: step.expand(B, K, V).contiguous(),
         "down": lambda: -step.expand(B, K, V).contiguous(), "equal": lambda: torch.full((B, K, V), -2.5, device="cuda"),
         "few allowed": lambda: torch.randn(B, K, V, generator=gen, device="cuda").masked_fill(
             torch.rand(B, K, V, generator=gen, device="cuda") < 0.9998, -math.inf),
         "last only": lambda: torch.full((B, K, V), -math.inf, device="cuda").index_fill(2, torch.tensor([V - 2], device="cuda"), 1.0)}[kind]()
    scores = -torch.arange(float(K), device="cuda").expand(B, K).contiguous() / 3
    out, tokens, parents, _ = got = _select(ma, x, scores, M)
    _check(tuple(t if t is None else t[:3] for t in got), x[:3], scores[:3], M)
    want = _candidates(x, scores, None, -1).flatten(1).sort(dim=1, descending=True, stable=True)
    best = want.values[:, :M]
    finite = torch.isfinite(best)
    assert torch.equal(torch.isfinite(out), finite) and bool((torch.where(finite, out - best, 0.0).abs() <= 2 * CLOSE + 2.0 ** -24 * 40).all())
    if kind != "random":
        assert torch.equal(parents.long() * V + tokens.long(), want.indices[:, :M])


def test_first_step_and_dead_beams(ma):
    """Only the first beam in use; none; beams without an allowed token, with NaN or with +infinity."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(1, 4, 9000, generator=gen, device="cuda")
    scores = torch.tensor([[0.0, -math.inf, -math.inf, -math.inf]], device="cuda")
    at, want = _check(_select(ma, x, scores, 8), x, scores, 8)
    assert torch.equal(at, want) and bool((at < 9000).all())
    for bad in (math.nan, math.inf, -math.inf):
        y = x.clone()
        if bad == -math.inf:
            y[0, 1] = bad
        else:
            y[0, 1, 8500] = bad
        s = torch.zeros(1, 4, device="cuda")
        at, _ = _check(_select(ma, y, s, 8), y, s, 8)
        assert bool((at // 9000 != 1).all())
    for s in (torch.full((1, 4), -math.inf, device="cuda"), torch.full((1, 4), math.nan, device="cuda")):
        out, tokens, parents, _ = _select(ma, x, s, 8)
        assert bool((out == -math.inf).all()) and tokens.tolist() == [list(range(8))] and bool((parents == 0).all())


def test_few_allowed(ma):
    """Fewer candidates than asked for: -infinity fills up, the lowest (beam, token) first; done beams among them."""
    x = torch.full((1, 3, 10), -math.inf, device="cuda")
    x[0, 1, 4], x[0, 1, 6], x[0, 2, 3] = 1.0, 2.0, 0.5
    scores = torch.tensor([[-1.0, -2.0, -3.0]], device="cuda")
    done = torch.tensor([[True, False, False]], device="cuda")
    got = _select(ma, x, scores, 8, done, 2)
    at, want = _check(got, x, scores, 8, done, 2)
    assert torch.equal(at, want) and at[0, :4].tolist() == [2, 16, 23, 14] and at[0, 4:].tolist() == [0, 1, 3, 4]
    everything = torch.ones(1, 3, dtype=torch.bool, device="cuda")
    got = _select(ma, x, scores, 6, everything, 9)
    at, want = _check(got, x, scores, 6, everything, 9)
    assert torch.equal(at, want) and at[0].tolist() == [9, 19, 29, 0, 1, 2] and bool(got[3][0, :3].all())


def test_scores_of_any_size(ma):
    """Within a beam the logits decide, also where a score leaves them no bits."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(1, 2, 20000, generator=gen, device="cuda")
    for size in (-1e9, -1e30, 1e6):
        s = torch.tensor([[size, -math.inf]], device="cuda")
        _, tokens, parents, _ = _select(ma, x, s, 1)
        assert int(tokens) == int(x[0, 0].argmax()) or abs(size) > 2.0 ** 50
        assert int(parents) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [40, 20000, 200003])
def test_order_within_a_beam(ma, V, dtype):
    """The larger logit comes first, then the lower token, also where the values of different logits are the same in 64 bits:
    under large scores, and of logits that are small beside the log of their sum.  Between beams the lower one."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(1, 3, V, generator=gen, device="cuda")
    tiny = 2.0 ** -24 if dtype == "f16" else 1e-20  # (fp16 has no smaller ones: a few different values)
    for scale, sizes in ((1.0, (-1e9, 1e6, -1e30, 1e30, 3e38, -3e38)), (tiny, (0.0, -1e30))):
        y = (x * scale).to(DTYPES[dtype])
        order = y[0].double().sort(dim=1, descending=True, stable=True).indices
        for size in sizes:
            for M in (1, 5, 32):
                for used in ([2], [0], [1, 2]):
                    if len(used) > 1 and scale == 1.0 and abs(size) < 1e29:
                        continue  # (values of two beams that differ)
                    s = torch.full((1, 3), -math.inf, device="cuda")
                    s[0, used] = size
                    out, tokens, parents, _ = _select(ma, y, s, M)
                    if scale == 1.0 or len(used) == 1 or dtype != "f16":  # (fp16: sums of two beams that may differ)
                        assert bool((parents == used[0]).all()), (size, M, used)
                        assert tokens[0].tolist() == order[used[0], :M].tolist(), (size, M, used)
                    want = _candidates(y, s, None, -1)[0, parents[0].long(), tokens[0].long()]
                    assert bool(((out[0] - want).abs() <= CLOSE + want.abs() * 2.0 ** -24).all()), (size, M, used)


def _check_far(got, logits, scores, M):
    """As _check, for finite logits of any size: they count relative to the largest of their row, from which 64 bits
    may round them alike; then within a beam the logits decide."""
    out, tokens, parents, _ = got
    B, K, V = logits.shape
    x = logits.double() - logits.double().amax(-1, keepdim=True)
    cand = scores.double()[..., None] + (x - x.exp().sum(-1, keepdim=True).log())
    at = parents.long() * V + tokens.long()
    assert bool(((parents >= 0) & (parents < K) & (tokens >= 0) & (tokens < V)).all())
    mine, best = cand.flatten(1).gather(1, at), cand.flatten(1).sort(dim=1, descending=True).values[:, :M]
    assert bool(((mine - best).abs() <= 2 * CLOSE + best.abs() * 2.0 ** -51).all())
    assert bool(((out.double() - mine).abs() <= CLOSE + mine.abs() * 2.0 ** -24).all())
    for b in range(B):
        assert len(set(at[b].tolist())) == M
        for k in range(K):
            mine_k = tokens[b][parents[b] == k].tolist()
            assert mine_k == logits[b, k].double().sort(descending=True, stable=True).indices[: len(mine_k)].tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [7, 9001, 100003])
def test_logits_of_any_size(ma, V, dtype):
    """Rows all of whose logits are the same finite value, the lowest and the largest of the type among them; and masks of
    such values beside ordinary logits, few or nearly all of them."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    dt = DTYPES[dtype]
    most = torch.finfo(dt).max
    scores = torch.tensor([[-0.5, -0.25, -1.0]], device="cuda")
    M = min(8, V)
    for size in (1e3, 3e4, 1e6, 1e9, 3e9, 1e10, 7e10, 1e20, 1e30, 3e37, 1e38, 2.3e38, 2.4e38, most):
        if size > most:
            continue
        for value in (-size, size):
            print(V, dtype, value, flush=True)
            x = torch.full((1, 3, V), value, device="cuda", dtype=dt)
            _check_far(_select(ma, x, scores, M), x, scores, M)  # all of one size
            y = torch.randn(1, 3, V, generator=gen, device="cuda").to(dt)
            for share in (0.001, 0.5, 0.999):
                some = torch.rand(1, 3, V, generator=gen, device="cuda") < share
                some[:, :, V // 2] = False
                z = y.masked_fill(some, value)
                _check_far(_select(ma, z, scores, M), z, scores, M)
                z[0, 1] = value
                _check_far(_select(ma, z, scores, M), z, scores, M)
            if V > 8192:  # the large ones in an early or a late chunk only
                for part in (slice(0, 8000), slice(V - 500, V)):
                    z = y.clone()
                    z[:, :, part] = value
                    _check_far(_select(ma, z, scores, M), z, scores, M)
    wide = torch.cat([torch.full((1, 3, V), f * most, device="cuda", dtype=dt) for f in (-1.0, 1.0)], 2)  # both ends of the range
    _check_far(_select(ma, wide, scores, M), wide, scores, M)
    many = (torch.randn(128, 4, V, generator=gen, device="cuda") * 3).to(dt).masked_fill(torch.rand(128, 4, V, generator=gen, device="cuda") < 0.98, -1e4)
    if dtype != "f16":
        many = many.masked_fill(many == many.min(), -7e10)
    s = torch.zeros(128, 4, device="cuda")
    got = _select(ma, many, s, M)
    _check_far(tuple(t if t is None else t[:2] for t in got), many[:2], s[:2], M)


def test_same_bits_again_and_on_two_streams(ma):
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = [(torch.randn(4, 4, 50001, generator=gen, device="cuda") * 3).bfloat16() for _ in range(2)]
    s = torch.zeros(4, 4, device="cuda")
    want = [_select(ma, t, s, 8) for t in x]
    streams = [torch.cuda.Stream() for _ in x]
    for _ in range(5):
        got = []
        for t, st in zip(x, streams):
            with torch.cuda.stream(st):
                o = (torch.zeros(4, 8, device="cuda"), *(torch.zeros(4, 8, dtype=torch.int32, device="cuda") for _ in range(2)))
                got.append(ma.monarch_attn_beam_select(t, s, *o))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b[:3]))


def _reordered(k, v, table, parents, lens, move):
    """Beam by beam, from a copy."""
    k2, v2, table2 = k.clone(), v.clone(), table.clone()
    B, K = parents.shape
    page = k.shape[2]
    for b in range(B):
        full, rest = divmod(max(0, int(lens[b * K])), page)
        for c in range(K):
            p = int(parents[b, c])
            if not 0 <= p < K:
                continue
            me, from_ = b * K + c, b * K + p
            if move:
                table2[me, :full] = table[from_, :full]
            if rest and full < table.shape[1]:
                dst, src = int(table[me, full]), int(table[from_, full])
                if 0 <= dst < k.shape[0] and 0 <= src < k.shape[0]:
                    k2[dst, :, :rest], v2[dst, :, :rest] = k[src, :, :rest], v[src, :, :rest]
    return k2, v2, table2


@pytest.mark.parametrize("move", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,K,lens,Hkv,d,page", [
    (1, 1, [5], 1, 8, 8), (2, 4, [0, 16], 2, 64, 16), (3, 3, [1, 15, 100], 1, 40, 16), (2, 8, [63, 64], 8, 128, 64), (1, 16, [1000], 3, 72, 32),
    (2, 32, [70, 9], 2, 96, 8), (1, 5, [300], 12, 64, 128), (3, 2, [4100, 3, 4096], 1, 128, 4096)])
def test_reorder(ma, B, K, lens, Hkv, d, page, dtype, move):
    print(B, K, lens, Hkv, d, page, dtype, move, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(7)
    blocks = max(lens) // page + 2
    k, v = (torch.randn(B * K * blocks + 1, Hkv, page, d, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    table = torch.randperm(B * K * blocks + 1, generator=gen, device="cuda")[: B * K * blocks].int().view(B * K, blocks)
    tokens = torch.tensor(lens, dtype=torch.int32, device="cuda").repeat_interleave(K)
    for parents in (torch.randint(0, K, (B, K), generator=gen, device="cuda"), torch.arange(K, device="cuda").flip(0).expand(B, K),
                    torch.zeros(B, K, device="cuda"), torch.arange(K, device="cuda").roll(1).expand(B, K)):
        parents = parents.int().contiguous()
        want = _reordered(k, v, table, parents, tokens, move)
        got = ma.monarch_attn_paged_reorder(k, v, table, parents, tokens, move_table=move)
        torch.cuda.synchronize()
        assert got[0] is k and got[1] is v and got[2] is table
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_reorder_of_what_is_not_there(ma):
    """Parents out of range, pages outside the cache and lengths beyond the table or below zero move nothing."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    k, v = (torch.randn(20, 2, 8, 32, generator=gen, device="cuda") for _ in range(2))
    table = torch.randperm(18, generator=gen, device="cuda").int().view(6, 3)
    table[1, 1], table[4, 0], table[5, 2] = -1, 99, 1 << 30
    for lens in ([13] * 6, [5] * 3 + [21] * 3, [1 << 30] * 6, [-3] * 6, [24] * 6):
        tokens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        parents = torch.tensor([[1, 0, 7], [-1, 2, 1]], dtype=torch.int32, device="cuda")
        if max(lens) > 24:  # more tokens than the table holds: all of its entries are of full pages
            want = _reordered(k, v, table, parents, torch.full_like(tokens, 24), True)
        else:
            want = _reordered(k, v, table, parents, tokens, True)
        got = ma.monarch_attn_paged_reorder(k, v, table, parents, tokens)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), lens


def test_captured(ma):
    """Selection and reorder in one graph, replayed with other logits."""
    s = torch.cuda.Stream()
    gen = torch.Generator(device="cuda").manual_seed(9)
    B, K, V, page = 3, 4, 20001, 8
    x = torch.randn(B, K, V, generator=gen, device="cuda")
    scores = torch.zeros(B, K, device="cuda")
    done, ended = torch.zeros(B, K, dtype=torch.bool, device="cuda"), torch.zeros(B, K, dtype=torch.bool, device="cuda")
    out, tokens, parents = torch.zeros(B, K, device="cuda"), *(torch.zeros(B, K, dtype=torch.int32, device="cuda") for _ in range(2))
    k, v = (torch.randn(60, 2, page, 64, generator=gen, device="cuda") for _ in range(2))
    table = torch.randperm(60, generator=gen, device="cuda").int().view(B * K, 5)
    lens = torch.full((B * K,), 21, dtype=torch.int32, device="cuda")

    def step():
        ma.monarch_attn_beam_select(x, scores, out, tokens, parents, done=done, done_out=ended, eos=1)
        ma.monarch_attn_paged_reorder(k, v, table, parents, lens)

    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    for i in range(4):
        x.copy_(torch.randn(B, K, V, generator=gen, device="cuda") * (i + 1))
        scores.copy_(out)
        done.copy_(ended)
        lens.fill_(18 + i)
        before = [t.clone() for t in (k, v, table)]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, tokens, parents, ended)]
        _check(got, x, scores, K, done, 1)
        assert all(torch.equal(a, b) for a, b in zip((k, v, table), _reordered(*before, parents, lens, True)))
        want = _select(ma, x, scores, K, done, 1)  # (an eager call between the replays)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
