"""The paged cache: its plan, the write of its rows and the attention that
reads it, alone against references and together as a serving loop uses them."""
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


def _cache(new, past, Hkv, d, page, dtype, gen, slack=3, extra=4):
    """Keys and values of every sequence, the pages that hold them (NaN elsewhere), block table and key counts."""
    kv = [max(0, a + b) for a, b in zip(new, past)]
    blocks = [-(-n // page) for n in kv]
    pages = sum(blocks) + extra
    ids = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((len(new), max(blocks + [0]) + slack), -1, dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((pages, Hkv, page, d), math.nan, device="cuda", dtype=DTYPES[dtype]) for _ in range(2))
    seqs, at = [], 0
    for i, n in enumerate(kv):
        mine = ids[at : at + blocks[i]]
        at += blocks[i]
        table[i, : blocks[i]] = mine
        k, v = (torch.randn(n, Hkv, d, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
        pos = torch.arange(n, device="cuda")
        for src, dst in ((k, kp), (v, vp)):
            if n:
                dst[mine[pos // page].long(), :, pos % page] = src
        seqs.append((k, v))
    return seqs, kp, vp, table, torch.tensor(kv, device="cuda", dtype=torch.int32)


def _attend(ma, q, kp, vp, cu, kv, table, causal=True, stream=None):
    out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype)
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table, causal, lse, stream=stream)
    torch.cuda.synchronize()
    return out, lse


def _check(out, lse, q, cu, seqs, past, causal=True):
    at = cu.tolist()
    assert bool((out[: at[0]] == 7).all()) and bool((out[at[-1]:] == 7).all()) and bool((lse[:, at[-1]:] == 7).all())
    for i, (a, z) in enumerate(zip(at[:-1], at[1:])):
        if a == z:
            continue
        ref = attention(q[a:z], *seqs[i], causal, past[i])
        for name, got in (("out", out[a:z]), ("lse", lse[:, a:z])):
            off = worst(got, *ref[name])
            assert off <= 1.0, f"{name} of sequence {i}: {off:.3g} of what rounding allows"


CASES = [
    # new tokens, tokens before them, Hq, Hkv, d, page
    ([1], [0], 1, 1, 64, 16),
    ([1], [499], 16, 4, 64, 16),
    ([1, 1, 1, 1], [0, 15, 16, 3000], 8, 2, 128, 16),
    ([1] * 20, [37 * i for i in range(20)], 4, 1, 128, 32),
    ([1, 1], [5000, 9], 12, 3, 96, 8),
    ([2, 0, 7, 1], [100, 50, 0, 1], 6, 2, 40, 64),
    ([33, 1, 128], [1000, 700, 0], 8, 1, 128, 16),
    ([300, 5], [77, 4000], 4, 4, 72, 128),
    ([1, 3], [2047, 2049], 32, 1, 64, 16),
    ([130], [9000], 2, 2, 64, 256),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,past,Hq,Hkv,d,page", CASES)
def test_paged_attention(ma, new, past, Hq, Hkv, d, page, dtype):
    print(new[:4], past[:4], Hq, Hkv, d, page, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    seqs, kp, vp, table, kv = _cache(new, past, Hkv, d, page, dtype, gen)
    cu = starts(new, "cuda", 1)
    q = torch.randn(sum(new) + 4, Hq, d, generator=gen, device="cuda").to(DTYPES[dtype])
    _check(*_attend(ma, q, kp, vp, cu, kv, table), q, cu, seqs, past)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_causal(ma, dtype):
    """Every new row sees the whole cache, as a decoder's attention over its encoder's keys."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    new, past = [5, 1, 40], [95, 2000, -39]
    seqs, kp, vp, table, kv = _cache(new, past, 2, 64, 16, dtype, gen)
    cu = starts(new, "cuda")
    q = torch.randn(sum(new), 4, 64, generator=gen, device="cuda").to(DTYPES[dtype])
    _check(*_attend(ma, q, kp, vp, cu, kv, table, causal=False), q, cu, seqs, past, causal=False)


@pytest.mark.parametrize("wide", [False, True])  # with a wide table the call is split over the keys
def test_rows_that_see_no_key(ma, wide):
    """Fewer keys than new tokens: the first rows see none and get zero and -inf; no keys at all the same."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    new, past = [10, 4, 3], [-6, -4, 20]
    seqs, kp, vp, table, kv = _cache(new, past, 2, 64, 16, "bf16", gen, slack=300 if wide else 3)
    cu = starts(new, "cuda")
    q = torch.randn(sum(new), 4, 64, generator=gen, device="cuda").bfloat16()
    out, lse = _attend(ma, q, kp, vp, cu, kv, table)
    _check(out, lse, q, cu, seqs, past)
    for rows in (slice(0, 6), slice(10, 14)):
        assert bool((out[rows] == 0).all()) and bool((lse[:, rows] == -math.inf).all())


@pytest.mark.parametrize("page_number", [-1, 1 << 20, -(1 << 31), (1 << 31) - 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("wide", [False, True])
def test_pages_outside_the_cache(ma, page_number, dtype, wide):
    """No read outside: the rows that see a token on such a page are NaN, the others as they would be."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    new, past = [40, 1, 1], [30, 200, 90]
    seqs, kp, vp, table, kv = _cache(new, past, 2, 64, 16, dtype, gen, slack=300 if wide else 3)
    cu = starts(new, "cuda")
    q = torch.randn(sum(new), 4, 64, generator=gen, device="cuda").to(DTYPES[dtype])
    good, _ = _attend(ma, q, kp, vp, cu, kv, table)
    table[0, 3], table[2, 0] = page_number, page_number  # tokens 48..63 of sequence 0: seen by its rows from 18 on
    out, _ = _attend(ma, q, kp, vp, cu, kv, table)
    assert bool(torch.isnan(out[18:40]).all()) and bool(torch.isnan(out[41]).all())
    assert torch.equal(out[:18], good[:18]) and torch.equal(out[40], good[40])


def test_keys_that_are_not_seen_have_no_effect(ma):
    """A later token of the chunk and what lies behind the last token in its page."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    new, past = [30, 1], [25, 70]
    seqs, kp, vp, table, kv = _cache(new, past, 2, 64, 16, "bf16", gen)
    cu = starts(new, "cuda")
    q = torch.randn(sum(new), 4, 64, generator=gen, device="cuda").bfloat16()
    good, _ = _attend(ma, q, kp, vp, cu, kv, table)
    for pages in (kp, vp):
        pages[table[0, 40 // 16].long(), :, 40 % 16] = math.inf
    out, _ = _attend(ma, q, kp, vp, cu, kv, table)
    assert torch.equal(out[:15], good[:15]) and not bool(torch.isfinite(out[15:30]).any(-1).all()) and torch.equal(out[30], good[30])


def test_key_counts_are_clamped(ma):
    gen = torch.Generator(device="cuda").manual_seed(6)
    seqs, kp, vp, table, kv = _cache([1, 1], [63, 31], 1, 64, 16, "bf16", gen, slack=0)
    cu = starts([1, 1], "cuda")
    q = torch.randn(2, 2, 64, generator=gen, device="cuda").bfloat16()
    kv[0], kv[1] = 1 << 30, -5  # 4 blocks of 16: 64 keys; none
    out, lse = _attend(ma, q, kp, vp, cu, kv, table)
    ref = attention(q[:1], *seqs[0], True, 63)
    assert worst(out[:1], *ref["out"]) <= 1.0 and bool((out[1] == 0).all()) and bool((lse[:, 1] == -math.inf).all())


def test_empty_cache_and_table(ma):
    q = torch.randn(3, 2, 64, device="cuda").bfloat16()
    kp = torch.empty(0, 1, 16, 64, device="cuda", dtype=torch.bfloat16)
    cu, kv = starts([3], "cuda"), torch.tensor([40], device="cuda", dtype=torch.int32)
    out, _ = _attend(ma, q, kp, kp, cu, kv, torch.empty(1, 0, device="cuda", dtype=torch.int32))
    assert bool((out == 0).all())
    out, _ = _attend(ma, q, kp, kp, cu, kv, torch.zeros(1, 4, device="cuda", dtype=torch.int32))
    assert bool(torch.isnan(out).all())  # page 0 of no pages


def test_cache_past_32_bits(ma):
    """Pages whose offset in the cache passes 2^32 bytes."""
    pages, Hkv, page, d = 40000, 8, 16, 128  # 1.3 GB elements: 2.6 GB... and the offsets of the last pages beyond 2^31
    pages = (1 << 32) // (Hkv * page * d * 2) * 2 + 100
    kp, vp = (torch.empty(pages, Hkv, page, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(7)
    n = 45
    k, v = (torch.randn(n, Hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.tensor([[pages - 1, 5, pages - 7]], device="cuda", dtype=torch.int32)
    pos = torch.arange(n, device="cuda")
    ma.monarch_attn_paged_write(k, v, kp, vp, table[0, pos // page].long() * page + pos % page)
    q = torch.randn(1, 16, d, generator=gen, device="cuda").bfloat16()
    out, _ = _attend(ma, q, kp, vp, starts([1], "cuda"), torch.tensor([n], device="cuda", dtype=torch.int32), table)
    assert worst(out, *attention(q, k, v, True, n - 1)["out"]) <= 1.0
    assert torch.equal(kp[pages - 7, :, 12], k[44])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Hkv,d,page,rows", [(1, 8, 8, 1), (3, 40, 16, 77), (8, 128, 32, 500), (12, 64, 256, 3)])
def test_write(ma, Hkv, d, page, rows, dtype):
    """Rows of strided tensors into their slots; slots outside the cache are skipped and everything else is left."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    joint = torch.randn(rows, 3 * Hkv * d, generator=gen, device="cuda").to(DTYPES[dtype])
    k, v = (joint[:, i * Hkv * d : (i + 1) * Hkv * d].unflatten(1, (Hkv, d)) for i in (0, 2))
    pages = rows // page + 3
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:rows]
    for i, bad in ((rows // 2, -1), (rows // 3, pages * page), (rows // 4, -(1 << 40)), (rows // 5, 1 << 40)):
        if rows > 3:
            slots[i] = bad
    kp, vp = (torch.randn(pages, Hkv, page, d, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    want = [kp.clone(), vp.clone()]
    for w, x in zip(want, (k, v)):
        for r, s in enumerate(slots.tolist()):
            if 0 <= s < pages * page:
                w[s // page, :, s % page] = x[r]
    got = ma.monarch_attn_paged_write(k, v, kp, vp, slots)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def _plan(ma, past, fresh, ring, free, table, page, capacity):
    ints = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    B = len(past)
    t = {"table": ints(table).reshape(B, -1) if B else torch.empty(0, 4, device="cuda", dtype=torch.int32),
         "cu": torch.full((B + 1,), -9, device="cuda", dtype=torch.int32),
         "kv": torch.full((B,), -9, device="cuda", dtype=torch.int32),
         "slots": torch.full((capacity,), -9, device="cuda", dtype=torch.int64), "left": ints([-9, -9]), "status": ints([-9])}
    ma.monarch_attn_paged_plan(ints(past), ints(fresh), ints(ring), ints(free), t["table"], t["cu"], t["kv"], t["slots"],
                               t["left"], t["status"], page)
    return {n: x.tolist() for n, x in t.items()}


def _plan_reference(past, fresh, ring, free, table, page, capacity):
    B, F = len(past), len(ring)
    table = [list(r) for r in table]
    width = len(table[0]) if B else 4
    first, count = (free[0] % F if F else 0), max(0, min(free[1], F))
    status, taken, rows, cu, kv, slots = 0, 0, 0, [0], [], []
    for b in range(B):
        if past[b] < 0 or fresh[b] < 0:
            status |= 4
        p, n = max(0, past[b]), max(0, fresh[b])
        if p + n > width * page:
            status |= 2
        had, have = -(-min(p, width * page) // page), -(-min(p + n, width * page) // page)
        for j in range(had, have):
            table[b][j] = ring[(first + taken) % F] if taken < count else -1
            taken += 1
        for pos in range(p, p + n):
            pg = table[b][pos // page] if pos // page < width else -1
            slots.append(pg * page + pos % page if pg >= 0 else -1)
        rows += n
        cu.append(min(rows, capacity))
        kv.append(min(p + n, width * page))
    if taken > count:
        status |= 1
    if rows > capacity:
        status |= 8
    slots = (slots + [-1] * capacity)[:capacity]
    used = min(taken, count)
    return {"table": table, "cu": cu, "kv": kv, "slots": slots,
            "left": [(first + used) % max(F, 1), count - used], "status": [status]}


@pytest.mark.parametrize("seed", range(12))
def test_plan(ma, seed):
    """Random requests: idle ones, new ones, pages that are full, a ring that wraps around, and, with odd seeds, too
    few pages, a table too narrow, too few slots or negative lengths."""
    import random

    rng = random.Random(seed)
    page = rng.choice((8, 16, 64))
    B = rng.choice((1, 3, 64, 300, 1000))
    past = [rng.choice((0, page, rng.randint(0, 5 * page))) for _ in range(B)]
    fresh = [rng.choice((0, 1, 1, rng.randint(0, 3 * page))) for _ in range(B)]
    had = [-(-p // page) for p in past]
    width = max(-(-(p + n) // page) for p, n in zip(past, fresh)) + 1
    capacity = sum(fresh) + rng.choice((0, 9))
    need = sum(-(-(p + n) // page) - h for p, n, h in zip(past, fresh, had))
    F = need + sum(had) + 7
    if seed % 4 == 1:
        width = max(1, width - 2)
    if seed % 8 == 3:
        capacity = max(0, capacity - 11)
    if seed % 8 == 7:
        fresh[0], past[B // 2] = -3, -(1 << 31)
    ids = list(range(F))
    rng.shuffle(ids)
    table = [[ids.pop() if j < had[b] else -1 for j in range(width)] for b in range(B)]
    ring = list(range(1000, 1000 + need + 5))
    rng.shuffle(ring)
    free = [rng.randint(-3, len(ring) + 3), len(ring) if seed % 2 == 0 else max(0, need - 2)]
    args = (past, fresh, ring, free, table, page, capacity)
    assert _plan(ma, *args) == _plan_reference(*args)


def test_plan_of_nothing(ma):
    r = _plan(ma, [], [], [], [0, 0], [], 16, 5)
    assert r["cu"] == [0] and r["slots"] == [-1] * 5 and r["left"] == [0, 0] and r["status"] == [0]
    r = _plan(ma, [3], [0], [1, 2], [1, 2], [[4, -1]], 16, 0)
    assert r["cu"] == [0, 0] and r["kv"] == [3] and r["left"] == [1, 2] and r["table"] == [[4, -1]]


def test_largest_plan(ma):
    B = ma.PLAN_MAX_B
    past, fresh = [i % 50 for i in range(B)], [i % 3 for i in range(B)]
    table, ring = [[i if j < 4 else -1 for j in range(5)] for i in range(B)], list(range(B))
    args = (past, fresh, ring, [5, B], table, 16, sum(fresh) + 1)
    assert _plan(ma, *args) == _plan_reference(*args)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("captured", [False, True])
def test_serving_loop(ma, captured, dtype):
    """Prompts in chunks, then token by token, requests of different lengths and one that joins late: every step plans,
    writes and attends, eagerly or as one captured graph that is replayed with the step's lengths; all outputs together
    are those of attention over the whole sequences."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    B, Hq, Hkv, d, page, blocks, pages, capacity = 3, 4, 2, 64, 16, 40, 64, 80
    steps = [(40, 17, 0), (30, 1, 0), (1, 1, 33), (1, 0, 1), (1, 1, 1), (7, 1, 1)]
    lens = [sum(s[i] for s in steps) for i in range(B)]
    seqs = [[torch.randn(n, h, d, generator=gen, device="cuda").to(DTYPES[dtype]) for h in (Hq, Hkv, Hkv)] for n in lens]
    ints = lambda *x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    kp, vp = (torch.full((pages, Hkv, page, d), math.nan, device="cuda", dtype=DTYPES[dtype]) for _ in range(2))
    past, fresh = torch.zeros(B, device="cuda", dtype=torch.int32), torch.zeros(B, device="cuda", dtype=torch.int32)
    ring = torch.randperm(pages, generator=gen, device="cuda").int()
    free, left, status = ints(60, pages), ints(0, 0), ints(0)
    table = torch.full((B, blocks), -1, device="cuda", dtype=torch.int32)
    cu, kv = ints(*[0] * (B + 1)), ints(*[0] * B)
    slots = torch.zeros(capacity, device="cuda", dtype=torch.int64)
    q, k, v = (torch.zeros(capacity, h, d, device="cuda", dtype=DTYPES[dtype]) for h in (Hq, Hkv, Hkv))
    out = torch.zeros_like(q)

    def step():
        ma.monarch_attn_paged_plan(past, fresh, ring, free, table, cu, kv, slots, left, status, page)
        ma.monarch_attn_paged_write(k, v, kp, vp, slots)
        ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table)
        past.copy_(kv)
        free.copy_(left)

    run = step
    if captured:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            step()  # no new tokens: sizes the stream's workspace, changes nothing
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        run = graph.replay
    done, got = [0] * B, [[] for _ in range(B)]
    for n in steps:
        fresh.copy_(ints(*n))
        for i, t in enumerate((q, k, v)):
            t.fill_(math.nan)
            rows = torch.cat([seqs[b][i][done[b] : done[b] + n[b]] for b in range(B)])
            t[: rows.shape[0]] = rows
        out.fill_(7.0)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        assert status.item() == 0 and bool((out[sum(n):] == 7).all())
        at = 0
        for b in range(B):
            got[b].append(out[at : at + n[b]].clone())
            at += n[b]
            done[b] += n[b]
    assert past.tolist() == lens and free.tolist()[1] == pages - sum(-(-x // page) for x in lens)
    for b in range(B):
        off = worst(torch.cat(got[b]), *attention(*seqs[b], True)["out"])
        assert off <= 1.0, (b, off)


def test_captured_split_call(ma):
    """A decoding call that is split over the keys, captured, and replayed with other contexts between eager calls."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    past = [3000, 100]
    seqs, kp, vp, table, kv = _cache([1, 1], past, 2, 64, 16, "bf16", gen)
    cu = starts([1, 1], "cuda")
    q = torch.randn(2, 8, 64, generator=gen, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table)
    for n in (3001, 1, 700, 2999):
        kv[0] = n
        q.copy_(torch.randn(2, 8, 64, generator=gen, device="cuda").bfloat16())
        want, _ = _attend(ma, q, kp, vp, cu, kv, table)
        graph.replay()
        with torch.cuda.stream(s):
            ma.monarch_attn_exact_paged_fwd(q, kp, vp, torch.zeros_like(q), cu, kv, table)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert worst(out[:1], *attention(q[:1], *(t[:n] for t in seqs[0]), True, n - 1)["out"]) <= 1.0


def test_capture_without_workspace_is_refused(ma):
    gen = torch.Generator(device="cuda").manual_seed(11)
    _, kp, vp, table, kv = _cache([1], [3000], 2, 64, 16, "bf16", gen)
    cu, q = starts([1], "cuda"), torch.randn(1, 8, 64, generator=gen, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    ma.monarch_attn_release_workspace()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(ma.MonarchAttnError) as e:
            ma.monarch_attn_exact_paged_fwd(q, kp, vp, out, cu, kv, table)
        out.add_(1)
    assert e.value.status == ma.MA_EUNSUPPORTED and "before capturing" in str(e.value)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_of_odd_lengths(ma, dtype):
    """Shares of the work that begin and end anywhere in 300 requests, some idle, some without a past."""
    gen = torch.Generator(device="cuda").manual_seed(71)
    new = [(0, 1, 1, 7, 40)[i % 5] for i in range(300)]
    past = [(i * 7919) % 3000 if i % 11 else 0 for i in range(300)]
    seqs, kp, vp, table, kv = _cache(new, past, 2, 64, 16, dtype, gen)
    q = torch.randn(sum(new) + 2, 6, 64, generator=gen, device="cuda").to(DTYPES[dtype])
    cu = starts(new, "cuda")
    out, lse = _attend(ma, q, kp, vp, cu, kv, table)
    _check(out, lse, q, cu, seqs, past)
    again = _attend(ma, q, kp, vp, cu, kv, table)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_decreasing_row_starts(ma):
    """Row starts that make more row tiles than the tensor's rows: what has no room is left out, and later calls are right."""
    gen = torch.Generator(device="cuda").manual_seed(72)
    seqs, kp, vp, table, kv = _cache([200], [2000], 2, 64, 16, "bf16", gen)
    q = torch.randn(200, 4, 64, generator=gen, device="cuda").bfloat16()
    cu = starts([200], "cuda")
    want = _attend(ma, q, kp, vp, cu, kv, table)
    bad = torch.tensor([0, 200] * 40 + [0], device="cuda", dtype=torch.int32)
    around = torch.full((600, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    ma.monarch_attn_exact_paged_fwd(q, kp, vp, around[200:400], bad, kv.repeat(80), table.repeat(80, 1))
    torch.cuda.synchronize()
    assert bool((around[:200] == 7).all()) and bool((around[400:] == 7).all())
    got = _attend(ma, q, kp, vp, cu, kv, table)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
