"""A decoder's operators where offsets pass 2^31 elements: far rows of k and v, far pages, far rows of logits."""
import pytest
import torch

from sequence_reference import attention, starts, worst

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ma():
    assert torch.cuda.is_available(), "no GPU visible"
    import paper_2505_18698_amd as lib

    return lib


def test_cross_attention_to_far_rows(ma):
    """600000 rows 4096 elements apart (2.4e9 elements): the last sequences, forward and gradient of contiguous k."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    keys, lens = [299000, 300500, 70, 430], [3, 0, 40, 5]
    cu, cu_k = starts(lens, "cuda"), starts(keys, "cuda")
    joint = torch.empty(sum(keys), 4096, device="cuda", dtype=torch.bfloat16)
    k, v = (x.unflatten(1, (-1, 64)) for x in (joint[:, :128], joint[:, 3968:]))
    far = int(cu_k[2])
    for t in (k, v):
        t[far:] = torch.randn(500, 2, 64, generator=gen, device="cuda").bfloat16()
        t[:299000] = 0.5
        t[299000:far] = float("nan")  # no query reads them
    q, dout = (torch.randn(48, 4, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    out, lse, rest = torch.zeros_like(q), torch.zeros(4, 48, device="cuda"), torch.zeros_like(q)
    ma.monarch_attn_exact_cross_fwd(q, k, v, out, cu, cu_k, None, lse, rest)
    dq, dk, dv = torch.zeros_like(q), *(torch.empty(sum(keys), 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ma.monarch_attn_exact_cross_bwd(q, k, v, out, lse, dout, dq, dk, dv, cu, cu_k, None, rest)
    torch.cuda.synchronize()
    assert bool((out[:3] == 0.5).all())
    for a, n, b, L in ((3, 40, far, 70), (43, 5, far + 70, 430)):
        rows, there = slice(a, a + n), slice(b, b + L)
        ref = attention(q[rows], k[there], v[there], False, 0, dout[rows])
        for name, x in (("out", out[rows]), ("dq", dq[rows]), ("dk", dk[there]), ("dv", dv[there])):
            assert worst(x, *ref[name]) <= 1.0, name
    assert bool((dk[299000:far] == 0).all()) and bool((dv[299000:far] == 0).all())


def test_append_and_reorder_of_far_pages(ma):
    """140000 pages of 8 heads of 16 rows of 128 columns: 2.3e9 elements a cache."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    pages = 140000
    k_pages, v_pages = (torch.zeros(pages, 8, 16, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.tensor([[pages - 1], [pages - 2], [3], [pages - 4]], dtype=torch.int32, device="cuda")
    lens = torch.full((4,), 6, dtype=torch.int32, device="cuda")
    cu, freq = starts([6] * 4, "cuda"), torch.ones(64, device="cuda")
    q, k, v = (torch.randn(24, h, 128, generator=gen, device="cuda").bfloat16() for h in (8, 8, 8))
    slots = (table.long() * 16 + torch.arange(6, device="cuda")).flatten()
    q_out, k_out = torch.zeros_like(q), torch.zeros_like(k)
    ma.monarch_attn_paged_append(q, k, v, q_out, k_pages, v_pages, freq, cu, lens, slots)
    ma.monarch_attn_rotate(q, k, torch.zeros_like(q), k_out, freq, cu, lens)
    rows = lambda cache: cache[table[:, 0].long()][:, :, :6].transpose(1, 2).flatten(0, 1)  # noqa: E731
    assert torch.equal(rows(k_pages), k_out) and torch.equal(rows(v_pages), v)
    parents = torch.tensor([[1, 1], [0, 0]], dtype=torch.int32, device="cuda")
    ma.monarch_attn_paged_reorder(k_pages, v_pages, table, parents, lens)
    at = torch.cat([torch.arange(6, device="cuda") + 6 * i for i in (1, 1, 2, 2)])
    assert torch.equal(rows(k_pages), k_out[at]) and torch.equal(rows(v_pages), v[at])
    used = torch.zeros(pages, dtype=torch.bool, device="cuda")
    used[table[:, 0].long()] = True
    assert int((k_pages.flatten(1) != 0).any(1).sum()) == 4 and bool((k_pages.flatten(1) != 0).any(1)[used].all())


def test_selection_of_far_rows(ma):
    """36 requests of 32 beams, rows 2^21 elements apart (2.4e9 elements)."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    B, K, V, M = 36, 32, 5000, 8
    whole = torch.empty(B, K, 1 << 21, device="cuda", dtype=torch.bfloat16)
    x = whole[:, :, 7: 7 + V]
    x.copy_(torch.randn(B, K, V, generator=gen, device="cuda"))
    scores = -torch.arange(float(K), device="cuda").expand(B, K).contiguous()
    out, tokens, parents = torch.zeros(B, M, device="cuda"), *(torch.zeros(B, M, dtype=torch.int32, device="cuda") for _ in range(2))
    ma.monarch_attn_beam_select(x, scores, out, tokens, parents)
    cand = scores.double()[..., None] + torch.log_softmax(x.double(), -1)
    best = cand.flatten(1).topk(M, dim=1).values
    got = cand.flatten(1).gather(1, parents.long() * V + tokens.long())
    assert float((got - best).abs().max()) <= 2.0 ** -16 and float((out - best).abs().max()) <= 2.0 ** -16 + 2.0 ** -24 * 32
