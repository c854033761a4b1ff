"""Operators of a decoder beside a converted encoder, for training and for beam search: what is measured of them, and
their plain forms.

An encoder whose attention is MonarchAttention feeds a decoder that reads its
states by cross attention; the decoder's own attention has rotary positions and
a paged cache, and answers are found by beam search:

cross   (`monarch_attn_exact_cross_fwd`): attention of packed queries to the
        encoder's states, of other lengths, packed or in a padded batch; and, with few
        queries a request, of the new tokens of its beams.
train   (`exact_cross_attention`): the same as a training step, forward and
        gradient through torch's autograd.
append  (`monarch_attn_paged_append`): the new tokens' queries and keys rotated
        by their positions, keys and values into the paged cache.
rotate  (`rotate_packed`): the rotation of packed sequences as a training step.
select  (`monarch_attn_beam_select`): the best continuations of a request's
        beams over the vocabulary.
reorder (`monarch_attn_paged_reorder`): the paged cache in the order of the beams chosen.

Lengths are spread over the logarithm and come from a case's `mix`. Queries and
keys have unit variance, as they leave a norm over the head.
"""
import math
import random

import torch

own = False  # whether run() calls the framework's operators or their plain form

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _cross(name, kind, B, n, keys, Hq, Hkv, d, dtype, padded=False, spare=0, mix=1):
    return {"name": name, "kind": kind, "B": B, "n_lo": n[0], "n_hi": n[1], "keys_lo": keys[0], "keys_hi": keys[1], "Hq": Hq,
            "Hkv": Hkv, "d": d, "dtype": dtype, "padded": padded, "spare": spare, "mix": mix}


def _rotary(name, kind, B, n, past, Hq, Hkv, d, rot, page, dtype, interleaved=False, spare=0, mix=1):
    return {"name": name, "kind": kind, "B": B, "n_lo": n[0], "n_hi": n[1], "past_lo": past[0], "past_hi": past[1], "Hq": Hq,
            "Hkv": Hkv, "d": d, "rot": rot, "page": page, "dtype": dtype, "interleaved": interleaved, "spare": spare, "mix": mix}


def _select(name, B, K, V, M, dtype, done=0.0, banned=0.0):
    return {"name": name, "kind": "select", "B": B, "K": K, "V": V, "M": M, "dtype": dtype, "done": done, "banned": banned}


def _reorder(name, B, K, tokens, Hkv, d, page, dtype, mix=1):
    return {"name": name, "kind": "reorder", "B": B, "K": K, "tokens_lo": tokens[0], "tokens_hi": tokens[1], "Hkv": Hkv, "d": d,
            "page": page, "dtype": dtype, "mix": mix}


def listed():
    return [
        # One text of 1000 tokens, four beams, a token each: latency.
        _cross("cross_one_f16", "cross", 1, (4, 4), (1000, 1000), 12, 12, 64, "f16"),
        # A decoding step of 32 requests with four beams each over encoded documents of 128 to 8192 tokens.
        _cross("cross_beams_32", "cross", 32, (4, 4), (128, 8192), 16, 16, 64, "bf16"),
        # Answers scored against a padded encoder batch: 24 texts of up to 2048 tokens.
        _cross("cross_scoring_padded", "cross", 24, (16, 512), (64, 2048), 12, 12, 64, "bf16", padded=True),
        # Fine-tuning a small encoder-decoder in fp32 on short and very short pairs.
        _cross("cross_train_f32", "train", 6, (1, 300), (1, 1000), 12, 12, 64, "f32"),
        # Training on long documents with short answers, 16 query heads on 4 key heads of 128.
        _cross("cross_train_8k", "train", 8, (100, 1024), (512, 8192), 16, 4, 128, "bf16"),
        # The new tokens of 64 decoding requests.
        _rotary("append_decode_64", "append", 64, (1, 1), (128, 8192), 32, 8, 128, 128, 16, "bf16"),
        # Prompts of 512 to 4096 tokens, cut from the layer's joint q, k, v projection.
        _rotary("append_prompts_16k", "append", 10, (512, 4096), (0, 64), 32, 8, 128, 128, 16, "bf16"),
        # A training step on packed documents, half of every head rotated, neighbouring columns as pairs.
        _rotary("rotate_train_8k", "rotate", 7, (100, 4096), (0, 0), 16, 4, 128, 64, 0, "bf16", interleaved=True, spare=33),
        # One request with four beams: latency.
        _select("select_one_f32", 1, 4, 32000, 8, "f32"),
        # 64 requests with eight beams, some of them done, some tokens banned.
        _select("select_64x8", 64, 8, 50001, 16, "bf16", done=0.1, banned=0.01),
        # The cache of one request with four beams.
        _reorder("reorder_one_f16", 1, 4, (1000, 1000), 12, 64, 16, "f16"),
        # 64 requests with eight beams, pages of 64 tokens.
        _reorder("reorder_64x8", 64, 8, (100, 4096), 8, 128, 64, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def _cost(w):
    return max(w["bytes"], w["flops"] / 100)


def draw(rng):
    top = max(_cost(work(c)) for c in listed())
    while True:
        kind = rng.choice(("cross", "cross", "cross", "train", "train", "append", "append", "rotate", "select", "select", "reorder"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f16", "f32"))
        Hkv = rng.choice((1, 2, 3, 4, 8, 12, 16))
        Hq = Hkv * rng.choice((1, 1, 1, 2, 4, 5))
        d = rng.choice((32, 40, 64, 64, 64, 80, 96, 128, 128))
        mix, spare = rng.randrange(1 << 30), rng.choice((0, 0, 1, 100))
        if kind in ("cross", "train"):
            few = kind == "cross" and rng.random() < 0.5
            n = rng.randint(1, 8) if few else _log_int(rng, 8, 2048)
            keys = _log_int(rng, 1, 12000)
            B = _log_int(rng, 1, max(1, min(64, 200000 // keys, 20000 // n)))
            case = _cross("", kind, B, (n if few else rng.choice((1, max(1, n // 4))), n), (rng.choice((0, 1, max(1, keys // 8))), keys),
                          Hq, Hkv, d, dtype, rng.random() < 0.3, spare, mix)
            size = B * Hq * n * keys
        elif kind in ("append", "rotate"):
            n = 1 if kind == "append" and rng.random() < 0.4 else _log_int(rng, 2, 4096)
            past = _log_int(rng, 1, 20000) if kind == "append" else 0
            rot = rng.choice([r for r in (8, 16, 24, 32, 64, 80, 96, 128, d, d) if r <= d])
            B = _log_int(rng, 1, max(1, min(128, 20000 // n, 200000 // max(1, past))))
            case = _rotary("", kind, B, (rng.choice((1, max(1, n // 4))), n), (0, past), Hq, Hkv, d, rot,
                           rng.choice((8, 16, 16, 32, 64)) if kind == "append" else 0, dtype, rng.random() < 0.5, spare, mix)
            size = B * (n + past) * Hkv * d
        elif kind == "select":
            K = rng.choice((1, 2, 3, 4, 5, 8, 16))
            V = _log_int(rng, 40, 200000)
            B = _log_int(rng, 1, 64)
            case = _select("", B, K, V, rng.choice((1, K, K, 2 * K, 2 * K)), dtype, rng.choice((0.0, 0.2)), rng.choice((0.0, 0.01, 0.5)))
            size = 4 * B * K * V
        else:
            K = rng.choice((1, 2, 3, 4, 5, 8, 16))
            tokens = _log_int(rng, 1, 4096)
            B = _log_int(rng, 1, max(1, min(64, 400000 // (tokens * K))))
            case = _reorder("", B, K, (1, tokens), Hkv, d, rng.choice((8, 16, 32, 64, 128)), dtype, mix)
            size = B * K * (tokens + 128) * Hkv * d
        del case["name"]
        if _cost(work(case)) <= top and size < 1e9:
            return case


def _spread(rng, B, lo, hi):
    """B lengths; the longest and the shortest are among them."""
    x = [_log_int(rng, lo, hi) for _ in range(B)]
    x[rng.randrange(B)] = hi
    if B > 1:
        x[rng.choice([i for i in range(B) if x[i] != hi] or [0])] = lo
    return x


def _lengths(case):
    """The two lengths of every sequence: (queries, keys), or (new, past) tokens."""
    rng = random.Random(case["mix"])
    what = "keys" if case["kind"] in ("cross", "train") else "past"
    return _spread(rng, case["B"], case["n_lo"], case["n_hi"]), _spread(rng, case["B"], case[what + "_lo"], case[what + "_hi"])


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, device="cuda", dtype=dtype)


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _key_rows(case, keys):
    """Where every sequence's keys start, and the rows of k and v in all."""
    width = case["keys_hi"]
    return [i * width for i in range(case["B"] + 1)] if case["padded"] else _starts(keys)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    dt = _DTYPES[case["dtype"]]
    state = {"kind": kind}
    if kind == "select":
        B, K, V, M = (case[x] for x in ("B", "K", "V", "M"))
        logits = _randn(gen, B, K, V) * 3
        if case["banned"]:
            logits = logits.masked_fill(torch.rand(B, K, V, generator=gen, device="cuda") < case["banned"], -math.inf)
        done = torch.rand(B, K, generator=gen, device="cuda") < case["done"]
        scores = -torch.rand(B, K, generator=gen, device="cuda").mul(8).cumsum(1)
        empty = lambda t: torch.zeros(B, M, device="cuda", dtype=t)  # noqa: E731
        return state | {"logits": logits.to(dt), "scores": scores, "done": done, "eos": 2, "scores_out": empty(torch.float32),
                        "tokens": empty(torch.int32), "parents": empty(torch.int32), "done_out": empty(torch.bool)}
    Hkv, d = case["Hkv"], case["d"]
    if kind == "reorder":
        B, K, page = case["B"], case["K"], case["page"]
        tokens = _spread(random.Random(case["mix"]), B, case["tokens_lo"], case["tokens_hi"])
        blocks = max(tokens) // page + 2
        table = torch.randperm(B * K * blocks, generator=gen, device="cuda").to(torch.int32).view(B * K, blocks)
        # full pages lie where an ancestor had them: the beams of a request share them; the started page is a beam's own
        full = (_ints(tokens) // page).repeat_interleave(K)[:, None]
        j = torch.arange(blocks, device="cuda")[None]
        shared = table.view(B, K, blocks)[torch.arange(B, device="cuda")[:, None, None],
                                          torch.randint(0, K, (B, K, blocks), generator=gen, device="cuda"), j[None]].view(B * K, blocks)
        return state | {"k_pages": _randn(gen, B * K * blocks, Hkv, page, d).to(dt), "v_pages": _randn(gen, B * K * blocks, Hkv, page, d).to(dt),
                        "table": torch.where(j < full, shared, table), "lens": _ints(tokens).repeat_interleave(K),
                        "parents": torch.randint(0, K, (B, K), generator=gen, device="cuda", dtype=torch.int32)}
    Hq = case["Hq"]
    new, other = _lengths(case)
    at = _starts(new)
    total = at[-1] + case["spare"]
    state["cu"] = _ints(at)
    if kind in ("cross", "train"):
        cu_k = _key_rows(case, other)
        rows = cu_k[-1] + case["spare"]
        state |= {"cu_k": _ints(cu_k), "k_lens": _ints(other) if case["padded"] else None, "longest": (max(new), max(max(other), 1))}
        q = _randn(gen, total, Hq, d).to(dt)
        if kind == "train":
            k, v = (_randn(gen, rows, Hkv, d).to(dt).requires_grad_() for _ in range(2))
            return state | {"qkv": (q.requires_grad_(), k, v), "dout": _randn(gen, total, Hq, d).to(dt)}
        joint = _randn(gen, rows, 2 * Hkv * d).to(dt)  # the projection of the encoder's states: k and v side by side
        k, v = (x.unflatten(1, (Hkv, d)) for x in joint.split(Hkv * d, dim=1))
        return state | {"qkv": (q, k, v), "out": torch.zeros(total, Hq, d, device="cuda", dtype=dt)}
    state["inv_freq"] = (10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])).float()
    state["interleaved"] = case["interleaved"]
    if kind == "rotate":
        leaf = [_randn(gen, total, h, d).to(dt) for h in (Hq, Hkv, Hq, Hkv)]
        return state | {"kv": None, "qk": tuple(x.requires_grad_() for x in leaf[:2]), "grads": tuple(leaf[2:])}
    page = case["page"]
    have = [-(-(p + n) // page) for p, n in zip(other, new)]
    ids = torch.randperm(sum(have) + 8, generator=gen, device="cuda")
    first = _ints(_starts(have), torch.int64)
    pos = torch.cat([torch.arange(p, p + n, device="cuda") for p, n in zip(other, new)])
    who = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), _ints(new, torch.int64))
    slots = ids[first[who] + pos // page] * page + pos % page
    joint = _randn(gen, total, (Hq + 2 * Hkv) * d).to(dt)  # what the layer's projection gives: q, k and v side by side
    return state | {"kv": _ints([p + n for p, n in zip(other, new)]), "page": page,
                    "slots": torch.cat((slots, torch.full((case["spare"],), -1, device="cuda", dtype=torch.int64))),
                    "qkv": tuple(x.unflatten(1, (-1, d)) for x in joint.split((Hq * d, Hkv * d, Hkv * d), dim=1)),
                    "q_out": torch.zeros(total, Hq, d, device="cuda", dtype=dt),
                    "k_pages": _randn(gen, len(ids), Hkv, page, d).to(dt), "v_pages": _randn(gen, len(ids), Hkv, page, d).to(dt)}


# ---- the plain forms ----

def _padded(first, lens, longest, total):
    """Rows [B, longest] of a packed tensor and which of them are real."""
    j = torch.arange(longest, device=first.device)
    return (first[:, None].long() + j).clamp(max=max(total - 1, 0)), j < lens[:, None]


def _heads(x, rows, real, Hkv):
    """[total, H, d] at rows [B, L] -> [B, Hkv, (H / Hkv) L, d] in fp32, zero where not real."""
    B, L = rows.shape
    H, d = x.shape[1:]
    if not x.shape[0]:
        return torch.zeros(B, Hkv, H // Hkv * L, d, device=x.device)
    x = x.float()[rows] * real[:, :, None, None]
    return x.view(B, L, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, H // Hkv * L, d)


def _unpacked(x, like, rows, real):
    """The inverse of _heads for the real rows; the other rows of the result are zero."""
    B, L = rows.shape
    H, d = like.shape[1:]
    x = x.view(B, -1, H * L // (x.shape[1] * L), L, d).permute(0, 3, 1, 2, 4).reshape(B * L, H, d)
    out = torch.zeros(like.shape[0] + 1, H, d, device=x.device, dtype=like.dtype)
    out[torch.where(real, rows, like.shape[0]).flatten()] = x.to(like.dtype)
    return out[:-1]


def _plain_cross(state):
    q, k, v = state["qkv"]
    cu, cu_k, k_lens = state["cu"], state["cu_k"], state["k_lens"]
    Hkv, d = k.shape[1:]
    s = 1.0 / math.sqrt(d)
    rows, real = _padded(cu[:-1], cu[1:] - cu[:-1], state["longest"][0], q.shape[0])
    rows_k, real_k = _padded(cu_k[:-1], cu_k[1:] - cu_k[:-1] if k_lens is None else k_lens, state["longest"][1], k.shape[0])
    qh, kh, vh = _heads(q, rows, real, Hkv), _heads(k, rows_k, real_k, Hkv), _heads(v, rows_k, real_k, Hkv)
    p = torch.where(real_k[:, None, None], torch.matmul(qh, kh.transpose(2, 3)) * s, -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True).clamp(min=-1e30))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = _unpacked(torch.matmul(p, vh), q, rows, real)
    if state["kind"] != "train":
        return out
    # dP = dO V^T, dS = P (dP - sum P dP), dQ = s dS K, dK = s dS^T Q, dV = P^T dO
    gh = _heads(state["dout"], rows, real, Hkv)
    dv = torch.matmul(p.transpose(2, 3), gh)
    ds = torch.matmul(gh, vh.transpose(2, 3))
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * s
    dq, dk = torch.matmul(ds, kh), torch.matmul(ds.transpose(2, 3), qh)
    return out, _unpacked(dq, q, rows, real), _unpacked(dk, k, rows_k, real_k), _unpacked(dv, v, rows_k, real_k)


def _angles(cu, kv, inv_freq, total):
    """cos and sin [total, pairs] of every row's position times the frequencies, and which rows are of a sequence."""
    row = torch.arange(total, device=cu.device)
    who = torch.searchsorted(cu[1:].contiguous(), row.int(), right=True).clamp(max=cu.shape[0] - 2)
    pos = row - cu[who] if kv is None else kv[who] - (cu[who + 1] - row)
    angle = pos.double()[:, None] * inv_freq.double()
    return angle.cos().float()[:, None], angle.sin().float()[:, None], (row < cu[-1])[:, None, None]


def _rotated(x, cos, sin, interleaved):
    pairs = cos.shape[-1]
    y = x.float()
    turned = y[..., : 2 * pairs]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., :pairs], turned[..., pairs:])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, y[..., 2 * pairs:]), -1).to(x.dtype)


def _plain_append(state):
    q, k, v = state["qkv"]
    cos, sin, real = _angles(state["cu"], state["kv"], state["inv_freq"], q.shape[0])
    state["q_out"].copy_(torch.where(real, _rotated(q, cos, sin, state["interleaved"]), state["q_out"]))
    slots, page = state["slots"], state["page"]
    at = torch.where(slots >= 0, slots, slots[0])  # a row without a slot writes the first row again
    for x, pages in ((_rotated(k, cos, sin, state["interleaved"]), state["k_pages"]), (v, state["v_pages"])):
        pages[at // page, :, at % page] = torch.where((slots >= 0)[:, None, None], x, x[0])
    return state["q_out"], state["k_pages"], state["v_pages"]


def _plain_rotate(state):
    cos, sin, real = _angles(state["cu"], None, state["inv_freq"], state["qk"][0].shape[0])
    there = [torch.where(real, _rotated(x, cos, sin, state["interleaved"]), 0) for x in state["qk"]]
    back = [torch.where(real, _rotated(x, cos, -sin, state["interleaved"]), 0) for x in state["grads"]]
    return (*there, *back)


def _plain_select(state):
    """In 64 bits: the order of candidates that are close to each other is part of the result."""
    x, scores, done = state["logits"].double(), state["scores"].double(), state["done"]
    B, K, V = x.shape
    M = state["tokens"].shape[1]
    top = x.amax(-1, keepdim=True).clamp(min=-1e300)
    cand = scores[..., None] + (x - top - (x - top).exp().sum(-1, keepdim=True).log())
    only = torch.where(torch.arange(V, device=x.device) == state["eos"], scores[..., None], -math.inf)
    cand = torch.where(done[..., None], only, cand)
    cand = torch.where(torch.isnan(cand), -math.inf, cand).view(B, K * V)
    # the M largest, of equal ones those with the lowest index
    least = cand.topk(M, dim=1).values[:, -1:]
    above, equal = cand > least, cand == least
    keep = above | (equal & (equal.cumsum(1) <= M - above.sum(1, keepdim=True)))
    index = torch.arange(K * V, device=x.device)
    at = torch.where(keep, K * V - index, 0).topk(M, dim=1).indices
    value, order = cand.gather(1, at).sort(dim=1, descending=True, stable=True)
    at = at.gather(1, order)
    parents, tokens = at // V, at % V
    return value.float(), tokens.int(), parents.int(), done.gather(1, parents) | (tokens == state["eos"])


def _plain_reorder(state):
    table, parents, lens, k, v = (state[x] for x in ("table", "parents", "lens", "k_pages", "v_pages"))
    B, K = parents.shape
    page, blocks = k.shape[2], table.shape[1]
    source = (torch.arange(B, device=table.device)[:, None] * K + parents).flatten()
    full = (lens // page)[:, None]
    r = torch.arange(page, device=table.device)
    mine = table.gather(1, full.long())[:, 0].long()
    theirs = mine[source]
    keep = (r < (lens % page)[:, None])[:, None, :, None]
    for x in (k, v):
        x[mine] = torch.where(keep, x[theirs], x[mine])
    table.copy_(torch.where(torch.arange(blocks, device=table.device) < full, table[source], table))
    return k, v, table


def run(state):
    kind = state["kind"]
    if own:
        import paper_2505_18698_amd as ma
        if kind == "cross":
            return ma.monarch_attn_exact_cross_fwd(*state["qkv"], state["out"], state["cu"], state["cu_k"], state["k_lens"])[0]
        if kind == "train":
            out = ma.exact_cross_attention(*state["qkv"], state["cu"], state["cu_k"], state["k_lens"])
            return (out.detach(), *torch.autograd.grad(out, state["qkv"], state["dout"]))
        if kind == "append":
            return ma.monarch_attn_paged_append(*state["qkv"], state["q_out"], state["k_pages"], state["v_pages"], state["inv_freq"],
                                                state["cu"], state["kv"], state["slots"], interleaved=state["interleaved"])
        if kind == "rotate":
            out = ma.rotate_packed(*state["qk"], state["inv_freq"], state["cu"], interleaved=state["interleaved"])
            return (*(x.detach() for x in out), *torch.autograd.grad(out, state["qk"], state["grads"]))
        if kind == "select":
            return ma.monarch_attn_beam_select(state["logits"], state["scores"], state["scores_out"], state["tokens"], state["parents"],
                                               done=state["done"], done_out=state["done_out"], eos=state["eos"])
        return ma.monarch_attn_paged_reorder(state["k_pages"], state["v_pages"], state["table"], state["parents"], state["lens"])
    with torch.no_grad():
        plain = {"cross": _plain_cross, "train": _plain_cross, "append": _plain_append, "rotate": _plain_rotate, "select": _plain_select,
                 "reorder": _plain_reorder}
        return plain[kind](state)


def work(case):
    """Every input read once and every output written once; of cross attention the pairs of query and key: two products
    forward, five more for the gradient."""
    kind = case["kind"]
    size = 4 if case["dtype"] == "f32" else 2
    if kind == "select":
        rows, out = case["B"] * case["K"], case["B"] * case["M"]
        return {"bytes": rows * (case["V"] * size + 5) + 13 * out, "flops": 0}
    Hkv, d = case["Hkv"], case["d"]
    if kind == "reorder":  # of parents at random (K - 1) / K differ from the beam itself, and 1 - (1 - 1 / K)^K of the beams are parents
        B, K, page = case["B"], case["K"], case["page"]
        tokens = _spread(random.Random(case["mix"]), B, case["tokens_lo"], case["tokens_hi"])
        moved = K - 1 + K * (1 - (1 - 1 / K) ** K) if K > 1 else 0
        return {"bytes": int(sum(moved * (4 * (n // page) + 2 * (n % page) * Hkv * d * size) for n in tokens)) + 8 * B * K, "flops": 0}
    Hq = case["Hq"]
    new, other = _lengths(case)
    n = sum(new)
    if kind == "append":
        return {"bytes": n * (2 * (Hq + 2 * Hkv) * d * size + 8) + 8 * case["B"], "flops": 0}
    if kind == "rotate":
        return {"bytes": (n + case["spare"]) * 4 * (Hq + Hkv) * d * size, "flops": 0}
    pairs, keys = sum(a * b for a, b in zip(new, other)), sum(other)
    if kind == "train":  # q, out, dout, dq; k, v, dk, dv
        return {"bytes": 4 * d * size * (n * Hq + keys * Hkv), "flops": 14 * d * Hq * pairs}
    return {"bytes": 2 * d * size * (n * Hq + keys * Hkv), "flops": 4 * d * Hq * pairs}


# ---- the definition in 64 bits ----

def _exact_cross(case, state):
    q, k, v = (x.detach() for x in state["qkv"])
    new, keys = _lengths(case)
    at, at_k = _starts(new), _key_rows(case, keys)
    G, scale = case["Hq"] // case["Hkv"], case["d"] ** -0.5
    outs = [torch.zeros(x.shape, device="cuda", dtype=torch.float64) for x in ((q, q, k, v) if case["kind"] == "train" else (q,))]
    for a, n, b, L in zip(at, new, at_k, keys):
        if n == 0 or L == 0:
            continue
        for h in range(case["Hq"]):
            Q, K, V = q[a:a + n, h].double(), k[b:b + L, h // G].double(), v[b:b + L, h // G].double()
            P = torch.softmax(Q @ K.T * scale, 1)
            O = P @ V
            outs[0][a:a + n, h] = O
            if case["kind"] == "train":
                g = state["dout"][a:a + n, h].double()
                dS = P * (g @ V.T - (g * O).sum(1, keepdim=True)) * scale
                outs[1][a:a + n, h] = dS @ K
                outs[2][b:b + L, h // G] += dS.T @ Q
                outs[3][b:b + L, h // G] += P.T @ g
    return tuple(outs) if case["kind"] == "train" else outs[0]


def _turn(x, pos, inv_freq, interleaved, sign=1.0):
    """Rotation as a product of complex numbers."""
    pairs = inv_freq.shape[0]
    y = x.detach().double().clone()
    phase = sign * torch.tensor(pos, device=y.device, dtype=torch.float64)[:, None, None] * inv_freq.double()
    turn = torch.polar(torch.ones_like(phase), phase)
    re, im = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    z = torch.complex(y[..., re], y[..., im]) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind in ("cross", "train"):
        return _exact_cross(case, state)
    if kind == "select":
        eos, M = state["eos"], case["M"]
        outs = [[], [], [], []]
        for x, score, done in zip(state["logits"], state["scores"].double(), state["done"].tolist()):
            cand = score[:, None] + torch.log_softmax(x.double(), dim=1)
            for k, ended in enumerate(done):
                if ended:
                    cand[k] = -math.inf
                    cand[k, eos] = score[k]
            value, at = cand.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).flatten().sort(dim=0, descending=True, stable=True)
            parent, token = at[:M] // case["V"], at[:M] % case["V"]
            for o, y in zip(outs, (value[:M], token, parent, torch.tensor(done, device="cuda")[parent] | (token == eos))):
                o.append(y)
        value, token, parent, ended = (torch.stack(o) for o in outs)
        return value, token.int(), parent.int(), ended
    if kind == "reorder":
        table, parents, lens = (state[x].tolist() for x in ("table", "parents", "lens"))
        K, page = case["K"], case["page"]
        old = [row[:] for row in table]
        caches = [state["k_pages"], state["v_pages"]]
        new = [x.double() for x in caches]
        for b in range(case["B"]):
            full, rows = divmod(lens[b * K], page)
            for c in range(K):
                source = b * K + parents[b][c]
                table[b * K + c][:full] = old[source][:full]
                for x, y in zip(caches, new):
                    y[old[b * K + c][full], :, :rows] = x[old[source][full], :, :rows].double()
        return (*new, _ints(table))
    new, past = _lengths(case)
    pos = [p + i for p, n in zip(past, new) for i in range(n)]
    turn = lambda x, sign=1.0: _turn(x[: len(pos)], pos, state["inv_freq"], case["interleaved"], sign)  # noqa: E731
    blank = lambda x, y: torch.cat((y, torch.zeros(x.shape[0] - len(pos), *x.shape[1:], device="cuda", dtype=torch.float64)))  # noqa: E731
    if kind == "rotate":
        return tuple(blank(x, turn(x, s)) for s, xs in ((1.0, state["qk"]), (-1.0, state["grads"])) for x in xs)
    q, k, v = state["qkv"]
    slots, page = state["slots"][: len(pos)], case["page"]
    caches = []
    for x, pages in ((turn(k), state["k_pages"]), (v[: len(pos)].double(), state["v_pages"])):
        flat = pages.double().transpose(1, 2).flatten(0, 1)
        flat[slots] = x
        caches.append(flat.unflatten(0, (-1, page)).transpose(1, 2).contiguous())
    return blank(q, turn(q)), *caches
