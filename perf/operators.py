"""Exact attention as language models train and serve with it: what is measured of it, and its plain form.

A model converted to MonarchAttention keeps exact attention in some of its
layers, and a decoder keeps it in all of them.  Four operators take it from
training to serving:

plan    (`monarch_attn_paged_plan`): from every request's cached and new tokens
        the row starts, key counts, block table and slot map of the next step,
        on the GPU, with pages taken from a ring of free ones.
write   (`monarch_attn_paged_write`): the new tokens' K and V rows into the paged
        cache, by slot.
packed  (`monarch_attn_exact_packed_fwd`): attention over whole prompts that lie
        one after another in one tensor, causal or not, with grouped heads.
train   (`exact_attention_packed`): the same as a training step, forward and
        gradient through torch's autograd.
paged   (`monarch_attn_exact_paged_fwd`): the new tokens of every request (one, or a
        chunk) over the keys and values of its pages.

A case: kind, the requests B, the shortest and longest number of new tokens
(new_lo, new_hi) and of tokens before them (past_lo, past_hi), rows behind
the last sequence (`spare`), heads Hq and Hkv, d, page, dtype, causal, and
`mix`, from which the lengths come.  Lengths are spread over the logarithm.
Queries and keys have unit variance, as they leave a norm over the head.
"""
import math
import random

import torch

own = False  # whether run() calls the framework's operators or their plain form

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(name, kind, B, new, past, Hq, Hkv, d, page, dtype, causal=True, spare=0, mix=1):
    return {"name": name, "kind": kind, "B": B, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
            "past_hi": past[1], "spare": spare, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "dtype": dtype,
            "causal": causal, "mix": mix}


def listed():
    return [
        # One decoding step of 64 requests: a token each, most of them on a page they already have.
        _case("plan_decode_64", "plan", 64, (1, 1), (128, 8192), 32, 8, 128, 16, "bf16"),
        # A step that admits prompts: 512 requests with up to 256 new tokens, some idle, in a padded batch.
        _case("plan_mixed_512", "plan", 512, (0, 256), (0, 4096), 32, 8, 128, 16, "bf16", spare=777),
        # The new rows of 64 decoding requests.
        _case("write_decode_64", "write", 64, (1, 1), (128, 1024), 32, 8, 128, 16, "bf16"),
        # The rows of prompts of 512 to 4096 tokens, cut from the layer's joint q, k, v projection.
        _case("write_prompts_16k", "write", 10, (512, 4096), (0, 64), 32, 8, 128, 16, "bf16"),
        # A small encoder on a ragged batch of 32 texts of up to 384 tokens without padding, no mask, one head a group.
        _case("packed_encoder_384_f16", "packed", 32, (16, 384), (0, 0), 12, 12, 64, 0, "f16", causal=False),
        # The prefill of one long prompt: 16384 tokens, the length of the long-sequence benchmark.
        _case("packed_causal_16k", "packed", 1, (16384, 16384), (0, 0), 16, 4, 128, 0, "bf16"),
        # Fine-tuning a decoder of 12 heads on documents of different lengths in fp32.
        _case("train_decoder_f32", "train", 6, (1, 1000), (0, 0), 12, 12, 64, 0, "f32"),
        # Training on packed documents in bf16, 16 query heads on 4 key heads of 128.
        _case("train_packed_8k", "train", 7, (100, 4096), (0, 0), 16, 4, 128, 0, "bf16"),
        # One request with a short context decodes one token: latency.
        _case("decode_one_f16", "paged", 1, (1, 1), (500, 500), 16, 4, 64, 16, "f16"),
        # A serving batch of 64 requests with contexts of 128 to 8192 tokens decodes one token each.
        _case("decode_64", "paged", 64, (1, 1), (128, 8192), 32, 8, 128, 16, "bf16"),
        # Two requests at the end of a very long context.
        _case("decode_long_128k", "paged", 2, (1, 1), (131000, 131000), 32, 8, 128, 64, "bf16"),
        # Chunked prefill: 8 requests add up to 512 tokens to contexts of up to 16384.
        _case("chunk_8_of_512", "paged", 8, (200, 512), (0, 16000), 32, 8, 128, 32, "bf16", spare=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng):
    top = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(("plan", "write", "packed", "packed", "train", "train", "paged", "paged", "paged"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f16", "f32"))
        Hkv = rng.choice((1, 2, 3, 4, 8, 12))
        Hq = Hkv * rng.choice((1, 1, 2, 4, 5, 8))
        d = rng.choice((32, 40, 64, 64, 80, 96, 128, 128))
        page = rng.choice((8, 16, 16, 32, 64, 128)) if kind in ("plan", "write", "paged") else 0
        past = (0, 0)
        if kind == "plan":
            B, new, past = _log_int(rng, 1, 1024), (rng.choice((0, 1)), _log_int(rng, 1, 300)), (0, _log_int(rng, 16, 8192))
        elif kind == "write":
            B, new, past = _log_int(rng, 1, 64), (1, _log_int(rng, 1, 500)), (0, 500)
        elif kind == "paged":
            n = 1 if rng.random() < 0.5 else _log_int(rng, 2, 600)
            B, new, past = _log_int(rng, 1, 96), (1, n), (0, _log_int(rng, 16, 20000))
        else:
            hi = _log_int(rng, 1, 6000)
            B, new = _log_int(rng, 1, max(1, min(64, 16000 // hi))), (rng.choice((0, 1, max(1, hi // 4))), hi)
        case = _case("", kind, B, new, past, Hq, Hkv, d, page, dtype, causal=kind == "paged" or rng.random() < 0.7,
                     spare=rng.choice((0, 0, 1, 100)), mix=rng.randrange(1 << 30))
        del case["name"]
        rows = (case["new_hi"] * Hq * (case["past_hi"] + case["new_hi"]) * B, B * Hkv * (new[1] + past[1]) * d)
        if work(case)["flops"] <= top / 3 and rows[0] < 2e9 and rows[1] < 4e8:
            return case


def _lengths(case):
    """(new, past) tokens of every request; the longest and the shortest are among them."""
    rng = random.Random(case["mix"])
    B = case["B"]
    new = [_log_int(rng, case["new_lo"], case["new_hi"]) for _ in range(B)]
    past = [_log_int(rng, case["past_lo"], case["past_hi"]) for _ in range(B)]
    if B > 1:
        new[rng.randrange(B)], past[rng.randrange(B)] = case["new_hi"], case["past_hi"]
        new[B - 1], past[B // 2] = case["new_lo"], case["past_lo"]
        new[0] = max(1, new[0])
    else:
        new, past = [case["new_hi"]], [case["past_hi"]]
    return new, past


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, device="cuda", dtype=dtype)


def _starts(new):
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    return at


def _pages(case, gen, new, past):
    """A ring of free pages, a block table in which the pages of the past are, and the same with all of them."""
    page, B = case["page"], case["B"]
    had = [-(-p // page) for p in past]
    all_ = [-(-(p + n) // page) for p, n in zip(past, new)]
    count = sum(all_) + max(8, sum(all_) // 8)
    ids = torch.randperm(count, generator=gen, device="cuda").to(torch.int32)
    width = max(all_) + 3
    j = torch.arange(width, device="cuda")[None]
    had, all_ = _ints(had)[:, None], _ints(all_)[:, None]
    first = all_.cumsum(0) - all_
    full = torch.where(j < all_, ids[(first + j).clamp(max=count - 1).long()], -1)
    return {"pages": count, "table": torch.where(j < had, full, -1).int(), "full": full.int()}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, Hq, Hkv, d, page = (case[x] for x in ("kind", "Hq", "Hkv", "d", "page"))
    dt = _DTYPES[case["dtype"]]
    new, past = _lengths(case)
    at = _starts(new)
    total = at[-1] + case["spare"]
    state = {"kind": kind, "causal": case["causal"], "page": page, "max_new": max(max(new), 1),
             "max_all": max(p + n for p, n in zip(past, new)), "cu": _ints(at)}
    if kind == "plan":
        paged = _pages(case, gen, new, past)
        ring = torch.randperm(paged["pages"], generator=gen, device="cuda").to(torch.int32)
        start = int(torch.randint(0, paged["pages"], (1,), generator=gen, device="cuda"))
        state |= {"past": _ints(past), "new": _ints(new), "ring": ring, "free": _ints([start, paged["pages"]]),
                  "table": paged["table"], "cu": torch.zeros(case["B"] + 1, device="cuda", dtype=torch.int32),
                  "kv": torch.zeros(case["B"], device="cuda", dtype=torch.int32),
                  "slots": torch.zeros(total, device="cuda", dtype=torch.int64),
                  "left": torch.zeros(2, device="cuda", dtype=torch.int32),
                  "status": torch.zeros(1, device="cuda", dtype=torch.int32)}
        return state
    if kind in ("write", "paged"):
        paged = _pages(case, gen, new, past)
        state |= {"k_pages": _randn(gen, paged["pages"], Hkv, page, d).to(dt),
                  "v_pages": _randn(gen, paged["pages"], Hkv, page, d).to(dt), "table": paged["full"],
                  "kv": _ints([p + n for p, n in zip(past, new)])}
    if kind == "train":
        leaf = [_randn(gen, total, h, d).to(dt) for h in (Hq, Hkv, Hkv, Hq)]
        state["qkv"], state["dout"] = tuple(x.requires_grad_() for x in leaf[:3]), leaf[3]
        return state
    joint = _randn(gen, total, (Hq + 2 * Hkv) * d).to(dt)  # what the layer's projection gives: q, k and v side by side
    state["qkv"] = tuple(x.unflatten(1, (-1, d)) for x in joint.split((Hq * d, Hkv * d, Hkv * d), dim=1))
    if kind == "write":
        pos = torch.cat([torch.arange(p, p + n, device="cuda") for p, n in zip(past, new)])
        who = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), _ints(new, torch.int64))
        slots = state["table"][who, pos // page].long() * page + pos % page
        state["slots"] = torch.cat((slots, torch.full((case["spare"],), -1, device="cuda", dtype=torch.int64)))
    else:
        state["out"] = torch.zeros(total, Hq, d, device="cuda", dtype=dt)
    return state


# ---- the plain forms ----

def _padded(cu, longest, total):
    """Rows [B, longest] of a packed tensor and which of them are real."""
    at = cu[:-1, None].long() + torch.arange(longest, device=cu.device)
    return at.clamp(max=total - 1), at < cu[1:, None]


def _heads(x, rows, Hkv):
    """[total, H, d] at rows [B, L] -> [B, Hkv, (H / Hkv) L, d] in fp32."""
    B, L = rows.shape
    H, d = x.shape[1:]
    x = x.float()[rows]  # [B, L, H, d]
    return x.view(B, L, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, H // Hkv * L, d)


def _unpacked(x, like, rows, real):
    """The inverse of _heads for the real rows; the other rows of the result are zero."""
    B, L = rows.shape
    H, d = like.shape[1:]
    x = x.view(B, -1, H * L // (x.shape[1] * L), L, d).permute(0, 3, 1, 2, 4).reshape(B * L, H, d)
    out = torch.zeros(like.shape[0] + 1, H, d, device=x.device, dtype=like.dtype)
    out[torch.where(real, rows, like.shape[0]).flatten()] = x.to(like.dtype)
    return out[:-1]


def _weights(q, k, see):
    """Softmax weights [B, Hkv, G Lq, Lk]; see [B, Lq, Lk].  A row that sees nothing has none."""
    B, Hkv, rows, d = q.shape
    Lq, Lk = see.shape[1:]
    s = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    s = s.view(B, Hkv, rows // Lq, Lq, Lk)
    see = see[:, None, None]
    s = torch.where(see, s, -math.inf)
    s = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e30))
    s = s / s.sum(-1, keepdim=True).clamp(min=1e-30)
    return s.view(B, Hkv, rows, Lk)


def _plain_attention(state):
    q, k, v = state["qkv"]
    rows, real = _padded(state["cu"], state["max_new"], q.shape[0])
    if state["kind"] == "paged":
        page, kv = state["page"], state["kv"]
        blocks = state["table"][:, : -(-state["max_all"] // page)].clamp(min=0).long()
        kh, vh = (x[blocks].float().transpose(1, 2).flatten(2, 3) for x in (state["k_pages"], state["v_pages"]))
        n = (state["cu"][1:] - state["cu"][:-1])[:, None, None]
        i = torch.arange(rows.shape[1], device=q.device)[None, :, None]
        j = torch.arange(kh.shape[2], device=q.device)[None, None, :]
        see = (j < kv[:, None, None]) & (i < n)
        see = see & (j <= kv[:, None, None] - n + i) if state["causal"] else see
    else:
        kh, vh = _heads(k, rows, k.shape[1]), _heads(v, rows, k.shape[1])
        see = real[:, :, None] & real[:, None, :]
        if state["causal"]:
            L = torch.arange(rows.shape[1], device=q.device)
            see = see & (L[:, None] >= L[None, :])
    qh = _heads(q, rows, kh.shape[1])
    p = _weights(qh, kh, see)
    out = _unpacked(torch.matmul(p, vh), q, rows, real)
    if state["kind"] != "train":
        return out
    # dP = dO V^T, dS = P (dP - sum P dP), dQ = s dS K, dK = s dS^T Q, dV = P^T dO
    gh = _heads(state["dout"], rows, kh.shape[1]) * real[:, None, None, :, None].expand(
        -1, kh.shape[1], q.shape[1] // kh.shape[1], -1, 1).reshape(*qh.shape[:3], 1)
    dv = torch.matmul(p.transpose(2, 3), gh)
    ds = torch.matmul(gh, vh.transpose(2, 3))
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * (1.0 / math.sqrt(q.shape[2]))
    dq, dk = torch.matmul(ds, kh), torch.matmul(ds.transpose(2, 3), qh)
    return out, _unpacked(dq, q, rows, real), _unpacked(dk, k, rows, real), _unpacked(dv, v, rows, real)


def _plain_write(state):
    slots, page = state["slots"], state["page"]
    real = (slots >= 0)[:, None, None]
    at = torch.where(slots >= 0, slots, slots[0])  # a row without a slot writes the first row again
    for x, pages in zip(state["qkv"][1:], (state["k_pages"], state["v_pages"])):
        pages[at // page, :, at % page] = torch.where(real, x, x[0])
    return state["k_pages"], state["v_pages"]


def _plain_plan(state):
    past, new, ring, free, table, page = (state[x] for x in ("past", "new", "ring", "free", "table", "page"))
    cu = torch.cat((torch.zeros_like(new[:1]), new.cumsum(0).int()))
    had, have = (past + page - 1) // page, (past + new + page - 1) // page
    need = have - had
    first = (need.cumsum(0) - need)[:, None]
    j = torch.arange(table.shape[1], device=past.device)[None]
    mine = (j >= had[:, None]) & (j < have[:, None])
    table = torch.where(mine, ring[(free[0] + first + j - had[:, None]) % ring.shape[0]], table)
    row = torch.arange(state["slots"].shape[0], device=past.device)
    who = torch.searchsorted(cu[1:].contiguous(), row.int(), right=True).clamp(max=past.shape[0] - 1)
    pos = (past[who] + row - cu[who]).clamp(min=0)
    slots = table[who, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    slots = torch.where(row < cu[-1], slots, -1)
    taken = need.sum()
    left = torch.stack(((free[0] + taken) % ring.shape[0], free[1] - taken)).int()
    return cu, past + new, table.int(), slots, left, torch.zeros_like(state["status"])


def run(state):
    kind = state["kind"]
    if own:
        import paper_2505_18698_amd as ma
        if kind == "plan":
            ma.monarch_attn_paged_plan(state["past"], state["new"], state["ring"], state["free"], state["table"],
                                       state["cu"], state["kv"], state["slots"], state["left"], state["status"],
                                       state["page"])
            return tuple(state[x] for x in ("cu", "kv", "table", "slots", "left", "status"))
        q, k, v = state["qkv"]
        if kind == "write":
            return ma.monarch_attn_paged_write(k, v, state["k_pages"], state["v_pages"], state["slots"])
        if kind == "paged":
            return ma.monarch_attn_exact_paged_fwd(q, state["k_pages"], state["v_pages"], state["out"], state["cu"],
                                                   state["kv"], state["table"], causal=state["causal"])[0]
        if kind == "packed":
            return ma.monarch_attn_exact_packed_fwd(q, k, v, state["out"], state["cu"], causal=state["causal"])[0]
        out = ma.exact_attention_packed(q, k, v, state["cu"], causal=state["causal"])
        return (out.detach(), *torch.autograd.grad(out, (q, k, v), state["dout"]))
    with torch.no_grad():
        if kind == "plan":
            return _plain_plan(state)
        if kind == "write":
            return _plain_write(state)
        return _plain_attention(state)


def work(case):
    """Every input read once and every output written once; of the products the pairs of query and key that see each
    other: two products forward, five more for the gradient."""
    new, past = _lengths(case)
    kind, Hq, Hkv, d, page = (case[x] for x in ("kind", "Hq", "Hkv", "d", "page"))
    size = 4 if case["dtype"] == "f32" else 2
    rows = sum(new)
    if kind == "plan":
        taken = sum(-(-(p + n) // page) - -(-p // page) for n, p in zip(new, past))
        return {"bytes": 8 * case["B"] + 8 * case["B"] + 8 * taken + 8 * (rows + case["spare"]) + 24, "flops": 0}
    if kind == "write":
        return {"bytes": rows * (8 + 4 * Hkv * d * size), "flops": 0}
    if case["causal"]:
        pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past))
    else:
        pairs = sum(n * (n + p) for n, p in zip(new, past))
    keys = sum(n + p for n, p in zip(new, past))
    reads = 2 * Hkv * d * size * keys + (4 * keys // page if page else 0)
    if kind == "train":  # q, k, v, out, dout and the gradients of q, k, v
        return {"bytes": rows * d * size * (4 * Hq + 4 * Hkv), "flops": 14 * d * Hq * pairs}
    return {"bytes": reads + 2 * rows * Hq * d * size, "flops": 4 * d * Hq * pairs}


# ---- the definition in 64 bits ----

def _exact_sequence(q, k, v, shift, causal, g):
    """q [n, H, d], k, v [L, Hkv, d] of one sequence in 64 bits, head by head; row i sees keys up to i + shift.
    With g, the gradient of <out, g> too."""
    n, H, d = q.shape
    G = H // k.shape[1]
    outs = [torch.zeros_like(x) for x in ((q, q, k, v) if g is not None else (q,))]
    step = max(1, int(2e8) // max(1, k.shape[0]))
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        for a in range(0, n, step):
            z = min(n, a + step)
            s = q[a:z, h] @ kh.T / math.sqrt(d)
            if causal:
                i = torch.arange(a, z, device=q.device)[:, None] + shift
                s = s.masked_fill(torch.arange(k.shape[0], device=q.device)[None] > i, -math.inf)
            p = torch.softmax(s, dim=-1)
            outs[0][a:z, h] = p @ vh
            if g is not None:
                dp = g[a:z, h] @ vh.T
                ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(d)
                outs[1][a:z, h] = ds @ kh
                outs[2][:, h // G] += ds.T @ q[a:z, h]
                outs[3][:, h // G] += p.T @ g[a:z, h]
    return outs


def exact(case, seed):
    state = prepare(case, seed)
    new, past = _lengths(case)
    at = _starts(new)
    kind, page = case["kind"], case["page"]
    if kind == "plan":
        ring, free = state["ring"].tolist(), state["free"].tolist()
        table, slots, first = state["table"].cpu().numpy(), [], free[0]
        for b, (n, p) in enumerate(zip(new, past)):
            for j in range(-(-p // page), -(-(p + n) // page)):
                table[b, j] = ring[first % len(ring)]
                first += 1
            slots += [int(table[b, x // page]) * page + x % page for x in range(p, p + n)]
        slots += [-1] * case["spare"]
        return (_ints(at), _ints([n + p for n, p in zip(new, past)]), torch.from_numpy(table), _ints(slots, torch.int64),
                _ints([first % len(ring), free[1] - (first - free[0])]), _ints([0]))
    if kind == "write":
        slots = state["slots"].tolist()
        caches = []
        for x, pages in zip(state["qkv"][1:], (state["k_pages"], state["v_pages"])):
            flat = pages.transpose(1, 2).reshape(-1, *x.shape[1:]).cpu()
            keep = [i for i, s in enumerate(slots) if s >= 0]
            flat[[slots[i] for i in keep]] = x.cpu()[keep]
            caches.append(flat.view(-1, page, *x.shape[1:]).transpose(1, 2).contiguous().double())
        return tuple(caches)
    q, k, v = (x.detach() for x in state["qkv"])
    if kind == "paged":
        outs = [torch.zeros(q.shape, device="cuda", dtype=torch.float64)]
    else:
        outs = [torch.zeros(x.shape, device="cuda", dtype=torch.float64) for x in ((q, q, k, v) if kind == "train" else (q,))]
    for b, (n, p) in enumerate(zip(new, past)):
        if n == 0:
            continue
        rows = slice(at[b], at[b + 1])
        if kind == "paged":
            ids = state["table"][b, : -(-(n + p) // page)].long()
            kb, vb = (x[ids].double().transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])[: n + p]
                      for x in (state["k_pages"], state["v_pages"]))
        else:
            kb, vb = k[rows].double(), v[rows].double()
        g = state["dout"][rows].double() if kind == "train" else None
        for dst, src in zip(outs, _exact_sequence(q[rows].double(), kb, vb, p, case["causal"], g)):
            dst[rows] = src
    return tuple(outs) if kind == "train" else outs[0]
