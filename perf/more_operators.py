"""Performance cases of the operators around the paged cache: rotation, a bounded cache, beam search.

``rotate``  norms of the query and key heads with the rotation by position, between the adapter apply and the cache.
``score``   the weight that a step's queries give to each cached token, added to what the token has gathered.
``evict``   each sequence cut to a budget of tokens by gathered weight; the kept ones' k, v and marks come back.
``select``  the best continuations over a request's beams and the vocabulary.
``copy``    the last pages of beams that go on, copied in every layer, and read back.

With ``own`` the calls go through ``paper_2608_03579_amd.salt``; without it the same operators are written with
elementary torch operations in 32 bits (angles, log-sum-exp and the order of candidates in 64).  torch owns the
activations; all work goes to torch's current stream.

A case is a dict of plain values:

``T, heads, kv_heads, dim, rot, inter, norm, far``
    rotate: tokens, head layout, values of a head that are rotated, pairs side by side or half a head apart,
    with norms or without, and the largest position.
``seqs, new, own, even, groups, prefix, page, fmt``
    a batch over the cache: sequences, new tokens of each (``even``: all have ``new``, else 1 to ``new``), their own
    tokens (``even``: ``own`` each, else spread over the logarithm up to it), domains with a shared prefix of up to
    ``prefix`` tokens (0: none), tokens to a page and the cache's format.
``window``
    score: only the last ``window`` new tokens of a sequence count (0: all).
``keep, recent``
    evict: the budget, and how many of the newest tokens stay whatever their weight.
``reqs, width, vocab, n_out, first``
    select: requests, beams of each, vocabulary, continuations to return, and whether only the first beam is live.
``pairs, layers, tokens``
    copy: pages copied, layers, and the most tokens in use of a page.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one user's next token: the smallest call there is
        dict(name="rotate_8b_T1", kind="rotate", dtype="bf16", T=1, heads=32, kv_heads=8, dim=128, rot=128,
             inter=False, norm=True, far=8191),
        # a chunk of prefill far into long texts, fp32, half of each head rotated in neighbouring pairs
        dict(name="rotate_half_f32_T203", kind="rotate", dtype="f32", T=203, heads=20, kv_heads=4, dim=64, rot=32,
             inter=True, norm=False, far=1000003),
        # a full prefill batch
        dict(name="rotate_8b_T8192", kind="rotate", dtype="bf16", T=8192, heads=32, kv_heads=8, dim=128, rot=128,
             inter=False, norm=True, far=131071),
        # a decode step of 64 users with up to 4096 tokens each
        dict(name="score_8b_decode_T64", kind="score", dtype="bf16", fmt="e4m3", heads=32, kv_heads=8, dim=128,
             page=64, seqs=64, new=1, own=4096, even=False, groups=0, prefix=0, window=0),
        # drafted tokens of users behind their domains' prompts, fp32, small pages
        dict(name="score_drafts_f32_int8", kind="score", dtype="f32", fmt="int8", heads=20, kv_heads=4, dim=64,
             page=16, seqs=23, new=4, own=1500, even=False, groups=5, prefix=1531, window=0),
        # two long prompts, every token of them counted: the largest
        dict(name="score_prompts_8b_T8192", kind="score", dtype="bf16", fmt="e4m3", heads=32, kv_heads=8, dim=128,
             page=64, seqs=2, new=4096, own=4096, even=True, groups=0, prefix=0, window=0),
        # prompts cut to their budget after the prefill
        dict(name="evict_8b_prompts", kind="evict", dtype="bf16", fmt="e4m3", heads=32, kv_heads=8, dim=128, page=64,
             seqs=16, own=8192, even=True, keep=512, recent=64),
        # every sequence one token over its budget, in fp32 with a small cache
        dict(name="evict_decode_f32_int8", kind="evict", dtype="f32", fmt="int8", heads=20, kv_heads=4, dim=64, page=16,
             seqs=40, own=257, even=True, keep=256, recent=32),
        # one request of four beams
        dict(name="select_w4", kind="select", dtype="bf16", reqs=1, width=4, vocab=128256, n_out=8, first=False),
        # 64 requests of eight beams, twice as many continuations as beams
        dict(name="select_r64_w8", kind="select", dtype="bf16", reqs=64, width=8, vocab=128256, n_out=16, first=False),
        # four beams' last pages, half full
        dict(name="copy_w4", kind="copy", dtype="bf16", fmt="e4m3", heads=32, kv_heads=8, dim=128, page=64, pairs=4,
             layers=16, tokens=40),
        # 128 beams' last pages in 28 layers
        dict(name="copy_w128", kind="copy", dtype="bf16", fmt="e4m3", heads=24, kv_heads=8, dim=128, page=64, pairs=128,
             layers=28, tokens=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), _cost(c))
    while True:
        kind = rng.choice(["rotate", "rotate", "score", "score", "score", "evict", "evict", "select", "select", "copy"])
        c = dict(kind=kind, dtype="f32" if rng.random() < 0.3 else "bf16")
        if kind == "select":
            width = rng.choice([1, 2, 3, 4, 5, 8, rng.randint(1, 16)])
            c.update(reqs=_log_int(rng, 1, 64), width=width, vocab=rng.choice([32000, 128256, _log_int(rng, 257, 200000)]),
                     n_out=min(64, width * rng.choice([1, 2, 2])), first=rng.random() < 0.2)
        else:
            kv = rng.choice([1, 2, 4, 8, 8])
            c.update(heads=kv * rng.choice([1, 3, 4, 5, 8]), kv_heads=kv, dim=rng.choice([64, 128, 128]))
        if kind == "rotate":
            c["dim"] = rng.choice([64, 128, 128, 256, 96, 80])
            c.update(T=_log_int(rng, 1, 8192), rot=rng.choice([c["dim"], c["dim"], 16 * rng.randint(1, c["dim"] // 16)]),
                     inter=rng.random() < 0.4, norm=rng.random() < 0.6, far=_log_int(rng, 1, 1 << 22))
        elif kind == "score":
            c.update(fmt=rng.choice(["e4m3", "e4m3", "int8"]), page=rng.choice([16, 32, 64, 128]), even=rng.random() < 0.3)
            if rng.random() < 0.6:
                new, seqs, top = rng.choice([1, 1, 1, rng.randint(2, 8)]), _log_int(rng, 1, 64), _log_int(rng, 16, 4096)
            else:
                new, seqs, top = _log_int(rng, 1, 2048), _log_int(rng, 1, 8), _log_int(rng, 1, 2048)
            groups = rng.choice([0, 0, 1, rng.randint(1, 8)])
            c.update(seqs=seqs, new=new, own=max(new, top), groups=groups, prefix=_log_int(rng, 1, 2048) if groups else 0,
                     window=rng.choice([0, 0, _log_int(rng, 1, 64)]))
        elif kind == "evict":
            top = _log_int(rng, 16, 8192)
            keep = max(1, min(top - 1, rng.choice([top - 1, _log_int(rng, 1, top)])))
            c.update(fmt=rng.choice(["e4m3", "e4m3", "int8"]), page=rng.choice([16, 32, 64, 128]), seqs=_log_int(rng, 1, 64),
                     own=top, even=rng.random() < 0.4, keep=keep, recent=rng.randint(0, keep))
        elif kind == "copy":
            page = rng.choice([16, 32, 64, 128])
            c.update(fmt=rng.choice(["e4m3", "e4m3", "int8"]), page=page, pairs=_log_int(rng, 1, 128),
                     layers=_log_int(rng, 1, 32), tokens=rng.randint(1, page))
        # (the plain form pads: it has to fit too)
        if _cost(c) <= most[kind] and _padded(c) <= 3e9:
            return c


# ---------------------------------------------------------------------------
# the batch of a case
# ---------------------------------------------------------------------------
def _batch(case, seed):
    """Per sequence its new tokens, its own tokens and its domain (-1: none); per domain its prefix's tokens.
    The batches of all seeds have the same sequences, in another order."""
    rng = np.random.default_rng([2608, 3591])
    if case["kind"] == "copy":
        n = case["pairs"]
        length = rng.integers(1, case["tokens"] + 1, size=n).astype(np.int32)
        return length, length, np.full(n, -1, np.int32), np.zeros(0, np.int32)
    n, most = case["seqs"], case["own"]
    new = case["new"] if case["kind"] == "score" else 0
    if case["even"]:
        q_len, length = np.full(n, new), np.full(n, most)
    else:
        q_len = rng.integers(1, new + 1, size=n) if new else np.zeros(n, int)
        length = np.exp(rng.uniform(0, math.log(most) if most > 1 else 0.0, size=n)).astype(np.int64)
        length = np.maximum(np.maximum(length, q_len), 1)
    rng = np.random.default_rng([2608, 3591, int(seed)])
    order = rng.permutation(n)
    q_len, length = q_len[order], length[order]
    groups = case.get("groups", 0)
    prefix = rng.integers(case["prefix"] // 2 + 1, case["prefix"] + 1, size=groups) if groups else np.zeros(0, int)
    group = rng.integers(-1, groups, size=n) if groups else np.full(n, -1)
    return q_len.astype(np.int32), length.astype(np.int32), group.astype(np.int32), prefix.astype(np.int32)


def _pages(case, seed):
    """Page tables in a random order of the pool's pages: (first page reference of each holder, the pages), the
    domains' prefixes before the sequences, and the pool's pages."""
    _, length, _, prefix = _batch(case, seed)
    tokens = np.concatenate([prefix, length])
    n = (tokens + case["page"] - 1) // case["page"]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(off[-1]) * (2 if case["kind"] == "copy" else 1) + 3
    pages = np.random.default_rng([2608, 3592, int(seed)]).permutation(total).astype(np.int32)
    return off, pages, total


def _slots(case, off, pages, tokens):
    """Where each holder's tokens lie in the pool, in order."""
    page, at = case["page"], [np.zeros(0, np.int64)]
    for i, n in enumerate(tokens):
        j = np.arange(n)
        at.append(pages[off[i] + j // page].astype(np.int64) * page + j % page)
    return np.concatenate(at)


def _padded(case):
    """Floats of the plain form's largest tensors."""
    if case["kind"] == "rotate":
        return 0
    if case["kind"] == "select":
        return 6 * case["reqs"] * case["width"] * case["vocab"]
    q_len, length, group, prefix = _batch(case, 0)
    kd = case["kv_heads"] * case["dim"]
    if case["kind"] == "copy":
        return 2 * kd * case["pairs"] * case["tokens"] * case["layers"]
    keys = int(length.max()) + (int(prefix.max()) if len(prefix) else 0)
    return kd * len(length) * keys + 3 * int(q_len.max()) * len(length) * case["heads"] * keys


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed, key):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + key * 7919 + 31) % (1 << 62))
    return g


def _normal(case, seed, key, shape, std=1.0, uneven=False):
    """Seeded N(0, std^2) on the GPU; `uneven`: a few of the last axis's columns are several times larger, as in activations."""
    g = _gen(seed, key)
    v = torch.randn(shape, generator=g, device="cuda")
    if uneven:
        n = shape[-1]
        v[..., torch.randint(0, n, (max(1, n // 64),), generator=g, device="cuda")] *= 8.0
    return (v * std).to(_DTYPE[case["dtype"]])


def _history(case, seed, layer=0):
    """k and v of every token of the prefixes and the sequences, holder after holder: [tokens][kv_heads][dim]."""
    _, length, _, prefix = _batch(case, seed)
    shape = (int(prefix.sum() + length.sum()), case["kv_heads"], case["dim"])
    return _normal(case, seed, 100 + 2 * layer, shape, uneven=True), _normal(case, seed, 101 + 2 * layer, shape)


def _marks(case, seed):
    """Gathered weight and position of every own token and kv head: heavy-tailed weights, positions with the gaps that
    earlier evictions left, in an order of their own for each head."""
    _, length, _, _ = _batch(case, seed)
    n, hk = int(length.sum()), case["kv_heads"]
    score = torch.exp(torch.randn((n, hk), generator=_gen(seed, 5), device="cuda") * 2 - 3)
    rng = np.random.default_rng([2608, 3593, int(seed)])
    pos = [np.stack([rng.permutation(3 * int(m))[: int(m)] for _ in range(hk)], 1) for m in length]
    return score, torch.from_numpy(np.concatenate(pos).astype(np.int32)).cuda()


def _frequencies(case):
    return 10000.0 ** (-np.arange(0, case["rot"], 2, dtype=np.float64) / case["rot"])


def _positions(case, seed):
    return torch.randint(0, case["far"] + 1, (case["T"],), generator=_gen(seed, 6), device="cuda", dtype=torch.int32)


def _step_positions(case, seed):
    """Positions of a step's new tokens: behind everything that the marks hold."""
    q_len, length, _, _ = _batch(case, seed)
    pos = [3 * int(m) + np.arange(int(q)) for q, m in zip(q_len, length)]
    return torch.from_numpy(np.concatenate(pos).astype(np.int32)).cuda()


def _beam_scores(case, seed):
    v = -torch.rand((case["reqs"], case["width"]), generator=_gen(seed, 8), device="cuda") * 12
    if case["first"]:
        v[:, 1:] = -math.inf
    return v.reshape(-1)


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _quantise_kv(x, fmt):
    """(codes, scale) of token-head vectors."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    if fmt == "int8":
        scale = (amax * (1.0 / 127.0)).clamp_min(2.0 ** -100)
        return torch.round(x * scale.reciprocal()).clamp(-127, 127).to(torch.int8), scale
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, (e - 9 + (m > 0.875)).clamp_min(-100), torch.zeros_like(e))
    scale = torch.ldexp(torch.ones_like(amax), e)
    return (x * torch.ldexp(torch.ones_like(amax), -e)).to(torch.float8_e4m3fn), scale


def _plain_cache(case, seed, layer=0):
    """The cache as it stands before the call: codes [pages x page][kv_heads][dim] and scales of k and of v."""
    off, pages, total = _pages(case, seed)
    _, length, _, prefix = _batch(case, seed)
    rows = torch.from_numpy(_slots(case, off, pages, np.concatenate([prefix, length]))).cuda()
    cache = []
    for x in _history(case, seed, layer):
        q, sc = _quantise_kv(x, case["fmt"])
        codes = torch.zeros(total * case["page"], *q.shape[1:], dtype=torch.uint8, device="cuda")
        scale = torch.zeros(total * case["page"], sc.shape[1], 1, device="cuda")
        codes[rows] = q.view(torch.uint8)
        scale[rows] = sc
        cache.append((codes.view(q.dtype), scale))
    return cache


def _plain_rotate(s):
    case, out = s["case"], []
    rot, half = case["rot"], case["rot"] // 2
    angle = s["pos"].double()[:, None, None] * s["freq"]
    c, sn = torch.cos(angle).float(), torch.sin(angle).float()
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        v = x.float().view(case["T"], -1, case["dim"])
        if case["norm"]:
            v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * w.float()
        r = v[..., :rot]
        a, b = (r[..., 0::2], r[..., 1::2]) if case["inter"] else (r[..., :half], r[..., half:])
        ra, rb = a * c - b * sn, b * c + a * sn
        r = torch.stack([ra, rb], -1).flatten(-2) if case["inter"] else torch.cat([ra, rb], -1)
        out.append(torch.cat([r, v[..., rot:]], -1).reshape(x.shape).to(x.dtype))
    return out


def _plain_score(s):
    f, case = s["index"], s["case"]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    G = H // Hk
    codes, scale = s["cache"][0]
    k = (codes[f["rows"]].float() * scale[f["rows"]]).permute(0, 2, 3, 1).contiguous()      # [R][Hk][D][keys]
    R, Q = f["q_row"].shape
    q = s["q"].float().view(-1, Hk, G, D)[f["q_row"]].permute(0, 2, 1, 3, 4).reshape(R, Hk, Q * G, D) * D ** -0.5
    logits = (q @ k).view(R, Hk, Q, G, -1)
    logits = logits.masked_fill(~f["seen"][:, None, :, None, :], -math.inf)
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    w = torch.where(f["counts"][:, None, :, None, None], p, torch.zeros((), device="cuda")).sum((2, 3))   # [R][Hk][keys]
    w = w[f["tok_seq"], :, f["tok_key"]]                                        # [own tokens][Hk]
    score, pos = s["marks"]
    new = f["is_new"][:, None]
    out = torch.where(new, torch.zeros((), device="cuda"), score) + w
    return [out, torch.where(new, f["new_pos"][:, None], pos)]


def _plain_evict(s):
    f, case, dt = s["index"], s["case"], _DTYPE[s["case"]["dtype"]]
    score, pos = s["marks"]
    most = f["place"].shape[1]
    there = f["there"][:, :, None]
    sc = torch.where(there, score[f["place"]], torch.full((), -math.inf, device="cuda"))    # [R][most][Hk]
    ps = torch.where(there, pos[f["place"]].long(), torch.full((), -1, device="cuda"))
    new = there & (ps > ps.amax(1, keepdim=True) - case["recent"])
    sc = torch.where(new, torch.full((), math.inf, device="cuda"), sc)
    order = torch.sort(sc, dim=1, descending=True, stable=True).indices
    rank = torch.zeros_like(order).scatter_(1, order, torch.arange(most, device="cuda")[None, :, None].expand_as(order))
    keep = f["keep"][:, None, None]
    stays = there & (rank < keep)
    at = torch.arange(most, device="cuda")[None, :, None]
    # holes before the budget, in order, take the kept ones behind it, in order
    hole, mover = ~stays & (at < keep), stays & (at >= keep)
    nth_hole, nth_mover = torch.cumsum(hole, 1) - 1, torch.cumsum(mover, 1) - 1
    by_nth = torch.zeros((sc.shape[0], most + 1, sc.shape[2]), dtype=torch.long, device="cuda")
    by_nth.scatter_(1, torch.where(mover, nth_mover, most), at.expand_as(order))
    source = torch.where(hole, torch.gather(by_nth, 1, nth_hole.clamp_min(0)), at)
    source = source[f["out_seq"], f["out_place"]]                               # [kept tokens][Hk]
    rows = f["slot"][f["out_seq"][:, None], source]
    head = torch.arange(case["kv_heads"], device="cuda")
    place = f["place"][f["out_seq"][:, None], source]
    kv = [(c.view(torch.uint8)[rows, head].view(c.dtype).float() * sl[rows, head]).to(dt) for c, sl in s["cache"]]
    return kv + [score[place, head], pos[place, head]]


def _plain_select(s):
    case = s["case"]
    R, W, N, V = case["reqs"], case["width"], case["n_out"], case["vocab"]
    x = s["logits"].float()
    m = x.amax(-1, keepdim=True)
    lse = m[:, 0].double() + torch.log(torch.exp(x.double() - m.double()).sum(-1))
    # keys that order as (value, lowest token) do
    bits = (x + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits)
    key = bits * (1 << 32) + (0xffffffff - torch.arange(V, device="cuda"))
    n = min(N, V)
    token = 0xffffffff - (torch.topk(key, n, -1).values & 0xffffffff)
    value = torch.gather(x, 1, token).double() + (s["score"].double() - lse)[:, None]
    value, token = value.view(R, W * n), token.view(R, W * n)
    if W * n < N:
        value = torch.nn.functional.pad(value, (0, N - W * n), value=-math.inf)
        token = torch.nn.functional.pad(token, (0, N - W * n))
    best, at = (t[:, :N] for t in torch.sort(value, dim=-1, descending=True, stable=True))
    none = best == -math.inf
    return [best.float(), torch.where(none, -1, at // n).int(),
            torch.where(none, -1, torch.gather(token, 1, at)).int()]


def _plain_copy(s):
    dt, out = _DTYPE[s["case"]["dtype"]], []
    for cache in s["caches"]:
        for codes, scale in cache:
            raw = codes.view(torch.uint8)
            raw[s["to"]] = raw[s["of"]]
            scale[s["to"]] = scale[s["of"]]
    for cache in s["caches"]:
        out += [(c.view(torch.uint8)[s["to"]].view(c.dtype).float() * sc[s["to"]]).to(dt) for c, sc in cache]
    return out


def _score_index(case, seed):
    """The batch as index tensors: every sequence's keys (prefix, then own), padded."""
    q_len, length, group, prefix = _batch(case, seed)
    off, pages, _ = _pages(case, seed)
    n_g, n = len(prefix), len(length)
    both = np.concatenate([prefix, length])
    slots = _slots(case, off, pages, both)
    first = np.concatenate([[0], np.cumsum(both)])
    pre = np.where(group >= 0, prefix[group] if n_g else 0, 0)
    most, Q = int((pre + length).max()), int(q_len.max())
    rows, seen = np.zeros((n, most), np.int64), np.zeros((n, Q, most), bool)
    q_row, counts = np.zeros((n, Q), np.int64), np.zeros((n, Q), bool)
    t0 = np.concatenate([[0], np.cumsum(q_len)])
    window = case["window"] or 1 << 30
    for i in range(n):
        p, m, q, g = int(pre[i]), int(length[i]), int(q_len[i]), int(group[i])
        rows[i, :p] = slots[first[g]: first[g] + p] if p else 0
        rows[i, p: p + m] = slots[first[n_g + i]: first[n_g + i] + m]
        q_row[i, :q] = t0[i] + np.arange(q)
        counts[i, max(0, q - window): q] = True
        seen[i, :q] = np.arange(most)[None, :] <= (p + m - q + np.arange(q))[:, None]
        seen[i, q:] = True
    seq = np.repeat(np.arange(n), length)
    place = np.arange(len(seq)) - np.concatenate([[0], np.cumsum(length)])[seq]
    at = place - (length - q_len)[seq]
    f = dict(rows=rows, seen=seen, q_row=q_row, counts=counts, tok_seq=seq, tok_key=pre[seq] + place, is_new=at >= 0)
    f = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in f.items()}
    f["new_pos"] = _step_positions(case, seed)[torch.from_numpy(np.where(at >= 0, t0[seq] + at, 0)).cuda()]
    return f


def _evict_index(case, seed):
    _, length, _, _ = _batch(case, seed)
    off, pages, _ = _pages(case, seed)
    n, most = len(length), int(length.max())
    slots = _slots(case, off, pages, length)
    first = np.concatenate([[0], np.cumsum(length)])
    j = np.minimum(np.arange(most)[None, :], length[:, None] - 1)
    place = first[:-1, None] + j
    keep = np.minimum(length, case["keep"])
    seq = np.repeat(np.arange(n), keep)
    f = dict(place=place, slot=slots[place], there=np.arange(most)[None, :] < length[:, None], keep=keep.astype(np.int64),
             out_seq=seq, out_place=np.arange(len(seq)) - np.concatenate([[0], np.cumsum(keep)])[seq])
    return {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in f.items()}


# ---------------------------------------------------------------------------
# the five functions
# ---------------------------------------------------------------------------
def _fill(case, seed, kv, stream, layer=0):
    """The history into the cache, as it came: each prefix and each sequence as new tokens."""
    _, length, _, prefix = _batch(case, seed)
    off, pages, _ = _pages(case, seed)
    both = np.concatenate([prefix, length])
    fill = kv.seqs(len(both), int(both.sum()), int(off[-1]))
    fill.set(both, both, off, pages, stream=stream)
    k, v = _history(case, seed, layer)
    fill.write(layer, k.data_ptr(), v.data_ptr(), stream)
    torch.cuda.synchronize()
    fill.close()


def prepare(case, seed):
    stream = torch.cuda.current_stream().cuda_stream
    s = dict(case=case, kind=case["kind"], stream=stream)
    dt, kind = _DTYPE[case["dtype"]], case["kind"]
    if own:
        from paper_2608_03579_amd import salt
    if kind == "select":
        rows = case["reqs"] * case["width"]
        s["logits"] = _normal(case, seed, 7, (rows, -(-case["vocab"] // 8) * 8), 2.5)[:, : case["vocab"]]
        s["score"] = _beam_scores(case, seed)
        if own:
            s["ctx"] = ctx = salt.Context(case["dtype"], [(128, 128)], 0, 0, 1, 0, 1)
            s["beams"] = ctx.beams(rows, case["n_out"])
            shape = (case["reqs"], case["n_out"])
            s["out"] = [torch.empty(shape, dtype=d, device="cuda") for d in (torch.float32, torch.int32, torch.int32)]
        return s
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if kind == "rotate":
        T = case["T"]
        s["q"] = _normal(case, seed, 1, (T, H * D), uneven=True)
        s["k"] = _normal(case, seed, 2, (T, Hk * D), uneven=True)
        s["qw"], s["kw"] = ((1 + 0.2 * _normal(case, seed, key, (D,)).float()).to(dt) for key in (3, 4))
        s["pos"] = _positions(case, seed)
        if own:
            s["ctx"] = ctx = salt.Context(case["dtype"], [(128, 128)], 0, 0, 1, 0, 1)
            norms = (s["qw"].data_ptr(), s["kw"].data_ptr()) if case["norm"] else (0, 0)
            s["rot"] = ctx.rotation(H, Hk, D, _frequencies(case), case["inter"], norms[0], norms[1], EPS)
            s["out"] = [torch.empty_like(s["q"]), torch.empty_like(s["k"])]
        else:
            s["freq"] = torch.from_numpy(_frequencies(case)).cuda()
        return s
    q_len, length, group, prefix = _batch(case, seed)
    off, pages, total = _pages(case, seed)
    T, n_g = int(q_len.sum()), len(prefix)
    if kind == "score":
        s["q"], s["new_pos"] = _normal(case, seed, 4, (T, H * D)), _step_positions(case, seed)
    if kind != "copy":
        s["marks"] = _marks(case, seed)
    if not own:
        if kind == "copy":
            s["caches"] = [_plain_cache(case, seed, i) for i in range(case["layers"])]
            s["of"] = torch.from_numpy(_slots(case, off, pages, length)).cuda()
            s["to"] = torch.from_numpy(_slots(case, off, pages[off[-1]:], length)).cuda()
        else:
            s["cache"] = _plain_cache(case, seed)
            s["index"] = (_score_index if kind == "score" else _evict_index)(case, seed)
        return s
    s["ctx"] = ctx = salt.Context(case["dtype"], [(H * D, H * D)], 0, 0, 1, 0, 1)
    s["kv"] = kv = ctx.kv_cache(case.get("layers", 1), H, Hk, D, case["page"], total, case["fmt"])
    if kind == "copy":
        for i in range(case["layers"]):
            _fill(case, seed, kv, stream, i)
        n = int(off[-1])
        s["lists"] = (pages[:n], pages[n: 2 * n], length)
        s["seqs"] = seqs = kv.seqs(len(length), 1, n)
        seqs.set(np.zeros_like(length), length, off, pages[n: 2 * n], stream=stream)
        s["out"] = [torch.empty((int(length.sum()), Hk, D), dtype=dt, device="cuda") for _ in range(2 * case["layers"])]
        return s
    kv.track()
    _fill(case, seed, kv, stream)
    own_off, own_pages = off[n_g:] - off[n_g], pages[off[n_g]: off[-1]]
    s["seqs"] = seqs = kv.seqs(len(length) + n_g, max(1, T), int(off[-1]))
    seqs.set(q_len, length, own_off, own_pages, group, prefix, off[: n_g + 1], pages[: off[n_g]], stream=stream)
    rows = int(length.sum())
    if kind == "evict":
        kept = np.minimum(length, case["keep"])
        s["left"] = left = kv.seqs(len(length), 1, int(off[-1]))
        left.set(q_len, kept, own_off, own_pages, stream=stream)
        rows = int(kept.sum())
        s["out"] = [torch.empty((rows, Hk, D), dtype=dt, device="cuda") for _ in range(2)]
    s["out_marks"] = [torch.empty((rows, Hk), dtype=d, device="cuda") for d in (torch.float32, torch.int32)]
    return s


def run(state):
    s, kind, case = state, state["kind"], state["case"]
    if not own:
        return {"rotate": _plain_rotate, "score": _plain_score, "evict": _plain_evict, "select": _plain_select,
                "copy": _plain_copy}[kind](s)
    st = s["stream"]
    if kind == "rotate":
        q, k = s["out"]
        s["ctx"].rotate(s["rot"], case["T"], s["pos"].data_ptr(), s["q"].data_ptr(), q.data_ptr(), s["k"].data_ptr(),
                        k.data_ptr(), st)
        return s["out"]
    if kind == "select":
        s["beams"].select(case["reqs"], case["width"], case["vocab"], s["logits"].data_ptr(), s["score"].data_ptr(),
                          case["n_out"], *[o.data_ptr() for o in s["out"]], st, ld=s["logits"].stride(0))
        return s["out"]
    if kind == "copy":
        s["kv"].copy(*s["lists"], stream=st)
        for i in range(case["layers"]):
            s["seqs"].read(i, "own", s["out"][2 * i].data_ptr(), s["out"][2 * i + 1].data_ptr(), st)
        return s["out"]
    # the sequences come with the marks they have gathered
    score, pos = s["marks"]
    s["seqs"].write_marks(0, score.data_ptr(), pos.data_ptr(), st)
    out_score, out_pos = s["out_marks"]
    if kind == "score":
        s["seqs"].score(0, s["q"].data_ptr(), s["new_pos"].data_ptr(), case["dim"] ** -0.5, case["window"], st)
        s["seqs"].read_marks(0, out_score.data_ptr(), out_pos.data_ptr(), st)
        return s["out_marks"]
    s["seqs"].evict(0, case["keep"], case["recent"], st)
    s["left"].read(0, "own", s["out"][0].data_ptr(), s["out"][1].data_ptr(), st)
    s["left"].read_marks(0, out_score.data_ptr(), out_pos.data_ptr(), st)
    return s["out"] + s["out_marks"]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "select":
        rows = case["reqs"] * case["width"]
        n = rows * case["vocab"]
        return dict(bytes=es * n + 4 * rows + 12 * case["reqs"] * case["n_out"], flops=4 * n)
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "rotate":
        n = case["T"] * (H + Hk) * D
        return dict(bytes=2 * es * n + 4 * case["T"], flops=7 * n)
    # the batch of seed 0 stands for those of the other seeds
    q_len, length, group, prefix = _batch(case, 0)
    n = int(length.sum())
    vec = Hk * (2 * D + 8)                      # a token in the cache: codes and scales of k and v
    if case["kind"] == "copy":                  # read, written, read and out
        return dict(bytes=case["layers"] * n * (3 * vec + 2 * es * Hk * D), flops=2 * case["layers"] * n * Hk * D)
    if case["kind"] == "evict":                 # marks in, the kept tokens' out, with their k and v
        kept = int(np.minimum(length, case["keep"]).sum())
        return dict(bytes=8 * Hk * (n + kept) + kept * (vec + 2 * es * Hk * D), flops=2 * kept * Hk * D)
    T = int(q_len.sum())
    used = np.unique(group[group >= 0])
    keys = q_len.astype(np.int64) * (length - q_len) + q_len.astype(np.int64) * (q_len + 1) // 2
    keys += q_len * np.where(group >= 0, prefix[group] if len(prefix) else 0, 0)
    if case["window"]:
        w = np.minimum(q_len, case["window"]).astype(np.int64)
        keys = w * (length - w) + w * (w + 1) // 2 + w * np.where(group >= 0, prefix[group] if len(prefix) else 0, 0)
    return dict(bytes=(n + int(prefix[used].sum())) * Hk * (D + 4) + 16 * n * Hk + es * T * H * D + 4 * T,
                flops=2 * int(keys.sum()) * H * D)


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _round_e4m3(v):
    """Nearest value with three bits behind the first, ties to even; steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(v)
    step = torch.exp2(torch.clamp(e - 1, min=-6).double() - 3)
    return torch.round(v / step) * step


def _exact_kv(x, fmt):
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    if fmt == "int8":
        s = (amax * float(np.float32(1.0 / 127.0))).float().clamp_min(2.0 ** -100)
        r = (1.0 / s.double()).float().double()
        return torch.round((x * r).float().double()).clamp(-127, 127) * s.double()
    s = torch.exp2(torch.ceil(torch.log2(amax.clamp_min(1e-300) / 448.0)))
    s = torch.where(amax / s > 448.0, s * 2, torch.where(amax / (s / 2) <= 448.0, s / 2, s)).clamp_min(2.0 ** -100)
    s = torch.where(amax > 0, s, torch.ones_like(s))
    return _round_e4m3(x / s) * s


def _exact_rotate(case, seed):
    T, D, rot = case["T"], case["dim"], case["rot"]
    pos, dt = _positions(case, seed).double(), _DTYPE[case["dtype"]]
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                    pos[:, None] * torch.from_numpy(_frequencies(case)).cuda()[None, :])[:, None, :]
    out = []
    for key, wkey, heads in ((1, 3, case["heads"]), (2, 4, case["kv_heads"])):
        x = _normal(case, seed, key, (T, heads * D), uneven=True).double().view(T, heads, D)
        if case["norm"]:
            w = (1 + 0.2 * _normal(case, seed, wkey, (D,)).float()).to(dt).double()
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS) * w
        r = x[..., :rot].reshape(T, heads, rot // 2, 2) if case["inter"] else x[..., :rot].reshape(
            T, heads, 2, rot // 2).transpose(-1, -2)
        r = torch.view_as_real(torch.view_as_complex(r.contiguous()) * z)
        r = r.reshape(T, heads, rot) if case["inter"] else r.transpose(-1, -2).reshape(T, heads, rot)
        out.append(torch.cat([r, x[..., rot:]], -1).reshape(T, heads * D))
    return out


def _exact_score(case, seed):
    q_len, length, group, prefix = _batch(case, seed)
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    G = H // Hk
    k = _exact_kv(_history(case, seed)[0], case["fmt"])
    q = _normal(case, seed, 4, (int(q_len.sum()), H * D)).double().view(-1, H, D)
    score, pos = (a.clone() for a in _marks(case, seed))
    score = score.double()
    step = _step_positions(case, seed)
    off = np.concatenate([[0], np.cumsum(np.concatenate([prefix, length]))])
    t, row = 0, 0
    for r in range(len(length)):
        a, b = int(off[len(prefix) + r]), int(off[len(prefix) + r + 1])
        n, m, g = int(q_len[r]), int(length[r]), int(group[r])
        pa, pb = (int(off[g]), int(off[g + 1])) if g >= 0 else (0, 0)
        kk = torch.cat([k[pa:pb], k[a:b]])
        score[row + m - n: row + m] = 0
        pos[row + m - n: row + m] = step[t: t + n, None]
        c0 = max(0, n - case["window"]) if case["window"] else 0
        limit = (pb - pa) + m - n + torch.arange(c0, n, device="cuda")
        hidden = torch.arange(kk.shape[0], device="cuda")[None, :] > limit[:, None]
        for h in range(H):
            logits = (q[t + c0: t + n, h] @ kk[:, h // G].T.contiguous()) / math.sqrt(D)
            p = torch.softmax(logits.masked_fill(hidden, -math.inf), -1)
            score[row: row + m, h // G] += p.sum(0)[pb - pa:]
        t, row = t + n, row + m
    return [score, pos]


def _exact_evict(case, seed):
    _, length, _, _ = _batch(case, seed)
    score, pos = (a.cpu().numpy() for a in _marks(case, seed))
    k, v = (_exact_kv(a, case["fmt"]) for a in _history(case, seed))
    row, at = 0, []
    for m in length:
        m = int(m)
        keep = min(m, case["keep"])
        here = np.empty((keep, case["kv_heads"]), np.int64)
        for h in range(case["kv_heads"]):
            sc, ps = score[row: row + m, h], pos[row: row + m, h].astype(np.int64)
            first = np.lexsort((np.arange(m), -sc.astype(np.float64), ~(ps > ps.max() - case["recent"])))
            stays = np.zeros(m, bool)
            stays[first[:keep]] = True
            src = np.arange(keep)
            src[~stays[:keep]] = keep + np.flatnonzero(stays[keep:])
            here[:, h] = row + src
        at.append(here)
        row += m
    at = np.concatenate(at)
    head = np.arange(case["kv_heads"])
    ix, hx = torch.from_numpy(at).cuda(), torch.from_numpy(head).cuda()
    return [k[ix, hx], v[ix, hx], torch.from_numpy(score[at, head]).double().cuda(), torch.from_numpy(pos[at, head]).cuda()]


def _exact_select(case, seed):
    rows, V, N = case["reqs"] * case["width"], case["vocab"], case["n_out"]
    x = _normal(case, seed, 7, (rows, -(-V // 8) * 8), 2.5)[:, :V]
    base = _beam_scores(case, seed).double().view(case["reqs"], -1)
    out = [torch.full((case["reqs"], N), -math.inf, dtype=torch.float64, device="cuda"),
           torch.full((case["reqs"], N), -1, dtype=torch.int32, device="cuda"),
           torch.full((case["reqs"], N), -1, dtype=torch.int32, device="cuda")]
    for r in range(case["reqs"]):
        lp = torch.log_softmax(x[r * case["width"]: (r + 1) * case["width"]].double(), -1) + base[r][:, None]
        v, i = torch.sort(lp.flatten(), descending=True, stable=True)
        n = min(N, int((v[:N] > -math.inf).sum()))
        out[0][r, :n], out[1][r, :n], out[2][r, :n] = v[:n], (i[:n] // V).int(), (i[:n] % V).int()
    return out


def exact(case, seed):
    if case["kind"] == "copy":
        return [_exact_kv(x, case["fmt"]) for i in range(case["layers"]) for x in _history(case, seed, i)]
    return {"rotate": _exact_rotate, "score": _exact_score, "evict": _exact_evict, "select": _exact_select}[case["kind"]](
        case, seed)
