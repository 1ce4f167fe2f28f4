"""Performance cases of the operators around the adapter apply: the rest of an adapted layer's attention block.

``base``    ``y = x W_base`` in 8-bit floating point, a scale for each block of 128: the
            product whose ``y`` the centroid + residual apply adds to.
``write``   k and v of a step quantised into the paged cache, and the step's tokens read back.
``read``    every token of the batch's sequences read back from the cache.
``attend``  attention over the cache for a batch whose domains share long prefixes.

With ``own`` the calls go through ``paper_2608_03579_amd.salt``; without it the same
operators are written with elementary torch operations in 32 bits.  torch owns the
activations; all work goes to torch's current stream.

A case is a dict of plain values:

``in_dim, outs``
    base: the product's input width, and the widths of the tables that share this x ("+" between them).
``heads, kv_heads, dim, page, fmt``
    attention layout, tokens to a page, and the cache's format.
``seqs, new, own, even``
    sequences; new tokens of each in this step (``even``: all of them have ``new``, else 1 to ``new``);
    their own tokens, the new ones included (``even``: ``own`` each, else spread over the logarithm up to it).
``groups, prefix``
    domains with a shared prefix of up to ``prefix`` tokens (0: none); sequences belong to one at random, and
    with ``even`` false some to none.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

STD = 0.02              # base-weight scale
BLOCK = 128
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # q_proj for one user's next token: the smallest call there is
        dict(name="base_q_3b_T1", kind="base", dtype="bf16", in_dim=3072, outs="3072", T=1),
        # q, k and v of a decode step of 64 users
        dict(name="base_qkv_8b_T64", kind="base", dtype="bf16", in_dim=4096, outs="4096+1024+1024", T=64),
        # o_proj of a decode step of 256 users
        dict(name="base_o_8b_T256", kind="base", dtype="bf16", in_dim=4096, outs="4096", T=256),
        # a chunk of prefill in fp32 with widths that fill no block evenly
        dict(name="base_ragged_f32_T203", kind="base", dtype="f32", in_dim=2056, outs="2056+520", T=203),
        # gate and up of a full prefill batch: the largest product
        dict(name="base_gateup_3b_T8192", kind="base", dtype="bf16", in_dim=3072, outs="8192+8192", T=8192),
        # the new token of 256 users goes into the cache
        dict(name="write_8b_decode_T256", kind="write", dtype="bf16", fmt="e4m3", heads=32, kv_heads=8, dim=128,
             page=64, seqs=256, new=1, own=1024, even=False, groups=0, prefix=0),
        # the prompts of a full prefill batch go into it
        dict(name="write_3b_prefill_T8192", kind="write", dtype="bf16", fmt="int8", heads=24, kv_heads=8, dim=128,
             page=64, seqs=16, new=512, own=512, even=True, groups=0, prefix=0),
        # sequences of a batch leave the cache as plain k and v, to be moved to another node
        dict(name="read_3b_seqs64", kind="read", dtype="bf16", fmt="e4m3", heads=24, kv_heads=8, dim=128, page=64,
             seqs=64, new=1, own=4096, even=False, groups=0, prefix=0),
        # a handful of interactive users at their lowest latency
        dict(name="attend_3b_decode_T4", kind="attend", dtype="bf16", fmt="e4m3", heads=24, kv_heads=8, dim=128,
             page=64, seqs=4, new=1, own=1024, even=False, groups=0, prefix=0),
        # 256 users of 16 domains decode behind their domain's prompt
        dict(name="attend_domains_8b_T256", kind="attend", dtype="bf16", fmt="e4m3", heads=32, kv_heads=8, dim=128,
             page=64, seqs=256, new=1, own=1024, even=False, groups=16, prefix=4096),
        # drafted tokens of a few users, fp32, small pages, some users without a domain
        dict(name="attend_drafts_f32_int8", kind="attend", dtype="f32", fmt="int8", heads=20, kv_heads=4, dim=64,
             page=16, seqs=23, new=4, own=1500, even=False, groups=5, prefix=1531),
        # prompts of 8 users prefill behind two long domain prompts: the largest attention
        dict(name="attend_chunk_3b_T2048", kind="attend", dtype="bf16", fmt="e4m3", heads=24, kv_heads=8, dim=128,
             page=64, seqs=8, new=256, own=256, even=True, groups=2, prefix=8192),
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
        kind = rng.choice(["base"] * 4 + ["attend"] * 5 + ["write", "write", "read"])
        f32 = rng.random() < 0.2
        c = dict(kind=kind, dtype="f32" if f32 else "bf16")
        if kind == "base":
            in_dim = rng.choice([3072, 4096, 8 * _log_int(rng, 8, 1024)])
            n = rng.choice([1, 1, 2, 3])
            outs = [rng.choice([1024, 3072, 4096, 8 * _log_int(rng, 8, 1024)]) for _ in range(n)]
            c.update(in_dim=in_dim, outs="+".join(str(o) for o in outs),
                     T=rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 8192)]))
        else:
            kv = rng.choice([1, 2, 4, 8, 8])
            c.update(fmt=rng.choice(["e4m3", "e4m3", "int8"]), heads=kv * rng.choice([1, 3, 4, 5, 8]), kv_heads=kv,
                     dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]))
            even = rng.random() < 0.3
            if kind == "attend" and rng.random() < 0.6 or kind == "read":
                new = rng.choice([1, 1, 1, rng.randint(2, 8)])      # decode, or drafts
                seqs = _log_int(rng, 1, 256)
                top = _log_int(rng, 16, 4096)
            else:
                new = _log_int(rng, 1, 700)                         # prompts
                seqs = _log_int(rng, 1, 32)
                top = _log_int(rng, 1, 1024)
            groups = rng.choice([0, 1, rng.randint(1, 16)]) if kind == "attend" else 0
            c.update(seqs=seqs, new=new, own=max(new, top), even=even, groups=groups,
                     prefix=_log_int(rng, 1, 8192) if groups else 0)
        # (the plain form pads: it has to fit too)
        if _cost(c) <= most[kind] and _padded(c) <= 3e9:
            return c


# ---------------------------------------------------------------------------
# the batch of a case
# ---------------------------------------------------------------------------
def _batch(case, seed):
    """Per sequence its new tokens, its own tokens and its domain (-1: none); per domain its prefix's tokens.
    The batches of all seeds have the same sequences, in another order."""
    rng = np.random.default_rng([2608, 3581])
    n, new, most = case["seqs"], case["new"], case["own"]
    if case["even"]:
        q_len, length = np.full(n, new), np.full(n, most)
    else:
        q_len = rng.integers(1, new + 1, size=n)
        length = np.exp(rng.uniform(0, math.log(most) if most > 1 else 0.0, size=n)).astype(np.int64)
        length = np.maximum(np.maximum(length, q_len), 1)
    rng = np.random.default_rng([2608, 3581, int(seed)])
    order = rng.permutation(n)
    q_len, length = q_len[order], length[order]
    groups = case["groups"]
    prefix = rng.integers(case["prefix"] // 2 + 1, case["prefix"] + 1, size=groups) if groups else np.zeros(0, int)
    if case["even"] and groups:
        prefix = np.full(groups, case["prefix"])
        group = np.arange(n) % groups
    else:
        group = rng.integers(-1, groups, size=n) if groups else np.full(n, -1)
    return q_len.astype(np.int32), length.astype(np.int32), group.astype(np.int32), prefix.astype(np.int32)


def _pages(case, seed):
    """Page tables in a random order of the pool's pages: (first page reference of each holder, the pages), the
    domains' prefixes before the sequences, and the pool's pages."""
    _, length, _, prefix = _batch(case, seed)
    tokens = np.concatenate([prefix, length])
    n = (tokens + case["page"] - 1) // case["page"]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(off[-1]) + 3
    pages = np.random.default_rng([2608, 3582, int(seed)]).permutation(total)[: off[-1]].astype(np.int32)
    return off, pages, total


def _padded(case):
    """Floats of the plain form's largest tensors."""
    if case["kind"] == "base":
        return 0
    q_len, length, group, prefix = _batch(case, 0)
    kd, p = case["kv_heads"] * case["dim"], int(prefix.max()) if len(prefix) else 0
    keys = p + int(length.max())
    return 2 * kd * (len(length) * int(length.max()) + len(prefix) * p) + 3 * int(q_len.max()) * len(length) * case["heads"] * keys


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(case, seed, key, shape, std=1.0, uneven=False):
    """Seeded N(0, std^2) on the GPU; `uneven`: a few of the last axis's columns are several times larger, as in activations."""
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + key * 7919 + 29) % (1 << 62))
    v = torch.randn(shape, generator=g, device="cuda")
    if uneven:
        n = shape[-1]
        v[..., torch.randint(0, n, (max(1, n // 64),), generator=g, device="cuda")] *= 8.0
    return (v * std).to(_DTYPE[case["dtype"]])


def _outs(case):
    return [int(o) for o in case["outs"].split("+")]


def _history(case, seed):
    """k and v of every token of the prefixes and the sequences, holder after holder: [tokens][kv_heads][dim]."""
    _, length, _, prefix = _batch(case, seed)
    shape = (int(prefix.sum() + length.sum()), case["kv_heads"], case["dim"])
    return _normal(case, seed, 1, shape, uneven=True), _normal(case, seed, 2, shape)


def _new_rows(case, seed):
    """Rows of the history that are the step's new tokens, in the order of q."""
    q_len, length, _, prefix = _batch(case, seed)
    end = int(prefix.sum()) + np.cumsum(length)
    return torch.from_numpy(np.concatenate([np.arange(e - q, e) for e, q in zip(end, q_len)])).cuda()


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _e4m3_block(x, dims):
    """(codes, scale) of blocks: scale = amax / 448 over `dims`, codes rounded to the 8-bit format."""
    amax = x.abs().amax(dims, keepdim=True)
    scale = (amax * (1.0 / 448.0)).clamp_min(2.0 ** -126)
    return (x * scale.reciprocal()).to(torch.float8_e4m3fn), scale


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


def _plain_base(s):
    x = s["x"].float()
    T, K = x.shape
    kb = -(-K // BLOCK)
    q, sx = _e4m3_block(torch.nn.functional.pad(x, (0, kb * BLOCK - K)).view(T, kb, BLOCK), 2)
    xd = (q.float() * sx).view(T, kb * BLOCK)[:, :K]
    ys = []
    for wq, sw in s["weights"]:
        rows = sw.repeat_interleave(BLOCK, 0)[:K]
        wd = wq.float() * rows.repeat_interleave(BLOCK, 1)[:, : wq.shape[1]]
        ys.append((xd @ wd).to(s["x"].dtype))
    return ys


def _plain_attend(s):
    f, case, dt = s["index"], s["case"], s["q"].dtype
    H, Hk, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    G = H // Hk
    T = s["q"].shape[0]
    q = s["q"].float().view(T, Hk, G, D) * D ** -0.5

    def gather(table, most):
        at = torch.arange(most, device="cuda")
        rows = table[:, at // page] * page + at % page                          # [holders][most]
        kv = [(c[rows].float() * sc[rows]).permute(0, 2, 1, 3).contiguous() for c, sc in s["cache"]]
        return kv                                                               # [holders][Hk][most][D]

    # own tokens: rows of a sequence against its keys, causal
    k, v = gather(f["own_table"], f["own_most"])
    R, Q = f["own_row"].shape
    qs = q[f["own_row"]].permute(0, 2, 1, 3, 4).reshape(R, Hk, Q * G, D)
    logits = (qs @ k.transpose(-1, -2).contiguous()).view(R, Hk, Q, G, -1)
    at = torch.arange(f["own_most"], device="cuda")
    logits = logits.masked_fill(~(at <= f["own_pos"][:, None, :, None, None]), -math.inf)
    own_logits = logits.permute(0, 2, 1, 3, 4)[f["seq"], f["in_seq"]]           # [T][Hk][G][keys]
    n_own = own_logits.shape[-1]
    if f["groups"]:
        pk, pv = gather(f["pre_table"], f["pre_most"])
        N, M = f["pre_row"].shape
        qs = q[f["pre_row"]].permute(0, 2, 1, 3, 4).reshape(N, Hk, M * G, D)
        logits = (qs @ pk.transpose(-1, -2).contiguous()).view(N, Hk, M, G, -1).permute(0, 2, 1, 3, 4)
        logits = logits[f["grp"], f["in_grp"]]
        at = torch.arange(f["pre_most"], device="cuda")
        logits = logits.masked_fill(~(at < f["pre_len"][:, None, None, None]), -math.inf)
        own_logits = torch.cat([own_logits, logits], -1)
    top = own_logits.amax(-1, keepdim=True)
    p = torch.exp(own_logits - top)
    p = p / p.sum(-1, keepdim=True)
    mine = torch.zeros(R, Q, Hk, G, n_own, device="cuda")
    mine[f["seq"], f["in_seq"]] = p[..., :n_own]
    o = (mine.permute(0, 2, 1, 3, 4).reshape(R, Hk, Q * G, n_own) @ v).view(R, Hk, Q, G, D)
    out = o.permute(0, 2, 1, 3, 4)[f["seq"], f["in_seq"]]
    if f["groups"]:
        shared = torch.zeros(N, M, Hk, G, f["pre_most"], device="cuda")
        shared[f["grp"], f["in_grp"]] = p[..., n_own:]
        o = (shared.permute(0, 2, 1, 3, 4).reshape(N, Hk, M * G, f["pre_most"]) @ pv).view(N, Hk, M, G, D)
        out = out + o.permute(0, 2, 1, 3, 4)[f["grp"], f["in_grp"]] * f["has"][:, None, None, None]
    return out.reshape(T, H * D).to(dt)


def _plain_index(case, seed):
    """The batch as index tensors: padded page tables, and where each row of q stands in its sequence and its domain."""
    q_len, length, group, prefix = _batch(case, seed)
    off, pages, _ = _pages(case, seed)
    n_g, n = len(prefix), len(length)

    def table(first, count):
        w = max(1, max(off[first + i + 1] - off[first + i] for i in range(count)))
        t = np.zeros((count, w), np.int64)
        for i in range(count):
            t[i, : off[first + i + 1] - off[first + i]] = pages[off[first + i]: off[first + i + 1]]
        return t

    seq = np.repeat(np.arange(n), q_len)
    first = np.concatenate([[0], np.cumsum(q_len)])
    in_seq = np.arange(len(seq)) - first[seq]
    row = np.zeros((n, q_len.max()), np.int64)
    pos = np.full((n, q_len.max()), -1, np.int64)
    row[seq, in_seq] = np.arange(len(seq))
    pos[seq, in_seq] = (length - q_len)[seq] + in_seq
    f = dict(own_table=table(n_g, n), own_most=int(length.max()), own_row=row, own_pos=pos, seq=seq, in_seq=in_seq,
             groups=n_g)
    if n_g:
        g = group[seq]
        grp = np.maximum(g, 0)
        order = np.argsort(grp, kind="stable")
        start = np.searchsorted(grp[order], np.arange(n_g))
        in_grp = np.empty(len(seq), np.int64)
        in_grp[order] = np.arange(len(seq)) - start[grp[order]]
        pre_row = np.zeros((n_g, int(in_grp.max()) + 1), np.int64)
        pre_row[grp, in_grp] = np.arange(len(seq))
        f.update(pre_table=table(0, n_g), pre_most=int(prefix.max()), pre_row=pre_row, grp=grp, in_grp=in_grp,
                 pre_len=np.where(g >= 0, prefix[grp], 0), has=(g >= 0).astype(np.float32))
    return {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in f.items()}


def _plain_cache(case, seed):
    """The cache as it stands before the call: codes [pages x page][kv_heads][dim] and scales of k and of v."""
    off, pages, total = _pages(case, seed)
    q_len, length, group, prefix = _batch(case, seed)
    rows = torch.from_numpy(_slots(case, off, pages, np.concatenate([prefix, length]))).cuda()
    cache = []
    for x in _history(case, seed):
        q, sc = _quantise_kv(x, case["fmt"])
        codes = torch.zeros(total * case["page"], *q.shape[1:], dtype=torch.uint8, device="cuda")
        scale = torch.zeros(total * case["page"], sc.shape[1], 1, device="cuda")
        codes[rows] = q.view(torch.uint8)
        scale[rows] = sc
        cache.append((codes.view(q.dtype), scale))
    return cache


def _slots(case, off, pages, tokens):
    """Where each holder's tokens lie in the pool, in order."""
    page, at = case["page"], []
    for i, n in enumerate(tokens):
        j = np.arange(n)
        at.append(pages[off[i] + j // page].astype(np.int64) * page + j % page)
    return np.concatenate(at)


# ---------------------------------------------------------------------------
# the five functions
# ---------------------------------------------------------------------------
def prepare(case, seed):
    s = dict(case=case, kind=case["kind"], stream=torch.cuda.current_stream().cuda_stream)
    dt = _DTYPE[case["dtype"]]
    if case["kind"] == "base":
        outs = _outs(case)
        s["x"] = _normal(case, seed, 3, (case["T"], case["in_dim"]), uneven=True)
        ws = [_normal(case, seed, 10 + i, (case["in_dim"], o), STD) for i, o in enumerate(outs)]
        if own:
            from paper_2608_03579_amd import salt
            s["ctx"] = ctx = salt.Context(case["dtype"], [(case["in_dim"], o) for o in outs], 0, 0, 1, 0, case["T"])
            for i, w in enumerate(ws):
                ctx.pin_base(i, w.data_ptr(), w.shape[1], s["stream"])
            s["tables"] = list(range(len(outs)))
            s["y"] = [torch.empty(case["T"], o, dtype=dt, device="cuda") for o in outs]
            s["y_ptr"] = [y.data_ptr() for y in s["y"]]
        else:
            s["weights"] = [_weight_blocks(w) for w in ws]
        return s
    q_len, length, group, prefix = _batch(case, seed)
    H, Hk, D, T = case["heads"], case["kv_heads"], case["dim"], int(q_len.sum())
    if case["kind"] == "attend":
        s["q"] = _normal(case, seed, 4, (T, H * D))
    if not own:
        s["cache"] = _plain_cache(case, seed)
        s["index"] = _plain_index(case, seed)
        if case["kind"] != "attend":
            off, pages, _ = _pages(case, seed)
            all_rows = _slots(case, off, pages, np.concatenate([prefix, length]))
            s["rows"] = torch.from_numpy(all_rows[int(prefix.sum()):]).cuda()
            if case["kind"] == "write":
                new = _new_rows(case, seed)
                s["rows"] = torch.from_numpy(all_rows).cuda()[new]
                s["k"], s["v"] = (a[new] for a in _history(case, seed))
        return s
    from paper_2608_03579_amd import salt
    off, pages, total = _pages(case, seed)
    n_g = len(prefix)
    tokens = int(prefix.sum() + length.sum())
    s["ctx"] = ctx = salt.Context(case["dtype"], [(H * D, H * D)], 0, 0, 1, 0, 1)
    s["kv"] = kv = ctx.kv_cache(1, H, Hk, D, case["page"], total, case["fmt"])
    # the history, written as it came: each prefix and each sequence as new tokens
    fill = kv.seqs(n_g + len(length), tokens, len(pages))
    both = np.concatenate([prefix, length])
    fill.set(both, both, off, pages, stream=s["stream"])
    k, v = _history(case, seed)
    fill.write(0, k.data_ptr(), v.data_ptr(), s["stream"])
    torch.cuda.synchronize()
    fill.close()
    s["seqs"] = seqs = kv.seqs(len(length) + n_g, T, len(pages))
    seqs.set(q_len, length, off[n_g:] - off[n_g], pages[off[n_g]:], group, prefix, off[: n_g + 1], pages[: off[n_g]],
             stream=s["stream"])
    if case["kind"] == "attend":
        s["out"] = torch.empty(T, H * D, dtype=dt, device="cuda")
        return s
    rows = T if case["kind"] == "write" else int(length.sum())
    if case["kind"] == "write":
        new = _new_rows(case, seed)
        s["k"], s["v"] = k[new], v[new]
    s["out"] = [torch.empty(rows, Hk, D, dtype=dt, device="cuda") for _ in range(2)]
    return s


def _weight_blocks(w):
    """A base weight in blocks of 128 x 128: codes [in][out] and scales."""
    K, N = w.shape
    kb, nb = -(-K // BLOCK), -(-N // BLOCK)
    p = torch.nn.functional.pad(w.float(), (0, nb * BLOCK - N, 0, kb * BLOCK - K)).view(kb, BLOCK, nb, BLOCK)
    q, sc = _e4m3_block(p, (1, 3))
    return q.view(kb * BLOCK, nb * BLOCK)[:K, :N].contiguous(), sc.view(kb, nb)


def run(state):
    s = state
    if not own:
        if s["kind"] == "base":
            return _plain_base(s)
        if s["kind"] == "attend":
            return _plain_attend(s)
        dt = _DTYPE[s["case"]["dtype"]]
        if s["kind"] == "write":
            for x, (codes, scale) in zip((s["k"], s["v"]), s["cache"]):
                q, sc = _quantise_kv(x, s["case"]["fmt"])
                codes.view(torch.uint8)[s["rows"]] = q.view(torch.uint8)
                scale[s["rows"]] = sc
        return [(codes.view(torch.uint8)[s["rows"]].view(codes.dtype).float() * scale[s["rows"]]).to(dt)
                for codes, scale in s["cache"]]
    if s["kind"] == "base":
        s["ctx"].base_product(s["tables"], s["case"]["T"], s["x"].data_ptr(), s["y_ptr"], s["stream"])
        return s["y"]
    if s["kind"] == "attend":
        s["seqs"].attend(0, s["q"].data_ptr(), s["out"].data_ptr(), s["case"]["dim"] ** -0.5, s["stream"])
        return s["out"]
    k, v = s["out"]
    if s["kind"] == "write":
        s["seqs"].write(0, s["k"].data_ptr(), s["v"].data_ptr(), s["stream"])
        s["seqs"].read(0, "new", k.data_ptr(), v.data_ptr(), s["stream"])
    else:
        s["seqs"].read(0, "own", k.data_ptr(), v.data_ptr(), s["stream"])
    return [k, v]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "base":
        K, N, T = case["in_dim"], sum(_outs(case)), case["T"]
        return dict(bytes=K * N + 4 * -(-K // BLOCK) * -(-N // BLOCK) + es * T * (K + N), flops=2 * T * K * N)
    # the batch of seed 0 stands for those of the other seeds
    q_len, length, group, prefix = _batch(case, 0)
    H, Hk, D, T = case["heads"], case["kv_heads"], case["dim"], int(q_len.sum())
    vec = Hk * (2 * D + 8)                      # a token in the cache: codes and scales of k and v
    if case["kind"] == "write":                 # in, into the cache, and out of it again
        return dict(bytes=T * (2 * es * 2 * Hk * D + 2 * vec), flops=8 * T * Hk * D)
    if case["kind"] == "read":
        n = int(length.sum())
        return dict(bytes=n * (vec + 2 * es * Hk * D), flops=2 * n * Hk * D)
    used = np.unique(group[group >= 0])
    keys = q_len.astype(np.int64) * (length - q_len) + q_len.astype(np.int64) * (q_len + 1) // 2
    keys += q_len * np.where(group >= 0, prefix[group] if len(prefix) else 0, 0)
    return dict(bytes=(int(length.sum()) + int(prefix[used].sum())) * vec + 2 * es * T * H * D,
                flops=4 * int(keys.sum()) * H * D)


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _round_e4m3(v):
    """Nearest value with three bits behind the first, ties to even; steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(v)
    step = torch.exp2(torch.clamp(e - 1, min=-6).double() - 3)
    return torch.round(v / step) * step


def _exact_block(x, dims):
    """What 8 bits hold of x (64 bits) in one block over `dims`; the scale and its reciprocal are 32-bit numbers."""
    c = float(np.float32(1.0 / 448.0))
    s = (x.abs().amax(dims, keepdim=True) * c).float().clamp_min(2.0 ** -126)
    r = (1.0 / s.double()).float().double()
    return _round_e4m3((x * r).float().double()) * s.double()


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


def exact(case, seed):
    if case["kind"] == "base":
        K = case["in_dim"]
        x = _normal(case, seed, 3, (case["T"], K), uneven=True).double()
        xd = torch.cat([_exact_block(x[:, k: k + BLOCK], 1) for k in range(0, K, BLOCK)], 1)
        res = []
        for i, o in enumerate(_outs(case)):
            w = _normal(case, seed, 10 + i, (K, o), STD).double()
            for k in range(0, K, BLOCK):
                for n in range(0, o, BLOCK):
                    w[k: k + BLOCK, n: n + BLOCK] = _exact_block(w[k: k + BLOCK, n: n + BLOCK], (0, 1))
            res.append(xd @ w)
        return res
    q_len, length, group, prefix = _batch(case, seed)
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    k, v = (_exact_kv(a, case["fmt"]) for a in _history(case, seed))
    if case["kind"] != "attend":
        rows = _new_rows(case, seed) if case["kind"] == "write" else slice(int(prefix.sum()), None)
        return [k[rows], v[rows]]
    q = _normal(case, seed, 4, (int(q_len.sum()), H * D)).double().view(-1, H, D)
    off = np.concatenate([[0], np.cumsum(np.concatenate([prefix, length]))])
    out, t = [], 0
    for r in range(len(length)):
        a, b = int(off[len(prefix) + r]), int(off[len(prefix) + r + 1])
        n, g = int(q_len[r]), int(group[r])
        pa, pb = (int(off[g]), int(off[g + 1])) if g >= 0 else (0, 0)
        kk = torch.cat([k[pa:pb], k[a:b]])
        vv = torch.cat([v[pa:pb], v[a:b]])
        limit = (pb - pa) + (b - a) - n + torch.arange(n, device="cuda")
        hidden = torch.arange(kk.shape[0], device="cuda")[None, :] > limit[:, None]
        o = torch.empty(n, H, D, dtype=torch.float64, device="cuda")
        for h in range(H):
            kh = h // (H // Hk)
            logits = (q[t: t + n, h] @ kk[:, kh].T.contiguous()) / math.sqrt(D)
            p = torch.softmax(logits.masked_fill(hidden, -math.inf), -1)
            o[:, h] = p @ vv[:, kh].contiguous()
        out.append(o.view(n, H * D))
        t += n
    return torch.cat(out)
