"""The attention block of an adapted decoder layer, prompts and then decode steps, through libsalt.

Users of two domains share their domain's prompt. Per step:

    q, k, v = x W_q, x W_k, x W_v       salt_base_product   (8-bit weights, blocks of 128)
    q, k, v += the users' adapters       salt_apply_batch    (domain centroid + user residual)
    q, k rotated by their positions      salt_rotate         (a user's tokens stand behind the prompt)
    k, v into the cache                  salt_kv_write       (pages, 8 bits)
    attention over prompt and history    salt_attend         (a domain's prompt is read once)
    y = attention W_o, += the adapters   salt_base_product, salt_apply

    python examples/attention_block.py [steps]

Runs on synthetic values (seeded) and compares the last step's output with float64 arithmetic on
unquantised weights and cache; prints the difference that the 8-bit formats make.
"""
from __future__ import annotations

import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

HIDDEN, HEADS, KV_HEADS, DIM = 512, 8, 2, 64
KV = KV_HEADS * DIM
DOMAINS, PROMPT, USERS, PAGE = 2, (200, 131), 6, 64
RANK_C, RANK_U = 16, 2
FREQ = 10000.0 ** (-np.arange(0, DIM, 2) / DIM)                                  # radians per position
TABLES = [(HIDDEN, HIDDEN), (HIDDEN, KV), (HIDDEN, KV), (HIDDEN, HIDDEN)]       # q, k, v, o
Q, K, V, O = range(4)


def bf16(a):
    """(bits, values) of an array rounded to bf16."""
    u = np.ascontiguousarray(a, np.float32).view(np.uint32).astype(np.uint64)
    bits = ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return bits, decode(bits)


def decode(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


class Layer:
    def __init__(self, seed=0, most_tokens=512):
        from paper_2608_03579_amd import hip, salt
        self.hip, self.salt = hip, salt
        rng = np.random.default_rng(seed)
        hip.set_device(0)
        self.stream = hip.Stream()
        self.ctx = ctx = salt.Context("bf16", TABLES, DOMAINS, RANK_C, USERS, RANK_U, most_tokens)
        self.w, self.cent, self.res = [], [], []
        for t, (n_in, n_out) in enumerate(TABLES):
            bits, w = bf16(rng.standard_normal((n_in, n_out)) / np.sqrt(n_in))
            dev = hip.DeviceArray.from_host(bits)
            ctx.pin_base(t, dev.ptr, n_out, self.stream.h)
            self.stream.synchronize()
            dev.free()
            self.w.append(w)
            at, b = bf16(rng.standard_normal((DOMAINS, RANK_C, n_in)) / np.sqrt(n_in)), bf16(
                rng.standard_normal((DOMAINS, RANK_C, n_out)) * 0.1)
            ctx.pin_centroids(t, at[0], b[0])
            self.cent.append((at[1], b[1]))
        for u in range(USERS):
            parts = [(bf16(rng.standard_normal((RANK_U, i)) / np.sqrt(i)), bf16(rng.standard_normal((RANK_U, o)) * 0.1))
                     for i, o in TABLES]
            ctx.load_residual(u, RANK_U, np.concatenate([p[0].reshape(-1) for ab in parts for p in ab]))
            self.res.append([(a[1], b[1]) for a, b in parts])
        ctx.wait_loads()
        self.plan = ctx.plan()
        self.rotation = ctx.rotation(HEADS, KV_HEADS, DIM, FREQ)
        # one layer's cache; every user and every domain's prompt has pages of its own
        self.kv = ctx.kv_cache(1, HEADS, KV_HEADS, DIM, PAGE, 64)
        self.step_seqs = self.kv.seqs(USERS + DOMAINS, most_tokens, 64)
        free = list(rng.permutation(64))
        self.prompt_pages = [[free.pop() for _ in range(-(-n // PAGE))] for n in PROMPT]
        self.user_pages = [[free.pop() for _ in range(4)] for _ in range(USERS)]
        self.lengths = [0] * USERS
        self.history = {}                                        # float64 k, v by ("prompt", d) or user

    def run(self, x_bits, domain_of, user_of, q_len, length, pages, domain=None):
        """One step of the block for a batch of sequences; returns the output rows."""
        # positions of the new tokens: behind the domain's prompt
        base = [0 if domain is None else PROMPT[domain[i]] for i in range(len(q_len))]
        pos = np.concatenate([b + n - q + np.arange(q) for b, n, q in zip(base, length, q_len)]).astype(np.int32)
        hip, ctx, s, T = self.hip, self.ctx, self.stream.h, len(x_bits)
        x = hip.DeviceArray.from_host(x_bits)
        y = [hip.DeviceArray((T, n_out), np.uint16) for _, n_out in TABLES]
        att, at = hip.DeviceArray((T, HIDDEN), np.uint16), hip.DeviceArray.from_host(pos)
        self.plan.set_maps(domain_of, user_of, None, s)
        self.plan.build(s)
        off = np.concatenate([[0], np.cumsum([len(p) for p in pages])])
        pre_off = np.concatenate([[0], np.cumsum([len(p) for p in self.prompt_pages])])
        self.step_seqs.set(q_len, length, off, np.concatenate(pages), domain, PROMPT, pre_off,
                           np.concatenate(self.prompt_pages), s)
        # q, k and v read one x: one product, one apply
        ctx.base_product([Q, K, V], T, x.ptr, [y[t].ptr for t in (Q, K, V)], s)
        ctx.apply_batch([Q, K, V], self.plan, [x.ptr] * 3, [y[t].ptr for t in (Q, K, V)], s)
        ctx.rotate(self.rotation, T, at.ptr, y[Q].ptr, y[Q].ptr, y[K].ptr, y[K].ptr, s)
        self.step_seqs.write(0, y[K].ptr, y[V].ptr, s)
        self.step_seqs.attend(0, y[Q].ptr, att.ptr, DIM ** -0.5, s)
        ctx.base_product([O], T, att.ptr, [y[O].ptr], s)
        ctx.apply(O, self.plan, att.ptr, y[O].ptr, s)
        self.stream.synchronize()
        out = decode(y[O].to_host())
        for d in [x, att, at, *y]:
            d.free()
        return out

    # ---- the same in float64, without any 8-bit format --------------------------------
    def project(self, t, x, d, u):
        y = x @ self.w[t]
        at, b = self.cent[t]
        y = y + (x @ at[d].T) @ b[d]
        if u >= 0:
            a, r = self.res[u][t]
            y = y + (x @ a.T) @ r
        return y

    @staticmethod
    def rotate(x, pos):
        """Heads of x [rows][heads * DIM]: values i and i + DIM / 2 turn by pos * FREQ[i]."""
        v = x.reshape(len(x), -1, 2, DIM // 2)
        t = (pos[:, None] * FREQ)[:, None, :]
        a, b = v[:, :, 0], v[:, :, 1]
        return np.stack([a * np.cos(t) - b * np.sin(t), b * np.cos(t) + a * np.sin(t)], 2).reshape(x.shape)

    def reference(self, x, holder, prompt, d, u):
        """x: a sequence's new rows; holder: where its history is kept; prompt: None or a domain."""
        q, k, v = (self.project(t, x, d, u) for t in (Q, K, V))
        hk, hv = self.history.get(holder, (np.zeros((0, KV)),) * 2)
        before = len(hk)
        pos = (PROMPT[prompt] if prompt is not None else 0) + before + np.arange(len(x))
        q, k = self.rotate(q, pos), self.rotate(k, pos)
        hk, hv = np.concatenate([hk, k]), np.concatenate([hv, v])
        self.history[holder] = hk, hv
        pk, pv = self.history[("prompt", prompt)] if prompt is not None else (np.zeros((0, KV)),) * 2
        out = np.zeros((len(x), HIDDEN))
        for i in range(len(x)):
            kk, vv = np.concatenate([pk, hk[: before + i + 1]]), np.concatenate([pv, hv[: before + i + 1]])
            for h in range(HEADS):
                g = h // (HEADS // KV_HEADS)
                s = kk[:, g * DIM:(g + 1) * DIM] @ q[i, h * DIM:(h + 1) * DIM] * DIM ** -0.5
                p = np.exp(s - s.max())
                out[i, h * DIM:(h + 1) * DIM] = (p / p.sum()) @ vv[:, g * DIM:(g + 1) * DIM]
        return self.project(O, out, d, u)

    def close(self):
        self.plan.close()
        self.ctx.close()
        self.stream.destroy()


def main(steps=4, seed=0):
    """Relative 2-norm difference of the last step's output from float64 on unquantised values."""
    rng = np.random.default_rng([seed, 1])
    layer = Layer(seed)
    try:
        # the domains' prompts, once, under the centroid alone
        x = [bf16(rng.standard_normal((n, HIDDEN))) for n in PROMPT]
        layer.run(np.concatenate([b for b, _ in x]), np.repeat(np.arange(DOMAINS), PROMPT).astype(np.int32),
                  np.full(sum(PROMPT), -1, np.int32), PROMPT, PROMPT, layer.prompt_pages)
        for d in range(DOMAINS):
            layer.reference(x[d][1], ("prompt", d), None, d, -1)
        # the users: a prompt of their own each, then one token at a time
        domain = np.arange(USERS) % DOMAINS
        for step in range(steps):
            q_len = np.asarray([5 + 3 * u if step == 0 else 1 for u in range(USERS)])
            layer.lengths = [n + int(q) for n, q in zip(layer.lengths, q_len)]
            bits, x = bf16(rng.standard_normal((int(q_len.sum()), HIDDEN)))
            user = np.repeat(np.arange(USERS), q_len)
            pages = [p[: -(-n // PAGE)] for p, n in zip(layer.user_pages, layer.lengths)]
            got = layer.run(bits, domain[user].astype(np.int32), user.astype(np.int32), q_len, layer.lengths, pages, domain)
            want = np.concatenate([layer.reference(x[user == u], u, int(domain[u]), int(domain[u]), u)
                                   for u in range(USERS)])
            far = float(np.linalg.norm(got - want) / np.linalg.norm(want))
            print(f"step {step}: {len(x)} rows, {far:.4f} from float64 without 8-bit formats", flush=True)
        return far
    finally:
        layer.close()


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 4)
