"""Plain reference of the paged calls, on the CPU: quantisation in IEEE
binary32 as the header defines it, everything else in 64 bits, one sequence at
a time.  Test infrastructure; shares no code with the library."""
import math

import numpy as np
import torch


def bf16_bits(x: np.ndarray) -> np.ndarray:
    """binary32 -> bf16 bits, nearest even (finite values)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint32)


def from_bf16(b: np.ndarray) -> np.ndarray:
    return (b.astype(np.uint32) << 16).view(np.float32)


def quantise(x: np.ndarray, group: int):
    """x [..., D] float32 -> codes [..., D] uint8, words [..., D/group] uint32."""
    x = np.where(np.isnan(x), np.float32(0), x).astype(np.float32)
    x = np.clip(x, np.float32(-2.0 ** 126), np.float32(2.0 ** 126))
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    mb = bf16_bits(g.min(-1))
    m = from_bf16(mb)
    span = np.maximum(g.max(-1) - m, np.float32(0))
    step = (span / np.float32(15)).astype(np.float32).view(np.uint32)
    step = (step + np.uint32(0x000FFFFF)) & np.uint32(0xFFF00000)
    s = step.view(np.float32)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(s > 0, np.clip(np.rint((g - m[..., None]) / s), 0, 15), 0)
    return q.reshape(x.shape).astype(np.uint8), (step >> 16) | (mb << 16)


def values(codes: np.ndarray, words: np.ndarray) -> np.ndarray:
    """The values that codes and words stand for, in 64 bits."""
    g = codes.reshape(words.shape + (codes.shape[-1] // words.shape[-1],)).astype(np.float64)
    s = from_bf16(words & 0xFFFF).astype(np.float64)[..., None]
    m = from_bf16(words >> 16).astype(np.float64)[..., None]
    return (g * s + m).reshape(codes.shape)


def key_order(D: int) -> np.ndarray:
    """Channel held by each nibble of a row of key codes."""
    n = np.arange(D)
    w, e = n // 8, n % 8
    return 32 * (w % (D // 32)) + 8 * (w // (D // 32)) + e


def pack(codes: np.ndarray) -> np.ndarray:
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(b: np.ndarray) -> np.ndarray:
    return np.stack((b & 15, b >> 4), -1).reshape(b.shape[:-1] + (2 * b.shape[-1],))


class Cache:
    """A cache's arrays on the host, filled by the rules of the header."""

    def __init__(self, n_pages, P, Hkv, D, group, seed=0):
        r = np.random.default_rng(seed)  # what nobody wrote: anything, words that are not finite among it
        self.P, self.D, self.group, self.Hkv, self.n_pages = P, D, group, Hkv, n_pages
        self.ck, self.cv = (r.integers(0, 256, (n_pages, Hkv, P, D // 2), dtype=np.uint8) for _ in range(2))
        self.sk, self.sv = (r.integers(0, 1 << 32, (n_pages, Hkv, P, D // group), dtype=np.uint32) for _ in range(2))
        self.sk[..., 0] |= 0x7FC07FC0
        self.sv[..., 0] |= 0x7FC07FC0

    def device(self, uc):
        return uc.PageCache(*(torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a.copy()).cuda().contiguous()
                              for a in (self.ck, self.cv, self.sk, self.sv)))

    def append(self, k, v, slots):
        """k, v [T, Hkv, D] float32."""
        order = key_order(self.D)
        for t, s in enumerate(slots):
            if s < 0 or s // self.P >= self.n_pages:
                continue
            p, r = divmod(int(s), self.P)
            qk, wk = quantise(k[t], self.group)
            qv, wv = quantise(v[t], self.group)
            self.ck[p, :, r], self.cv[p, :, r] = pack(qk[:, order]), pack(qv)
            self.sk[p, :, r], self.sv[p, :, r] = wk, wv

    def copy(self, copies):
        for a, b, n in copies:
            if a >= 0:
                for x in (self.ck, self.cv, self.sk, self.sv):
                    x[b, :, :n] = x[a, :, :n]

    def rows(self, slots):
        """Values of the slots: k, v [T, Hkv, D] in 64 bits."""
        p, r = np.asarray(slots) // self.P, np.asarray(slots) % self.P
        back = np.empty(self.D, np.int64)
        back[key_order(self.D)] = np.arange(self.D)
        return (values(unpack(self.ck[p, :, r])[..., back], self.sk[p, :, r]),
                values(unpack(self.cv[p, :, r]), self.sv[p, :, r]))


def slots_of(table_row, n, P):
    j = np.arange(n)
    return np.asarray(table_row)[j // P].astype(np.int64) * P + j % P


def attend(cache, q, q_start, lens, table, scale):
    """q [T, Hq, D] float64 -> o [T, Hq, D], lse [T, Hq] (rows of no sequence: NaN)."""
    T, Hq, D = q.shape
    G = Hq // cache.Hkv
    o, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    for s, n_rows in enumerate(lens):
        a, b = int(q_start[s]), int(q_start[s + 1])
        if b <= a:
            continue
        k, v = cache.rows(slots_of(table[s], n_rows, cache.P)) if n_rows else (np.zeros((0, cache.Hkv, D)),) * 2
        for i in range(b - a):
            sees = max(0, n_rows - (b - a) + i + 1)
            for h in range(Hq):
                if sees == 0:
                    o[a + i, h], lse[a + i, h] = 0, -np.inf
                    continue
                x = k[:sees, h // G] @ q[a + i, h] * scale
                m = x.max()
                p = np.exp(x - m)
                o[a + i, h] = p @ v[:sees, h // G] / p.sum()
                lse[a + i, h] = m + math.log(p.sum())
    return o, lse


def sizes(cache, q, q_start, lens, table, scale, lse, unit):
    """What a row's errors are measured by: sum_j p_j M_j per channel, with M_j
    the largest size in the channel's group of value j, and the same sums of
    d_j (lse's error) and d_j M_j, where d_j = unit * scale * sum |q| M'_j, M'_j
    likewise of key j, is the error of a logit and p_j is taken with it."""
    T, Hq, D = q.shape
    G = Hq // cache.Hkv
    size, d_size, d_lse = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for s, n_rows in enumerate(lens):
        a, b = int(q_start[s]), int(q_start[s + 1])
        if b <= a or n_rows == 0:
            continue
        k, v = cache.rows(slots_of(table[s], n_rows, cache.P))
        most = []
        for x in (k, v):
            g = np.abs(x).reshape(n_rows, cache.Hkv, D // cache.group, cache.group)
            most.append(np.broadcast_to(g.max(-1, keepdims=True), g.shape).reshape(x.shape))
        for i in range(b - a):
            sees = max(0, n_rows - (b - a) + i + 1)
            for h in range(Hq if sees else 0):
                x = k[:sees, h // G] @ q[a + i, h] * scale
                d = most[0][:sees, h // G] @ np.abs(q[a + i, h]) * scale * unit
                p = np.exp(np.minimum(x + d - lse[a + i, h], 0))
                size[a + i, h], d_lse[a + i, h] = p @ most[1][:sees, h // G], p @ d
                d_size[a + i, h] = (p * np.minimum(d, 1)) @ most[1][:sees, h // G]
    return size, d_size, d_lse


def free_pages(table, lens, P, n_pages):
    held = {int(p) for row, n in zip(table, lens) for p in row[:min(-(-max(int(n), 0) // P), len(row))]}
    return [p for p in range(n_pages) if p not in held]


def step(lens, new, table, P, n_pages, free, pool, n_slots):
    """-> table, len_out, q_start, slots, pool_out, refused."""
    table = np.array(table)
    left = max(min(pool[1], n_pages) - pool[0], 0)
    pages = tokens = taken = 0
    len_out, start, slots, refused = [], [0], [-1] * n_slots, []
    for s, (n, k) in enumerate(zip(lens, new)):
        n, k = max(int(n), 0), max(int(k), 0)
        need = -(-(n + k) // P) - -(-n // P)
        pages, tokens = pages + need, tokens + k
        ok = (need == 0 or pages <= left) and -(-(n + k) // P) <= table.shape[1] and tokens <= n_slots
        if ok:
            held = -(-n // P)
            table[s, held:held + need] = free[pool[0] + pages - need:pool[0] + pages]
            for i in range(k):
                p = table[s, (n + i) // P]
                slots[tokens - k + i] = p * P + (n + i) % P if 0 <= p < n_pages else -1
            taken = max(taken, pages) if need else taken
        start.append(min(tokens, n_slots))
        len_out.append(n + k if ok else n)
        refused.append(not ok)
    return table, len_out, start, slots, [pool[0] + taken, pool[1]], refused


def beam_select(logits, score, done, eos, pad):
    """float64 [R, W, V] -> score, parent, token, done."""
    R, W, V = logits.shape
    out = []
    for r in range(R):
        with np.errstate(all="ignore"):
            x = np.where(np.isnan(logits[r]), -np.inf, logits[r])
            m = x.max(-1, keepdims=True)
            t = score[r][:, None] + ((x - m) - np.log(np.exp(x - m).sum(-1, keepdims=True)))
        for b in range(W):
            if done[r, b]:
                t[b] = -np.inf
                t[b, pad] = score[r, b]
            elif not np.isfinite(m[b]).all() or not np.isfinite(score[r, b]):
                t[b] = -np.inf
        t = np.where(np.isfinite(t), t, -np.inf).reshape(-1)
        best = np.argsort(-t, kind="stable")[:W]
        par, tok = best // V, best % V
        out.append((t[best], par, tok, (done[r][par] != 0) | (tok == eos)))
    return [np.stack([o[i] for o in out]) for i in range(4)]


def beam_reorder(parent, table, lens, P):
    """-> the table's entries that hold rows (others as they are), copies."""
    R, W = parent.shape
    out, copies = np.array(table), np.tile(np.array([-1, -1, 0]), (R * W, 1))
    for r in range(R):
        n = int(lens[r * W])
        full, part = n // P, n % P
        lost = [b for b in range(W) if b not in set(parent[r].tolist())]
        seen = set()
        for b in range(W):
            p = int(parent[r, b])
            out[r * W + b, :full] = table[r * W + p, :full]
            if part:
                out[r * W + b, full] = table[r * W + p, full]
                if p in seen:
                    out[r * W + b, full] = table[r * W + lost.pop(0), full]
                    copies[r * W + b] = table[r * W + p, full], out[r * W + b, full], part
            seen.add(p)
    return out, copies
