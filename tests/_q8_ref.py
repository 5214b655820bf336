"""The paged 8-bit cache in 64 bits, written from its definition (numpy; not
collected by pytest). Pages are kept as the values they stand for."""
from __future__ import annotations

import numpy as np
import torch

TOP = 448.0


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value of |y| <= 448, ties to the even one: four significant bits,
    steps of 2^-9 below 2^-6. NaN stays."""
    y = np.asarray(y, dtype=np.float64)
    _, x = np.frexp(np.where(np.isfinite(y), y, 0.0))        # |y| = m 2^x, m in [0.5, 1)
    step = np.exp2(np.maximum(x - 4, -9).astype(np.float64))
    return np.rint(y / step) * step                          # rint: ties to even


def exponent(amax: float) -> int:
    """The smallest e >= -126 with amax <= 448 * 2^e."""
    e = -126
    while amax > TOP * 2.0 ** e:
        e += 1
    return e


def allocate(old, new, B, tables, stack, rows=0, n_slots=0):
    """block_tables on lists: ``tables`` and ``stack`` (top last) are changed."""
    gone = []
    for s in range(len(old)):
        for j in range(-(-new[s] // B), -(-old[s] // B)):
            gone.append(tables[s][j])
            tables[s][j] = -1
    stack.extend(reversed(gone))
    slots, cu = [], [0]
    for s in range(len(old)):
        for j in range(-(-old[s] // B), -(-new[s] // B)):
            tables[s][j] = stack.pop()
        got = [tables[s][p // B] * B + p % B for p in range(old[s], new[s])]
        slots += got + [-1] * (rows - len(got)) if rows else got
        cu.append(cu[-1] + len(got))
    return slots + [-1] * (n_slots - len(slots)), cu, [x - 1 for x in new]


class Pool:
    """Keys and values [page][head][place][d] as stored values, exponents [page][head]."""

    def __init__(self, n_pages, h, B, d):
        self.B = B
        self.x = {n: np.zeros((n_pages, h, B, d)) for n in "kv"}
        self.e = {n: np.full((n_pages, h), -127, dtype=np.int64) for n in "kv"}

    def append(self, k, v, slots):
        """k, v [h][N][d] float64; slots [N]. Later tokens win over earlier ones."""
        pages = {}
        for i, sl in enumerate(slots):
            if 0 <= sl < self.x["k"].shape[0] * self.B:
                pages.setdefault(sl // self.B, {})[sl % self.B] = i
        for pg, places in pages.items():
            off, tok = list(places), list(places.values())
            for n, x in (("k", k), ("v", v)):
                for h in range(x.shape[0]):
                    new = x[h, tok]
                    fin = np.abs(new[np.isfinite(new)])
                    e = exponent(fin.max() if fin.size else 0.0)
                    if 0 not in places:
                        old = self.e[n][pg, h]
                        e = max(e, old)
                        if e > old:
                            self.x[n][pg, h] = round_e4m3(self.x[n][pg, h] / 2.0 ** e) * 2.0 ** e
                    self.e[n][pg, h] = e
                    put = np.where(np.isfinite(new), new, np.nan)
                    self.x[n][pg, h, off] = round_e4m3(put / 2.0 ** e) * 2.0 ** e

    def tokens(self, n, table, positions):
        """Stored values [h][len][d] of a sequence's positions (0 without a page)."""
        out = np.zeros((self.x[n].shape[1], len(positions), self.x[n].shape[3]))
        for i, p in enumerate(positions):
            j = p // self.B
            if j < len(table) and 0 <= table[j] < self.x[n].shape[0]:
                out[:, i] = self.x[n][table[j], :, p % self.B]
        return out


def cache_values(cache, layer=None):
    """The stored values of a device cache: k, v [page][head][place][d] and exponents."""
    c = cache if layer is None else {n: t[layer] for n, t in cache.items()}
    e = {n: c[n + "_scale"].cpu().numpy().astype(np.int64) - 127 for n in "kv"}
    k = c["k"].cpu().float().numpy().astype(np.float64)
    v = c["v"].cpu().float().numpy().astype(np.float64).transpose(0, 1, 3, 2)
    return {"k": k * np.exp2(e["k"].astype(np.float64))[..., None, None],
            "v": v * np.exp2(e["v"].astype(np.float64))[..., None, None]}, e


def attention(q, K, V, scale):
    """q [h_q][d], K, V [h_kv][T][d] in 64 bits -> (o, a, top): the output, the weighted
    mean of |v| (what rounded weights are off by a share of) and each head's largest
    sum of |q_i k_i| times the scale (what a rounded logit is off by a share of)."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    G = q.shape[0] // K.shape[0]
    o, a, top = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[0])
    for u in range(q.shape[0]):
        k, v = K[u // G], V[u // G]
        if k.shape[0] == 0:
            continue
        s = k @ q[u] * scale
        w = np.exp(s - s.max())
        w /= w.sum()
        o[u], a[u] = w @ v, w @ np.abs(v)
        top[u] = (np.abs(k) @ np.abs(q[u])).max() * scale
    return o, a, top


def attention_bound(dtype, o, a, top, d, T):
    """How far the kernel's output may be from ``attention``'s.

    A logit is a sum of d products in 32 bits, times two factors: off by at most
    (d + 4) 2^-24 of sum |q_i k_i|, which counts twice (in the weight and in the sum
    it is divided by), as do the rounding of the exponential's argument (the same
    factor covers it) and 4 ulp of the exponential. Sums over tokens: a wavefront adds at most
    T / 64 + 1 groups of 64, which one matrix instruction adds 32 of, then the merge
    adds up to 4 * 32 partial sums: T / 64 + 200 additions of 2^-24. bf16 weights: half a
    step, 2^-8; the output's own rounding 2^-8 of it (2^-24 in 32 bits). Values below
    1e-30 are left out of consideration."""
    u = 2.0 ** -24
    share = 2 * (d + 8) * u * top[:, None] + (8 + T / 64 + 200) * u
    if dtype == torch.bfloat16:
        return (share + 2.0 ** -8) * a * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(o) + 1e-30
    return share * a + u * np.abs(o) + 1e-30
