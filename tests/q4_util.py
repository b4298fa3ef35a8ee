"""The cache in 4 bits in numpy, element by element from its description in include/specpv.h, and the attention, the account of
attention weight and the eviction in 64 bits.  Shares no code with the library."""
from __future__ import annotations

import numpy as np
import torch

HALF_BF16, HALF_F32 = 2.0 ** -8, 2.0 ** -24  # half a step, relative


def bf16(x) -> np.ndarray:
    """Nearest bfloat16 of float64 values, ties to even (rounded once), as float64."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        m, e = np.frexp(x)
        step = np.ldexp(1.0, np.maximum(e, -125) - 8)  # eight significant bits, down to the subnormals
        y = np.rint(x / step) * step
        y = np.where(np.abs(y) > 3.3895313892515355e38, np.sign(y) * np.inf, y)
    return np.where(np.isfinite(x), y, x)


def bf16_bits(x) -> np.ndarray:
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).float().bfloat16().view(torch.int16).numpy().view(np.uint16)


def from_bits(b) -> np.ndarray:
    return (np.asarray(b).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def quantise(x):
    """Rows [.., d] (float64 holding what the library is given) -> codes, scale, offset (float64 holding bfloat16)."""
    x32 = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        lo, hi = x32.min(-1), x32.max(-1)
        scale = bf16((hi - lo) / np.float32(15))
        s = scale.astype(np.float32)
        offset = bf16((lo.astype(np.float64) - 16 * scale).astype(np.float32))
        base = offset.astype(np.float32) + np.float32(16) * s
        n = np.rint((x32 - base[..., None]) / s[..., None])
    bad = ~(np.isfinite(x32).all(-1) & np.isfinite(scale) & np.isfinite(offset) & np.isfinite(base))
    n = np.clip(np.nan_to_num(n, nan=0.0, posinf=15, neginf=0), 0, 15).astype(np.int64)
    n[bad] = 0
    return n, np.where(bad, np.nan, scale), np.where(bad, np.nan, offset)


def values(n, scale, offset):
    with np.errstate(all="ignore"):
        return bf16((16.0 + n) * np.asarray(scale)[..., None] + np.asarray(offset)[..., None])


def element_bit(i):
    return (4 * (i // 2) + 16 * (i % 2) + 3) % 32


def read_page(raw: np.ndarray, bs: int, d: int):
    """One page of one KV head -> key codes, value codes [bs][d] and parameters [4][bs]."""
    words = raw[: bs * d].view(np.uint32)
    k, v = np.zeros((bs, d), np.int64), np.zeros((bs, d), np.int64)

    def field(w, i):
        w = int(w)
        return ((w | w << 32) >> element_bit(i)) & 15

    for t in range(bs):
        for c in range(d):
            k[t, c] = field(words[((c // 32) * bs + t) * 4 + c % 32 // 8], c % 8)
            v[t, c] = field(words[bs * d // 8 + ((t // 16) * d + c) * 2 + t % 16 // 8], t % 8)
    return k, v, from_bits(raw[bs * d:].view(np.uint16)).reshape(4, bs)


def write_page(k, v, params) -> np.ndarray:
    """The inverse of read_page; params [4][bs] as bfloat16 bits."""
    bs, d = k.shape
    t, c = np.meshgrid(np.arange(bs), np.arange(d), indexing="ij")
    words = np.zeros(bs * d // 4, np.uint64)
    bit = np.array([element_bit(i) for i in range(8)], np.uint64)

    def put(at, n, e):
        x = n.astype(np.uint64) << bit[e]
        np.bitwise_or.at(words, at, (x | x >> np.uint64(32)) & np.uint64(0xFFFFFFFF))

    put(((c // 32) * bs + t) * 4 + c % 32 // 8, k, c % 8)
    put(bs * d // 8 + ((t // 16) * d + c) * 2 + t % 16 // 8, v, t % 8)
    return np.concatenate([words.astype(np.uint32).view(np.uint8), np.ascontiguousarray(params).reshape(-1).view(np.uint8)])


class Q4:
    """A cache in 4 bits of random rows for given lengths: the pool for the library and the values for the reference.  Everything
    that no sequence holds is filled with ones (NaN as a scale)."""

    def __init__(self, layers, Hkv, d, bs, lens, seed=0, shuffle=True, spare=1, max_blocks=None, amplitude=1.0):
        rng = np.random.default_rng(seed)
        self.layers, self.Hkv, self.d, self.bs, self.lens = layers, Hkv, d, bs, list(lens)
        batch = len(lens)
        self.max_blocks = max_blocks or max(max(-(-n // bs) for n in lens), 1)
        n_pages = batch * self.max_blocks + spare
        order = rng.permutation(n_pages) if shuffle else np.arange(n_pages)
        self.table = order[: batch * self.max_blocks].reshape(batch, -1).astype(np.int32)
        self.pool = np.full((layers, n_pages, Hkv, bs * (d + 8)), 0xFF, np.uint8)
        self.k = [np.zeros((layers, Hkv, n, d)) for n in lens]
        self.v = [np.zeros((layers, Hkv, n, d)) for n in lens]
        for b, n in enumerate(lens):
            for i in range(-(-n // bs)):
                held = min(bs, n - i * bs)
                for l in range(layers):
                    for h in range(Hkv):
                        loud = amplitude * np.where(rng.random((held, 1)) < 0.1, 3.0, 1.0)
                        kc, ks, ko = quantise(bf16(rng.standard_normal((held, d)) * loud))
                        vc, vs, vo = quantise(bf16(rng.standard_normal((held, d)) * loud))
                        self.k[b][l, h, i * bs: i * bs + held] = values(kc, ks, ko)
                        self.v[b][l, h, i * bs: i * bs + held] = values(vc, vs, vo)
                        full = [np.full((bs, d), 15) for _ in range(2)]
                        full[0][:held], full[1][:held] = kc, vc
                        par = np.full((4, bs), 0xFFFF, np.uint16)
                        for j, x in enumerate((ks, ko, vs, vo)):
                            par[j, :held] = bf16_bits(x)
                        self.pool[l, self.table[b, i], h] = write_page(*full, par)

    def cache(self, B, device="cuda", max_seq_len=None):
        return B.CacheQ4(torch.from_numpy(self.pool).to(device), torch.from_numpy(self.table).to(device),
                         torch.tensor(self.lens, dtype=torch.int32, device=device), max(self.lens) if max_seq_len is None else max_seq_len)


def attention(q, k, v, kn, vn, seen, G, scale):
    """q [M][Hq][d], k, v [Hkv][n][d], kn, vn [M][Hkv][d], seen [M][M] -> out [M][Hq][d], lse [M][Hq], the weighted mean of |v| and
    a bound of |error of a score| / 2^-23: the sum of |q k| over the channels, which are summed in float32."""
    M, Hq, d = q.shape
    n = k.shape[1]
    out, lse = np.zeros((M, Hq, d)), np.full((M, Hq), -np.inf)
    mean_abs, slack = np.zeros((M, Hq, d)), np.zeros((M, Hq))
    for h in range(Hq):
        kk = np.concatenate([k[h // G], kn[:, h // G]])
        vv = np.concatenate([v[h // G], vn[:, h // G]])
        see = np.concatenate([np.ones((M, n), bool), seen], 1)
        for j in range(M):
            at = see[j]
            if not at.any():
                continue
            with np.errstate(all="ignore"):
                s = kk[at] @ q[j, h] * scale
                slack[j, h] = (np.abs(kk[at]) @ np.abs(q[j, h])).max() * scale
                top = s.max()
                w = np.exp(s - top)
                lse[j, h] = top + np.log(w.sum())
                w /= w.sum()
                out[j, h] = w @ vv[at]
                mean_abs[j, h] = w @ np.abs(vv[at])
    return out, lse, mean_abs, slack
