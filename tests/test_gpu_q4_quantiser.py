"""The quantiser of the cache in 4 bits where it decides: ranges beside a tie of the scale, elements beside a tie of the code, and many
rows, bit for bit against numpy from the format's description in include/specpv.h."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests import q4_util as Q

pytestmark = pytest.mark.gpu

FIFTEENTH = np.float32(1) / np.float32(15)


def quantise(x):
    """Rows [.., d] of float32 -> codes, scale, offset, every step rounded as the description says."""
    x = np.asarray(x, dtype=np.float32)
    lo, hi = x.min(-1), x.max(-1)
    scale = Q.bf16((hi - lo) * FIFTEENTH)
    s = scale.astype(np.float32)
    offset = Q.bf16(lo - np.float32(16) * s)
    base = offset.astype(np.float32) + np.float32(16) * s
    with np.errstate(all="ignore"):
        n = np.rint((x - base[..., None]) / s[..., None])
    n = np.clip(np.nan_to_num(n, nan=0.0, posinf=15, neginf=0), 0, 15).astype(np.int64)
    bad = ~np.isfinite(x).all(-1)  # stored as NaN
    return n, np.where(bad, np.nan, scale), np.where(bad, np.nan, offset)


def codes_of(pages, bs, d):
    """Pages [.., bs (d + 8)] of bytes -> codes of keys and values [.., bs, d]."""
    lead = pages.shape[:-1]
    words = np.ascontiguousarray(pages[..., : bs * d]).view(np.uint32).reshape(*lead, 2, bs * d // 8).astype(np.uint64)
    bit = np.array([Q.element_bit(i) for i in range(8)], np.uint64)
    codes = ((words | words << np.uint64(32))[..., None] >> bit & np.uint64(15)).astype(np.int64)
    k = codes[..., 0, :, :].reshape(*lead, d // 32, bs, 32)
    v = codes[..., 1, :, :].reshape(*lead, bs // 16, d, 16)
    return np.swapaxes(k, -3, -2).reshape(*lead, bs, d), np.swapaxes(v, -2, -1).reshape(*lead, bs, d)


def check(k, v, bs):
    """k, v [tokens][Hkv][d] of float32, committed as a chunk to an empty cache."""
    n, Hkv, d = k.shape
    cfg = B.make_config(1, Hkv, Hkv, d, bs, "fp32", 1, 1, 4, 16)
    blocks = -(-n // bs)
    cache = B.CacheQ4(B.new_q4_pool(cfg, blocks), torch.arange(blocks, dtype=torch.int32, device="cuda")[None].contiguous(),
                      torch.zeros(1, dtype=torch.int32, device="cuda"), blocks * bs)
    kt, vt = (torch.from_numpy(x)[None, None].contiguous().cuda() for x in (k, v))
    kv, vv = torch.zeros_like(kt), torch.zeros_like(vt)
    ws = B.new_workspace(cfg, 1, 1, 64, 8)
    B.specpv_commit_accepted_q4(cfg, 0, 1, kt, vt, n, None, torch.tensor([n], dtype=torch.int32, device="cuda"), n, cache, None, None, kv,
                                vv, ws)
    assert B.specpv_poll_status(ws)[0] == 0 and cache.seq_lens.tolist() == [n]
    pool = cache.pool.cpu().numpy()[0]                                                      # [blocks][Hkv][bytes]
    codes = [np.swapaxes(c, 1, 2).reshape(blocks * bs, Hkv, d)[:n] for c in codes_of(pool, bs, d)]
    params = np.ascontiguousarray(pool[..., bs * d:]).view(np.uint16).reshape(blocks, Hkv, 4, bs).transpose(0, 3, 1, 2)
    params = params.reshape(blocks * bs, Hkv, 4)[:n]
    for x, got, seen, at in ((k, codes[0], kv, 0), (v, codes[1], vv, 2)):
        want, scale, offset = quantise(x)
        assert np.array_equal(Q.from_bits(params[..., at]), scale, equal_nan=True)
        assert np.array_equal(Q.from_bits(params[..., at + 1]), offset, equal_nan=True)
        some = np.isfinite(scale)  # (a row of NaN has no codes to speak of)
        assert np.array_equal(got[some], want[some])
        assert np.array_equal(seen[0, 0].cpu().double().numpy(), Q.values(want, scale, offset), equal_nan=True)


def beside(x, steps):
    """Neighbours of float32 values: `steps` last places away."""
    return (np.asarray(x, np.float32).view(np.int32) + np.asarray(steps, np.int32)).view(np.float32)


@pytest.mark.parametrize("d,bs", [(64, 16), (128, 64)])
def test_ranges_beside_a_tie_of_the_scale(d, bs):
    """Ranges whose fifteenth lies within a few last places of half-way between two bfloat16 numbers."""
    rng = np.random.default_rng(d)
    n, Hkv = 1500, 4
    half = (256 + rng.integers(0, 256, (2, n, Hkv)) // 2 * 2 + 1) / 256.0  # odd numerators of nine bits: ties
    tie = (15.0 * half * np.exp2(rng.integers(-20, 20, half.shape).astype(np.float64))).astype(np.float32)
    reach = beside(tie, rng.integers(-3, 4, tie.shape))
    x = (rng.random((2, n, Hkv, d)) * reach[..., None]).astype(np.float32)
    x[..., 5], x[..., d - 1] = 0.0, reach  # the row's ends
    x = np.minimum(x, reach[..., None])
    check(x[0], x[1], bs)


@pytest.mark.parametrize("d,bs", [(64, 16), (128, 64)])
def test_elements_beside_a_tie_of_the_code(d, bs):
    """Elements within a few last places of half-way between two codes (a last place below zero is NaN: such rows are among them)."""
    rng = np.random.default_rng(d + 1)
    n, Hkv = 1500, 4
    x = (rng.standard_normal((2, n, Hkv, d)) * np.exp(rng.standard_normal((2, n, Hkv, 1)))).astype(np.float32)
    _, scale, offset = quantise(x)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    at = (offset + 16 * scale)[..., None] + (rng.integers(0, 15, x.shape) + 0.5) * scale[..., None]
    y = beside(at.astype(np.float32), rng.integers(-2, 3, x.shape))
    ends = (x == lo) | (x == hi) | (y <= lo) | (y >= hi)  # the row's range stays what it is
    check(*np.where(ends, x, y), bs)


@pytest.mark.parametrize("d,bs", [(64, 32), (128, 64)])
def test_many_rows(d, bs):
    """Rows enough for ranges to meet ties of the scale by chance (about one in 85000)."""
    rng = np.random.default_rng(d + 2)
    x = rng.standard_normal((2, 25000, 8, d), dtype=np.float32)
    x *= 1 + 2 * (rng.random((2, 25000, 8, 1)) < 0.02).astype(np.float32)
    check(x[0], x[1], bs)
