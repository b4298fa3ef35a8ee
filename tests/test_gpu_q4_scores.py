"""Attention over a cache in 4 bits where scores, rows or values leave the ordinary: huge scores, NaN, infinities of no weight."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests import q4_util as Q
from tests.test_gpu_q4 import config, random_masks, rows, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M", [1, 4, 8, 20])
def test_parts_of_a_long_cache_weigh_what_their_scores_say(M, d):
    """Scores of 5600 whose differences across the cache are a few units: parts of the cache are weighed by their references' difference,
    and rounding a reference of that size costs 2e-4 of a weight.  Everything is exact here: keys are whole numbers up to 15 (scale 1),
    the softmax scale makes scores whole powers of two's logarithms, so weights are powers of two."""
    rng = np.random.default_rng(M + d)
    Hq, Hkv, bs, n = 8, 2, 64, 5000
    cfg = config(1, Hq, Hkv, d, bs, "bf16", out_f32=1, softmax_scale=float(np.float32(np.log(2.0))))
    assert np.float32(cfg.softmax_scale) * np.float32(1.4426950408889634) == 1
    blocks = -(-n // bs)
    cache = B.CacheQ4(B.new_q4_pool(cfg, blocks), torch.randperm(blocks)[None].int().cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                      blocks * bs)
    key = rng.integers(0, 16, (n, Hkv, d)).astype(np.float64)
    key[..., 0], key[..., d - 1] = 15, 0               # the row's range: scale 1, offset -16
    key[..., 1] = (rng.integers(3, 15, (blocks, Hkv))).repeat(bs, 0)[:n]  # what tells tokens apart goes by the page
    value = rng.integers(0, 16, (blocks, Hkv, d)).repeat(bs, 0)[:n].astype(np.float64)
    value[..., 0], value[..., d - 1] = 15, 0
    ws = B.new_workspace(cfg, 1, 1, blocks * bs, M)
    k, v = (torch.from_numpy(x)[None, None].bfloat16().cuda().contiguous() for x in (key, value))
    kv, vv = torch.zeros_like(k), torch.zeros_like(v)
    B.specpv_commit_accepted_q4(cfg, 0, 1, k, v, n, None, torch.tensor([n], dtype=torch.int32, device="cuda"), n, cache, None, None, kv, vv, ws)
    assert torch.equal(k, kv) and torch.equal(v, vv)
    q64 = np.zeros((1, 1, M, Hq, d))
    q64[..., 0], q64[..., 1] = 544, rng.choice([1.0, 0.5, -1.0], (1, 1, M, Hq))
    q = torch.from_numpy(q64).bfloat16().cuda()
    _, mask = random_masks(rng, 1, M, 0.0)             # of the step's tokens nothing is seen
    new = torch.zeros(1, 1, M, Hkv, d, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros(1, 1, M, Hq, d, device="cuda"), torch.zeros(1, 1, M, Hq, device="cuda")
    B.specpv_verify_full_q4(cfg, 0, 1, q, new, new, mask, None, M, cache, out, lse, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    out, lse = out.cpu().double().numpy()[0, 0], lse.cpu().double().numpy()[0, 0]
    for j in range(M):
        for h in range(Hq):
            s = key[:, h // 4] @ q64[0, 0, j, h]
            w = np.exp2(s - s.max())
            want = w @ value[:, h // 4] / w.sum()
            # weights are powers of two or (half units) off by 2^-8 in bfloat16, of either sign, over 64 tokens of a page and more; numerator
            # and denominator are sums in float32 of 5000 numbers, 2^-23 of each 64 tokens
            half = q64[0, 0, j, h, 1] == 0.5
            assert np.all(np.abs(out[j, h] - want) <= (2.0 ** -16 + (Q.HALF_BF16 if half else 0)) * want), (j, h)
            # a reference times ln 2 (half a step of each), the logarithm, their sum
            top = s.max() * np.log(2.0)
            assert abs(lse[j, h] - (top + np.log(w.sum()))) <= 2 * 2.0 ** -23 * top


@pytest.mark.parametrize("dtype,M", [("bf16", 1), ("bf16", 2), ("bf16", 4), ("bf16", 20), ("bf16", 40), ("fp32", 3)])
@pytest.mark.parametrize("log2_q", [28, 29, 33, 60, 100])
def test_scores_far_past_the_whole_numbers_of_float32(dtype, M, log2_q):
    """Scores of 2^26 to 2^100, whose neighbours in float32 lie 8 to 2^77 apart: references climb from tile to tile and come to rest.  A query
    is a power of two in one channel, and the key value of that channel decides: a row is the mean of the values of its largest keys,
    wherever they are."""
    rng = np.random.default_rng(log2_q + M)
    # every sequence over the same pages; warps go from chunk to chunk, CTAs from tile to tile
    Hq, Hkv, d, bs, n, batch = 32, 8, 64, 64, 3000, 24 if M < 8 else 4
    cfg = config(1, Hq, Hkv, d, bs, dtype, out_f32=1)
    q4 = Q.Q4(1, Hkv, d, bs, [n], seed=3)
    cache = q4.cache(B)
    cache.block_table = cache.block_table.expand(batch, -1).contiguous()
    cache.seq_lens = cache.seq_lens.expand(batch).contiguous()
    q64 = np.zeros((1, batch, M, Hq, d))
    channel = rng.integers(0, d, (batch, M, Hq))
    np.put_along_axis(q64[0], channel[..., None], 2.0 ** log2_q * rng.choice([-1.0, 1.0], (batch, M, Hq, 1)), -1)
    q = torch.from_numpy(q64).to(torch_dtype(dtype)).cuda()
    k, k64 = rows(rng, (1, batch, M, Hkv, d), "bf16")
    v, v64 = rows(rng, (1, batch, M, Hkv, d), "bf16")
    k, v = k.to(q.dtype), v.to(q.dtype)
    seen, mask = random_masks(rng, batch, M)
    out, lse = torch.zeros(1, batch, M, Hq, d, device="cuda"), torch.zeros(1, batch, M, Hq, device="cuda")
    ws = B.new_workspace(cfg, 1, batch, n, M)
    B.specpv_verify_full_q4(cfg, 0, 1, q, k, v, mask, None, M, cache, out, lse, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    out, lse = out.cpu().double().numpy()[0], lse.cpu().double().numpy()[0]
    for b in range(batch):
        for h in range(Hq):
            kk, vv = (np.concatenate([x[0][0, h // 4], y[0, b, :, h // 4]]) for x, y in ((q4.k, k64), (q4.v, v64)))
            for j in range(M):
                there = np.concatenate([np.ones(n, bool), seen[b, j]])
                s = kk[:, channel[b, j, h]] * q64[0, b, j, h, channel[b, j, h]] / 8
                top = s[there].max()
                w = np.where(there & (s == top), 1.0, 0.0)  # (the next key, 2^-8 of it or more below, weighs exp(-2^18) or less)
                want = w @ vv / w.sum()
                # equal scores, rounded alike: weights of 1, sums of a few values in float32.  Each of the other parts of the cache, 64 at most,
                # weighs 2^-149 (so that infinite values come through) of sums of at most 3000 values of weight 2^16: 2^-149 2^6 2^12 2^16
                assert np.all(np.abs(out[b, j, h] - want) <= 2.0 ** -20 * (w @ np.abs(vv) / w.sum()) + 2.0 ** -115 * np.abs(vv).max())
                # the score: scaled by a float32 factor and back, three roundings, which also hold the logarithm
                assert abs(lse[b, j, h] - (top + np.log(w.sum()))) <= 2.0 ** -21 * np.abs(top)


def verify(dtype, Hq, Hkv, d, q4, q, k, v, mask, M, out_f32=0):
    cfg = config(1, Hq, Hkv, d, q4.bs, dtype, out_f32=out_f32)
    out = torch.full((1, 1, M, Hq, d), 7.0, dtype=torch.float32 if out_f32 else torch_dtype(dtype), device="cuda")
    lse = torch.full((1, 1, M, Hq), 7.0, device="cuda")
    ws = B.new_workspace(cfg, 1, 1, max(q4.lens), M)
    B.specpv_verify_full_q4(cfg, 0, 1, q, k, v, mask, None, M, q4.cache(B), out, lse, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    return out[0, 0].cpu(), lse[0, 0].cpu()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M", [1, 3, 20])
@pytest.mark.parametrize("where", ["q", "k", "cache"])
def test_nan_among_the_parts_of_a_long_cache(dtype, d, M, where):
    """A cache long enough to be split many times: a NaN that is all that one of the parts sees is not left out when they meet."""
    rng = np.random.default_rng(d + M)
    Hq, Hkv, n = 8, 2, 2000
    q4 = Q.Q4(1, Hkv, d, 64, [n], seed=2)
    q, _ = rows(rng, (1, 1, M, Hq, d), dtype)
    k, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    v, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    seen, mask = random_masks(rng, 1, M, 0.0)
    seen[0, range(M), range(M)] = True  # every row sees itself alone
    mask = torch.zeros_like(mask)
    for j in range(M):
        mask[0, j, j // 64] = 1 << (j % 64)
    clean, clean_lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, mask, M)
    assert clean.isfinite().all() and clean_lse.isfinite().all()
    hit = torch.zeros(M, Hq, dtype=torch.bool)
    if where == "q":
        q[0, 0, M - 1, 3, 5] = float("nan")
        hit[M - 1, 3] = True
    elif where == "k":
        k[0, 0, M - 1, 1, 5] = float("nan")
        hit[M - 1, 4:] = True
    else:  # a cached key that was stored as NaN: all rows of its KV head see it
        par = q4.pool[0, q4.table[0, 7], 0, 64 * d:].view(np.uint16).reshape(4, 64)
        par[:2, 9] = 0x7FC0
        hit[:, :4] = True
    out, lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, mask, M)
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M,n", [(1, 2000), (3, 2000), (20, 2000), (100, 200), (100, 2000)])
def test_infinite_values_of_hardly_any_weight(dtype, d, M, n):
    """An infinite value reaches the rows that see its token however little the token weighs: exp(-150) is no float32, but it is not 0."""
    rng = np.random.default_rng(d + M)
    Hq, Hkv = 8, 2
    q4 = Q.Q4(1, Hkv, d, 64, [n], seed=2)
    q, _ = rows(rng, (1, 1, M, Hq, d), dtype, 150.0)
    k = torch.zeros(1, 1, M, Hkv, d, dtype=q.dtype, device="cuda")
    k[..., M // 2:, :, :] = -q[0, 0, M // 2:, ::Hq // Hkv] / 150  # half of the step's tokens lie far below the others for their own rows
    v, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    seen = rng.random((M, M)) < 0.4
    seen[range(M), range(M)] = True
    words = np.zeros((1, M, (M + 63) // 64), np.uint64)
    for j in range(M):
        words[0, :, j // 64] |= seen[:, j].astype(np.uint64) << np.uint64(j % 64)
    mask = torch.from_numpy(words.view(np.int64)).cuda()
    clean, clean_lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, mask, M)
    token, channel = (M - 1, 0), (3, d - 1)
    v[0, 0, M - 1, 0, 3], v[0, 0, 0, 1, d - 1] = float("inf"), -float("inf")
    out, lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, mask, M)
    assert torch.equal(lse, clean_lse)
    for h in range(Hq):
        e = h // 4
        hit = torch.from_numpy(seen[:, token[e]])
        assert torch.all(out[hit, h, channel[e]] == (float("inf"), -float("inf"))[e])
        out[hit, h, channel[e]] = clean[hit, h, channel[e]]
        assert torch.equal(out[:, h], clean[:, h])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M,n", [(4, 150), (4, 2000), (12, 150), (40, 700)])
def test_infinite_keys_reach_only_the_rows_that_see_them(dtype, d, M, n):
    """A score of -infinity is a token that is not there, one of +infinity no number; other rows keep every bit."""
    rng = np.random.default_rng(M + d)
    Hq, Hkv = 8, 2
    q4 = Q.Q4(1, Hkv, d, 64, [n], seed=2)
    q, _ = rows(rng, (1, 1, M, Hq, d), dtype)
    q[..., 5] = q[..., 5].abs().clamp(min=0.5) * torch.from_numpy(rng.choice([-1.0, 1.0], (1, 1, M, Hq))).to(q.dtype).cuda()
    k, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    v, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    seen = rng.random((M, M)) < 0.5
    seen[range(M), range(M)] = True

    def words(s):
        w = np.zeros((1, M, (M + 63) // 64), np.uint64)
        for j in range(M):
            w[0, :, j // 64] |= s[:, j].astype(np.uint64) << np.uint64(j % 64)
        return torch.from_numpy(w.view(np.int64)).cuda()

    clean, clean_lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, words(seen), M)
    without = seen.copy()
    without[:, 2] = False
    less, less_lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, words(without), M)
    k[0, 0, 2, :, 5] = float("inf")
    out, lse = verify(dtype, Hq, Hkv, d, q4, q, k, v, words(seen), M)
    for j in range(M):
        for h in range(Hq):
            if not seen[j, 2]:
                assert torch.equal(out[j, h], clean[j, h]) and lse[j, h] == clean_lse[j, h]
            elif q[0, 0, j, h, 5] < 0:
                assert torch.equal(out[j, h], less[j, h]) and lse[j, h] == less_lse[j, h]
            else:
                assert out[j, h].isnan().all() and lse[j, h].isnan()
