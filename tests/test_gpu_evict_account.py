"""The account of attention weight where its terms are exact: no more may be off than float32 takes."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests.test_gpu_evict import config, make_cache, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bs", [(64, 16), (128, 64)])
@pytest.mark.parametrize("size", [10.0, 80.0, 1000.0, -1000.0])
def test_exact_products_and_a_large_log_sum_exp(dtype, d, bs, size):
    """Queries of one power of two, so that a score is one exact product, and log-sum-exps of about `size`: what is left are the roundings of the
    difference, of its exponential and of the sums."""
    rng = np.random.default_rng(d + int(abs(size)))
    Hq, Hkv, n, M, A = 8, 2, 333, 6, 4
    cfg = config(1, Hq, Hkv, d, bs, dtype, softmax_scale=0.125)
    cache, _, _ = make_cache(1, Hkv, d, bs, [n], dtype, rng)
    # channel 1 holds the scores: 8 bits, within 4 of `size`
    score = torch.from_numpy(size + rng.integers(-8, 9, (n, Hkv)) / 2).bfloat16().double()
    for t in range(n):
        cache.k_pool[0, cache.block_table[0, t // bs].item(), :, t % bs, 1] = score[t].to(cache.k_pool.dtype)
    score = score.numpy()
    q = torch.zeros(1, 1, M, Hq, d, dtype=torch_dtype(dtype), device="cuda")
    q[..., 1] = 8.0
    lse = (size + torch.from_numpy(rng.random((1, 1, M, Hq)) * 3)).float()
    acc = torch.zeros(1, 1, Hkv, cache.block_table.shape[1] * bs, device="cuda")
    rows = torch.tensor([[0, 2, 3, 5]], dtype=torch.int32, device="cuda")
    ws = B.new_workspace(cfg, 1, 1, n, M)
    B.specpv_accumulate_attention(cfg, 0, 1, q, lse.cuda(), M, rows, torch.tensor([A], dtype=torch.int32, device="cuda"), A, cache, acc, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    got, e = acc[0, 0].cpu().double().numpy(), lse[0, 0].double().numpy()
    for h in range(Hkv):
        want, tol = np.zeros(n), np.zeros(n)
        for i, r in enumerate((0, 2, 3, 5)):
            for g in range(Hq // Hkv):
                x = score[: n - A + i + 1, h] - e[r, h * 4 + g]
                w = np.exp(x)
                want[: len(w)] += w
                # the difference, the factor and their product, 2^-24 of it each; the exponential
                tol[: len(w)] += w * (4 * 2.0 ** -24 * np.abs(x) + 2.0 ** -21)
        tol += 16 * 2.0 ** -24 * want  # a sum of 16
        assert np.all(np.abs(got[h, :n] - want) <= tol), (np.abs(got[h, :n] - want) / want).max()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [1e-36, 1e-38, 1e-40, 1e-44])
def test_scales_too_small_to_divide_by(dtype, scale):
    """Scores of nothing: what counts is the log-sum-exp, which divided by such a scale is no float32."""
    rng = np.random.default_rng(0)
    Hq, Hkv, d, bs, n, M = 8, 2, 64, 16, 100, 3
    cfg = config(1, Hq, Hkv, d, bs, dtype, softmax_scale=scale)
    cache, _, _ = make_cache(1, Hkv, d, bs, [n], dtype, rng)
    q = torch.from_numpy(rng.standard_normal((1, 1, M, Hq, d))).to(torch_dtype(dtype)).cuda()
    lse = torch.from_numpy(np.log(n) + rng.standard_normal((1, 1, M, Hq))).float()
    lse[0, 0, 0, 0], lse[0, 0, 1, 7] = -50.0, float("inf")
    acc = torch.zeros(1, 1, Hkv, cache.block_table.shape[1] * bs, device="cuda")
    ws = B.new_workspace(cfg, 1, 1, n, M)
    B.specpv_accumulate_attention(cfg, 0, 1, q, lse.cuda(), M, None, torch.tensor([M], dtype=torch.int32, device="cuda"), M, cache, acc, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    got, w = acc[0, 0].cpu().double().numpy(), np.exp(-lse[0, 0].double().numpy()).reshape(M, Hkv, -1).sum(-1)
    for h in range(Hkv):
        for t in range(n):
            want = sum(w[i, h] for i in range(M) if t < n - M + i + 1)
            # scores below 1e-34; the log-sum-exp times log2(e), in float32, its exponential, a sum of 12
            assert abs(got[h, t] - want) <= want * (2 * 2.0 ** -24 * 50 * 1.45 + 2.0 ** -21 + 12 * 2.0 ** -24)
