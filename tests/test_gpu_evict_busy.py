"""Eviction beside other work on the GPU, again and again: rows that a late warp moves are the same ones."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests.test_gpu_evict import config, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,n,keep", [("bf16", 64, 300, 200), ("bf16", 128, 900, 700), ("bf16", 128, 4352, 4096), ("fp32", 128, 1500, 1100)])
def test_eviction_beside_other_work(dtype, d, n, keep):
    """One to many rounds per cluster, with a second stream that keeps the SMs busy, so that warps of a CTA drift apart."""
    rng = np.random.default_rng(n)
    layers, Hkv, bs, sink, local = 2, 4, 64, 4, 32
    cfg = config(layers, Hkv, Hkv, d, bs, dtype)
    cache, _, _ = make_cache(layers, Hkv, d, bs, [n, n - 7], dtype, rng, fill=3.0)
    tokens = cache.block_table.shape[1] * bs
    acc0 = torch.from_numpy(np.exp(2 * rng.standard_normal((layers, 2, Hkv, tokens)))).float().cuda()
    pools, lens = [cache.k_pool.clone(), cache.v_pool.clone()], cache.seq_lens.clone()
    acc, idx = acc0.clone(), torch.zeros(layers, 2, Hkv, keep, dtype=torch.int32, device="cuda")
    ws = B.new_workspace(cfg, layers, 2, tokens, 4)
    table = cache.block_table.long()
    a, b = (torch.randn(2048, 2048, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    noise, side = torch.randn(1 << 24, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(100):
        with torch.cuda.stream(side):
            for _ in range(3):
                torch.matmul(a, b)
                noise.mul_(1.0)
        cache.k_pool.copy_(pools[0])
        cache.v_pool.copy_(pools[1])
        cache.seq_lens.copy_(lens)
        acc.copy_(acc0)
        B.specpv_evict_tokens(cfg, cache, acc, keep, sink, local, idx, ws)
        # what the indexes say, by indexing
        t = idx.long().permute(0, 2, 1, 3)                                   # [layers][Hkv][seqs][keep]
        layer = torch.arange(layers, device="cuda")[:, None, None, None]
        head = torch.arange(Hkv, device="cuda")[None, :, None, None]
        seq = torch.arange(2, device="cuda")[None, None, :, None]
        to = torch.arange(keep, device="cuda").expand_as(t)
        for got, old in zip((cache.k_pool, cache.v_pool), pools):
            new = old.clone()
            new[layer, table[seq, to // bs], head, to % bs] = old[layer, table[seq, t // bs], head, t % bs]
            wrong += (got != new).sum()
        wrong += (acc[..., :keep] != acc0.gather(-1, idx.long())).sum()
    torch.cuda.synchronize()
    assert wrong.item() == 0
    assert B.specpv_poll_status(ws)[0] == 0 and cache.seq_lens.tolist() == [keep, keep]
