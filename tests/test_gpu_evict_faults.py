"""What an eviction leaves behind when the block table names pages that do not exist."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests.test_gpu_evict import config, kept_tokens, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,bs", [("bf16", 64, 16), ("fp32", 128, 32)])
@pytest.mark.parametrize("bad", [{5: -3}, {1: 2 ** 31 - 1}, {0: 10 ** 6, 2: -1}])
def test_rows_of_good_pages_move_and_nothing_else_is_written(dtype, d, bs, bad):
    rng = np.random.default_rng(len(bad))
    Hkv, n, keep, sink, local = 2, 6 * bs - 6, 3 * bs - 8, 4, bs + 4
    cfg = config(1, Hkv, Hkv, d, bs, dtype)
    cache, _, _ = make_cache(1, Hkv, d, bs, [n, n - 1], dtype, rng, fill=3.0)
    tokens = 6 * bs
    acc = torch.rand(1, 2, Hkv, tokens, device="cuda")
    before, table = acc.cpu().numpy(), cache.block_table.cpu().numpy()
    want = [cache.k_pool.clone(), cache.v_pool.clone()]
    idx = torch.full((1, 2, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    ws = B.new_workspace(cfg, 1, 2, tokens, 4)
    for block, page in bad.items():
        cache.block_table[0, block] = page  # of the first sequence alone
    B.specpv_evict_tokens(cfg, cache, acc, keep, sink, local, idx, ws)
    st, info = B.specpv_poll_status(ws)
    assert B.STATUS_NAMES[st] == "BAD_BLOCK_TABLE" and info[0] == 0 and info[1] in bad and info[2] == bad[info[1]]
    assert cache.seq_lens.tolist() == [keep, keep]
    for b, length in enumerate((n, n - 1)):
        for h in range(Hkv):
            stay = np.array(kept_tokens(before[0, b, h], length, keep, sink, local))
            assert np.array_equal(idx[0, b, h].cpu().numpy(), stay)
            account = before[0, b, h].copy()
            account[:keep], account[keep:length] = account[stay], 0
            assert np.array_equal(acc[0, b, h].cpu().numpy(), account)
            for pool in want:
                old = pool.clone()
                for j, t in enumerate(stay):
                    if b == 1 or (j // bs not in bad and t // bs not in bad):
                        pool[0, table[b, j // bs], h, j % bs] = old[0, table[b, t // bs], h, t % bs]
    assert torch.equal(cache.k_pool, want[0]) and torch.equal(cache.v_pool, want[1])
