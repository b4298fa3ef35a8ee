"""Pages far into large pools (byte offsets past 2^32, element numbers past 2^32): every call gives what it gives with the same pages at
the head of a small pool, and one graph of all of them gives it again."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests import q4_util as Q
from tests.test_gpu_q4 import config, random_masks, rows

pytestmark = pytest.mark.gpu

Hq, Hkv, d, bs, blocks, n = 8, 8, 128, 64, 8, 450
FAR = 66000  # pages: 4.6 GB in 4 bits, 8.7 GB of bfloat16


def pools(pages, shape, dtype, far):
    """The pages, alone or scattered over the end of a pool; and where they are."""
    if not far:
        return pages.clone(), torch.arange(blocks, dtype=torch.int32, device="cuda")[None].contiguous()
    at = FAR - 1 - 3 * torch.arange(blocks, device="cuda")
    pool = torch.zeros(1, FAR, *shape, dtype=dtype, device="cuda")
    pool[:, at] = pages
    return pool, at[None].int().contiguous()


def inputs():
    rng = np.random.default_rng(0)
    q4 = Q.Q4(1, Hkv, d, bs, [n], seed=1, shuffle=False, spare=0, max_blocks=blocks)
    x = dict(q4=torch.from_numpy(q4.pool).cuda())
    for name in "kv":
        x[name] = torch.from_numpy(rng.standard_normal((1, blocks, Hkv, bs, d))).bfloat16().cuda()
    for M in (1, 40):
        x[M] = [rows(rng, (1, 1, M, h, d), "bf16")[0] for h in (Hq, Hkv, Hkv)] + [random_masks(rng, 1, M)[1]]
    return x


def run(x, far, dtype="bf16", graph=False):
    cfg = config(1, Hq, Hkv, d, bs, dtype, budget_blocks=4, buffer_tokens=16)
    cast = (lambda t: t.float()) if dtype == "fp32" else (lambda t: t)
    pool, table = pools(x["q4"], (Hkv, bs * (d + 8)), torch.uint8, far)
    full = B.CacheQ4(pool, table, torch.tensor([n], dtype=torch.int32, device="cuda"), blocks * bs)
    ws = B.new_workspace(cfg, 1, 1, blocks * bs, 40)
    one = torch.tensor([3], dtype=torch.int32, device="cuda")
    outs, calls = [], []
    for M in (1, 40):
        q, k, v = (cast(t) for t in x[M][:3])
        out, lse = torch.zeros_like(q), torch.zeros(1, 1, M, Hq, device="cuda")
        calls.append(lambda q=q, k=k, v=v, M=M, out=out, lse=lse: B.specpv_verify_full_q4(cfg, 0, 1, q, k, v, x[M][3], None, M, full, out, lse, ws))
        outs += [out, lse]
    k, v = (cast(t) for t in x[40][1:3])
    kmax, kmin = (torch.zeros(1, 1, Hkv, blocks, d, dtype=k.dtype, device="cuda") for _ in range(2))
    calls.append(lambda: B.specpv_commit_accepted_q4(cfg, 0, 1, k, v, 40, None, one, 3, full, kmax, kmin, None, None, ws))
    parts = [torch.zeros(1, FAR if far else 5, Hkv, bs, d, dtype=k.dtype, device="cuda") if dtype == "bf16" else
             torch.zeros(1, 5, Hkv, bs, d, device="cuda") for _ in range(2)]
    part_table = (parts[0].shape[1] - 5 + torch.arange(5, device="cuda"))[None].int().contiguous()
    part = B.Cache(*parts, part_table, torch.zeros(1, dtype=torch.int32, device="cuda"), 5 * bs)
    idx = torch.tensor([0, 3, 5, 7], dtype=torch.int32, device="cuda").expand(1, 1, Hkv, 4).contiguous()
    count = torch.tensor([4], dtype=torch.int32, device="cuda")
    calls.append(lambda: B.specpv_refresh_partial_q4(cfg, full, idx, count, part, part.seq_lens, ws))
    acc = torch.zeros(1, 1, Hkv, 5 * bs, device="cuda")
    calls.append(lambda: B.specpv_accumulate_attention(cfg, 0, 1, cast(x[40][0]) if dtype == "fp32" else x[40][0], outs[3], 40, None, one, 3, part, acc, ws))
    kept = torch.zeros(1, 1, Hkv, 100, dtype=torch.int32, device="cuda")
    calls.append(lambda: B.specpv_evict_tokens(cfg, part, acc, 100, 4, 16, kept, ws))
    start = [full.pool.clone() if graph else None, acc.clone()]
    if graph:
        for call in calls:  # (before the capture: modules are loaded)
            call()
        full.pool.copy_(start[0])
        full.seq_lens.fill_(n)
        for t in (acc, kmax, kmin, kept, *parts, *outs):
            t.zero_()
        g, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=stream):
            for call in calls:
                call()
        g.replay()
    else:
        for call in calls:
            call()
    assert B.specpv_poll_status(ws)[0] == 0
    held = [t[:, part_table[0].long()].clone() for t in parts]
    return [*outs, kmax, kmin, full.pool[:, table[0].long()].clone(), full.seq_lens, *held, part.seq_lens, acc, kept]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_far_pages(dtype):
    x = inputs()
    near = run(x, False, dtype)
    assert near[-3].tolist() == [100] and all(t.isfinite().all() for t in near[:4])
    far = run(x, True, dtype)
    for a, b in zip(near, far):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_all_calls_in_one_graph(dtype):
    x = inputs()
    for a, b in zip(run(x, False, dtype), run(x, False, dtype, graph=True)):
        assert torch.equal(a, b)
