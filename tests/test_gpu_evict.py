"""The account of attention weight and the eviction by it, against numpy in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B

pytestmark = pytest.mark.gpu


def torch_dtype(dtype):
    return torch.float32 if dtype == "fp32" else torch.bfloat16


def config(layers, Hq, Hkv, d, bs, dtype, **over):
    return B.make_config(layers, Hq, Hkv, d, bs, dtype, 1, 1, 4, 16, **over)


def make_cache(layers, Hkv, d, bs, lens, dtype, rng, max_blocks=None, fill=float("nan")):
    """Pools whose unused places hold `fill`, and the tokens' rows per sequence in 64 bits."""
    batch = len(lens)
    blocks = max_blocks or max(max(-(-n // bs) for n in lens), 1)
    pages = batch * blocks + 1
    table = rng.permutation(pages)[: batch * blocks].reshape(batch, blocks).astype(np.int32)
    pools, held = [], []
    for _ in range(2):
        pool = torch.full((layers, pages, Hkv, bs, d), fill, dtype=torch_dtype(dtype))
        per = []
        for b, n in enumerate(lens):
            x = torch.from_numpy(rng.standard_normal((layers, Hkv, n, d))).to(pool.dtype)
            for t0 in range(0, n, bs):
                pool[:, table[b, t0 // bs], :, : min(bs, n - t0)] = x[:, :, t0:t0 + bs]
            per.append(x.double().numpy())
        pools.append(pool.cuda())
        held.append(per)
    cache = B.Cache(*pools, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), blocks * bs)
    return cache, held[0], held[1]


def run_accumulate(dtype, Hq, Hkv, d, bs, M, lens, taken, A, layers=2, layer0=0, n_call=None, seed=0, scale=0.0, empty_row=False):
    rng = np.random.default_rng(seed)
    batch, n_call, G = len(lens), n_call or layers, Hq // Hkv
    cfg = config(layers, Hq, Hkv, d, bs, dtype, softmax_scale=scale)
    cache, k64, _ = make_cache(layers, Hkv, d, bs, lens, dtype, rng)
    q = torch.from_numpy(rng.standard_normal((n_call, batch, M, Hq, d))).to(torch_dtype(dtype)).cuda()
    q64 = q.cpu().double().numpy()
    lse = torch.from_numpy(rng.standard_normal((n_call, batch, M, Hq)) + 5).float()
    n_taken = [min(A, n) if taken is None else len(t) for n, t in zip(lens, taken or lens)]
    rows = [list(range(n)) if taken is None else t for n, t in zip(n_taken, taken or lens)]
    if empty_row:
        lse[:, 0, rows[0][0]] = -float("inf")
    accepted = None
    if taken is not None:
        accepted = torch.full((batch, A), -9, dtype=torch.int32)
        for b, t in enumerate(taken):
            accepted[b, : len(t)] = torch.tensor(t, dtype=torch.int32)
        accepted = accepted.cuda()
    tokens = cache.block_table.shape[1] * bs
    acc = torch.from_numpy(rng.random((layers, batch, Hkv, tokens))).float().cuda()
    want = acc.cpu().double().numpy()
    tol = np.zeros_like(want)
    s = scale or d ** -0.5
    for l in range(n_call):
        for b, n in enumerate(lens):
            for h in range(Hkv):
                for i, r in enumerate(rows[b]):
                    end = n - n_taken[b] + i + 1
                    for g in range(G):
                        e = float(lse[l, b, r, h * G + g])
                        if e == -np.inf:
                            continue
                        k, qq = k64[b][layer0 + l, h, :end], q64[l, b, r, h * G + g]
                        w = np.exp(k @ qq * s - e)
                        # a score summed in float32 over d channels, the difference, its exponential, and the sum over the rows
                        err = (d + 4) * 2.0 ** -23 * (np.abs(k) @ np.abs(qq)) * s + 2.0 ** -22 * abs(e) + 2.0 ** -20 + n_taken[b] * G * 2.0 ** -24
                        want[layer0 + l, b, h, :end] += w
                        tol[layer0 + l, b, h, :end] += w * err
    tol += 2.0 ** -23 * np.abs(want)
    ws = B.new_workspace(cfg, n_call, batch, tokens, M)
    n_dev = torch.tensor(n_taken, dtype=torch.int32, device="cuda")
    before = acc.clone()
    B.specpv_accumulate_attention(cfg, layer0, n_call, q, lse.cuda(), M, accepted, n_dev, A, cache, acc, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    got = acc.cpu().double().numpy()
    assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / np.maximum(tol, 1e-300)).max()
    for b, n in enumerate(lens):
        assert torch.equal(acc[:, b, :, n:], before[:, b, :, n:])  # behind the sequence
    other = torch.ones(layers, dtype=torch.bool)
    other[layer0:layer0 + n_call] = False
    assert torch.equal(acc[other], before[other])
    again = before.clone()
    B.specpv_accumulate_attention(cfg, layer0, n_call, q, lse.cuda(), M, accepted, n_dev, A, cache, again, ws)
    assert torch.equal(again, acc)  # the same sums at every run


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bs", [(128, 64), (64, 16), (128, 16), (64, 32)])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 127, 128, 129, 300])
def test_account_at_the_edges_of_pages_and_tiles(dtype, d, bs, n):
    run_accumulate(dtype, 8, 2, d, bs, 9, [n, n + 5], [[3] if n == 1 else [0, 7], [8, 1, 4]], 4, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,Hkv,A", [(1, 1, 1), (8, 1, 1), (5, 1, 3), (8, 2, 4), (16, 1, 9), (8, 1, 17), (8, 1, 128), (160, 1, 2), (12, 3, 33)])
def test_account_of_any_number_of_rows(dtype, Hq, Hkv, A):
    run_accumulate(dtype, Hq, Hkv, 128, 64, max(A, 4), [200], None, A, layers=1, seed=A)
    run_accumulate(dtype, Hq, Hkv, 64, 32, max(A, 4), [333, 40], None, A, layers=2, layer0=1, n_call=1, seed=A)


def test_account_of_no_rows_empty_rows_and_an_empty_cache():
    run_accumulate("bf16", 8, 2, 128, 64, 4, [100, 50, 0], [[], [1], []], 2)
    run_accumulate("bf16", 8, 2, 128, 64, 4, [100], [[2, 3]], 2, empty_row=True)
    run_accumulate("fp32", 8, 2, 64, 16, 4, [100], [[2, 3]], 3, empty_row=True, scale=0.3)


def test_account_of_one_row_many_times():
    run_accumulate("bf16", 8, 2, 128, 64, 4, [100], [[2, 2, 2]], 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("A", [1, 3])
def test_account_of_infinite_keys(dtype, A):
    """A score of -infinity adds nothing, one of +infinity an infinity, and both to their own token alone; rows that are not there, and
    those whose lse is -infinity, add nothing even so."""
    rng = np.random.default_rng(A)
    cfg = config(1, 2, 1, 64, 16, dtype)
    cache, k64, _ = make_cache(1, 1, 64, 16, [50], dtype, rng)
    q = torch.from_numpy(rng.standard_normal((1, 1, 4, 2, 64))).to(torch_dtype(dtype)).cuda()
    q[..., 7] = -q[..., 7].abs() - 0.5
    q[..., 9] = 1.0
    page, at = cache.block_table[0, 1].item(), 3
    cache.k_pool[0, page, 0, at, 7] = float("inf")       # token 19
    cache.k_pool[0, page, 0, at + 1, 7] = -float("inf")  # token 20
    cache.k_pool[0, page, 0, at + 2, 9] = -float("inf")  # token 21
    lse = torch.full((1, 1, 4, 2), 5.0, device="cuda")
    lse[0, 0, 2] = -float("inf")
    acc = torch.ones(1, 1, 1, 64, device="cuda")
    ws = B.new_workspace(cfg, 1, 1, 64, 4)
    n = torch.tensor([A], dtype=torch.int32, device="cuda")
    B.specpv_accumulate_attention(cfg, 0, 1, q, lse, 4, None, n, A, cache, acc, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    a = acc[0, 0, 0].cpu().numpy()
    assert a[19] == 1.0 and a[20] == np.inf and a[21] == 1.0
    assert np.all(np.isfinite(np.delete(a, 20))) and np.all(a[50:] == 1.0)
    assert np.all(np.delete(a[: 50 - A], [19, 20, 21]) > 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_account_faults_are_reported(dtype):
    rng = np.random.default_rng(0)
    cfg = config(1, 4, 2, 64, 16, dtype)
    cache, _, _ = make_cache(1, 2, 64, 16, [40, 33], dtype, rng)
    q = torch.randn(1, 2, 3, 4, 64, device="cuda").to(torch_dtype(dtype))
    lse = torch.full((1, 2, 3, 4), 5.0, device="cuda")
    acc = torch.zeros(1, 2, 2, 48, device="cuda")
    ws = B.new_workspace(cfg, 1, 2, 48, 3)
    n = torch.tensor([1, 2], dtype=torch.int32, device="cuda")

    def call(rows):
        a = torch.tensor(rows, dtype=torch.int32, device="cuda")
        B.specpv_accumulate_attention(cfg, 0, 1, q, lse, 3, a, n, 2, cache, acc, ws)
        return B.STATUS_NAMES[B.specpv_poll_status(ws)[0]]

    assert call([[0, 0], [1, 2]]) == "OK"
    assert call([[0, 0], [1, 3]]) == "INVALID_ARG"
    assert call([[-1, 0], [1, 2]]) == "INVALID_ARG"
    assert acc.isfinite().all()
    cache.block_table[1, 1] = 99
    assert call([[0, 0], [1, 2]]) == "BAD_BLOCK_TABLE"
    assert acc.isfinite().all()


# ---- eviction ----------------------------------------------------------------------------------------------------
def kept_tokens(acc, n, keep, sink, local):
    """The definition: sink, the heaviest of the rest, local; ties to the lower token, NaN last."""
    middle = list(range(sink, n - local))
    middle.sort(key=lambda t: (np.isnan(acc[t]), -acc[t] if not np.isnan(acc[t]) else 0.0, t))
    return sorted([*range(sink), *middle[: keep - sink - local], *range(n - local, n)])


def run_evict(dtype, Hkv, d, bs, lens, keep, sink, local, layers=2, seed=0, shared=0, change=None, max_blocks=None):
    rng = np.random.default_rng(seed)
    batch = len(lens)
    cfg = config(layers, Hkv, Hkv, d, bs, dtype, select_shared=shared)
    cache, k64, v64 = make_cache(layers, Hkv, d, bs, lens, dtype, rng, fill=3.0, max_blocks=max_blocks)
    tokens = cache.block_table.shape[1] * bs
    acc = torch.from_numpy(np.exp(2 * rng.standard_normal((layers, batch, Hkv, tokens)))).float()
    if change:
        change(acc)
    before = acc.numpy().copy()
    acc = acc.cuda()
    idx = torch.full((layers, batch, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    ws = B.new_workspace(cfg, layers, batch, tokens, 4)
    pools = [cache.k_pool.clone(), cache.v_pool.clone()]
    B.specpv_evict_tokens(cfg, cache, acc, keep, sink, local, idx, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    assert cache.seq_lens.tolist() == [min(n, keep) for n in lens]
    got_idx, got_acc, table = idx.cpu().numpy(), acc.cpu().numpy(), cache.block_table.cpu().numpy()
    want = [p.clone() for p in pools]
    for l in range(layers):
        for b, n in enumerate(lens):
            for h in range(Hkv):
                a = before[l, b, h]
                if n <= keep:
                    stay = list(range(n))
                    assert np.array_equal(got_acc[l, b, h], a, equal_nan=True)
                else:
                    rank = a
                    if shared:  # in float32, heads in order
                        rank = np.zeros(tokens, np.float32)
                        for g in range(Hkv):
                            rank = rank + before[l, b, g]
                        rank = rank * np.float32(1 / Hkv)
                    stay = kept_tokens(rank, n, keep, sink, local)
                    want_acc = a.copy()
                    want_acc[:keep] = a[stay]
                    want_acc[keep:n] = 0
                    assert np.array_equal(got_acc[l, b, h], want_acc, equal_nan=True)
                    for new, old, x in ((want[0], pools[0], k64), (want[1], pools[1], v64)):
                        rows = old[l, table[b, np.array(stay) // bs], h, np.array(stay) % bs]
                        new[l, table[b, np.arange(keep) // bs], h, np.arange(keep) % bs] = rows
                        assert np.array_equal(rows.cpu().double().numpy(), x[b][l, h, stay])
                assert got_idx[l, b, h, : len(stay)].tolist() == stay
                assert np.all(got_idx[l, b, h, len(stay):] == -1)
    assert torch.equal(cache.k_pool, want[0]) and torch.equal(cache.v_pool, want[1])  # and nothing else was written


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bs", [(128, 64), (64, 16), (128, 32)])
@pytest.mark.parametrize("n,keep,sink,local", [(100, 60, 4, 8), (100, 99, 0, 1), (100, 100, 4, 8), (100, 200, 4, 8), (100, 1, 0, 0),
                                               (100, 13, 12, 0), (100, 13, 0, 12), (777, 700, 32, 128), (777, 130, 1, 1), (65, 64, 63, 0)])
def test_eviction(dtype, d, bs, n, keep, sink, local):
    run_evict(dtype, 2, d, bs, [n, max(n - 30, 0), 0, 1], keep, sink, local, layers=1, seed=n + keep)


@pytest.mark.parametrize("n,keep", [(2500, 1111), (4999, 4500), (9000, 5000), (17500, 300), (17500, 17000)])
def test_eviction_from_long_lists(n, keep):
    run_evict("bf16", 2, 64, 64, [n], keep, 4, 32, layers=1, seed=n)


@pytest.mark.parametrize("n,keep,shared", [(24001, 8192, 0), (24001, 23000, 1), (70001, 5000, 0), (70001, 69000, 1)])
def test_eviction_from_lists_past_the_registers(n, keep, shared):
    run_evict("bf16", 2, 64, 64, [n, 20000], keep, 32, 100, layers=1, seed=n, shared=shared)
    run_evict("bf16", 1, 64, 64, [n], keep, 0, 0, layers=1, shared=shared, change=lambda acc: acc.fill_(2.0))


def test_eviction_of_many_units_and_layers():
    run_evict("bf16", 8, 64, 16, [200, 150], 128, 4, 16, layers=12)
    run_evict("bf16", 3, 64, 16, [200, 150], 128, 4, 16, layers=2, shared=1)


def test_eviction_with_ties_infinities_and_nan():
    def change(acc):
        acc[..., 10:60] = 1.0
        acc[..., 70] = float("inf")
        acc[..., 71] = float("nan")
        acc[..., 72] = -0.0
        acc[..., 73] = 0.0
        acc[..., 74] = -float("inf")
    run_evict("bf16", 2, 64, 16, [100], 50, 3, 5, change=change)
    run_evict("fp32", 2, 64, 16, [100], 95, 3, 5, change=change)
    run_evict("bf16", 2, 64, 16, [100], 50, 3, 5, change=lambda acc: acc.fill_(0.0))


def test_eviction_reports_bad_pages():
    rng = np.random.default_rng(0)
    cfg = config(1, 2, 2, 64, 16, "bf16")
    cache, _, _ = make_cache(1, 2, 64, 16, [90], "bf16", rng)
    acc = torch.rand(1, 1, 2, 96, device="cuda")
    idx = torch.zeros(1, 1, 2, 40, dtype=torch.int32, device="cuda")
    ws = B.new_workspace(cfg, 1, 1, 96, 4)
    cache.block_table[0, 5] = -3
    B.specpv_evict_tokens(cfg, cache, acc, 40, 4, 20, idx, ws)
    assert B.STATUS_NAMES[B.specpv_poll_status(ws)[0]] == "BAD_BLOCK_TABLE"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_loop_with_eviction(dtype):
    """Attention, commit, account, eviction, step by step, against the same loop in 64 bits: what is kept is followed exactly."""
    rng = np.random.default_rng(7)
    layers, Hq, Hkv, d, bs, M, keep, sink, local = 2, 8, 2, 64, 16, 6, 60, 4, 8
    dt = torch_dtype(dtype)
    cfg = config(layers, Hq, Hkv, d, bs, dtype)
    cache, k64, v64 = make_cache(layers, Hkv, d, bs, [70, 41], dtype, rng, max_blocks=6)
    acc = torch.zeros(layers, 2, Hkv, 6 * bs, device="cuda")
    ws = B.new_workspace(cfg, layers, 2, 6 * bs, M)
    idx = torch.zeros(layers, 2, Hkv, keep, dtype=torch.int32, device="cuda")
    k64, v64 = [list(k64), list(v64)]
    total = [np.zeros((layers, Hkv, 6 * bs)) for _ in range(2)]
    for step in range(12):
        q, k, v = (torch.from_numpy(rng.standard_normal((layers, 2, M, n, d))).to(dt) for n in (Hq, Hkv, Hkv))
        mask = torch.tensor([[[(1 << (j + 1)) - 1] for j in range(M)]] * 2, dtype=torch.int64, device="cuda")
        out, lse = torch.zeros(layers, 2, M, Hq, d, dtype=dt, device="cuda"), torch.zeros(layers, 2, M, Hq, device="cuda")
        qc, kc, vc = q.cuda(), k.cuda(), v.cuda()
        B.specpv_verify_full(cfg, 0, layers, qc, kc, vc, mask, None, M, cache, out, lse, ws)
        n_acc = [1 + step % 4, 1 + (step + 1) % 3]
        rows = torch.arange(4, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()
        n_dev = torch.tensor(n_acc, dtype=torch.int32, device="cuda")
        B.specpv_commit_accepted(cfg, 0, layers, kc, vc, M, rows, n_dev, 4, cache, None, None, ws)
        B.specpv_accumulate_attention(cfg, 0, layers, qc, lse, M, rows, n_dev, 4, cache, acc, ws)
        for b in range(2):
            k64[b] = np.concatenate([k64[b], k[:, b, : n_acc[b]].double().numpy().transpose(0, 2, 1, 3)], 2)
            v64[b] = np.concatenate([v64[b], v[:, b, : n_acc[b]].double().numpy().transpose(0, 2, 1, 3)], 2)
            n = k64[b].shape[2]
            for l in range(layers):
                for h in range(Hq):
                    for i in range(n_acc[b]):
                        s = k64[b][l, h // 4, : n - n_acc[b] + i + 1] @ q[l, b, i, h].double().numpy() / 8
                        w = np.exp(s - s.max())
                        total[b][l, h // 4, : len(s)] += w / w.sum()
        # a step adds at most 4 rows x 4 heads weights of at most 1 to an account, each off by the errors of its score and of the
        # log-sum-exp: sums of 64 products in float32, 2 x 68 x 2^-23 of the products' magnitudes (below 12 here)
        assert np.abs(acc.cpu().double().numpy() - np.stack(total, 1)).max() <= 16 * 2 * 68 * 2.0 ** -23 * 12 * (step + 1)
        if step % 3 == 2:
            account = acc.cpu().numpy()
            B.specpv_evict_tokens(cfg, cache, acc, keep, sink, local, idx, ws)
            for b in range(2):
                n = k64[b].shape[2]
                if n <= keep:
                    continue
                stay = np.array([[kept_tokens(account[l, b, h], n, keep, sink, local) for h in range(Hkv)] for l in range(layers)])
                assert np.array_equal(stay, idx[:, b].cpu().numpy())
                at = stay[..., None]
                k64[b], v64[b] = (np.take_along_axis(x[b], at, 2) for x in (k64, v64))
                total[b][:, :, :keep] = np.take_along_axis(total[b], stay, 2)
                total[b][:, :, keep:] = 0
        assert B.specpv_poll_status(ws)[0] == 0
        assert cache.seq_lens.tolist() == [x.shape[2] for x in k64]
    table = cache.block_table.cpu().numpy()
    for b in range(2):
        t = np.arange(k64[b].shape[2])
        for pool, x in ((cache.k_pool, k64), (cache.v_pool, v64)):
            got = pool.cpu().double().numpy()[:, table[b, t // bs], :, t % bs]  # [tokens][layers][heads][d]
            assert np.array_equal(got.transpose(1, 2, 0, 3), x[b])


def test_eviction_captured_and_replayed():
    rng = np.random.default_rng(3)
    cfg = config(2, 2, 2, 64, 16, "bf16")
    cache, _, _ = make_cache(2, 2, 64, 16, [90], "bf16", rng, fill=3.0)
    acc0 = torch.rand(2, 1, 2, 96, device="cuda")
    acc, idx = acc0.clone(), torch.zeros(2, 1, 2, 40, dtype=torch.int32, device="cuda")
    ws = B.new_workspace(cfg, 2, 1, 96, 4)
    start = cache.k_pool.clone()
    B.specpv_evict_tokens(cfg, cache, acc, 40, 4, 20, idx, ws)
    want = [x.clone() for x in (cache.k_pool, acc, idx)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        B.specpv_evict_tokens(cfg, cache, acc, 40, 4, 20, idx, ws)
    for _ in range(2):
        cache.k_pool.copy_(start)
        acc.copy_(acc0)
        idx.zero_()
        cache.seq_lens.fill_(90)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((cache.k_pool, acc, idx), want)) and cache.seq_lens.item() == 40
