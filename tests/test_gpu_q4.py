"""The cache in 4 bits: attention, commit and refresh against numpy in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from tests import q4_util as Q

pytestmark = pytest.mark.gpu


def config(layers, Hq, Hkv, d, bs, dtype, **over):
    kw = dict(sink_blocks=1, local_blocks=1, budget_blocks=4, buffer_tokens=16)
    kw.update(over)
    return B.make_config(layers, Hq, Hkv, d, bs, dtype, **kw)


def torch_dtype(dtype):
    return torch.float32 if dtype == "fp32" else torch.bfloat16


def rows(rng, shape, dtype, scale=1.0):
    """A step's tensor on the GPU, and what it holds."""
    x = rng.standard_normal(shape) * scale
    t = torch.from_numpy(x).to(torch_dtype(dtype)).cuda()
    return t, t.cpu().double().numpy()


def random_masks(rng, batch, M, density=0.5):
    """Any mask, not only trees; a row may see nothing among the step's tokens."""
    seen = rng.random((batch, M, M)) < density
    words = np.zeros((batch, M, (M + 63) // 64), np.uint64)
    for j in range(M):
        words[..., j // 64] |= seen[..., j].astype(np.uint64) << np.uint64(j % 64)
    return seen, torch.from_numpy(words.view(np.int64)).cuda()


def check_attention(out, lse, ref, dtype, out_f32, n_tokens, plain, v_unit=1.0):
    """The errors that arithmetic allows.  A score is a sum of d products in float32 (each addition off by at most 2^-23 of the sum of
    the magnitudes, d additions and the scaling), weights are exp of it (2^-21 for the exponential and its argument) and, on the tensor
    cores, rounded to bfloat16 (2^-8); sums over the tokens are in float32 (2^-23 each, the tensor core's truncated)."""
    want, want_lse, mean_abs, slack = ref
    d = want.shape[-1]
    score = (d + 4) * 2.0 ** -23 * slack + 2.0 ** -21
    sums = (n_tokens / 16 + 64) * 2.0 ** -23
    weight = score + sums + (0 if plain else Q.HALF_BF16)
    some = np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(want_lse))
    lse_tol = score + sums + 4 * Q.HALF_F32 * np.abs(np.where(some, want_lse, 0))
    assert np.all(np.abs(lse[some] - want_lse[some]) <= lse_tol[some])
    tol = 2 * weight[..., None] * mean_abs  # the numerator's, and the denominator's
    if not (out_f32 or dtype == "fp32"):
        tol = tol * (1 + Q.HALF_BF16) + Q.HALF_BF16 * np.abs(want)
    tol = tol + 1e-30 * v_unit  # weights below 2^-126 of the largest are 0: n_tokens 2^-126 times the largest value
    assert np.all(np.isfinite(out))
    assert np.all(np.abs(out - want) <= tol), (np.abs(out - want) / tol).max()


def run_attention(dtype, Hq, Hkv, d, bs, M, lens, q_lens=None, layers=2, seed=0, out_f32=0, layer0=0, n_call=None, scale=0.0,
                  q_scale=1.0, density=0.5, shuffle=True, poison=True, v_log2=0, ws_skip=0):
    rng = np.random.default_rng(seed)
    batch, n_call = len(lens), n_call or layers
    cfg = config(layers, Hq, Hkv, d, bs, dtype, out_f32=out_f32, softmax_scale=scale)
    q4 = Q.Q4(layers, Hkv, d, bs, lens, seed=seed + 1, shuffle=shuffle)
    if v_log2:  # the values times a power of two: exact in their scales and offsets
        params = q4.pool[..., bs * d:].view(np.uint16).reshape(*q4.pool.shape[:3], 4, bs)[..., 2:, :]
        params[params != 0xFFFF] += np.uint16(v_log2 << 7)
        q4.v = [x * 2.0 ** v_log2 for x in q4.v]
    q, q64 = rows(rng, (n_call, batch, M, Hq, d), dtype, q_scale)
    k, k64 = rows(rng, (n_call, batch, M, Hkv, d), dtype)
    v, v64 = rows(rng, (n_call, batch, M, Hkv, d), dtype, 2.0 ** v_log2)
    seen, mask = random_masks(rng, batch, M, density)
    used = [M] * batch if q_lens is None else q_lens
    if poison:  # what no row sees does not matter
        for b, n in enumerate(used):
            k[:, b, n:], v[:, b, n:] = float("nan"), float("inf")
            q[:, b, n:] = float("nan")
    out = torch.full((n_call, batch, M, Hq, d), 7.0, dtype=torch.float32 if out_f32 else torch_dtype(dtype), device="cuda")
    lse = torch.full((n_call, batch, M, Hq), 7.0, device="cuda")
    ws = B.new_workspace(cfg, n_call, batch, max(lens), M)
    if ws_skip:  # as large as it has to be, and no better aligned
        ws = torch.zeros(ws.numel() + ws_skip, dtype=torch.uint8, device="cuda")[ws_skip:]
    ql = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    B.specpv_verify_full_q4(cfg, layer0, n_call, q, k, v, mask, ql, M, q4.cache(B), out, lse, ws)
    st, info = B.specpv_poll_status(ws)
    assert st == 0, (st, info)
    got, got_lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for l in range(n_call):
        for b, n in enumerate(used):
            assert np.all(got[l, b, n:] == 7.0) and np.all(got_lse[l, b, n:] == 7.0)  # rows past the step's are not written
            if n == 0:
                continue
            ref = Q.attention(q64[l, b, :n], q4.k[b][layer0 + l], q4.v[b][layer0 + l], k64[l, b, :n], v64[l, b, :n],
                              seen[b][:n, :n], Hq // Hkv, scale or d ** -0.5)
            check_attention(got[l, b, :n], got_lse[l, b, :n], ref, dtype, out_f32, lens[b] + n, dtype == "fp32", 2.0 ** v_log2)
    return got, got_lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bs", [(128, 64), (128, 16), (64, 32), (64, 16), (128, 32), (64, 64)])
@pytest.mark.parametrize("n", [0, 1, 15, 63, 64, 65, 127, 128, 129, 500])
def test_attention_at_the_edges_of_pages_and_tiles(dtype, d, bs, n):
    run_attention(dtype, 8, 2, d, bs, 3, [n, max(n - 1, 0)], layers=1, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,Hkv,M", [(2, 2, 1), (8, 2, 1), (8, 1, 1), (5, 1, 7), (8, 2, 16), (8, 2, 17), (8, 2, 32), (8, 2, 33), (8, 2, 60),
                                      (7, 1, 19), (16, 1, 4), (16, 1, 5), (8, 1, 128), (48, 1, 3), (160, 1, 2)])
def test_attention_for_any_number_of_rows(dtype, Hq, Hkv, M):
    run_attention(dtype, Hq, Hkv, 128, 64, M, [333], layers=1, seed=Hq + M)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_of_a_ragged_batch_with_row_counts(dtype):
    run_attention(dtype, 8, 2, 128, 32, 40, [700, 0, 31, 257], q_lens=[40, 5, 0, 17], layers=2)
    run_attention(dtype, 8, 2, 64, 64, 9, [1000, 3], q_lens=[1, 9], layers=3, layer0=1, n_call=2)


def test_attention_split_over_a_long_cache():
    run_attention("bf16", 8, 1, 128, 64, 5, [9001], layers=1, out_f32=1)
    run_attention("bf16", 8, 1, 128, 64, 33, [9001], layers=1, out_f32=1, seed=3)


@pytest.mark.parametrize("q_scale", [8.0, 60.0])
def test_attention_with_scores_that_climb_far_past_the_first_tile(q_scale):
    """Scores of hundreds: the first tile's reference has to give way."""
    for M in (2, 20):
        run_attention("bf16", 8, 2, 128, 64, M, [700], layers=1, q_scale=q_scale, seed=M)


@pytest.mark.parametrize("M", [4, 8, 20])
def test_attention_with_large_values_and_scores_that_climb(M):
    """Values of 2^100: sums of weights that are measured by an old reference must not carry them past float32.  (A cache long enough
    for every warp of the kernel for few rows to go from chunk to chunk.)"""
    run_attention("bf16", 16, 8, 64, 64, M, [30000] if M < 20 else [3000], layers=1, q_scale=30.0, v_log2=100, out_f32=1, seed=M)


@pytest.mark.parametrize("dtype,M", [("bf16", 1), ("bf16", 4), ("bf16", 9), ("fp32", 1)])
def test_attention_of_many_sequences(dtype, M):
    """More sequences than a warp has lanes, empty ones and ones without rows among them."""
    rng = np.random.default_rng(M)
    lens = [int(x) for x in rng.integers(0, 300, 70)]
    lens[0] = lens[33] = lens[69] = 0
    q_lens = [int(x) for x in rng.integers(0, M + 1, 70)]
    run_attention(dtype, 8, 2, 64, 16, M, lens, q_lens=q_lens, layers=1)
    run_attention(dtype, 4, 1, 64, 32, M, lens, layers=2, layer0=1, n_call=1)


@pytest.mark.parametrize("dtype,M", [("bf16", 1), ("bf16", 16), ("bf16", 40), ("fp32", 5)])
def test_workspace_of_the_least_alignment(dtype, M):
    run_attention(dtype, 8, 1, 128, 64, M, [2500], layers=1, ws_skip=16)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_see_nothing_are_zero(dtype):
    """Empty cache, empty rows of the mask."""
    got, lse = run_attention(dtype, 8, 2, 128, 64, 6, [0, 0], layers=1, density=0.0)
    assert np.all(got == 0) and np.all(np.isneginf(lse))
    run_attention(dtype, 8, 2, 128, 64, 6, [0, 70], layers=1, density=0.1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["k", "v"])
def test_infinities_and_nan_reach_only_the_rows_that_see_them(dtype, d, where):
    rng = np.random.default_rng(5)
    M, Hq, Hkv, bs, lens = 12, 8, 2, 64, [150]
    cfg = config(1, Hq, Hkv, d, bs, dtype)
    q4 = Q.Q4(1, Hkv, d, bs, lens, seed=2)
    q, _ = rows(rng, (1, 1, M, Hq, d), dtype)
    k, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    v, _ = rows(rng, (1, 1, M, Hkv, d), dtype)
    seen, mask = random_masks(rng, 1, M)
    ws = B.new_workspace(cfg, 1, 1, 150, M)

    def run():
        out, lse = torch.zeros(1, 1, M, Hq, d, dtype=torch_dtype(dtype), device="cuda"), torch.zeros(1, 1, M, Hq, device="cuda")
        B.specpv_verify_full_q4(cfg, 0, 1, q, k, v, mask, None, M, q4.cache(B), out, lse, ws)
        return out.cpu(), lse.cpu()

    clean, clean_lse = run()
    (k if where == "k" else v)[0, 0, 4, 1, 3] = float("nan")
    (k if where == "k" else v)[0, 0, 7, 0, 5] = float("inf") if where == "v" else float("nan")
    out, lse = run()
    for j in range(M):
        for h in range(Hq):
            hit = seen[0, j, 4] if h >= Hq // 2 else seen[0, j, 7]
            c = 3 if h >= Hq // 2 else 5
            if not hit:
                assert torch.equal(out[0, 0, j, h], clean[0, 0, j, h]) and lse[0, 0, j, h] == clean_lse[0, 0, j, h]
            elif where == "k":
                assert out[0, 0, j, h].isnan().all() and lse[0, 0, j, h].isnan()
            else:
                x = out[0, 0, j, h, c]
                assert x.isnan() if h >= Hq // 2 else x == float("inf")
                others = torch.arange(d) != c
                assert torch.equal(out[0, 0, j, h][others], clean[0, 0, j, h][others])


def test_a_bad_page_is_reported():
    for dtype in ("fp32", "bf16"):
        cfg = config(1, 8, 2, 64, 16, dtype)
        q4 = Q.Q4(1, 2, 64, 16, [100, 100])
        rng = np.random.default_rng(0)
        q, _ = rows(rng, (1, 2, 4, 8, 64), dtype)
        k, _ = rows(rng, (1, 2, 4, 2, 64), dtype)
        _, mask = random_masks(rng, 2, 4)
        out = torch.zeros_like(q)
        ws = B.new_workspace(cfg, 1, 2, 100, 4)
        good = q4.table.copy()
        for bad in (-1, q4.pool.shape[1], 2 ** 31 - 1):
            q4.table = good.copy()
            q4.table[1, 2] = bad
            B.specpv_verify_full_q4(cfg, 0, 1, q, k, k, mask, None, 4, q4.cache(B), out, None, ws)
            st, info = B.specpv_poll_status(ws)
            assert st == B.STATUS_NAMES.index("BAD_BLOCK_TABLE") and info[:3] == [1, 2, bad]
        q4.table = good
        B.specpv_verify_full_q4(cfg, 0, 1, q, k, k, mask, None, 4, q4.cache(B), out, None, ws)
        assert B.specpv_poll_status(ws)[0] == 0


# ---- commit ------------------------------------------------------------------------------------------------------
def run_commit(dtype, Hkv, d, bs, M, lens, taken, A, layers=2, with_values=True, with_summaries=True, seed=0, make=None, groups=None):
    """taken: per sequence the row numbers, or None for rows 0 .. A - 1."""
    rng = np.random.default_rng(seed)
    batch = len(lens)
    cfg = config(layers, 2 * Hkv, Hkv, d, bs, dtype)
    q4 = Q.Q4(layers, Hkv, d, bs, lens, seed=seed + 1, max_blocks=max(-(-(n + A) // bs) for n in lens))
    k, k64 = rows(rng, (layers, batch, M, Hkv, d), dtype)
    v, v64 = rows(rng, (layers, batch, M, Hkv, d), dtype)
    if make:
        make(k, v)
        k64, v64 = k.cpu().double().numpy(), v.cpu().double().numpy()
    n_taken = [A if taken is None else len(t) for t in (taken or lens)]
    accepted = None
    if taken is not None:
        accepted = torch.full((batch, A), -5, dtype=torch.int32)
        for b, t in enumerate(taken):
            accepted[b, : len(t)] = torch.tensor(t, dtype=torch.int32)
        accepted = accepted.cuda()
    shape = (layers, batch, Hkv, q4.max_blocks, d)
    kmax, kmin = (torch.full(shape, 7.0, dtype=torch_dtype(dtype), device="cuda") for _ in range(2))
    kv, vv = (torch.full((layers, batch, A, Hkv, d), 7.0, dtype=torch_dtype(dtype), device="cuda") for _ in range(2))
    ws = B.new_workspace(cfg, layers, batch, 64, 8)
    cache = q4.cache(B, max_seq_len=q4.max_blocks * bs)
    before = cache.pool.clone()
    n_dev = torch.tensor(n_taken, dtype=torch.int32, device="cuda")
    for l0, nl in groups or [(0, layers)]:
        B.specpv_commit_accepted_q4(cfg, l0, nl, k[l0:l0 + nl].contiguous(), v[l0:l0 + nl].contiguous(), M, accepted, n_dev, A, cache,
                                    kmax if with_summaries else None, kmin if with_summaries else None,
                                    kv[l0:l0 + nl] if with_values else None, vv[l0:l0 + nl] if with_values else None, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    assert cache.seq_lens.tolist() == [n + a for n, a in zip(lens, n_taken)]
    pool = cache.pool.cpu().numpy()
    want_pool = before.cpu().numpy().copy()
    want_max, want_min = np.full(shape, 7.0), np.full(shape, 7.0)
    want_k, want_v = np.full(kv.shape, 7.0), np.full(kv.shape, 7.0)
    for b, n in enumerate(lens):
        src = list(range(n_taken[b])) if taken is None else taken[b]
        for l in range(layers):
            for h in range(Hkv):
                pages = {}
                parts = []
                for x in (k64, v64):
                    r = x[l, b, src, h].reshape(len(src), d)
                    parts.append(Q.quantise(r))
                for a in range(len(src)):
                    i, t = divmod(n + a, bs)
                    if i not in pages:
                        pages[i] = [*Q.read_page(want_pool[l, q4.table[b, i], h], bs, d)[:2],
                                    want_pool[l, q4.table[b, i], h][bs * d:].view(np.uint16).reshape(4, bs).copy()]
                    for j in range(2):
                        pages[i][j][t] = parts[j][0][a]
                        pages[i][2][2 * j, t], pages[i][2][2 * j + 1, t] = Q.bf16_bits(parts[j][1][a]), Q.bf16_bits(parts[j][2][a])
                    want_k[l, b, a, h] = Q.values(parts[0][0][a], parts[0][1][a], parts[0][2][a])
                    want_v[l, b, a, h] = Q.values(parts[1][0][a], parts[1][1][a], parts[1][2][a])
                for i, (kc, vc, par) in pages.items():
                    want_pool[l, q4.table[b, i], h] = Q.write_page(kc, vc, par)
                    held = min(bs, n + len(src) - i * bs)
                    x = Q.values(kc[:held], Q.from_bits(par[0, :held]), Q.from_bits(par[1, :held]))
                    if np.isnan(x).any():
                        x = x[~np.isnan(x).any(1)]  # NaN loses against numbers
                    if len(x):
                        want_max[l, b, h, i], want_min[l, b, h, i] = x.max(0), x.min(0)
    if make is None:  # (NaN has many bit patterns)
        assert np.array_equal(pool, want_pool)
    if with_values:
        assert np.array_equal(kv.cpu().double().numpy(), want_k, equal_nan=True)
        assert np.array_equal(vv.cpu().double().numpy(), want_v, equal_nan=True)
    if with_summaries:
        assert np.array_equal(kmax.cpu().double().numpy(), want_max) and np.array_equal(kmin.cpu().double().numpy(), want_min)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bs", [(128, 64), (64, 16), (128, 32), (64, 64)])
@pytest.mark.parametrize("n", [0, 1, 7, 8, 15, 16, 63, 70])
def test_commit_of_accepted_rows(dtype, d, bs, n):
    run_commit(dtype, 2, d, bs, 20, [n, n + 3], [[0, 3, 4, 9, 19], [2]], 5, seed=n)


def test_commit_of_a_chunk_and_of_nothing():
    run_commit("bf16", 2, 128, 64, 150, [30, 64], None, 150, layers=1)
    run_commit("fp32", 1, 64, 16, 37, [5], None, 33, layers=1)
    run_commit("bf16", 1, 64, 32, 5, [10, 0], [[], [1, 1, 0]], 3, with_values=False)
    run_commit("bf16", 1, 64, 32, 5, [31], [[4, 2]], 2, with_summaries=False, layers=3, groups=[(0, 1), (1, 2)])


def test_commit_of_equal_tiny_huge_and_unholdable_rows():
    def make(k, v):
        k[:, :, 0], v[:, :, 0] = 0.0, -2.5
        k[:, :, 1], v[:, :, 1] = 1e-30, 1e-38
        k[:, :, 1, :, ::2] = 3e-30
        k[:, :, 2] *= 1e30
        v[:, :, 2] *= 1e-30
        k[:, :, 3, :, 5] = float("inf")
        v[:, :, 3, :, 2] = float("nan")
        k[:, :, 4, :, 0], k[:, :, 4, :, 1] = 3.3e38, -3.3e38  # their difference is no float32
    run_commit("bf16", 2, 64, 16, 6, [3], None, 6, make=make)
    run_commit("fp32", 2, 128, 32, 6, [3], None, 6, make=make)


def test_commit_faults_are_reported_and_skipped():
    cfg = config(1, 2, 1, 64, 16, "bf16")
    x = torch.randn(1, 2, 8, 1, 64, device="cuda").bfloat16()
    ws = B.new_workspace(cfg, 1, 2, 64, 8)
    n = torch.tensor([2, 2], dtype=torch.int32, device="cuda")
    for accepted, table, lens, status, want_lens in (
            ([[0, 1], [0, 1]], [[0, 1], [2, 3]], [31, 4], "CAPACITY", [31, 6]),
            ([[0, 8], [-1, 3]], [[0, 1], [2, 3]], [3, 4], "INVALID_ARG", [5, 6]),
            ([[0, 1], [0, 1]], [[0, 1], [4, 3]], [3, 4], "BAD_BLOCK_TABLE", [5, 6])):
        cache = B.CacheQ4(B.new_q4_pool(cfg, 4), torch.tensor(table, dtype=torch.int32, device="cuda"),
                          torch.tensor(lens, dtype=torch.int32, device="cuda"), 32)
        B.specpv_commit_accepted_q4(cfg, 0, 1, x, x, 8, torch.tensor(accepted, dtype=torch.int32, device="cuda"), n, 2, cache, None, None,
                                    None, None, ws)
        st, _ = B.specpv_poll_status(ws)
        assert B.STATUS_NAMES[st] == status and cache.seq_lens.tolist() == want_lens


# ---- refresh -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,bs", [(128, 64), (64, 16), (128, 16), (64, 32)])
def test_refresh_opens_the_selected_blocks(dtype, d, bs):
    rng = np.random.default_rng(1)
    layers, Hkv, budget = 2, 3, 6
    lens = [bs * 11 + 5, bs * 3, 0, bs * 6 + 1]
    cfg = config(layers, 3, Hkv, d, bs, dtype, budget_blocks=budget, buffer_tokens=10)
    q4 = Q.Q4(layers, Hkv, d, bs, lens, seed=4)
    count = [min(-(-n // bs), budget) for n in lens]
    idx = np.zeros((layers, 4, Hkv, budget), np.int32)
    blocks = budget + -(-10 // bs)
    table = rng.permutation(4 * blocks).reshape(4, blocks).astype(np.int32)
    pk, pv = (torch.full((layers, 4 * blocks, Hkv, bs, d), 7.0, dtype=torch_dtype(dtype), device="cuda") for _ in range(2))
    want_k, want_v = np.full(pk.shape, 7.0), np.full(pk.shape, 7.0)
    for b, n in enumerate(lens):
        nb = -(-n // bs)
        for l in range(layers):
            for h in range(Hkv):
                if nb:
                    pick = np.sort(np.append(rng.permutation(nb - 1)[: count[b] - 1], nb - 1))
                    idx[l, b, h, : count[b]] = pick
                    for s, i in enumerate(pick):
                        held = min(bs, n - i * bs)
                        want_k[l, table[b, s], h, :held] = q4.k[b][l, h, i * bs: i * bs + held]
                        want_v[l, table[b, s], h, :held] = q4.v[b][l, h, i * bs: i * bs + held]
    plens = torch.full((4,), -1, dtype=torch.int32, device="cuda")
    part = B.Cache(pk, pv, torch.from_numpy(table).cuda(), plens, blocks * bs)
    ws = B.new_workspace(cfg, layers, 4, 64, 8)
    B.specpv_refresh_partial_q4(cfg, q4.cache(B), torch.from_numpy(idx).cuda(), torch.tensor(count, dtype=torch.int32, device="cuda"), part,
                                plens, ws)
    assert B.specpv_poll_status(ws)[0] == 0
    assert np.array_equal(pk.cpu().double().numpy(), want_k) and np.array_equal(pv.cpu().double().numpy(), want_v)
    assert plens.tolist() == [(c - 1) * bs + n - (-(-n // bs) - 1) * bs if c else 0 for c, n in zip(count, lens)]
    # a block number past the sequence, and page ids outside the pools
    idx_t = torch.from_numpy(idx).cuda()
    for change, status in ((lambda: idx_t.__setitem__((1, 0, 2, 3), 12), "INVALID_ARG"),
                           (lambda: part.block_table.__setitem__((0, 1), 4 * blocks), "BAD_BLOCK_TABLE")):
        change()
        B.specpv_refresh_partial_q4(cfg, q4.cache(B), idx_t, torch.tensor(count, dtype=torch.int32, device="cuda"), part, plens, ws)
        assert B.STATUS_NAMES[B.specpv_poll_status(ws)[0]] == status
        idx_t.copy_(torch.from_numpy(idx))


# ---- together ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_decode_loop_over_a_cache_in_4_bits(dtype, d):
    """Prefill in chunks, scores on the summaries, selection, refresh, full and partial verification, commit: the 4-bit cache gives
    what an ordinary cache of the values that it stands for gives."""
    torch.manual_seed(0)
    layers, Hq, Hkv, bs, M, budget = 2, 8, 2, 16, 10, 8
    dt = torch_dtype(dtype)
    cfg = config(layers, Hq, Hkv, d, bs, dtype, sink_blocks=2, local_blocks=2, budget_blocks=budget, buffer_tokens=24)
    blocks, prompt = 30, [300, 211]
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    table = torch.randperm(2 * blocks).reshape(2, blocks).int().cuda()
    q4 = B.CacheQ4(B.new_q4_pool(cfg, 2 * blocks), table, lens, blocks * bs)
    pools = [torch.zeros(layers, 2 * blocks, Hkv, bs, d, dtype=dt, device="cuda") for _ in range(2)]
    plain = B.Cache(*pools, table, torch.zeros_like(lens), blocks * bs)
    kmax, kmin = (torch.zeros(layers, 2, Hkv, blocks, d, dtype=dt, device="cuda") for _ in range(2))
    pmax, pmin = torch.zeros_like(kmax), torch.zeros_like(kmin)
    ws = B.new_workspace(cfg, layers, 2, blocks * bs, 128)

    def append(k, v, accepted, n, A):
        kv, vv = (torch.zeros(layers, 2, A, Hkv, d, dtype=dt, device="cuda") for _ in range(2))
        B.specpv_commit_accepted_q4(cfg, 0, layers, k, v, k.shape[2], accepted, n, A, q4, kmax, kmin, kv, vv, ws)
        order = torch.arange(A, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()
        B.specpv_commit_accepted(cfg, 0, layers, kv, vv, A, order, n, A, plain, pmax, pmin, ws)

    done = [0, 0]
    while any(a < b for a, b in zip(done, prompt)):
        n = [min(100, b - a) for a, b in zip(done, prompt)]
        append(torch.randn(layers, 2, 100, Hkv, d, device="cuda").to(dt), torch.randn(layers, 2, 100, Hkv, d, device="cuda").to(dt), None,
               torch.tensor(n, dtype=torch.int32, device="cuda"), 100)
        done = [a + b for a, b in zip(done, n)]
    part_blocks = budget + 4
    parts = [B.Cache(*(torch.zeros(layers, 2 * part_blocks, Hkv, bs, d, dtype=dt, device="cuda") for _ in range(2)),
                     torch.arange(2 * part_blocks, dtype=torch.int32, device="cuda").reshape(2, -1).contiguous(),
                     torch.zeros(2, dtype=torch.int32, device="cuda"), part_blocks * bs) for _ in range(2)]
    for step in range(4):
        q = torch.randn(layers, 2, M, Hq, d, device="cuda").to(dt)
        k, v = (torch.randn(layers, 2, M, Hkv, d, device="cuda").to(dt) for _ in range(2))
        mask = torch.tensor([[[(1 << (j + 1)) - 1] for j in range(M)]] * 2, dtype=torch.int64, device="cuda")
        out, lse = (torch.zeros(2, layers, 2, M, Hq, *s, dtype=t, device="cuda") for s, t in (((d,), dt), ((), torch.float32)))
        B.specpv_verify_full_q4(cfg, 0, layers, q, k, v, mask, None, M, q4, out[0], lse[0], ws)
        B.specpv_verify_full(cfg, 0, layers, q, k, v, mask, None, M, plain, out[1], lse[1], ws)
        # both round their weights (twice 2^-8 of a mean of |v| < 1.5, for numerator and denominator) and outputs (2^-8 of < 1)
        tol = 8 * Q.HALF_BF16 if dtype == "bf16" else 1e-5
        assert (out[0].float() - out[1].float()).abs().max() <= tol and (lse[0] - lse[1]).abs().max() <= tol
        accepted = torch.arange(3, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()
        append(k, v, accepted, torch.tensor([3, 1 + step % 2], dtype=torch.int32, device="cuda"), 3)
        assert torch.equal(q4.seq_lens, plain.seq_lens) and torch.equal(kmax, pmax) and torch.equal(kmin, pmin)
        scores = torch.zeros(layers, 2, Hkv, blocks, device="cuda")
        idx, count = torch.zeros(layers, 2, Hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        B.specpv_score_blocks(cfg, 0, layers, q, None, M, None, kmax, kmin, plain, scores, ws)
        B.specpv_select_partial_kv(cfg, layers, scores, q4.seq_lens, 2, blocks, idx, count, ws)
        B.specpv_refresh_partial_q4(cfg, q4, idx, count, parts[0], parts[0].seq_lens, ws)
        B.specpv_refresh_partial(cfg, plain, idx, count, parts[1], parts[1].seq_lens, ws)
        assert torch.equal(parts[0].seq_lens, parts[1].seq_lens)
        assert torch.equal(parts[0].k_pool, parts[1].k_pool) and torch.equal(parts[0].v_pool, parts[1].v_pool)
        B.specpv_verify_partial(cfg, 0, layers, q, k, v, mask, None, M, parts[0], out[0], lse[0], ws)
        assert B.specpv_poll_status(ws)[0] == 0 and out[0].isfinite().all()


def test_captured_and_replayed():
    """Attention and commit in a CUDA graph, replayed with other inputs, on a stream of its own."""
    torch.manual_seed(1)
    cfg = config(1, 8, 2, 128, 64, "bf16")
    q4 = Q.Q4(1, 2, 128, 64, [400], max_blocks=8)
    cache = q4.cache(B, max_seq_len=512)
    q, k, v = (torch.randn(1, 1, 6, h, 128, device="cuda").bfloat16() for h in (8, 2, 2))
    mask = torch.tensor([[[(1 << (j + 1)) - 1] for j in range(6)]], dtype=torch.int64, device="cuda")
    n, out = torch.tensor([2], dtype=torch.int32, device="cuda"), torch.zeros_like(q)
    ws = B.new_workspace(cfg, 1, 1, 512, 6)

    def step():
        B.specpv_verify_full_q4(cfg, 0, 1, q, k, v, mask, None, 6, cache, out, None, ws)
        B.specpv_commit_accepted_q4(cfg, 0, 1, k, v, 6, None, n, 2, cache, None, None, None, None, ws)

    start = cache.pool.clone()
    want = []
    for _ in range(3):
        step()
        want.append(out.clone())
    final = cache.pool.clone()
    cache.pool.copy_(start)
    cache.seq_lens.fill_(400)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for x in want:
        graph.replay()
        torch.cuda.synchronize()
        # the number of splits goes by max_seq_len, so the sums are the same ones
        assert torch.equal(out, x)
    assert torch.equal(cache.pool, final) and cache.seq_lens.item() == 406


def test_two_streams_at_once():
    """Two calls under way together, a workspace each, over one cache, give what they give one after the other."""
    rng = np.random.default_rng(0)
    cfg = config(1, 8, 2, 128, 64, "bf16")
    q4 = Q.Q4(1, 2, 128, 64, [3000])
    cache = q4.cache(B)
    calls = []
    for M in (1, 40):
        q, _ = rows(rng, (1, 1, M, 8, 128), "bf16")
        k, _ = rows(rng, (1, 1, M, 2, 128), "bf16")
        _, mask = random_masks(rng, 1, M)
        calls.append((M, q, k, mask, torch.zeros_like(q), B.new_workspace(cfg, 1, 1, 3000, M), torch.cuda.Stream()))

    def run(c, stream):
        M, q, k, mask, out, ws, _ = c
        with torch.cuda.stream(stream):
            B.specpv_verify_full_q4(cfg, 0, 1, q, k, k, mask, None, M, cache, out, None, ws)

    want = []
    for c in calls:
        run(c, torch.cuda.current_stream())
        torch.cuda.synchronize()
        want.append(c[4].clone())
        c[4].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for c in calls:
            run(c, c[6])
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert torch.equal(c[4], w) and B.specpv_poll_status(c[5])[0] == 0


def test_two_graphs_over_one_workspace():
    """Captured calls of both kernels, replayed in turn on one stream, each against a cache that grows between replays."""
    rng = np.random.default_rng(1)
    cfg = config(1, 8, 2, 128, 64, "bf16")
    q4 = Q.Q4(1, 2, 128, 64, [2000], max_blocks=40)
    cache = q4.cache(B, max_seq_len=40 * 64)
    ws = B.new_workspace(cfg, 1, 1, 40 * 64, 40)
    stream = torch.cuda.Stream()
    calls = []
    for M in (1, 40):
        q, _ = rows(rng, (1, 1, M, 8, 128), "bf16")
        k, _ = rows(rng, (1, 1, M, 2, 128), "bf16")
        _, mask = random_masks(rng, 1, M)
        calls.append((M, q, k, mask, torch.zeros_like(q), torch.zeros(1, 1, M, 8, device="cuda")))

    def run(c):
        M, q, k, mask, out, lse = c
        B.specpv_verify_full_q4(cfg, 0, 1, q, k, k, mask, None, M, cache, out, lse, ws)

    graphs = []
    with torch.cuda.stream(stream):
        for c in calls:
            run(c)
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                run(c)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    for step in range(6):
        for c, graph in zip(calls, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
                replayed = c[4].clone(), c[5].clone()
                run(c)
            torch.cuda.synchronize()
            assert torch.equal(replayed[0], c[4]) and torch.equal(replayed[1], c[5])
            B.specpv_commit_accepted_q4(cfg, 0, 1, c[2], c[2], c[0], None, one, 1, cache, None, None, None, None, ws)
            torch.cuda.synchronize()
    assert cache.seq_lens.tolist() == [2012] and B.specpv_poll_status(ws)[0] == 0
