"""Arguments that the calls around the 4-bit cache and the eviction refuse on the host (no GPU needed), and the format's reference."""
import ctypes

import numpy as np
import pytest

from paper_2512_02337_b200 import binding as B
from paper_2512_02337_b200 import build as build_mod
from tests import q4_util as Q

OK, INVALID, SHAPE, BUDGET, CAPACITY = 0, 1, 2, 3, 4


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


@pytest.fixture()
def env():
    buf = np.zeros(4096, dtype=np.float32)  # 16-byte aligned host memory stands in for device pointers: nothing is launched
    ptr = buf.ctypes.data + (-buf.ctypes.data) % 16
    cfg = B.make_config(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, block_tokens=64, dtype="bf16", sink_blocks=1, local_blocks=2,
                        budget_blocks=8, buffer_tokens=64)
    return buf, ptr, cfg


def q4(p, **over):
    return B.PagedQ4(**{**dict(pool=p, block_table=p, seq_lens=p, batch=1, max_blocks=16, n_pages=16, max_seq_len=1024), **over})


def kv(p, **over):
    return B.PagedKV(**{**dict(k_pool=p, v_pool=p, block_table=p, seq_lens=p, batch=1, max_blocks=16, n_pages=16, max_seq_len=1024), **over})


BAD_CACHES = [(dict(block_table=None), INVALID), (dict(seq_lens=None), INVALID), (dict(batch=0), INVALID), (dict(max_blocks=0), INVALID),
              (dict(n_pages=0), INVALID), (dict(max_seq_len=-1), INVALID), (dict(max_seq_len=1025), CAPACITY)]


def test_attention(env):
    _, p, cfg = env

    def call(cache=None, layer0=0, n=1, q=p, k=p, v=p, mask=p, M=16, out=p, ws=p, size=1 << 30):
        c = cache or q4(p)
        return B.lib().specpv_verify_full_q4(ctypes.byref(cfg), layer0, n, q, k, v, mask, None, M, ctypes.byref(c), out, None, ws, size, None)
    for over, want in BAD_CACHES + [(dict(pool=None), INVALID), (dict(pool=p + 8), INVALID)]:
        assert call(q4(p, **over)) == want, over
    for name in ("q", "k", "v", "mask", "out", "ws"):
        assert call(**{name: None}) == INVALID
        if name != "mask":
            assert call(**{name: p + 2}) == INVALID
    assert call(layer0=2) == INVALID and call(layer0=-1) == INVALID and call(n=3) == INVALID and call(n=0) == INVALID
    assert call(M=0) == INVALID and call(M=129) == CAPACITY and call(size=1024) == CAPACITY
    assert B.lib().specpv_verify_full_q4(ctypes.byref(cfg), 0, 1, p, p, p, p, None, 16, None, p, None, p, 1 << 30, None) == INVALID


def test_commit(env):
    _, p, cfg = env

    def call(cache=None, layer0=0, n=1, k=p, v=p, M=16, accepted=p, taken=p, A=4, kmax=None, kmin=None, kv=None, vv=None, ws=p, size=4096):
        c = cache or q4(p)
        return B.lib().specpv_commit_accepted_q4(ctypes.byref(cfg), layer0, n, k, v, M, accepted, taken, A, ctypes.byref(c), kmax, kmin,
                                                 kv, vv, ws, size, None)
    for over, want in BAD_CACHES + [(dict(pool=None), INVALID), (dict(pool=p + 8), INVALID)]:
        assert call(q4(p, **over)) == want, over
    for name in ("k", "v", "taken", "ws"):
        assert call(**{name: None}) == INVALID
    assert call(k=p + 4) == INVALID and call(v=p + 4) == INVALID
    assert call(kmax=p) == INVALID and call(kmin=p) == INVALID and call(kv=p) == INVALID and call(vv=p) == INVALID
    assert call(kv=p + 4, vv=p) == INVALID
    assert call(M=0) == INVALID and call(A=0) == INVALID and call(n=3) == INVALID and call(size=8) == INVALID
    assert call(accepted=None, A=17) == CAPACITY  # more rows than there are


def test_refresh(env):
    _, p, cfg = env

    def call(cache=None, part=None, idx=p, count=p, lens=p, ws=p, size=4096):
        c, t = cache or q4(p), part or kv(p)
        return B.lib().specpv_refresh_partial_q4(ctypes.byref(cfg), ctypes.byref(c), idx, count, ctypes.byref(t), lens, ws, size, None)
    for over, want in BAD_CACHES + [(dict(pool=None), INVALID), (dict(pool=p + 8), INVALID)]:
        assert call(q4(p, **over)) == want, over
    for name in ("idx", "count", "lens", "ws"):
        assert call(**{name: None}) == INVALID
    for over, want in [(dict(k_pool=None), INVALID), (dict(v_pool=p + 8), INVALID), (dict(batch=2), INVALID), (dict(n_pages=0), INVALID),
                       (dict(max_blocks=8), CAPACITY)]:  # eight blocks of budget, a buffer behind them
        assert call(part=kv(p, **over)) == want, over


def test_account(env):
    _, p, cfg = env

    def call(cache=None, layer0=0, n=1, q=p, lse=p, M=16, accepted=p, taken=p, A=4, acc=p, ws=p, size=4096):
        c = cache or kv(p)
        return B.lib().specpv_accumulate_attention(ctypes.byref(cfg), layer0, n, q, lse, M, accepted, taken, A, ctypes.byref(c), acc, ws,
                                                   size, None)
    for over, want in BAD_CACHES + [(dict(k_pool=None), INVALID), (dict(k_pool=p + 8), INVALID)]:
        assert call(kv(p, **over)) == want, over
    for name in ("q", "lse", "taken", "acc", "ws"):
        assert call(**{name: None}) == INVALID
    assert call(q=p + 8) == INVALID and call(acc=p + 4) == INVALID
    assert call(M=0) == INVALID and call(A=0) == INVALID and call(layer0=2) == INVALID and call(size=8) == INVALID
    assert call(M=129) == CAPACITY and call(accepted=None, A=17) == CAPACITY


def test_eviction(env):
    _, p, cfg = env

    def call(cache=None, acc=p, keep=64, sink=4, local=8, idx=p, ws=p, size=4096, cfg=cfg):
        c = cache or kv(p)
        return B.lib().specpv_evict_tokens(ctypes.byref(cfg), ctypes.byref(c), acc, keep, sink, local, idx, ws, size, None)
    for over, want in BAD_CACHES + [(dict(k_pool=None), INVALID), (dict(v_pool=p + 8), INVALID), (dict(batch=40000), CAPACITY)]:
        assert call(kv(p, **over)) == want, over
    for name in ("acc", "idx", "ws"):
        assert call(**{name: None}) == INVALID
    assert call(acc=p + 4) == INVALID and call(size=8) == INVALID
    assert call(keep=12) == BUDGET and call(keep=0, sink=0, local=0) == BUDGET and call(sink=-1) == BUDGET and call(local=-1) == BUDGET
    assert call(sink=2 ** 31 - 1, local=2 ** 31 - 1) == BUDGET  # their sum is no int32


def test_binding_takes_descriptors_of_the_cache():
    import torch
    cfg = B.make_config(2, 8, 2, 64, 16, "bf16", 1, 2, 8, 64)
    pool = B.new_q4_pool(cfg, 5, device="cpu")
    assert tuple(pool.shape) == (2, 5, 2, 16 * 72) and pool.dtype == torch.uint8 and not pool.any()
    table, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    d = B.CacheQ4(pool, table, lens, 60).desc()
    assert (d.pool, d.block_table, d.seq_lens) == (pool.data_ptr(), table.data_ptr(), lens.data_ptr())
    assert (d.batch, d.max_blocks, d.n_pages, d.max_seq_len) == (3, 4, 5, 60)


# ---- the reference of the format ---------------------------------------------------------------------------------
@pytest.mark.parametrize("d,bs", [(64, 16), (128, 64)])
def test_pages_are_read_as_they_are_written(d, bs):
    rng = np.random.default_rng(0)
    k, v = rng.integers(0, 16, (2, bs, d))
    par = rng.integers(0, 65536, (4, bs)).astype(np.uint16)
    raw = Q.write_page(k, v, par)
    assert raw.shape == (bs * (d + 8),)
    k2, v2, p2 = Q.read_page(raw, bs, d)
    assert np.array_equal(k, k2) and np.array_equal(v, v2) and np.array_equal(p2, Q.from_bits(par), equal_nan=True)


def test_bfloat16_of_the_reference():
    import torch
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(20000) * np.exp2(rng.integers(-140, 127, 20000)), [0.0, 1e-45, 3.4e38, -3.4e38, np.inf]])
    x = x.astype(np.float32).astype(np.float64)
    assert np.array_equal(Q.bf16(x), torch.from_numpy(x).float().bfloat16().double().numpy())


def test_quantisation_is_off_by_half_a_step():
    """A value is at most half a step from its row's element, plus what the rounding of scale, offset and value to bfloat16 adds."""
    rng = np.random.default_rng(2)
    x = Q.bf16(rng.standard_normal((400, 128)) * np.exp(rng.standard_normal((400, 1))))
    n, s, o = Q.quantise(x)
    y = Q.values(n, s, o)
    size = np.abs(x).max(-1)
    # half a step; at the ends of the range, fifteen roundings of the scale; the offset's; the value's own
    assert np.all(np.abs(y - x) <= (s / 2 + 31 * s * Q.HALF_BF16 + np.abs(o) * Q.HALF_BF16)[:, None] + Q.HALF_BF16 * size[:, None])
    assert n.min() == 0 and n.max() == 15


def test_what_launches_cannot_number_is_refused(env):
    """More than 65535 (layer, sequence) pairs in a call, row counts and capacities past int32: an error before any launch."""
    _, p, cfg = env
    many, long = dict(batch=40000), dict(max_blocks=2 ** 31 // 16)
    huge = 2 ** 31 - 1
    lib, c = B.lib(), ctypes.byref(cfg)
    for over in (many, long):
        a, b = ctypes.byref(q4(p, **over)), ctypes.byref(kv(p, **over))
        assert lib.specpv_verify_full_q4(c, 0, 2, p, p, p, p, None, 16, a, p, None, p, 1 << 40, None) == CAPACITY
        assert lib.specpv_commit_accepted_q4(c, 0, 2, p, p, 16, p, p, 4, a, None, None, None, None, p, 4096, None) == CAPACITY
        part = ctypes.byref(kv(p, **many)) if over is many else ctypes.byref(kv(p))
        assert lib.specpv_refresh_partial_q4(c, a, p, p, part, p, p, 4096, None) == CAPACITY
        assert lib.specpv_accumulate_attention(c, 0, 2, p, p, 16, p, p, 4, b, p, p, 4096, None) == CAPACITY
        assert lib.specpv_evict_tokens(c, b, p, 64, 4, 8, p, p, 4096, None) == CAPACITY
    a, b = ctypes.byref(q4(p)), ctypes.byref(kv(p))
    assert lib.specpv_commit_accepted_q4(c, 0, 1, p, p, 16, p, p, huge, a, None, None, None, None, p, 4096, None) == CAPACITY
    assert lib.specpv_accumulate_attention(c, 0, 1, p, p, 16, p, p, huge, b, p, p, 4096, None) == CAPACITY
