"""The binding tells the two kinds of cache apart (no GPU needed: nothing is launched)."""
import pytest
import torch

from paper_2512_02337_b200 import binding as B
from paper_2512_02337_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


@pytest.fixture(params=["native", "ctypes"])
def calls(request, monkeypatch):
    if request.param == "ctypes":
        monkeypatch.setattr(B, "_pycalls", B._CtypesCalls())


def caches():
    cfg = B.make_config(1, 4, 2, 64, 16, "bf16", 1, 1, 4, 16)
    table, lens = torch.zeros(1, 6, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    plain = B.Cache(*(torch.zeros(1, 6, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)), table, lens, 96)
    return cfg, plain, B.CacheQ4(B.new_q4_pool(cfg, 6, device="cpu"), table, lens, 96)


def test_an_ordinary_cache_in_place_of_one_in_4_bits_is_refused(calls):
    cfg, plain, q4 = caches()
    x, ints, ws = torch.zeros(1, 1, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 16, dtype=torch.int32), torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(TypeError):
        B.specpv_verify_full_q4(cfg, 0, 1, x, x, x, ints, None, 2, plain, x, None, ws, stream=0)
    with pytest.raises(TypeError):
        B.specpv_commit_accepted_q4(cfg, 0, 1, x, x, 2, None, ints, 2, plain, None, None, None, None, ws, stream=0)
    with pytest.raises(TypeError):
        B.specpv_refresh_partial_q4(cfg, plain, ints, ints, plain, ints, ws, stream=0)


def test_a_cache_in_4_bits_in_place_of_an_ordinary_one_is_refused(calls):
    cfg, plain, q4 = caches()
    x, ints, ws = torch.zeros(1, 1, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 16, dtype=torch.int32), torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(TypeError):
        B.specpv_refresh_partial_q4(cfg, q4, ints, ints, q4, ints, ws, stream=0)
    with pytest.raises(TypeError):
        B.specpv_accumulate_attention(cfg, 0, 1, x, x, 2, None, ints, 2, q4, x, ws, stream=0)
    with pytest.raises(TypeError):
        B.specpv_evict_tokens(cfg, q4, x, 8, 1, 1, ints, ws, stream=0)
    with pytest.raises(TypeError):
        B.specpv_verify_full(cfg, 0, 1, x, x, x, ints, None, 2, q4, x, None, ws, stream=0)
