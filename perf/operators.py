"""Timing cases of the calls around a KV cache held in 4 bits, and of eviction by accumulated attention weight.

Kinds of pass
  attend      tree-masked attention of a step's tokens over a full cache held in 4 bits
  commit      a step's accepted rows, or a chunk of a prefill, quantised and appended to such a cache, with the summaries
              of the blocks they touch and the values that the rows now stand for
  refresh     the selected blocks of such a cache, copied into an ordinary partial cache
  accumulate  the attention weight that every cached token received from a step's accepted rows, added to its account
  evict       the tokens with the least accumulated weight leave a cache, the others close up

A cache in 4 bits.  A page holds, per KV head, the codes of its keys, those of its values and four rows of bfloat16
numbers, one per token: key scale, key offset, value scale, value offset.  Code n (0 .. 15) stands for
bfloat16((16 + n) * scale + offset).  Key codes are laid out [d / 32][token][16 bytes], value codes [token / 16][d]
[8 bytes]; a 32-bit word holds eight of them, of consecutive channels (keys) or tokens (values): element 2 i in bits
4 i .. 4 i + 3, element 2 i + 1 in bits 16 + 4 i .., the whole word then rotated left by three bits.
A row is quantised to scale = bfloat16((max - min) / 15), offset = bfloat16(min - 16 scale) and the nearest codes.
"""
from __future__ import annotations

import math

import torch

own = False

BASE = dict(layers=32, hq=32, hkv=8, d=128, bs=64, dtype="bf16", m=60, shuffle=False)
HEAD = 256 << 10  # what every workspace begins with


def _case(name, kind, ctx, **over):
    c = dict(BASE, kind=kind, ctx=ctx, **over)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decoded token over a short context, one layer: latency
        _case("attend_token_2k", "attend", "2047", layers=1, m=1),
        # plain decoding of four long sequences, pages in any order
        _case("attend_batch4_token", "attend", "98304,114688,122881,131072", layers=4, m=1, shuffle=True),
        # a draft tree of 60 nodes over 128K tokens: the full verification of a refresh
        _case("attend_tree_128k", "attend", "131072", layers=8),
        # the tiny float32 configuration, pages of 16 tokens
        _case("attend_fp32_tiny", "attend", "2048", layers=1, hq=8, hkv=2, d=64, bs=16, dtype="fp32", m=16),
        # the accepted tokens of a step, all layers
        _case("commit_step", "commit", "32700", rows=5),
        # a chunk of a prompt, some layers
        _case("commit_prefill", "commit", "6001", layers=16, m=2048, rows=2048),
        # the 4096-token partial cache rebuilt at 32K tokens, all layers
        _case("refresh_4k", "refresh", "32768", budget=64),
        # two sequences, head size 64, 16-token pages and the 512-token budget
        _case("refresh_512_d64", "refresh", "7001,9000", layers=8, d=64, bs=16, budget=32, shuffle=True),
        # after a partial step: 5 accepted rows over the partial cache, all layers
        _case("accumulate_4k", "accumulate", "4261", rows=5),
        # after a step over a long cache
        _case("accumulate_96k", "accumulate", "98309", layers=12, rows=7),
        # a cache of 4096 tokens and a buffer that has filled up, all layers
        _case("evict_4k", "evict", "4352", keep=4096, sink=32, local=128),
        # a long prompt cut down after its prefill, two sequences
        _case("evict_prompt", "evict", "24001,19999", layers=8, keep=8192, sink=32, local=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "commit", "refresh", "accumulate", "evict"])
    over = dict(bs=rng.choice([16, 32, 64, 64]), d=rng.choice([64, 128, 128]), shuffle=rng.random() < 0.4)
    over["hq"] = rng.choice([8, 16, 32, 32, 40, 64])
    over["dtype"] = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    small = over["dtype"] == "fp32"
    batch = rng.choice([1, 1, 2, 3, 4])
    top = {"attend": 4000 if small else 131072, "commit": 65536, "refresh": 65536, "accumulate": 16384 if small else 131072,
           "evict": 32768}[kind]
    longest = _log_int(rng, 200, top)
    ctx = [longest if b == 0 else rng.randint(longest // 2, longest) for b in range(batch)]
    # the cache, in bytes of 16 or 32 bits, up to which a listed case of the kind goes
    most = {"attend": 1e8 if small else 4e9, "commit": 4e9, "refresh": 4e9, "accumulate": 0.5e9 if small else 4e9, "evict": 1.5e9}[kind]
    width = 4 if small and kind in ("accumulate", "evict") else 2
    layers = int(most / (batch * longest * 8 * 2 * over["d"] * width))
    over["layers"] = max(1, min(rng.choice([1, 4, 8, 16, 32]), layers))
    if kind == "attend":
        over["m"] = rng.choice([1, 1, 2, rng.randint(3, 16), rng.randint(17, 64)])
    elif kind == "commit":
        over["m"] = rng.choice([rng.randint(8, 64), rng.randint(8, 64), _log_int(rng, 100, 1500)])
        over["rows"] = over["m"] if over["m"] > 64 else rng.randint(1, 8)
        over["layers"] = min(over["layers"], max(1, 16384 // (batch * over["rows"])))
    elif kind == "refresh":
        over["budget"] = max(11, rng.choice([256, 512, 1024, 2048, 4096]) // over["bs"])
    elif kind == "accumulate":
        over["m"] = rng.randint(8, 64)
        over["rows"] = rng.randint(1, 8)
    else:
        over["keep"] = rng.randint(max(150, longest // 3), max(160, longest - 1))
        over["sink"] = rng.choice([0, 4, 32])
        over["local"] = rng.choice([1, 64, 100])
    case = _case(None, kind, ",".join(str(c) for c in ctx), **over)
    largest = [work(c) for c in listed()]
    while case["layers"] > 1 and any(work(case)[k] > 0.9 * max(w[k] for w in largest) for k in ("bytes", "flops")):
        case["layers"] -= case["layers"] // 4 or 1  # no more than the largest listed case
    return case


# ---- the cache in 4 bits -------------------------------------------------------------------------------------------
def _pack(e):
    """[.., 8] codes -> [..] int32 words."""
    n = (e[..., 0] | e[..., 2] << 4 | e[..., 4] << 8 | e[..., 6] << 12 | e[..., 1] << 16 | e[..., 3] << 20 | e[..., 5] << 24 | e[..., 7] << 28)
    return n << 3 | (n >> 29) & 7


def _unpack(w):
    """[..] int32 words -> [.., 8] codes."""
    n = (w >> 3) & 0x1FFFFFFF | w << 29
    shifts = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], dtype=torch.int32, device=w.device)
    return n[..., None] >> shifts & 15


def _pages(k, v, params, d):
    """Codes [.., bs, d] of keys and values and params [.., 4, bs] (bfloat16) -> pages [.., bs * (d + 8)] of bytes."""
    lead, bs = k.shape[:-2], k.shape[-2]
    kw = _pack(k.reshape(*lead, bs, d // 32, 4, 8)).transpose(-3, -2)                               # [d / 32][bs][4]
    vw = _pack(v.reshape(*lead, bs // 16, 2, 8, d).permute(*range(len(lead)), -4, -1, -3, -2))      # [bs / 16][d][2]
    parts = [kw.reshape(*lead, -1), vw.reshape(*lead, -1), params.contiguous().reshape(*lead, 4 * bs)]
    return torch.cat([x.contiguous().view(torch.uint8) for x in parts], -1)


def _codes(pages, bs, d):
    """Pages -> codes of keys and values [.., bs, d] and params [.., 4, bs]."""
    lead, n = pages.shape[:-1], bs * d // 2
    kw, vw = (pages[..., i * n:(i + 1) * n].contiguous().view(torch.int32) for i in range(2))
    k = _unpack(kw.reshape(*lead, d // 32, bs, 4)).transpose(-4, -3).reshape(*lead, bs, d)
    v = _unpack(vw.reshape(*lead, bs // 16, d, 2)).permute(*range(len(lead)), -4, -2, -1, -3).reshape(*lead, bs, d)
    return k, v, pages[..., 2 * n:].contiguous().view(torch.bfloat16).reshape(*lead, 4, bs)


def _values(codes, scale, offset):
    """What codes [.., bs, d] with scale and offset [.., bs] stand for, in float32."""
    return ((codes + 16) * scale.float()[..., None] + offset.float()[..., None]).bfloat16().float()


def _quantise(x):
    """Rows [.., d] -> codes, scale, offset."""
    x = x.float()
    lo, hi = x.amin(-1), x.amax(-1)
    scale = ((hi - lo) / 15).bfloat16()
    s = scale.float()
    offset = (lo - 16 * s).bfloat16()
    base = offset.float() + 16 * s
    n = ((x - base[..., None]) / s[..., None]).round().nan_to_num(0.0).clamp(0, 15)
    return n.int(), scale, offset


def _page_table(case, n_blocks, gen):
    batch = len(_ctx(case))
    order = torch.randperm(batch * n_blocks, generator=gen, device="cuda") if case["shuffle"] else torch.arange(batch * n_blocks, device="cuda")
    return order.reshape(batch, n_blocks).int().contiguous()


# ---- what a program holds before the call --------------------------------------------------------------------------
def _ctx(case):
    return [int(c) for c in case["ctx"].split(",")]


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _workspace_bytes(case, rows):
    """Room for the partial results of a call over all its layers, the sizes that the library asks for."""
    g = case["hq"] // case["hkv"]
    tok = 128 // g
    packed = max(-(-rows * g // 256) * 256, -(-rows // (2 * tok)) * 256)
    base = case["hkv"] * case["layers"] * len(_ctx(case))
    return HEAD + (8 * 148 + base) * packed * (case["d"] + 2) * 4 + 256


def _q4_cache(case, n_blocks, gen):
    """Keys and values ~ N(0, 1), 2 % of the tokens three times as large, quantised page by page."""
    batch, d, bs = len(_ctx(case)), case["d"], case["bs"]
    pool = torch.empty(case["layers"], batch * n_blocks, case["hkv"], bs * (d + 8), dtype=torch.uint8, device="cuda")
    for layer in range(case["layers"]):
        shape = (batch * n_blocks, case["hkv"], bs)
        loud = 1 + 2 * (torch.rand(shape, generator=gen, device="cuda") < 0.02).float()[..., None]
        k, ks, ko = _quantise(torch.randn(*shape, d, generator=gen, device="cuda") * loud)
        v, vs, vo = _quantise(torch.randn(*shape, d, generator=gen, device="cuda") * loud)
        pool[layer] = _pages(k, v, torch.stack([ks, ko, vs, vo], -2), d)
    return pool


def _cache(case, n_blocks, gen):
    """An ordinary cache with the same kind of keys and values."""
    shape = (case["layers"], len(_ctx(case)) * n_blocks, case["hkv"], case["bs"], case["d"])
    out = []
    for _ in range(2):
        x = torch.empty(shape, dtype=_dtype(case), device="cuda")
        for layer in range(case["layers"]):
            loud = 1 + 2 * (torch.rand(shape[1:-1], generator=gen, device="cuda") < 0.02).float()[..., None]
            x[layer] = torch.randn(shape[1:], generator=gen, device="cuda") * loud
        out.append(x)
    return out


def _tree(m, gen):
    """Visibility [m, m] of a draft tree: every node sees itself and its ancestors."""
    pick = torch.rand(m, generator=gen).tolist()
    seen = torch.zeros(m, m, dtype=torch.bool)
    for i in range(m):
        if i:
            seen[i] = seen[max(0, i - 1 - int(pick[i] * 8))]
        seen[i, i] = True
    return seen


def _mask_words(seen):
    m = seen.shape[-1]
    words = torch.zeros(*seen.shape[:-1], -(-m // 64), dtype=torch.int64)
    for j in range(m):
        words[..., j // 64] |= seen[..., j].long() << (j % 64)
    return words


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 1)
    host = torch.Generator().manual_seed(seed * 7919 + 2)
    ctx, d, bs, hkv, layers, m = _ctx(case), case["d"], case["bs"], case["hkv"], case["layers"], case["m"]
    batch, dt = len(ctx), _dtype(case)

    def randn(*shape, dtype=dt):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    s = dict(case=case, lens=ints(ctx), top=max(ctx))
    if case["kind"] == "attend":
        n_blocks = -(-max(ctx) // bs)
        s["pool"] = _q4_cache(case, n_blocks, gen)
        s["q"] = randn(layers, batch, m, case["hq"], d)
        s["k_new"], s["v_new"] = (randn(layers, batch, m, hkv, d) for _ in range(2))
        seen = torch.stack([_tree(m, host) for _ in ctx])
        s["seen"], s["mask"] = seen.cuda(), _mask_words(seen).cuda().contiguous()
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(layers, batch, m, case["hq"], device="cuda")
    elif case["kind"] == "commit":
        rows = case["rows"]
        n_blocks = -(-(max(ctx) + rows) // bs)
        s["top"] = n_blocks * bs
        s["pool"] = _q4_cache(case, n_blocks, gen)
        s["k_new"], s["v_new"] = (randn(layers, batch, m, hkv, d) for _ in range(2))
        s["taken"] = None if rows == m else torch.stack([torch.randperm(m, generator=host)[:rows].sort().values for _ in ctx]).int().cuda()
        s["n_taken"] = ints([max(1, rows - b) for b in range(batch)])
        s["kmax"], s["kmin"] = (torch.zeros(layers, batch, hkv, n_blocks, d, dtype=dt, device="cuda") for _ in range(2))
        s["k_values"], s["v_values"] = (torch.zeros(layers, batch, rows, hkv, d, dtype=dt, device="cuda") for _ in range(2))
        s["lens0"] = s["lens"].clone()
    elif case["kind"] == "refresh":
        n_blocks, budget = -(-max(ctx) // bs), case["budget"]
        s["pool"] = _q4_cache(case, n_blocks, gen)
        used = [-(-c // bs) for c in ctx]
        count = [min(u, budget) for u in used]
        idx = torch.zeros(layers, batch, hkv, budget, dtype=torch.int32, device="cuda")
        for b, (u, c) in enumerate(zip(used, count)):
            score = torch.rand(layers, hkv, u, generator=gen, device="cuda")
            score[..., -1] = 2.0  # the last block stays
            idx[:, b, :, :c] = score.topk(c, -1).indices.sort(-1).values.int()
        s["idx"], s["count"] = idx, ints(count)
        s["part_blocks"] = budget + -(-(20 + m) // bs)
        s["part_table"] = torch.arange(batch * s["part_blocks"], dtype=torch.int32, device="cuda").reshape(batch, -1)
        s["part_k"], s["part_v"] = (torch.zeros(layers, batch * s["part_blocks"], hkv, bs, d, dtype=dt, device="cuda") for _ in range(2))
        s["part_lens"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
    elif case["kind"] == "accumulate":
        n_blocks, rows = -(-max(ctx) // bs), case["rows"]
        s["k"], s["v"] = _cache(case, n_blocks, gen)
        s["q"] = randn(layers, batch, m, case["hq"], d)
        # the rows' log-sum-exps: about what unit queries over unit keys give
        s["lse"] = torch.log(s["lens"].float())[None, :, None, None] + 0.6 + 0.2 * randn(layers, batch, m, case["hq"], dtype=torch.float32)
        s["taken"] = torch.stack([torch.randperm(m, generator=host)[:rows].sort().values for _ in ctx]).int().cuda()
        s["n_taken"] = ints([max(1, rows - b) for b in range(batch)])
        s["acc"] = torch.rand(layers, batch, hkv, n_blocks * bs, generator=gen, device="cuda") * 1e-3
    else:
        n_blocks = -(-max(ctx) // bs)
        s["k"], s["v"] = _cache(case, n_blocks, gen)
        # accumulated weights: a few tokens have most of it
        s["acc0"] = torch.randn(layers, batch, hkv, n_blocks * bs, generator=gen, device="cuda").mul(2).exp()
        s["acc"], s["lens0"] = s["acc0"].clone(), s["lens"].clone()
        s["idx"] = torch.zeros(layers, batch, hkv, case["keep"], dtype=torch.int32, device="cuda")
    s["table"] = _page_table(case, n_blocks, gen)
    s["workspace"] = torch.zeros(_workspace_bytes(case, min(m, 128)) if case["kind"] == "attend" else HEAD, dtype=torch.uint8, device="cuda")
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _tokens(pool, table):
    """[layers][pages][heads][bs][..] through a table [batch][blocks] -> [layers][batch][heads][tokens][..]."""
    x = pool[:, table.long()].transpose(2, 3)
    return x.reshape(*x.shape[:3], -1, *x.shape[5:])


def _plain_attend(s):
    case = s["case"]
    layers, batch, m, hkv, d = case["layers"], len(_ctx(case)), case["m"], case["hkv"], case["d"]
    g = case["hq"] // hkv
    kc, vc, params = _codes(s["pool"], case["bs"], d)
    k = _tokens(_values(kc, params[..., 0, :], params[..., 1, :]), s["table"])
    del kc
    v = _tokens(_values(vc, params[..., 2, :], params[..., 3, :]), s["table"])
    del vc
    q = s["q"].float().reshape(layers, batch, m, hkv, g, d).permute(0, 1, 3, 2, 4, 5).reshape(layers, batch, hkv, m * g, d)
    kn, vn = (s[x].float().transpose(2, 3) for x in ("k_new", "v_new"))
    old = torch.arange(k.shape[3], device="cuda")[None] < s["lens"][:, None]
    a = (q @ k.transpose(-1, -2)).mul_(d ** -0.5).masked_fill_(~old[None, :, None, None], -math.inf)
    b = (q @ kn.transpose(-1, -2)).mul_(d ** -0.5).masked_fill_(~s["seen"].repeat_interleave(g, 1)[None, :, None], -math.inf)
    top = torch.maximum(a.amax(-1), b.amax(-1))[..., None]
    a, b = a.sub_(top).exp_(), b.sub_(top).exp_()
    total = a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True)
    v = v.masked_fill(~old[None, :, None, :, None], 0.0)
    out = (a @ v + b @ vn) / total
    lse = (top + total.log())[..., 0]
    s["out"].copy_(out.reshape(layers, batch, hkv, m, g, d).permute(0, 1, 3, 2, 4, 5).reshape(layers, batch, m, -1, d))
    s["lse"].copy_(lse.reshape(layers, batch, hkv, m, g).permute(0, 1, 3, 2, 4).reshape(layers, batch, m, -1))
    return s["out"], s["lse"]


def _taken_rows(x, taken, rows):
    """Rows of a step's tensor [layers][batch][m][heads][d], by number."""
    if taken is None:
        return x[:, :, :rows]
    return x.gather(2, taken.long()[None, :, :, None, None].expand(x.shape[0], -1, -1, x.shape[3], x.shape[4]))


def _plain_commit(s):
    case = s["case"]
    layers, batch, rows, hkv, d, bs = case["layers"], len(_ctx(case)), case["rows"], case["hkv"], case["d"], case["bs"]
    s["lens"].copy_(s["lens0"])
    lens = s["lens"].long()
    parts = []
    for x in (_taken_rows(s["k_new"], s["taken"], rows), _taken_rows(s["v_new"], s["taken"], rows)):
        parts.append(_quantise(x))  # codes [layers][batch][rows][heads][d], scale and offset without the d
    # the pages that the rows fall on, opened, filled and closed again
    n_touched = min(-(-rows // bs) + 1, s["table"].shape[1])
    first = lens // bs
    blocks = first[:, None] + torch.arange(n_touched, device="cuda")
    there = blocks < s["table"].shape[1]
    pages = s["table"].long().gather(1, blocks.clamp(max=s["table"].shape[1] - 1))
    kc, vc, params = _codes(s["pool"][:, pages], bs, d)  # [layers][batch][touched][heads][bs][d]
    token = blocks[..., None] * bs + torch.arange(bs, device="cuda")  # [batch][touched][bs]
    row = token - lens[:, None, None]
    new = (row >= 0) & (row < s["n_taken"].long()[:, None, None])
    which = row.clamp(0, rows - 1).reshape(batch, -1)
    pick = torch.arange(batch, device="cuda")[:, None]

    def placed(old, fresh):  # fresh [layers][batch][rows][heads][..] to the place of its tokens
        x = fresh[:, pick, which].reshape(layers, batch, n_touched, bs, hkv, *fresh.shape[4:]).transpose(3, 4)
        return torch.where(new[None, :, :, None].reshape(1, batch, n_touched, 1, bs, *([1] * (fresh.dim() - 4))), x, old)

    kc, vc = placed(kc, parts[0][0]), placed(vc, parts[1][0])
    params = torch.stack([placed(params[..., i, :], parts[i // 2][1 + i % 2]) for i in range(4)], -2)
    closed = _pages(kc, vc, params, d)
    s["pool"][:, pages[there]] = closed[:, there]
    # summaries of those blocks over the tokens that they now hold
    held = token < (lens + s["n_taken"])[:, None, None]
    k = _values(kc, params[..., 0, :], params[..., 1, :])
    touched = there & new.any(-1)
    b_at, t_at = touched.nonzero(as_tuple=True)
    at = (slice(None), b_at, slice(None), blocks[b_at, t_at])
    out_of = ~held[None, :, :, None, :, None]
    s["kmax"][at] = k.masked_fill(out_of, -math.inf).amax(-2)[:, b_at, t_at].transpose(0, 1).to(s["kmax"].dtype)
    s["kmin"][at] = k.masked_fill(out_of, math.inf).amin(-2)[:, b_at, t_at].transpose(0, 1).to(s["kmin"].dtype)
    there_row = torch.arange(rows, device="cuda")[None] < s["n_taken"][:, None]
    for name, (n, scale, offset) in zip(("k_values", "v_values"), parts):
        s[name].copy_(torch.where(there_row[None, :, :, None, None], _values(n, scale, offset), s[name].float()))
    s["lens"].add_(s["n_taken"])
    return s["k_values"], s["v_values"], s["kmax"], s["kmin"], s["lens"]


def _plain_refresh(s):
    case = s["case"]
    d, bs, budget, hkv = case["d"], case["bs"], case["budget"], case["hkv"]
    layers, batch = case["layers"], len(_ctx(case))
    block = s["idx"].long()
    page = s["table"].long()[torch.arange(batch, device="cuda")[None, :, None, None], block]
    layer = torch.arange(layers, device="cuda")[:, None, None, None]
    head = torch.arange(hkv, device="cuda")[None, None, :, None]
    kc, vc, params = _codes(s["pool"][layer, page, head], bs, d)  # [layers][batch][heads][budget][bs][d]
    to = s["part_table"].long()[None, :, None, :budget]
    some = torch.arange(budget, device="cuda")[None, None, None, :, None] < s["count"][None, :, None, None, None]
    valid = some & (block[..., None] * bs + torch.arange(bs, device="cuda") < s["lens"][None, :, None, None, None])
    for pool, codes, i in ((s["part_k"], kc, 0), (s["part_v"], vc, 2)):
        x = _values(codes, params[..., i, :], params[..., i + 1, :]).to(pool.dtype)
        pool[layer, to, head] = torch.where(valid[..., None], x, pool[layer, to, head])
    used = -(-s["lens"] // bs)
    s["part_lens"].copy_((s["count"] - 1) * bs + s["lens"] - (used - 1) * bs)
    return s["part_k"], s["part_v"], s["part_lens"]


def _plain_accumulate(s):
    case = s["case"]
    layers, batch, rows, hkv, d = case["layers"], len(_ctx(case)), case["rows"], case["hkv"], case["d"]
    g = case["hq"] // hkv
    k = _tokens(s["k"], s["table"]).float()
    q = _taken_rows(s["q"], s["taken"], rows).float().reshape(layers, batch, rows, hkv, g, d).permute(0, 1, 3, 2, 4, 5).reshape(layers, batch, hkv, -1, d)
    lse = s["lse"].gather(2, s["taken"].long()[None, :, :, None].expand(layers, -1, -1, case["hq"]))
    lse = lse.reshape(layers, batch, rows, hkv, g).permute(0, 1, 3, 2, 4).reshape(layers, batch, hkv, -1, 1)
    # accepted row i sees the tokens up to its own, which is the last but n - 1 - i
    row = torch.arange(rows, device="cuda").repeat_interleave(g)[None]
    end = torch.where(row < s["n_taken"][:, None], s["lens"][:, None] - s["n_taken"][:, None] + row + 1, 0)
    seen = torch.arange(k.shape[3], device="cuda") < end[..., None]
    w = (q @ k.transpose(-1, -2)).mul_(d ** -0.5).sub_(lse).exp_().masked_fill_(~seen[None, :, None], 0.0)
    s["acc"].add_(w.sum(-2))
    return s["acc"]


def _plain_evict(s):
    case = s["case"]
    keep, sink, local = case["keep"], case["sink"], case["local"]
    layers, batch, hkv = case["layers"], len(_ctx(case)), case["hkv"]
    s["lens"].copy_(s["lens0"])
    s["acc"].copy_(s["acc0"])
    lens = s["lens"].long()
    token = torch.arange(s["acc"].shape[-1], device="cuda")
    kept_always = (token < sink) | (token >= lens[:, None] - local)
    score = s["acc"].masked_fill(kept_always[None, :, None], math.inf).masked_fill((token >= lens[:, None])[None, :, None], -math.inf)
    # the `keep` best, ties to the lower token, in ascending order; tokens past the end sort behind all others
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    best = best.sort(-1).values
    n = lens.clamp(max=keep)
    there = torch.arange(keep, device="cuda") < n[:, None]  # [batch][keep]
    best = torch.where(there[None, :, None], best, 0)
    s["idx"].copy_(torch.where(there[None, :, None], best.int(), s["idx"]))
    layer = torch.arange(layers, device="cuda")[:, None, None, None]
    head = torch.arange(hkv, device="cuda")[None, None, :, None]
    seq = torch.arange(batch, device="cuda")[None, :, None, None]
    bs = case["bs"]
    table = s["table"].long()
    to = token[:keep].expand(layers, batch, hkv, keep)
    to = torch.where(there[None, :, None], to, 0)  # places that nothing is moved to take token 0, which stays, on themselves
    source = torch.where(there[None, :, None] & (best >= 0), best, 0)
    first = source[..., :1]
    source = torch.where(there[None, :, None], source, first)
    for x in (s["k"], s["v"]):
        rows = x[layer, table[seq, source // bs], head, source % bs]
        x[layer, table[seq, to // bs], head, to % bs] = rows
    a = torch.zeros_like(s["acc"])
    a[..., :keep] = torch.where(there[None, :, None], s["acc"].gather(-1, source), 0.0)
    past = (token >= lens[:, None])[None, :, None]  # behind the sequence: left as it was
    s["acc"].copy_(torch.where(past, s["acc"], a))
    s["lens"].copy_(n)
    return s["k"], s["v"], s["acc"], s["idx"], s["lens"]


# ---- the calls of the library --------------------------------------------------------------------------------------
def _handle(s):
    """Configuration and cache descriptors, which a program makes once."""
    from paper_2512_02337_b200 import binding as B

    c = s["case"]
    h = dict(B=B, cfg=B.make_config(c["layers"], c["hq"], c["hkv"], c["d"], c["bs"], c["dtype"], -(-32 // c["bs"]), -(-128 // c["bs"]),
                                    c.get("budget", 64), 20 + min(c["m"], 128)))
    if "pool" in s:
        h["q4"] = B.CacheQ4(s["pool"], s["table"], s["lens"], s["top"])
    if "part_k" in s:
        h["part"] = B.Cache(s["part_k"], s["part_v"], s["part_table"], s["part_lens"], s["part_blocks"] * c["bs"])
    if "k" in s:
        h["kv"] = B.Cache(s["k"], s["v"], s["table"], s["lens"], s["top"])
    return h


def _own_run(s):
    h = s["handle"] if "handle" in s else s.setdefault("handle", _handle(s))
    B, cfg, c, ws = h["B"], h["cfg"], s["case"], s["workspace"]
    if c["kind"] == "attend":
        B.specpv_verify_full_q4(cfg, 0, c["layers"], s["q"], s["k_new"], s["v_new"], s["mask"], None, c["m"], h["q4"], s["out"], s["lse"], ws)
        return s["out"], s["lse"]
    if c["kind"] == "commit":
        s["lens"].copy_(s["lens0"])
        B.specpv_commit_accepted_q4(cfg, 0, c["layers"], s["k_new"], s["v_new"], c["m"], s["taken"], s["n_taken"], c["rows"], h["q4"],
                                    s["kmax"], s["kmin"], s["k_values"], s["v_values"], ws)
        return s["k_values"], s["v_values"], s["kmax"], s["kmin"], s["lens"]
    if c["kind"] == "refresh":
        B.specpv_refresh_partial_q4(cfg, h["q4"], s["idx"], s["count"], h["part"], s["part_lens"], ws)
        return s["part_k"], s["part_v"], s["part_lens"]
    if c["kind"] == "accumulate":
        B.specpv_accumulate_attention(cfg, 0, c["layers"], s["q"], s["lse"], c["m"], s["taken"], s["n_taken"], c["rows"], h["kv"], s["acc"], ws)
        return s["acc"]
    s["lens"].copy_(s["lens0"])
    s["acc"].copy_(s["acc0"])
    B.specpv_evict_tokens(cfg, h["kv"], s["acc"], c["keep"], c["sink"], c["local"], s["idx"], ws)
    return s["k"], s["v"], s["acc"], s["idx"], s["lens"]


def run(state):
    if own:
        return _own_run(state)
    return {"attend": _plain_attend, "commit": _plain_commit, "refresh": _plain_refresh, "accumulate": _plain_accumulate,
            "evict": _plain_evict}[state["case"]["kind"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    ctx, layers, hq, hkv, d, m, bs = _ctx(case), case["layers"], case["hq"], case["hkv"], case["d"], case["m"], case["bs"]
    es = 4 if case["dtype"] == "fp32" else 2
    n, batch = sum(ctx), len(ctx)
    if case["kind"] == "attend":
        step = layers * batch * m * (2 * hq * d * es + 2 * hkv * d * es + 4 * hq)
        return {"bytes": layers * n * hkv * (d + 8) + step, "flops": 4.0 * layers * hq * d * m * (n + batch * (m + 1) / 2)}
    if case["kind"] == "commit":
        rows = sum(max(1, case["rows"] - b) for b in range(batch))
        touched = sum(-(-(c + max(1, case["rows"] - b)) // bs) - c // bs for b, c in enumerate(ctx))
        old = sum(c % bs for c in ctx)  # tokens that share a block with new ones: their keys enter its summary
        return {"bytes": layers * hkv * (rows * (2 * d * es + d + 8 + 2 * d * es) + old * (d // 2 + 4) + touched * 2 * d * es), "flops": 20.0 * layers * hkv * rows * d}
    if case["kind"] == "refresh":
        kept = sum(min(-(-c // bs), case["budget"]) for c in ctx)
        return {"bytes": layers * hkv * (kept * bs * (d + 8 + 2 * d * es) + 4 * kept), "flops": 4.0 * layers * hkv * kept * bs * d}
    if case["kind"] == "accumulate":
        rows = sum(max(1, case["rows"] - b) * c for b, c in enumerate(ctx))
        few = sum(max(1, case["rows"] - b) for b in range(batch))
        return {"bytes": layers * (n * hkv * (d * es + 8) + few * hq * (d * es + 4)), "flops": 2.0 * layers * hq * d * rows}
    kept = [min(c, case["keep"]) for c in ctx]
    moved = sum(k - case["sink"] for k, c in zip(kept, ctx) if k < c)
    return {"bytes": layers * hkv * (4 * n + 8 * sum(kept) + moved * 4 * d * es), "flops": 2.0 * layers * hkv * n}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def _exact_field(words, i):
    """Element i of every word: its four bits stand at 4 (i / 2) + 16 (i % 2) + 3, counted around the word."""
    at = (4 * (i // 2) + 16 * (i % 2) + 3) % 32
    w = words.long() & 0xFFFFFFFF
    return ((w | w << 32) >> at) & 15


def _exact_page_values(pages, bs, d, dtype=torch.float64):
    """Keys and values [.., bs, d] of pages, element by element of the layout."""
    raw = pages.contiguous()
    lead = raw.shape[:-1]
    n = bs * d // 2
    p = raw[..., 2 * n:].contiguous().view(torch.bfloat16).double().reshape(*lead, 4, bs)
    k = torch.empty(*lead, bs, d, dtype=dtype, device=raw.device)
    v = torch.empty_like(k)
    kw = raw[..., :n].contiguous().view(torch.int32).reshape(*lead, d // 32, bs, 4)
    vw = raw[..., n:2 * n].contiguous().view(torch.int32).reshape(*lead, bs // 16, d, 2)
    for i in range(8):
        kf = _exact_field(kw, i)
        for j in range(d // 32):
            for w in range(4):
                k[..., 32 * j + 8 * w + i] = ((kf[..., j, :, w] + 16) * p[..., 0, :] + p[..., 1, :]).bfloat16().to(dtype)
        vf = _exact_field(vw, i)
        for u in range(bs // 16):
            for w in range(2):
                t = 16 * u + 8 * w + i
                v[..., t, :] = ((vf[..., u, :, w] + 16) * p[..., 2, t, None] + p[..., 3, t, None]).bfloat16().to(dtype)
    return k, v


def _exact_attend(case, s):
    ctx, d, g, m = _ctx(case), case["d"], case["hq"] // case["hkv"], case["m"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for layer in range(case["layers"]):
        for b, n in enumerate(ctx):
            pages = s["pool"][layer][s["table"][b, : -(-n // case["bs"])].long()]
            k, v = _exact_page_values(pages, case["bs"], d)
            for h in range(case["hkv"]):
                kk = torch.cat([k[:, h].reshape(-1, d)[:n], s["k_new"][layer, b, :, h].double()])
                vv = torch.cat([v[:, h].reshape(-1, d)[:n], s["v_new"][layer, b, :, h].double()])
                q = s["q"][layer, b, :, h * g:(h + 1) * g].double()
                logits = torch.einsum("mgd,td->mgt", q, kk) / math.sqrt(d)
                logits[..., n:] = logits[..., n:].masked_fill(~s["seen"][b][:, None], -math.inf)
                lse[layer, b, :, h * g:(h + 1) * g] = torch.logsumexp(logits, -1)
                out[layer, b, :, h * g:(h + 1) * g] = torch.einsum("mgt,td->mgd", torch.softmax(logits, -1), vv)
    return out, lse


def _exact_quantised(x):
    """Values of one set of rows [.., d] after quantisation, in 64 bits but for the stored numbers, which have 16."""
    x = x.double()
    lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    # the range and the division by 15 are taken in 32 bits, as the format says
    scale = ((hi.float() - lo.float()) / 15).bfloat16().double()
    offset = (lo - 16 * scale).float().bfloat16().double()
    n = torch.round(((x - (offset + 16 * scale)).float() / scale.float()).double()).clamp(0, 15)
    return ((n + 16) * scale + offset).bfloat16().double()


def _exact_commit(case, s):
    ctx, bs = _ctx(case), case["bs"]
    kv = [s["k_values"].double(), s["v_values"].double()]
    kmax, kmin = s["kmax"].double(), s["kmin"].double()
    for b, n in enumerate(ctx):
        take = int(s["n_taken"][b])
        rows = torch.arange(take, device="cuda") if s["taken"] is None else s["taken"][b, :take].long()
        for name, to in zip(("k_new", "v_new"), kv):
            to[:, b, :take] = _exact_quantised(s[name][:, b, rows])
        for block in range(n // bs, (n + take - 1) // bs + 1):
            old, _ = _exact_page_values(s["pool"][:, int(s["table"][b, block])], bs, case["d"])  # [layers][heads][bs][d]
            t0 = block * bs
            had = max(0, min(bs, n - t0))
            fresh = kv[0][:, b, max(0, t0 - n):max(0, min(take, t0 + bs - n))].transpose(1, 2)
            k = torch.cat([old[:, :, :had], fresh], 2)
            kmax[:, b, :, block], kmin[:, b, :, block] = k.amax(2), k.amin(2)
    return kv[0], kv[1], kmax, kmin, None


def _exact_refresh(case, s):
    bs, d = case["bs"], case["d"]
    part = [s["part_k"].double(), s["part_v"].double()]
    for b, n in enumerate(_ctx(case)):
        for i in range(int(s["count"][b])):
            to = int(s["part_table"][b, i])
            for layer in range(case["layers"]):
                block = s["idx"][layer, b, :, i].long()
                pages = s["pool"][layer, s["table"][b, block].long(), torch.arange(case["hkv"], device="cuda")]
                there = (block[:, None] * bs + torch.arange(bs, device="cuda") < n)[..., None]
                for pool, x in zip(part, _exact_page_values(pages, bs, d)):
                    pool[layer, to] = torch.where(there, x, pool[layer, to])
    return part[0], part[1], None


def _exact_accumulate(case, s):
    ctx, d, g = _ctx(case), case["d"], case["hq"] // case["hkv"]
    acc = s["acc"].double()
    for b, n in enumerate(ctx):
        take = int(s["n_taken"][b])
        pages = s["table"][b, : -(-n // case["bs"])].long()
        for layer in range(case["layers"]):
            for h in range(case["hkv"]):
                k = s["k"][layer, pages, h].double().reshape(-1, d)[:n]
                for i in range(take):
                    r, end = int(s["taken"][b, i]), n - take + i + 1
                    heads = slice(h * g, (h + 1) * g)
                    w = torch.exp(k[:end] @ s["q"][layer, b, r, heads].double().T / math.sqrt(d) - s["lse"][layer, b, r, heads].double())
                    acc[layer, b, h, :end] += w.sum(-1)
    return acc


def _exact_evict(case, s):
    keep, sink, local, bs = case["keep"], case["sink"], case["local"], case["bs"]
    k, v, acc = s["k"].clone(), s["v"].clone(), s["acc"].double()
    for b, n in enumerate(_ctx(case)):
        if n <= keep:
            continue
        page = s["table"][b].long().repeat_interleave(bs)
        slot = torch.arange(page.numel(), device="cuda") % bs
        middle = acc[:, b, :, sink:n - local]
        order = torch.argsort(-middle, dim=-1, stable=True)[..., : keep - sink - local] + sink
        ends = [torch.arange(*r, device="cuda").expand(*order.shape[:2], -1) for r in ((0, sink), (n - local, n))]
        stay = torch.cat([ends[0], order, ends[1]], -1).sort(-1).values
        for layer in range(case["layers"]):
            for h in range(case["hkv"]):
                at = stay[layer, h]
                for x in (k, v):
                    x[layer, page[:keep], h, slot[:keep]] = x[layer, page[at], h, slot[at]]
                acc[layer, b, h, :keep] = acc[layer, b, h, at]
        acc[:, b, :, keep:n] = 0
    return k.double(), v.double(), acc, None, None


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "commit": _exact_commit, "refresh": _exact_refresh, "accumulate": _exact_accumulate,
            "evict": _exact_evict}[case["kind"]](case, s)
