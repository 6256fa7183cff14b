"""Performance cases of the 8-bit draft cache and of attention over many rows:
the calls that keep a paged cache in 8 bits beside the caches of the context's
own type, and the attention of tokens, drafts and prompts over either.

kinds
  append   per-head RMS norm of queries and keys and their rotation in one pass
           over the fused projection rows; keys and values quantised as they
           are written to the paged cache
  pack     a cache of the context's type written to the 8-bit one
  unpack   and read back
  attend   attention of one or more rows per sequence, each over the slots up
           to its own (`window` > 0: over the last `window` of them and the
           first `first`), of a cache in the context's type or in 8 bits

An 8-bit cache holds e4m3 codes and one power-of-two scale per block, KV head
and pool (keys, values).  A block's scale is 2^e with the least e for which its
largest finite magnitude is at most 448 * 2^e (e in -110 .. 119); a code is the
value over the scale, rounded once to the nearest.  A block that holds rows
keeps its scale unless the new rows need a larger one; then the codes that it
holds are rounded again, to the new scale.

A case is a dict of plain values.  prepare() makes what a serving program
holds before the call, run() is one call, exact() the same from the
definitions in 64 bits.

Values: keys, values and queries N(0, 1) as normalised heads have them, times
a factor of each KV head (the queries of attention N(0, 2), so that some slots
stand out), norm gains around 1.  Blocks are scattered over the pools in a
random order, as an allocator leaves them; slots that hold nothing are NaN.
Lengths and row counts of a batch are spread evenly over their ranges, each in
an order that the seed gives.
"""
import functools
import math
import types

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-5
F8 = torch.float8_e4m3fn
E_MIN, E_MAX = -110, 119

# query heads, KV heads, head dim, RoPE base: the repository's workloads, and
# generic smaller and other ones
HEADS = {
    "llama3_8b": (32, 8, 128, 500000.0),
    "llama3_70b": (64, 8, 128, 500000.0),
    "llama2_7b": (32, 32, 128, 10000.0),
    "medium": (16, 4, 128, 500000.0),
    "wide": (16, 4, 256, 10000.0),
    "small": (8, 2, 64, 500000.0),
    "small_odd": (6, 2, 64, 10000.0),
    "narrow": (7, 1, 32, 10000.0),
    "tiny": (4, 4, 64, 10000.0),
}


def _case(name, kind, heads, batch, ctx_lo, ctx_hi, **kw):
    c = dict(name=name, kind=kind, heads=heads, dtype="bf16", batch=batch, ctx_lo=ctx_lo,
             ctx_hi=ctx_hi, block=16, new_lo=0, new_hi=0)
    if kind in ("append", "attend"):
        c.update(new_lo=1, new_hi=1)
    if kind == "attend":
        c.update(bits=8, window=0, first=0, lse=False)
    if kind in ("pack", "unpack"):
        c.update(start=0.0)
    c.update(kw)
    return c


def listed():
    return [
        # a decoding step of a serving batch: one new token per sequence
        _case("append_8b_bs16", "append", "llama3_8b", 16, 512, 4096),
        # prompts of a ragged batch entering the cache
        _case("append_8b_prompts", "append", "llama3_8b", 8, 0, 0, new_lo=129, new_hi=1531),
        # one user's drafted context, put away in 8 bits
        _case("pack_7b_bs1", "pack", "llama2_7b", 1, 4096, 4096),
        # a ragged batch put away, of which the first half was before
        _case("pack_8b_bs16", "pack", "llama3_8b", 16, 8191, 32767, start=0.5),
        # one user's context, brought back to be drafted on
        _case("unpack_8b_bs1", "unpack", "llama3_8b", 1, 2048, 2048),
        # a batch of long contexts brought back
        _case("unpack_8b_bs16", "unpack", "llama3_8b", 16, 8191, 32767),
        # the smallest call, fp32: launches and latency
        _case("attend_tiny_f32", "attend", "tiny", 1, 127, 127, dtype="f32", bits=32, window=64,
              first=4, lse=True),
        # a batch of long contexts decoding over the last slots and the first ones
        _case("window_8b_bs16", "attend", "llama3_8b", 16, 4099, 32771, bits=16, window=4096, first=4),
        # the largest model's heads, a large batch of long contexts in 8 bits
        _case("attend8_70b_bs32", "attend", "llama3_70b", 32, 32767, 32767),
        # five drafts and the token before them, scored for each of a ragged batch
        _case("verify8_8b_bs16", "attend", "llama3_8b", 16, 512, 16384, new_lo=6, new_hi=6),
        # one long prompt with multi-head attention
        _case("prompt_7b_bs1", "attend", "llama2_7b", 1, 0, 0, bits=16, new_lo=8192, new_hi=8192),
        # a chunk of a long prompt under a window, over an 8-bit cache
        _case("chunk8_70b_window", "attend", "llama3_70b", 1, 12288, 12288, new_lo=2048, new_hi=2048,
              window=4096, first=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "pack", "unpack", "attend", "attend", "attend", "attend"])
    heads = rng.choice(list(HEADS))
    nq, nkv, d, _ = HEADS[heads]
    dtype = "f32" if heads == "tiny" or rng.random() < 0.15 else "bf16"
    batch = _log(rng, 1, 48)
    # at most 10^9 keys in all, 131072 slots of a sequence
    most = min(131072, int(1e9 / (nkv * d * batch)))
    c = _case("", kind, heads, batch, 0, 0, dtype=dtype, block=rng.choice([16, 16, 16, 32, 64, 12]))
    del c["name"]
    if kind in ("append", "attend"):
        n = rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 8, max(9, min(4096, 8192 // batch)))])
        c.update(new_lo=max(1, min(n, rng.choice([1, n // 2, n]))), new_hi=n)
    if kind == "attend":
        # at most 2^31 pairs of a query head's row and a slot, 2^30 in 32 bits
        pairs = 2 ** 31 if dtype == "bf16" else 2 ** 30
        most = max(16, min(most, pairs // (nq * batch * c["new_hi"])))
        c.update(bits=rng.choice([8, 8, 16 if dtype == "bf16" else 32]), lse=rng.random() < 0.3)
        if rng.random() < 0.5:
            c.update(window=_log(rng, 16, 8192), first=rng.choice([0, 1, 4, 33]))
    hi = _log(rng, 16, min(most, 4096 if kind == "append" else most))
    c.update(ctx_hi=hi, ctx_lo=rng.choice([hi, hi // 2, hi // 8, 1, 0]))
    if kind in ("pack", "unpack"):
        c.update(start=rng.choice([0.0, 0.0, 0.5, 0.97]))
    return c


# ------------------------------------------------------------------- inputs
def _dims(case):
    nq, nkv, d, theta = HEADS[case["heads"]]
    return types.SimpleNamespace(nq=nq, nkv=nkv, d=d, theta=theta, g=nq // nkv)


def _spread(lo, hi, n):
    """n whole numbers spread evenly over lo .. hi (hi alone for one)."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lens(case):
    return _spread(case["ctx_lo"], case["ctx_hi"], case["batch"])


def _news(case):
    return _spread(case["new_lo"], case["new_hi"], case["batch"])


def _blocks_per_seq(case):
    """Block-table columns: the longest sequence and its new rows."""
    return max(1, -(-(case["ctx_hi"] + case["new_hi"]) // case["block"]))


def _exponent(amax):
    """Exponents of the scales that magnitudes up to amax take."""
    m, e = torch.frexp(amax)
    need = e.to(torch.int64) - 9 + (m > 0.875)
    return torch.where(amax > 0, need, torch.full_like(need, E_MIN)).clamp(E_MIN, E_MAX)


def _codes(x, e):
    """Codes of fp32 values whose scales are 2^e: one rounding, by the cast."""
    y = torch.ldexp(x, -e)
    return torch.where(torch.isfinite(y), y.clamp(-448.0, 448.0), torch.full_like(y, float("nan"))).to(F8)


def _quantised(x, held):
    """Codes and scales of blocks x [n, nkv, bs, d] of which held [n, bs] are there."""
    there = held[:, None, :, None]
    amax = x.abs().masked_fill_(~there, 0.0).amax((2, 3)).float()
    e = _exponent(amax)
    codes = _codes(x.float(), e[:, :, None, None]).view(torch.uint8).masked_fill_(~there, 0x7f).view(F8)
    scale = torch.ldexp(torch.ones_like(amax), e).masked_fill_(~held.any(1)[:, None], float("nan"))
    return codes, scale


def _inputs(case, seed):
    """Everything a case's call reads, from the seed alone."""
    m, B, bs = _dims(case), case["batch"], case["block"]
    kind = case["kind"]
    rng = np.random.default_rng([int(seed), 29])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(shape, std=1.0, dtype=dt):
        t = torch.randn(shape, generator=gen, device=DEV, dtype=dtype)
        return t.mul_(std) if std != 1.0 else t

    def int32(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    x = types.SimpleNamespace(case=case)
    nb = _blocks_per_seq(case)
    n = B * nb
    lens, counts = rng.permutation(_lens(case)), rng.permutation(_news(case))
    x.lens, x.table = int32(lens), int32(rng.permutation(n).reshape(B, nb))
    x.counts = torch.tensor(counts, device=DEV)
    x.offsets = int32(np.concatenate([[0], np.cumsum(counts)]))
    T = int(counts.sum())
    x.row_seq = torch.tensor(np.repeat(np.arange(B), counts), device=DEV)
    x.start = int32((lens * case["start"]).astype(np.int64)) if case.get("start") else None

    def held(upto):
        """[n, bs]: slots below upto [B] of the blocks of x.table."""
        t = torch.arange(nb * bs, device=DEV)
        h = torch.zeros((n, bs), dtype=torch.bool, device=DEV)
        h[x.table.long().view(-1)] = (t[None, :] < upto[:, None]).view(-1, bs)
        return h

    eight = kind != "attend" or case["bits"] == 8
    before = {"append": x.lens, "pack": x.start if x.start is not None else torch.zeros_like(x.lens),
              "unpack": x.lens, "attend": x.lens + x.counts}[kind]
    h = held(before)
    std = torch.exp2(normal((2, m.nkv), 0.7, torch.float32)).to(dt)
    pools = [normal((n, m.nkv, bs, m.d)).mul_(std[i][None, :, None, None]) for i in range(2)]
    if eight:
        packed = [_quantised(p, h) for p in pools]
        x.k8, x.v8 = packed[0][0], packed[1][0]
        x.scales = torch.stack([packed[0][1], packed[1][1]], 2).contiguous()
    if kind in ("pack", "attend"):
        gone = ~(h if kind == "attend" else held(x.lens))
        for p in pools:
            p.masked_fill_(gone[:, None, :, None], float("nan"))
    if kind == "unpack":
        for p in pools:
            p.fill_(float("nan"))
    if kind in ("pack", "unpack") or not eight:
        x.k_pool, x.v_pool = pools
    del pools
    if kind in ("pack", "unpack"):          # the two caches have blocks of their own
        order = torch.tensor(rng.permutation(n), device=DEV)
        x.table_kv = order[x.table.long()].to(torch.int32)
        if kind == "pack":
            x.k_pool, x.v_pool = (torch.empty_like(p).index_copy_(0, order, p) for p in (x.k_pool, x.v_pool))
    if kind == "append":
        x.qkv = normal((T, m.nq + 2 * m.nkv, m.d))
        x.qkv[:, m.nq + m.nkv:] *= std[1][:, None]
        x.qkv = x.qkv.view(T, -1)
        x.q_gain = (1.0 + 0.1 * normal((m.d,), dtype=torch.float32)).to(dt)
        x.k_gain = (1.0 + 0.1 * normal((m.d,), dtype=torch.float32)).to(dt)
        # positions run ahead of the slots where a cache was evicted before
        x.positions = x.lens + int32(rng.integers(0, 1 << 16, B))
    if kind == "attend":
        x.q = normal((T, m.nq, m.d), 2.0)
    return x


@functools.lru_cache(maxsize=None)
def _drafter(heads, dtype, block, batch, blocks_per_seq):
    """The program's drafting context: one per model and capacity."""
    from paper_2602_01762_amd import Drafter
    nq, nkv, d, theta = HEADS[heads]
    return Drafter(types.SimpleNamespace(
        hidden=512, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=512, vocab=4096, M=1, n_steps=1,
        feat_width=512, rope_theta=theta, rms_eps=EPS, dtype=dtype, kv_block_size=block, batch=batch,
        blocks_per_seq=blocks_per_seq, tree_width=0, tree_nodes=0, max_new_rows=0))


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:
        x.dr = _drafter(case["heads"], case["dtype"], case["block"], case["batch"], _blocks_per_seq(case))
        if hasattr(x, "k8"):
            x.kv8 = x.dr.cache8(x.lens, x.k8, x.v8, x.scales, x.table)
        if hasattr(x, "k_pool"):
            x.kv = x.dr.cache(x.lens, x.k_pool, x.v_pool, getattr(x, "table_kv", x.table))
    return x


# ------------------------------------------------------ the framework's calls
def _own(x):
    case, dr = x.case, x.dr
    kind = case["kind"]
    single = case["new_lo"] == case["new_hi"] == 1
    if kind == "append":
        q = dr.cache8_append(x.kv8, x.qkv, q_gain=x.q_gain, k_gain=x.k_gain,
                             offsets=None if single else x.offsets, positions=x.positions)
        return {"q": q, "k8": x.k8, "v8": x.v8, "scales": x.scales}
    if kind == "pack":
        dr.cache8_pack(x.kv8, x.kv, start=x.start, max_len=case["ctx_hi"])
        return {"k8": x.k8, "v8": x.v8, "scales": x.scales}
    if kind == "unpack":
        dr.cache8_unpack(x.kv8, x.kv, start=x.start, max_len=case["ctx_hi"])
        return {"k": x.k_pool, "v": x.v_pool}
    r = dr.cache_attend_rows(x.kv8 if case["bits"] == 8 else x.kv, x.q, offsets=None if single else x.offsets,
                             n_new=1, window=case["window"], n_first=case["first"],
                             max_len=case["ctx_hi"] + case["new_hi"], lse=case["lse"])
    return r if case["lse"] else {"out": r["out"]}


# ------------------------------------------------------------ the plain forms
def _encode64(x, e):
    """Codes of fp64 values whose scales are 2^e, rounded once to the nearest
    (the cast from fp64 would round to fp32 first)."""
    y = torch.ldexp(x, -e).clamp(-448.0, 448.0)
    step = torch.frexp(y).exponent.clamp(min=-5) - 4          # of 3 fraction bits, or of 2^-9
    return torch.ldexp(torch.round(torch.ldexp(y, -step)), step).float().to(F8)


def _grow(codes, scale, e):
    """Codes of blocks [n, nkv, bs, d] with scale [n, nkv], rounded to the scales 2^e."""
    return (codes.float() * torch.ldexp(scale, -e)[:, :, None, None]).to(F8)


def _write(x, which, rows, blk, off, amax, encode):
    """Rows [N, nkv, d] (amax [N, nkv]) to the slots off [N] of the blocks blk
    [N] of pool `which`, of which the block of each sequence's first new slot
    may hold rows."""
    bs = x.case["block"]
    pool, scales = (x.k8, x.v8)[which], x.scales[..., which]
    n = pool.shape[0]
    begin = x.lens.long() if x.case["kind"] == "append" else (
        torch.zeros_like(x.lens).long() if x.start is None else x.start.long())
    top = torch.zeros((n, rows.shape[1]), dtype=amax.dtype, device=DEV)
    top.scatter_reduce_(0, blk[:, None].expand_as(amax), amax, "amax")
    e = _exponent(top)
    new = torch.zeros(n, dtype=torch.bool, device=DEV)
    new[blk] = True
    # blocks that hold rows already: their scales do not shrink, their codes follow
    at = begin % bs
    first = x.table.long().gather(1, (begin // bs).clamp(max=x.table.shape[1] - 1)[:, None]).view(-1)
    part = first[(at > 0) & new[first]]
    have = at[(at > 0) & new[first]]
    old_e = torch.frexp(scales[part]).exponent.long() - 1
    e[part] = torch.maximum(e[part], old_e)
    grown = _grow(pool.view(torch.uint8)[part].view(F8), scales[part], e[part]).view(torch.uint8)
    stay = (torch.arange(bs, device=DEV) < have[:, None])[:, None, :, None]
    raw = pool.view(torch.uint8)
    raw[part] = torch.where(stay, grown, raw[part])
    scales[new] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)[new]
    raw[blk, :, off] = encode(rows, e[blk][:, :, None]).view(torch.uint8)


def _append_plain(x):
    case, m = x.case, _dims(x.case)
    T = x.qkv.shape[0]
    at = torch.arange(T, device=DEV) - x.offsets.long()[x.row_seq]
    pos = x.positions.long()[x.row_seq] + at
    i = torch.arange(m.d // 2, device=DEV, dtype=torch.float64)
    ang = pos.double()[:, None] * torch.pow(torch.tensor(m.theta, dtype=torch.float64, device=DEV),
                                            -2.0 * i / m.d)
    c, s = torch.cos(ang)[:, None, :], torch.sin(ang)[:, None, :]

    def normed_rotated(h, gain, c, s):
        h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * gain.to(h.dtype)
        a, b = h[..., : m.d // 2], h[..., m.d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    h = x.qkv.view(T, m.nq + 2 * m.nkv, m.d)
    q = normed_rotated(h[:, : m.nq].float(), x.q_gain, c.float(), s.float()).to(x.qkv.dtype)
    # keys in 64 bits: a value next to the border between two codes
    k = normed_rotated(h[:, m.nq: m.nq + m.nkv].double(), x.k_gain, c, s)
    v = h[:, m.nq + m.nkv:].float()
    slot = x.lens.long()[x.row_seq] + at
    blk = x.table.long()[x.row_seq, slot // case["block"]]
    _write(x, 0, k, blk, slot % case["block"], k.abs().amax(-1), _encode64)
    _write(x, 1, v, blk, slot % case["block"], v.abs().amax(-1), _codes)
    return {"q": q, "k8": x.k8, "v8": x.v8, "scales": x.scales}


def _moved(x):
    """Blocks in the 8-bit pools and in the others, and slots in them, of the
    slots that a pack or unpack moves."""
    bs = x.case["block"]
    t = torch.arange(x.table.shape[1] * bs, device=DEV)
    go = t < x.lens[:, None]
    if x.start is not None:
        go &= t >= x.start[:, None]
    b, t = go.nonzero(as_tuple=True)
    return x.table.long()[b, t // bs], x.table_kv.long()[b, t // bs], t % bs


def _pack_plain(x):
    blk, src, off = _moved(x)
    for which, pool in enumerate((x.k_pool, x.v_pool)):
        rows = pool[src, :, off].float()
        _write(x, which, rows, blk, off, rows.abs().amax(-1), _codes)
    return {"k8": x.k8, "v8": x.v8, "scales": x.scales}


def _unpack_plain(x):
    blk, dst, off = _moved(x)
    for which, (codes, pool) in enumerate(((x.k8, x.k_pool), (x.v8, x.v_pool))):
        rows = codes.view(torch.uint8)[blk, :, off].view(F8).float() * x.scales[blk, :, which][:, :, None]
        pool[dst, :, off] = rows.to(pool.dtype)
    return {"k": x.k_pool, "v": x.v_pool}


def _attend_plain(x):
    case, m = x.case, _dims(x.case)
    B, bs, R = case["batch"], case["block"], case["new_hi"]
    nb = x.table.shape[1]
    blk = x.table.long()

    def rows(which):
        """Keys or values [B, nkv, nb * bs, d] in 32 bits."""
        if case["bits"] == 8:
            t = (x.k8, x.v8)[which].view(torch.uint8)[blk].view(F8).float()
            t *= x.scales[..., which][blk][..., None, None]
        else:
            t = (x.k_pool, x.v_pool)[which][blk].float()
        return t.transpose(1, 2).reshape(B, m.nkv, nb * bs, m.d)

    # rows of every sequence, padded to R
    i = torch.arange(R, device=DEV)
    there = i < x.counts[:, None]                                          # [B, R]
    at = (x.offsets.long()[:-1, None] + i).clamp(max=x.q.shape[0] - 1)
    q = x.q[at].float().view(B, R, m.nkv, m.g, m.d).permute(0, 2, 1, 3, 4).reshape(B, m.nkv, R * m.g, m.d)
    s = torch.matmul(q, rows(0).transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(m.d)).view(B, m.nkv, R, m.g, -1)
    t = torch.arange(nb * bs, device=DEV)
    v = (x.lens.long()[:, None] + 1 + i)[..., None]                        # slots up to each row's own
    seen = t < v
    if case["window"]:
        seen &= (t >= v - case["window"]) | (t < case["first"])
    s.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = s.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    held = t < (x.lens + x.counts)[:, None]
    values = rows(1).masked_fill_(~held[:, None, :, None], 0.0)
    o = torch.matmul(e.view(B, m.nkv, R * m.g, -1), values).view(B, m.nkv, R, m.g, m.d) / total

    def packed(y):
        """[B, nkv, R, g, ...] -> [T, nq, ...]"""
        return y.transpose(1, 2)[there].reshape(x.q.shape[0], m.nq, -1)

    r = {"out": packed(o).to(x.q.dtype)}
    if case["lse"]:
        r["lse"] = packed(top + torch.log(total)).squeeze(-1)
    return r


PLAIN = {"append": _append_plain, "pack": _pack_plain, "unpack": _unpack_plain, "attend": _attend_plain}


def run(x):
    return _own(x) if own else PLAIN[x.case["kind"]](x)


# ------------------------------------------------------------------ work, exact
def work(case):
    m = _dims(case)
    e = 2 if case["dtype"] == "bf16" else 4
    lens, news = _lens(case), _news(case)
    if case["kind"] == "append":
        T = sum(news)
        return {"bytes": float(T * m.d * ((2 * m.nq + 2 * m.nkv) * e + 2 * m.nkv)),
                "flops": 8.0 * T * (m.nq + 2 * m.nkv) * m.d}
    if case["kind"] in ("pack", "unpack"):
        n = sum(L - int(L * case["start"]) for L in lens) * 2.0 * m.nkv * m.d
        return {"bytes": n * (e + 1), "flops": n}
    held = seen = 0
    for L, n in zip(lens, news):
        v = L + 1 + np.arange(n)
        W, F = case["window"] or 1 << 30, case["first"]
        low = np.maximum(0, v - W)
        seen += int((v - low + np.minimum(low, F)).sum())
        if n:
            held += int(v[-1] - low[0] + min(low[0], F))
    return {"bytes": 2.0 * held * m.nkv * m.d * case["bits"] / 8 + 2.0 * sum(news) * m.nq * m.d * e,
            "flops": 4.0 * seen * m.nq * m.d}


def _nearest_code(y):
    """y [.., d] in 64 bits to the nearest of the values that e4m3 holds, ties to
    the even code: by search in the table of them."""
    grid = [(8 + f) / 8 * 2.0 ** (k - 7) if k else f / 8 * 2.0 ** -6 for k in range(16) for f in range(8)][:127]
    grid = torch.tensor(grid, dtype=torch.float64, device=DEV)
    a = y.abs().clamp(max=448.0)
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    take = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(grid[take], y)


def _exact_write(pool, scale, rows, table, slots, bs, fresh_from):
    """Rows [n, nkv, d] to these slots of one sequence, block by block."""
    for i in range(int(slots[0]) // bs, int(slots[-1]) // bs + 1):
        pick = (slots // bs) == i
        y, off = rows[pick], slots[pick] % bs
        b = int(table[i])
        top = y.abs().amax((0, 2))
        least = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
        # the logarithm may be off by a rounding next to a whole number
        least = torch.where(top <= 448.0 * torch.exp2(least - 1), least - 1, least)
        least = torch.where(top > 448.0 * torch.exp2(least), least + 1, least).clamp(E_MIN, E_MAX)
        e = torch.exp2(least)
        keep = fresh_from - i * bs
        if keep > 0:
            old = scale[b].clone()
            e = torch.maximum(e, old)
            pool[b, :, :keep] = _nearest_code(pool[b, :, :keep] * (old / e)[:, None, None])
        pool[b][:, off] = _nearest_code(y / e[None, :, None]).transpose(0, 1)
        scale[b] = e


def _exact_attend(x):
    case, m, bs = x.case, _dims(x.case), x.case["block"]
    out = torch.zeros(x.q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(x.q.shape[:2], dtype=torch.float64, device=DEV)
    lens, off = x.lens.tolist(), x.offsets.tolist()
    for b in range(case["batch"]):
        r0, r1 = off[b], off[b + 1]
        n = r1 - r0
        if n == 0:
            continue
        slots = torch.arange(lens[b] + n, device=DEV)
        blk = x.table[b].long()[slots // bs]
        own_slot = lens[b] + torch.arange(n, device=DEV)
        ago = own_slot[:, None] - slots[None, :]
        hidden = ago < 0
        if case["window"]:
            hidden |= (ago >= case["window"]) & (slots[None, :] >= case["first"])
        for j in range(m.nkv):
            K, V = ((p.view(torch.uint8)[blk, j, slots % bs].view(F8).double() * x.scales[blk, j, w].double()[:, None]
                     if case["bits"] == 8 else p[blk, j, slots % bs].double())
                    for w, p in enumerate((x.k8, x.v8) if case["bits"] == 8 else (x.k_pool, x.v_pool)))
            for h in range(j * m.g, (j + 1) * m.g):
                s = torch.mm(x.q[r0:r1, h].double(), K.t().contiguous()) / math.sqrt(m.d)
                s.masked_fill_(hidden, float("-inf"))
                lse[r0:r1, h] = torch.logsumexp(s, 1)
                out[r0:r1, h] = torch.mm(torch.softmax(s, 1), V)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    x = _inputs(case, seed)
    m, B, bs, kind = _dims(case), case["batch"], case["block"], case["kind"]
    if kind == "attend":
        return _exact_attend(x)
    lens = x.lens.tolist()
    start = [0] * B if x.start is None else x.start.tolist()
    if kind == "unpack":
        r = [p.double() for p in (x.k_pool, x.v_pool)]
        for b in range(B):
            t = torch.arange(start[b], lens[b], device=DEV)
            src, dst = x.table[b].long()[t // bs], x.table_kv[b].long()[t // bs]
            for w, codes in enumerate((x.k8, x.v8)):
                r[w][dst, :, t % bs] = codes.view(torch.uint8)[src, :, t % bs].view(F8).double() * \
                    x.scales[src, :, w].double()[:, :, None]
        return {"k": r[0], "v": r[1]}
    touched = sum(_news(case)) if kind == "append" else sum(a - b for a, b in zip(lens, start))
    if touched // bs + B > 12000:
        return None                      # a few steps for each block: over 20 seconds
    pools, scale = [x.k8.double(), x.v8.double()], [x.scales[..., w].double() for w in range(2)]
    if kind == "pack":
        for b in range(B):
            t = torch.arange(start[b], lens[b], device=DEV)
            if t.numel():
                src = x.table_kv[b].long()[t // bs]
                for w, p in enumerate((x.k_pool, x.v_pool)):
                    _exact_write(pools[w], scale[w], p[src, :, t % bs].double(), x.table[b], t, bs, start[b])
        return {"k8": pools[0], "v8": pools[1], "scales": torch.stack(scale, 2)}
    h = x.qkv.double().view(-1, m.nq + 2 * m.nkv, m.d)
    q = torch.zeros((h.shape[0], m.nq, m.d), dtype=torch.float64, device=DEV)
    off, pos = x.offsets.tolist(), x.positions.tolist()
    half = torch.arange(m.d // 2, device=DEV, dtype=torch.float64)
    freq = torch.exp(half * (-2.0 * math.log(m.theta) / m.d))
    for b in range(B):
        n = off[b + 1] - off[b]
        if n == 0:
            continue
        y = h[off[b]: off[b + 1]]
        i = torch.arange(n, device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(n, m.d // 2),
                           (pos[b] + i).double()[:, None] * freq)[:, None]

        def head(z, gain):
            z = z / torch.sqrt(z.square().sum(-1, keepdim=True) / m.d + EPS) * gain.double()
            z = torch.complex(z[..., : m.d // 2], z[..., m.d // 2:]) * turn
            return torch.cat([z.real, z.imag], -1)

        q[off[b]: off[b + 1]] = head(y[:, : m.nq], x.q_gain)
        k = head(y[:, m.nq: m.nq + m.nkv], x.k_gain)
        for w, rows in enumerate((k, y[:, m.nq + m.nkv:])):
            _exact_write(pools[w], scale[w], rows, x.table[b], lens[b] + i, bs, lens[b])
    return {"q": q, "k8": pools[0], "v8": pools[1], "scales": torch.stack(scale, 2)}
