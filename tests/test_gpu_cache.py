"""Long-context draft cache on the GPU against the fp64 oracle.

Tolerances.  u = 2^-24.  A dot product of d stored values in fp32 is off by at
most (d + 4) u sum|q_c k_c|, so a score by delta = (d + 4) u max_t sum_c |q_c
k_tc| / sqrt(d), and a probability by the factor 1 + 2 delta.  The weighted sum
of n values adds at most (n + 64) u times sum_t p_t |v_t| in fp32 (n: the
largest number of terms that one accumulator or one join takes in a row, at
most 1024 here), and in bf16 caches the products may take p as a hi/lo pair of
bf16, 2^-16.  An output in bf16 is rounded once: half a step, 2^-8 of the value.
"""
import types

import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import widen
from synth import to_host

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"
U = 2.0 ** -24
EPS = 1e-5


def f64(t):
    return widen(to_host(t)).astype(np.float64) if t.dtype != torch.float32 else t.detach().cpu().numpy().astype(np.float64)


def drafter(nq, nkv, d, dtype, bs, batch, columns, theta=1e4):
    from paper_2602_01762_amd import Drafter
    return Drafter(types.SimpleNamespace(
        hidden=512, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=512, vocab=512, M=1, n_steps=1,
        feat_width=512, rope_theta=theta, rms_eps=EPS, dtype=dtype, kv_block_size=bs, batch=batch,
        blocks_per_seq=columns, tree_width=0, tree_nodes=0, max_new_rows=0))


class Cache:
    """A context and a batch of sequences whose blocks are scattered over a
    pool; every slot that holds nothing is NaN."""

    def __init__(self, nq, nkv, d, dtype, bs, lens, columns, spare=3, seed=0):
        self.nq, self.nkv, self.d, self.bs, self.g = nq, nkv, d, bs, nq // nkv
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.B, self.columns = len(lens), columns
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)
        self.dr = drafter(nq, nkv, d, dtype, bs, self.B, columns)
        n = self.B * columns + spare
        self.n_lens = list(lens)
        perm = self.rng.permutation(n)
        self.table_h = perm[: self.B * columns].reshape(self.B, columns)
        self.free = perm[self.B * columns:]
        self.k, self.v = self.normal((n, nkv, bs, d)), self.normal((n, nkv, bs, d))
        self.table = torch.tensor(self.table_h, dtype=torch.int32, device=DEV)
        self.lens = torch.tensor(self.n_lens, dtype=torch.int32, device=DEV)
        dead = torch.ones((n, bs), dtype=torch.bool)
        for b, L in enumerate(lens):
            for i in range(columns):
                dead[int(self.table_h[b, i]), : max(0, min(bs, L - i * bs))] = False
        dead = dead.to(DEV)[:, None, :, None]
        self.k.masked_fill_(dead, float("nan"))
        self.v.masked_fill_(dead, float("nan"))

    def normal(self, shape, std=1.0):
        return (std * torch.randn(shape, generator=self.gen, device=DEV)).to(self.dt)

    def weights(self, zero=0.0):
        w = torch.exp(torch.randn(self.k.shape[:3], generator=self.gen, device=DEV))
        return w.masked_fill_(torch.rand(w.shape, generator=self.gen, device=DEV) < zero, 0.0)

    def kv(self):
        return self.dr.cache(self.lens, self.k, self.v, self.table)

    def rows(self, pool_h, b, j, slots, table=None):
        t = self.table_h if table is None else table
        slots = np.asarray(slots, dtype=np.int64)
        return pool_h[t[b, slots // self.bs], j, slots % self.bs]

    def close(self, status=0):
        assert self.dr.device_status() == status
        self.dr.close()


HEADS = [(4, 4, 64, "f32"), (8, 2, 64, "bf16"), (32, 8, 128, "bf16"), (7, 1, 32, "bf16"),
         (4, 1, 256, "bf16"), (3, 3, 128, "bf16"), (8, 1, 128, "bf16"), (8, 1, 128, "f32"),
         (2, 1, 256, "f32"), (6, 2, 32, "f32")]


# ------------------------------------------------------------------- append
def check_append(c, counts, with_gain=True, positions=None, weights=False, pad=0):
    T = int(sum(counts)) + pad
    nh = c.nq + 2 * c.nkv
    qkv = c.normal((T, nh * c.d), 1.5)
    qkv[T - pad:] = float("nan")
    g = [(1 + 0.1 * c.normal((c.d,)).float()).to(c.dt) if with_gain else None for _ in range(2)]
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    w = c.weights() if weights else None
    w0 = w.clone() if weights else None
    out = torch.full((T, c.nq, c.d), 7.0, dtype=c.dt, device=DEV)
    k0, v0 = c.k.clone(), c.v.clone()
    r = c.dr.cache_append(c.kv(), qkv, g[0], g[1], offsets=off, positions=pos, weights=w, out=out)
    torch.cuda.synchronize()
    assert r is out
    x = f64(qkv).reshape(T, nh, c.d)
    gains = [None if t is None else f64(t) for t in g]
    got_q, kh, vh = f64(out), f64(c.k), f64(c.v)
    step = 2.0 ** -8 if c.dt == torch.bfloat16 else 0.0
    touched = torch.zeros(c.k.shape[:1] + (c.bs,), dtype=torch.bool)
    r0 = 0
    for b, n in enumerate(counts):
        for i in range(n):
            p = (c.n_lens[b] if positions is None else positions[b]) + i
            wq, wk, wv = C.append_row(x[r0 + i], c.nq, c.nkv, p, 1e4, EPS, *gains)
            slot = c.n_lens[b] + i
            blk = int(c.table_h[b, slot // c.bs])
            touched[blk, slot % c.bs] = True
            # normed head before its rotation: |x1 c| + |x2 s| <= |x1| + |x2|
            lim = {}
            for name, want, h0, gain in (("q", wq, 0, gains[0]), ("k", wk, c.nq, gains[1])):
                y = x[r0 + i, h0: h0 + len(want)]
                if gain is not None:
                    y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + EPS) * gain
                a = np.abs(y[:, : c.d // 2]) + np.abs(y[:, c.d // 2:])
                lim[name] = step * np.abs(want) + (c.d / 2 + 10) * U * (np.concatenate([a, a], -1) + np.abs(want))
            assert np.all(np.abs(got_q[r0 + i] - wq) <= lim["q"])
            assert np.all(np.abs(kh[blk, :, slot % c.bs] - wk) <= lim["k"])
            assert np.array_equal(vh[blk, :, slot % c.bs], wv)
        r0 += n
    assert np.all(got_q[r0:] == 7.0)                       # rows behind the last sequence
    same = ~touched.to(DEV)[:, None, :].expand(c.k.shape[:3])
    for new, old in ((c.k, k0), (c.v, v0)):                # every other slot, NaN bits included
        view = torch.int16 if c.dt == torch.bfloat16 else torch.int32
        assert torch.equal(new.view(view)[same], old.view(view)[same])
    if weights:
        assert torch.equal(w[same], w0[same]) and float(w[~same].abs().max()) == 0.0


@pytest.mark.parametrize("heads", HEADS)
def test_append_ragged_rows(heads):
    c = Cache(*heads, 16, [0, 5, 31, 16], 4)
    check_append(c, [3, 0, 17, 1], positions=[0, 70000, 3, 2 ** 30], weights=True, pad=2)
    c.close()


@pytest.mark.parametrize("bs", [1, 7, 12, 64])
def test_append_block_sizes(bs):
    c = Cache(8, 2, 64, "bf16", bs, [0, 11], -(-40 // bs))
    check_append(c, [29, 28])
    c.close()


def test_append_without_gains_and_without_offsets():
    c = Cache(8, 2, 64, "bf16", 16, [4, 16, 0], 3)
    check_append(c, [2, 1, 3], with_gain=False)
    c.close()
    c = Cache(8, 2, 64, "bf16", 16, [4, 16, 0], 3)
    qkv = c.normal((3, 12 * 64))
    q = c.dr.cache_append(c.kv(), qkv)
    d = Cache(8, 2, 64, "bf16", 16, [4, 16, 0], 3)
    q2 = d.dr.cache_append(d.kv(), qkv, offsets=torch.arange(4, dtype=torch.int32, device=DEV))
    assert torch.equal(q, q2)
    assert torch.equal(c.k.view(torch.int16), d.k.view(torch.int16))
    c.close()
    d.close()


def test_append_many_sequences_and_rows():
    lens = [(37 * b) % 50 for b in range(64)]
    c = Cache(6, 2, 32, "f32", 16, lens, 6)
    check_append(c, [(b * 7) % 5 for b in range(64)])
    c.close()


def test_append_flags_what_it_cannot_store():
    c = Cache(8, 2, 64, "bf16", 16, [30, 30], 2)
    k0 = c.k.clone()
    qkv = c.normal((8, 12 * 64))
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device=DEV)
    c.dr.cache_append(c.kv(), qkv, offsets=off)             # slots 32, 33 are past the table
    assert c.dr.device_status() == -7
    assert not torch.isnan(c.k[int(c.table_h[0, 1]), :, 14:16].float()).any()
    c.k.copy_(k0)
    c.table[0, 1] = c.k.shape[0]                            # a block that the pool does not hold
    c.dr.cache_append(c.kv(), qkv[:2].contiguous(), offsets=torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV))
    assert c.dr.device_status() == -7
    assert torch.isnan(c.k[int(c.table_h[0, 1]), :, 14].float()).all()
    c.k.copy_(k0)
    for bad in ([0, 5, 4], [1, 4, 8], [0, 4, 9], [-1, 4, 8]):
        c.dr.cache_append(c.kv(), qkv, offsets=torch.tensor(bad, dtype=torch.int32, device=DEV))
        assert c.dr.device_status() == -1, bad
    assert torch.equal(c.k.view(torch.int16), k0.view(torch.int16))
    c.lens[1] = -3
    c.dr.cache_append(c.kv(), qkv[:2].contiguous())
    c.close(-7)


# ---------------------------------------------------------------- attention
def check_attend(c, q, res, n_new=0, blocks=None, w=None, w0=None):
    qh, kh, vh = f64(q), f64(c.k), f64(c.v)
    out = f64(res["out"])
    lse = None if res["lse"] is None else res["lse"].cpu().numpy().astype(np.float64)
    wn = None if w is None else w.cpu().numpy().astype(np.float64)
    wo = None if w is None else w0.cpu().numpy().astype(np.float64)
    seen_w = np.zeros(c.k.shape[:3], bool)
    bf = c.dt == torch.bfloat16
    for b in range(c.B):
        n = c.n_lens[b] + n_new
        for j in range(c.nkv):
            slots = np.arange(n)
            if blocks is not None:
                ids = [i for i in blocks[b, j].tolist() if i >= 0]
                slots = np.array([i * c.bs + s for i in ids for s in range(c.bs) if i * c.bs + s < n], dtype=np.int64)
            K, V = c.rows(kh, b, j, slots), c.rows(vh, b, j, slots)
            qq = qh[b, j * c.g: (j + 1) * c.g]
            want, p, want_lse = C.attend(qq, K, V)
            got = out[b, j * c.g: (j + 1) * c.g]
            if len(slots) == 0:
                assert np.all(got == 0)
                assert lse is None or np.all(np.isneginf(lse[b, j * c.g: (j + 1) * c.g]))
                continue
            delta = (c.d + 4) * U * (np.abs(qq) @ np.abs(K).T).max(axis=1)[:, None] / np.sqrt(c.d)
            run = min(len(slots), 1024) + 64
            rel = 2 * delta + run * U + (2.0 ** -16 if bf else 0.0)
            lim = (2.0 ** -8 if bf else 0.0) * np.abs(want) + rel * (p @ np.abs(V))
            assert np.all(np.abs(got - want) <= lim), (b, j, float(np.max(np.abs(got - want) / lim)))
            if lse is not None:
                e = np.abs(lse[b, j * c.g: (j + 1) * c.g] - want_lse)
                assert np.all(e <= delta[:, 0] + run * U + 4 * U * (1 + np.abs(want_lse)))
            if w is not None:
                blk = c.table_h[b, slots // c.bs]
                add = p.sum(axis=0)
                lim = (4 * delta.max() + 2 * run * U + 2.0 ** -20) * add + 2 * U * np.abs(wo[blk, j, slots % c.bs] + add)
                e = np.abs(wn[blk, j, slots % c.bs] - wo[blk, j, slots % c.bs] - add)
                assert np.all(e <= lim), (b, j, float(np.max(e / lim)))
                seen_w[blk, j, slots % c.bs] = True
    if w is not None:
        assert np.array_equal(wn[~seen_w], wo[~seen_w])


LENS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 129, 333, 640]


@pytest.mark.parametrize("heads", HEADS)
def test_attend_lengths(heads):
    c = Cache(*heads, 16, LENS, 41)
    q = c.normal((c.B, c.nq, c.d), 2.0)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, lse=True))
    w = c.weights()
    w0 = w.clone()
    r = c.dr.cache_attend(c.kv(), q, weights=w, max_len=640, lse=True)
    check_attend(c, q, r, w=w, w0=w0)
    c.close()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("bs", [16, 12])
def test_attend_block_lists(heads, bs):
    cols = -(-641 // bs)
    c = Cache(*heads, bs, LENS, cols)
    q = c.normal((c.B, c.nq, c.d), 2.0)
    n = 9
    lists = np.full((c.B, c.nkv, n), -1, np.int32)
    for b, L in enumerate(LENS):
        have = -(-L // bs)
        for j in range(c.nkv):
            m = min(have, int(c.rng.integers(0, n + 1)))
            pick = c.rng.choice(have, m, replace=False) if m else []
            if m and j == 0:
                pick[0] = have - 1 if have - 1 not in pick[1:] else pick[0]    # a block that ends inside
            lists[b, j, :m] = np.sort(pick)
    bl = torch.tensor(lists, device=DEV)
    w = c.weights()
    w0 = w.clone()
    r = c.dr.cache_attend(c.kv(), q, blocks=bl, weights=w, lse=True)
    check_attend(c, q, r, blocks=lists, w=w, w0=w0)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, blocks=bl), blocks=lists)
    # more entries than the table has columns: the rest is not read
    more = torch.full((c.B, c.nkv, cols + 5), -1, dtype=torch.int32, device=DEV)
    more[..., :n] = bl
    more[..., cols:] = 10 ** 6
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, blocks=more), blocks=lists)
    c.close()


@pytest.mark.parametrize("bs", [1, 7, 64, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_block_sizes(bs, dtype):
    lens = [300, 1, 65]
    c = Cache(8, 2, 64, dtype, bs, lens, -(-301 // bs))
    q = c.normal((3, 8, 64), 2.0)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, lse=True))
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (4, 1, 256, "bf16"), (2, 1, 256, "f32")])
def test_attend_long_sequences(heads):
    lens = [2049, 5000, 1023, 1024, 1025, 2048]
    c = Cache(*heads, 16, lens, 313)
    q = c.normal((c.B, c.nq, c.d), 2.0)
    w = c.weights()
    w0 = w.clone()
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, weights=w, lse=True), w=w, w0=w0)
    c.close()


@pytest.mark.parametrize("top", [1, 64, 65, 129, 511, 512, 513])
@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 8, 128, "bf16"), (4, 1, 256, "bf16"), (7, 1, 32, "bf16"),
                                   (8, 1, 128, "f32"), (3, 3, 64, "f32")])
def test_attend_short_sequences(heads, top):
    """Around the bound up to which a segment is one workgroup's."""
    lens = [0, 1, top // 2, top, max(1, top - 1)]
    c = Cache(*heads, 16, lens, 33)
    q = c.normal((c.B, c.nq, c.d), 2.0)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, max_len=top, lse=True))
    w = c.weights()
    w0 = w.clone()
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, max_len=top, weights=w, lse=True), w=w, w0=w0)
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 4, 64, "bf16"), (5, 5, 128, "f32")])
def test_attend_sixty_four_sequences(heads):
    """Below and above the number of segments that fill the chip."""
    lens = [(b * 131) % 1025 for b in range(64)]
    lens[3] = 1024
    c = Cache(*heads, 16, lens, 65)
    q = c.normal((64, c.nq, c.d), 2.0)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, max_len=1024, lse=True))
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, max_len=1025, lse=True))
    c.close()


@pytest.mark.parametrize("top", [512, 513, 1000, 1024, 1025])
def test_scratch_sized_for_the_largest_batch(top):
    """serves the calls of every smaller one."""
    import ctypes
    from paper_2602_01762_amd import binding as B
    lens = [(b * 131) % (top + 1) for b in range(64)]
    lens[3] = top
    c = Cache(8, 8, 32, "bf16", 16, lens, -(-top // 16))
    q = c.normal((64, c.nq, c.d), 2.0)
    n = B.prism_cache_scratch(c.dr.ctx, B.PRISM_CACHE_ATTEND, 64, top)
    scratch = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    for nb in (64, 33, 32, 31, 16, 5, 1):
        kv = c.dr.cache(c.lens[:nb], c.k, c.v, c.table[:nb])
        out = torch.empty((nb, c.nq, c.d), dtype=c.dt, device=DEV)
        io = B.prism_cache_attention()
        io.kv, io.max_len, io.d_q, io.d_out = ctypes.addressof(kv), top, B.ptr(q), B.ptr(out)
        io.d_scratch, io.scratch_bytes = B.ptr(scratch), n
        B.prism_cache_attend(c.dr.ctx, io)
        assert torch.equal(out, c.dr.cache_attend(kv, q[:nb], max_len=top)["out"])
    c.close()


def test_attend_sees_the_appended_row():
    c = Cache(8, 2, 64, "bf16", 16, [0, 47, 48], 4)
    q = c.dr.cache_append(c.kv(), c.normal((3, 12 * 64)))
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, n_new=1, max_len=49, lse=True), n_new=1)
    c.close()


def test_attend_flags_what_it_cannot_read():
    c = Cache(8, 2, 64, "bf16", 16, [100, 100], 8)
    q = c.normal((2, 8, 64))
    ref = c.dr.cache_attend(c.kv(), q)["out"]
    assert c.dr.device_status() == 0
    cut = c.dr.cache_attend(c.kv(), q, max_len=64)["out"]   # longer than its bound: cut to it
    assert c.dr.device_status() == -7
    c.n_lens = [64, 64]
    check_attend(c, q, {"out": cut, "lse": None})
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.table[0, 3] = bad
        out = c.dr.cache_attend(c.kv(), q)["out"]
        assert c.dr.device_status() == -7
        assert torch.equal(out[1], ref[1]) and not torch.isnan(out.float()).any()
    c.table[0, 3] = int(c.table_h[0, 3])
    c.lens[0] = -5
    out = c.dr.cache_attend(c.kv(), q)["out"]
    assert c.dr.device_status() == -7
    assert float(out[0].float().abs().max()) == 0.0 and torch.equal(out[1], ref[1])
    c.lens[0] = 100
    for bad in ([0, 0, -1], [3, 1, 2], [-2, 1, 2], [0, 7, 2 ** 31 - 1], [0, 1, 7]):
        lst = torch.tensor([[bad, bad], [[0, 1, -1]] * 2], dtype=torch.int32, device=DEV)
        out = c.dr.cache_attend(c.kv(), q, blocks=lst)["out"]
        assert c.dr.device_status() == -1, bad
        assert not torch.isnan(out.float()).any()
    c.close()


def entries_read(lst, n_blocks):
    """Of a block list, the entries that are larger than all before them, up
    to the first -1; the others as -1."""
    top, out = -1, []
    for i in lst:
        out.append(i if top < i < n_blocks else -1)
        top = max(top, 2 ** 31 if i == -1 else i)
    return out


def check_malformed(c, lists):
    q = c.normal((c.B, c.nq, c.d), 2.0)
    read = np.array([[entries_read(row, -(-c.n_lens[b] // c.bs)) for row in rows] for b, rows in enumerate(lists)])
    bl = torch.tensor(lists, dtype=torch.int32, device=DEV)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, blocks=bl, lse=True), blocks=read)
    assert c.dr.device_status() == -1
    w = c.weights()
    w0 = w.clone()
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, blocks=bl, weights=w, lse=True), blocks=read, w=w, w0=w0)
    assert c.dr.device_status() == -1


@pytest.mark.parametrize("bad", [[3, -1, 3, -1], [3, 1, 3, -1], [0, 5, 3, 5], [5, 3, 4, -1], [-1, 0, -1, 2], [0, 1, -5, 1],
                                 [1, 2 ** 31 - 1, 2, -1], [6, 0, 7, 6], [-2 ** 31, 0, 0, -1]])
def test_attend_reads_no_block_of_a_list_twice(bad):
    """whatever stands between the repeats."""
    c = Cache(8, 2, 64, "bf16", 16, [100, 100], 8)
    check_malformed(c, [[bad, bad], [bad, [0, 1, 6, -1]]])
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (4, 1, 128, "f32"), (2, 1, 256, "bf16")])
@pytest.mark.parametrize("bs,n", [(1, 130), (1, 500), (1, 700), (4, 128), (4, 300), (16, 150)])
def test_attend_long_malformed_lists(heads, bs, n):
    """Lists of more entries than a wave looks at together, each with an entry
    out of its order, by one workgroup each and joined."""
    lens = [bs * 900, bs * 800 - 1, bs * 700, bs * 900, bs * 650 + 1]
    c = Cache(*heads, bs, lens, 900)
    lists = []
    for b in range(c.B):
        rows = []
        for j in range(c.nkv):
            m = int(c.rng.integers(n // 2, n + 1))
            row = np.full(n, -1, np.int64)
            row[:m] = np.sort(c.rng.choice(-(-lens[b] // bs), m, replace=False))
            at = [int(c.rng.integers(1, m)), m - 1, m // 2, 66, 64][b]
            row[at] = [row[int(c.rng.integers(0, at))], row[0], -1, 10 ** 6, -7][b]
            if b == 2:
                row[m - 1] = row[3]                          # behind the -1
            rows.append(row.tolist())
        lists.append(rows)
    check_malformed(c, lists)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_infinities_and_nan(dtype):
    """-inf scores take no part; a row of them gives zeros; NaN in a visible
    key, or a +inf score, reaches its own KV head's outputs only."""
    lens = [80, 80, 80, 80]
    c = Cache(4, 2, 64, dtype, 16, lens, 6)
    q = c.normal((4, 4, 64)).abs() + 0.5                     # positive: the sign of k decides
    def put(pool, b, slot, value):
        pool[int(c.table_h[b, slot // 16]), 0, slot % 16] = value
    for s in range(80):
        put(c.k, 0, s, float("-inf"))                        # every score -inf
    for s in range(3, 80):
        put(c.k, 1, s, float("-inf"))                        # three slots left
    put(c.k, 2, 70, float("nan"))
    put(c.k, 3, 5, float("inf"))
    r = c.dr.cache_attend(c.kv(), q, lse=True)
    out, lse = r["out"].float(), r["lse"]
    assert float(out[0, :2].abs().max()) == 0.0 and torch.isneginf(lse[0, :2]).all()
    assert torch.isnan(out[2, :2]).all() and torch.isnan(out[3, :2]).all()
    assert not torch.isnan(out[:, 2:]).any()
    kh, vh = f64(c.k), f64(c.v)
    want, _, _ = C.attend(f64(q)[1, :2], c.rows(kh, 1, 0, np.arange(3)), c.rows(vh, 1, 0, np.arange(3)))
    assert np.all(np.abs(out[1, :2].cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 1e-4)
    c.close()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", [[1, 17, 333], [1, 700, 2100]])
def test_attend_infinite_values(heads, lens):
    """Every probability is above 0, so an infinity among the values gives its
    channel that infinity, both signs NaN, and leaves the other channels and
    KV heads alone: by one workgroup, joined, with slot weights, by a list."""
    c = Cache(*heads, 16, lens, -(-lens[-1] // 16))
    q = c.normal((c.B, c.nq, c.d))
    for b, n in enumerate(lens):
        def put(slot, channel, value):
            c.v[int(c.table_h[b, slot // 16]), 0, slot % 16, channel] = value
        put(n - 1, 0, float("inf"))
        put(n // 2, 1, float("-inf"))
        put(0, 2, float("inf"))
        put(n - 1, 2, float("-inf"))
        for slot in range(0, n, 3):
            put(slot, 7, float("-inf"))
    qh, kh, vh = f64(q), f64(c.k), f64(c.v)
    every = torch.full((c.B, c.nkv, c.columns), -1, dtype=torch.int32, device=DEV)
    for b, n in enumerate(lens):
        every[b, :, : -(-n // 16)] = torch.arange(-(-n // 16), device=DEV)
    for kw in (dict(), dict(weights=c.weights()), dict(blocks=every)):
        out = f64(c.dr.cache_attend(c.kv(), q, max_len=lens[-1], **kw)["out"])
        for b, n in enumerate(lens):
            for j in range(c.nkv):
                K, V = c.rows(kh, b, j, np.arange(n)), c.rows(vh, b, j, np.arange(n))
                qq = qh[b, j * c.g: (j + 1) * c.g]
                p = C.attend(qq, K, np.zeros_like(V))[1]
                with np.errstate(invalid="ignore"):
                    want = (p[:, :, None] * V).sum(axis=1)
                got = out[b, j * c.g: (j + 1) * c.g]
                fin = np.isfinite(want)
                assert np.array_equal(got[~fin], want[~fin], equal_nan=True), (b, j)
                delta = (c.d + 4) * U * (np.abs(qq) @ np.abs(K).T).max() / np.sqrt(c.d)
                rel = 2 * delta + (min(n, 1024) + 64) * U
                lim = (2.0 ** -8 if c.dt == torch.bfloat16 else 0.0) * np.abs(want[fin])
                lim = lim + rel * (p[:, :, None] * np.abs(V)).sum(axis=1)[fin]
                assert np.all(np.abs(got[fin] - want[fin]) <= lim), (b, j)
    c.close()


def test_attend_rows_beyond_four_gigabytes():
    """Blocks at the end of pools of more than 2^32 bytes."""
    nkv, d, bs = 8, 128, 16
    n = (1 << 32) // (nkv * d * bs * 2) + 40
    c = Cache(8, 8, 128, "bf16", 16, [70, 33], 5)
    k, v = c.k, c.v
    big_k = torch.full((n, nkv, bs, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    big_v = torch.full((n, nkv, bs, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    m = k.shape[0]
    big_k[n - m:], big_v[n - m:] = k, v
    q = c.normal((2, 8, 128), 2.0)
    w = torch.zeros((n, nkv, bs), device=DEV)
    ref = c.dr.cache_attend(c.kv(), q)["out"]
    kv = c.dr.cache(c.lens, big_k, big_v, c.table + (n - m))
    assert torch.equal(c.dr.cache_attend(kv, q, weights=w)["out"], ref)
    assert abs(float(w.sum()) - 2 * 8) < 1e-3 and float(w[: n - m].abs().max()) == 0.0
    s = c.dr.summary_buffer(kv)
    c.dr.cache_summarize(kv, s)
    s0 = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    assert torch.equal(s[n - m:].view(torch.int16), s0.view(torch.int16))
    new = c.table.flip(1) + (n - m)
    new[:, 0] = torch.tensor([n - m - 1, n - m - 2], dtype=torch.int32)
    r = c.dr.cache_evict(kv, new, w, 9)
    assert r["lens"].tolist() == [9, 9]
    for b in range(2):
        for j in range(nkv):
            kept = r["kept"][b, j].long().cpu()
            blk = torch.tensor(c.table_h[b])[kept // bs]
            assert torch.equal(big_k[int(new[b, 0]), j, :9], k[blk.to(DEV), j, (kept % bs).to(DEV)])
    c.close()


@pytest.mark.parametrize("L", [-1, -3, -2 ** 31])
@pytest.mark.parametrize("n_new", [1, 5])
def test_a_negative_length_sees_nothing(L, n_new):
    """also with new slots behind it, and is flagged by every call."""
    c = Cache(8, 2, 64, "bf16", 16, [40, 40], 4)
    q, w = c.normal((2, 8, 64)), c.weights()
    s0 = torch.full((c.k.shape[0], c.nkv, 2, c.d), 3.0, dtype=c.dt, device=DEV)
    c.lens.copy_(torch.tensor([40 - n_new, 40 - n_new], dtype=torch.int32))
    ref = c.dr.cache_attend(c.kv(), q, n_new=n_new)["out"]
    s_ref = c.dr.cache_summarize(c.kv(), s0.clone(), n_new=n_new)
    blocks_ref = c.dr.cache_select(c.kv(), q, s_ref, 2, n_new=n_new)
    assert c.dr.device_status() == 0
    c.lens[0] = L
    w0 = w.clone()
    lst = torch.tensor([[[0, 1, -1]] * 2] * 2, dtype=torch.int32, device=DEV)
    lst[0] = -1
    for kw in (dict(), dict(weights=w), dict(blocks=lst), dict(max_len=40)):
        r = c.dr.cache_attend(c.kv(), q, n_new=n_new, lse=True, **kw)
        assert c.dr.device_status() == -7
        assert float(r["out"][0].float().abs().max()) == 0.0 and torch.isneginf(r["lse"][0]).all()
        if "blocks" not in kw and "weights" not in kw:
            assert torch.equal(r["out"][1], ref[1])
    first = torch.tensor(c.table_h[0], device=DEV)
    assert torch.equal(w[first], w0[first])
    s = c.dr.cache_summarize(c.kv(), s0.clone(), n_new=n_new)
    assert c.dr.device_status() == -7
    assert float((s[first] - 3).abs().max()) == 0.0
    other = torch.tensor(c.table_h[1], device=DEV)
    assert torch.equal(s[other].view(torch.int16), s_ref[other].view(torch.int16))
    blocks = c.dr.cache_select(c.kv(), q, s_ref, 2, n_new=n_new)
    assert c.dr.device_status() == -7
    assert (blocks[0] == -1).all() and torch.equal(blocks[1], blocks_ref[1])
    c.close()


# ------------------------------------------------- summaries and selection
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("bs", [16, 7])
def test_summaries(heads, bs):
    lens = [0, 1, 6, 7, 8, 16, 100, 113]
    c = Cache(*heads, bs, lens, -(-114 // bs))
    s = torch.full((c.k.shape[0], c.nkv, 2, c.d), 9.0, dtype=c.dt, device=DEV)
    assert c.dr.cache_summarize(c.kv(), s) is s
    got, kh = f64(s), f64(c.k)
    untouched = np.ones(c.k.shape[0], bool)
    for b, L in enumerate(lens):
        for j in range(c.nkv):
            want = C.summarize(c.rows(kh, b, j, np.arange(L)), bs)
            blk = c.table_h[b, : len(want)]
            assert np.array_equal(got[blk, j], want)
            untouched[blk] = False
    assert np.all(got[untouched] == 9.0)
    # the last slots only: the blocks that hold them, nothing else
    for span, n_new in ((1, 0), (bs, 0), (bs + 1, 0), (3, 1), (10 ** 6, 0)):
        c.n_lens = [L - n_new if L >= n_new else 0 for L in lens]
        c.lens.copy_(torch.tensor(c.n_lens, dtype=torch.int32))
        part = torch.full_like(s, 9.0)
        c.dr.cache_summarize(c.kv(), part, n_new=n_new, span=span)
        want = np.full(got.shape, 9.0)
        for b in range(c.B):
            n = c.n_lens[b] + n_new
            if n == 0 or lens[b] == 0:
                continue
            for i in range(max(0, n - span) // bs, -(-n // bs)):
                want[c.table_h[b, i]] = got[c.table_h[b, i]]
        if n_new == 0:
            assert np.array_equal(f64(part), want), span
        else:
            ok = [b for b in range(c.B) if lens[b] > 0]
            blk = np.concatenate([c.table_h[b] for b in ok])
            assert np.array_equal(f64(part)[blk], want[blk])
    c.close()


def test_summaries_pass_over_nan_keys():
    c = Cache(4, 1, 32, "bf16", 16, [16], 1)
    blk = int(c.table_h[0, 0])
    c.k[blk, 0, 3, :8] = float("nan")
    c.k[blk, 0, 5, 8] = float("inf")
    c.k[blk, 0, 6, 9] = float("-inf")
    s = f64(c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv())))[blk, 0]
    kh = f64(c.k)[blk, 0]
    assert np.array_equal(s[0], np.nanmin(kh, axis=0)) and np.array_equal(s[1], np.nanmax(kh, axis=0))
    c.close()


def check_select(c, q, s, out, n_blocks, first, last, n_new=0):
    qh, sh, got = f64(q), f64(s), out.cpu().numpy()
    for b in range(c.B):
        n = c.n_lens[b] + n_new
        nblk = -(-n // c.bs)
        for j in range(c.nkv):
            score = C.block_scores(qh[b, j * c.g: (j + 1) * c.g], sh[c.table_h[b, :nblk], j])
            want = C.choose(score, n_blocks, first, last)
            assert got[b, j, : len(want)].tolist() == want.tolist(), (b, j)
            assert np.all(got[b, j, len(want):] == -1)


@pytest.mark.parametrize("heads", HEADS)
def test_select(heads):
    c = Cache(*heads, 16, LENS, 41)
    q = c.normal((c.B, c.nq, c.d), 2.0)
    s = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    for n, first, last in ((1, 0, 0), (5, 1, 2), (40, 0, 3), (60, 2, 2), (4, 4, 0), (4, 0, 4)):
        check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, n, first, last), n, first, last)
        check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, n, first, last, max_len=640), n, first, last)
    c.close()


def test_select_ties_and_nan():
    c = Cache(4, 2, 64, "bf16", 4, [400, 399], 101)
    q = c.normal((2, 4, 64))
    s = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    for b in range(2):                                       # groups of equal summaries, some NaN
        for i in range(100):
            s[int(c.table_h[b, i])] = s[int(c.table_h[b, i % 3])]
        for i in (0, 7, 50):
            s[int(c.table_h[b, i]), 1] = float("nan")
    for n in (1, 2, 33, 34, 35, 66, 67, 98, 99, 100):
        check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, n), n, 0, 0)
    s.zero_()
    for n in (1, 50, 99):
        check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, n, 0, 1), n, 0, 1)
    c.close()


def test_select_many_blocks():
    c = Cache(4, 1, 32, "bf16", 1, [9000, 4097, 1025], 9000)
    q = c.normal((3, 4, 32))
    s = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    for n, first, last in ((1, 0, 0), (300, 3, 7), (4097, 0, 1), (8999, 1, 0)):
        check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, n, first, last), n, first, last)
    c.close()


# ---------------------------------------------------------------- eviction
def check_evict(c, w, n_keep, first, recent, max_len=0):
    nb = -(-n_keep // c.bs)
    new_h = np.full((c.B, c.columns), -1, np.int64)
    new_h[:, :nb] = c.free[: c.B * nb].reshape(c.B, nb)
    new = torch.tensor(new_h, dtype=torch.int32, device=DEV)
    k0, v0, w0 = c.k.clone(), c.v.clone(), w.clone()
    r = c.dr.cache_evict(c.kv(), new, w, n_keep, first, recent, max_len=max_len)
    kept, lens = r["kept"].cpu().numpy(), r["lens"].tolist()
    wh = w0.cpu().numpy()
    view = torch.int16 if c.dt == torch.bfloat16 else torch.int32
    want = [k0.view(view).clone(), v0.view(view).clone(), w0.view(torch.int32).clone()]
    for b, L in enumerate(c.n_lens):
        assert lens[b] == min(n_keep, L)
        for j in range(c.nkv):
            pick = C.choose(c.rows(wh, b, j, np.arange(L)), n_keep, first, recent)
            assert kept[b, j, : len(pick)].tolist() == pick.tolist(), (b, j)
            assert np.all(kept[b, j, len(pick):] == -1)
            i = np.arange(len(pick))
            src, dst = c.table_h[b, pick // c.bs], new_h[b, i // c.bs]
            for t in want:
                t[dst, j, i % c.bs] = t[src, j, pick % c.bs]
    assert torch.equal(c.k.view(view), want[0]) and torch.equal(c.v.view(view), want[1])
    assert torch.equal(w.view(torch.int32), want[2])
    return r, new_h


@pytest.mark.parametrize("heads", HEADS)
def test_evict(heads):
    c = Cache(*heads, 16, LENS, 41, spare=12 * 41)
    for n, first, recent in ((1, 0, 0), (64, 4, 16), (333, 0, 333), (640, 3, 5), (200, 200, 0)):
        check_evict(c, c.weights(0.2), n, first, recent, max_len=640 if n == 64 else 0)
    c.close()


def test_select_from_more_blocks_than_fit_on_chip():
    c = Cache(2, 1, 32, "bf16", 1, [30000, 24577, 5], 30000)
    q = c.normal((3, 2, 32))
    s = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    for n, first, last in ((100, 0, 0), (12000, 2, 5)):
        check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, n, first, last), n, first, last)
    c.close()


@pytest.mark.parametrize("bs", [1, 7, 64])
def test_evict_block_sizes(bs):
    lens = [0, 1, 130, 301]
    cols = -(-301 // bs)
    c = Cache(8, 2, 64, "bf16", bs, lens, cols, spare=4 * cols)
    for n in (5, 64, 129, 301):
        check_evict(c, c.weights(0.1), n, min(2, n), min(3, n - 2))
    c.close()


def test_evict_weights_that_tie_or_are_no_numbers():
    c = Cache(4, 2, 32, "bf16", 16, [500, 257], 32, spare=64)
    w = torch.zeros(c.k.shape[:3], device=DEV)
    check_evict(c, w, 100, 0, 0)                             # all equal: the lowest slots
    w = torch.randint(0, 3, c.k.shape[:3], generator=c.gen, device=DEV).float()
    for n in (1, 90, 255, 256):
        check_evict(c, w.clone(), n, 2 if n > 2 else 0, 3 if n > 5 else 0)
    w = torch.randn(c.k.shape[:3], generator=c.gen, device=DEV)
    r = torch.rand(w.shape, generator=c.gen, device=DEV)
    w[r < 0.3] = float("nan")
    w[(r > 0.3) & (r < 0.4)] = float("inf")
    w[(r > 0.4) & (r < 0.5)] = float("-inf")
    w[(r > 0.5) & (r < 0.6)] = -0.0
    w[(r > 0.6) & (r < 0.7)] = 0.0
    w[(r > 0.7) & (r < 0.8)] = -float("nan")
    for n in (10, 60, 130, 200, 250):
        check_evict(c, w.clone(), n, 1, 4)
    c.close()


def test_evict_long_sequences():
    c = Cache(2, 1, 32, "bf16", 16, [40000, 33000, 1024], 2500, spare=3 * 700)
    for n in (1, 1025, 11000):
        check_evict(c, c.weights(0.3), n, min(4, n), n // 4 if n > 8 else 0)
    c.close()


@pytest.mark.parametrize("lens", [[40000, 25000, 24577], [24576, 20000, 9000]])
def test_evict_many_equal_weights(lens):
    """More slots with the weight of the cut than the choice lists."""
    c = Cache(2, 2, 32, "bf16", 16, lens, 2500, spare=3 * 700)
    for n, first, recent in ((11000, 4, 100), (3000, 0, 0)):
        check_evict(c, c.weights(0.9), n, first, recent, max_len=max(lens))
    w = c.weights(0.5)
    check_evict(c, torch.where(w > 0, 1.0 + torch.floor(w), w), 9000, 1, 1, max_len=max(lens))
    c.close()


def test_evict_flags_blocks_it_cannot_use():
    c = Cache(4, 2, 32, "bf16", 16, [60, 60], 4, spare=8)
    w = c.weights()
    new = torch.tensor([[int(c.free[0]), c.k.shape[0], -1, -1], [int(c.free[1]), int(c.free[2]), -1, -1]],
                       dtype=torch.int32, device=DEV)
    r = c.dr.cache_evict(c.kv(), new, w, 32)
    assert c.dr.device_status() == -7
    for b, i in ((0, 0), (1, 1)):                            # the good blocks are filled
        kept = r["kept"][b, 1].cpu().numpy()[16 * i: 16 * i + 16]
        blk = torch.tensor(c.table_h[b, kept // 16], device=DEV)
        assert torch.equal(c.k[int(new[b, i]), 1], c.k[blk, 1, torch.tensor(kept % 16, device=DEV).long()])
    c.table[0, 1] = -1                                       # source slots without storage rank last
    new[0, 1] = int(c.free[3])
    r = c.dr.cache_evict(c.kv(), new, w, 32)
    assert c.dr.device_status() == -7
    kept = r["kept"][0].cpu().numpy()
    assert not ((kept >= 16) & (kept < 32)).any()
    c.close()


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 1, 128, "f32"), (32, 8, 128, "bf16")])
def test_a_cache_filled_read_evicted_and_selected_from(heads):
    c = Cache(*heads, 16, [150, 0, 333], 24, spare=3 * 24)
    w = torch.zeros(c.k.shape[:3], device=DEV)
    wo = np.zeros(c.k.shape[:3])
    for _ in range(3):
        q = c.dr.cache_append(c.kv(), c.normal((c.B, (c.nq + 2 * c.nkv) * c.d), 1.5), weights=w)
        c.dr.cache_attend(c.kv(), q, n_new=1, weights=w)
        c.lens += 1
        c.n_lens = [n + 1 for n in c.n_lens]
        kh = f64(c.k)
        for b in range(c.B):
            for j in range(c.nkv):
                s = np.arange(c.n_lens[b])
                _, p, _ = C.attend(f64(q)[b, j * c.g: (j + 1) * c.g], c.rows(kh, b, j, s), c.rows(kh, b, j, s))
                wo[c.table_h[b, s // c.bs], j, s % c.bs] += p.sum(0)
    assert np.max(np.abs(w.cpu().numpy() - wo)) < 1e-4
    r, new_h = check_evict(c, w, 100, 4, 32)
    c.table_h, c.n_lens = new_h, r["lens"].tolist()
    c.table, c.lens = torch.tensor(new_h, dtype=torch.int32, device=DEV), r["lens"]
    s = c.dr.summary_buffer(c.kv())
    c.dr.cache_summarize(c.kv(), s)
    qkv = c.normal((c.B, (c.nq + 2 * c.nkv) * c.d), 1.5)
    pos = torch.tensor([153, 3, 336], dtype=torch.int32, device=DEV)
    q = c.dr.cache_append(c.kv(), qkv, positions=pos, weights=w)
    c.dr.cache_summarize(c.kv(), s, n_new=1, span=1)
    full = c.dr.cache_summarize(c.kv(), torch.zeros_like(s), n_new=1)
    assert torch.equal(s.view(torch.uint8), full.view(torch.uint8))
    blocks = c.dr.cache_select(c.kv(), q, s, 4, n_first=1, n_last=1, n_new=1)
    check_select(c, q, s, blocks, 4, 1, 1, n_new=1)
    r = c.dr.cache_attend(c.kv(), q, n_new=1, blocks=blocks, lse=True)
    check_attend(c, q, r, n_new=1, blocks=blocks.cpu().numpy())
    c.close()


def test_drafting_goes_on_over_an_evicted_cache():
    """A drafting chain over the evicted cache equals the oracle's over the
    same slots (each KV head with the tokens that it kept)."""
    from harness import check_chain, oracle_for
    from paper_2602_01762_amd import Drafter
    from synth import SMALL_BF16_CHAIN, make_inputs, make_weights
    cfg = SMALL_BF16_CHAIN.with_(batch=2, ctx_range=(200, 333), n_steps=3)
    wt, inp = make_weights(cfg, DEV), make_inputs(cfg, DEV, extra_blocks=2 * 6)
    dr = Drafter(cfg)
    dr.load(wt)
    used = set(inp.block_table.flatten().tolist())
    free = [i for i in range(inp.k_pool.shape[0]) if i not in used]
    new = torch.full_like(inp.block_table, -1)
    new[:, :6] = torch.tensor(free[:12], dtype=torch.int32).view(2, 6)
    w = torch.rand(inp.k_pool.shape[:3], device=DEV)
    kv = dr.cache(inp.ctx_lens, inp.k_pool, inp.v_pool, inp.block_table)
    r = dr.cache_evict(kv, new, w, 77, n_first=4, n_recent=20)
    inp.block_table, inp.ctx_lens = new, r["lens"]
    orc, hi = oracle_for(cfg, wt, inp)
    out = dr.chain(inp, logits=True, hidden=True)
    torch.cuda.synchronize()
    assert dr.device_status() == 0
    check_chain(cfg, out, orc, hi, [0, 1], inp=inp)
    dr.close()


def test_drafting_at_the_true_positions_after_an_eviction():
    """The kept keys carry the rotation of their old positions: draft steps at
    the positions that follow those, in the slots that follow the kept ones,
    equal the oracle's."""
    from harness import LOGIT_TOL, check_draft_kv, check_token, oracle_for
    from paper_2602_01762_amd import Drafter
    from synth import SMALL_BF16_CHAIN, make_inputs, make_weights
    cfg = SMALL_BF16_CHAIN.with_(batch=2, ctx_range=(200, 333), n_steps=3)
    wt, inp = make_weights(cfg, DEV), make_inputs(cfg, DEV, extra_blocks=2 * 6)
    dr = Drafter(cfg)
    dr.load(wt)
    used = set(inp.block_table.flatten().tolist())
    free = [i for i in range(inp.k_pool.shape[0]) if i not in used]
    new = torch.full_like(inp.block_table, -1)
    new[:, :6] = torch.tensor(free[:12], dtype=torch.int32).view(2, 6)
    w = torch.rand(inp.k_pool.shape[:3], device=DEV)
    kv = dr.cache(inp.ctx_lens, inp.k_pool, inp.v_pool, inp.block_table)
    r = dr.cache_evict(kv, new, w, 77, n_first=4, n_recent=20)
    old = inp.ctx_lens.clone()
    inp.block_table, inp.ctx_lens = new, r["lens"]
    assert (old > inp.ctx_lens).all()
    orc, hi = oracle_for(cfg, wt, inp)
    caches = [orc.new_cache(hi, b) for b in range(2)]
    tokens, feat, want_feat = inp.tokens, inp.features, f64(inp.features)
    for k in range(3):
        rows = {"tokens": tokens, "feat": feat, "seq": torch.arange(2, dtype=torch.int32, device=DEV),
                "pos": old + k, "slot": inp.ctx_lens + k}
        st = dr.step(k + 1, inp, rows, logits=True)
        torch.cuda.synchronize()
        assert dr.device_status() == 0
        slots = [int(n) + k for n in inp.ctx_lens]
        h, lg = orc.forward(cfg.fmap[k], tokens.tolist(), want_feat, [int(n) + k for n in old], caches, [0, 1], slots,
                            [list(range(s + 1)) for s in slots])
        got = st["logits"].cpu().numpy()
        assert np.max(np.abs(got - lg)) <= LOGIT_TOL[cfg.dtype]
        for b in range(2):
            check_token(lg[b], int(st["ids"][b, 0]), "seq %d step %d" % (b, k + 1))
        tokens, feat, want_feat = st["ids"][:, 0].contiguous(), st["hidden"], h
    check_draft_kv(cfg, inp, {b: caches[b]["draft"] for b in range(2)}, [0, 1])
    dr.close()


def test_a_row_appended_in_the_same_step_is_kept():
    """Append, attention and eviction of one decoding step: once the lengths
    have been advanced, the new row is a candidate, and the most recent one."""
    c = Cache(8, 2, 64, "bf16", 16, [100, 47], 8, spare=4)
    w = torch.zeros(c.k.shape[:3], device=DEV)
    kv = c.kv()
    q = c.dr.cache_append(kv, c.normal((2, 12 * 64)), weights=w)
    c.dr.cache_attend(kv, q, n_new=1, weights=w)
    c.lens += 1
    c.n_lens = [101, 48]
    r, _ = check_evict(c, w, 32, 4, 8)
    assert r["lens"].tolist() == [32, 32]
    assert (r["kept"][0, :, -1] == 100).all() and (r["kept"][1, :, -1] == 47).all()
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 1, 128, "f32")])
def test_a_batch_without_any_slot(heads):
    c = Cache(*heads, 16, [0, 0, 0], 4, spare=6)
    q, w = c.normal((3, c.nq, c.d)), c.weights()
    kv, w0, k0 = c.kv(), w.clone(), c.k.clone()
    s = torch.full((c.k.shape[0], c.nkv, 2, c.d), 3.0, dtype=c.dt, device=DEV)
    c.dr.cache_summarize(kv, s)
    c.dr.cache_summarize(kv, s, span=5)
    assert float((s - 3).abs().max()) == 0.0
    blocks = c.dr.cache_select(kv, q, s, 2, 1, 1)
    assert (blocks == -1).all()
    for kw in (dict(), dict(weights=w), dict(blocks=blocks), dict(blocks=blocks, weights=w), dict(max_len=1)):
        r = c.dr.cache_attend(kv, q, lse=True, out=torch.full_like(q, 5.0), **kw)
        assert float(r["out"].float().abs().max()) == 0.0 and torch.isneginf(r["lse"]).all()
    new = torch.full((3, 4), -1, dtype=torch.int32, device=DEV)
    new[:, :2] = torch.tensor(c.free[:6].reshape(3, 2), device=DEV)
    r = c.dr.cache_evict(kv, new, w, 20, 1, 2)
    assert r["lens"].tolist() == [0, 0, 0] and (r["kept"] == -1).all()
    assert torch.equal(w, w0) and torch.equal(c.k.view(torch.uint8), k0.view(torch.uint8))
    c.close()


def test_blocks_that_the_pool_does_not_hold():
    """Summaries and scores skip them and flag; every other block is right."""
    c = Cache(8, 2, 64, "bf16", 16, [160, 160], 10)
    q = c.normal((2, 8, 64))
    good = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    keep = c.table.clone()
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1):
        c.table.copy_(keep)
        c.table[0, 4] = bad
        s = torch.zeros_like(good)
        c.dr.cache_summarize(c.kv(), s)
        assert c.dr.device_status() == -7
        want = good.clone()
        want[int(keep[0, 4])] = 0
        assert torch.equal(s.view(torch.int16), want.view(torch.int16))
        blocks = c.dr.cache_select(c.kv(), q, good, 9)
        assert c.dr.device_status() == -7
        assert blocks[0].tolist() == [[0, 1, 2, 3, 5, 6, 7, 8, 9]] * 2       # ranks last
    c.table.copy_(keep)
    c.lens[0] = 400                                          # past the capacity
    for call in (lambda: c.dr.cache_summarize(c.kv(), s), lambda: c.dr.cache_select(c.kv(), q, good, 3),
                 lambda: c.dr.cache_select(c.kv(), q, good, 3, max_len=160)):
        call()
        assert c.dr.device_status() == -7
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (6, 2, 32, "f32")])
def test_sequences_that_share_a_prefix(heads):
    """Full blocks in the tables of several sequences are read, summarised,
    chosen and evicted from for each."""
    c = Cache(*heads, 16, [150, 100, 48, 49], 10, spare=4 * 3)
    for b in (1, 2, 3):
        c.table_h[b, :3] = c.table_h[0, :3]
        for i in range(3, -(-c.n_lens[b] // 16)):           # (its own blocks hold slots already)
            assert not torch.isnan(c.k[int(c.table_h[b, i]), :, 0].float()).any()
    c.table.copy_(torch.tensor(c.table_h, dtype=torch.int32))
    q = c.normal((c.B, c.nq, c.d), 2.0)
    check_attend(c, q, c.dr.cache_attend(c.kv(), q, lse=True))
    s = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    got, kh = f64(s), f64(c.k)
    for b, L in enumerate(c.n_lens):
        for j in range(c.nkv):
            want = C.summarize(c.rows(kh, b, j, np.arange(L)), 16)
            assert np.array_equal(got[c.table_h[b, : len(want)], j], want)
    again = s.clone()
    c.dr.cache_summarize(c.kv(), again, span=60)
    assert torch.equal(again, s)
    check_select(c, q, s, c.dr.cache_select(c.kv(), q, s, 3, 1, 1), 3, 1, 1)
    check_evict(c, c.weights(0.1), 40, 2, 9)
    c.close()


def test_a_drafting_batch_serves_the_cache_calls():
    from paper_2602_01762_amd import Drafter
    from synth import SMALL_BF16_CHAIN, make_inputs
    cfg = SMALL_BF16_CHAIN.with_(batch=2, ctx_range=(20, 33), n_steps=2)
    inp = make_inputs(cfg, DEV)
    dr = Drafter(cfg)
    q = torch.randn((2, cfg.n_q_heads, cfg.head_dim), device=DEV).to(torch.bfloat16)
    w = torch.zeros(inp.k_pool.shape[:3], device=DEV)
    a = dr.cache_attend(dr.batch(inp), q, weights=w)["out"]
    b = dr.cache_attend(dr.cache(inp.ctx_lens, inp.k_pool, inp.v_pool, inp.block_table), q)["out"]
    assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())
    assert abs(float(w.sum()) - 2 * cfg.n_q_heads) < 1e-3
    assert dr.device_status() == 0
    dr.close()


def test_calls_repeat_bit_for_bit_and_replay_in_a_graph():
    c = Cache(32, 8, 128, "bf16", 16, [1, 700, 333, 64], 48, spare=4 * 8)
    q = c.normal((4, 32, 128), 2.0)
    s = c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv()))
    new = torch.full((4, 48), -1, dtype=torch.int32, device=DEV)
    new[:, :8] = torch.tensor(c.free[:32].reshape(4, 8), device=DEV)
    w = c.weights()
    kv = c.kv()

    def same(x, y):             # bits: slots that a longer length uncovers hold NaN
        return torch.equal(x.view(torch.uint8), y.view(torch.uint8))

    def step():
        bl = c.dr.cache_select(kv, q, s, 6, 1, 1)
        a = c.dr.cache_attend(kv, q, blocks=bl)["out"]
        b = c.dr.cache_attend(kv, q, lse=True)
        e = c.dr.cache_evict(kv, new, w, 128, 2, 9)
        return [bl, a, b["out"], b["lse"], e["kept"], e["lens"]]

    eager = [t.clone() for t in step()]
    again = step()
    assert all(same(x, y) for x, y in zip(eager, again))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        c.lens.copy_(torch.tensor([1 + i, 700 - 37 * i, 333, 64 * i], dtype=torch.int32))
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = step()
        assert all(same(x, y) for x, y in zip(out, want)), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    assert all(same(x, y) for x, y in zip(other, step()))
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 1, 128, "f32")])
def test_a_decoding_step_replays_in_two_graphs(heads):
    """Append, weighted attention, summaries, selection and the attention over
    the chosen blocks, captured once for each of two halves of a batch that
    share the pools; replayed at once on two streams, over growing lengths,
    with eager steps of a copy between the replays."""
    lens = [0, 700, 15, 333]
    a, b = (Cache(*heads, 16, lens, 48, seed=5) for _ in range(2))
    width = (a.nq + 2 * a.nkv) * a.d
    qkv = a.normal((6, 4, width))
    w = [torch.zeros(c.k.shape[:3], device=DEV) for c in (a, b)]
    s = [c.dr.cache_summarize(c.kv(), c.dr.summary_buffer(c.kv())) for c in (a, b)]
    kvs = [[c.dr.cache(c.lens[i: i + 2], c.k, c.v, c.table[i: i + 2]) for i in (0, 2)] for c in (a, b)]
    rows = [torch.empty((2, width), dtype=a.dt, device=DEV) for _ in range(2)]

    def step(c, x, half, src):
        kv = kvs[x][half]
        q = c.dr.cache_append(kv, src, weights=w[x])
        full = c.dr.cache_attend(kv, q, n_new=1, weights=w[x], lse=True)
        c.dr.cache_summarize(kv, s[x], n_new=1, span=1)
        blocks = c.dr.cache_select(kv, q, s[x], 5, 1, 1, n_new=1)
        part = c.dr.cache_attend(kv, q, n_new=1, blocks=blocks)["out"]
        return [q, full["out"], full["lse"], blocks, part]

    def same(x, y):
        return torch.equal(x.view(torch.uint8), y.view(torch.uint8))

    torch.cuda.synchronize()
    graphs, outs = [], []
    for half in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(a, 0, half, rows[half]))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(6):
        for half in range(2):
            rows[half].copy_(qkv[i, 2 * half: 2 * half + 2])
        torch.cuda.synchronize()
        for half, st in enumerate(streams):
            with torch.cuda.stream(st):
                graphs[half].replay()
        torch.cuda.synchronize()
        for half in range(2):
            want = step(b, 1, half, qkv[i, 2 * half: 2 * half + 2].contiguous())
            assert all(same(x, y) for x, y in zip(outs[half], want)), (i, half)
        for x, y in ((a.k, b.k), (a.v, b.v), (w[0], w[1]), (s[0], s[1])):
            assert same(x, y), i
        a.lens += 1
        b.lens += 1
    a.close()
    b.close()


def test_two_streams_at_once():
    """Calls of one context on two streams do not share anything."""
    c = Cache(8, 2, 64, "bf16", 16, [3000, 2000], 190)
    qs = [c.normal((2, 8, 64), 2.0) for _ in range(2)]
    kv = c.kv()
    want = [c.dr.cache_attend(kv, q)["out"].clone() for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(c.dr.cache_attend(kv, qs[i])["out"])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])
    c.close()


# ------------------------------------------------------------------ refusals
def test_refusals():
    from paper_2602_01762_amd import PrismError, binding as B
    c = Cache(8, 2, 64, "bf16", 16, [20, 20], 4, spare=8)
    kv, q, w = c.kv(), c.normal((2, 8, 64)), c.weights()
    s = c.dr.summary_buffer(kv)
    new = torch.full((2, 4), -1, dtype=torch.int32, device=DEV)
    new[:, 0] = torch.tensor(c.free[:2], device=DEV)
    bad = [
        lambda: c.dr.cache_append(kv, c.normal((3, 12 * 64))),                 # 3 rows, no offsets
        lambda: c.dr.cache_append(kv, c.normal((0, 12 * 64)), offsets=torch.zeros(3, dtype=torch.int32, device=DEV)),
        lambda: c.dr.cache_attend(kv, q, max_len=65),
        lambda: c.dr.cache_attend(kv, q, max_len=-1),
        lambda: c.dr.cache_attend(kv, q, n_new=-1),
        lambda: c.dr.cache_summarize(kv, s, span=-1),
        lambda: c.dr.cache_summarize(kv, s, n_new=65),
        lambda: c.dr.cache_select(kv, q, s, 0),
        lambda: c.dr.cache_select(kv, q, s, 3, n_first=2, n_last=2),
        lambda: c.dr.cache_select(kv, q, s, 3, n_first=-1),
        lambda: c.dr.cache_evict(kv, new, w, 0),
        lambda: c.dr.cache_evict(kv, new, w, 65),
        lambda: c.dr.cache_evict(kv, new, w, 8, n_first=5, n_recent=4),
        lambda: c.dr.cache_evict(kv, new, w, 8, n_recent=-1),
        lambda: c.dr.cache_evict(kv, c.table, w, 8),                           # onto itself
    ]
    for i, call in enumerate(bad):
        with pytest.raises(PrismError) as e:
            call()
        assert e.value.status == -1 and str(e.value), i
    io = B.prism_cache_attention()
    import ctypes
    io.kv = ctypes.addressof(kv)
    out, scratch = torch.empty_like(q), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    io.d_q, io.d_out, io.d_scratch, io.scratch_bytes = B.ptr(q), B.ptr(out), B.ptr(scratch), 1 << 20
    io.max_len = 0
    io.d_weights = B.ptr(w)                                                    # a call that needs scratch
    for field, value in (("scratch_bytes", 16), ("d_scratch", 0), ("d_q", 0), ("d_q", B.ptr(q) + 2),
                         ("d_out", B.ptr(out) + 8), ("kv", None)):
        keep = getattr(io, field)
        setattr(io, field, value)
        with pytest.raises(PrismError) as e:
            B.prism_cache_attend(c.dr.ctx, io)
        assert e.value.status == -1, field
        setattr(io, field, keep)
    with pytest.raises(PrismError):
        B.prism_cache_scratch(c.dr.ctx, 4, 1, 0)
    with pytest.raises(PrismError):
        B.prism_cache_scratch(c.dr.ctx, 0, 3, 0)
    more = c.dr.cache(torch.zeros(3, dtype=torch.int32, device=DEV), c.k, c.v,
                      torch.zeros((3, 4), dtype=torch.int32, device=DEV))
    with pytest.raises(PrismError) as e:                                       # 3 sequences, max_batch 2
        c.dr.cache_summarize(more, s)
    assert e.value.status == -1
    big = c.dr.cache(c.lens, c.k, c.v, c.table)
    big.n_pool_blocks = 1 << 27                                                # 2^32 rows
    with pytest.raises(PrismError) as e:
        B.prism_cache_summarize(c.dr.ctx, big, 0, 0, s)
    assert e.value.status == -2
    assert c.dr.device_status() == 0
    c.close()
