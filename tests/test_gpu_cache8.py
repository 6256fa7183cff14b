"""The 8-bit cache on the GPU against the fp64 oracle.

Codes and scales are compared for equality.  Values are exact; keys that are
normalised and rotated go through some tens of fp64 operations, so a key is off by
less than 2^-44 of its head's largest magnitude, and takes another code than the
oracle's only next to the border of two.  That an input lies there is a matter of
10^-11 for each (2^-44 of magnitudes of some 2^2 against steps of 2^-9 or more of
the scale, twice), and inputs are seeded.  Queries are normalised and rotated in
fp32: (d / 2 + 10) 2^-24 of the two channels of a pair together and of the value (the
mean of d squares, halved by the root, and some ten operations behind it), and in
bf16 one rounding more, half a step, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from oracle import cache8 as C8
from test_gpu_cache import EPS, Cache, f64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"
F8 = torch.float8_e4m3fn
TABLE = C8.e4m3_table()


def values(codes):
    return TABLE[codes.view(torch.uint8).cpu().numpy()]


class Cache8(Cache):
    """A batch with a cache of the context's type (Cache) and an 8-bit one in
    blocks of its own, whose first `packed[b]` slots the oracle has written; codes
    of slots that hold nothing and scales of blocks that hold nothing are NaN."""

    def __init__(self, nq, nkv, d, dtype, bs, lens, columns, packed=None, seed=0, spread=1.0, **kw):
        super().__init__(nq, nkv, d, dtype, bs, lens, columns, seed=seed, **kw)
        n = self.k.shape[0]
        self.table8_h = self.rng.permutation(n)[: self.B * columns].reshape(self.B, columns)
        self.table8 = torch.tensor(self.table8_h, dtype=torch.int32, device=DEV)
        self.codes_h = np.full((2, n, nkv, bs, d), np.nan)          # values of the codes
        self.exp_h = np.full((n, nkv, 2), -999)
        self.packed = list(lens if packed is None else packed)
        for b, m in enumerate(self.packed):
            rows = self.rng.normal(size=(2, m, nkv, d)) * np.exp(spread * self.rng.normal(size=(2, 1, nkv, 1)))
            for w in range(2):
                self.oracle_write(b, w, 0, rows[w])
        self.k8, self.v8 = (self.to_codes(x) for x in self.codes_h)
        self.scales = self.to_scales(self.exp_h)

    @staticmethod
    def to_codes(x):
        return torch.tensor(np.where(np.isnan(x), 0.0, x), dtype=torch.float32).to(F8).view(torch.uint8).masked_fill_(
            torch.tensor(np.isnan(x)), 0x7f).to(DEV).view(F8)

    @staticmethod
    def to_scales(e):
        return torch.tensor(np.where(e == -999, np.nan, np.exp2(e.astype(np.float64))), dtype=torch.float32, device=DEV)

    def oracle_write(self, b, w, slot, rows):
        """rows [n, nkv, d] to the slots from `slot` on of pool w, in the oracle's copy."""
        done = 0
        while done < len(rows):
            t = slot + done
            off = t % self.bs
            n = min(self.bs - off, len(rows) - done)
            blk = int(self.table8_h[b, t // self.bs])
            for j in range(self.nkv):
                v, e = C8.write_block(self.codes_h[w, blk, j, :off], int(self.exp_h[blk, j, w]), rows[done: done + n, j])
                self.codes_h[w, blk, j, : off + n] = v
                self.exp_h[blk, j, w] = e
            done += n

    def kv8(self):
        return self.dr.cache8(self.lens, self.k8, self.v8, self.scales, self.table8)

    def check8(self):
        """Codes and scales are the oracle's, whole pools."""
        assert np.array_equal(self.scales.cpu().numpy(), self.to_scales(self.exp_h).cpu().numpy(), equal_nan=True)
        for got, want in zip((self.k8, self.v8), self.codes_h):
            assert np.array_equal(values(got), want, equal_nan=True)

    def dequantised(self):
        """Keys and values [n, nkv, bs, d] that the codes stand for."""
        s = np.exp2(np.where(self.exp_h == -999, 0, self.exp_h).astype(np.float64))
        return [self.codes_h[w] * s[:, :, None, None, w] for w in range(2)]


HEADS = [(4, 4, 64, "f32"), (8, 2, 64, "bf16"), (32, 8, 128, "bf16"), (7, 1, 32, "bf16"),
         (4, 1, 256, "bf16"), (8, 1, 128, "f32"), (2, 1, 256, "f32"), (6, 2, 32, "f32")]


# ------------------------------------------------------------------- append
def append(c, counts, positions=None, gains=True, pad=0, std=1.5, offsets=True, put=()):
    T, nh = int(sum(counts)) + pad, c.nq + 2 * c.nkv
    qkv = c.normal((T, nh, c.d), std)
    qkv[T - pad:] = float("nan")
    for row, head, dim, value in put:
        qkv[row, head, dim] = value
    g = [(1 + 0.1 * c.normal((c.d,)).float()).to(c.dt) if gains else None for _ in range(2)]
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV) if offsets else None
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    out = torch.full((T, c.nq, c.d), 7.0, dtype=c.dt, device=DEV)
    r = c.dr.cache8_append(c.kv8(), qkv.view(T, -1), g[0], g[1], offsets=off, positions=pos, out=out)
    assert r is out
    torch.cuda.synchronize()
    x, got = f64(qkv), f64(out)
    gains64 = [None if t is None else f64(t) for t in g]
    half = 2.0 ** -8 if c.dt == torch.bfloat16 else 0.0
    r0 = 0
    for b, n in enumerate(counts):
        rows = np.zeros((2, n, c.nkv, c.d))
        for i in range(n):
            p = (c.n_lens[b] if positions is None else positions[b]) + i
            with np.errstate(invalid="ignore"):
                q, rows[0, i], rows[1, i] = C8.append_row(x[r0 + i], c.nq, c.nkv, p, 1e4, float(np.float32(EPS)), *gains64)
            top = np.abs(q).max(axis=1, keepdims=True)
            y = x[r0 + i, : c.nq]
            if gains64[0] is not None:
                y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + EPS) * gains64[0]
            pair = np.abs(y[:, : c.d // 2]) + np.abs(y[:, c.d // 2:])
            lim = half * np.abs(q) + (c.d / 2 + 10) * 2.0 ** -24 * (np.concatenate([pair, pair], -1) + np.abs(q))
            lim = lim + p * 2.0 ** -50 * top
            over = float(np.max(np.abs(got[r0 + i] - q) / lim))
            assert over <= 1, (b, i, over)
        for w in range(2):
            c.oracle_write(b, w, c.n_lens[b], rows[w])
        r0 += n
    assert np.all(got[r0:] == 7.0)
    c.check8()


@pytest.mark.parametrize("heads", HEADS)
def test_append_ragged_rows(heads):
    c = Cache8(*heads, 16, [0, 5, 31, 16, 15], 5)
    append(c, [3, 0, 17, 1, 40], positions=[0, 70000, 3, 2 ** 30, 9], pad=2)
    c.close()


@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (6, 2, 32, "f32"), (8, 1, 128, "bf16"), (4, 1, 256, "bf16")])
@pytest.mark.parametrize("bs", [1, 7, 12, 64, 100])
def test_append_block_sizes(heads, bs):
    """Blocks of more rows than stay in registers, and of one."""
    c = Cache8(*heads, bs, [0, 11, 64], -(-150 // bs))
    append(c, [70, 47, 33])
    c.close()


def test_append_one_row_each():
    c = Cache8(32, 8, 128, "bf16", 16, [4, 16, 0, 31, 200], 14)
    append(c, [1] * 5, offsets=False)
    c.close()
    c = Cache8(8, 2, 64, "bf16", 16, [(37 * b) % 50 for b in range(64)], 6)
    append(c, [(b * 7) % 5 for b in range(64)], gains=False)
    c.close()


def test_scales_grow_and_stay():
    """A block whose scale a later row raises, by little, by a lot, and not."""
    for std in (0.01, 3.0, 5e4, 1e-30, 1e30):
        c = Cache8(8, 2, 64, "bf16", 16, [5, 21, 16], 4)
        append(c, [2, 1, 3], gains=False, std=std)
        c.close()


def test_append_step_by_step_keeps_a_block():
    """One row at a time for three blocks: the oracle's every time."""
    c = Cache8(8, 2, 64, "bf16", 16, [0, 13], 5)
    for i in range(48):
        append(c, [1, 1], std=1.5 if i % 11 else 9.0, gains=False)
        c.lens += 1
        c.n_lens = [n + 1 for n in c.n_lens]
    c.close()


def test_append_what_is_not_finite():
    """is NaN in its place and no more: the scale is the others'.  (Keys without
    gains, at position 0, where a rotation leaves pairs alone but for NaN.)"""
    inf, nan = float("inf"), float("nan")
    c = Cache8(4, 2, 64, "bf16", 16, [0, 3], 2)
    # heads 0 .. 3 queries, 4, 5 keys, 6, 7 values
    append(c, [2, 2], gains=False, put=[(0, 6, 1, inf), (1, 6, 2, -inf), (2, 7, 63, nan), (3, 7, 0, inf)])
    v = values(c.v8)[int(c.table8_h[0, 0]), 0]
    assert np.isnan(v[0, 1]) and np.isnan(v[1, 2]) and np.isfinite(v[0, 2])
    c.close()
    c = Cache8(4, 2, 64, "bf16", 16, [0, 0], 2)
    append(c, [2, 1], gains=False, put=[(0, 6, d, nan) for d in range(64)] + [(1, 6, d, 0.0) for d in range(64)])
    c.close()
    # values of no magnitude, and beyond the largest scale
    c = Cache8(4, 2, 64, "f32", 16, [0, 0], 2)
    append(c, [1, 2], gains=False, put=[(r, 6, d, 0.0) for r in range(3) for d in range(64)] +
           [(0, 7, 5, 3.3e38), (0, 7, 6, 1e38), (1, 7, 0, 2e-38), (1, 7, 1, 1e-44)])
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_keys_beyond_the_largest_fp32(dtype):
    """Two finite channels of 3e38 that a rotation adds to 4.2e38: a finite key, so the
    largest code over the largest scale (448 * 2^119), of either sign."""
    c = Cache8(4, 2, 64, dtype, 16, [0, 3], 2)
    # heads 4, 5 are keys; at position 7 the first pair turns by 7 rad: cos 0.75, sin 0.66
    append(c, [2, 1], gains=False, positions=[7, 7],
           put=[(0, 4, 0, 3e38), (0, 4, 32, -3e38), (2, 5, 0, -3e38), (2, 5, 32, 3e38)])
    v, s = values(c.k8), c.scales.cpu().numpy()
    a, b = int(c.table8_h[0, 0]), int(c.table8_h[1, 0])
    assert v[a, 0, 0, 0] == 448.0 and s[a, 0, 0] == 2.0 ** 119
    assert v[b, 1, 3, 0] == -448.0 and s[b, 1, 0] == 2.0 ** 119
    c.close()


def test_keys_next_to_a_border():
    """Keys that lie halfway between two codes, and next to it, without a rotation
    (position 0) and gains: ties go to the even code, the others to the nearer."""
    c = Cache8(1, 1, 32, "f32", 16, [0], 1)
    t = TABLE[:127]
    mid = ((t[1:] + t[:-1]) / 2)[20:20 + 31 * 3]
    qkv = torch.zeros((9, 3, 32), device=DEV)
    for k, f in enumerate((1.0, 1 + 2.0 ** -22, 1 - 2.0 ** -22)):
        for r in range(3):
            qkv[3 * k + r, 1, :31] = torch.tensor(mid[31 * r: 31 * r + 31] * f, dtype=torch.float32)
    qkv[0, 1, 31] = 448.0                                              # the scale is 1
    qkv[:, 2] = qkv[:, 1]
    off = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    for r in range(9):                                                 # each at position 0
        c.dr.cache8_append(c.kv8(), qkv[r: r + 1].reshape(1, -1).contiguous(), offsets=off,
                           positions=torch.zeros(1, dtype=torch.int32, device=DEV))
        c.lens += 1
    x = f64(qkv)
    blk = int(c.table8_h[0, 0])
    for pool, h in ((c.k8, 1), (c.v8, 2)):
        assert np.array_equal(values(pool)[blk, 0, :9], C8.e4m3_round(x[:, h]))
    assert float(c.scales[blk].max()) == 1.0
    c.close()


def test_append_flags_what_it_cannot_store():
    c = Cache8(8, 2, 64, "bf16", 16, [30, 30], 2)
    k0, s0 = c.k8.view(torch.uint8).clone(), c.scales.clone()
    qkv = c.normal((8, 12 * 64))
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device=DEV)
    q = c.dr.cache8_append(c.kv8(), qkv, offsets=off)       # slots 32, 33 are past the table
    assert c.dr.device_status() == -7 and not torch.isnan(q.float()).any()
    assert not np.isnan(values(c.k8)[int(c.table8_h[0, 1]), :, 14:16]).any()

    def restore():
        c.k8.view(torch.uint8).copy_(k0)
        c.scales.copy_(s0)

    restore()
    c.table8[0, 1] = c.k8.shape[0]                          # a block that the pool does not hold
    two = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    c.dr.cache8_append(c.kv8(), qkv[:2].contiguous(), offsets=two)
    assert c.dr.device_status() == -7
    assert np.isnan(values(c.k8)[int(c.table8_h[0, 1]), :, 14]).all()
    restore()
    for bad in ([0, 5, 4], [1, 4, 8], [0, 4, 9], [-1, 4, 8]):
        c.dr.cache8_append(c.kv8(), qkv, offsets=torch.tensor(bad, dtype=torch.int32, device=DEV))
        assert c.dr.device_status() == -1, bad
    assert torch.equal(c.k8.view(torch.uint8), k0) and torch.equal(c.scales.view(torch.int32), s0.view(torch.int32))
    c.lens[1] = -3
    c.dr.cache8_append(c.kv8(), qkv[:2].contiguous())
    c.close(-7)


# ------------------------------------------------------------- pack, unpack
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("bs", [16, 12])
def test_pack_and_unpack(heads, bs):
    lens = [0, 1, 15, 16, 17, 100, 333]
    start = [0, 0, 3, 16, 16, 57, 200]
    c = Cache8(*heads, bs, lens, -(-334 // bs), packed=start)
    kh, vh = f64(c.k), f64(c.v)
    c.dr.cache8_pack(c.kv8(), c.kv(), start=torch.tensor(start, dtype=torch.int32, device=DEV), max_len=333)
    for b, L in enumerate(lens):
        slots = np.arange(start[b], L)
        for w, p in enumerate((kh, vh)):
            blk = c.table_h[b, slots // bs]
            c.oracle_write(b, w, start[b], p[blk, :, slots % bs])
    c.check8()
    # and back, from other slots on
    k0, v0 = c.k.clone(), c.v.clone()
    back = [0, 1, 0, 5, 17, 99, 31]
    c.dr.cache8_unpack(c.kv8(), c.kv(), start=torch.tensor(back, dtype=torch.int32, device=DEV))
    want = [f64(k0), f64(v0)]
    for b, L in enumerate(lens):
        slots = np.arange(back[b], L)
        for w, x in enumerate(c.dequantised()):
            want[w][c.table_h[b, slots // bs], :, slots % bs] = x[c.table8_h[b, slots // bs], :, slots % bs]
    for got, x in zip((c.k, c.v), want):
        assert np.array_equal(f64(got), x, equal_nan=True)
    c.check8()                                               # the 8-bit cache is left as it was
    c.close()


@pytest.mark.parametrize("bs", [1, 7, 64, 200])
def test_pack_block_sizes(bs):
    c = Cache8(8, 2, 64, "bf16", bs, [300, 65, 1], -(-302 // bs), packed=[0, 40, 0])
    c.dr.cache8_pack(c.kv8(), c.kv(), start=torch.tensor([0, 40, 0], dtype=torch.int32, device=DEV))
    kh, vh = f64(c.k), f64(c.v)
    for b, s in enumerate([0, 40, 0]):
        slots = np.arange(s, c.n_lens[b])
        for w, p in enumerate((kh, vh)):
            c.oracle_write(b, w, s, p[c.table_h[b, slots // bs], :, slots % bs])
    c.check8()
    c.close()


def test_pack_takes_the_new_rows_too_and_is_cut_at_max_len():
    c = Cache8(8, 2, 64, "bf16", 16, [32, 20], 4, packed=[0, 0])
    c.lens -= 1
    kh, vh = f64(c.k), f64(c.v)
    c.dr.cache8_pack(c.kv8(), c.kv(), n_new=1, max_len=25)
    assert c.dr.device_status() == -7                         # 32 slots, 25 of them taken
    for b, n in enumerate([25, 20]):
        slots = np.arange(n)
        for w, p in enumerate((kh, vh)):
            c.oracle_write(b, w, 0, p[c.table_h[b, slots // 16], :, slots % 16])
    c.check8()
    c.close()


def test_moves_flag_what_they_cannot_reach():
    c = Cache8(8, 2, 64, "bf16", 16, [40, 40], 3)
    k0 = c.k.clone()
    c.dr.cache8_unpack(c.kv8(), c.kv(), start=torch.tensor([-1, 40], dtype=torch.int32, device=DEV))
    assert c.dr.device_status() == -1
    c.dr.cache8_unpack(c.kv8(), c.kv(), start=torch.tensor([2 ** 31 - 1, 41], dtype=torch.int32, device=DEV))
    assert c.dr.device_status() == 0
    assert torch.equal(c.k.view(torch.int16), k0.view(torch.int16))
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.table[0, 1] = bad
        c.table8[1, 2] = bad
        c.dr.cache8_unpack(c.kv8(), c.kv())
        assert c.dr.device_status() == -7
        c.dr.cache8_pack(c.kv8(), c.kv())
        assert c.dr.device_status() == -7
    c.lens[0] = -7
    c.dr.cache8_pack(c.kv8(), c.kv())
    c.close(-7)


def test_pack_what_is_not_finite():
    c = Cache8(4, 2, 64, "bf16", 16, [20], 2, packed=[0])
    blk = int(c.table_h[0, 0])
    c.k[blk, 0, 3, 5] = float("inf")
    c.v[blk, 1, 15, 0] = float("nan")
    c.v[blk, 0] = float("-inf")
    kh, vh = f64(c.k), f64(c.v)
    c.dr.cache8_pack(c.kv8(), c.kv())
    slots = np.arange(20)
    for w, p in enumerate((kh, vh)):
        c.oracle_write(0, w, 0, p[c.table_h[0, slots // 16], :, slots % 16])
    c.check8()
    c.close()


# ------------------------------------------------------------------ together
def test_calls_repeat_and_replay_in_a_graph():
    """Append, pack and unpack captured, replayed over growing lengths with eager
    work between: the eager copy's bits every time."""
    a, b = (Cache8(8, 2, 64, "bf16", 16, [0, 70, 33], 8, seed=3) for _ in range(2))
    qkv = a.normal((6, 3, 12 * 64), 2.0)
    src = torch.empty((3, 12 * 64), dtype=a.dt, device=DEV)
    start = torch.tensor([0, 5, 33], dtype=torch.int32, device=DEV)

    def step(c, rows):
        q = c.dr.cache8_append(c.kv8(), rows)
        c.dr.cache8_unpack(c.kv8(), c.kv(), start=start, n_new=1)
        c.dr.cache8_pack(c.kv8(), c.kv(), start=start, n_new=1)
        return q

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    kv8, kv = a.kv8(), a.kv()
    with torch.cuda.graph(g):
        q = a.dr.cache8_append(kv8, src)
        a.dr.cache8_unpack(kv8, kv, start=start, n_new=1)
        a.dr.cache8_pack(kv8, kv, start=start, n_new=1)
    for i in range(6):
        src.copy_(qkv[i])
        g.replay()
        torch.cuda.synchronize()
        want = step(b, qkv[i].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(q.view(torch.int16), want.view(torch.int16)), i
        for x, y in ((a.k, b.k), (a.v, b.v), (a.k8, b.k8), (a.v8, b.v8), (a.scales, b.scales)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i
        a.lens += 1
        b.lens += 1
    a.close()
    b.close()


def test_blocks_beyond_four_gigabytes():
    """Blocks at the end of pools of more than 2^32 codes."""
    nkv, d, bs = 8, 128, 16
    n = (1 << 32) // (nkv * d * bs) + 40
    from test_gpu_cache import drafter
    dr = drafter(8, nkv, d, "bf16", bs, 1, 4)
    k8, v8 = (torch.empty((n, nkv, bs, d), dtype=torch.uint8, device=DEV).view(F8) for _ in range(2))
    scales = torch.ones((n, nkv, 2), device=DEV)
    tab = torch.tensor([[n - 1, n - 2, n - 7, n - 3]], dtype=torch.int32, device=DEV)
    lens = torch.tensor([0], dtype=torch.int32, device=DEV)
    kv8 = dr.cache8(lens, k8, v8, scales, tab)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v = (torch.randn((5, nkv, bs, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    src = torch.tensor([[3, 1, 0, 4]], dtype=torch.int32, device=DEV)
    lens.fill_(50)
    dr.cache8_pack(kv8, dr.cache(lens, k, v, src))
    got, want = torch.zeros_like(k), torch.zeros_like(k)
    dr.cache8_unpack(kv8, dr.cache(lens, got, torch.zeros_like(v), src))
    for i, (b, p) in enumerate(zip([3, 1, 0, 4], [n - 1, n - 2, n - 7, n - 3])):
        rows = min(16, 50 - 16 * i)
        if rows > 0:
            want[b, :, :rows] = (k8[p].float() * scales[p, :, 0][:, None, None])[:, :rows].to(torch.bfloat16)
            e = (k[b, :, :rows].float() - want[b, :, :rows].float()).abs()
            # half a step of a code, 2^-4 of the value, or of the subnormal codes
            assert bool((e <= 2.0 ** -4 * k[b, :, :rows].float().abs() + 2.0 ** -10 * scales[p, :, 0][:, None, None]).all())
    assert torch.equal(got, want)
    assert dr.device_status() == 0
    dr.close()


def test_refusals():
    from paper_2602_01762_amd import PrismError, binding as B
    import ctypes
    c = Cache8(8, 2, 64, "bf16", 16, [20, 20], 4)
    kv8, kv = c.kv8(), c.kv()
    one = c.dr.cache(c.lens[:1], c.k, c.v, c.table[:1])
    bad = [
        lambda: c.dr.cache8_append(kv8, c.normal((3, 12 * 64))),               # 3 rows, no offsets
        lambda: c.dr.cache8_append(kv8, c.normal((0, 12 * 64)), offsets=torch.zeros(3, dtype=torch.int32, device=DEV)),
        lambda: c.dr.cache8_pack(kv8, one),
        lambda: c.dr.cache8_unpack(kv8, kv, max_len=65),
        lambda: c.dr.cache8_unpack(kv8, kv, n_new=-1),
        lambda: c.dr.cache8_pack(c.dr.cache8(torch.zeros(3, dtype=torch.int32, device=DEV), c.k8, c.v8, c.scales,
                                             torch.zeros((3, 4), dtype=torch.int32, device=DEV)), kv),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(PrismError) as e:
            call()
        assert e.value.status == -1 and str(e.value), i
    qkv, q = c.normal((2, 12 * 64)), c.normal((2, 8, 64))
    io = B.prism_cache8_rows()
    io.kv8, io.rows, io.d_qkv, io.d_q = ctypes.addressof(kv8), 2, B.ptr(qkv), B.ptr(q)
    for field, value in (("kv8", None), ("d_qkv", 0), ("d_q", B.ptr(q) + 2), ("d_q_gain", B.ptr(q) + 2), ("rows", 0)):
        keep = getattr(io, field)
        setattr(io, field, value)
        with pytest.raises(PrismError) as e:
            B.prism_cache8_append(c.dr.ctx, io)
        assert e.value.status == -1, field
        setattr(io, field, keep)
    for field, value, st in (("d_scales", 0, -1), ("d_k_codes", B.ptr(c.k8) + 8, -1), ("d_scales", B.ptr(c.scales) + 4, -1),
                             ("d_ctx_lens", 0, -1), ("n_pool_blocks", 0, -1), ("batch", 0, -1), ("n_pool_blocks", 1 << 27, -2)):
        k = c.kv8()
        setattr(k, field, value)
        with pytest.raises(PrismError) as e:
            c.dr.cache8_pack(k, kv)
        assert e.value.status == st, field
    assert c.dr.device_status() == 0
    c.close()
