"""Attention of several rows per sequence on the GPU against the fp64 oracle.

Tolerances as for the attention of one row (test_gpu_cache.py): u = 2^-24, a score
is off by delta = (d + 4) u max_t sum_c |q_c k_tc| / sqrt(d), a probability by the
factor 1 + 2 delta, sums of n terms by (n + 64) u of their magnitudes, at most 1024 +
64 in a row; in bf16 contexts the products may take p as a hi/lo pair of bf16, 2^-16,
and an output is rounded once, half a step, 2^-8 of the value.  Prompts in bf16
contexts may take p rounded to bf16, half a step, 2^-8 of each product.  The values
of an 8-bit cache are exact.
"""
import numpy as np
import pytest
import torch

from oracle import cache8 as C8
from test_gpu_cache import U, Cache, f64
from test_gpu_cache8 import Cache8, F8, values

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"
HEADS = [(4, 4, 64, "f32"), (8, 2, 64, "bf16"), (32, 8, 128, "bf16"), (7, 1, 32, "bf16"),
         (4, 1, 256, "bf16"), (3, 3, 128, "bf16"), (8, 1, 128, "bf16"), (8, 1, 128, "f32"),
         (2, 1, 256, "f32"), (6, 2, 32, "f32"), (5, 1, 128, "bf16")]


def pools(c, eight):
    """What the keys and values stand for, and the table that leads to them."""
    return (c.dequantised(), c.table8_h) if eight else ((f64(c.k), f64(c.v)), c.table_h)


def check(c, q, counts, r, eight=False, n_new=1, window=0, n_first=0, rows=None, max_len=None, rounded=False):
    """rows: of each sequence, the ones that are compared (None: all); rounded: every
    sequence goes by the kernel of prompts."""
    (kh, vh), table = pools(c, eight)
    qh, out = f64(q), f64(r["out"])
    lse = None if r["lse"] is None else r["lse"].cpu().numpy().astype(np.float64)
    bf = c.dt == torch.bfloat16
    r0 = 0
    for b, n in enumerate(counts):
        top = min(c.n_lens[b] + n_new + n - 1, max_len or 1 << 30)
        slots = np.arange(max(top, 0))
        prompt = bf and (n * c.g > 16 or rounded)
        for j in range(c.nkv):
            K, V = kh[table[b, slots // c.bs], j, slots % c.bs], vh[table[b, slots // c.bs], j, slots % c.bs]
            for i in range(n) if rows is None else [i for i in rows if i < n]:
                at, hs = r0 + i, slice(j * c.g, (j + 1) * c.g)
                v = min(c.n_lens[b] + n_new + i, top)
                want, p, want_lse, s = C8.attend_row(qh[at, hs], K, V, v, window, n_first)
                got = out[at, hs]
                if len(s) == 0:
                    assert np.all(got == 0) and (lse is None or np.all(np.isneginf(lse[at, hs])))
                    continue
                delta = (c.d + 4) * U * (np.abs(qh[at, hs]) @ np.abs(K[s]).T).max(axis=1)[:, None] / np.sqrt(c.d)
                run = min(len(s), 1024) + 64
                rel = 2 * delta + run * U + (2.0 ** -16 if bf else 0.0) + (2.0 ** -8 if prompt else 0.0)
                lim = (2.0 ** -8 if bf else 0.0) * np.abs(want) + rel * (p @ np.abs(V[s]))
                e = np.abs(got - want)
                assert np.all(e <= lim), (b, j, i, float(np.max(e / lim)))
                if lse is not None:
                    e = np.abs(lse[at, hs] - want_lse)
                    assert np.all(e <= delta[:, 0] + run * U + 4 * U * (1 + np.abs(want_lse))), (b, j, i)
        r0 += n


def setup(heads, bs, lens, counts, eight, columns=None, seed=0, pad=0):
    """A cache that holds the rows too, while its lengths do not count them."""
    held = [L + n for L, n in zip(lens, counts)]
    columns = columns or max(1, -(-max(held) // bs))
    c = (Cache8 if eight else Cache)(*heads, bs, held, columns, seed=seed)
    c.n_lens = list(lens)
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    T = sum(counts) + pad
    q = c.normal((T, c.nq, c.d), 2.0)
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)
    return c, q, off


def sequences(c, eight):
    return c.kv8() if eight else c.kv()


LENS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 129, 333, 640]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads", HEADS)
def test_one_row_each(heads, eight):
    """A decoding step, by one workgroup each and joined."""
    c, q, off = setup(heads, 16, LENS, [1] * 12, eight)
    kv = sequences(c, eight)
    for window, n_first in ((0, 0), (64, 4), (1, 0), (100, 33)):
        kw = dict(window=window, n_first=n_first)
        check(c, q, [1] * 12, c.dr.cache_attend_rows(kv, q, n_new=1, lse=True, **kw), eight, **kw)
        check(c, q, [1] * 12, c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, max_len=641, **kw), eight, **kw)
    check(c, q, [1] * 12, c.dr.cache_attend_rows(kv, q, lse=True), eight, n_new=0)     # nothing seen by the first
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads", HEADS)
def test_drafts_to_score(heads, eight):
    """A few rows of each sequence, also none."""
    counts = [6, 0, 1, 3, 8, 5, 2, 7, 1, 6, 4, 6]
    c, q, off = setup(heads, 16, LENS, counts, eight, pad=2)
    kv = sequences(c, eight)
    for window, n_first in ((0, 0), (64, 4), (3, 1), (1000, 7)):
        out = torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
        kw = dict(window=window, n_first=n_first)
        r = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True, out=out, **kw)
        assert r["out"] is out and bool((out[sum(counts):] == 7.0).all())
        check(c, q, counts, r, eight, **kw)
    check(c, q, counts, c.dr.cache_attend_rows(kv, q, offsets=off, n_new=0), eight, n_new=0)
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,n_first", [(0, 0), (50, 4), (200, 70)])
def test_prompts(heads, eight, window, n_first):
    """Ragged prompts, with and without a context before them, single tokens
    among them."""
    lens, counts = [0, 300, 0, 77, 512, 5], [129, 200, 1, 64, 1, 33]
    c, q, off = setup(heads, 16, lens, counts, eight, pad=1)
    out = torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
    r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True,
                               out=out)
    assert bool((out[sum(counts):] == 7.0).all())
    check(c, q, counts, r, eight, window=window, n_first=n_first)
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("bs", [1, 7, 12, 64, 256])
@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (4, 1, 128, "f32")])
def test_block_sizes(heads, bs, eight):
    lens, counts = [300, 0, 65, 511], [1, 70, 6, 40]
    c, q, off = setup(heads, bs, lens, counts, eight)
    for window, n_first in ((0, 0), (90, 5)):
        r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, n_new=1, window=window, n_first=n_first)
        check(c, q, counts, r, eight, window=window, n_first=n_first)
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 8, 128, "bf16"), (4, 1, 256, "bf16"), (8, 1, 128, "f32")])
def test_long_contexts(heads, eight):
    """Split over the length and joined: few rows, and a chunk of a prompt."""
    lens, counts = [5000, 1023, 2048, 0], [3, 1, 6, 2]
    c, q, off = setup(heads, 16, lens, counts, eight)
    kv = sequences(c, eight)
    for window, n_first in ((0, 0), (700, 4), (4096, 0)):
        r = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        check(c, q, counts, r, eight, window=window, n_first=n_first)
    c.close()
    lens, counts = [3000, 100], [150, 90]
    c, q, off = setup(heads, 16, lens, counts, eight)
    kv = sequences(c, eight)
    for window, n_first in ((0, 0), (700, 4)):
        r = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        check(c, q, counts, r, eight, window=window, n_first=n_first, rows=[0, 1, 15, 16, 31, 32, 63, 64, 88, 89, 127, 128, 149])
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    lens = [(b * 131) % 900 for b in range(64)]
    counts = [(b * 5) % 9 for b in range(64)]
    c, q, off = setup((6, 2, 32, dtype), 16, lens, counts, False)
    check(c, q, counts, c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1, window=300, n_first=2, lse=True),
          window=300, n_first=2)
    c.close()


def test_a_long_prompt_among_single_tokens():
    lens, counts = [0, 2000, 700, 3], [1500, 1, 1, 1]
    c, q, off = setup((8, 2, 128, "bf16"), 16, lens, counts, False)
    r = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1, lse=True)
    check(c, q, counts, r, rows=[0, 1, 2, 63, 64, 127, 128, 500, 1023, 1024, 1498, 1499])
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n", [0, 1, 13, 70])
def test_a_lone_sequence_with_rows_behind_it(n, eight):
    """A buffer of more rows than the one sequence has: by the kernel of prompts, which
    rounds probabilities to bf16 (half a step, 2^-8 of each product), split over the
    length, however few they are."""
    c, q, off = setup((8, 2, 64, "bf16"), 16, [2500], [n], eight, columns=170, pad=200 - n)
    out = torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
    r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, n_new=1, lse=True, out=out)
    assert bool((out[n:] == 7.0).all())
    check(c, q, [n], r, eight, rounded=True)
    c.close()


@pytest.mark.parametrize("counts", [[1, 1], [7, 3], [90, 40]])
def test_on_another_stream(counts):
    c, q, off = setup((8, 2, 64, "bf16"), 16, [700, 90], counts, True, columns=60)
    kv = sequences(c, True)
    want = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1)["out"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1)["out"]
    side.synchronize()
    assert torch.equal(got, want)
    c.close()


def test_scratch_sized_for_the_largest_call():
    """serves smaller batches and fewer rows, whatever their window."""
    import ctypes
    from paper_2602_01762_amd import binding as B
    lens, counts = [900, 40, 1500, 700], [60, 1, 9, 130]
    c, q, off = setup((8, 2, 64, "bf16"), 16, lens, counts, False)
    n = B.prism_cache_rows_scratch(c.dr.ctx, 4, 200, 0)
    scratch = torch.empty(n, dtype=torch.uint8, device=DEV)
    for nb in (4, 3, 2, 1):
        kv = c.dr.cache(c.lens[:nb], c.k, c.v, c.table[:nb])
        T = sum(counts[:nb])
        for window, n_first in ((0, 0), (600, 3)):
            out = torch.empty((T, c.nq, c.d), dtype=c.dt, device=DEV)
            io = B.prism_cache_row_attention()
            io.kv, io.rows, io.d_offsets, io.n_new = ctypes.addressof(kv), T, B.ptr(off), 1
            io.window, io.n_first, io.d_q, io.d_out = window, n_first, B.ptr(q), B.ptr(out)
            io.d_scratch, io.scratch_bytes = B.ptr(scratch), n
            B.prism_cache_attend_rows(c.dr.ctx, io)
            want = c.dr.cache_attend_rows(kv, q[:T], offsets=off[: nb + 1], n_new=1, window=window, n_first=n_first)
            assert torch.equal(out, want["out"])
    c.close()


# ------------------------------------------------- what is not seen, not finite
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (8, 2, 64, "f32"), (4, 1, 256, "bf16"), (4, 4, 128, "bf16"),
                                   (4, 2, 32, "bf16")])
@pytest.mark.parametrize("counts", [[6, 5], [90, 40]])
def test_what_a_row_does_not_see_does_not_reach_it(heads, eight, counts):
    """NaN and infinities in keys and values of slots that some rows of a tile see
    and others do not: the others' outputs are those of a cache without them."""
    lens, window, n_first = [100, 30], 40, 3
    c, q, off = setup(heads, 16, lens, counts, eight)
    kw = dict(offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
    clean = c.dr.cache_attend_rows(sequences(c, eight), q, **kw)
    table = c.table8_h if eight else c.table_h
    bad = {0: [101, 63, 2, 103], 1: [32, 33, 1]}                # behind, before, at the edge of some rows' windows
    for b, slots in bad.items():
        for x, s in enumerate(slots):
            blk = int(table[b, s // 16])
            for w in range(2):
                if eight:
                    (c.k8, c.v8)[w].view(torch.uint8)[blk, 0, s % 16, 5 + x] = 0x7f if x % 2 else 0xff
                else:
                    (c.k, c.v)[w][blk, 0, s % 16, 5 + x] = [float("nan"), float("inf"), float("-inf"), float("nan")][x]
    r = c.dr.cache_attend_rows(sequences(c, eight), q, **kw)
    r0 = touched = 0
    for b, n in enumerate(counts):
        for i in range(n):
            s = set(C8.seen_slots(lens[b] + 1 + i, window, n_first).tolist())
            if s & set(bad[b]):
                touched += 1
                assert not bool(torch.isfinite(r["out"][r0 + i, : c.g].float()).all())
            else:
                assert torch.equal(r["out"][r0 + i], clean["out"][r0 + i]) or \
                    float((r["out"][r0 + i].float() - clean["out"][r0 + i].float()).abs().max()) < 0.02
                assert bool(torch.isfinite(r["lse"][r0 + i]).all())
            assert torch.equal(r["out"][r0 + i, c.g:], clean["out"][r0 + i, c.g:])      # other KV heads
        r0 += n
    assert touched
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5, 80])
def test_scores_that_are_infinite(dtype, n):
    """-inf scores take no part; a row of nothing else gives zeros."""
    lens = [80, 80]
    c, q, off = setup((4, 2, 64, dtype), 16, lens, [n, n], False)
    q = q.abs() + 0.5
    for s in range(80 + n):
        for b in range(2):
            if b == 0 or s >= 3:
                c.k[int(c.table_h[b, s // 16]), 0, s % 16] = float("-inf")
    r = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1, lse=True)
    assert float(r["out"][:n, :2].abs().max()) == 0.0 and bool(torch.isneginf(r["lse"][:n, :2]).all())
    assert bool(torch.isfinite(r["out"]).all())
    kh, vh = f64(c.k), f64(c.v)
    for i in range(n):
        K, V = c.rows(kh, 1, 0, np.arange(3)), c.rows(vh, 1, 0, np.arange(3))
        want, p, _, _ = C8.attend_row(f64(q)[n + i, :2], K, V, 3, 0, 0)
        assert np.all(np.abs(f64(r["out"])[n + i, :2] - want) <= 2.0 ** -7 * (p @ np.abs(V)) + 1e-4)
    c.close()


@pytest.mark.parametrize("n", [1, 40])
def test_infinite_values_that_are_seen(n):
    lens = [50]
    c, q, off = setup((8, 2, 64, "bf16"), 16, lens, [n], False)
    def put(slot, dim, x):
        c.v[int(c.table_h[0, slot // 16]), 0, slot % 16, dim] = x
    put(3, 0, float("inf"))
    put(40, 1, float("-inf"))
    put(3, 2, float("inf"))
    put(40, 2, float("-inf"))
    out = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1)["out"].float()
    assert bool((out[:, :4, 0] == float("inf")).all()) and bool((out[:, :4, 1] == float("-inf")).all())
    assert bool(torch.isnan(out[:, :4, 2]).all()) and bool(torch.isfinite(out[:, :4, 3:]).all())
    assert bool(torch.isfinite(out[:, 4:]).all())
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,counts", [([80, 80], [1, 1]), ([80, 80], [5, 3]), ([80], [90]), ([1500, 80], [5, 3]), ([1500], [90])])
def test_values_that_are_not_finite_behind_scores_of_minus_infinity(lens, counts, dtype):
    """A row whose every score is -inf gives zeros, whatever its values are; in tiles
    that one workgroup walks, in prompts, and joined."""
    c, q, off = setup((4, 2, 64, dtype), 16, lens, counts, False)
    q = q.abs() + 0.5
    for b, n in enumerate(counts):
        blocks = [int(x) for x in c.table_h[b]]
        c.k[blocks, 0] = float("-inf")
        for s, dim, x in ((0, 0, "inf"), (17, 1, "-inf"), (40, 2, "nan"), (lens[b], 3, "inf")):
            c.v[int(c.table_h[b, s // 16]), 0, s % 16, dim] = float(x)
    r = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1, lse=True)
    assert bool((r["out"][:, :2] == 0).all()) and bool(torch.isneginf(r["lse"][:, :2]).all())
    assert bool(torch.isfinite(r["out"]).all())
    c.close()


@pytest.mark.parametrize("eight", [False, True])
def test_other_rows_do_not_reach_a_prompt(eight):
    """Other queries in other rows, of the same sequence and of another one, change no
    bit of a row's output."""
    for lens, counts, changed in (([100], [200], slice(1, None, 2)), ([0, 50], [150, 201], slice(0, 150)),
                                  ([0, 2500], [150, 201], slice(0, 150))):
        c, q, off = setup((8, 2, 64, "bf16"), 16, lens, counts, eight)
        kv = sequences(c, eight)
        kept = torch.ones(q.shape[0], dtype=torch.bool, device=DEV)
        kept[changed] = False
        was = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True)
        q[changed] *= 30
        now = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True)
        for x in ("out", "lse"):
            assert torch.equal(was[x][kept], now[x][kept]), (x, lens)
            assert not torch.equal(was[x][~kept], now[x][~kept])
        c.close()


@pytest.mark.parametrize("L", [200, 3000])
def test_large_values_of_a_prompt(L):
    """Values of 1e37 on 20 slots whose score lies 2^7.9 above those before them: their
    average is finite, and so is every sum that leads to it."""
    c, q, off = setup((4, 1, 64, "bf16"), 16, [L], [64], False)
    c.k.zero_()
    c.v.zero_()
    q.zero_()
    q[:, :, 0] = 8.0
    for s in range(130, 150):
        blk = int(c.table_h[0, s // 16])
        c.k[blk, 0, s % 16, 0] = 7.9 * np.log(2.0)                # the score, 8 k / sqrt(64)
        c.v[blk, 0, s % 16] = 1e37
    r = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1, lse=True)
    assert bool(torch.isfinite(r["out"]).all()) and float(r["out"].float().min()) > 5e36 * min(1.0, 1000 / L)
    check(c, q, [64], r, rounded=True)
    c.close()


# ------------------------------------------------------------------- together
@pytest.mark.parametrize("heads", [(8, 2, 64, "bf16"), (32, 8, 128, "bf16"), (4, 1, 128, "f32")])
def test_a_cache_in_eight_bits_from_prompt_to_drafting(heads):
    """A prompt appended to the 8-bit cache and attended to, decoding steps over a
    window, drafts scored, and the cache read back: the attention over what was
    read back is the same."""
    lens = [0, 0, 0]
    c = Cache8(*heads, 16, lens, 12)
    counts = [90, 33, 1]
    off = torch.tensor([0, 90, 123, 124], dtype=torch.int32, device=DEV)
    width = (c.nq + 2 * c.nkv) * c.d
    total = [0, 0, 0]

    def held():
        """The oracle's copy of the caches: what they hold now."""
        c.codes_h = np.stack([values(c.k8), values(c.v8)])
        s = c.scales.cpu().numpy().astype(np.float64)
        with np.errstate(invalid="ignore"):
            c.exp_h = np.where(np.isnan(s), -999, np.log2(np.where(s > 0, s, 1.0)).astype(np.int64))

    for counts, window, n_first in (([90, 33, 1], 0, 0), ([1, 1, 1], 40, 4), ([1, 1, 1], 40, 4), ([6, 6, 6], 0, 0)):
        off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)
        q = c.dr.cache8_append(c.kv8(), c.normal((sum(counts), width), 1.5), offsets=off)
        r = c.dr.cache_attend_rows(c.kv8(), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        held()
        check(c, q, counts, r, True, window=window, n_first=n_first)
        total = [a + n for a, n in zip(total, counts)]
        c.n_lens = total
        c.lens.copy_(torch.tensor(total, dtype=torch.int32))
    c.dr.cache8_unpack(c.kv8(), c.kv())
    q = c.normal((3, c.nq, c.d), 2.0)
    a = c.dr.cache_attend_rows(c.kv8(), q, lse=True)
    b = c.dr.cache_attend_rows(c.kv(), q, lse=True)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])   # the same values, the same order
    d = c.dr.cache_attend(c.kv(), q, lse=True)
    assert float((d["out"].float() - b["out"].float()).abs().max()) <= 2.0 ** -7 * float(b["out"].float().abs().max())
    c.close()


def test_drafting_goes_on_over_a_cache_that_was_put_away():
    """A drafting batch's cache packed, its pools lost, read back: the chain drafts
    as over the same values."""
    from paper_2602_01762_amd import Drafter
    from synth import SMALL_BF16_CHAIN, make_inputs, make_weights
    cfg = SMALL_BF16_CHAIN.with_(batch=2, ctx_range=(20, 90), n_steps=3)
    inp = make_inputs(cfg, DEV)
    dr = Drafter(cfg)
    dr.load(make_weights(cfg, DEV))
    n = inp.k_pool.shape[0]
    k8, v8, scales = dr.cache8_buffers(n)
    kv8 = dr.cache8(inp.ctx_lens, k8, v8, scales, inp.block_table)
    kv = dr.cache(inp.ctx_lens, inp.k_pool, inp.v_pool, inp.block_table)
    dr.cache8_pack(kv8, dr.batch(inp))
    dr.cache8_unpack(kv8, kv)                               # what the codes stand for
    pools = inp.k_pool.clone(), inp.v_pool.clone()
    first = dr.chain(inp)["tokens"].clone()
    inp.k_pool.fill_(7.0)
    inp.v_pool.fill_(7.0)
    dr.cache8_unpack(kv8, kv)
    held = torch.zeros((n, cfg.kv_block_size), dtype=torch.bool, device=DEV)
    for b, L in enumerate(inp.ctx_lens.tolist()):
        for t in range(L):
            held[int(inp.block_table[b, t // cfg.kv_block_size]), t % cfg.kv_block_size] = True
    for p, was in zip((inp.k_pool, inp.v_pool), pools):
        assert torch.equal(p.transpose(1, 2)[held], was.transpose(1, 2)[held])
    assert torch.equal(dr.chain(inp)["tokens"], first)
    assert dr.device_status() == 0
    dr.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("counts", [[1, 1, 1], [3, 1, 6], [70, 2, 33]])
def test_replays_in_two_graphs_at_once(eight, counts):
    """One row each, drafts and prompts, captured twice with other windows, replayed
    together on two streams over growing lengths: the eager bits every time."""
    c, q, off = setup((8, 2, 64, "bf16"), 16, [0, 900, 333], counts, eight, columns=75)
    kv = sequences(c, eight)
    modes = [dict(), dict(window=100, n_first=4)]

    def call(kw):
        r = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True, **kw)
        return [r["out"], r["lse"]]

    eager = [call(kw) for kw in modes]
    assert all(torch.equal(x, y) for e, kw in zip(eager, modes) for x, y in zip(e, call(kw)))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for kw in modes:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(kw))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for step in range(5):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, kw in zip(outs, modes):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(o, call(kw))), step
        c.lens -= torch.tensor([0, 41, 7], dtype=torch.int32, device=DEV)
    c.close()


def test_rows_beyond_four_gigabytes():
    """Blocks at the end of pools of more than 2^32 bytes, both forms."""
    from test_gpu_cache import drafter
    nkv, d, bs = 8, 128, 16
    n = (1 << 32) // (nkv * d * bs) + 40
    dr = drafter(16, nkv, d, "bf16", bs, 1, 4)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    ids = [n - 1, n - 2, n - 7, n - 3]
    tab = torch.tensor([ids], dtype=torch.int32, device=DEV)
    lens = torch.tensor([50], dtype=torch.int32, device=DEV)
    k8, v8 = (torch.zeros((n, nkv, bs, d), dtype=torch.uint8, device=DEV).view(F8) for _ in range(2))
    scales = torch.ones((n, nkv, 2), device=DEV)
    small = [torch.randn((4, nkv, bs, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]
    near = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    kv8 = dr.cache8(lens, k8, v8, scales, tab)
    dr.cache8_pack(kv8, dr.cache(lens, *small, near))
    dr.cache8_unpack(kv8, dr.cache(lens, *small, near))
    for T in (1, 40):
        q = torch.randn((T, 16, d), generator=g, device=DEV).to(torch.bfloat16)
        off = torch.tensor([0, T], dtype=torch.int32, device=DEV)
        lens.fill_(50 - T)
        want = dr.cache_attend_rows(dr.cache(lens, *small, near), q, offsets=off, n_new=1)["out"]
        assert torch.equal(dr.cache_attend_rows(kv8, q, offsets=off, n_new=1)["out"], want)
        lens.fill_(50)
    del k8, v8, kv8
    big = [torch.zeros((n // 2 + 40, nkv, bs, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    m = big[0].shape[0]
    far = torch.tensor([[m - 1, m - 5, m - 2, m - 3]], dtype=torch.int32, device=DEV)
    for p, s in zip(big, small):
        p[far[0].long()] = s
    for T in (1, 40):
        q = torch.randn((T, 16, d), generator=g, device=DEV).to(torch.bfloat16)
        off = torch.tensor([0, T], dtype=torch.int32, device=DEV)
        lens.fill_(50 - T)
        want = dr.cache_attend_rows(dr.cache(lens, *small, near), q, offsets=off, n_new=1)["out"]
        assert torch.equal(dr.cache_attend_rows(dr.cache(lens, *big, far), q, offsets=off, n_new=1)["out"], want)
    assert dr.device_status() == 0
    dr.close()


# ------------------------------------------------------------- flags, refusals
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("counts", [[4, 4], [60, 50]])
def test_flags_what_it_cannot_read(eight, counts):
    lens = [100, 100]
    c, q, off = setup((8, 2, 64, "bf16"), 16, lens, counts, eight)
    kv = sequences(c, eight)
    kw = dict(offsets=off, n_new=1)
    ref = c.dr.cache_attend_rows(kv, q, **kw)["out"]
    assert c.dr.device_status() == 0
    cut = c.dr.cache_attend_rows(kv, q, max_len=64, **kw)           # longer than the bound: cut to it
    assert c.dr.device_status() == -7
    check(c, q, counts, cut, eight, max_len=64)
    table, table_h = (c.table8, c.table8_h) if eight else (c.table, c.table_h)
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        table[0, 3] = bad
        out = c.dr.cache_attend_rows(kv, q, **kw)["out"]
        assert c.dr.device_status() == -7
        assert torch.equal(out[counts[0]:], ref[counts[0]:]) and not torch.isnan(out.float()).any()
    table[0, 3] = int(table_h[0, 3])
    for L in (-5, -2 ** 31):
        c.lens[0] = L
        out = c.dr.cache_attend_rows(kv, q, **kw)["out"]
        assert c.dr.device_status() == -7
        assert float(out[: counts[0]].float().abs().max()) == 0.0 and torch.equal(out[counts[0]:], ref[counts[0]:])
    c.lens[0] = 2 ** 31 - 1                                         # cut at the capacity
    c.dr.cache_attend_rows(kv, q, **kw)
    assert c.dr.device_status() == -7
    c.lens[0] = 100
    for bad in ([0, 5, 4], [1, 4, 8], [0, 4, 10 ** 6], [-1, 4, 8]):
        out = torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
        c.dr.cache_attend_rows(kv, q, offsets=torch.tensor(bad, dtype=torch.int32, device=DEV), n_new=1, out=out)
        assert c.dr.device_status() == -1, bad
        assert bool((out == 7.0).all())
    c.close()


def test_refusals():
    from paper_2602_01762_amd import PrismError, binding as B
    import ctypes
    c = Cache8(8, 2, 64, "bf16", 16, [20, 20], 64)
    kv, q = c.kv(), c.normal((2, 8, 64))
    off = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    bad = [
        lambda: c.dr.cache_attend_rows(kv, c.normal((3, 8, 64))),              # 3 rows, no offsets
        lambda: c.dr.cache_attend_rows(kv, c.normal((0, 8, 64)), offsets=off),
        lambda: c.dr.cache_attend_rows(kv, q, max_len=1025),
        lambda: c.dr.cache_attend_rows(kv, q, max_len=-1),
        lambda: c.dr.cache_attend_rows(kv, q, n_new=-1),
        lambda: c.dr.cache_attend_rows(kv, q, window=-1),
        lambda: c.dr.cache_attend_rows(kv, q, window=5, n_first=-1),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(PrismError) as e:
            call()
        assert e.value.status == -1 and str(e.value), i
    out, scratch = torch.empty_like(q), torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    kv8 = c.kv8()
    io = B.prism_cache_row_attention()
    io.kv, io.rows, io.d_q, io.d_out = ctypes.addressof(kv), 2, B.ptr(q), B.ptr(out)
    io.d_scratch, io.scratch_bytes = B.ptr(scratch), B.prism_cache_rows_scratch(c.dr.ctx, 2, 2, 0)
    assert 0 < io.scratch_bytes <= 1 << 26
    B.prism_cache_attend_rows(c.dr.ctx, io)
    for field, value in (("scratch_bytes", 16), ("d_scratch", 0), ("d_q", 0), ("d_q", B.ptr(q) + 2),
                         ("d_out", B.ptr(out) + 8), ("kv", None), ("kv8", ctypes.addressof(kv8)), ("rows", 3)):
        keep = getattr(io, field)
        setattr(io, field, value)
        with pytest.raises(PrismError) as e:
            B.prism_cache_attend_rows(c.dr.ctx, io)
        assert e.value.status == -1, field
        setattr(io, field, keep)
    for args in ((0, 1, 0), (3, 1, 0), (1, 0, 0), (1, 1, 1025), (1, 1, -1)):
        with pytest.raises(PrismError):
            B.prism_cache_rows_scratch(c.dr.ctx, *args)
    io.rows, io.d_offsets = 2 ** 30, B.ptr(off)
    with pytest.raises(PrismError) as e:
        B.prism_cache_attend_rows(c.dr.ctx, io)
    assert e.value.status == -2
    assert c.dr.device_status() == 0
    c.close()
