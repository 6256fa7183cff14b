"""Attention of several rows on the GPU, each kernel held to its own precision, and
the prompts' kernel in the calls that rows_plan.py lists (test_rows_plan.py checks
that they reach it).

Tolerances as in test_gpu_attend_rows.py: u = 2^-24, a score is off by delta = (d + 4)
u max_t sum_c |q_c k_tc| / sqrt(d), a probability by the factor 1 + 2 delta, sums of n
terms by (min(n, 1024) + 64) u of their magnitudes, an output in bf16 by half a step, 2^-8.
Probabilities of prompts are rounded to bf16, half a step, 2^-8 of each product;
tiles of 32 columns take them as 8 bits cut off and the rest (below 2^-7) rounded to 8
bits, so 2^-7 2^-9 = 2^-16 of the probability at most; tiles of 16 columns as 24 bits.
"""
import ctypes

import numpy as np
import pytest
import torch

import rows_plan as R
from oracle import cache8 as C8
from test_gpu_attend_rows import pools, sequences, setup
from test_gpu_cache import U, f64
from test_gpu_cache8 import Cache8, values

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"


def some_rows(n):
    """The rows of a sequence that are compared: the ends, around tiles, and some."""
    return sorted({i for i in list(range(4)) + [15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 255, 256] + list(range(5, n, 23)) +
                   list(range(n - 3, n)) if 0 <= i < n})


def check(c, q, counts, r, eight=False, n_new=1, window=0, n_first=0, max_len=None, every=False):
    (kh, vh), table = pools(c, eight)
    qh, out = f64(q), f64(r["out"])
    lse = None if r["lse"] is None else r["lse"].cpu().numpy().astype(np.float64)
    bf = c.dt == torch.bfloat16
    p_ = R.plan((c.nq, c.nkv, c.d, "bf16" if bf else "f32"), len(counts), q.shape[0], max_len or c.bs * c.columns, window, n_first)
    r0 = 0
    for b, n in enumerate(counts):
        top = min(c.n_lens[b] + n_new + n - 1, max_len or 1 << 30)
        slots = np.arange(max(top, 0))
        parts = 0.0 if not bf else 2.0 ** -8 if R.is_prompt(p_, n) else 2.0 ** -16 if p_.cols == 32 else 0.0
        for j in range(c.nkv):
            K, V = kh[table[b, slots // c.bs], j, slots % c.bs], vh[table[b, slots // c.bs], j, slots % c.bs]
            for i in range(n) if every else some_rows(n):
                at, hs = r0 + i, slice(j * c.g, (j + 1) * c.g)
                want, p, want_lse, s = C8.attend_row(qh[at, hs], K, V, min(c.n_lens[b] + n_new + i, top), window, n_first)
                if len(s) == 0:
                    assert np.all(out[at, hs] == 0) and (lse is None or np.all(np.isneginf(lse[at, hs])))
                    continue
                delta = (c.d + 4) * U * (np.abs(qh[at, hs]) @ np.abs(K[s]).T).max(axis=1)[:, None] / np.sqrt(c.d)
                run = min(len(s), 1024) + 64
                lim = (2.0 ** -8 if bf else 0.0) * np.abs(want) + (2 * delta + run * U + parts) * (p @ np.abs(V[s]))
                e = np.abs(out[at, hs] - want)
                assert np.all(e <= lim), (b, j, i, float(np.max(e / lim)))
                if lse is not None:
                    e = np.abs(lse[at, hs] - want_lse)
                    assert np.all(e <= delta[:, 0] + run * U + 4 * U * (1 + np.abs(want_lse))), (b, j, i)
        r0 += n


def make(case, eight, **kw):
    heads, bs, lens, counts = case
    return setup(heads, bs, lens, counts, eight, columns=R.columns_of(bs, lens, counts), **kw)


# ------------------------------------------------------- tiles, at their own precision
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads,bs,lens,counts", [
    (R.SMALL, 1, [300, 0, 65, 511], [1, 70, 6, 40]), (R.SMALL, 12, [300, 0, 65, 511], [1, 70, 6, 40]),
    (R.SMALL, 256, [300, 0, 65, 511], [1, 70, 6, 40]), (R.MANY, 16, [3000, 100], [60, 50]), (R.NARROW, 7, [200, 30, 0], [9, 0, 33]),
    (R.SMALL, 16, [5000, 1023, 2048, 0], [3, 1, 6, 2]), (R.ODD, 16, [700, 3000, 1], [6, 12, 16]), (R.WIDE, 16, [700, 90], [33, 12]),
    ((4, 1, 128, "f32"), 16, [300, 0, 2000], [1, 70, 33]),
])
def test_rows_in_tiles(heads, bs, lens, counts, eight):
    """Probabilities in two parts or three, wherever no prompt is: their low parts
    are not lost."""
    c, q, off = make((heads, bs, lens, counts), eight)
    for window, n_first in ((0, 0), (90, 5)):
        assert not R.plan(heads, len(lens), sum(counts), bs * c.columns, window, n_first).prompt_segments
        r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        check(c, q, counts, r, eight, window=window, n_first=n_first)
    c.close()


# ------------------------------------------------------------------ prompts
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", R.BLOCKS)
def test_block_sizes(case, eight):
    c, q, off = make(case, eight, pad=3)
    for window, n_first in R.BLOCK_WINDOWS:
        out = torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
        r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True, out=out)
        assert bool((out[sum(case[3]):] == 7.0).all())
        check(c, q, case[3], r, eight, window=window, n_first=n_first)
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", R.SPLIT)
def test_windows_split_over_their_length(case, eight):
    c, q, off = make(case, eight)
    for window, n_first in R.SPLIT_WINDOWS:
        r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        check(c, q, case[3], r, eight, window=window, n_first=n_first)
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", R.NEW)
def test_numbers_of_new_rows(case, eight):
    """Rows that see the slots before them only (the first of an empty sequence sees
    nothing), and rows with others in the cache behind them."""
    heads, bs, lens, counts = case
    c, q, off = setup(heads, bs, lens, [n + 9 for n in counts], eight)
    q = q[: sum(counts)].contiguous()
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)
    for n_new in (0, 2, 9):
        for window, n_first in ((0, 0), (30, 2)):
            kw = dict(n_new=n_new, window=window, n_first=n_first)
            check(c, q, counts, c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, lse=True, **kw), eight, **kw)
    c.close()


@pytest.mark.parametrize("case", R.CROWD)
def test_many_sequences(case):
    c, q, off = make(case, True)
    for window, n_first in ((0, 0), (200, 3)):
        r = c.dr.cache_attend_rows(c.kv8(), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        check(c, q, case[3], r, True, window=window, n_first=n_first)
    c.close()


@pytest.mark.parametrize("n", [1, 5, 20])
@pytest.mark.parametrize("case", R.LONG)
def test_the_end_of_the_largest_capacity(case, n):
    """Slots up to 2^20, in blocks of 7: by tiles and as a prompt."""
    heads, bs, lens, (most,) = case
    c, q, off = make(case, False)
    q, off = q[:n].contiguous(), torch.tensor([0, n], dtype=torch.int32, device=DEV)
    for window, n_first in ((0, 0), (9000, 5)):
        r = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1 + most - n, window=window, n_first=n_first, lse=True)
        check(c, q, [n], r, n_new=1 + most - n, window=window, n_first=n_first)
    c.close()


# slots, and whether some row sees none of them: among the first ones that every row
# sees too; that only the first rows still see; that only later rows see
BAD = [({0: [101, 63, 2, 103], 1: [32, 33, 1]}, False), ({0: [63, 62], 1: [32, 33]}, True), ({0: [101, 103], 1: [60, 61]}, True)]
ODD_VALUES = [float("nan"), float("inf"), float("-inf"), float("nan")]


def spoil(c, eight, which, bad):
    """What is not finite at the bad slots of the first KV head, in the keys' or
    values' pool or both: channel 5 + x of the x-th slot."""
    table = c.table8_h if eight else c.table_h
    for b in range(c.B):
        for x, s in enumerate(bad[b]):
            blk = int(table[b, s // c.bs])
            for w in which:
                if eight:
                    (c.k8, c.v8)[w].view(torch.uint8)[blk, 0, s % c.bs, 5 + x] = 0x7f if x % 2 else 0xff
                else:
                    (c.k, c.v)[w][blk, 0, s % c.bs, 5 + x] = ODD_VALUES[x]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("bad,hidden", BAD)
@pytest.mark.parametrize("case", R.HIDDEN + R.HIDDEN_TILES)
def test_what_a_row_does_not_see_does_not_reach_it(case, bad, hidden, eight):
    """Rows that do not see them: the bits of a cache without them.  Rows that see a
    value that is not finite: that in its channel, the same bits in the others."""
    _, bs, lens, counts = case
    window, n_first = R.HIDDEN_WINDOW
    kw = dict(n_new=1, window=window, n_first=n_first, lse=True)
    c, q, off = make(case, eight)
    clean = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, **kw)
    for what in ((1,), (0, 1)):                             # values, then keys too
        spoil(c, eight, what, bad)
        r = c.dr.cache_attend_rows(sequences(c, eight), q, offsets=off, **kw)
        got, want = r["out"].float().cpu(), clean["out"].float().cpu()
        assert torch.equal(got[:, c.g:], want[:, c.g:])     # other KV heads
        r0 = touched = 0
        for b, n in enumerate(counts):
            for i in range(n):
                seen = [x for x, s in enumerate(bad[b]) if s in C8.seen_slots(lens[b] + 1 + i, window, n_first)]
                y, z = got[r0 + i, : c.g], want[r0 + i, : c.g]
                if not seen:
                    assert torch.equal(y, z), (b, i)
                    assert torch.equal(r["lse"][r0 + i], clean["lse"][r0 + i]), (b, i)
                elif 0 in what:
                    assert not bool(torch.isfinite(y).all())
                else:
                    z = z.clone()
                    for x in seen:
                        z[:, 5 + x] = float("nan") if eight else ODD_VALUES[x]
                    assert np.array_equal(y.numpy(), z.numpy(), equal_nan=True), (b, i, seen)
                touched += bool(seen)
            r0 += n
        assert touched and (touched < r0) == hidden
    c.close()


@pytest.mark.parametrize("case", R.INFINITE)
def test_scores_that_are_infinite(case):
    """-inf scores take no part; a row of nothing else gives zeros."""
    c, q, off = make(case, False)
    n = case[3][0]
    q = q.abs() + 0.5
    c.k[[int(x) for x in c.table_h[0]], 0] = float("-inf")
    for s in range(3, 80 + n):
        c.k[int(c.table_h[1, s // 16]), 0, s % 16] = float("-inf")
    r = c.dr.cache_attend_rows(c.kv(), q, offsets=off, n_new=1, lse=True)
    assert float(r["out"][:n, :2].abs().max()) == 0.0 and bool(torch.isneginf(r["lse"][:n, :2]).all())
    assert bool(torch.isfinite(r["out"]).all())
    K, V = (c.rows(f64(p), 1, 0, np.arange(3)) for p in (c.k, c.v))
    qh, out = f64(q), f64(r["out"])
    for i in range(n):
        want, p, _, _ = C8.attend_row(qh[n + i, :2], K, V, 3, 0, 0)
        delta = (c.d + 4) * U * (np.abs(qh[n + i, :2]) @ np.abs(K).T).max() / np.sqrt(c.d)
        # half a step of the probabilities and of the output, and of 3 slots (3 + 64) u
        lim = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * delta + 67 * U) * (p @ np.abs(V))
        assert np.all(np.abs(out[n + i, :2] - want) <= lim), i
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", R.FLAGS)
def test_flags_what_it_cannot_read(case, eight):
    counts = case[3]
    c, q, off = make(case, eight)
    kv = sequences(c, eight)
    kw = dict(offsets=off, n_new=1)
    ref = c.dr.cache_attend_rows(kv, q, **kw)["out"]
    assert c.dr.device_status() == 0
    cut = c.dr.cache_attend_rows(kv, q, max_len=64, lse=True, **kw)     # longer than the bound: cut to it
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
    B, T = len(counts), q.shape[0]
    for bad in ([0, T + 1, T][: B + 1], [1, T, T][: B + 1], [0] + [T] * (B - 1) + [10 ** 6], [-1, T, T][: B + 1]):
        out = torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
        c.dr.cache_attend_rows(kv, q, offsets=torch.tensor(bad, dtype=torch.int32, device=DEV), n_new=1, out=out)
        assert c.dr.device_status() == -1, bad
        assert bool((out == 7.0).all())
    c.close()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", R.GRAPHS)
def test_replays_in_two_graphs_at_once(case, eight):
    """Captured with two windows, replayed together on two streams over shorter and
    shorter lengths, with eager calls between: the eager bits every time."""
    c, q, off = make(case, eight)
    kv = sequences(c, eight)

    def call(window, n_first):
        r = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True, window=window, n_first=n_first)
        return [r["out"], r["lse"]]

    for w in R.GRAPH_WINDOWS:
        call(*w)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for w in R.GRAPH_WINDOWS:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(*w))
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
        for o, w in zip(outs, R.GRAPH_WINDOWS):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(o, call(*w))), step
        c.lens -= torch.tensor([0, 41, 7] if len(case[2]) == 3 else [37], dtype=torch.int32, device=DEV)
    c.close()


@pytest.mark.parametrize("case", R.EIGHT)
def test_a_prompt_appended_in_eight_bits_and_attended_to(case):
    _, bs, lens, counts = case
    c = Cache8(*case[0], bs, lens, R.columns_of(bs, lens, counts))
    off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)
    for window, n_first in ((0, 0), (40, 4)):
        q = c.dr.cache8_append(c.kv8(), c.normal((sum(counts), (c.nq + 2 * c.nkv) * c.d), 1.5), offsets=off)
        r = c.dr.cache_attend_rows(c.kv8(), q, offsets=off, n_new=1, window=window, n_first=n_first, lse=True)
        c.codes_h = np.stack([values(c.k8), values(c.v8)])
        s = c.scales.cpu().numpy().astype(np.float64)
        with np.errstate(invalid="ignore"):
            c.exp_h = np.where(np.isnan(s), -999, np.log2(np.where(s > 0, s, 1.0)).astype(np.int64))
        check(c, q, counts, r, True, window=window, n_first=n_first)
    c.close()


# ------------------------------------------------- streams and scratch
def on_side(fill, call):
    """call() on a stream of its own, behind work that keeps that stream busy and then
    writes the call's input: a launch on another stream would not wait for it."""
    side = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):                                  # a few ms
            busy = busy @ busy * 1e-2
        fill()
        r = call()
    side.synchronize()
    torch.cuda.synchronize()
    return r


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("case", R.STREAMS + [(R.SMALL, 16, [700, 90], [1, 1]), (R.SMALL, 16, [700, 90], [7, 3])])
def test_attention_waits_for_its_stream(case, eight):
    c, q, off = make(case, eight)
    kv, src = sequences(c, eight), q.clone()
    want = c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True)
    q.zero_()
    got = on_side(lambda: q.copy_(src), lambda: c.dr.cache_attend_rows(kv, q, offsets=off, n_new=1, lse=True))
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    c.close()


def test_the_8_bit_cache_waits_for_its_stream():
    a, b = (Cache8(8, 2, 64, "bf16", 16, [0, 70, 33], 8, seed=3) for _ in range(2))
    rows = a.normal((3, 12 * 64), 2.0)
    start = torch.tensor([0, 5, 33], dtype=torch.int32, device=DEV)
    off = torch.arange(4, dtype=torch.int32, device=DEV)

    def step(c, qkv):
        q = c.dr.cache8_append(c.kv8(), qkv, offsets=off)
        c.dr.cache8_unpack(c.kv8(), c.kv(), start=start, n_new=1)
        c.dr.cache8_pack(c.kv8(), c.kv(), start=start, n_new=1)
        return q

    want = step(a, rows)
    src = torch.zeros_like(rows)
    got = on_side(lambda: src.copy_(rows), lambda: step(b, src))
    assert torch.equal(got, want)
    for x, y in ((a.k, b.k), (a.v, b.v), (a.k8, b.k8), (a.v8, b.v8), (a.scales, b.scales)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    a.close()
    b.close()


def test_nothing_is_written_behind_the_scratch():
    """Sized for the largest call, for each batch, and to the byte that a call asks for."""
    from paper_2602_01762_amd import binding as B
    heads, bs, lens, counts = R.SCRATCH
    c, q, off = make(R.SCRATCH, False)
    most = B.prism_cache_rows_scratch(c.dr.ctx, 4, sum(counts), 0)
    for nb in (4, 3, 2, 1):
        kv = c.dr.cache(c.lens[:nb], c.k, c.v, c.table[:nb])
        T = sum(counts[:nb])
        for n in {most, B.prism_cache_rows_scratch(c.dr.ctx, nb, T, 0)}:
            for window, n_first in ((0, 0), (600, 3)):
                out = torch.empty((T, c.nq, c.d), dtype=c.dt, device=DEV)
                scratch = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
                io = B.prism_cache_row_attention()
                io.kv, io.rows, io.d_offsets, io.n_new = ctypes.addressof(kv), T, B.ptr(off), 1
                io.window, io.n_first, io.d_q, io.d_out = window, n_first, B.ptr(q), B.ptr(out)
                io.d_scratch, io.scratch_bytes = B.ptr(scratch), n
                B.prism_cache_attend_rows(c.dr.ctx, io)
                assert bool((scratch[n:] == 0xa5).all())
                want = c.dr.cache_attend_rows(kv, q[:T], offsets=off[: nb + 1], n_new=1, window=window, n_first=n_first)
                assert torch.equal(out, want["out"])
    c.close()
