"""The plan that the runtime makes for an attention of rows (csrc/cache_plan.h,
compiled for the host), and the calls that the tests of the prompts' kernel make:
their plans are checked without a GPU, so that no limit of the dispatch can move
them to the other kernel unnoticed."""
import ctypes
import functools
import os
import subprocess
import tempfile
import types

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_01762_amd", "csrc")

_CODE = r"""
#include "plan.h"
extern "C" void plan(int bf16, int nkv, int g, int d, int batch, int rows, int one_each, int max_len, int window,
                     int n_first, int *out) {
  using namespace prism;
  const RowsPlan p = rows_plan(bf16, nkv, g, d, batch, rows, one_each, max_len, window, n_first,
                               cache_waves(d * (bf16 ? 2 : 4)));
  const int v[] = {p.cols, p.few, p.segments, p.direct, p.prompt_segments, p.splits};
  for (int i = 0; i < 6; ++i) out[i] = v[i];
}
"""


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "p.cc"), os.path.join(d, "p.so")
        with open(src, "w") as f:
            f.write(_CODE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
        return ctypes.CDLL(lib)


def plan(heads, batch, rows, max_len, window=0, n_first=0, one_each=False):
    """cols, few, segments, direct, prompt_segments, splits of a call over max_len
    slots at most."""
    nq, nkv, d, dtype = heads
    out = (ctypes.c_int * 6)()
    _lib().plan(dtype == "bf16", nkv, nq // nkv, d, batch, rows, one_each, max_len, window, n_first, out)
    return types.SimpleNamespace(**dict(zip(("cols", "few", "segments", "direct", "prompt_segments", "splits"), out)))


def is_prompt(p, n):
    """Whether a sequence of n rows goes by the prompts' kernel."""
    return p.prompt_segments > 0 and (n > p.few or not p.segments)


def columns_of(bs, lens, counts):
    """Table columns that hold the rows too."""
    return max(1, -(-max(L + n for L, n in zip(lens, counts)) // bs))


NARROW, SMALL, ODD, ONE, WIDE, MANY = ((7, 1, 32, "bf16"), (8, 2, 64, "bf16"), (6, 2, 128, "bf16"), (3, 3, 128, "bf16"),
                                       (4, 1, 256, "bf16"), (8, 8, 128, "bf16"))
# heads, block size, lengths, rows, windows
BLOCKS = [(SMALL, bs, [300, 0, 65, 511], [1, 220, 6, 40]) for bs in (1, 7, 12, 64, 256)] + \
         [(heads, bs, [333], [70]) for heads, bs in ((SMALL, 1), (NARROW, 7), (ONE, 12), (WIDE, 7), (WIDE, 100), (ODD, 48))] + \
         [(ONE, 7, [40, 0, 5], [1030, 1, 49])]
BLOCK_WINDOWS = [(0, 0), (90, 5)]
# a window and splits
SPLIT = [(SMALL, 16, [5000], [40]), (MANY, 16, [5000], [90]), (ONE, 12, [5000], [70]), (WIDE, 16, [3000], [33]),
         (SMALL, 16, [5000, 1023], [300, 5]), (NARROW, 16, [3000, 0, 7], [150, 1, 30])]
SPLIT_WINDOWS = [(0, 0), (700, 4), (2100, 0), (513, 300)]
# slots that some rows see and others do not, under a window of 40 and 3 first ones
HIDDEN = [(SMALL, 16, [100, 30], [250, 60]), (SMALL, 12, [100], [90]), (WIDE, 16, [100, 30], [250, 60]), (MANY, 16, [100], [90]),
          ((4, 2, 32, "bf16"), 16, [100, 30], [420, 120]), (NARROW, 7, [100], [40])]
HIDDEN_WINDOW = (40, 3)
# the same in tiles of 16 and 32 columns
HIDDEN_TILES = [((8, 2, 64, "f32"), 16, [100, 30], [6, 60]), (SMALL, 16, [100, 30], [6, 60]), (WIDE, 7, [100, 30], [9, 60]),
                (MANY, 16, [100, 30], [33, 60]), ((4, 2, 32, "bf16"), 16, [100, 30], [5, 60])]
FLAGS = [(SMALL, 16, [100, 100], [260, 50]), (SMALL, 16, [100], [90])]
GRAPHS = [(SMALL, 16, [0, 900, 333], [270, 2, 33]), (SMALL, 16, [3000], [130]), (MANY, 16, [900], [70])]
GRAPH_WINDOWS = [(0, 0), (100, 4)]
INFINITE = [((4, 2, 64, "bf16"), 16, [80, 80], [300, 300])]
STREAMS = [(SMALL, 16, [700, 90], [260, 40]), (SMALL, 16, [3000], [100])]
EIGHT = [(SMALL, 16, [0, 0, 0], [300, 33, 1])]
# other numbers of new rows; many sequences; the end of the largest capacity, 2^20 slots
NEW = [(SMALL, 16, [0, 100], [200, 90]), ((5, 1, 128, "bf16"), 16, [60], [70]), ((8, 1, 64, "bf16"), 16, [0, 3], [130, 20])]
CROWD = [((6, 2, 32, "bf16"), 16, [(b * 131) % 500 for b in range(64)], [(b * 7) % 40 for b in range(64)])]
LONG = [(NARROW, 7, [2 ** 20 - 44], [20])]
# a batch that needs the scratch of both kernels
SCRATCH = (SMALL, 16, [900, 40, 1500, 700], [60, 1, 9, 230])
