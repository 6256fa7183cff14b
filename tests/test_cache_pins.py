"""Pins of the cache oracle (CPU): facts that follow from the definitions, and
the argument checks and launch plans of the cache calls that need no GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import softmax_attend, rope
from oracle import cache as C
from paper_2602_01762_amd import binding as B
from paper_2602_01762_amd.drafter import Drafter

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attend_is_the_softmax_average_of_each_head():
    rng = np.random.default_rng(0)
    q, K, V = rng.normal(size=(3, 8)), rng.normal(size=(21, 8)), rng.normal(size=(21, 8))
    out, p, lse = C.attend(q, K, V)
    for h in range(3):
        assert np.allclose(out[h], softmax_attend(q[h], K, V), atol=1e-14)
    assert np.allclose(p.sum(axis=1), 1.0)
    assert np.allclose(lse, np.log(np.exp(q @ K.T / np.sqrt(8)).sum(axis=1)))
    # two halves joined by their log-sums
    a, b = C.attend(q, K[:9], V[:9]), C.attend(q, K[9:], V[9:])
    w = 1.0 / (1.0 + np.exp(b[2] - a[2]))[:, None]
    assert np.allclose(out, w * a[0] + (1 - w) * b[0])


def test_append_normalises_then_rotates():
    rng = np.random.default_rng(1)
    x, g = rng.normal(size=(4, 8)), 1 + 0.1 * rng.normal(size=8)
    q, k, v = C.append_row(x, 2, 1, 0, 1e4, 0.0, g, None)
    assert np.allclose(np.sqrt(np.mean((q / g) ** 2, axis=-1)), 1.0)      # position 0 does not rotate
    assert np.allclose(k, x[2:3]) and np.array_equal(v, x[3:4])
    q7, _, _ = C.append_row(x, 2, 1, 7, 1e4, 0.0, g, None)
    assert np.allclose(q7, rope(q, 7, 1e4))
    assert np.allclose((q7 ** 2).sum(-1), (q ** 2).sum(-1))               # a rotation keeps the norm


def test_a_block_score_bounds_its_keys():
    rng = np.random.default_rng(2)
    q, K = rng.normal(size=(4, 16)), rng.normal(size=(50, 16))
    s = C.block_scores(q, C.summarize(K, 8))
    for i in range(len(s)):
        assert s[i] >= (q @ K[8 * i: 8 * i + 8].T).max() - 1e-6
    one = C.block_scores(q, C.summarize(K, 1))                            # one key per block: exact
    assert np.allclose(one, (q @ K.T).max(axis=0), atol=1e-5)


def test_choice_order():
    v = np.array([1.0, 3.0, np.nan, 3.0, -np.inf, 2.0, np.inf])
    assert C.choose(v, 1, 0, 0).tolist() == [6]
    assert C.choose(v, 2, 0, 0).tolist() == [1, 6]                        # the tie goes to 1
    assert C.choose(v, 3, 1, 1).tolist() == [0, 1, 6]
    assert C.choose(v, 6, 0, 0).tolist() == [0, 1, 3, 4, 5, 6]            # NaN last
    assert C.choose(v, 9, 0, 0).tolist() == list(range(7))


# ---- argument checks of the wrapper (nothing reaches the library)
def _fake():
    dr = object.__new__(Drafter)
    dr.ctx = None
    dr.device = torch.device("cpu")
    dr.cfg = B.prism_config(n_q_heads=4, n_kv_heads=2, head_dim=32, kv_block_size=16,
                            max_blocks_per_seq=5, max_batch=3, dtype=B.PRISM_BF16)
    dr._cache_setup()
    return dr


def _kv(dr, **kw):
    t = dict(lens=torch.zeros(3, dtype=torch.int32), k_pool=torch.zeros(9, 2, 16, 32, dtype=torch.bfloat16),
             v_pool=torch.zeros(9, 2, 16, 32, dtype=torch.bfloat16),
             block_table=torch.zeros(3, 5, dtype=torch.int32))
    t.update(kw)
    return dr.cache(**t)


@pytest.mark.parametrize("kw,err", [
    (dict(lens=torch.zeros(3)), TypeError),
    (dict(lens=torch.zeros(2, dtype=torch.int32)), ValueError),           # table of 3 sequences
    (dict(k_pool=torch.zeros(9, 2, 16, 32)), TypeError),
    (dict(v_pool=torch.zeros(8, 2, 16, 32, dtype=torch.bfloat16)), ValueError),
    (dict(k_pool=torch.zeros(9, 16, 2, 32, dtype=torch.bfloat16).transpose(1, 2)), ValueError),
    (dict(block_table=torch.zeros(3, 4, dtype=torch.int32)), ValueError),
    (dict(block_table=torch.zeros(3, 5, dtype=torch.int64)), TypeError),
])
def test_cache_refuses_other_tensors(kw, err):
    with pytest.raises(err):
        _kv(_fake(), **kw)


def test_calls_refuse_other_tensors():
    dr = _fake()
    kv = _kv(dr)
    bf = dict(dtype=torch.bfloat16)
    q, w = torch.zeros(3, 4, 32, **bf), torch.zeros(9, 2, 16)
    summ, new = torch.zeros(9, 2, 2, 32, **bf), torch.zeros(3, 5, dtype=torch.int32)
    bad = [
        (TypeError, lambda: dr.cache_append(kv, torch.zeros(3, 256))),
        (ValueError, lambda: dr.cache_append(kv, torch.zeros(3, 255, **bf))),
        (ValueError, lambda: dr.cache_append(kv, torch.zeros(3, 512, **bf)[:, ::2])),
        (ValueError, lambda: dr.cache_append(kv, torch.zeros(3, 256, **bf), q_gain=torch.zeros(31, **bf))),
        (ValueError, lambda: dr.cache_append(kv, torch.zeros(3, 256, **bf), offsets=torch.zeros(3, dtype=torch.int32))),
        (TypeError, lambda: dr.cache_append(kv, torch.zeros(3, 256, **bf), weights=w.double())),
        (ValueError, lambda: dr.cache_attend(kv, q[:2])),
        (ValueError, lambda: dr.cache_attend(kv, q, weights=w[:8])),
        (TypeError, lambda: dr.cache_attend(kv, q, blocks=torch.zeros(3, 2, 4))),
        (ValueError, lambda: dr.cache_attend(kv, q, blocks=torch.zeros(3, 1, 4, dtype=torch.int32))),
        (ValueError, lambda: dr.cache_attend(kv, q, blocks=torch.zeros(3, 2, 0, dtype=torch.int32))),
        (ValueError, lambda: dr.cache_attend(kv, q, out=q.transpose(0, 1).contiguous())),
        (ValueError, lambda: dr.cache_summarize(kv, summ[:, :1])),
        (TypeError, lambda: dr.cache_select(kv, q, summ.float(), 2)),
        (ValueError, lambda: dr.cache_select(kv, q, summ, 2, out=torch.zeros(3, 2, 3, dtype=torch.int32))),
        (ValueError, lambda: dr.cache_evict(kv, new[:, :4], w, 8)),
        (TypeError, lambda: dr.cache_evict(kv, new, w.to(torch.bfloat16), 8)),
        (TypeError, lambda: dr.cache_evict(kv, new, None, 8)),
    ]
    for err, call in bad:
        with pytest.raises(err):
            call()


def test_struct_layouts(tmp_path):
    """The binding's structs of the cache calls have the header's layout."""
    structs = ("prism_cache_rows", "prism_cache_attention", "prism_cache_selection", "prism_cache_eviction")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "prism_draft.h"', "int main(void) {"]
    for st in structs:
        lines.append('  printf("%s %%zu\\n", sizeof(%s));' % (st, st))
        for f, _ in getattr(B, st)._fields_:
            lines.append('  printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (st, f, st, f))
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;\n}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    ref = dict(ln.split() for ln in out.splitlines())
    for st in structs:
        cls = getattr(B, st)
        assert ctypes.sizeof(cls) == int(ref[st])
        for f, _ in cls._fields_:
            assert getattr(cls, f).offset == int(ref["%s.%s" % (st, f)])


@pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")
def test_null_context_is_refused():
    L = B.lib()
    n = ctypes.c_uint64()
    assert L.prism_cache_scratch(None, 0, 1, 0, ctypes.byref(n)) == -1
    assert L.prism_cache_append(None, None, None) == -1
    assert L.prism_cache_attend(None, None, None) == -1
    assert L.prism_cache_summarize(None, None, 0, 0, None, None) == -1
    assert L.prism_cache_select(None, None, None) == -1
    assert L.prism_cache_evict(None, None, None) == -1


def test_attention_runs_cover_every_granule(tmp_path):
    """The runs that a plan's waves take over random lengths: every granule of
    every (sequence, KV head) once, each (wave, segment) its own partial below
    waves + segments, and a segment's partials next to each other, where the
    join looks for them."""
    src, exe = tmp_path / "plan.cc", tmp_path / "plan"
    src.write_text(r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "plan.h"
using namespace prism;
int main() {
  srand(1);
  for (int it = 0; it < 4000; ++it) {
    const int B = 1 + rand() % 64, nkv = 1 + rand() % 8, top = 1 << (rand() % 18);
    std::vector<int> len(B);
    int span = 1;
    for (int &n : len) { n = rand() % 3 ? rand() % (top + 1) : 0; span = n > span ? n : span; }
    const bool weights = rand() % 2;
    const CachePlan p = cache_plan(B * nkv, span, weights);
    if (p.waves < 1 || p.waves > (p.direct ? B * nkv : CACHE_WAVES)) return 1;
    if (p.direct && (span > (B * nkv >= CACHE_DIRECT_UNITS ? CACHE_DIRECT_MANY : CACHE_DIRECT) || weights)) return 2;
    std::vector<long> begin(B), count(B);
    long total = 0;
    for (int b = 0; b < B; ++b) {
      count[b] = p.direct ? 1 : (len[b] + CACHE_GRAN - 1) / CACHE_GRAN;
      begin[b] = total;
      total += count[b] * nkv;
    }
    long per = (total + p.waves - 1) / p.waves;
    if (per < 1) per = 1;
    std::vector<int> owner(p.waves + (long)B * nkv, -1), seen(total, 0);
    for (long w = 0; w < p.waves; ++w) {
      long u = w * per, last = u + per < total ? u + per : total;
      while (u < last) {
        int b = 0;
        while (begin[b] + count[b] * nkv <= u) ++b;
        const long j = (u - begin[b]) / count[b], first = u - begin[b] - j * count[b];
        long m = count[b] - first;
        if (m > last - u) m = last - u;
        for (long i = 0; i < m; ++i) ++seen[u + i];
        const long part = w + (long)b * nkv + j, g0 = begin[b] + j * count[b];
        if (part >= (long)owner.size() || owner[part] != -1) return 3;
        owner[part] = b * nkv + (int)j;
        const long w0 = g0 / per, w1 = (g0 + count[b] - 1) / per;   // the join's range
        if (w < w0 || w > w1) return 4;
        u += m;
      }
    }
    for (int s : seen) if (s != 1) return 5;
    for (int b = 0; b < B; ++b)
      for (int j = 0; j < nkv && count[b]; ++j) {
        const long g0 = begin[b] + j * count[b];
        for (long w = g0 / per; w <= (g0 + count[b] - 1) / per; ++w)
          if (owner[w + (long)b * nkv + j] != b * nkv + j) return 6;
      }
  }
  return 0;
}
""")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2602_01762_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_scratch_of_a_batch_serves_every_smaller_one(tmp_path):
    """Some larger batches need none where smaller ones do (and the size for a
    batch that needs none alone is not 0 then)."""
    src, exe = tmp_path / "scratch.cc", tmp_path / "scratch"
    src.write_text(r"""
#include "plan.h"
using namespace prism;
int main() {
  const int spans[] = {1, 64, 511, 512, 513, 700, 1000, 1023, 1024, 1025, 4096, 131072};
  const int nkvs[] = {1, 2, 5, 8, 32}, gs[] = {1, 4, 8}, ds[] = {32, 256};
  int grows = 0;
  for (int span : spans)
    for (int nkv : nkvs)
      for (int g : gs)
        for (int d : ds)
          for (int weights = 0; weights < 2; ++weights) {
            size_t most = 0;
            for (int b = 1; b <= 64; ++b) {
              const size_t need = cache_attend_scratch(b, nkv, g, d, span, weights);
              const size_t size = cache_attend_scratch_up_to(b, nkv, g, d, span, weights);
              most = need > most ? need : most;
              if (size != most) return 1;
              grows += need < size;
              if (span <= 512 && !weights && size) return 2;
            }
          }
  return grows ? 0 : 3;
}
""")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2602_01762_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_attention_runs_by_the_functions_that_the_kernels_call(tmp_path):
    """Over random lengths, with plan.h's own numbering: every granule is one
    run's, no two runs share a partial, all lie inside the scratch, and the
    join's range of a segment holds its partials, in order and no others."""
    src, exe = tmp_path / "runs.cc", tmp_path / "runs"
    src.write_text(r"""
#include <cstdlib>
#include <vector>
#include "plan.h"
using namespace prism;
int main() {
  srand(2);
  for (int it = 0; it < 4000; ++it) {
    const int B = 1 + rand() % 64, nkv = 1 + rand() % 8, top = 1 << (rand() % 18), g = 1 + rand() % 8, d = 32 << (rand() % 4);
    std::vector<int> len(B);
    int span = 1;
    for (int &n : len) { n = rand() % 3 ? rand() % (top + 1) : 0; span = n > span ? n : span; }
    const bool weights = rand() % 2;
    const int waves = cache_waves(d * (rand() % 2 ? 4 : 2));
    const CachePlan p = cache_plan(B * nkv, span, weights, waves);
    if (p.waves > (p.direct ? B * nkv : waves)) return 9;
    std::vector<int> begin(B), count(B);
    int total = 0;
    for (int b = 0; b < B; ++b) {
      count[b] = p.direct ? 1 : cache_granules(len[b]);
      begin[b] = total;
      total += count[b] * nkv;
    }
    const int run = cache_run(total, p.waves);
    if ((long)run * p.waves < total) return 1;
    std::vector<int> owner(cache_partials(p.waves, B * nkv), -1), seen(total, 0);
    const size_t bytes = cache_attend_scratch(B, nkv, g, d, span, weights, waves);
    if (p.direct ? bytes : bytes < owner.size() * g * (d + 2) * 4 + (weights ? (size_t)B * nkv * g * span * 4 : 0)) return 2;
    for (int w = 0; w < p.waves; ++w) {
      int u = w * run;
      const int last = u + run < total ? u + run : total;
      while (u < last) {
        int b = 0;
        while (begin[b] + count[b] * nkv <= u) ++b;
        const CacheRun r = cache_run_at(u - begin[b], count[b], last - u);
        if (r.granules < 1 || r.head >= nkv) return 3;
        for (int i = 0; i < r.granules; ++i) {
          if (begin[b] + r.head * count[b] + r.first + i != u + i) return 4;
          ++seen[u + i];
        }
        const int part = cache_partial(w, b * nkv + r.head);
        if (part >= (int)owner.size() || owner[part] != -1) return 5;
        owner[part] = b * nkv + r.head;
        u += r.granules;
      }
    }
    for (int s : seen) if (s != 1) return 6;
    int joined = 0;
    for (int b = 0; b < B; ++b)
      for (int j = 0; j < nkv; ++j) {
        const CacheParts c = cache_parts(begin[b] + j * count[b], count[b], run);
        for (int i = 0; i < c.n; ++i, ++joined)
          if (owner[cache_partial(c.wave, b * nkv + j) + i] != b * nkv + j) return 7;
      }
    for (int o : owner) joined -= o >= 0;
    if (joined) return 8;
  }
  return 0;
}
""")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2602_01762_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
