"""Pins of the oracle of the 8-bit cache and of the attention of several rows (CPU),
and what their calls refuse and plan without a GPU."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import cache8 as C8
from paper_2602_01762_amd import binding as B
from paper_2602_01762_amd.drafter import Drafter

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_01762_amd", "csrc")
F8 = torch.float8_e4m3fn


def test_code_values():
    t = C8.e4m3_table()
    assert t[0x7e] == 448.0 and t[0x08] == 2.0 ** -6 and t[0x01] == 2.0 ** -9 and t[0xc0] == -2.0
    assert np.isnan(t[0x7f]) and np.isnan(t[0xff])
    want = torch.arange(256, dtype=torch.uint8).view(F8).double().numpy()
    assert np.array_equal(t, want, equal_nan=True)


def test_rounding_to_codes():
    t = C8.e4m3_table()[:127]
    assert np.array_equal(C8.e4m3_round(t), t) and np.array_equal(C8.e4m3_round(-t), -t)
    mid = (t[1:] + t[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, t[:-1], t[1:])
    assert np.array_equal(C8.e4m3_round(mid), even)                 # ties to the even code
    assert np.array_equal(C8.e4m3_round(mid * (1 + 1e-12)), t[1:])
    assert np.array_equal(C8.e4m3_round(mid * (1 - 1e-12)), t[:-1])
    x = np.random.default_rng(0).normal(size=4000) * 100
    assert np.array_equal(C8.e4m3_round(x.astype(np.float32).astype(np.float64)),
                          torch.tensor(x, dtype=torch.float32).to(F8).double().numpy())
    assert C8.e4m3_round(np.array([460.0, -1e9])).tolist() == [448.0, -448.0]
    assert np.isnan(C8.e4m3_round(np.array([np.inf, np.nan]))).all()


def test_scales_are_the_least_that_hold_a_block():
    for top, e in ((448.0, 0), (448.0 * (1 + 2e-16), 1), (449.0, 1), (224.0, -1), (1.75, -8), (1.76, -7),
                   (1.0, -8), (0.0, -110), (1e-40, -110), (3e38, 119)):
        assert C8.scale_exponent(np.array([0.0, -top, np.nan, np.inf])) == e, top


def test_a_block_written_row_by_row_is_one_written_at_once():
    """but for values that a later scale makes subnormal: those are rounded twice,
    each time by half a step of 2^-9 of the scale at most."""
    rng = np.random.default_rng(3)
    for grow in (1.0, 1.6, 3.0):
        rows = rng.normal(size=(16, 32)) * grow ** np.arange(16)[:, None]
        held, e = np.zeros((0, 32)), None
        for r in rows:
            held, e = C8.write_block(held, e, r[None])
        once, e1 = C8.write_block(np.zeros((0, 32)), None, rows)
        assert e == e1
        normal = np.abs(rows) >= 2.0 ** (e - 6) * 1.1
        assert np.array_equal(held[normal], once[normal])
        assert np.abs(held - rows * 2.0 ** -e)[~normal].max(initial=0.0) <= 2 * 2.0 ** -10


def test_rows_are_those_of_the_cache_oracle():
    """but for its angles, whose cosines and sines it rounds to fp32."""
    rng = np.random.default_rng(6)
    x, g = rng.normal(size=(5, 16)), 1 + 0.1 * rng.normal(size=16)
    for pos in (0, 1, 77, 5000):
        for a, b in zip(C8.append_row(x, 3, 1, pos, 1e4, 1e-5, g, None), C.append_row(x, 3, 1, pos, 1e4, 1e-5, g, None)):
            assert np.allclose(a, b, atol=2.0 ** -22 * np.abs(x).max())


def test_rows_see_their_window_and_the_first_slots():
    assert C8.seen_slots(5, 0, 0).tolist() == [0, 1, 2, 3, 4]
    assert C8.seen_slots(9, 3, 2).tolist() == [0, 1, 6, 7, 8]
    assert C8.seen_slots(4, 3, 2).tolist() == [0, 1, 2, 3]
    assert C8.seen_slots(3, 9, 0).tolist() == [0, 1, 2]
    assert C8.seen_slots(0, 3, 2).tolist() == [] == C8.seen_slots(-4, 0, 0).tolist()
    rng = np.random.default_rng(4)
    q, K, V = rng.normal(size=(2, 8)), rng.normal(size=(20, 8)), rng.normal(size=(20, 8))
    out, p, lse, s = C8.attend_row(q, K, V, 13, 4, 2)
    want = C.attend(q, K[[0, 1, 9, 10, 11, 12]], V[[0, 1, 9, 10, 11, 12]])
    assert np.array_equal(out, want[0]) and np.array_equal(lse, want[2])


# ---- argument checks of the wrapper (nothing reaches the library)
def _fake():
    dr = object.__new__(Drafter)
    dr.ctx = None
    dr.device = torch.device("cpu")
    dr.cfg = B.prism_config(n_q_heads=4, n_kv_heads=2, head_dim=32, kv_block_size=16,
                            max_blocks_per_seq=5, max_batch=3, dtype=B.PRISM_BF16)
    dr._cache_setup()
    return dr


def _codes(*shape):
    return torch.zeros(shape, dtype=torch.uint8).view(F8)


def _kv8(dr, **kw):
    t = dict(lens=torch.zeros(3, dtype=torch.int32), k_codes=_codes(9, 2, 16, 32), v_codes=_codes(9, 2, 16, 32),
             scales=torch.ones(9, 2, 2), block_table=torch.zeros(3, 5, dtype=torch.int32))
    t.update(kw)
    return dr.cache8(**t)


def _kv(dr):
    p = torch.zeros(9, 2, 16, 32, dtype=torch.bfloat16)
    return dr.cache(torch.zeros(3, dtype=torch.int32), p, p.clone(), torch.zeros(3, 5, dtype=torch.int32))


@pytest.mark.parametrize("kw,err", [
    (dict(lens=torch.zeros(3)), TypeError),
    (dict(lens=torch.zeros(2, dtype=torch.int32)), ValueError),
    (dict(k_codes=torch.zeros(9, 2, 16, 32, dtype=torch.uint8)), TypeError),
    (dict(v_codes=_codes(8, 2, 16, 32)), ValueError),
    (dict(k_codes=_codes(9, 16, 2, 32).transpose(1, 2)), ValueError),
    (dict(scales=torch.ones(9, 2)), ValueError),
    (dict(scales=torch.ones(9, 2, 2).half()), TypeError),
    (dict(block_table=torch.zeros(3, 4, dtype=torch.int32)), ValueError),
])
def test_cache8_refuses_other_tensors(kw, err):
    with pytest.raises(err):
        _kv8(_fake(), **kw)


def test_buffers_make_a_cache():
    dr = _fake()
    k, v, s = dr.cache8_buffers(7)
    kv8 = dr.cache8(torch.zeros(3, dtype=torch.int32), k, v, s, torch.zeros(3, 5, dtype=torch.int32))
    assert kv8.n_pool_blocks == 7 and k.dtype == F8 and not bool(k.view(torch.uint8).any())


def test_calls_refuse_other_tensors():
    dr = _fake()
    kv8, kv = _kv8(dr), _kv(dr)
    bf = dict(dtype=torch.bfloat16)
    q, i32 = torch.zeros(3, 4, 32, **bf), dict(dtype=torch.int32)
    bad = [
        (TypeError, lambda: dr.cache8_append(kv, torch.zeros(3, 256, **bf))),
        (TypeError, lambda: dr.cache8_append(kv8, torch.zeros(3, 256))),
        (ValueError, lambda: dr.cache8_append(kv8, torch.zeros(3, 255, **bf))),
        (ValueError, lambda: dr.cache8_append(kv8, torch.zeros(3, 256, **bf), k_gain=torch.zeros(31, **bf))),
        (ValueError, lambda: dr.cache8_append(kv8, torch.zeros(3, 256, **bf), offsets=torch.zeros(3, **i32))),
        (TypeError, lambda: dr.cache8_append(kv8, torch.zeros(3, 256, **bf), positions=torch.zeros(3))),
        (ValueError, lambda: dr.cache8_append(kv8, torch.zeros(3, 256, **bf), out=q[:2])),
        (TypeError, lambda: dr.cache8_pack(kv, kv8)),
        (TypeError, lambda: dr.cache8_unpack(kv8, kv8)),
        (ValueError, lambda: dr.cache8_pack(kv8, kv, start=torch.zeros(2, **i32))),
        (TypeError, lambda: dr.cache8_unpack(kv8, kv, start=torch.zeros(3))),
        (TypeError, lambda: dr.cache_attend_rows(None, q)),
        (TypeError, lambda: dr.cache_attend_rows(kv8, q.float())),
        (ValueError, lambda: dr.cache_attend_rows(kv, q[:, :3])),
        (ValueError, lambda: dr.cache_attend_rows(kv, q.transpose(0, 1).contiguous().transpose(0, 1))),
        (ValueError, lambda: dr.cache_attend_rows(kv8, q, offsets=torch.zeros(3, **i32))),
        (TypeError, lambda: dr.cache_attend_rows(kv8, q, out=q.float())),
        (TypeError, lambda: dr.cache_attend(kv8, q)),
        (TypeError, lambda: dr.cache_append(kv8, torch.zeros(3, 256, **bf))),
        (TypeError, lambda: dr.cache_summarize(kv8, q)),
        (TypeError, lambda: dr.cache_select(kv8, q, q, 1)),
        (TypeError, lambda: dr.cache_evict(kv8, q, q, 1)),
    ]
    for i, (err, call) in enumerate(bad):
        with pytest.raises(err):
            call()


def test_calls_take_subclasses_of_their_structs(monkeypatch):
    """A program's own descriptions, derived from the binding's, reach the library."""
    class Batch(B.prism_batch):
        pass

    class Held(B.prism_cache8):
        pass

    def as_a(cls, kv):
        own = cls.from_buffer_copy(kv)
        own.__dict__.update(kv.__dict__)
        return own

    dr = _fake()
    kv, kv8 = as_a(Batch, _kv(dr)), as_a(Held, _kv8(dr))
    bf = dict(dtype=torch.bfloat16)
    q, qkv, w = torch.zeros(3, 4, 32, **bf), torch.zeros(3, 256, **bf), torch.zeros(9, 2, 16)
    summary, table = torch.zeros(9, 2, 2, 32, **bf), torch.zeros(3, 5, dtype=torch.int32)
    monkeypatch.setattr(Drafter, "_stream", lambda self: 0)
    calls = {name: [] for name in B.EXPORTS if name.startswith("prism_cache")}
    for name, got in calls.items():
        if name.endswith("scratch"):
            monkeypatch.setattr(B, name, lambda *a: 16)
        else:
            monkeypatch.setattr(B, name, lambda ctx, io, *a, got=got: got.append(io))
    dr.cache_append(kv, qkv)
    assert calls["prism_cache_append"][0].kv == ctypes.addressof(kv)
    dr.cache_attend(kv, q)
    dr.cache_summarize(kv, summary)
    dr.cache_select(kv, q, summary, 1)
    dr.cache_evict(kv, table, w, 1)
    dr.cache8_append(kv8, qkv)
    dr.cache8_pack(kv8, kv)
    dr.cache8_unpack(kv8, kv)
    io = dr._io[6]
    dr.cache_attend_rows(kv8, q)
    assert io.kv is None and io.kv8 == ctypes.addressof(kv8)
    dr.cache_attend_rows(kv, q)
    assert io.kv == ctypes.addressof(kv) and io.kv8 is None
    assert all(len(got) == (2 if name == "prism_cache_attend_rows" else 1)
               for name, got in calls.items() if not name.endswith("scratch"))


STRUCTS = ("prism_cache8", "prism_cache8_rows", "prism_cache8_move", "prism_cache_row_attention")


def test_structs_mirror_the_header(tmp_path):
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "prism_draft.h"', "int main(void) {"]
    for st in STRUCTS:
        lines.append('  printf("%s %%zu\\n", sizeof(%s));' % (st, st))
        lines += ['  printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (st, f, st, f) for f, _ in getattr(B, st)._fields_]
    (tmp_path / "l.c").write_text("\n".join(lines + ["  return 0;\n}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout
    ref = {k: int(v) for k, v in (ln.split() for ln in out.splitlines())}
    header = open(os.path.join(ROOT, "include", "prism_draft.h")).read()
    for st in STRUCTS:
        cls = getattr(B, st)
        assert ctypes.sizeof(cls) == ref[st], st
        for f, _ in cls._fields_:
            assert getattr(cls, f).offset == ref["%s.%s" % (st, f)], (st, f)
        body = re.sub(r"/\*.*?\*/", "", header[: header.index("} %s;" % st)], flags=re.S).rsplit("{", 1)[1]
        assert len(re.findall(r"\b\w+\s*(?=[;,])", body)) == len(cls._fields_), st


@pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")
def test_null_context():
    L = B.lib()
    n = ctypes.c_uint64()
    assert L.prism_cache_rows_scratch(None, 1, 1, 0, ctypes.byref(n)) == -1
    assert L.prism_cache8_append(None, None, None) == -1
    assert L.prism_cache8_pack(None, None, None) == -1
    assert L.prism_cache8_unpack(None, None, None) == -1
    assert L.prism_cache_attend_rows(None, None, None) == -1


def _host(tmp_path, name, code):
    src, exe = tmp_path / (name + ".cc"), tmp_path / name
    src.write_text(code)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], capture_output=True, text=True)


def test_rows_plans(tmp_path):
    """The segments that random rows make are within the plan's, scratch for a
    batch and rows serves every smaller call, and counts stay below 2^31."""
    r = _host(tmp_path, "rows", r"""
#include <cstdlib>
#include <vector>
#include "plan.h"
using namespace prism;
int main() {
  srand(5);
  for (int it = 0; it < 20000; ++it) {
    const int B = 1 + rand() % 64, nkv = 1 + rand() % 8, g = 1 + rand() % 8, d = 32 << (rand() % 4);
    const int top = 1 << (rand() % 12), max_len = 1 + rand() % (1 << (rand() % 18 + 1));
    long T = 0;
    std::vector<int> counts;
    for (int b = 0; b < B; ++b) {
      const int n = rand() % 4 ? rand() % (top + 1) : 0;
      T += n;
      counts.push_back(n);
    }
    T += rand() % 3;
    if (T < 1) T = 1;
    const int window = rand() % 2 ? 1 + rand() % 5000 : 0, n_first = rand() % 40, waves = cache_waves(d * 2);
    const bool bf16 = rand() % 2;
    const RowsPlan p = rows_plan(bf16, nkv, g, d, B, (int)T, false, max_len, window, n_first, waves);
    const int span = rows_span(g, p.cols, max_len, window, n_first), rt = rows_per_tile(g, p.cols);
    if (span < 1 || span > max_len) return 2;
    if (rt < 1 || rt * g > p.cols || (p.cols != 16 && p.cols != 32)) return 1;
    long few = 0, many = 0;                       // segments of each kernel
    int longest = 0;
    for (int b = 0; b < B; ++b) {
      if (counts[b] > p.few) many += (counts[b] + prompt_rows(g, d) - 1) / prompt_rows(g, d) * nkv;
      else few += (counts[b] + rt - 1) / rt * nkv;
      longest = counts[b] > longest ? counts[b] : longest;
    }
    if (!p.segments) {                            // the prompts' kernel alone: one sequence
      if (B != 1 || !p.prompt_segments) return 3;
      many = (longest + prompt_rows(g, d) - 1) / prompt_rows(g, d) * nkv;
      few = 0;
    }
    if (few > p.segments || many > p.prompt_segments) return 4;
    if (!bf16 && p.prompt_segments) return 5;
    if (p.splits < 1 || p.splits > PROMPT_SPLITS || (p.splits > 1 && span < p.splits * PROMPT_PART)) return 6;
    if (p.segments && p.direct && p.waves != p.segments) return 7;
    if (p.segments && !p.direct && (p.waves < 1 || p.waves > waves || (long)p.segments * cache_granules(max_len) >= 1l << 31)) return 8;
    const size_t need = rows_scratch(g, d, p) + prompt_scratch(nkv * g, d, (int)T, p);
    const size_t up = rows_scratch_up_to(bf16, nkv, g, d, B, (int)T, max_len, waves);
    if (need > up) return 9;
    if (p.segments && !p.direct && need < (size_t)cache_partials(p.waves, p.segments) * rt * g * (d + 2) * 4) return 10;
    if (rows_scratch_up_to(bf16, nkv, g, d, 1 + rand() % B, 1 + rand() % (int)T, 1 + rand() % max_len, waves) > up) return 11;
  }
  return 0;
}
""")
    assert r.returncode == 0, r.returncode


def test_fp64_rotation(tmp_path):
    r = _host(tmp_path, "rot", r"""
#define __host__
#define __device__
#include <cstdio>
#include <cstring>
#include <math.h>
#include "rotation.h"
int main() {
  double worst = 0;
  for (int i = 0; i < 400000; ++i) {
    const double a = i < 1000 ? i * 0.0015707963 - 0.785 : (i - 200000) * 0.7310585 * (i % 7 ? 1 : 30);
    double c, s;
    prism::rotation_cos_sin64(a, c, s);
    const double tol = 4e-16 + fabs(a) * 3e-17;     // the angle's own reduction: two words of pi / 2
    const double e = fmax(fabs(c - cos(a)), fabs(s - sin(a))) / tol;
    worst = e > worst ? e : worst;
  }
  printf("%g", worst);
  return worst <= 1 ? 0 : 1;
}
""")
    assert r.returncode == 0, r.stdout
