"""The calls of test_gpu_rows_prompts.py reach the kernel that they test (CPU)."""
import pytest

import rows_plan as R


def _plan(case, window=(0, 0)):
    heads, bs, lens, counts = case
    return R.plan(heads, len(lens), sum(counts), bs * R.columns_of(bs, lens, counts), *window)


@pytest.mark.parametrize("cases,windows", [
    (R.BLOCKS, R.BLOCK_WINDOWS), (R.SPLIT, R.SPLIT_WINDOWS), (R.HIDDEN, [R.HIDDEN_WINDOW]), (R.FLAGS, [(0, 0)]),
    (R.GRAPHS, R.GRAPH_WINDOWS), (R.INFINITE, [(0, 0)]), (R.STREAMS, [(0, 0)]), (R.EIGHT, [(0, 0)]),
    (R.NEW, [(0, 0), (30, 2)]), (R.CROWD, [(0, 0), (200, 3)]), (R.LONG, [(0, 0), (9000, 5)]), ([R.SCRATCH], [(0, 0)]),
])
def test_prompts_go_by_their_kernel(cases, windows):
    for case in cases:
        for window in windows:
            p = _plan(case, window)
            assert p.prompt_segments > 0 and any(R.is_prompt(p, n) for n in case[3]), (case, window)


def test_cases_cover_both_ways():
    assert not any(_plan(c, R.HIDDEN_WINDOW).prompt_segments for c in R.HIDDEN_TILES)
    assert {_plan(c, R.HIDDEN_WINDOW).cols for c in R.HIDDEN_TILES} == {16, 32}
    assert all(_plan(c, w).splits > 1 for c in R.SPLIT for w in R.SPLIT_WINDOWS)
    assert any(_plan(c).splits > 1 for c in R.GRAPHS + R.STREAMS) and any(_plan(c).splits == 1 for c in R.HIDDEN)
    p = _plan(R.SCRATCH)
    assert p.segments and not p.direct and p.prompt_segments and p.splits > 1
    one = [c for c in R.BLOCKS + R.SPLIT if c[0][0] == c[0][1]]
    assert any(len(c[2]) == 1 for c in one) and any(len(c[2]) > 1 for c in one)
    assert {c[0][2] for c in R.BLOCKS} == {32, 64, 128, 256} and {c[1] for c in R.BLOCKS} >= {1, 7, 12, 64, 256}


def test_which_sequences_are_prompts():
    small = ("bf16",)
    assert not R.plan((8, 2, 64) + small, 4, 117, 600).prompt_segments            # 468 columns in four sequences
    assert R.is_prompt(R.plan((8, 2, 64) + small, 1, 13, 600), 13)                # one of its own
    assert not R.plan((8, 2, 64) + small, 1, 12, 600).prompt_segments
    p = R.plan((8, 2, 64) + small, 3, 300, 600)
    assert R.is_prompt(p, 13) and not R.is_prompt(p, 12)
    assert not R.plan((8, 2, 64, "f32"), 1, 500, 600).prompt_segments
    assert not R.plan((8, 2, 64) + small, 64, 64, 600, one_each=True).prompt_segments
