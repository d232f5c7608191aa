"""The planner of laser_attend (csrc/attend_plan.hpp), compiled with the host compiler: which kernel takes a
span and over how many workgroups its keys are split, over sizes from one row and no key to the longest."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_31580_amd", "csrc")
MAIN = """
#include <cstdio>
#include <vector>
#include "attend_plan.hpp"
int main() {
  int n, hq, hkv, hd, cus, es, i8, io16, mode;
  while (std::scanf("%d %d %d %d %d %d %d %d %d", &n, &hq, &hkv, &hd, &cus, &es, &i8, &io16, &mode) == 9) {
    std::vector<laser::AttendSize> s(n);
    for (auto& x : s) std::scanf("%d %d %d", &x.n, &x.pages, &x.rows_pages);
    laser::plan_attend(s.data(), n, hq, hkv, hd, cus, es, i8, io16, mode);
    for (auto& x : s) std::printf("%d %d %d ", x.kind, x.tiles, x.nsplit);
    std::printf("\\n");
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", f"-I{CSRC}", "-o", str(d / "plan"), str(d / "main.cpp")], check=True)

    def call(spans, hq=28, hkv=4, hd=128, cus=256, es=1, io16=1, mode=0, i8=None):
        line = f"{len(spans)} {hq} {hkv} {hd} {cus} {es} {int(es == 1 if i8 is None else i8)} {io16} {mode} " + " ".join(f"{n} {p} {r}" for n, p, r in spans)
        out = [int(x) for x in subprocess.run([str(d / "plan")], input=line, capture_output=True, text=True, check=True).stdout.split()]
        return [tuple(out[3 * i:3 * i + 3]) for i in range(len(spans))]

    return call


def span(n, end):
    """n rows that end at position `end`, causal."""
    return (n, -(-end // 16), min(n, end) // 16)


def test_kernels_and_bounds(plan):
    rng = random.Random(3)
    for _ in range(60):
        hq, hkv = rng.choice([(28, 4), (32, 8), (12, 2), (16, 1), (3, 3)])
        es, io16 = rng.choice([(1, 1), (1, 0), (2, 1), (2, 0), (4, 0), (4, 1)])
        mode = rng.choice([0, 0, 1, 2])
        spans = []
        for _ in range(rng.choice([1, 1, 2, 8, 64])):
            n = int(2 ** rng.uniform(0, 13))
            spans.append(span(n, int(2 ** rng.uniform(0, 16)) if rng.random() < 0.95 else 0))
        for (n, pages, _), (kind, tiles, splits) in zip(spans, plan(spans, hq, hkv, rng.choice([64, 128]), 256, es, io16, mode)):
            cols = n * hq // hkv
            assert (kind != 2 or mode != 1) and (mode != 2 or es == 4 or cols <= 64 or kind == 2)
            assert kind in ((0,) if es == 4 else (0, 1, 2)) and not (kind == 1 and not io16)
            assert (kind != 1 or cols > 16) and (kind != 2 or cols > 64)
            assert tiles == -(-cols // {0: 16, 1: 32, 2: 256}[kind])
            assert 1 <= splits <= 128 and splits <= max(1, pages)


def test_one_long_request_fills_the_card(plan):
    ((kind, _, splits),) = plan([span(1, 14336)])
    assert kind == 0 and splits * 4 >= 128
    ((kind, tiles, splits),) = plan([span(128, 14000)], mode=2)
    assert kind == 2 and 128 <= tiles * 4 * splits <= 512


def test_short_keys_and_full_cards_are_not_split(plan):
    assert plan([span(1, 500)]) == [(0, 1, 1)]
    assert all(s == 1 for _, _, s in plan([span(1, 50 + 9 * i) for i in range(64)], 32, 8))
    ((_, _, splits),) = plan([span(4096, 8192)], 32, 8)
    assert splits == 1
    for mode, kind in ((1, 1), (2, 2)):
        assert plan([span(512, 512)], mode=mode)[0][::2] == (kind, 1)


def test_partials_are_bounded(plan):
    """However many rows a call has, its splits are at most 64 workgroups per CU beyond one per tile."""
    for es, io16, mode in ((4, 0, 0), (1, 1, 1), (2, 0, 1), (1, 1, 0)):
        for spans in ([(200000, 4000, 0)], [(20000, 4000, 10)] * 3, [(900, 3000, 0)] * 20, [(1, 4000, 0)] * 200, [(7, 900, 0)] * 900):
            got = plan(spans, 28, 4, es=es, io16=io16, mode=mode)
            tiles = sum(t * 4 for _, t, _ in got)
            assert sum(t * 4 * s for _, t, s in got) <= tiles + 64 * 256, (es, io16, spans[0], got[0])


def test_tiles_pay_from_some_work_on(plan):
    """Prompts of a few hundred rows through row kernels, long ones and chunks behind long contexts through tiles."""
    for n, end, kind in ((64, 64, 1), (512, 512, 1), (2048, 2048, 2), (512, 14000, 2), (4096, 16384, 2)):
        assert plan([span(n, end)])[0][0] == kind, (n, end)


def test_tiles_are_filled(plan):
    """Long contexts, so that work is no question: tiles of which few columns are in use go through the row kernels, per span."""
    def kinds(n, **kw):
        return [k for k, _, _ in plan([span(n, 9000)] * 16, 32, 8, **kw)]
    for kw, few, enough in ((dict(), 40, 48), (dict(i8=0), 24, 28), (dict(es=2), 24, 28), (dict(es=2, io16=0), 32, 40), (dict(i8=0, io16=0), 40, 48),
                            (dict(io16=0), 50, 64)):
        assert set(kinds(few, **kw)) <= {0, 1} and set(kinds(enough, **kw)) == {2}, kw
    assert [k for k, _, _ in plan([span(20, 9000)] * 8 + [span(64, 9000)] * 8, 32, 8)] == [1] * 8 + [2] * 8
    assert set(kinds(20, mode=2)) == {2}
    for es, i8, io16 in ((1, 1, 1), (1, 0, 1), (2, 0, 1), (1, 1, 0), (2, 0, 0)):
        assert plan([span(1000, 8000)], 32, 8, es=es, i8=i8, io16=io16)[0][0] == 2


def test_ragged_tiles_get_like_shares(plan):
    """Spans of different lengths: a workgroup's pages differ by less than a factor of two where spans are split."""
    spans = [span(60, 1000 + 530 * i) for i in range(16)]
    got = plan(spans, 32, 8)
    assert {k for k, _, _ in got} == {2}
    shares = [-(-p // s) for (_, p, _), (_, _, s) in zip(spans, got)]
    split = [x for x, (_, _, s) in zip(shares, got) if s > 1]
    assert split and max(shares) <= 2 * min(split)
    assert got[-1][2] > got[4][2] >= got[0][2]
