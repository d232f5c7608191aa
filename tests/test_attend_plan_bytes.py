"""How much memory the partials of a laser_attend call take (csrc/attend_plan.hpp), whatever the number of its rows."""
import random

import pytest

from test_attend_plan import plan, span  # noqa: F401  (plan: a fixture)

MOST = 288 << 20


def size(got, spans, hq, hd):
    """Bytes of the partials: head_dim + 2 floats per row, head and split where a span is split."""
    return sum(n * hq * s * (hd + 2) * 4 for (n, _, _), (_, _, s) in zip(spans, got) if s > 1)


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("es,i8,io16", [(1, 1, 1), (1, 0, 1), (2, 0, 1), (2, 0, 0), (4, 0, 0), (1, 1, 0)])
def test_partials_have_a_bound_in_bytes(plan, es, i8, io16, mode):
    rng = random.Random(5)
    calls = [([(8, 700, 0)] * 2047, 32, 8), ([(30000, 3000, 1875)], 32, 8), ([(2759, 4039, 172)] * 16, 32, 8),
             ([(60724, 4096, 3795)] * 2, 12, 2), ([(200000, 4000, 0)], 28, 4), ([(20, 4000, 0)] * 600, 16, 1)]
    for _ in range(20):
        n = int(2 ** rng.uniform(4, 16))
        calls.append(([span(max(1, int(n * rng.uniform(0.3, 1))), rng.randint(1, 65536)) for _ in range(rng.choice([1, 3, 16, 64]))],
                      *rng.choice([(28, 4), (32, 8), (12, 2), (16, 1)])))
    for spans, hq, hkv in calls:
        got = plan(spans, hq, hkv, 128, 256, es, io16, mode, i8)
        assert size(got, spans, hq, 128) <= MOST, (spans[0], len(spans), got[0])


def test_the_bound_leaves_ordinary_calls_alone(plan):
    """Long contexts of few rows are split as far as before; chunks of thousands of rows behind long contexts too."""
    assert all(s >= 16 for _, _, s in plan([span(1, 60000)] * 64, 32, 8))
    assert plan([span(512, 14000)])[0][2] > 1 and plan([span(2048, 16000)])[0][2] > 1
