"""How an attention of several new tokens is cut (host only: no GPU call)."""
import math
import random

import pytest

from tests.prompt_plan import plan, workspace
from tests.test_gpu_prompt_tiles import CUT, SHAPES, SIZES, SOME


def total(sizes):
    return sum(n for n, _ in sizes)


@pytest.mark.parametrize("sizes,heads,group,d,page", [(SIZES, *s) for s in SHAPES] + [(SOME, 52, 1, 64, 16), (CUT, 128, 1, 128, 64)])
def test_shapes_of_the_tests_take_tiles_of_128_rows(sizes, heads, group, d, page):
    p = plan("bf16", total(sizes), len(sizes), heads, group, d, page, -(-max(n for _, n in sizes) // page))
    assert p.rows == 128 and p.splits == (2 if sizes is CUT else 1)


def test_workspace_holds_every_plan_and_never_falls():
    rng = random.Random(5)
    log = lambda lo, hi: max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi))))))
    seen = set()
    for _ in range(20_000):
        page, group, heads, d = rng.choice((16, 64, 1024)), log(1, 64), log(1, 256), 16 * rng.randint(1, 16)
        b = log(1, 2 ** 23 // (heads * group))
        t = log(1, 2 ** 29 // (heads * group))
        pages = log(1, 2 ** 30 // page)
        window, prefix = rng.choice((0, 0, log(1, 2 ** 31 - 1))), rng.random() < 0.5
        p = plan("bf16", t, b, heads, group, d, page, pages, window, prefix)
        # what the kernel writes: a slot for every row of every part of every unit
        used = p.tiles * heads * p.splits * p.rows * (p.dp + 2) * 4 if p.splits > 1 else 0
        if b > 1024:                                         # and a sum for every 256 sequences
            used += -(-(-(-b // 256) * 4) // 256) * 256
        have = workspace("bf16", t, b, heads, group, d, page, pages)
        assert used <= have
        assert p.tiles >= t * group // p.rows + min(b, t) and p.tiles * heads * p.splits < 2 ** 24
        more = (t + log(1, t), b, pages) if rng.random() < 0.4 else (t, b + log(1, b), pages) if rng.random() < 0.5 else (t, b, pages + log(1, pages))
        if more[0] * heads * group <= 2 ** 29 and more[1] * heads * group <= 2 ** 23 and more[2] * page <= 2 ** 30:
            assert have <= workspace("bf16", more[0], more[1], heads, group, d, page, more[2])
        seen.add((p.rows, p.splits > 1))
    assert len(seen) == 4
