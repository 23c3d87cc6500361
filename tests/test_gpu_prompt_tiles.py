"""GPU parity of attention of several new tokens by the row tiles that a call
takes: those of 128 (four waves that share their keys) where there are at least
256 tiles times key-value heads, else those of 32; against the float64 oracle, or
what the call said before a change that must not reach it.

Tolerances as in test_gpu_prompt_whole.py, the weights' part by the plan that
the call takes: half a step of the type where one part carries a weight, 2^-16
where two do (tiles of 32 rows, and f16 queries over e4m3).  Beside that, a
weight is a float32 relative to its row's running maximum, so that 2^-126 of the
heaviest and less may count as 0, and over e4m3 its product with the value's
scale is an operand of 16 bits, which may count as 0 below 2^-126 as well: n
tokens of 2^-126 |v| over the sum of weights (at least 1), and of 2^-126 448.
Over f16 caches a weight is within half a step however light, but for 2^-25 of
the result (half of f16's smallest step); in two parts it is within 2^-16 or
2^-37 of the row's heaviest (half of f16's smallest step, the heaviest at 2^12).
"""
import numpy as np
import pytest
import torch

from tests.gpu_check import say
from tests.prompt_plan import plan_of
from tests.test_gpu_prompt_ops import KINDS, ROUND, TINY, U, f64, gen, stored
from tests.test_gpu_prompt_whole import FEW, RULES, make_prompt, run_prompt
from tests.test_gpu_prompt_whole import SIZES as SMALL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def apc():
    import paper_2502_06798_amd as apc
    apc.load()
    assert torch.cuda.is_available()
    return apc


def check(orc, cache, dtype, made, scale, got, heads=None, **kw):
    """A call's results against the oracle's, for all key-value heads or some."""
    pool, table, q, starts, lens = made
    out, lse = got
    two = plan_of(made, cache, **kw).rows == 32 or (cache == "e4m3" and dtype == "f16")
    group = q.shape[1] // pool[0].shape[1]
    if heads is not None:
        rows = [h * group + a for h in heads for a in range(group)]
        pool = tuple(None if p is None else p[:, heads] for p in pool)
        q, out, lse = q[:, rows], out[:, rows], lse[:, rows]
        if kw.get("slopes") is not None:
            kw = dict(kw, slopes=kw["slopes"][rows])
    k, v, ks, vs = pool
    host = lambda x: None if x is None else x.cpu().numpy()
    cap, slopes = kw.get("cap", 0.0), host(kw.get("slopes"))
    with np.errstate(invalid="ignore", over="ignore"):
        ro, rl, spread, top, heavy, away = orc.attend_prompt(
            cache, f64(q), host(starts), stored(k.contiguous()), stored(v.contiguous()), host(ks), host(vs), host(table), host(lens),
            scale, kw.get("window", 0), cap, slopes, host(kw.get("prefix")))
    n = table.shape[1] * k.shape[2]
    e = (q.shape[2] + 24) * U * top + cap * 2.0 ** -21
    if slopes is not None:
        e = e + 4 * U * np.abs(slopes).astype(np.float64) * away
    weight = spread * (2.0 ** -16 if two else ROUND[dtype])
    if cache == "f16":
        weight = np.minimum(weight + n * 2.0 ** -37 * heavy, spread * ROUND[dtype]) + 2.0 ** -25
    tol = spread * (4 * e + 2 * (n + 64) * U)[..., None] + weight
    tol = tol + np.abs(ro) * ROUND[dtype] * 1.001 + TINY[dtype]
    tol = tol + n * 2.0 ** -126 * (heavy + (448.0 if cache == "e4m3" else 0.0))
    g, gl = f64(out), f64(lse)
    none = np.isnan(rl)                                      # rows of no sequence
    assert (g[none] == 7).all() and (gl[none] == 7).all()
    # infinity is a right rounding of what is half a step below the type's last value, or more, and within the tolerance
    end = {"f16": 65520.0, "bf16": (2.0 - 2.0 ** -8) * 2.0 ** 127}[dtype]
    over = np.isinf(g) & (np.sign(g) == np.sign(ro)) & (np.abs(ro) + tol >= end)
    bad = ~(np.abs(g - ro) <= tol) & ~none[..., None] & ~over
    assert not bad.any(), (np.argwhere(bad)[:4], bad.sum(), np.abs(g - ro)[bad].max())
    empty = np.isneginf(rl)
    assert np.array_equal(np.isneginf(gl), empty) and (g[empty] == 0).all()
    some = ~none & ~empty
    assert (np.abs(gl[some] - rl[some]) <= (2 * e + (n + 64) * U)[some] + 2.0 ** -20 * np.abs(rl[some])).all()


def tall(made, cache, splits=1, **kw):
    """The call takes tiles of 128 rows, its keys cut into so many parts."""
    p = plan_of(made, cache, **kw)
    assert (p.rows, p.splits) == (128, splits)
    return made


# every way new tokens and lengths can end in a row tile, a tile of keys and a page, sequences of none and of one among them
SIZES = [(1, 1), (2, 40), (0, 10), (33, 33), (17, 100), (0, 0), (129, 130), (65, 200), (1, 200), (31, 31), (64, 64), (128, 128),
         (127, 200), (130, 140)]
SHAPES = [(19, 1, 16, 16), (12, 4, 64, 16), (19, 1, 48, 32), (10, 5, 80, 16), (6, 8, 128, 64), (15, 3, 128, 16), (3, 16, 128, 128),
          (19, 1, 64, 256), (19, 2, 96, 256), (12, 4, 176, 16), (7, 7, 256, 16), (19, 2, 32, 1024), (19, 1, 208, 32)]
SOME = [(40, 100), (70, 208), (150, 207), (50, 20), (9, 50)]                 # with 52 heads
CUT = [(70, 2100), (150, 2500)]                                              # with 128 heads: keys in two parts


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("heads,group,d,page", SHAPES)
def test_tiles_lengths(apc, orc, cache, dtype, heads, group, d, page):
    say(f"tiles {dtype} over {cache} heads={heads} group={group} d={d} page={page}")
    made = tall(make_prompt(d + page, SIZES, heads, group, d, page, -(-200 // page), cache, dtype, pad=3), cache)
    check(orc, cache, dtype, made, d ** -0.5, run_prompt(apc, *made, d ** -0.5))


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("rule", RULES, ids=[" ".join(f"{k}={v}" for k, v in r.items()) for r in RULES])
def test_tiles_rules(apc, orc, cache, dtype, rule):
    """Windows, caps, slopes and prefixes, alone and together."""
    for d in (64, 128, 160):
        say(f"tiles {rule} {dtype} over {cache} d={d}")
        made = make_prompt(d, SIZES, 15, 3, d, 16, 13, cache, dtype, 2.0)
        kw = dict(rule)
        if "slopes" in kw:
            kw["slopes"] = kw["slopes"] * torch.arange(1, 46, device="cuda", dtype=torch.float32) / 20
        if "prefix" in kw:
            kw["prefix"] = torch.full((len(SIZES),), kw["prefix"], dtype=torch.int32, device="cuda")
            kw["prefix"][1] = 3
        tall(made, cache, **kw)
        check(orc, cache, dtype, made, d ** -0.5, run_prompt(apc, *made, d ** -0.5, **kw), heads=[0, 4, 9, 14], **kw)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_cut_keys(apc, orc, cache, dtype, d):
    """Keys in two parts, units whose keys are too few for that beside them; and many keys in one."""
    for sizes, splits in ((CUT, 2), ([(150, 2500), (70, 1030)], 2), (CUT + [(40, 2300)], 1)):
        for kw in (dict(), dict(window=2100, slopes=torch.linspace(0.0, 0.02, 128, device="cuda"))):
            say(f"tiles cut {dtype} over {cache} d={d} {sizes} {list(kw)}")
            made = tall(make_prompt(d, sizes, 128, 1, d, 64, 40, cache, dtype, 1.5), cache, splits, **kw)
            got = run_prompt(apc, *made, d ** -0.5, **kw)
            check(orc, cache, dtype, made, d ** -0.5, got, heads=[0, 77, 127], **kw)
            for a, b in zip(got, run_prompt(apc, *made, d ** -0.5, **kw)):
                assert torch.equal(a, b)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_absent_pages_and_odd_tables(apc, orc, cache, dtype, d):
    """Page entries outside the pool leave their tokens out; lengths below 0 and past the table are cut; sequences with
    more new tokens than they hold."""
    sizes = [(40, 200), (30, 100), (70, 208), (50, 20), (90, 50), (35, 5), (60, 130)]
    made = pool, table, q, starts, lens = make_prompt(17, sizes, 38, 1, d, 16, 13, cache, dtype, pad=4)
    n_pages = pool[0].shape[0]
    table[0, 0], table[0, 5:7], table[1, 6], table[2, 3:] = -1, n_pages, -2 ** 31, 2 ** 31 - 1
    table[4, :], table[6, 7] = -7, n_pages
    lens[2], lens[5] = 5000, -3
    pre = torch.tensor([0, 5, 300, 10, 9, 2, 70], dtype=torch.int32, device="cuda")
    for kw in (dict(), dict(prefix=pre), dict(window=30, prefix=pre)):
        say(f"tiles absent {dtype} over {cache} d={d} {list(kw)}")
        check(orc, cache, dtype, tall(made, cache, **kw), 0.2, run_prompt(apc, *made, 0.2, **kw), heads=[0, 9, 37], **kw)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("heads,group,d,page", [(2, 4, 64, 16), (2, 5, 80, 16), (1, 8, 128, 64), (1, 7, 256, 16), (3, 1, 48, 32)])
def test_small_calls_carry_weights_in_two_parts(apc, orc, cache, dtype, heads, group, d, page):
    """Calls in tiles of 32 rows hold the weights to 2^-16, however many rows their sequences have."""
    for sizes in (SMALL, FEW, [(200, 5000), (1, 3000)]):
        say(f"two parts {dtype} over {cache} heads={heads} group={group} d={d} n={len(sizes)}")
        made = make_prompt(d + 5, sizes, heads, group, d, page, -(-max(n for _, n in sizes) // page), cache, dtype, pad=3)
        assert plan_of(made, cache).rows == 32
        check(orc, cache, dtype, made, d ** -0.5, run_prompt(apc, *made, d ** -0.5))


STARTS = {"cut": [-4, 37, 60, 60, 10 ** 6, 10 ** 6 + 5, 2 ** 31 - 1], "falling": [100, 140, 143, 20, 60, 90, -3],
          "turned": [2 ** 31 - 1, 150, 230, 40, 150, 3, -2 ** 31]}


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("name", STARTS)
@pytest.mark.parametrize("heads", [2, 128])
def test_starts_are_cut_and_falling_ones_have_no_row(apc, orc, cache, dtype, name, heads):
    """Starts outside the rows, falling ones among them (no row stands in two sequences): sequences' rows are right, and
    the others stay as they were."""
    say(f"starts {name} {dtype} over {cache} heads={heads}")
    pool, table, q, _, lens = make_prompt(71, [(40, 200), (30, 150), (60, 208), (50, 60), (40, 90), (35, 40)], heads, 2, 64, 16, 13, cache, dtype)
    starts = torch.tensor(STARTS[name], dtype=torch.int32, device="cuda")
    made = pool, table, q, starts, lens
    assert plan_of(made, cache).rows == (32 if heads == 2 else 128)
    some = [0, 1] if heads == 2 else [0, 50, 127]
    cut = starts.clamp(0, q.shape[0]).tolist()
    rows = [r for a, b in zip(cut, cut[1:]) for r in range(a, b)]
    assert len(set(rows)) == len(rows) and (name == "cut" or 0 < len(rows) < q.shape[0])
    for kw in (dict(), dict(prefix=torch.tensor([5, 0, 300, 9, 2, 40], dtype=torch.int32, device="cuda"), window=50)):
        got = run_prompt(apc, *made, 0.2, **kw)
        check(orc, cache, dtype, made, 0.2, got, heads=some, **kw)
        rest = [r for r in range(q.shape[0]) if r not in set(rows)]
        assert (got[0][rest] == 7).all() and (got[1][rest] == 7).all()


def spoil(pool, keep, fill):
    """Bytes of `fill` in every token (page x place) that is not to be kept."""
    for t in pool:
        if t is not None:
            m = keep[:, None, :].expand(t.shape[:3])
            m = m[..., None].expand(t.shape) if t.dim() == 4 else m
            raw = t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])
            bad = torch.empty_like(raw)
            bad.view(torch.uint8).fill_(fill)
            raw.copy_(torch.where(m, raw, bad))


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("fill", [0xff, 0x7f, 0x7c])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_unseen_slots_hold_anything(apc, cache, dtype, fill, d):
    """NaN, infinities and huge values past the lengths and in pages that no table names: bit for bit the same results; in
    the last token of each sequence, which its own row alone sees: the other rows' within the other order of their sums."""
    for sizes, heads, splits, pages in ((SOME, 52, 1, 4), (CUT, 128, 2, 40)):
        pool, table, q, starts, lens = made = tall(make_prompt(13, sizes, heads, 1, d, 64, pages, cache, dtype), cache, splits)
        want = run_prompt(apc, *made, 0.125)
        seen = torch.zeros((pool[0].shape[0], 64), dtype=torch.bool, device="cuda")
        for i, (_, n) in enumerate(sizes):
            j = torch.arange(n, device="cuda")
            seen[table[i][j // 64].long(), j % 64] = True
        say(f"tiles unseen 0x{fill:x} {dtype} over {cache} d={d} past the lengths {len(sizes)}")
        spoil(pool, seen, fill)
        for a, b in zip(want, run_prompt(apc, *made, 0.125)):
            assert torch.equal(a, b)
        say(f"tiles unseen 0x{fill:x} {dtype} over {cache} d={d} later tokens {len(sizes)}")
        for i, (_, n) in enumerate(sizes):
            seen[table[i, (n - 1) // 64].item(), (n - 1) % 64] = False
        spoil(pool, seen, fill)
        got = run_prompt(apc, *made, 0.125)
        last = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
        last[(starts[1:] - 1).long()] = True
        assert torch.isfinite(got[0][~last].float()).all()
        # (the rows' own sums, rounded otherwise: each call within half a step for the weights, of values of which the largest
        # is `most`, and half a step of the output)
        most = (pool[1].float() if pool[3] is None else pool[1].float() * pool[3][..., None])[seen[:, None].expand(pool[1].shape[:3])].abs().max()
        diff = (got[0][~last].float() - want[0][~last].float()).abs()
        assert (diff <= 2 * ROUND[dtype] * (most + want[0][~last].float().abs())).all()
        ends = torch.isneginf(want[1][~last])
        assert torch.equal(torch.isneginf(got[1][~last]), ends) and (got[1][~last] - want[1][~last])[~ends].abs().max() < 1e-5


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_infinite_values(apc, orc, dtype, d):
    """Infinite and NaN values reach the elements that they stand in of the rows that see them, and nothing else."""
    for sizes, heads, splits, pages in ((SOME, 52, 1, 4), (CUT, 128, 2, 40)):
        say(f"tiles infinite {dtype} d={d} {sizes}")
        pool, table, q, starts, lens = made = tall(make_prompt(19, sizes, heads, 1, d, 64, pages, dtype, dtype), dtype, splits)
        want, wl = run_prompt(apc, *made, d ** -0.5)
        n0, n1 = sizes[0][1], sizes[1][1]
        put = [(0, n0 - 3, 3, float("inf")), (0, n0 - 2, 3, float("-inf")), (0, n0 - 2, 5, float("-inf")), (1, n1 - 1, 7, float("nan")),
               (1, 20, d - 1, float("inf"))]
        for i, j, e, x in put:
            pool[1][table[i, j // 64].item(), 5, j % 64, e] = x
        got, gl = run_prompt(apc, *made, d ** -0.5)
        expect = want.float().clone()
        for i, (n, length) in enumerate(sizes[:2]):
            for r in range(n):
                sums = {}
                for i2, j, e, x in put:
                    if i2 == i and j <= length - n + r:
                        sums[e] = sums.get(e, 0.0) + x
                for e, x in sums.items():
                    expect[int(starts[i]) + r, 5, e] = x
        g = got.float()
        assert torch.equal(torch.isnan(g), torch.isnan(expect)) and torch.equal(torch.isinf(g), torch.isinf(expect))
        assert torch.equal(g[torch.isinf(g)], expect[torch.isinf(expect)])
        fine = torch.isfinite(expect)
        most = pool[1].float()[torch.isfinite(pool[1])].abs().max()
        assert ((g - expect).abs()[fine] <= 2 * ROUND[dtype] * (expect.abs()[fine] + most)).all()
        ends = torch.isneginf(wl)
        assert torch.equal(torch.isneginf(gl), ends) and (gl - wl)[~ends].abs().max() < 1e-5
        others = [h for h in range(heads) if h != 5]
        assert torch.equal(got[:, others], want[:, others]) and torch.equal(gl[:, others], wl[:, others])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tiles_scores_at_the_ends(apc, dtype):
    """Keys that score -inf drop out; a +inf score makes its row NaN, as a float32 softmax does; others stay."""
    pool, table, q, starts, lens = made = tall(make_prompt(29, SOME, 52, 1, 64, 16, 13, dtype, dtype), dtype)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    want = run_prompt(apc, *made, 0.125)
    k, at = pool[0], lambda j: (table[0, j // 16].item(), 3, j % 16)
    keep = k[at(99)].clone()
    k[at(99)][0] = float("inf")                              # seen by the first sequence's last row alone
    got = run_prompt(apc, *made, 0.125)
    assert torch.isnan(got[0][39, 3]).all() and torch.isnan(got[1][39, 3])
    rest = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    rest[39, 3] = False
    # (the NaN row's tile of 128 goes over its keys again: each call within half a step for the weights and for the output)
    diff, most = (got[0][rest].float() - want[0][rest].float()).abs(), pool[1].float().abs().max()
    assert (diff <= 2 * ROUND[dtype] * (most + want[0][rest].float().abs())).all()
    ends = torch.isneginf(want[1][rest])
    assert torch.equal(torch.isneginf(got[1][rest]), ends) and (got[1][rest] - want[1][rest])[~ends].abs().max() < 1e-5
    rest[:40, 3] = False
    assert torch.equal(got[0][rest], want[0][rest]) and torch.equal(got[1][rest], want[1][rest])
    k[at(99)] = keep
    for j in range(61):
        k[at(j)][0] = float("-inf")                          # all that the first row sees
    got = run_prompt(apc, *made, 0.125)
    assert not got[0][0, 3].any() and torch.isneginf(got[1][0, 3])
    assert torch.isfinite(got[0].float()).all() and torch.isfinite(got[1][1:40]).all()


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_tiles_scale_signs(apc, orc, cache, dtype, d, scale):
    made = tall(make_prompt(31, SIZES, 19, 2, d, 16, 13, cache, dtype), cache)
    check(orc, cache, dtype, made, scale, run_prompt(apc, *made, scale), heads=[0, 18])


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_light_weights(apc, orc, cache, dtype, d):
    """A heavy token whose value is 0 and many light ones that make the output."""
    pool, table, q, starts, lens = made = tall(make_prompt(37, [(70, 1000), (150, 2100)], 128, 1, d, 64, 40, cache, dtype), cache, 2)
    q.zero_()
    q[:, :, 0] = 1.0
    pool[0].view(torch.uint8).zero_()
    if pool[2] is not None:
        pool[2].fill_(1.0)
    for i in (0, 1):
        heavy = (table[i, 0].item(), slice(None), 5)
        pool[0][heavy][:, 0] = 14.0
        pool[1][heavy].view(torch.uint8).zero_()
    check(orc, cache, dtype, made, 1.0, run_prompt(apc, *made, 1.0), heads=[0, 64, 127])


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("slope", [1e6, 1e30, 3e38])
def test_tiles_steep_slopes(apc, cache, dtype, slope):
    """Slopes that leave each token itself alone: its value, and its own score."""
    for d in (64, 128, 256):
        say(f"tiles slope {slope} {dtype} over {cache} d={d}")
        made = tall(make_prompt(51, SIZES, 19, 2, d, 16, 13, cache, dtype), cache)
        out, lse = run_prompt(apc, *made, 0.125, slopes=torch.full((38,), slope, device="cuda"))
        alone, one = run_prompt(apc, *made, 0.125, window=1)
        at = torch.isfinite(one) & (one != 7)
        assert torch.equal(torch.isfinite(lse), torch.isfinite(one))
        # a weight rounded to the type over a sum of it unrounded, then the output's rounding, in each call: within
        # 2 ROUND (1 + ROUND) of the value each, 4.16 ROUND apart relative to a result
        diff = (out.float() - alone.float()).abs()[at]
        assert (diff <= 4.16 * ROUND[dtype] * alone.float().abs()[at] + TINY[dtype]).all()
        assert (lse - one)[at].abs().max() < 1e-4


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("size", [1e7, 1e12, 1e30])
def test_tiles_huge_scores(apc, cache, dtype, size):
    """Scores whose float32 steps are many times 1: a mean of the values with finite weights."""
    for d in (64, 128, 256):
        say(f"tiles scores of {size} {dtype} over {cache} d={d}")
        pool, table, q, starts, lens = made = tall(make_prompt(57, SIZES, 19, 2, d, 16, 13, cache, dtype), cache)
        out, lse = run_prompt(apc, *made, size)
        _, one = run_prompt(apc, *made, 0.0)
        v = pool[1].float() if pool[3] is None else pool[1].float() * pool[3][..., None]
        assert torch.isfinite(out.float()).all() and torch.equal(torch.isfinite(lse), torch.isfinite(one))
        # a mean lies within the values; its weights and itself are rounded
        assert out.float().abs().max() <= v.abs().max() * (1 + 3 * ROUND[dtype])


@pytest.mark.parametrize("cache,dtype", KINDS)
def test_tiles_cap_ends(apc, orc, cache, dtype):
    """Caps so small that every score is 0 but for less than float32 tells, and so large that none is bent."""
    made = tall(make_prompt(53, SIZES, 19, 2, 64, 16, 13, cache, dtype), cache)
    want = run_prompt(apc, *made, 0.125)
    some = torch.isfinite(want[1])
    v = made[0][1].float() if made[0][3] is None else made[0][1].float() * made[0][3][..., None]
    for cap in (1e-30, 1e-44, 1e30, 3.4e38):
        say(f"tiles cap {cap} {dtype} over {cache}")
        got = run_prompt(apc, *made, 0.125, cap=cap)
        if cap < 1:
            check(orc, cache, dtype, made, 0.0, got, heads=[0, 18])
        else:
            # (tanh is linear there: float32 carries x / cap as exactly as x)
            assert (got[1] - want[1])[some].abs().max() < 1e-4
            diff = (got[0].float() - want[0].float()).abs()
            assert (diff <= 2 * ROUND[dtype] * (want[0].float().abs() + v.abs().max())).all()


def test_tiles_views(apc):
    """Queries inside a fused product's rows, head-major outputs, page tables inside wider ones, no lse."""
    pool, table, q, starts, lens = made = tall(make_prompt(41, SIZES, 12, 4, 80, 16, 13, "bf16", "bf16", pad=2), "bf16")
    want, _ = run_prompt(apc, *made, 0.1)
    t, b = q.shape[0], len(SIZES)
    wide = torch.randn((t, 53, 83), device="cuda").to(torch.bfloat16)
    wide[:, 2:50, 1:81] = q
    out = torch.full((48, t, 90), 7.0, device="cuda").to(torch.bfloat16)
    tables = torch.full((b, 29), -9, dtype=torch.int32, device="cuda")
    tables[:, 3:16] = table
    c = apc.KvCache(*pool)
    ws = apc.attend_prompt_workspace_tensor(c, t, b, 48, 13)
    apc.apc_attend_prompt(c, wide[:, 2:50, 1:81], starts, tables[:, 3:16], lens, 0.1, out.transpose(0, 1)[:, :, 5:85], ws)
    torch.cuda.synchronize()
    assert torch.equal(out.transpose(0, 1)[:, :, 5:85], want)
    assert (out[:, :, :5] == 7).all() and (out[:, :, 85:] == 7).all()


def test_tiles_streams_and_graph(apc):
    """Calls with cut keys on two streams at once, with workspaces of their own, and captured and replayed with other
    queries in the same buffers: the results of calls alone."""
    work = []
    for seed, cache in ((1, "bf16"), (2, "e4m3")):
        pool, table, q, starts, lens = made = tall(make_prompt(seed, CUT, 128, 1, 64, 64, 40, cache, "bf16"), cache, 2)
        c = apc.KvCache(*pool)
        ws = apc.attend_prompt_workspace_tensor(c, q.shape[0], len(CUT), 128, 40)
        work.append((c, made, ws, torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")))

    def go(w, stream=None):
        c, (pool, table, q, starts, lens), ws, out, lse = w
        apc.apc_attend_prompt(c, q, starts, table, lens, 0.125, out, ws, lse, stream=stream)

    alone = []
    for w in work:
        go(w)
        torch.cuda.synchronize()
        alone.append((w[3].clone(), w[4].clone()))
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(5):
        for w in work:
            w[3].fill_(3.0)
        torch.cuda.synchronize()
        for w, s in zip(work, streams):
            go(w, s)
        torch.cuda.synchronize()
        for w, (o, l) in zip(work, alone):
            assert torch.equal(w[3], o) and torch.equal(w[4], l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for w in work:
            go(w)
    for turn in range(4):
        for w in work:
            w[1][2].copy_(torch.randn(w[1][2].shape, device="cuda", generator=gen(turn)))
            w[3].fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [(w[3].clone(), w[4].clone()) for w in work]
        for w, (o, l) in zip(work, got):
            go(w)
            torch.cuda.synchronize()
            assert torch.equal(w[3], o) and torch.equal(w[4], l)


def test_tiles_offsets_past_32_bits(apc, orc):
    """Pages, queries and outputs whose elements lie past 2^31."""
    page, heads, d, group = 1024, 8, 256, 4
    k = torch.zeros((1100, heads, page, d), dtype=torch.bfloat16, device="cuda")      # 2.3e9 elements
    v = torch.zeros_like(k)
    g = gen(3)
    for p in (0, 1098, 1099):
        k[p].copy_(torch.randn(k[p].shape, device="cuda", generator=g))
        v[p].copy_(torch.randn(v[p].shape, device="cuda", generator=g))
    table = torch.tensor([[1098, 0], [0, 1099]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([1500, 1030], dtype=torch.int32, device="cuda")
    t, hq, row = 1030, heads * group, 2_200_000              # 1,029 rows of it: 2.26e9 elements
    starts = torch.tensor([0, 700, t], dtype=torch.int32, device="cuda")
    big = torch.zeros(t * row, dtype=torch.bfloat16, device="cuda")
    q = big.as_strided((t, hq, d), (row, d, 1))
    q.copy_(torch.randn((t, hq, d), device="cuda", generator=g))
    tall(((k, v, None, None), table, q), "bf16")
    c = apc.KvCache(k, v)
    ws = apc.attend_prompt_workspace_tensor(c, t, 2, hq, 2)
    out, lse = big.as_strided((t, hq, d), (row, d, 1), hq * d), torch.empty((t, hq), device="cuda")
    apc.apc_attend_prompt(c, q, starts, table, lens, d ** -0.5, out, ws, lse)
    torch.cuda.synchronize()
    small = [torch.stack([x[1098], x[0], x[1099]]) for x in (k, v)]
    at = torch.tensor([[0, 1], [1, 2]], dtype=torch.int32, device="cuda")
    check(orc, "bf16", "bf16", ((small[0], small[1], None, None), at, q, starts, lens), d ** -0.5, (out, lse), heads=[0, 7])


# (sizes, heads, rows of a tile, parts of the keys) with pages of 64 tokens
FORMS = {"32 rows": ([(40, 300), (70, 100), (1, 129)], 2, 32, 1), "32 rows, cut": ([(1, 5000), (20, 2100)], 1, 32, 9),
         "128 rows": (SOME, 52, 128, 1), "128 rows, cut": (CUT, 128, 128, 2)}


def make_form(form, seed, group, d, cache, dtype, spread=1.0):
    sizes, heads, rows, splits = FORMS[form]
    made = make_prompt(seed, sizes, heads, group, d, 64, -(-max(n for _, n in sizes) // 64), cache, dtype, spread)
    p = plan_of(made, cache)
    assert (p.rows, p.splits) == (rows, splits), (p.rows, p.splits)
    return made, [h for h in (0, 30, 127) if h < heads]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_means_at_the_end_of_the_range(apc, orc, cache, form, d):
    """bf16 and scaled e4m3 values up to 3.36e38, all of a column of one sign, with like and unlike weights: their mean, not
    the sum's infinity; and huge values so far apart that each wave's, or each part's, sum is finite and not all of them."""
    made, heads = make_form(form, 73, 1, d, cache, "bf16")
    pool, table, q, starts, lens = made
    g, v = gen(9), pool[1]
    sign = torch.randint(0, 2, (d,), device="cuda", generator=g) * 2.0 - 1.0
    size = 0.5 + 0.49 * torch.rand(v.shape, device="cuda", generator=g)
    if cache == "e4m3":
        v.copy_(sign * size * 448.0)
        pool[3].fill_(3.39e38 / 448.0)
    else:
        v.copy_(sign * size * 3.39e38)
    for scale in (0.0, 0.125):
        say(f"range end {cache} {form} d={d} scale={scale}")
        check(orc, cache, "bf16", made, scale, run_prompt(apc, *made, scale), heads=heads)
    say(f"range end {cache} {form} d={d} apart")
    far = 32 if form == "32 rows" else 512 if form == "32 rows, cut" else 40 if form == "128 rows" else 1040
    for i, (_, n) in enumerate(FORMS[form][0]):
        j = torch.arange(n, device="cuda")
        j = j[j % far != 0]
        v.view(torch.uint8 if cache == "e4m3" else torch.int16)[table[i][j // 64].long(), :, j % 64] = 0
    check(orc, cache, "bf16", made, 0.0, run_prompt(apc, *made, 0.0), heads=heads)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("scale", [3e38, -3.4e38])
def test_scales_at_the_end_of_the_range(apc, orc, cache, dtype, form, scale):
    """Scales whose product with log2(e) is beyond float32: products of 0 score 0, and tiny ones what they should."""
    made, heads = make_form(form, 79, 1, 64, cache, dtype)
    pool, table, q, starts, lens = made
    say(f"scale {scale} {dtype} over {cache} {form}")
    p = torch.randint(-2, 3, pool[0].shape[:3], device="cuda", generator=gen(4)).float()
    q.zero_()
    pool[0].view(torch.uint8).zero_()
    # products of p 2^-122, scores of 56 p and more; f16 holds none so small
    if cache == "e4m3":
        pool[0][..., 0] = p.to(pool[0].dtype)
        q[..., 0] = 2.0 ** -10
        pool[2].fill_(2.0 ** -112)
    elif cache == "bf16":
        pool[0][..., 0] = (p * 2.0 ** -61).to(pool[0].dtype)
        q[..., 0] = 2.0 ** -61
    check(orc, cache, dtype, made, scale, run_prompt(apc, *made, scale), heads=heads)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_light_weights_over_f16_keep_their_bits(apc, orc, form, d):
    """Tokens of 2^-17 to 2^-47 of the heaviest weight, whose value is 0: they are the output, down to f16's last bits."""
    made, heads = make_form(form, 83, 1, d, "f16", "f16")
    pool, table, q, starts, lens = made
    q.zero_()
    q[:, :, :2] = 1.0
    pool[1].copy_(pool[1].abs().clamp(max=3.0) * 2.0e4)
    for gap in (12.0, 15.5, 19.0, 22.0, 25.0, 28.0, 32.0):
        say(f"light f16 {form} d={d} gap={gap}")
        pool[0][..., 2:] = 0
        pool[0][..., 0] = 0
        pool[0][..., 1].copy_(torch.rand(pool[0].shape[:3], device="cuda", generator=gen(5)))
        for i in range(len(lens)):
            for j in (0, 37):
                heavy = (table[i, 0].item(), slice(None), j)
                pool[0][heavy][:, 0] = gap
                pool[1][heavy] = 0
        check(orc, "f16", "f16", made, 1.0, run_prompt(apc, *made, 1.0), heads=heads)


MANY = {"32 rows": (3000, 3, 2, 32, 1), "128 rows": (1100, 90, 2, 128, 1), "empty": (2500, 0, 1, 32, 9)}


@pytest.mark.parametrize("name", MANY)
@pytest.mark.parametrize("cache,dtype", KINDS)
def test_many_sequences(apc, orc, cache, dtype, name):
    """More sequences than are looked through one by one, with rows of all of them, and of few whose keys are cut."""
    b, most, group, rows, splits = MANY[name]
    rng = np.random.default_rng(b)
    new = rng.integers(0, most + 1, b)
    sizes = [(int(n), int(n) + int(p)) for n, p in zip(new, rng.integers(0, 20, b))]
    if name == "empty":
        sizes[1023], sizes[1024], sizes[2499] = (2, 4700), (1, 30), (1, 5000)
        sizes = [(n, max(n, length if length > 20 else 0)) for n, length in sizes]
    else:
        sizes[700], sizes[b - 1] = (140, 150), (33, 40)
    say(f"many {name} {dtype} over {cache}")
    # (a pool that sequences share: random pages of it)
    pool, _, q, starts, lens = make_prompt(87, [(sum(n for n, _ in sizes), 5000)], 1, group, 64, 64, 79, cache, dtype, pad=5)
    starts = torch.from_numpy(np.concatenate([[0], np.cumsum([n for n, _ in sizes])])).to(torch.int32).cuda()
    lens = torch.tensor([n for _, n in sizes], dtype=torch.int32, device="cuda")
    pages = -(-max(n for _, n in sizes) // 64)
    table = torch.randint(0, pool[0].shape[0], (b, pages), dtype=torch.int32, device="cuda", generator=gen(6))
    made = pool, table, q, starts, lens
    p = plan_of(made, cache)
    assert (p.rows, p.splits) == (rows, splits), (p.rows, p.splits)
    check(orc, cache, dtype, made, 0.125, run_prompt(apc, *made, 0.125))


def test_a_million_sequences(apc):
    """Their time is not the square of their number, and each is what it is in a small call."""
    b = 2 ** 20
    pool, _, q, _, _ = make_prompt(89, [(b, 16 * 1000)], 1, 1, 16, 16, 1000, "bf16", "bf16")
    table = torch.randint(0, 1000, (b, 1), dtype=torch.int32, device="cuda", generator=gen(6))
    lens = torch.randint(0, 17, (b,), dtype=torch.int32, device="cuda", generator=gen(7))
    starts = torch.arange(b + 1, dtype=torch.int32, device="cuda")
    run_prompt(apc, pool, table[:2000], q[:2000], starts[:2001], lens[:2000], 0.25)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    say("a million sequences")
    begin.record()
    out, lse = run_prompt(apc, pool, table, q, starts, lens, 0.25)
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 500.0                   # (ms; each looked through one by one: 4,000)
    for i in (0, 500_000, b - 700):
        some = slice(i, i + 700)
        a, e = run_prompt(apc, pool, table[some], q[some], starts[:701], lens[some], 0.25)
        assert torch.equal(a, out[some]) and torch.equal(e, lse[some])
