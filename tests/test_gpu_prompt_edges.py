"""Corners of the prompt model's operators against float64."""
import numpy as np
import pytest
import torch

from tests.gpu_check import say
from tests.test_gpu_prompt_ops import KINDS, ROUND, TINY, TORCH, U, check_attend, check_norm, f64, gen, make_attend, run_attend, stored

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def apc():
    import paper_2502_06798_amd as apc
    apc.load()
    assert torch.cuda.is_available()
    return apc


# ---- attention: many query heads -----------------------------------------------

@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("group,d", [(8193, 64), (8193, 128), (4097, 256), (20000, 128)])
def test_attend_more_query_tiles_than_compute_units(apc, orc, cache, dtype, group, d):
    """One key-value head for thousands of query heads over tables that are cut: every output is written."""
    say(f"attend query tiles {dtype} over {cache} group={group} d={d}")
    lens = [3000, 0, 70]
    pool, table, q = make_attend(group + d, len(lens), 1, group, d, 64, 47, cache, dtype)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, pool, table, q, n, d ** -0.5)
    assert torch.equal(torch.isneginf(lse).all(dim=1).cpu(), torch.tensor([False, True, False]))
    assert (out[1] == 0).all() and not (out[::2] == 7.0).all(dim=2).any() and not (lse == 7.0).any()
    at = torch.tensor([0, 15, 16, 31, 32, group // 2, group - 2, group - 1], device="cuda")
    check_attend(orc, cache, dtype, pool, table, q[:, at], n, d ** -0.5, 0, out[:, at], lse[:, at])


def test_attend_empty_sequence_of_2_to_31_elements(apc):
    """A sequence that holds nothing, its output of 2^31 elements: all of them are written."""
    heads, group, d, page = 1 << 19, 16, 256, 16
    say("attend 2^31 elements of an empty sequence")
    k, v = (torch.empty((1, heads, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = apc.KvCache(k, v)
    q = torch.empty((1, heads * group, d), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    table, lens = torch.zeros((1, 128), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    apc.apc_attend(c, q, table, lens, 0.1, out, apc.attend_workspace_tensor(c, 1, heads * group, 128), lse)
    torch.cuda.synchronize()
    assert not out.view(torch.int32).any() and torch.isneginf(lse).all()


# ---- attention: chosen scores and values ------------------------------------------

def one_sequence(cache, dtype, n, d, page=64):
    """A pool with one sequence of n tokens, keys and values 0; setters of a token's row (exact in the cache's type)."""
    mp = -(-n // page)
    pool = [torch.zeros((mp, 1, page, d), device="cuda").to(TORCH[cache]) for _ in range(2)]
    pool += [torch.ones((mp, 1, page), device="cuda") if cache == "e4m3" else None for _ in range(2)]
    table = torch.arange(mp, dtype=torch.int32, device="cuda")[None].contiguous()
    return pool, table, torch.tensor([n], dtype=torch.int32, device="cuda")


def put(pool, j, row):
    """row into token j of the pool's first sequence (pages in order)."""
    page = pool.shape[2]
    raw = row.to(pool.dtype)
    if pool.element_size() == 1:
        pool.view(torch.uint8)[j // page, 0, j % page] = raw.view(torch.uint8)
    else:
        pool[j // page, 0, j % page] = raw


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("below,value", [(15.0, 1.0), (17.4, 1.0), (17.4, 96.0), (22.0, 96.0), (25.0, 208.0)])
def test_attend_light_weights_beside_a_heavy_one(apc, cache, dtype, below, value):
    """One token takes nearly all the weight and has the value 0; the others' many small weights make the output."""
    n, d, at = 32769, 64, 12345
    say(f"attend light {dtype} over {cache} below={below} value={value}")
    pool, table, lens = one_sequence(cache, dtype, n, d)
    pool[1].copy_(torch.full(pool[1].shape, value, device="cuda"))
    heavy = torch.zeros(d, device="cuda")
    heavy[0] = below                                         # exact in every type (e4m3: 15, 17.4 -> 18, 22, 25 -> 24 or 26)
    put(pool[0], at, heavy)
    put(pool[1], at, torch.zeros(d, device="cuda"))
    q = torch.zeros((1, 3, d), device="cuda").to(TORCH[dtype])
    q[..., 0] = 1.0
    out, lse = run_attend(apc, pool, table, q, lens, 1.0)
    s = float(pool[0].float()[at // 64, 0, at % 64, 0])      # the heavy score as the cache holds it
    rest = (n - 1) * np.exp(-s)
    want = value * rest / (1 + rest)
    # one score of one product, the others 0: the exponent's argument to 2 u s, the sums of n equal terms to n u at most
    # and in blocks here (at most n / 128 + 64 additions on any path), weights to 2^-16
    tol = want * (4 * U * s + 2 * (n / 128 + 64) * U + 2.0 ** -16 + ROUND[dtype] * 1.001) + TINY[dtype]
    assert (np.abs(f64(out) - want) <= tol).all(), (f64(out).ravel()[0], want)
    assert (np.abs(f64(lse) - (s + np.log1p(rest))) <= 2.0 ** -20 * s + 64 * U).all()


def reference(q, k, v, scale):
    """(out, lse, tol of out without the output's rounding) of one sequence and head, float64 rows k, v; tokens whose
    score is -inf leave the sums (their weight is 0) but for infinite and NaN values, which 0 turns into NaN."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (k @ q)
        w = np.exp(s - s.max())
        out = (w[:, None] * v).sum(axis=0) / w.sum()
        some = np.isfinite(s)
        e = (k.shape[1] + 24) * U * (np.abs(scale) * (np.abs(k[some]) @ np.abs(q)).max())
        spread = (w[some, None] * np.abs(v[some])).sum(axis=0) / w.sum()
        return out, s.max() + np.log(w.sum()), spread * (4 * e + 2 * (len(s) + 64) * U + 2.0 ** -16), 2 * e + (len(s) + 64) * U


def rows_of(orc, cache, pool, scale, table, n):
    """float64 rows of the first n tokens of the only sequence, head 0."""
    x = orc.kv_values(cache, stored(pool))
    with np.errstate(invalid="ignore"):
        if scale is not None:
            x = x * scale.cpu().numpy().astype(np.float64)[..., None]
    return np.concatenate([x[p, 0] for p in table[0].tolist()])[:n]


def check_one(orc, cache, dtype, pool, table, q, n, scale, out, lse):
    k, v = rows_of(orc, cache, pool[0], pool[2], table, n), rows_of(orc, cache, pool[1], pool[3], table, n)
    got, gl = f64(out)[0], f64(lse)[0]
    for h in range(q.shape[1]):
        want, wl, tol, ltol = reference(f64(q)[0, h], k, v, scale)
        some = np.isfinite(want)
        assert np.array_equal(got[h][~some], want[~some], equal_nan=True), (got[h][~some], want[~some])
        bad = ~(np.abs(got[h] - want)[some] <= (tol + np.abs(want) * ROUND[dtype] * 1.001 + TINY[dtype])[some])
        assert not bad.any(), (np.abs(got[h] - want)[some][bad].max())
        assert abs(gl[h] - wl) <= ltol + 2.0 ** -20 * abs(wl)


LONG = [5, 70, 333, 5000]


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("group,d", [(1, 16), (3, 64), (5, 80), (4, 128), (20, 128), (2, 192), (18, 256)])
def test_attend_infinite_values(apc, orc, cache, dtype, group, d):
    """An infinite value of a token with weight makes its element infinite, two of different sign or a NaN make it NaN,
    and the other elements are what they were."""
    for n in LONG:
        say(f"attend infinite values {dtype} over {cache} group={group} d={d} n={n}")
        pool, table, q = make_attend(d + n, 1, 1, group, d, 16, -(-n // 16), cache, dtype)
        lens = torch.tensor([n], dtype=torch.int32, device="cuda")
        at = lambda j: (table[0, j // 16].item(), 0, j % 16)
        if cache == "e4m3":
            code = pool[1].view(torch.uint8)
            code[at(n - 1)][:6] = torch.tensor([0x7e, 0xfe, 0x00, 0x01, 0x81, 0x7f], dtype=torch.uint8, device="cuda")
            pool[3][at(n - 1)] = float("inf")
        else:
            v = pool[1]
            v[at(0)][1], v[at(n - 1)][2] = float("inf"), float("-inf")
            v[at(n // 2)][3], v[at(1)][3] = float("inf"), float("inf")
            v[at(n // 3)][4], v[at(n - 1)][4] = float("inf"), float("-inf")
            v[at(n // 2)][5], v[at(n - 1)][d - 1] = float("nan"), float("inf")
        scale = 0.02 if cache == "e4m3" else d ** -0.5       # no token's weight vanishes
        pool[2] is None or pool[2].clamp_(max=0.3)
        out, lse = run_attend(apc, pool, table, q, lens, scale)
        check_one(orc, cache, dtype, pool, table, q, n, scale, out, lse)
        again = run_attend(apc, pool, table, q, lens, scale)
        assert torch.equal(out.view(torch.int16), again[0].view(torch.int16)) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group,d", [(1, 16), (2, 48), (3, 64), (5, 80), (2, 96), (4, 128), (20, 112), (2, 144), (2, 192), (4, 256)])
def test_attend_infinite_keys(apc, orc, dtype, group, d):
    """A key that scores minus infinity has no weight, whatever its other elements and the head's size."""
    for n in LONG:
        say(f"attend infinite keys {dtype} group={group} d={d} n={n}")
        pool, table, q = make_attend(d + n, 1, 1, group, d, 16, -(-n // 16), dtype, dtype)
        lens = torch.tensor([n], dtype=torch.int32, device="cuda")
        at = lambda j: (table[0, j // 16].item(), 0, j % 16)
        for e in (0, 7, d - 1):
            q[..., e] = q[..., e].abs() + 0.25
        for j, e in ((0, 0), (n - 2, 7), (n // 2, d - 1)):
            pool[0][at(j)][e] = float("-inf")
        pool[0][at(n // 2)][0] = float("-inf")
        out, lse = run_attend(apc, pool, table, q, lens, d ** -0.5)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        check_one(orc, dtype, dtype, pool, table, q, n, d ** -0.5, out, lse)
        pool[0][table[0].long(), 0, :, 0] = float("-inf")     # no token scores above it
        out, lse = run_attend(apc, pool, table, q, lens, d ** -0.5)
        assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("n", [300, 9000])
def test_attend_values_at_the_end_of_the_range(apc, orc, cache, dtype, n):
    """Two tokens of values near float32's largest, the later one with the larger score: their mean is finite."""
    say(f"attend large values {dtype} over {cache} n={n}")
    d = 64
    pool, table, lens = one_sequence(cache, dtype, n, d)
    for j, score in ((0, 0.0), (256, 4.0)):
        row = torch.zeros(d, device="cuda")
        row[0], row[1] = score, 30.0
        put(pool[0], j, row)
        put(pool[1], j, torch.full((d,), 448.0 if cache == "e4m3" else 3.0e38, device="cuda"))
        if cache == "e4m3":
            pool[3][j // 64, 0, j % 64] = 6.7e35
    q = torch.zeros((1, 2, d), device="cuda").to(TORCH[dtype])
    q[..., 0], q[..., 1] = 1.0, 1.0
    out, lse = run_attend(apc, pool, table, q, lens, 1.0)
    assert torch.isfinite(out).all()
    check_one(orc, cache, dtype, pool, table, q, n, 1.0, out, lse)


# ---- norm ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("to8", [False, True])
@pytest.mark.parametrize("size,weight", [(1e16, 1e25), (1e-15, 1e-30), (1e-18, 1e-25), (1e-8, 1e-33)])
def test_norm_weights_far_from_one(apc, orc, dtype, to8, size, weight):
    """h w leaves float32's range, or its normal part, where the normed row times w does not."""
    for n, d in ((3, 3), (5, 48), (2, 999), (3, 4096), (2, 20000)):
        say(f"norm extremes {dtype} to8={to8} n={n} d={d} size={size} weight={weight}")
        g = gen(n + d)
        x = (torch.randn((n, d), device="cuda", generator=g) * size).to(TORCH[dtype])
        w = ((1 + torch.rand(d, device="cuda", generator=g)) * weight).to(TORCH[dtype])
        out = torch.zeros((n, d), device="cuda").to(TORCH["e4m3" if to8 else dtype])
        scale = torch.zeros(n, device="cuda") if to8 else None
        apc.apc_norm_rows(x, out, w, None, None, scale, 0.0)
        torch.cuda.synchronize()
        check_norm(orc, x, None, w, out, scale, None, 0.0, dtype)
