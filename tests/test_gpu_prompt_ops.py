"""GPU parity of the prompt model's operators against the float64 oracle.

Tolerances, u = 2^-24 (a float32 operation's rounding), ulp(out) the output
type's unit roundoff:
* norm: the sum of d squares takes at most 64 additions in a row on any path
  (a thread's, then a tree), halved by the square root; with the residual's
  addition, root, division and two products at most 40 u, taken as 64 u =
  2^-18.  Then one rounding to the output's type.  e4m3: the scale within
  2^-17, and each code nearest to y / scale within that.
* cache: bit for bit.
* attention: a score's error is at most e = (d + 16) u top + 8 u |s| (top =
  scale * sum |q k|, a d-term sum, the scales and the exponent's argument), so
  weights are off by a factor of at most 1 + 2 e and the output by 2 (2 e)
  spread; its own sums and the sum of weights by 2 (n + 64) u spread (n
  tokens); the weights' two 16-bit parts hold them to 2^-16.  Then one
  rounding to the output's type.  lse: 2 e + (n + 64) u + 2^-20 |lse|.
"""
import numpy as np
import pytest
import torch

from tests.gpu_check import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}   # half the smallest subnormal


@pytest.fixture(scope="module")
def apc():
    import paper_2502_06798_amd as apc
    apc.load()
    assert torch.cuda.is_available()
    return apc


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---- norm --------------------------------------------------------------------

def half_step(v):
    """Half the distance between neighbouring e4m3 values around |v| (the larger one at a power of two)."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def check_norm(orc, x, res, w, out, scale, total, eps, dtype):
    y, h = orc.norm_rows(f64(x), None if res is None else f64(res), None if w is None else f64(w), eps)
    if total is not None:
        assert (np.abs(f64(total) - h) <= np.abs(h) * (ROUND[dtype] + U) * 1.0001 + TINY[dtype]).all()
    if scale is None:
        got = f64(out)
        tol = np.abs(y) * (2.0 ** -18 + ROUND[dtype] * 1.001) + TINY[dtype] + 1e-44
        assert np.array_equal(np.isnan(got), np.isnan(y))
        bad = np.abs(got - y) > tol
        assert not bad[~np.isnan(y)].any(), np.abs(got - y)[bad].max()
        return
    s = f64(scale)
    top = np.abs(y).max(axis=1)
    want = np.where(top > 0, top / 448.0, 1.0)
    assert (np.abs(s - want) <= want * 2.0 ** -17).all()
    t, got = y / s[:, None], f64(out)
    assert (np.abs(got - t) <= half_step(np.maximum(np.abs(t), np.abs(got))) + np.abs(t) * 2.0 ** -16).all()


SHAPES = [(1, 1), (3, 2), (5, 15), (1, 64), (257, 77), (64, 256), (33, 511), (33, 512), (16, 768), (7, 999), (9, 1000),
          (5, 1024), (5, 1025), (3, 2047), (1030, 2048), (3, 2056), (4, 4096), (2, 4097), (2, 5000), (3, 8192),
          (2, 8200), (1, 16384), (2, 16388), (2, 32767), (1, 32768)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("to8", [False, True])
def test_norm_shapes(apc, orc, dtype, to8):
    for n, d in SHAPES:
        for mode in ("plain", "res", "res+sum"):
            say(f"norm {dtype} to8={to8} n={n} d={d} {mode}")
            g = gen(n * 7 + d)
            mk = lambda: (torch.randn((n, d), device="cuda", generator=g)
                          * torch.exp(torch.randn((n, 1), device="cuda", generator=g) * 2)).to(TORCH[dtype])
            x, w = mk(), (1 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(TORCH[dtype])
            res = mk() if mode != "plain" else None
            total = torch.full((n, d), 7.0, device="cuda").to(TORCH[dtype]) if mode == "res+sum" else None
            out = torch.zeros((n, d), device="cuda").to(TORCH["e4m3" if to8 else dtype])
            scale = torch.zeros(n, device="cuda") if to8 else None
            apc.apc_norm_rows(x, out, w if mode != "res" else None, res, total, scale, 1e-6)
            torch.cuda.synchronize()
            check_norm(orc, x, res, w if mode != "res" else None, out, scale, total, 1e-6, dtype)


@pytest.mark.parametrize("dtype,d,pad,shift", [("f32", 768, 4, 0), ("f32", 999, 6, 1), ("f16", 768, 8, 8),
                                               ("f16", 768, 3, 5), ("bf16", 4096, 8, 0), ("bf16", 1001, 1, 3),
                                               ("bf16", 512, 2, 2), ("f16", 40, 24, 8)])
@pytest.mark.parametrize("to8", [False, True])
def test_norm_strided_rows(apc, orc, dtype, d, pad, shift, to8):
    """Views into wider rows, at any element; what lies between the rows stays as it was."""
    say(f"norm strided {dtype} d={d} pad={pad} shift={shift} to8={to8}")
    n, g = 37, gen(d + pad)
    wide = lambda: torch.randn((n, d + pad + shift), device="cuda", generator=g).to(TORCH[dtype])
    xw, rw, sw = wide(), wide(), wide()
    ow = torch.full((n, d + pad + shift), 3.0, device="cuda").to(TORCH["e4m3" if to8 else dtype])
    before = sw.clone()
    cut = lambda t: t[:, shift:shift + d]
    w = torch.randn(d + 1, device="cuda", generator=g).to(TORCH[dtype])[1:]
    scale = torch.zeros(n + 1, device="cuda")[1:] if to8 else None
    apc.apc_norm_rows(cut(xw), cut(ow), w, cut(rw), cut(sw), scale, 1e-5)
    torch.cuda.synchronize()
    check_norm(orc, cut(xw), cut(rw), w, cut(ow), scale, cut(sw), 1e-5, dtype)
    for t, was in ((sw, before.float()), (ow, torch.full_like(ow, 3.0).float())):
        t = t.float()
        assert torch.equal(t[:, :shift], was[:, :shift]) and torch.equal(t[:, shift + d:], was[:, shift + d:])


@pytest.mark.parametrize("dtype,d", [("f32", 768), ("bf16", 4096), ("f16", 999), ("bf16", 16384)])
def test_norm_in_place(apc, orc, dtype, d):
    """The residual updated in place, and the norm over x's own rows, equal the calls with buffers of their own."""
    g = gen(d)
    x, r = (torch.randn((19, d), device="cuda", generator=g).to(TORCH[dtype]) for _ in range(2))
    out, total = torch.empty_like(x), torch.empty_like(x)
    apc.apc_norm_rows(x, out, None, r, total)
    x2, r2 = x.clone(), r.clone()
    apc.apc_norm_rows(x2, x2, None, r2, r2)
    x3, out3 = x.clone(), torch.empty_like(x)
    apc.apc_norm_rows(x3, out3, None, r, x3)
    torch.cuda.synchronize()
    check_norm(orc, x, r, None, out, None, total, 1e-6, dtype)
    assert torch.equal(x2, out) and torch.equal(r2, total) and torch.equal(x3, total) and torch.equal(out3, out)


@pytest.mark.parametrize("d", [48, 999, 4096])
def test_norm_special_rows(apc, d):
    """Zero rows, NaN, infinity, overflowing squares; a neighbour's row is not touched by any of it."""
    x = torch.randn((6, d), device="cuda", generator=gen(3))
    x[0] = 0.0
    x[1, d // 2] = float("nan")
    x[2, d - 1] = float("inf")
    x[3] = 1e30
    x[4] = 1e-30
    out, codes, s = torch.empty_like(x), torch.empty((6, d), dtype=TORCH["e4m3"], device="cuda"), torch.empty(6, device="cuda")
    apc.apc_norm_rows(x, out)
    apc.apc_norm_rows(x, codes, out_scale=s)
    alone, alone_s = torch.empty((1, d), dtype=TORCH["e4m3"], device="cuda"), torch.empty(1, device="cuda")
    apc.apc_norm_rows(x[5:], alone, out_scale=alone_s)
    torch.cuda.synchronize()
    o, c = out.cpu(), codes.float().cpu()
    assert (o[0] == 0).all() and (c[0] == 0).all() and s[0] == 1
    assert o[1].isnan().all() and c[1].isnan().all() and s[1] == 1
    assert o[2, -1].isnan() and (o[2, :-1] == 0).all()               # inf * 0, and finite * 0
    assert (o[3] == 0).all() and (c[3] == 0).all()                   # the sum of squares overflows
    assert torch.allclose(o[4], x[4].cpu() * 1e3, rtol=1e-5)         # eps rules
    assert torch.equal(codes[5:].view(torch.uint8), alone.view(torch.uint8)) and torch.equal(s[5:], alone_s)
    z = torch.zeros((1, d), device="cuda")
    apc.apc_norm_rows(z, z, eps=0.0)
    torch.cuda.synchronize()
    assert z.isnan().all()


def test_norm_rows_are_queries(apc, orc):
    """e4m3 rows and scales from the norm are what apc_match_batch takes: each row finds itself."""
    x = torch.randn((300, 768), device="cuda", generator=gen(5)).to(torch.bfloat16)
    e, s = torch.empty((300, 768), dtype=TORCH["e4m3"], device="cuda"), torch.empty(300, device="cuda")
    apc.apc_norm_rows(x, e, out_scale=s)
    c = apc.apc_build_cache(e, s)
    ts, ti = torch.empty((300, 1), device="cuda"), torch.empty((300, 1), dtype=torch.int32, device="cuda")
    apc.apc_match_batch(c, e, s, 1, ts, ti, apc.workspace_tensor(c, 300, 1))
    torch.cuda.synchronize()
    assert torch.equal(ti[:, 0].cpu(), torch.arange(300, dtype=torch.int32))
    c.close()


def test_norm_many_rows(apc, orc):
    """More rows than one launch has workgroups for."""
    n, d = (1 << 20) * 5 + 3, 8
    x = torch.randn((n, d), device="cuda", generator=gen(6)).to(torch.float16)
    out = torch.zeros_like(x)
    apc.apc_norm_rows(x, out)
    torch.cuda.synchronize()
    at = np.r_[0:50, (1 << 20) - 3:(1 << 20) + 3, (1 << 22) - 3:(1 << 22) + 3, n - 50:n]
    check_norm(orc, x[at], None, None, out[at], None, None, 1e-6, "f16")
    assert (out.abs().amax(dim=1) > 0).all()


# ---- cache -------------------------------------------------------------------

def stored(t):
    """Host copy of a pool's stored elements."""
    return t.view(torch.uint8).cpu().numpy() if t.element_size() == 1 else \
        t.view(torch.int16).cpu().numpy().view(np.float16 if t.dtype == torch.float16 else np.uint16)


def make_pool(n_pages, heads, page, d, dtype, fill=None):
    """Pages filled with a byte (stale memory: codes, halves and scales that decode to anything)."""
    k, v = (torch.empty((n_pages, heads, page, d), dtype=TORCH[dtype], device="cuda") for _ in range(2))
    ks, vs = ((torch.empty((n_pages, heads, page), device="cuda") for _ in range(2)) if dtype == "e4m3" else (None, None))
    for t in (k, v, ks, vs):
        if t is not None and t.numel():
            t.view(torch.uint8).fill_(0x3c if fill is None else fill)
    return k, v, ks, vs


def same_bits(a, b):
    return np.array_equal(a.view(np.uint8), b.view(np.uint8))


@pytest.mark.parametrize("cache", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_kv_write_read_bit_exact(apc, orc, cache, dtype):
    for t, heads, d, page, how in ((1, 1, 16, 16, "plain"), (5, 3, 64, 16, "fused"), (33, 2, 80, 32, "odd"),
                                   (130, 8, 128, 64, "fused"), (19, 5, 176, 128, "heads"), (40, 12, 64, 1024, "plain"),
                                   (7, 1, 256, 16, "odd"), (9, 2, 48, 16, "expand")):
        say(f"kv {dtype}->{cache} t={t} heads={heads} d={d} page={page} {how}")
        g, n_pages = gen(t + d), max(1, 2 * t // page) + 1
        rows = lambda *s: (torch.randn(s, device="cuda", generator=g)
                           * torch.exp(torch.randn(s[:-1] + (1,), device="cuda", generator=g) * 3)).to(TORCH[dtype])
        if how == "fused":                                # views into one product's rows
            x = rows(t, 3 * heads, d)
            k, v = x[:, heads:2 * heads], x[:, 2 * heads:]
        elif how == "odd":                                # rows that start at any element
            k, v = rows(t, heads, d + 3)[..., 3:], rows(t, heads, d + 1)[..., :d]
        elif how == "heads":                              # heads outermost
            k, v = rows(heads, t, d).transpose(0, 1), rows(heads, t, d).transpose(0, 1)
        elif how == "expand":                             # one row for every head
            k, v = rows(t, 1, d).expand(t, heads, d), rows(t, 1, d).expand(t, heads, d)
        else:
            k, v = rows(t, heads, d), rows(t, heads, d)
        if how == "plain":
            k[0, 0], v[0, 0, 3], v[t // 2, heads - 1] = 0.0, float("nan"), 1e-7
            k[t - 1, heads - 1, d - 1] = float("inf")
            k[t // 3, 0, ::2], v[0, 0, :3] = -0.0, -0.0
            v[t // 3, 0], v[t // 4, 0] = -0.0, 3e-39
        slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:t].to(torch.int32)
        if t > 4:
            slots[1], slots[2], slots[3], slots[4] = -1, n_pages * page, -2 ** 31, 2 ** 31 - 1
        kp, vp, ks, vs = make_pool(n_pages, heads, page, d, cache)
        want = [stored(p).copy() for p in (kp, vp)]
        wants = [None if s is None else s.cpu().numpy().copy() for s in (ks, vs)]
        c = apc.KvCache(kp, vp, ks, vs)
        apc.apc_kv_write(c, k, v, slots)
        torch.cuda.synchronize()
        for x, pool, w, s, ws in ((k, kp, want[0], ks, wants[0]), (v, vp, want[1], vs, wants[1])):
            orc.kv_write(cache, w, ws, x.float().cpu().numpy(), slots.cpu().numpy())
            assert same_bits(stored(pool), w)
            assert s is None or same_bits(s.cpu().numpy(), ws)
        for out in ("f32", "f16", "bf16"):
            ko, vo = torch.full((t, heads, d + 2), 5.0, device="cuda").to(TORCH[out]), torch.empty((heads, t, d), device="cuda").to(TORCH[out])
            apc.apc_kv_read(c, slots, ko[..., :d] if how == "odd" else ko[..., 2:], vo.transpose(0, 1))
            torch.cuda.synchronize()
            for got, w, ws in ((ko[..., :d] if how == "odd" else ko[..., 2:], want[0], wants[0]), (vo.transpose(0, 1), want[1], wants[1])):
                ref = orc.kv_read(cache, w, ws, slots.cpu().numpy(), out)
                ref = ref if out == "f32" else orc.kv_values(out, ref)
                a, b = f64(got), np.asarray(ref, dtype=np.float64)
                assert np.array_equal(a, b, equal_nan=True)
            edge = ko[..., d:] if how == "odd" else ko[..., :2]
            assert (edge == 5.0).all()


def test_kv_empty_and_many(apc, orc):
    """No tokens, no pages; and more rows than one launch has workgroups for."""
    kp, vp, ks, vs = make_pool(0, 2, 16, 32, "e4m3")
    c = apc.KvCache(kp, vp, ks, vs)
    z = torch.zeros((3, 2, 32), device="cuda")
    apc.apc_kv_write(c, z[:0], z[:0], torch.zeros(0, dtype=torch.int32, device="cuda"))
    apc.apc_kv_write(c, z, z, torch.arange(3, dtype=torch.int32, device="cuda"))        # every slot is outside
    o = torch.ones_like(z)
    apc.apc_kv_read(c, torch.arange(3, dtype=torch.int32, device="cuda"), o, o.clone())
    torch.cuda.synchronize()
    assert (o == 0).all()
    heads, d, page, n_pages = 64, 16, 1024, 160
    t = n_pages * page
    kp, vp, ks, vs = make_pool(n_pages, heads, page, d, "e4m3")
    x = torch.randn((t, heads, d), device="cuda", generator=gen(8)).to(torch.bfloat16)
    slots = torch.randperm(t, device="cuda", generator=gen(9)).to(torch.int32)
    c = apc.KvCache(kp, vp, ks, vs)
    apc.apc_kv_write(c, x, -x, slots)
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    apc.apc_kv_read(c, slots, ko, vo)
    torch.cuda.synchronize()
    assert torch.equal(ko, -vo)
    at = np.r_[0:20, t // 2:t // 2 + 20, t - 20:t]
    rows, sc = orc.quantize_rows("e4m3", x[at].float().cpu().numpy().reshape(-1, d))
    want = (orc.kv_values("e4m3", rows).astype(np.float32) * sc[:, None]).reshape(len(at), heads, d)
    assert np.array_equal(f64(ko[at]), f64(torch.from_numpy(want).to(torch.bfloat16)))


@pytest.mark.parametrize("cache", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("t,heads,d", [(8195, 32, 32), (8197, 17, 64), (4099, 16, 80), (2051, 17, 176)])
def test_kv_large_calls_are_small_calls(apc, cache, dtype, t, heads, d):
    """Calls whose lanes go on to several tokens leave the bits that calls of 300 tokens leave, slots outside the pool among them."""
    say(f"kv large {dtype}->{cache} t={t} heads={heads} d={d}")
    page, g = 64, gen(t + d)
    n_pages = t // page + 3
    x = (torch.randn((t, 2 * heads, d), device="cuda", generator=g)
         * torch.exp(torch.randn((t, 2 * heads, 1), device="cuda", generator=g) * 3)).to(TORCH[dtype])
    k, v = x[:, :heads], x[:, heads:]
    slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:t].to(torch.int32)
    slots[::7] = -1
    slots[t - 2] = n_pages * page
    one, many = (apc.KvCache(*make_pool(n_pages, heads, page, d, cache)) for _ in range(2))
    apc.apc_kv_write(one, k, v, slots)
    for i in range(0, t, 300):
        apc.apc_kv_write(many, k[i:i + 300], v[i:i + 300], slots[i:i + 300])
    for a, b in zip((one.k, one.v, one.k_scale, one.v_scale), (many.k, many.v, many.k_scale, many.v_scale)):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    got, want = (torch.full((2, t, heads, d), 5.0, device="cuda").to(TORCH[dtype]) for _ in range(2))
    apc.apc_kv_read(one, slots, got[0], got[1])
    for i in range(0, t, 300):
        apc.apc_kv_read(one, slots[i:i + 300], want[0, i:i + 300], want[1, i:i + 300])
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    out = (slots < 0) | (slots >= n_pages * page)
    top = torch.stack([k, v])[:, ~out].float().abs().amax(dim=3)
    some = torch.isfinite(top) & (top > 1e-4)                # a half's rows reach infinity here and there
    assert some.float().mean() > 0.9
    assert (got[:, out] == 0).all() and (got[:, ~out].float().abs().amax(dim=3)[some] > 0).all()


# ---- attention ---------------------------------------------------------------

def make_attend(seed, b, heads, group, d, page, max_pages, cache, dtype, extra=3, spread=1.0):
    g, n_pages = gen(seed), b * max_pages + extra
    kp, vp, ks, vs = make_pool(n_pages, heads, page, d, cache)
    for p, s in ((kp, ks), (vp, vs)):
        x = torch.randn((n_pages, heads, page, d), device="cuda", generator=g)
        if s is None:
            p.copy_(x)
        else:
            s.copy_(x.abs().amax(dim=3) / 448 * torch.exp(torch.randn(s.shape, device="cuda", generator=g)))
            p.copy_((torch.randint(-448, 449, x.shape, device="cuda", generator=g)).float())
            s.mul_(0.3)
    table = torch.randperm(n_pages, device="cuda", generator=g)[:b * max_pages].to(torch.int32).reshape(b, max_pages)
    q = (torch.randn((b, heads * group, d), device="cuda", generator=g) * spread).to(TORCH[dtype])
    return (kp, vp, ks, vs), table, q


def run_attend(apc, pool, table, q, lens, scale, window=0, stream=None, **kw):
    c = apc.KvCache(*pool)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    ws = apc.attend_workspace_tensor(c, q.shape[0], q.shape[1], table.shape[1])
    ws.fill_(0xff)                                           # nothing in it needs to start at zero
    apc.apc_attend(c, q, table, lens, scale, out, ws, lse, window)
    torch.cuda.synchronize()
    return out, lse


def check_attend(orc, cache, dtype, pool, table, q, lens, scale, window, out, lse):
    k, v, ks, vs = pool
    host = lambda t: None if t is None else t.cpu().numpy()
    d, n = q.shape[2], table.shape[1] * k.shape[2]
    with np.errstate(invalid="ignore", over="ignore"):
        ro, rl, spread, top = orc.attend(cache, f64(q), stored(k), stored(v), host(ks), host(vs), host(table), host(lens),
                                         scale, window)
    e = (d + 16) * U * top + 8 * U * top
    got, gl = f64(out), f64(lse)
    tol = spread * (4 * e + 2 * (n + 64) * U + 2.0 ** -16)[..., None] + np.abs(ro) * ROUND[dtype] * 1.001 + TINY[dtype]
    bad = ~(np.abs(got - ro) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - ro)[bad].max())
    assert np.array_equal(np.isneginf(gl), np.isneginf(rl))
    some = ~np.isneginf(rl)
    assert (np.abs(gl - rl)[some] <= (2 * e + (n + 64) * U + 2.0 ** -20 * np.abs(rl))[some]).all()
    assert (got[np.isneginf(rl)] == 0).all()


KINDS = [("f16", "f16"), ("bf16", "bf16"), ("e4m3", "f16"), ("e4m3", "bf16")]
LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 300, 511, 513]


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("heads,group,d,page", [(1, 1, 16, 16), (2, 4, 64, 16), (3, 1, 64, 32), (2, 5, 80, 16),
                                                (1, 8, 128, 64), (2, 3, 128, 16), (1, 16, 128, 32), (1, 24, 128, 128),
                                                (1, 40, 64, 16), (2, 2, 96, 256), (1, 4, 176, 16), (1, 4, 192, 64),
                                                (1, 7, 256, 16), (1, 2, 32, 1024), (1, 17, 256, 64)])
def test_attend_lengths(apc, orc, cache, dtype, heads, group, d, page):
    """Every way a length can end in a page and a tile, nothing held among them."""
    say(f"attend {dtype} over {cache} heads={heads} group={group} d={d} page={page}")
    mp = -(-513 // page)
    pool, table, q = make_attend(d + page, len(LENS), heads, group, d, page, mp, cache, dtype)
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    scale = d ** -0.5
    out, lse = run_attend(apc, pool, table, q, lens, scale)
    check_attend(orc, cache, dtype, pool, table, q, lens, scale, 0, out, lse)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("window", [1, 2, 16, 31, 33, 100, 4096])
def test_attend_window(apc, orc, cache, dtype, window):
    say(f"attend window={window} {dtype} over {cache}")
    pool, table, q = make_attend(11, len(LENS), 2, 4, 64, 16, 33, cache, dtype)
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, pool, table, q, lens, 0.125, window)
    check_attend(orc, cache, dtype, pool, table, q, lens, 0.125, window, out, lse)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("fill", [0xff, 0x7f, 0x7c])
def test_attend_unseen_slots_hold_anything(apc, orc, cache, dtype, fill):
    """NaN, infinities and huge values past the length, before the window and in pages that no table names."""
    say(f"attend unseen 0x{fill:x} {dtype} over {cache}")
    page, mp, b = 16, 9, 12
    pool, table, q = make_attend(13, b, 2, 4, 64, page, mp, cache, dtype)
    lens = torch.tensor([0, 1, 5, 16, 17, 40, 47, 64, 100, 130, 143, 144], dtype=torch.int32, device="cuda")
    window = 50
    want = run_attend(apc, pool, table, q, lens, 0.125, window)
    check_attend(orc, cache, dtype, pool, table, q, lens, 0.125, window, *want)
    seen = torch.zeros((pool[0].shape[0], page), dtype=torch.bool, device="cuda")
    for i, n in enumerate(lens.tolist()):
        for j in range(max(0, n - window), n):
            seen[table[i, j // page].item(), j % page] = True
    for t in pool:
        if t is not None:
            bad = torch.empty_like(t)
            bad.view(torch.uint8).fill_(fill)
            m = seen[:, None, :].expand(t.shape[:3])
            m = m[..., None].expand(t.shape) if t.dim() == 4 else m
            raw = t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16 if t.element_size() == 2 else torch.int32)
            raw.copy_(torch.where(m, raw, bad.view(raw.dtype)))
    got = run_attend(apc, pool, table, q, lens, 0.125, window)
    for a, b2 in zip(want, got):
        assert torch.equal(a, b2)


@pytest.mark.parametrize("cache,dtype", KINDS)
def test_attend_absent_pages(apc, orc, cache, dtype):
    """Page entries outside the pool leave their tokens out; a sequence of such entries alone attends to nothing."""
    pool, table, q = make_attend(17, 6, 2, 4, 128, 32, 12, cache, dtype)
    n_pages = pool[0].shape[0]
    table[0, 0], table[1, 3:5], table[2, 11], table[3, :] = -1, n_pages, -2 ** 31, 2 ** 31 - 1
    table[4, :10] = -7
    lens = torch.tensor([384, 300, 384, 200, 321, 10], dtype=torch.int32, device="cuda")
    for window in (0, 70):
        out, lse = run_attend(apc, pool, table, q, lens, 0.1, window)
        check_attend(orc, cache, dtype, pool, table, q, lens, 0.1, window, out, lse)
        assert torch.isneginf(lse[3]).all()


@pytest.mark.parametrize("cache,dtype", KINDS)
def test_attend_lengths_outside_the_table(apc, orc, cache, dtype):
    pool, table, q = make_attend(19, 4, 1, 2, 64, 16, 3, cache, dtype)
    lens = torch.tensor([-5, 49, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, pool, table, q, lens, 0.2)
    check_attend(orc, cache, dtype, pool, table, q, lens, 0.2, 0, out, lse)
    out, lse = run_attend(apc, pool, table[:, :0], q, lens, 0.2)                # no page at all
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("b,heads,group,d,page,lens", [(1, 2, 4, 128, 64, [5000]), (1, 1, 8, 64, 16, [9001]),
                                                       (3, 1, 5, 80, 32, [4097, 1, 2500]),
                                                       (5, 2, 1, 256, 128, [1, 0, 6000, 3, 777]),
                                                       (2, 1, 33, 128, 16, [3333, 1111])])
def test_attend_split_lengths(apc, orc, cache, dtype, b, heads, group, d, page, lens):
    """Few sequences, long: the length is split and joined."""
    say(f"attend split {dtype} over {cache} b={b} heads={heads} group={group} d={d} page={page} lens={lens}")
    mp = -(-max(lens) // page) + 1
    pool, table, q = make_attend(23, b, heads, group, d, page, mp, cache, dtype)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for window in (0, 2000):
        out, lse = run_attend(apc, pool, table, q, n, d ** -0.5, window)
        check_attend(orc, cache, dtype, pool, table, q, n, d ** -0.5, window, out, lse)
        again = run_attend(apc, pool, table, q, n, d ** -0.5, window)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])       # no order of arrival in the result


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("heads,group,d,page", [(1, 1, 16, 16), (3, 2, 64, 64), (2, 5, 80, 16), (2, 4, 128, 32),
                                                (1, 24, 128, 16), (1, 3, 256, 128), (1, 40, 64, 16)])
def test_attend_short_sequences_in_a_long_table(apc, orc, cache, dtype, heads, group, d, page):
    """The table could hold 16,384 tokens a sequence, most of its entries stale."""
    say(f"attend long table {dtype} over {cache} heads={heads} group={group} d={d} page={page}")
    pool, table, q = make_attend(d + page, len(LENS), heads, group, d, page, -(-513 // page), cache, dtype)
    wide = torch.full((len(LENS), 16384 // page), 2 ** 30, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    for window in (0, 70):
        out, lse = run_attend(apc, pool, wide, q, lens, d ** -0.5, window)
        check_attend(orc, cache, dtype, pool, table, q, lens, d ** -0.5, window, out, lse)


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("b,heads,group,d,cap,most", [(300, 1, 2, 64, 8192, 40), (1000, 2, 1, 16, 16384, 100),
                                                      (257, 1, 3, 128, 4096, 700), (5000, 1, 1, 16, 64, 64),
                                                      (2600, 1, 2, 32, 8192, 33)])
def test_attend_many_sequences(apc, orc, cache, dtype, b, heads, group, d, cap, most):
    """Batches past 256 sequences, a third of them empty in runs, in short tables and long ones."""
    say(f"attend many {dtype} over {cache} b={b} heads={heads} group={group} d={d} cap={cap} most={most}")
    page, g = 16, gen(b)
    pages = -(-most // page)
    pool, small, q = make_attend(b, b, heads, group, d, page, pages, cache, dtype)
    table = torch.full((b, cap // page), -3, dtype=torch.int32, device="cuda")
    table[:, :pages] = small
    lens = torch.randint(0, most + 1, (b,), device="cuda", generator=g).to(torch.int32)
    lens[b // 5:b // 3] = 0
    lens[-b // 6:] = 0
    lens[b // 2] = most
    for window in (0, 20):
        out, lse = run_attend(apc, pool, table, q, lens, 0.3, window)
        check_attend(orc, cache, dtype, pool, small, q, lens, 0.3, window, out, lse)
    lens.zero_()                                                     # nothing anywhere
    out, lse = run_attend(apc, pool, table, q, lens, 0.3)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("b,heads,group,d,page,most", [(1200, 1, 3, 16, 16, 32), (130, 8, 5, 80, 32, 256), (130, 8, 20, 128, 64, 256),
                                                       (520, 2, 1, 64, 16, 200), (264, 4, 40, 64, 16, 100), (130, 8, 2, 192, 32, 256),
                                                       (130, 16, 4, 256, 64, 960), (1030, 2, 17, 256, 16, 70)])
def test_attend_a_wave_to_a_unit(apc, orc, cache, dtype, b, heads, group, d, page, most):
    """Many (sequence, head) pairs of a few tiles each, the sequences on a pool of shared pages."""
    say(f"attend wave a unit {dtype} over {cache} b={b} heads={heads} group={group} d={d} page={page} most={most}")
    rows, g = 16, gen(b + d)
    pool, few, q = make_attend(b + d, rows, heads, group, d, page, -(-most // page), cache, dtype)
    q = torch.randn((b, heads * group, d), device="cuda", generator=g).to(q.dtype)
    table = few[torch.randint(0, rows, (b,), device="cuda", generator=g)].contiguous()
    lens = torch.randint(0, most + 1, (b,), device="cuda", generator=g).to(torch.int32)
    lens[b // 5:b // 4], lens[b // 2], lens[-1] = 0, most, most
    at = torch.cat([torch.arange(0, 8), torch.arange(b // 5 - 2, b // 5 + 2), torch.arange(b // 2 - 2, b // 2 + 2),
                    torch.arange(b - 12, b)]).cuda()
    for window in (0, 50):
        out, lse = run_attend(apc, pool, table, q, lens, d ** -0.5, window)
        check_attend(orc, cache, dtype, pool, table[at], q[at], lens[at], d ** -0.5, window, out[at], lse[at])
        assert torch.equal(torch.isneginf(lse).all(dim=1), lens == 0) and (out[lens > 0].float().abs().amax(dim=2) > 0).all()
        again = run_attend(apc, pool, table, q, lens, d ** -0.5, window)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("b,heads,group,d,page,cap", [(260, 8, 2, 256, 64, 960), (20, 8, 4, 128, 64, 960), (300, 8, 24, 256, 16, 960)])
def test_attend_workspace_of_a_larger_batch(apc, orc, cache, dtype, b, heads, group, d, page, cap):
    """One workspace, made for the largest batch and table, with every smaller call's: uncut units next to cut ones."""
    say(f"attend one workspace {dtype} over {cache} b={b} heads={heads} d={d}")
    rows, g = 6, gen(b + d)
    pool, few, _ = make_attend(b + d, rows, heads, group, d, page, cap // page, cache, dtype)
    c = apc.KvCache(*pool)
    ws = apc.attend_workspace_tensor(c, b, heads * group, cap // page)
    for n in (b, 100, 15, 3, 1):
        if n > b:
            continue
        q = torch.randn((n, heads * group, d), device="cuda", generator=g).to(TORCH[dtype])
        table = few[torch.arange(n, device="cuda") % rows].contiguous()
        lens = torch.randint(cap // 2, cap + 1, (n,), device="cuda", generator=g).to(torch.int32)
        for window in (0, 700):
            out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
            ws.fill_(0xff)
            apc.apc_attend(c, q, table, lens, d ** -0.5, out, ws, lse, window)
            torch.cuda.synchronize()
            check_attend(orc, cache, dtype, pool, table[-4:], q[-4:], lens[-4:], d ** -0.5, window, out[-4:], lse[-4:])


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("b,heads,group,d,page,lens", [(4, 1, 24, 256, 16, [0, 1, 37, 500]), (3, 2, 33, 192, 64, [4100, 2, 1500]),
                                                       (2, 1, 64, 144, 32, [2049, 700]), (1, 1, 32, 256, 128, [9000])])
def test_attend_many_heads_of_wide_rows(apc, orc, cache, dtype, b, heads, group, d, page, lens):
    """More than 16 query heads to a key-value head with heads wider than 128: uncut, cut, several query tiles."""
    say(f"attend wide {dtype} over {cache} b={b} heads={heads} group={group} d={d} lens={lens}")
    pool, table, q = make_attend(d + group, b, heads, group, d, page, -(-max(lens) // page), cache, dtype)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for window in (0, 333):
        out, lse = run_attend(apc, pool, table, q, n, d ** -0.5, window)
        check_attend(orc, cache, dtype, pool, table, q, n, d ** -0.5, window, out, lse)


def test_attend_more_units_than_workgroups(apc, orc):
    """Short sequences in more (sequence, head) pairs than a launch has workgroups for."""
    b, heads, d, page = 9000, 8, 16, 16
    pool, table, q = make_attend(61, b, heads, 1, d, page, 1, "f16", "f16")
    lens = torch.randint(0, 17, (b,), device="cuda", generator=gen(62)).to(torch.int32)
    out, lse = run_attend(apc, pool, table, q, lens, 0.25)
    at = torch.cat([torch.arange(0, 30), torch.arange(8150, 8230), torch.arange(b - 30, b)]).cuda()
    check_attend(orc, "f16", "f16", pool, table[at], q[at], lens[at], 0.25, 0, out[at], lse[at])
    assert torch.equal(torch.isneginf(lse).all(dim=1), lens == 0) and (out[lens > 0].abs().amax(dim=2) > 0).all()


@pytest.mark.parametrize("cap", [64, 16384])
def test_attend_without_pages(apc, cap):
    """A pool of no pages: every entry is outside it."""
    pool = make_pool(0, 2, 16, 64, "bf16")
    q = torch.randn((3, 4, 64), device="cuda", generator=gen(63)).to(torch.bfloat16)
    table = torch.zeros((3, cap // 16), dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, pool, table, q, torch.tensor([cap, 5, 0], dtype=torch.int32, device="cuda"), 0.1)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_attend_peaked_flat_and_rising_scores(apc, orc, cache, dtype, scale):
    """One token that takes all the weight at either end, equal weights, scores that rise along the sequence."""
    pool, table, q = make_attend(29, 4, 1, 4, 64, 16, 20, cache, dtype, spread=0.5)
    k = pool[0]
    flat = k.view(-1, 64)
    for i, place in ((0, 0), (1, 311), (2, 160)):
        flat_row = table[i, place // 16].item() * 16 + place % 16
        flat[flat_row] = (q[i, 0].float() * 30).clamp(-400, 400).to(k.dtype)
    ramp = torch.linspace(0, 4, 320, device="cuda")
    for j in range(320):
        row = table[3, j // 16].item() * 16 + j % 16
        flat[row] = (q[3, 0].float() * ramp[j]).to(k.dtype)
    lens = torch.tensor([312, 312, 312, 320], dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, pool, table, q, lens, scale)
    check_attend(orc, cache, dtype, pool, table, q, lens, scale, 0, out, lse)


@pytest.mark.parametrize("cache,dtype", KINDS)
def test_attend_strides(apc, orc, cache, dtype):
    """Queries in a fused product's rows, at odd elements, heads outermost; outputs into wider rows; a table's slice."""
    b, heads, group, d = 5, 2, 3, 64
    pool, wide, _ = make_attend(31, b, heads, group, d, 16, 12, cache, dtype)
    lens = torch.tensor([190, 3, 64, 0, 99], dtype=torch.int32, device="cuda")
    g = gen(37)
    big = torch.randn((b, heads * group + 2 * heads, d), device="cuda", generator=g).to(TORCH[dtype])
    odd = torch.randn((b, heads * group, d + 5), device="cuda", generator=g).to(TORCH[dtype])
    outer = torch.randn((heads * group, b, d), device="cuda", generator=g).to(TORCH[dtype])
    c = apc.KvCache(*pool)
    for q in (big[:, :heads * group], odd[..., 3:3 + d], outer.transpose(0, 1)):
        table = wide[:, :9]
        buf = torch.full((b, heads * group, d + 7), 5.0, device="cuda").to(TORCH[dtype])
        lse = torch.empty((b, heads * group), device="cuda")
        apc.apc_attend(c, q, table, lens, 0.125, buf[..., 1:1 + d], apc.attend_workspace_tensor(c, b, heads * group, 9), lse)
        torch.cuda.synchronize()
        check_attend(orc, cache, dtype, pool, table, q, lens, 0.125, 0, buf[..., 1:1 + d], lse)
        assert (buf[..., :1] == 5).all() and (buf[..., 1 + d:] == 5).all()
        out2 = torch.empty((b, heads * group, d), device="cuda").to(TORCH[dtype])
        apc.apc_attend(c, q, table, lens, 0.125, out2, apc.attend_workspace_tensor(c, b, heads * group, 9))    # no lse
        torch.cuda.synchronize()
        assert torch.equal(out2, buf[..., 1:1 + d])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_offsets_past_32_bits(apc, orc, cache):
    """A pool of more than 2^32 bytes and, for e4m3, elements: tokens written, read and attended at its end."""
    heads, page, d = 8, 128, 128
    n_pages = (1 << 32) // (heads * page * d) + (9 if cache == "e4m3" else 1000)
    kp, vp = (torch.zeros((n_pages, heads, page, d), dtype=torch.uint8 if cache == "e4m3" else TORCH[cache],
                          device="cuda").view(TORCH[cache]) for _ in range(2))
    ks, vs = ((torch.zeros((n_pages, heads, page), device="cuda") for _ in range(2)) if cache == "e4m3" else (None, None))
    c = apc.KvCache(kp, vp, ks, vs)
    t = 4 * page - 5
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    slots = (table.view(-1, 1).long() * page + torch.arange(page, device="cuda")).reshape(-1)[:t].to(torch.int32)
    x = torch.randn((t, 2, heads, d), device="cuda", generator=gen(41)).to(torch.bfloat16)
    apc.apc_kv_write(c, x[:, 0], x[:, 1], slots)
    ko, vo = (torch.empty((t, heads, d), device="cuda") for _ in range(2))
    apc.apc_kv_read(c, slots, ko, vo)
    q = torch.randn((1, heads * 4, d), device="cuda", generator=gen(43)).to(torch.bfloat16)
    lens = torch.tensor([t], dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, (kp, vp, ks, vs), table, q, lens, 0.09)
    torch.cuda.synchronize()
    rows, sc = orc.quantize_rows(cache, x[:, 0].float().cpu().numpy().reshape(-1, d))
    want = orc.kv_values(cache, rows).astype(np.float32) * (1 if sc is None else sc[:, None])
    assert np.array_equal(ko.cpu().numpy().reshape(-1, d), want)
    sub = [None if p is None else p[table[0].long()] if p.dtype != torch.float8_e4m3fn else
           p.view(torch.uint8)[table[0].long()].view(p.dtype) for p in (kp, vp, ks, vs)]
    check_attend(orc, cache, "bf16", sub, torch.arange(4, dtype=torch.int32, device="cuda")[None], q, lens, 0.09, 0, out, lse)


def test_prompt_ops_on_their_own_stream(apc, orc):
    """Calls on a stream of their own follow that stream's work."""
    s = torch.cuda.Stream()
    pool, table, q = make_attend(47, 3, 2, 4, 64, 16, 20, "e4m3", "bf16")
    lens = torch.tensor([300, 7, 99], dtype=torch.int32, device="cuda")
    c = apc.KvCache(*pool)
    ws = apc.attend_workspace_tensor(c, 3, 8, 20)
    x = torch.randn((3, 512), device="cuda", generator=gen(48))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        a = torch.randn((4000, 4000), device="cuda")
        for _ in range(4):
            a = a @ a * 1e-4                                         # keeps the stream busy before the inputs are there
        q2, x2 = torch.zeros_like(q), torch.zeros_like(x)
        q2.copy_(q)
        x2.copy_(x)
        out, normed = torch.empty_like(q), torch.empty_like(x)
        apc.apc_attend(c, q2, table, lens, 0.125, out, ws)
        apc.apc_norm_rows(x2, normed)
    q3 = torch.empty_like(q)
    torch.cuda.synchronize()
    want, lse = run_attend(apc, pool, table, q, lens, 0.125)
    assert torch.equal(out, want)
    check_norm(orc, x, None, None, normed, None, None, 1e-6, "f32")
    apc.apc_attend(c, q, table, lens, 0.125, q3, ws, stream=s)       # the stream as an argument
    torch.cuda.synchronize()
    assert torch.equal(q3, want)


def test_prompt_step_graph_replays(apc, orc):
    """A step's calls captured as a graph; every replay, with eager work between, equals the eager result."""
    pool, table, q = make_attend(53, 4, 2, 4, 64, 16, 40, "e4m3", "bf16")
    lens = torch.tensor([640, 1, 333, 0], dtype=torch.int32, device="cuda")
    c = apc.KvCache(*pool)
    ws = apc.attend_workspace_tensor(c, 4, 8, 40)
    h = torch.randn((4, 512), device="cuda", generator=gen(54)).to(torch.bfloat16)
    kv = torch.randn((4, 4, 64), device="cuda", generator=gen(55)).to(torch.bfloat16)
    slots = torch.tensor([table[0, 39].item() * 16 + 15, table[1, 0].item() * 16, table[2, 20].item() * 16 + 12, -1],
                         dtype=torch.int32, device="cuda")
    codes, s = torch.empty((4, 512), dtype=TORCH["e4m3"], device="cuda"), torch.empty(4, device="cuda")
    out, lse, ko, vo = torch.empty_like(q), torch.empty((4, 8), device="cuda"), *torch.empty((2, 4, 2, 64), device="cuda")

    def step():
        apc.apc_kv_write(c, kv[:, :2], kv[:, 2:], slots)
        apc.apc_attend(c, q, table, lens, 0.125, out, ws, lse)
        apc.apc_kv_read(c, slots, ko, vo)
        apc.apc_norm_rows(out.view(4, 512), codes, None, h, h, s)

    h0 = h.clone()
    results = lambda: [t.clone() for t in (out, lse, ko, vo, codes.view(torch.uint8), s, h)]
    step()
    torch.cuda.synchronize()
    ref = results()
    h.copy_(h0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(4):
        h.copy_(h0)
        for t in (out, lse, ko, vo, s):
            t.fill_(-7)
        ws.fill_(0xff)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(ref, results()):
            assert torch.equal(a, b), f"replay {rep} differs"
