"""The float64 oracle of the prompt model's operators, pinned to independent
formulations: the norm to its unit mean square and to torch, the cache to the
pinned row storage, attention to a softmax over a dense gather, to invariances
and to one-token and empty cases."""
import numpy as np
import pytest
import torch


def test_norm_rows(orc):
    rng = np.random.default_rng(1)
    x, r, w = rng.standard_normal((5, 33)), rng.standard_normal((5, 33)), rng.standard_normal(33)
    y, h = orc.norm_rows(x, r, w, 1e-6)
    assert np.array_equal(h, x + r)
    t = torch.from_numpy(x + r)
    want = torch.nn.functional.rms_norm(t, (33,), torch.from_numpy(w), 1e-6).numpy()
    assert np.abs(y - want).max() < 1e-12
    y, _ = orc.norm_rows(x, None, None, 0.0)
    assert np.allclose((y * y).mean(axis=1), 1.0, atol=1e-12)            # unit mean square
    y7, _ = orc.norm_rows(x * 7, None, None, 0.0)
    assert np.allclose(y, y7, atol=1e-12)                                # scale invariance
    z, _ = orc.norm_rows(np.zeros((1, 4)), None, None, 1e-6)
    assert np.array_equal(z, np.zeros((1, 4)))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "e4m3"])
def test_kv_write_then_read(orc, dtype):
    rng = np.random.default_rng(2)
    t, heads, page, d, n_pages = 9, 3, 16, 32, 2
    x = rng.standard_normal((t, heads, d)).astype(np.float32)
    slots = np.array([5, 31, -1, 0, 16, 32, 7, 30, 1])                   # -1 and 32 are outside
    rows, sc = orc.quantize_rows(dtype, x.reshape(-1, d))
    pool = np.zeros((n_pages, heads, page, d), rows.dtype)
    scale = np.full((n_pages, heads, page), 9.0, np.float32) if dtype == "e4m3" else None
    orc.kv_write(dtype, pool, scale, x, slots)
    back = orc.kv_read(dtype, pool, scale, slots, "f32")
    ok = (slots >= 0) & (slots < 32)
    want = orc.kv_values(dtype, rows).reshape(t, heads, d) * (1.0 if sc is None else sc.reshape(t, heads, 1))
    assert np.array_equal(back[ok], want[ok].astype(np.float32))
    assert np.array_equal(back[~ok], np.zeros_like(back[~ok]))
    untouched = np.ones((n_pages, page), bool)
    untouched[slots[ok] // page, slots[ok] % page] = False
    assert not pool.swapaxes(1, 2)[untouched].any()
    if scale is not None:
        assert (scale.swapaxes(1, 2)[untouched] == 9.0).all()


def _cache(rng, n_pages, heads, page, d):
    return [rng.standard_normal((n_pages, heads, page, d)).astype(np.float16) for _ in range(2)]


def test_attend_is_softmax_over_the_gathered_tokens(orc):
    rng = np.random.default_rng(3)
    heads, group, page, d = 2, 3, 16, 16
    k, v = _cache(rng, 7, heads, page, d)
    pages = np.array([[4, 2, 6], [0, 5, 1]], np.int32)
    lengths = np.array([37, 48], np.int32)
    q = rng.standard_normal((2, heads * group, d))
    for window in (0, 1, 20, 100):
        out, lse, _, _ = orc.attend("f16", q, k, v, None, None, pages, lengths, 0.25, window)
        for i in range(2):
            kk = torch.from_numpy(k[pages[i]].astype(np.float64)).permute(1, 0, 2, 3).reshape(heads, -1, d)
            vv = torch.from_numpy(v[pages[i]].astype(np.float64)).permute(1, 0, 2, 3).reshape(heads, -1, d)
            n = int(lengths[i])
            f = max(0, n - window) if window else 0
            qq = torch.from_numpy(q[i]).view(heads, group, d)
            s = 0.25 * qq @ kk[:, f:n].transpose(1, 2)
            assert np.abs(out[i] - (torch.softmax(s, -1) @ vv[:, f:n]).reshape(-1, d).numpy()).max() < 1e-12
            assert np.abs(lse[i] - torch.logsumexp(s, -1).reshape(-1).numpy()).max() < 1e-12


def test_attend_corners(orc):
    rng = np.random.default_rng(4)
    k, v = _cache(rng, 3, 1, 16, 16)
    q = rng.standard_normal((3, 2, 16))
    pages = np.array([[1], [2], [-1]], np.int32)
    out, lse, _, _ = orc.attend("f16", q, k, v, None, None, pages, np.array([1, 0, 9]), 1.0)
    assert np.allclose(out[0], v[1, 0, 0].astype(np.float64)[None])       # one token: its value
    assert np.array_equal(out[1:], np.zeros((2, 2, 16))) and np.isneginf(lse[1:]).all()   # nothing held, no page
    # a page order change with the tokens moved along changes nothing; what lies past the length neither
    full = np.array([[0, 1, 2]], np.int32)
    a = orc.attend("f16", q[:1], k, v, None, None, full, np.array([40]), 1.0)
    perm = np.array([2, 0, 1])
    k2, v2 = k[perm].copy(), v[perm].copy()
    k2[0, :, 8:], v2[0, :, 8:] = np.nan, np.inf
    b = orc.attend("f16", q[:1], k2, v2, None, None, np.array([[1, 2, 0]]), np.array([40]), 1.0)
    for x, y in zip(a, b):
        assert np.array_equal(x, y)


def test_attend_scales_are_the_values_factors(orc):
    rng = np.random.default_rng(5)
    codes = [rng.integers(0, 120, (2, 1, 16, 16)).astype(np.uint8) for _ in range(2)]
    ks, vs = (rng.uniform(0.01, 0.1, (2, 1, 16)).astype(np.float32) for _ in range(2))
    q = rng.standard_normal((1, 1, 16))
    pages = np.array([[1, 0]], np.int32)
    out, lse, _, _ = orc.attend("e4m3", q, codes[0], codes[1], ks, vs, pages, np.array([30]), 0.3)
    val = orc.e4m3_values()
    kk = np.concatenate([val[codes[0][p, 0]] * ks[p, 0][:, None].astype(np.float64) for p in (1, 0)])[:30]
    vv = np.concatenate([val[codes[1][p, 0]] * vs[p, 0][:, None].astype(np.float64) for p in (1, 0)])[:30]
    w = np.exp(0.3 * (kk @ q[0, 0]))
    assert np.allclose(out[0, 0], w @ vv / w.sum(), rtol=1e-12) and np.isclose(lse[0, 0], np.log(w.sum()))
