"""The float64 oracle of the operators that read whole prompts, pinned to
independent formulations: rotation to complex products and invariances,
attention of many new tokens to attention of one, to a dense softmax with the
mask written out, and to its corner cases."""
import numpy as np
import pytest


def test_rotary_freqs(orc):
    f = orc.rotary_freqs(8, 10000.0, 1.0, 0.0, 1.0, 4.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-14)
    assert np.allclose(orc.rotary_freqs(8, 10000.0, 4.0, 0.0, 1.0, 4.0), f / 4)
    # 100 positions: 15.9, 1.59, 0.159 and 0.0159 turns
    g = orc.rotary_freqs(8, 10000.0, 4.0, 100.0, 1.0, 4.0)
    part = (100 * 0.1 / (2 * np.pi) - 1) / 3
    assert np.allclose(g, [1.0, part * 0.1 + (1 - part) * 0.025, 0.0025, 0.00025])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_is_a_complex_product(orc, interleaved):
    rng = np.random.default_rng(1)
    x, at, f = rng.standard_normal((5, 3, 10)), np.array([0, 1, 77, -1, 10 ** 6]), rng.uniform(0, 1, 4)
    y = orc.rotate(x, at, f, interleaved, 1.5)
    assert np.array_equal(y[3], x[3]) and np.array_equal(y[..., 8:], x[..., 8:])
    z = x[..., 0:8:2] + 1j * x[..., 1:8:2] if interleaved else x[..., :4] + 1j * x[..., 4:8]
    z = 1.5 * z * np.exp(1j * (at[:, None] * f))[:, None]
    got = y[..., 0:8:2] + 1j * y[..., 1:8:2] if interleaved else y[..., :4] + 1j * y[..., 4:8]
    assert np.allclose(got[[0, 1, 2, 4]], z[[0, 1, 2, 4]], atol=1e-9)
    # a product of a query and a key goes by their distance alone
    a = orc.rotate(x, at + 13, f, interleaved)
    b = orc.rotate(x, at, f, interleaved)
    turned = np.einsum("thd,thd->th", a[[0, 1, 2]], orc.rotate(x, at + 20, f, interleaved)[[0, 1, 2]])
    assert np.allclose(turned, np.einsum("thd,thd->th", b[[0, 1, 2]], orc.rotate(x, at + 7, f, interleaved)[[0, 1, 2]]))
    assert np.allclose(orc.rotate(b, at, -f, interleaved), x, atol=1e-9)       # and back


def _cache(rng, n_pages, heads, page, d):
    return [rng.standard_normal((n_pages, heads, page, d)).astype(np.float16) for _ in range(2)]


def test_one_token_is_attend(orc):
    rng = np.random.default_rng(2)
    k, v = _cache(rng, 9, 2, 16, 16)
    pages = rng.permutation(9).astype(np.int32).reshape(3, 3)
    pages[1, 0] = -1
    lens = np.array([40, 48, 0])
    q = rng.standard_normal((3, 6, 16))
    for window in (0, 1, 20):
        a = orc.attend("f16", q, k, v, None, None, pages, lens, 0.3, window)
        b = orc.attend_prompt("f16", q, np.arange(4), k, v, None, None, pages, lens, 0.3, window)
        for x, y in zip(a, b):
            assert np.allclose(x, y, rtol=1e-12, atol=1e-13)


@pytest.mark.parametrize("cap,slope,window,prefix", [(0, 0, 0, None), (2.0, 0, 0, None), (0, 0.1, 0, None), (0, 0, 7, None),
                                                     (0, 0, 0, 20), (1.5, 0.2, 9, 25), (0, 0, 0, 99), (0, 0.3, 5, 99)])
def test_attend_prompt_is_a_masked_softmax(orc, cap, slope, window, prefix):
    rng = np.random.default_rng(3)
    heads, group, page, d, n, length = 2, 2, 16, 16, 11, 30
    k, v = _cache(rng, 4, heads, page, d)
    pages = np.array([[2, 1]], np.int32)
    q = rng.standard_normal((n + 2, heads * group, d))                  # two rows of no sequence
    slopes = slope * np.arange(1, heads * group + 1) if slope else None
    out, lse, spread, _, _, away = orc.attend_prompt("f16", q, np.array([1, n + 1]), k, v, None, None, pages,
                                                     np.array([length]), 0.25, window, cap, slopes,
                                                     None if prefix is None else np.array([prefix]))
    assert np.isnan(out[[0, -1]]).all() and np.isnan(lse[[0, -1]]).all()
    flat = lambda x, h: x[[2, 1], h].reshape(-1, d)[:length].astype(np.float64)
    for r in range(n):
        p = length - n + r
        see = [j for j in range(length) if (j <= p or (prefix is not None and j < prefix)) and (not window or abs(p - j) < window)]
        assert away[r + 1, 0] == max(abs(p - j) for j in see)
        for a in range(heads * group):
            s = 0.25 * flat(k, a // group)[see] @ q[r + 1, a]
            s = cap * np.tanh(s / cap) if cap else s
            s = s - (slopes[a] * np.abs(p - np.array(see)) if slope else 0)
            w = np.exp(s)
            assert np.isclose(lse[r + 1, a], np.log(w.sum()))
            assert np.allclose(out[r + 1, a], w @ flat(v, a // group)[see] / w.sum())
            assert (spread[r + 1, a] >= np.abs(out[r + 1, a]) - 1e-12).all()


def test_rows_that_see_nothing(orc):
    rng = np.random.default_rng(4)
    k, v = _cache(rng, 2, 1, 16, 16)
    q = rng.standard_normal((9, 1, 16))
    # five new tokens of a sequence of three; nothing held; no page there
    out, lse, _, _, _, _ = orc.attend_prompt("f16", q, np.array([0, 5, 7, 9]), k, v, None, None,
                                             np.array([[0], [1], [-1]], np.int32), np.array([3, 0, 16]), 1.0)
    assert np.isneginf(lse[[0, 1, 5, 6, 7, 8], 0]).all() and not out[[0, 1, 5, 6, 7, 8]].any()
    assert np.isfinite(lse[2:5]).all()
    assert np.array_equal(out[2, 0], v[0, 0, 0].astype(np.float64))      # sees one token
    # a prefix is seen from negative positions too
    _, lse, _, _, _, _ = orc.attend_prompt("f16", q[:5], np.array([0, 5]), k, v, None, None, np.array([[0]], np.int32),
                                           np.array([3]), 1.0, prefix=np.array([2]))
    assert np.isfinite(lse).all()
