"""Refusals of the calls that read whole prompts: every bad argument returns its
status before the GPU is touched (CPU only: no compute calls)."""
import ctypes
import os

import numpy as np
import pytest

from tests.test_api_prompt import BAD_KV, BF16, E4M3, E_ARG, E_DTYPE, E_WORKSPACE, F16, F32, FAKE, ODD, _kv

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2502_06798_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("libapc.so not built")
    return binding.load()


def test_rotary_freqs(lib, orc):
    import paper_2502_06798_amd as apc
    for args in ((64, 10000.0, 1.0, 0.0, 1.0, 4.0), (2, 10000.0, 4.0, 0.0, 0.0, 0.0), (256, 5e5, 8.0, 8192.0, 1.0, 4.0),
                 (90, 1e6, 40.0, 4096.0, 1.0, 32.0)):
        got, want = apc.apc_rotary_freqs(*args), orc.rotary_freqs(*args)
        assert got.shape == (args[0] // 2,) and np.allclose(got, want, rtol=1e-13, atol=0)
    buf = np.zeros(256)

    def call(rot=64, base=1e4, factor=1.0, original=0.0, low=1.0, high=4.0, out=buf.ctypes.data):
        return lib.apc_rotary_freqs(rot, base, factor, original, low, high, out)

    assert call() == 0 and call(low=4.0, high=1.0) == 0                 # not looked at without an original length
    for rot in (0, -2, 3, 258):
        assert call(rot=rot) == E_ARG
    for bad in (0.0, -1.0, NAN, INF):
        assert call(base=bad) == E_ARG and call(factor=bad) == E_ARG
    assert call(original=-1.0) == E_ARG and call(original=NAN) == E_ARG and call(original=INF) == E_ARG
    assert call(original=9.0, low=4.0, high=4.0) == E_ARG and call(original=9.0, high=NAN) == E_ARG
    assert call(original=9.0, low=-INF) == E_ARG
    assert call(out=None) == E_ARG
    with pytest.raises(apc.ApcError):
        apc.apc_rotary_freqs(63)


def test_rotate_refusals(lib):
    from paper_2502_06798_amd import binding

    def call(rot=64, il=0, mag=1.0, freq=0x100000, dt=F16, t=3, heads=2, d=64, x=FAKE, xt=128, xh=64, pos=FAKE, out=FAKE,
             ot=128, oh=64, r=True):
        desc = binding._RotaryStruct(rot, il, mag, freq)
        return lib.apc_rotate(ctypes.byref(desc) if r else None, dt, t, heads, d, x, xt, xh, pos, out, ot, oh, None)

    assert call(t=0) == 0 and call(t=0, x=None, out=None, pos=None, freq=0) == 0
    assert call(r=False) == E_ARG
    assert call(dt=E4M3) == E_DTYPE and call(dt=7) == E_DTYPE
    assert call(d=0) == E_ARG and call(d=257, xh=300, oh=300) == E_ARG
    for rot in (0, -2, 1, 63, 66):
        assert call(rot=rot) == E_ARG
    assert call(il=2) == E_ARG and call(il=-1) == E_ARG
    assert call(mag=NAN) == E_ARG and call(mag=INF) == E_ARG
    assert call(heads=0) == E_ARG and call(t=-1) == E_ARG and call(t=1 << 30) == E_ARG
    for name in ("xt", "xh", "ot", "oh"):
        assert call(**{name: -1}) == E_ARG
    assert call(x=None) == E_ARG and call(out=None) == E_ARG and call(pos=None) == E_ARG and call(freq=0) == E_ARG
    assert call(x=ODD) == E_ARG and call(out=ODD) == E_ARG and call(freq=0x100004) == E_ARG
    assert call(pos=ctypes.c_void_p(0x100002)) == E_ARG and call(dt=F32, x=ctypes.c_void_p(0x100002)) == E_ARG
    # rows of out on top of each other
    assert call(oh=63) == E_ARG and call(ot=63, oh=1000) == E_ARG and call(ot=64, oh=64) == E_ARG
    assert call(ot=0, oh=64) == E_ARG


@pytest.mark.parametrize("bad,status", BAD_KV)
def test_cache_descriptions(lib, bad, status):
    c, n = ctypes.byref(_kv(**bad)), ctypes.c_size_t()
    assert lib.apc_attend_prompt_workspace(c, 3, 1, 2, 4, ctypes.byref(n)) == status
    assert lib.apc_attend_prompt(c, F16, 3, FAKE, 128, 64, 1, FAKE, 2, FAKE, 4, 4, FAKE, None, None, 0, 0.0, 1.0, FAKE,
                                 128, 64, None, FAKE, 1 << 40, None) == status


def test_attend_prompt_refusals(lib):
    n = ctypes.c_size_t()

    def call(cache=None, dt=F16, t=7, q=FAKE, qr=256, qh=64, b=2, starts=FAKE, hq=4, pages=FAKE, mp=4, lp=4, lens=FAKE,
             prefix=None, slopes=None, window=0, cap=0.0, scale=1.0, out=FAKE, o_r=256, oh=64, lse=None, ws=FAKE,
             wb=1 << 40):
        c = cache if cache is not None else ctypes.byref(_kv())
        return lib.apc_attend_prompt(c, dt, t, q, qr, qh, b, starts, hq, pages, mp, lp, lens, prefix, slopes, window, cap,
                                     scale, out, o_r, oh, lse, ws, wb, None)

    assert call(b=0) == 0 and call(t=0) == 0 and call(t=0, q=None, out=None, ws=None, wb=0) == 0
    assert call(dt=F32) == E_DTYPE and call(dt=E4M3) == E_DTYPE
    assert call(cache=ctypes.byref(_kv(dt=F16, ks=None, vs=None)), dt=BF16) == E_DTYPE
    assert call(b=-1) == E_ARG and call(hq=0) == E_ARG and call(hq=3) == E_ARG
    assert call(b=1 << 22) == E_ARG                                     # 2^24 sequences x heads
    assert call(t=-1) == E_ARG and call(t=(1 << 30) + 1, hq=2) == E_ARG and call(t=1 << 28) == E_ARG
    assert call(mp=-1) == E_ARG and call(mp=(1 << 26) + 1, lp=1 << 27) == E_ARG and call(lp=3) == E_ARG
    assert call(window=-1) == E_ARG
    for bad in (NAN, INF):
        assert call(scale=bad) == E_ARG and call(cap=bad) == E_ARG
    assert call(cap=-1.0) == E_ARG
    for name in ("qr", "qh", "o_r", "oh"):
        assert call(**{name: -1}) == E_ARG
    for name in ("q", "starts", "pages", "lens", "out"):
        assert call(**{name: None}) == E_ARG
    for name in ("q", "starts", "pages", "lens", "prefix", "slopes", "out", "lse"):
        assert call(**{name: ODD}) == E_ARG
    # long tables need a workspace
    assert lib.apc_attend_prompt_workspace(ctypes.byref(_kv()), 7, 2, 4, 4096, ctypes.byref(n)) == 0 and n.value > 0
    assert call(mp=4096, lp=4096, wb=n.value - 1) == E_WORKSPACE
    assert call(mp=4096, lp=4096, ws=None) == E_ARG
    assert call(mp=4096, lp=4096, ws=ctypes.c_void_p(0x100004)) == E_ARG
    assert lib.apc_attend_prompt_workspace(ctypes.byref(_kv()), 7, 2, 4, 4096, None) == E_ARG


def test_workspace_never_falls(lib):
    n = ctypes.c_size_t()
    for heads, group, d, page in ((1, 1, 64, 16), (8, 4, 128, 64), (3, 5, 256, 128), (12, 1, 64, 16)):
        c = ctypes.byref(_kv(heads=heads, d=d, page=page))

        def need(t, b, mp):
            assert lib.apc_attend_prompt_workspace(c, t, b, heads * group, mp, ctypes.byref(n)) == 0
            return n.value

        ts, bs, mps = (0, 1, 2, 31, 32, 33, 200, 5000, 100_000), (0, 1, 2, 7, 64, 300, 1000), (0, 1, 16, 64, 500, 4000)
        for t in ts:
            for b in bs:
                for mp in mps:
                    x = need(t, b, mp)
                    assert x >= max(need(t2, b, mp) for t2 in ts if t2 <= t)
                    assert x >= max(need(t, b2, mp) for b2 in bs if b2 <= b)
                    assert x >= max(need(t, b, m2) for m2 in mps if m2 <= mp)


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    import paper_2502_06798_amd as apc
    with pytest.raises(ValueError):
        apc.Rotary(torch.zeros(8))                                      # not float64
    with pytest.raises(ValueError):
        apc.Rotary(torch.zeros((2, 4), dtype=torch.float64))
    with pytest.raises(ValueError):
        apc.Rotary(torch.zeros(8, dtype=torch.float64))                 # not on a device
