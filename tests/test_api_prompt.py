"""Refusals of the prompt model's calls: every bad argument returns its status
before the GPU is touched (CPU only: no compute calls)."""
import ctypes
import os

import pytest

E_ARG, E_DTYPE, E_WORKSPACE = 1, 2, 6
F32, F16, BF16, E4M3 = 0, 1, 2, 3
FAKE = ctypes.c_void_p(0x100000)       # never dereferenced: every call below fails its checks first
ODD = ctypes.c_void_p(0x100001)


@pytest.fixture(scope="module")
def lib():
    from paper_2502_06798_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("libapc.so not built")
    return binding.load()


def test_norm_rows_refusals(lib):
    def call(dt=F16, odt=E4M3, n=4, d=64, x=FAKE, lx=64, res=FAKE, lr=64, w=FAKE, eps=1e-6, s=FAKE, ls=64, out=FAKE,
             lo=64, sc=FAKE):
        return lib.apc_norm_rows(dt, odt, n, d, x, lx, res, lr, w, eps, s, ls, out, lo, sc, None)

    assert call(n=0) == 0                               # nothing to do
    assert call(dt=E4M3) == E_DTYPE and call(dt=9) == E_DTYPE
    assert call(odt=BF16, sc=None) == E_DTYPE           # neither x's type nor e4m3
    assert call(n=-1) == E_ARG and call(n=1 << 31) == E_ARG
    assert call(d=0) == E_ARG and call(d=32769, lx=32769, lr=32769, ls=32769, lo=32769) == E_ARG
    assert call(lx=63) == E_ARG and call(lr=63) == E_ARG and call(ls=63) == E_ARG and call(lo=63) == E_ARG
    assert call(x=None) == E_ARG and call(out=None) == E_ARG
    assert call(x=ODD) == E_ARG and call(w=ODD) == E_ARG and call(s=ODD) == E_ARG and call(sc=ODD) == E_ARG
    assert call(res=None) == E_ARG                      # a sum without a residual
    assert call(sc=None) == E_ARG                       # e4m3 without scales
    assert call(odt=F16) == E_ARG                       # scales for f16
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == E_ARG
    assert lib.apc_last_error()


def _kv(dt=E4M3, heads=2, d=64, page=16, n=4, k=0x100000, v=0x100000, ks=0x100000, vs=0x100000):
    from paper_2502_06798_amd import binding
    return binding._KvStruct(dt, heads, d, page, n, k, v, ks, vs)


BAD_KV = [(dict(dt=F32), E_DTYPE), (dict(dt=9), E_DTYPE), (dict(heads=0), E_ARG), (dict(d=0), E_ARG),
          (dict(d=24), E_ARG), (dict(d=272), E_ARG), (dict(page=8), E_ARG), (dict(page=48), E_ARG),
          (dict(page=2048), E_ARG), (dict(n=-1), E_ARG), (dict(n=1 << 27), E_ARG), (dict(k=0), E_ARG),
          (dict(v=0x100008), E_ARG), (dict(ks=0), E_ARG), (dict(vs=0x100004), E_ARG),
          (dict(dt=F16), E_ARG)]                        # scales of a cache that has none


@pytest.mark.parametrize("bad,status", BAD_KV)
def test_cache_descriptions(lib, bad, status):
    c = ctypes.byref(_kv(**bad))
    n = ctypes.c_size_t()
    assert lib.apc_kv_write(c, F32, 1, FAKE, 128, 64, FAKE, 128, 64, FAKE, None) == status
    assert lib.apc_kv_read(c, F32, 1, FAKE, FAKE, 128, 64, FAKE, 128, 64, None) == status
    assert lib.apc_attend_workspace(c, 1, 2, 4, ctypes.byref(n)) == status
    assert lib.apc_attend(c, F16, FAKE, 128, 64, 1, 2, FAKE, 4, 4, FAKE, 0, 1.0, FAKE, 128, 64, None, FAKE, 1 << 40,
                          None) == status


def test_kv_rows_refusals(lib):
    c = ctypes.byref(_kv())
    for read in (False, True):
        def call(dt=F16, t=3, k=FAKE, kt=128, kh=64, v=FAKE, vt=128, vh=64, s=FAKE, cache=c):
            if read:
                return lib.apc_kv_read(cache, dt, t, s, k, kt, kh, v, vt, vh, None)
            return lib.apc_kv_write(cache, dt, t, k, kt, kh, v, vt, vh, s, None)

        assert call(t=0) == 0
        assert call(cache=None) == E_ARG
        assert call(dt=E4M3) == E_DTYPE and call(dt=1 << 30) == E_DTYPE
        assert call(t=-1) == E_ARG and call(t=1 << 31) == E_ARG
        assert call(kt=-1) == E_ARG and call(kh=-1) == E_ARG and call(vt=-1) == E_ARG and call(vh=-1) == E_ARG
        assert call(k=None) == E_ARG and call(v=None) == E_ARG and call(s=None) == E_ARG
        assert call(k=ODD) == E_ARG and call(dt=F32, v=ctypes.c_void_p(0x100002)) == E_ARG
        assert call(s=ctypes.c_void_p(0x100002)) == E_ARG


def test_attend_refusals(lib):
    kv = ctypes.byref(_kv())
    need = ctypes.c_size_t()
    assert lib.apc_attend_workspace(kv, 3, 4, 4, ctypes.byref(need)) == 0

    def call(c=kv, dt=F16, q=FAKE, qr=256, qh=64, b=3, heads=4, pages=FAKE, mp=4, lp=4, lens=FAKE, window=0, scale=0.125,
             out=FAKE, orow=256, oh=64, lse=None, ws=FAKE, nb=None):
        return lib.apc_attend(c, dt, q, qr, qh, b, heads, pages, mp, lp, lens, window, scale, out, orow, oh, lse, ws,
                              need.value if nb is None else nb, None)

    assert call(b=0) == 0
    assert call(c=None) == E_ARG
    assert call(dt=F32) == E_DTYPE and call(dt=E4M3) == E_DTYPE
    half = ctypes.byref(_kv(dt=BF16, ks=0, vs=0))
    assert call(c=half, dt=F16) == E_DTYPE              # another 16-bit type than the cache's
    assert call(b=-1) == E_ARG and call(heads=0) == E_ARG and call(heads=3) == E_ARG
    assert call(b=1 << 29) == E_ARG
    assert call(mp=-1) == E_ARG and call(mp=1 << 27, lp=1 << 27) == E_ARG and call(lp=3) == E_ARG
    assert call(window=-1) == E_ARG
    assert call(scale=float("nan")) == E_ARG and call(scale=float("inf")) == E_ARG
    assert call(qr=-1) == E_ARG and call(qh=-1) == E_ARG and call(orow=-1) == E_ARG and call(oh=-1) == E_ARG
    assert call(q=None) == E_ARG and call(out=None) == E_ARG and call(lens=None) == E_ARG and call(pages=None) == E_ARG
    assert call(q=ODD) == E_ARG and call(out=ODD) == E_ARG and call(lens=ODD) == E_ARG and call(lse=ODD) == E_ARG
    if need.value:
        assert call(ws=None) == E_ARG and call(ws=ctypes.c_void_p(0x100008)) == E_ARG
        assert call(nb=need.value - 1) == E_WORKSPACE
    assert lib.apc_attend_workspace(kv, 3, 4, 4, None) == E_ARG


def test_attend_workspace_never_falls(lib):
    for dt, ks in ((F16, 0), (E4M3, 0x100000)):
        for heads, d, page in ((1, 16, 16), (8, 128, 64), (12, 64, 32)):
            kv = ctypes.byref(_kv(dt=dt, heads=heads, d=d, page=page, ks=ks, vs=ks))
            for group in (1, 4, 24):
                last_b = 0
                for b in (1, 2, 3, 7, 16, 31, 64, 100, 256, 1000, 5000):
                    last = last_b
                    for mp in (0, 1, 2, 5, 30, 64, 200, 1000, 4000, 20000):
                        n = ctypes.c_size_t()
                        assert lib.apc_attend_workspace(kv, b, heads * group, mp, ctypes.byref(n)) == 0
                        if mp == 0:
                            assert n.value >= last_b
                            last_b = n.value
                            last = n.value
                        assert n.value >= last
                        last = n.value


@pytest.mark.parametrize("dt,ks", [(F16, 0), (E4M3, 0x100000)])
@pytest.mark.parametrize("heads,d,page", [(8, 128, 64), (8, 256, 64), (16, 192, 32), (12, 64, 16), (200, 128, 16), (2, 32, 1024)])
@pytest.mark.parametrize("group", [1, 8, 24])
def test_attend_workspace_serves_every_smaller_call(lib, dt, ks, heads, d, page, group):
    """No batch and no table within a call's asks for more, where the kernel that takes it changes with either."""
    kv = ctypes.byref(_kv(dt=dt, heads=heads, d=d, page=page, ks=ks, vs=ks))
    tables = [t * 16 // page for t in range(0, 300, 3) if t * 16 % page == 0] + [2000]
    above = [0] * len(tables)
    for b in (1, 2, 10, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 255, 256, 300, 1023, 1024, 2048):
        if b * heads * group > 1 << 23:                       # refused
            break
        left = 0
        for i, mp in enumerate(tables):
            n = ctypes.c_size_t()
            assert lib.apc_attend_workspace(kv, b, heads * group, mp, ctypes.byref(n)) == 0
            assert n.value >= above[i] and n.value >= left, (b, mp)
            above[i] = left = n.value


def test_binding_refuses_host_and_misshapen_tensors():
    import torch

    import paper_2502_06798_amd as apc
    x = torch.zeros(2, 32)
    with pytest.raises(ValueError):
        apc.apc_norm_rows(x, torch.zeros(2, 32))                         # host tensors
    with pytest.raises(ValueError):
        apc.apc_norm_rows(x, torch.zeros(2, 31))
    with pytest.raises(ValueError):
        apc.apc_norm_rows(x, torch.zeros(2, 32), weight=torch.zeros(31))
    with pytest.raises(ValueError):
        apc.KvCache(torch.zeros(2, 1, 16, 16), torch.zeros(2, 1, 16, 32))
    with pytest.raises(ValueError):
        apc.KvCache(torch.zeros(2, 16, 16), torch.zeros(2, 16, 16))
