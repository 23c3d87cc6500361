"""The plan that the library makes for an attention of several new tokens (host
only): rows of a tile, tiles, parts of the keys.  Not part of the C ABI: the
structure mirrors PromptPlan in csrc/apc_internal.h, and plan() checks that the
two agree."""
import ctypes

import paper_2502_06798_amd as apc
from paper_2502_06798_amd import binding

DT = {"f16": 1, "bf16": 2, "e4m3": 3}


class Plan(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int32) for f in ("shift", "dp", "rows", "tiles", "splits", "unit_rows", "min_tiles")] +
                [("to_cap", ctypes.c_float), ("bias", ctypes.c_int32), ("lift", ctypes.c_int32)])


def cache(dtype, heads, d, page, n_pages=1000):
    """A cache's description without its memory: addresses that no host call follows."""
    scale = 4096 if dtype == "e4m3" else None
    return binding._KvStruct(DT[dtype], heads, d, page, n_pages, 4096, 4096, scale, scale)


def plan(dtype, t, b, heads, group, d, page, max_pages, window=0, prefix=False):
    f = apc.load()._ZN3apc11plan_promptERK6apc_kvliiiib
    f.argtypes = [ctypes.c_void_p, ctypes.c_int64] + [ctypes.c_int32] * 4 + [ctypes.c_bool]
    f.restype = Plan
    c = cache(dtype, heads, d, page)
    p = f(ctypes.addressof(c), t, b, heads * group, max_pages, window if window < 2 ** 30 else 0, prefix)
    assert 1 << p.shift == page and p.dp >= d and p.rows in (32, 128) and (p.to_cap, p.bias, p.lift) == (0, 0, 0)
    return p


def workspace(dtype, t, b, heads, group, d, page, max_pages):
    n, c = ctypes.c_size_t(), cache(dtype, heads, d, page)
    f = apc.load().apc_attend_prompt_workspace
    assert f(ctypes.byref(c), t, b, heads * group, max_pages, ctypes.byref(n)) == 0
    return n.value


def plan_of(made, cache, window=0, prefix=None, **_):
    """The plan of a call over (pool, table, queries, starts, lengths)."""
    pool, table, q = made[:3]
    _, heads, page, d = pool[0].shape
    return plan(cache, q.shape[0], table.shape[0], heads, q.shape[1] // heads, d, page, table.shape[1], window,
                prefix is not None)
