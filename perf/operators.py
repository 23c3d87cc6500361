"""The prompt model's operators: what a step of it costs, in plain torch and through the library's entry points.

Three operators, in the order a step of the text model calls them for its new tokens:

* ``norm``    the residual's addition and root-mean-square norm of rows, to the rows' type or to e4m3 rows with a scale
              each (the form in which the matching step takes queries);
* ``write``   keys and values of new tokens into a paged cache, rounded or quantised (e4m3 codes, a scale per token and
              head) as they are written, and ``read``: cached tokens back as rows;
* ``attend``  attention of one new token per sequence over its cached tokens, query heads sharing key-value heads.

Hidden states are Gaussian rows of varying magnitude with a few strong channels; keys and values are Gaussian rows, each
head with a magnitude of its own, and queries such that a sequence's weights spread over some tens of its tokens. Pages
of a sequence lie anywhere in the pool. A slot or a page entry below zero stands for none.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------------------------------

def _norm(name, n, d, dtype, out, res, pad=0):
    return {"name": name, "kind": "norm", "n": n, "d": d, "dtype": dtype, "out": out, "res": res, "pad": pad}


def _write(name, tokens, heads, d, dtype, cache, page, skip, spread=False):
    return {"name": name, "kind": "write", "tokens": tokens, "heads": heads, "d": d, "dtype": dtype, "cache": cache,
            "page": page, "skip": skip, "spread": spread}


def _read(name, tokens, heads, d, cache, out, page, skip, spread=False):
    return {"name": name, "kind": "read", "tokens": tokens, "heads": heads, "d": d, "cache": cache, "dtype": out,
            "page": page, "skip": skip, "spread": spread}


def _attend(name, b, lo, hi, group, heads, d, dtype, cache, page, window=0, empty=0):
    return {"name": name, "kind": "attend", "b": b, "lo": lo, "hi": hi, "group": group, "heads": heads, "d": d,
            "dtype": dtype, "cache": cache, "page": page, "window": window, "empty": empty}


def listed():
    return [
        # one prompt's newest token, between two layers
        _norm("norm_n1_d768_f16", 1, 768, "f16", "f16", True),
        # float32 states of an odd width and number, views into wider rows, to e4m3 rows
        _norm("norm_n1001_d999_f32_e4m3", 1_001, 999, "f32", "e4m3", False, 6),
        # all tokens of a large batch of prompts, residual kept, 8-bit rows out
        _norm("norm_n65536_d4096_bf16_e4m3", 65_536, 4_096, "bf16", "e4m3", True),
        # one new token of each of 16 prompts
        _write("write_t16_h12_d64_f16", 16, 12, 64, "f16", "f16", 16, 0, True),
        # a large batch of whole prompts, quantised; its last tokens are padding
        _write("write_t65536_h8_d128_bf16_e4m3", 65_536, 8, 128, "bf16", "e4m3", 64, 1_500),
        # a few prompts' tokens handed on as rows, off every tile
        _read("read_t777_h5_d80_f16_f32", 777, 5, 80, "f16", "f32", 32, 7),
        # the cached prefixes of a large batch
        _read("read_t100003_h8_d128_e4m3_bf16", 100_003, 8, 128, "e4m3", "bf16", 64, 0),
        # one prompt of 77 tokens, a head of its own for every query head
        _attend("attend_b1_n77_g1_h12_d64_f16", 1, 77, 77, 1, 12, 64, "f16", "f16", 16),
        # odd sizes, a window, two sequences that hold nothing yet
        _attend("attend_b7_n3001_g5_h2_d80_f16_e4m3", 7, 1, 3_001, 5, 2, 80, "f16", "e4m3", 16, 1_000, 2),
        # an ordinary batch of prompts of mixed length
        _attend("attend_b256_n2048_g4_h8_d128_bf16", 256, 100, 2_048, 4, 8, 128, "bf16", "bf16", 32),
        # one long document
        _attend("attend_b1_n131072_g8_h8_d128_bf16_e4m3", 1, 131_072, 131_072, 8, 8, 128, "bf16", "e4m3", 64),
        # the largest: many long contexts
        _attend("attend_b64_n32768_g4_h8_d128_bf16_e4m3", 64, 16_384, 32_768, 4, 8, 128, "bf16", "e4m3", 64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "write", "read", "attend", "attend", "attend", "attend"))
    half = rng.choice(("f16", "bf16"))
    if kind == "norm":
        d = _log(rng, 64, 16_384)
        if rng.random() < 0.6:
            d = (d + 15) // 16 * 16
        dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
        n = _log(rng, 1, 65_536 * 4_096 * 2 // (SIZE[dtype] * d))
        return {k: v for k, v in _norm("", n, d, dtype, rng.choice((dtype, "e4m3", "e4m3")), rng.random() < 0.6,
                                       rng.choice((0, 0, 8, 3))).items() if k != "name"}
    heads, page = rng.randint(1, 16), rng.choice((16, 32, 64, 128, 256))
    d = rng.choice((64, 64, 128, 128, 128, 256, 16 * rng.randint(1, 16)))
    cache = rng.choice((half, "e4m3"))
    if kind in ("write", "read"):
        dtype = rng.choice(("f32", half, half))
        t = _log(rng, 1, 65_536 * 1_024 // (heads * d))
        make = (lambda *a: _write("", t, heads, d, dtype, cache, *a)) if kind == "write" else \
            (lambda *a: _read("", t, heads, d, cache, dtype, *a))
        return {k: v for k, v in make(page, rng.choice((0, t // 9)), rng.random() < 0.3).items() if k != "name"}
    group = rng.choice((1, 2, 4, 4, 5, 8, 8, 16, 24))
    b = _log(rng, 1, 256)
    most = min(131_072, 64 * 24_576 * 8 * 128 // (b * heads * d * SIZE[cache] * (2 if group > 8 else 1)))
    hi = _log(rng, 1, max(1, most))
    lo = rng.choice((hi, 1 + hi // 2, 1))
    return {k: v for k, v in _attend("", b, lo, hi, group, heads, d, half, cache, page,
                                     rng.choice((0, 0, 0, 1 + hi // 3)), rng.choice((0, b // 5))).items() if k != "name"}


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + stream * 7_919 + 24_691) & ((1 << 62) - 1))
    return g


def _states(n, d, dtype, pad, g):
    """Rows of d values in rows of d + pad."""
    x = torch.randn((n, d + pad), device="cuda", generator=g)
    x *= torch.exp(torch.randn((n, 1), device="cuda", generator=g) * 0.5)
    x *= 1.0 + 9.0 * (torch.rand(d + pad, device="cuda", generator=g) < 0.01)
    return x.to(DTYPE[dtype])[:, :d]


def _pool(pages, heads, page, d, dtype, g):
    """A pool's pages as a cache holds them after many writes: values or codes, and the scales (e4m3)."""
    out = torch.empty((pages, heads, page, d), dtype=DTYPE[dtype], device="cuda")
    scale = torch.empty((pages, heads, page), device="cuda") if dtype == "e4m3" else None
    size = 0.5 + torch.rand((heads, 1, 1), device="cuda", generator=g)
    step = max(1, (1 << 28) // (heads * page * d))
    for p0 in range(0, pages, step):
        p1 = min(pages, p0 + step)
        x = torch.randn((p1 - p0, heads, page, d), device="cuda", generator=g) * size
        if scale is not None:
            s = x.abs().amax(dim=3) / 448.0
            scale[p0:p1] = s
            x = (x / s[..., None]).clamp_(-448.0, 448.0)
        out[p0:p1] = x.to(out.dtype)
    return out, scale


def _lengths(case):
    """Lengths of the sequences, evenly from lo to hi, the first `empty` of them 0 (their order comes from the seed)."""
    b, lo, hi = case["b"], case["lo"], case["hi"]
    n = [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]
    return [0] * case["empty"] + n[:b - case["empty"]]


def _kept(case):
    w = case["window"]
    return [min(n, w) if w else n for n in _lengths(case)]


def prepare(case, seed):
    g, dt = _gen(seed, 1), DTYPE[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "norm":
        n, d = case["n"], case["d"]
        st["x"] = _states(n, d, case["dtype"], case["pad"], g)
        st["res"] = _states(n, d, case["dtype"], case["pad"], g) if case["res"] else None
        st["w"] = (1.0 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(dt)
        st["sum"] = torch.empty((n, d), dtype=dt, device="cuda") if case["res"] else None
        st["out"] = torch.empty((n, d), dtype=DTYPE[case["out"]], device="cuda")
        st["scale"] = torch.empty(n, device="cuda") if case["out"] == "e4m3" else None
        return st
    heads, page, d = case["heads"], case["page"], case["d"]
    if case["kind"] in ("write", "read"):
        t = case["tokens"]
        pages = -(-t // page) + 3
        if case["spread"]:          # single tokens of many sequences, anywhere
            slots = torch.randperm(pages * page, device="cuda", generator=g)
        else:                       # whole pages, in any order
            slots = (torch.randperm(pages, device="cuda", generator=g)[:, None] * page
                     + torch.arange(page, device="cuda")).reshape(-1)
        slots = slots[:t].to(torch.int32)
        if case["skip"]:
            slots[t - case["skip"]:] = -1
        st["slots"] = slots
        st["kp"], st["ks"] = _pool(pages, heads, page, d, case["cache"], g)
        st["vp"], st["vs"] = _pool(pages, heads, page, d, case["cache"], g)
        if case["kind"] == "write":
            # what the product of the hidden states gives: queries, keys and values of a token side by side
            qkv = torch.randn((t, 3 * heads, d), device="cuda", generator=g).to(dt)
            st["k"], st["v"] = qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
        else:
            st["k"], st["v"] = (torch.empty((t, heads, d), dtype=dt, device="cuda") for _ in range(2))
    else:
        b, group = case["b"], case["group"]
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        st["lens"] = lens[torch.randperm(b, device="cuda", generator=g)].contiguous()
        per = max(1, -(-case["hi"] // page))
        st["table"] = torch.randperm(b * per, device="cuda", generator=g).to(torch.int32).reshape(b, per)
        st["kp"], st["ks"] = _pool(b * per, heads, page, d, case["cache"], g)
        st["vp"], st["vs"] = _pool(b * per, heads, page, d, case["cache"], g)
        st["q"] = (torch.randn((b, heads * group, d), device="cuda", generator=g) * 2.0).to(dt)
        st["scale"] = d ** -0.5
        st["out"] = torch.empty((b, heads * group, d), dtype=dt, device="cuda")
        st["lse"] = torch.empty((b, heads * group), device="cuda")
    if own:
        # the handle and the workspace that a program keeps for a pool; they hold nothing of the inputs
        import paper_2502_06798_amd as apc
        st["cache"] = apc.KvCache(st["kp"], st["vp"], st["ks"], st["vs"])
        if case["kind"] == "attend":
            st["ws"] = apc.attend_workspace_tensor(st["cache"], b, heads * group, per)
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------

def _run_own(st):
    import paper_2502_06798_amd as apc
    case = st["case"]
    if case["kind"] == "norm":
        apc.apc_norm_rows(st["x"], st["out"], st["w"], st["res"], st["sum"], st["scale"], EPS)
        return {"out": st["out"], "scale": st["scale"], "sum": st["sum"]}
    if case["kind"] == "write":
        apc.apc_kv_write(st["cache"], st["k"], st["v"], st["slots"])
        return {"k": st["kp"], "v": st["vp"], "ks": st["ks"], "vs": st["vs"]}
    if case["kind"] == "read":
        apc.apc_kv_read(st["cache"], st["slots"], st["k"], st["v"])
        return {"k": st["k"], "v": st["v"]}
    apc.apc_attend(st["cache"], st["q"], st["table"], st["lens"], st["scale"], st["out"], st["ws"], st["lse"],
                   case["window"])
    return {"out": st["out"], "lse": st["lse"]}


def _codes(y):
    """e4m3 values of rows (last axis) and their scales."""
    s = y.abs().amax(dim=-1) / 448.0
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (y / s[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), s


def _norm_plain(st):
    case = st["case"]
    h = st["x"].float()
    if st["res"] is not None:
        h = h + st["res"].float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * st["w"].float()
    total = None if st["res"] is None else h.to(st["x"].dtype)
    if case["out"] == "e4m3":
        codes, s = _codes(y)
        return {"out": codes, "scale": s, "sum": total}
    return {"out": y.to(st["x"].dtype), "scale": None, "sum": total}


def _put(pool, scale, x, page, off):
    if scale is None:
        pool[page, :, off] = x.float().to(pool.dtype)
        return
    codes, s = _codes(x.float())
    pool.view(torch.uint8)[page, :, off] = codes.view(torch.uint8)
    scale[page, :, off] = s


def _write_plain(st):
    size = st["case"]["page"]
    keep = (st["slots"] >= 0).nonzero().reshape(-1)
    slots = st["slots"][keep].long()
    page, off = slots // size, slots % size
    _put(st["kp"], st["ks"], st["k"][keep], page, off)
    _put(st["vp"], st["vs"], st["v"][keep], page, off)
    return {"k": st["kp"], "v": st["vp"], "ks": st["ks"], "vs": st["vs"]}


def _get(pool, scale, page, off, some, dtype):
    x = pool.view(torch.uint8)[page, :, off].view(pool.dtype).float() if scale is not None else pool[page, :, off].float()
    if scale is not None:
        x = x * scale[page, :, off][..., None]
    return torch.where(some, x, torch.zeros_like(x)).to(dtype)


def _read_plain(st):
    size = st["case"]["page"]
    slots = st["slots"].clamp(min=0).long()
    page, off, some = slots // size, slots % size, (st["slots"] >= 0)[:, None, None]
    return {"k": _get(st["kp"], st["ks"], page, off, some, st["k"].dtype),
            "v": _get(st["vp"], st["vs"], page, off, some, st["v"].dtype)}


def _tokens(pool, scale, table, seen):
    """float32 rows of every sequence's tokens: b x heads x (pages x page) x d, zeros where none is seen."""
    x = pool.view(torch.uint8)[table].view(pool.dtype).float() if scale is not None else pool[table].float()
    if scale is not None:
        x *= scale[table][..., None]
    b, pages, heads, page, d = x.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(b, heads, pages * page, d)
    return x.masked_fill_(~seen[:, None, :, None], 0.0)


def _attend_plain(st):
    case = st["case"]
    b, heads, group, d = case["b"], case["heads"], case["group"], case["d"]
    at = torch.arange(st["table"].shape[1] * case["page"], device="cuda")
    lens = st["lens"][:, None]
    seen = at < lens
    if case["window"]:
        seen &= at >= lens - case["window"]
    table = st["table"].long()
    q = st["q"].float().view(b, heads, group, d)
    s = torch.matmul(q, _tokens(st["kp"], st["ks"], table, seen).transpose(-1, -2)) * st["scale"]
    s.masked_fill_(~seen[:, None, None, :], -math.inf)
    m = s.amax(dim=-1, keepdim=True).clamp(min=-3.0e38)
    p = torch.exp(s - m)
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p, _tokens(st["vp"], st["vs"], table, seen)) / total.clamp(min=1e-38)
    return {"out": out.reshape(b, heads * group, d).to(st["q"].dtype),
            "lse": (m + torch.log(total)).reshape(b, heads * group)}


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _norm_plain, "write": _write_plain, "read": _read_plain, "attend": _attend_plain}[
        state["case"]["kind"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] == "norm":
        n, d = case["n"], case["d"]
        per = e + SIZE[case["out"]] + (2 * e if case["res"] else 0)
        return {"bytes": n * d * per + d * e + (4 * n if case["out"] == "e4m3" else 0), "flops": n * d * 6}
    heads, d, ec = case["heads"], case["d"], SIZE[case["cache"]]
    scales = 8 if case["cache"] == "e4m3" else 0
    if case["kind"] in ("write", "read"):
        t = case["tokens"] - case["skip"]
        rows = case["tokens"] if case["kind"] == "read" else t          # skipped tokens are read back as zeros
        return {"bytes": 2 * heads * d * (rows * e + t * ec) + t * heads * scales + 4 * case["tokens"],
                "flops": 2 * t * heads * d * (3 if ec == 1 else 1)}
    kept, hq = sum(_kept(case)), heads * case["group"]
    entries = sum(-(-n // case["page"]) for n in _kept(case))
    return {"bytes": kept * heads * (2 * d * ec + scales) + case["b"] * hq * (2 * d * e + 4) + 4 * (entries + case["b"]),
            "flops": 4 * kept * hq * d}


# ---- 64 bits -----------------------------------------------------------------------------------------------------

def _exact_rows(pool, scale, seq, page, heads):
    """float64 tokens of one sequence (heads x tokens x d) from its page numbers."""
    x = pool.float()[seq].double() if scale is None else pool.view(torch.uint8)[seq].view(pool.dtype).double()
    if scale is not None:
        x = x * scale[seq].double().unsqueeze(-1)
    return torch.cat(list(x), dim=1) if len(seq) else x.new_zeros((heads, 0, pool.shape[3]))


def _exact_attend(case, st):
    page, heads, group = case["page"], case["heads"], case["group"]
    outs, lses = [], []
    lens = st["lens"].tolist()
    for i, n in enumerate(lens):
        q = st["q"][i].double().reshape(heads, group, case["d"])
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            outs.append(torch.zeros_like(q).reshape(-1, case["d"]))
            lses.append(torch.full((heads * group,), -math.inf, dtype=torch.float64, device="cuda"))
            continue
        seq = st["table"][i, :-(-n // page)].long()
        k = _exact_rows(st["kp"], st["ks"], seq, page, heads)[:, first:n]
        v = _exact_rows(st["vp"], st["vs"], seq, page, heads)[:, first:n]
        rows, logs = [], []
        for h in range(heads):
            s = (q[h] @ k[h].t().contiguous()) * st["scale"]
            logs.append(torch.logsumexp(s, dim=1))
            rows.append(torch.softmax(s, dim=1) @ v[h])
        outs.append(torch.cat(rows))
        lses.append(torch.cat(logs))
    return {"out": torch.stack(outs), "lse": torch.stack(lses)}


def _exact_write(case, st):
    def pool(p, s, x):
        new, news = p.float().double(), None if s is None else s.double()
        for i in range(heads):
            rows = x[:, i].double()[ok]
            if s is not None:
                top = rows.abs().max(dim=1).values
                unit = torch.where(top > 0, top / 448.0, torch.ones_like(top))
                rows = rows / unit[:, None]
                news[at // page, i, at % page] = unit
            new[at // page, i, at % page] = rows
        return new, news

    page, heads = case["page"], case["heads"]
    ok = st["slots"] >= 0
    at = st["slots"][ok].long()
    (k, ks), (v, vs) = pool(st["kp"], st["ks"], st["k"]), pool(st["vp"], st["vs"], st["v"])
    return {"k": k, "v": v, "ks": ks, "vs": vs}


def _exact_read(case, st):
    def rows(p, s):
        x = p.float().double() if s is None else p.float().double() * s.double().unsqueeze(-1)
        flat = x.transpose(1, 2).reshape(-1, case["heads"], case["d"])
        out = torch.zeros((case["tokens"], case["heads"], case["d"]), dtype=torch.float64, device="cuda")
        ok = st["slots"] >= 0
        out[ok] = flat.index_select(0, st["slots"][ok].long())
        return out

    return {"k": rows(st["kp"], st["ks"]), "v": rows(st["vp"], st["vs"])}


def _exact_norm(case, st):
    h = st["x"].double()
    if case["res"]:
        h = st["res"].double() + h
    length = torch.sqrt(h.pow(2).sum(dim=1) / case["d"] + EPS)
    y = h / length[:, None] * st["w"].double()
    total = h if case["res"] else None
    if case["out"] != "e4m3":
        return {"out": y, "scale": None, "sum": total}
    top = y.abs().max(dim=1).values
    unit = torch.where(top > 0, top / 448.0, torch.ones_like(top))
    return {"out": y / unit[:, None], "scale": unit, "sum": total}


def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["kind"]](case, st)
