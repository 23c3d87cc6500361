"""Prompts read whole: what the prompt model's positions and its attention over many new tokens cost, in plain torch and
through the library's entry points.

Two operators, in the order a layer of the text model calls them when it reads whole prompts, or the next piece of them:

* ``rotate``  rotary positions of the new tokens' queries and keys (views of the fused product's output): both layouts,
              a part of the head, frequencies scaled for long contexts;
* ``attend``  attention of several new tokens of each sequence over its cached tokens, theirs among them: causal, with a
              prefix that every token sees or both ways, within a window, scores capped by a tanh or lowered with the
              distance; single tokens are its smallest form.

Hidden rows are Gaussian. Keys and values are Gaussian rows, each head with a magnitude of its own, and queries such that
a token's weights spread over some tens of the tokens it sees. Pages of a sequence lie anywhere in the pool; new tokens'
rows stand one sequence after the other.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}


# ---- cases -------------------------------------------------------------------------------------------------------

def _rotate(name, tokens, heads, other, d, rot, dtype, interleaved, factor=1.0, original=0, far=2_048):
    """heads: rotated ones; other: heads of the same rows that are not (the values). far: positions are below it."""
    return {"name": name, "kind": "rotate", "tokens": tokens, "heads": heads, "other": other, "d": d, "rot": rot,
            "dtype": dtype, "interleaved": interleaved, "factor": factor, "original": original, "far": far}


def _attend(name, b, new, past, group, heads, d, dtype, cache, page, window=0, cap=0.0, bias=False, prefix="none", empty=0):
    """new, past: (least, most) new tokens of a sequence, and tokens cached before them. prefix: what every token sees."""
    return {"name": name, "kind": "attend", "b": b, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
            "past_hi": past[1], "group": group, "heads": heads, "d": d, "dtype": dtype, "cache": cache, "page": page,
            "window": window, "cap": cap, "bias": bias, "prefix": prefix, "empty": empty}


def listed():
    return [
        # one prompt's newest token: 12 query and 4 key heads
        _rotate("rotate_t1_h16_d64_f16", 1, 16, 4, 64, 64, "f16", False),
        # half of each head, neighbouring elements in pairs, an odd number of tokens in float32
        _rotate("rotate_t1001_h7_d80_rot40_f32_pairs", 1_001, 7, 0, 80, 40, "f32", True),
        # all tokens of a large batch of prompts, at far positions of a context that was made longer
        _rotate("rotate_t65536_h40_d128_bf16_scaled", 65_536, 40, 8, 128, 128, "bf16", False, 8.0, 8_192, 131_072),
        # one prompt of a text encoder
        _attend("attend_b1_n77_g1_h12_d64_f16", 1, (77, 77), (0, 0), 1, 12, 64, "f16", "f16", 16),
        # a batch of prompts read both ways, scores lowered with the distance
        _attend("attend_b16_n77_g1_h12_d64_f16_bias_both", 16, (5, 77), (0, 0), 1, 12, 64, "f16", "f16", 16, bias=True, prefix="all"),
        # odd sizes: new tokens behind ragged pasts, a window, capped scores, two sequences without a token
        _attend("attend_b7_n333_g5_h2_d80_f16_e4m3_window_cap", 7, (1, 333), (0, 1_500), 5, 2, 80, "f16", "e4m3", 16, 700, 20.0, empty=2),
        # an ordinary batch of whole prompts, scores capped
        _attend("attend_b8_n2048_g4_h8_d128_bf16_cap", 8, (1_000, 2_048), (0, 0), 4, 8, 128, "bf16", "bf16", 32, cap=30.0),
        # the next piece of prompts over what is cached, a third of the piece seen by all of it
        _attend("attend_b16_n512_past1536_g4_h8_d128_bf16_e4m3_prefix", 16, (300, 512), (500, 1_536), 4, 8, 128, "bf16", "e4m3", 32, prefix="part"),
        # the largest in operations: two long documents
        _attend("attend_b2_n8192_g4_h8_d128_bf16", 2, (8_192, 8_192), (0, 0), 4, 8, 128, "bf16", "bf16", 64),
        # a piece of one document against its long past, scores lowered with the distance
        _attend("attend_b1_n1024_past64512_g8_h4_d128_bf16_bias", 1, (1_024, 1_024), (64_512, 64_512), 8, 4, 128, "bf16", "bf16", 64, bias=True),
        # one new token of one long document, capped
        _attend("attend_b1_n1_past131071_g8_h8_d128_bf16_e4m3_cap", 1, (1, 1), (131_071, 131_071), 8, 8, 128, "bf16", "e4m3", 64, cap=30.0),
        # the largest in bytes: one new token of each of many long contexts
        _attend("attend_b64_n1_past32767_g4_h8_d128_bf16_e4m3_bias", 64, (1, 1), (16_383, 32_767), 4, 8, 128, "bf16", "e4m3", 64, bias=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    half = rng.choice(("f16", "bf16"))
    if rng.random() < 0.3:
        d = rng.choice((64, 64, 128, 128, 256, 2 * rng.randint(8, 128)))
        rot = rng.choice((d, d, d // 4 * 2, 2 * rng.randint(1, d // 2)))
        heads, dtype = rng.randint(1, 64), rng.choice(("f32", half, half))
        t = _log(rng, 1, 65_536 * 40 * 128 * 2 // (heads * d * SIZE[dtype]))
        factor = rng.choice((1.0, 1.0, 4.0, 8.0))
        case = _rotate("", t, heads, rng.choice((0, 4)), d, rot, dtype, rng.random() < 0.4, factor,
                       rng.choice((0, 4_096)) if factor > 1.0 else 0, _log(rng, 128, 1 << 20))
        del case["name"]
        return case
    group, heads, page = rng.choice((1, 2, 4, 4, 5, 8, 8, 16)), rng.randint(1, 12), rng.choice((16, 32, 64, 128, 256))
    d = rng.choice((64, 64, 128, 128, 128, 256, 16 * rng.randint(1, 16)))
    cache = rng.choice((half, "e4m3"))
    q_heads = group * heads
    if rng.random() < 0.35:         # single tokens, or a few, of each sequence
        b = _log(rng, 1, 256)
        new = rng.choice(((1, 1), (1, 1), (1, 4)))
        most = min(131_072, 64 * 24_576 * 8 * 128 // (b * heads * d * SIZE[cache] * (2 if group > 8 else 1)))
        past = _log(rng, 1, max(1, most // new[1]))
        past = (rng.choice((past, past // 2, 0)), past)
    else:                           # prompts, or pieces of them
        b = _log(rng, 1, 32)
        pairs = (1 << 31) * 128 // (max(128, d) * b * q_heads)      # of a new token and a token
        most = min(8_192, int(math.sqrt(pairs)))
        n = _log(rng, 1, max(1, most))
        new = (rng.choice((n, 1 + n // 2, 1)), n)
        room = max(1, min(pairs // n, 65_536, (1 << 30) // (b * heads * d)) - n)
        past = rng.choice((0, 0, _log(rng, 1, room)))
        past = (rng.choice((past, past // 2, 0)), past)
    hi = new[1] + past[1]
    case = _attend("", b, new, past, group, heads, d, half, cache, page, rng.choice((0, 0, 0, 1 + hi // 3)),
                   rng.choice((0.0, 0.0, 20.0, 50.0)), rng.random() < 0.3, rng.choice(("none", "none", "part", "all")),
                   rng.choice((0, 0, b // 5)))
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + stream * 7_919 + 50_021) & ((1 << 62) - 1))
    return g


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


def _spread(lo, hi, b):
    return [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]


def _sizes(case):
    """(new tokens, all tokens) of each sequence, before the seed puts them into another order: the longest pasts stand
    with the fewest new tokens, the first `empty` sequences hold nothing."""
    b = case["b"]
    new, past = _spread(case["new_lo"], case["new_hi"], b), _spread(case["past_lo"], case["past_hi"], b)[::-1]
    return [(0, 0) if i < case["empty"] else (n, n + p) for i, (n, p) in enumerate(zip(new, past))]


def _prefix(case, n, length):
    return {"none": 0, "part": length - n + n // 3, "all": length}[case["prefix"]]


def _seen(case, n, length, at):
    """First token that the token at position `at` (a tensor) sees, and the end of those it sees."""
    end = torch.clamp(at + 1, min=_prefix(case, n, length))
    first = torch.zeros_like(at)
    if case["window"]:
        first = torch.clamp(at + 1 - case["window"], min=0)
        end = torch.minimum(end, at + case["window"])
    return first, torch.clamp(end, max=length)


def _frequencies(case):
    """Angle of one position for each pair, in float64: base 10,000, divided by the factor, or (for a context of `original`
    positions made longer) by a factor that goes from 1 for what turns 4 times or more in it to the whole for what turns once or less."""
    half = case["rot"] // 2
    f = 10_000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    if not case["original"]:
        return f / case["factor"]
    part = ((case["original"] * f / (2.0 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
    return part * f + (1.0 - part) * f / case["factor"]


def prepare(case, seed):
    g, dt = _gen(seed, 1), DTYPE[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "rotate":
        t, heads, d = case["tokens"], case["heads"], case["d"]
        # what the product of the hidden states gives: queries, keys and values of a token side by side
        st["x"] = torch.randn((t, heads + case["other"], d), device="cuda", generator=g).to(dt)[:, :heads]
        st["at"] = torch.randint(0, case["far"], (t,), device="cuda", generator=g, dtype=torch.int32)
        st["freq"] = _frequencies(case).cuda()
        st["out"] = torch.empty((t, heads, d), dtype=dt, device="cuda")
        if own:
            # the description of the positions that a program keeps with its model
            import paper_2502_06798_amd as apc
            st["rotary"] = apc.Rotary(st["freq"], interleaved=case["interleaved"])
        return st
    b, heads, group, page, d = case["b"], case["heads"], case["group"], case["page"], case["d"]
    order = torch.randperm(b, device="cuda", generator=g).tolist()
    sizes = [_sizes(case)[i] for i in order]
    new, lens = torch.tensor([n for n, _ in sizes]), [n for _, n in sizes]
    t, per = int(new.sum()), max(1, -(-max(lens) // page))
    st["starts"] = torch.cat([new.new_zeros(1), new.cumsum(0)]).to(torch.int32).cuda()
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["prefix"] = None
    if case["prefix"] != "none":
        st["prefix"] = torch.tensor([_prefix(case, *s) for s in sizes], dtype=torch.int32, device="cuda")
    st["slopes"] = None
    if case["bias"]:
        st["slopes"] = torch.exp2(-8.0 * (torch.arange(heads * group, device="cuda") + 1.0) / (heads * group))
    # where each new token's row is in a rectangle of b x (most new tokens): for the plain form
    st["most"] = int(new.max())
    st["seq"] = torch.repeat_interleave(torch.arange(b), new).cuda()
    st["row"] = torch.cat([torch.arange(n) for n, _ in sizes]).cuda()
    st["table"] = torch.randperm(b * per, device="cuda", generator=g).to(torch.int32).reshape(b, per)
    st["kp"], st["ks"] = _pool(b * per, heads, page, d, case["cache"], g)
    st["vp"], st["vs"] = _pool(b * per, heads, page, d, case["cache"], g)
    st["q"] = (torch.randn((t, heads * group, d), device="cuda", generator=g) * 2.0).to(dt)
    st["scale"] = d ** -0.5
    st["out"] = torch.empty((t, heads * group, d), dtype=dt, device="cuda")
    st["lse"] = torch.empty((t, heads * group), device="cuda")
    if own:
        # the handle and the workspace that a program keeps for a pool; they hold nothing of the inputs
        import paper_2502_06798_amd as apc
        st["cache"] = apc.KvCache(st["kp"], st["vp"], st["ks"], st["vs"])
        st["ws"] = apc.attend_prompt_workspace_tensor(st["cache"], t, b, heads * group, per)
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------

def _run_own(st):
    import paper_2502_06798_amd as apc
    case = st["case"]
    if case["kind"] == "rotate":
        apc.apc_rotate(st["rotary"], st["x"], st["at"], st["out"])
        return {"out": st["out"]}
    apc.apc_attend_prompt(st["cache"], st["q"], st["starts"], st["table"], st["lens"], st["scale"], st["out"], st["ws"],
                          st["lse"], window=case["window"], cap=case["cap"], slopes=st["slopes"], prefix=st["prefix"])
    return {"out": st["out"], "lse": st["lse"]}


def _rotate_plain(st):
    case = st["case"]
    rot, half = case["rot"], case["rot"] // 2
    angle = st["at"].double()[:, None] * st["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = st["x"].float()
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return {"out": torch.cat((turned, x[..., rot:]), dim=-1).to(st["x"].dtype)}


def _tokens(pool, scale, table, length):
    """float32 rows of every sequence's tokens: b x heads x (pages x page) x d, zeros past its length."""
    x = pool.view(torch.uint8)[table].view(pool.dtype).float() if scale is not None else pool[table].float()
    if scale is not None:
        x *= scale[table][..., None]
    b, pages, heads, page, d = x.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(b, heads, pages * page, d)
    return x.masked_fill_((torch.arange(pages * page, device="cuda") >= length[:, None])[:, None, :, None], 0.0)


def _attend_plain(st):
    case = st["case"]
    b, heads, group, d, most = case["b"], case["heads"], case["group"], case["d"], st["most"]
    table = st["table"].long()
    length = st["lens"].long()
    q = torch.zeros((b, most, heads, group, d), device="cuda")
    q[st["seq"], st["row"]] = st["q"].float().view(-1, heads, group, d)
    q = q.permute(0, 2, 3, 1, 4).reshape(b, heads, group * most, d)
    k = _tokens(st["kp"], st["ks"], table, length)
    s = torch.matmul(q, k.transpose(-1, -2)).view(b, heads, group, most, -1)
    del k
    s *= st["scale"]
    if case["cap"]:
        s = torch.tanh(s / case["cap"]) * case["cap"]
    new = st["starts"].long().diff()
    at = (length - new)[:, None, None] + torch.arange(most, device="cuda")[:, None]
    token = torch.arange(s.shape[-1], device="cuda")
    away = (at - token).abs()                                               # b x most x tokens
    if case["bias"]:
        s -= st["slopes"].view(1, heads, group, 1, 1) * away[:, None, None]
    seen = token <= at
    if st["prefix"] is not None:
        seen |= token < st["prefix"][:, None, None]
    if case["window"]:
        seen &= away < case["window"]
    seen &= token < length[:, None, None]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(dim=-1, keepdim=True).clamp(min=-3.0e38)
    p = torch.exp(s - m)
    del s
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p.view(b, heads, group * most, -1), _tokens(st["vp"], st["vs"], table, length))
    out = (out.view(b, heads, group, most, d) / total.clamp(min=1e-38)).permute(0, 3, 1, 2, 4)[st["seq"], st["row"]]
    lse = (m + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2)[st["seq"], st["row"]]
    return {"out": out.reshape(-1, heads * group, d).to(st["q"].dtype), "lse": lse.reshape(-1, heads * group)}


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _rotate_plain, "attend": _attend_plain}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] == "rotate":
        rows = case["tokens"] * case["heads"]
        return {"bytes": 2 * rows * case["d"] * e + 4 * case["tokens"] + 4 * case["rot"], "flops": 3 * rows * case["rot"]}
    heads, d, ec, hq = case["heads"], case["d"], SIZE[case["cache"]], case["heads"] * case["group"]
    scales = 8 if case["cache"] == "e4m3" else 0
    pairs = kept = entries = t = 0
    for n, length in _sizes(case):
        if n == 0:
            continue
        first, end = _seen(case, n, length, torch.arange(length - n, length))
        lo, hi = int(first.min()), int(end.max())
        pairs += int((end - first).clamp(min=0).sum())
        kept += hi - lo
        entries += (hi - 1) // case["page"] - lo // case["page"] + 1
        t += n
    return {"bytes": kept * heads * (2 * d * ec + scales) + t * hq * (2 * d * e + 4) + 4 * (entries + 2 * case["b"]),
            "flops": 4 * pairs * hq * d}


# ---- 64 bits -----------------------------------------------------------------------------------------------------

def _exact_rotate(case, st):
    half = case["rot"] // 2
    turns = torch.outer(st["at"].double(), st["freq"])
    by = torch.polar(torch.ones_like(turns), turns)[:, None]                # e^(i angle)
    x = st["x"].double()
    even = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
    odd = even + (1 if case["interleaved"] else half)
    z = torch.complex(x[..., even], x[..., odd]) * by
    y = x.clone()
    y[..., even], y[..., odd] = z.real, z.imag
    return {"out": y}


def _exact_rows(pool, scale, pages, h):
    """float64 tokens of head h of one sequence from its page numbers."""
    x = pool.view(torch.uint8)[pages, h].view(pool.dtype).double() if scale is not None else pool[pages, h].double()
    if scale is not None:
        x = x * scale[pages, h].double().unsqueeze(-1)
    return x.flatten(0, 1)


def _exact_attend(case, st):
    heads, group, d, page = case["heads"], case["group"], case["d"], case["page"]
    outs = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lses = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    starts, lens = st["starts"].tolist(), st["lens"].tolist()
    for i, length in enumerate(lens):
        n = starts[i + 1] - starts[i]
        if n == 0:
            continue
        at = torch.arange(length - n, length, device="cuda")
        first, end = _seen(case, n, length, at)
        j = torch.arange(length, device="cuda")
        hidden = (j < first[:, None]) | (j >= end[:, None])
        pages = st["table"][i, :-(-length // page)].long()
        rows = slice(starts[i], starts[i + 1])
        for h in range(heads):
            k, v = (_exact_rows(st[p], st[c], pages, h)[:length] for p, c in (("kp", "ks"), ("vp", "vs")))
            for a in range(h * group, (h + 1) * group):
                s = (st["q"][rows, a].double() @ k.t().contiguous()) * st["scale"]
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["bias"]:
                    s -= float(st["slopes"][a]) * (at[:, None] - j).abs()
                s.masked_fill_(hidden, -math.inf)
                lses[rows, a] = torch.logsumexp(s, dim=1)
                outs[rows, a] = torch.softmax(s, dim=1) @ v
    return {"out": outs, "lse": lses}


def exact(case, seed):
    st = prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend}[case["kind"]](case, st)
