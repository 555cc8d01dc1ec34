"""A cache held in 4 bits, the attention over it, and the norms of queries and keys with their rotation:
the calls over the range in which a serving program makes them, each also in a plain form of elementary
torch operations.

"quant": a step's keys and values are quantised into MXFP4 pages (blocks of 32 dims: E2M1 codes and a
power of two), and the chunk's rows are read back as the values that later steps will see.
"read": the cached context of a batch is read back as bf16 rows.
"attn": attention of a varlen batch's chunks over MXFP4 pages that hold prefix and chunk.
"norm": queries and keys of a projected row are normed for each head and rotated; keys and values go
into bf16 or e4m3 pages, or ("none") the keys into rows of their own.

`own` picks the framework's calls; otherwise the plain form runs, in 32 bits (angles in 64) whatever the
inputs' type, rounded at the end.  Keys for e4m3 pages are first rounded to bf16, as the separate calls
round them; such pages come back as float8 values, without their head's scale.
"""
import math
import random

import torch

own = False

DEV = "cuda"
D, PAGE = 128, 16
BLOCK = 32                      # dims that share a power of two
RUN = PAGE * (D // 2 + D // BLOCK)   # bytes of one page of one kv head: codes, then scales
SCALE = D ** -0.5
MOST_SCORES = 1 << 31           # of a group of requests that the plain form of attention takes at once


def _case(name, op, **kw):
    case = dict(op=op, reqs=1, p_lo=0, p_hi=0, c_lo=1, c_hi=1, c_mode="uniform", lens=1, hq=32, hkv=8)
    if op == "norm":
        case.update(kv="bf16", rot=128, layout="halves", weights="bf16", offset=0.0)
    case.update(kw)
    return dict(name=name, **case)


def listed():
    return [
        # the smallest step of a decoding request: one row into its page and back, so latency and nothing else
        _case("quant_one", "quant", p_lo=2047, p_hi=2047),
        # a full mixed step: chunks from one token to 2048
        _case("quant_mixed", "quant", reqs=64, p_lo=0, p_hi=32768, c_lo=1, c_hi=2048, c_mode="lognormal", lens=4),
        # contexts of a few requests on their way to a place that takes values: odd lengths
        _case("read_contexts", "read", reqs=8, p_lo=1001, p_hi=16384, lens=5),
        # one decoding request's layer: a 2048-token context
        _case("attn_one", "attn", p_lo=2047, p_hi=2047),
        # a decode batch at ragged contexts, 70B-like heads
        _case("attn_decode", "attn", reqs=64, p_lo=1, p_hi=16384, hq=64, lens=2),
        # few rows over very long contexts, which 4 bits are kept for
        _case("attn_decode_long", "attn", reqs=4, p_lo=120000, p_hi=131071, lens=3),
        # a streamed chunk on 8192 cached tokens
        _case("attn_chunk", "attn", p_lo=8192, p_hi=8192, c_lo=512, c_hi=512),
        # a full mixed step: chunks from one token to 2048 on up to 32768 cached tokens
        _case("attn_mixed", "attn", reqs=32, p_lo=0, p_hi=32768, c_lo=1, c_hi=2048, c_mode="lognormal", lens=6),
        # one decoding row, normed, rotated and appended
        _case("norm_append_one", "norm", p_lo=2047, p_hi=2047),
        # a decode batch into e4m3 pages, 70B-like heads, fp32 weights
        _case("norm_append_decode_fp8", "norm", reqs=64, p_lo=1, p_hi=16384, hq=64, kv="fp8", weights="fp32", lens=2),
        # a chunk of a layer without pages: adjacent pairs, half of the dims rotated, weights kept as their distance from one
        _case("norm_chunk", "norm", reqs=3, c_lo=389, c_hi=1024, hkv=32, kv="none", rot=64, layout="adjacent", offset=1.0, lens=7),
        # a full mixed step
        _case("norm_append_mixed", "norm", reqs=64, p_lo=0, p_hi=32768, c_lo=1, c_hi=2048, c_mode="lognormal", lens=4),
    ]


MAX_COST = {"quant": 3.2e8, "read": 4.5e8, "attn": 6.8e10, "norm": 8.6e8}   # about the largest listed cases


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["attn", "attn", "attn", "quant", "read", "norm", "norm"])
        kind = "decode" if op == "read" else rng.choice(["decode", "stream", "batch", "mixed"])
        kw = dict(lens=rng.randrange(1 << 20))
        kw["hq"], kw["hkv"] = rng.choice([(8, 2), (16, 4), (32, 8), (64, 8), (8, 1), (16, 16)])
        if op == "norm":
            kw.update(kv=rng.choice(["bf16", "bf16", "fp8", "none"]), rot=rng.choice([128, 128, 64, 96, 32, 16]),
                      layout=rng.choice(["halves", "halves", "adjacent"]), weights=rng.choice(["bf16", "fp32"]), offset=rng.choice([0.0, 1.0]))
        if kind == "decode":
            hi = _log_int(rng, 64, 131072 if op == "attn" else 32768)
            kw.update(reqs=_log_int(rng, 1, 96), p_lo=max(1, hi // 16), p_hi=hi, c_lo=1, c_hi=1 if op == "read" else rng.choice([1, 1, 4]))
        elif kind == "stream":
            p, c = rng.choice([0, _log_int(rng, 16, 65536)]), _log_int(rng, 2, 4096)
            kw.update(p_lo=p, p_hi=p, c_lo=c, c_hi=c)
        elif kind == "batch":
            kw.update(reqs=rng.randint(2, 16), p_lo=0, p_hi=_log_int(rng, 64, 32768), c_lo=_log_int(rng, 3, 512), c_hi=1024)
        else:
            kw.update(reqs=rng.randint(8, 48), p_lo=0, p_hi=_log_int(rng, 512, 32768), c_lo=1, c_hi=2048, c_mode="lognormal")
        case = _case("", op, **kw)
        del case["name"]
        w = work(case)
        if max(w["bytes"], w["flops"] / 50) <= MAX_COST[op]:
            return case


def lengths(case):
    """Cached and new tokens of the requests."""
    rng = random.Random(1000003 * case["lens"] + case["reqs"])
    P, C = [], []
    for _ in range(case["reqs"]):
        P.append(rng.randint(case["p_lo"], case["p_hi"]))
        if case["c_mode"] == "lognormal":
            C.append(min(case["c_hi"], max(case["c_lo"], int(rng.lognormvariate(math.log(64.0), 4.118)))))
        else:
            C.append(rng.randint(case["c_lo"], case["c_hi"]))
    return P, C


def work(case):
    P, C = lengths(case)
    T, hq, hkv, row = sum(C), case["hq"], case["hkv"], 2 * D
    held = RUN // PAGE                                     # bytes of a quantised row of a head
    if case["op"] == "quant":
        return {"bytes": 2 * T * hkv * (row + held + row), "flops": 2 * T * hkv * D * 2}
    if case["op"] == "read":
        return {"bytes": 2 * sum(P) * hkv * (held + row), "flops": 2 * sum(P) * hkv * D}
    if case["op"] == "attn":
        pairs = sum(c * p + c * (c + 1) // 2 for p, c in zip(P, C))
        return {"bytes": 2 * (sum(P) + T) * hkv * held + 2 * T * hq * row, "flops": 4 * pairs * hq * D}
    moved = 2 * T * row * (hq + hkv)
    if case["kv"] != "none":
        moved += T * hkv * (row + (0 if case["kv"] == "bf16" else -2 * D) + row)
    return {"bytes": moved, "flops": T * (hq + hkv) * (4 * D + 3 * case["rot"])}


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    P, C = lengths(case)
    op, T, R, hq, hkv = case["op"], sum(C), len(P), case["hq"], case["hkv"]
    s = dict(case=case, T=T, R=R)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)  # noqa: E731
    s["P"], s["C"], s["cu"] = ints(P), ints(C), ints([sum(C[:r]) for r in range(R + 1)])
    # channels of keys and values differ in size, as a model's do
    channels = lambda: torch.exp(0.5 * torch.randn((hkv, D), generator=gen, device=DEV))  # noqa: E731

    # pages in any order; where only the new tokens' pages are met, the ones before them are one shared page
    whole = op in ("attn", "read")
    first = [0 if whole else p // PAGE for p in P]
    last = [(p + (0 if op == "read" else c) + PAGE - 1) // PAGE for p, c in zip(P, C)]
    pages = 1 + sum(b - a for a, b in zip(first, last))
    order = 1 + torch.randperm(pages - 1, generator=torch.Generator().manual_seed(seed))
    tables = torch.zeros((R, max(max(last), max((p + c + PAGE - 1) // PAGE for p, c in zip(P, C)))), dtype=torch.int32)
    at = 0
    for r in range(R):
        n = last[r] - first[r]
        tables[r, first[r]:last[r]] = order[at:at + n].int()
        at += n
    s["tables"] = tables.to(DEV)

    if op == "norm":
        pairs = case["rot"] // 2
        qkv = normal(T, hq + 2 * hkv, D)                   # one projected row a token: queries, keys, values
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_out"] = torch.empty((T, hq, D), dtype=torch.bfloat16, device=DEV)
        s["inv_freq"] = (10000.0 ** -(torch.arange(pairs, dtype=torch.float64) / pairs)).float().to(DEV)
        s["eps"] = 1e-6
        weight = lambda: (1 - case["offset"] + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(  # noqa: E731
            torch.float32 if case["weights"] == "fp32" else torch.bfloat16)
        s["q_weight"], s["k_weight"] = weight(), weight()
        if case["kv"] == "none":
            s["k_out"] = torch.empty((T, hkv, D), dtype=torch.bfloat16, device=DEV)
        elif case["kv"] == "fp8":
            s["k_scale"], s["v_scale"] = (0.01 + 0.01 * torch.rand(hkv, generator=gen, device=DEV) for _ in range(2))
            s["k_pages"], s["v_pages"] = (torch.empty((pages, hkv, PAGE, D), device=DEV).normal_(0, 50, generator=gen).to(torch.float8_e4m3fn) for _ in range(2))
        else:
            s["k_pages"], s["v_pages"] = normal(pages, hkv, PAGE, D), normal(pages, hkv, PAGE, D)
    else:
        s["k_pages"], s["v_pages"] = (_held(normal(pages, hkv, PAGE, D).float() * channels()[:, None]) for _ in range(2))
    if op == "quant":
        s["k"], s["v"] = ((normal(T, hkv, D).float() * channels()).to(torch.bfloat16) for _ in range(2))
    if op in ("quant", "read"):
        n = [p if op == "read" else c for p, c in zip(P, C)]
        s["begin"], s["count"], s["rows"] = (s["P"] if op == "quant" else 0 * s["P"]), ints(n), sum(n)
        s["cu_out"] = ints([sum(n[:r]) for r in range(R + 1)])
        s["k_out"], s["v_out"] = (torch.empty((sum(n), hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if op == "attn":
        s["q"] = normal(T, hq, D)
        s["out"] = torch.empty((T, hq, D), dtype=torch.bfloat16, device=DEV)
        s["groups"] = _groups(P, C, hq)

    if own:   # the framework's objects for the same tensors
        import paper_2604_16395_amd as s2l
        s["batch"] = s2l.Batch(P, C, tables.numpy())
        if op == "norm":
            s["rope"] = s2l.Rope(s["inv_freq"], adjacent=case["layout"] == "adjacent")
            s["norm"] = s2l.QKNorm(s["q_weight"], s["k_weight"], s["eps"], case["offset"])
        if op != "norm" or case["kv"] == "bf16":
            s["cache"] = s2l.PagedKVCache(s["k_pages"], s["v_pages"])
        elif case["kv"] == "fp8":
            s["cache"] = s2l.PagedKVCache(s["k_pages"].view(torch.uint8), s["v_pages"].view(torch.uint8), s["k_scale"], s["v_scale"])
        if op == "attn":   # planned once for all layers of a step
            s["ws"] = torch.empty(s2l.s2l_attn_workspace_bytes(s["batch"], hq, hkv), dtype=torch.uint8, device=DEV)
            s["plan"] = s2l.s2l_attn_plan(s["batch"], hq, hkv, s["ws"])
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2604_16395_amd as s2l
        if op == "quant":
            s2l.s2l_kv_append(s["cache"], s["batch"], s["k"], s["v"])
            s2l.s2l_kv_read(s["cache"], s["batch"], s2l.S2L_READ_CHUNK, s["cu_out"], s["k_out"], s["v_out"])
        elif op == "read":
            s2l.s2l_kv_read(s["cache"], s["batch"], s2l.S2L_READ_PREFIX, s["cu_out"], s["k_out"], s["v_out"])
        elif op == "attn":
            s2l.s2l_chunk_prefill_attn(s["cache"], s["batch"], s["q"], s["case"]["hq"], SCALE, s["out"], None, s["plan"], s["ws"])
        elif s["case"]["kv"] == "none":
            s2l.s2l_norm_rope_qk(s["batch"], s["norm"], s["rope"], s["q"], s["q_out"], s["k"], s["k_out"])
        else:
            s2l.s2l_norm_rope_kv_append(s["cache"], s["batch"], s["norm"], s["rope"], s["q"], s["q_out"], s["k"], s["v"])
    else:
        {"quant": _plain_quant, "read": _plain_read, "attn": _plain_attn, "norm": _plain_norm}[op](s)
    if op == "attn":
        return {"out": s["out"]}
    if op == "norm" and s["case"]["kv"] != "none":
        return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return {"q": s["q_out"], "k": s["k_out"]} if op == "norm" else {"k": s["k_out"], "v": s["v_out"]}


# ---- the plain forms ----

def _quantised(x):
    """fp32 [..., 128]: the E2M1 code of each dim, and each block's scale byte."""
    x = x.unflatten(-1, (D // BLOCK, BLOCK))
    scale = (torch.frexp(x.abs().amax(-1))[1] - 3).clamp(-125, 125)
    y = torch.ldexp(x, -scale[..., None])
    a = y.abs()
    # ties go to the even code
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5).byte())
    return (code + 8 * torch.signbit(y).byte()).flatten(-2), (scale + 127).byte()


def _held(x):
    """Pages [pages][heads][16][128] in the form in which they are held: codes two a byte, then the scales."""
    code, scale = _quantised(x)
    return torch.cat([(code[..., 0::2] + 16 * code[..., 1::2]).flatten(-2), scale.flatten(-2)], -1)


def _values(held, scale):
    """fp32 values of codes two a byte [..., 64] and scales [..., 4]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    table = torch.cat([table, -table])
    code = torch.stack([held & 15, held >> 4], -1).flatten(-2)
    return torch.ldexp(table[code.int()].unflatten(-1, (D // BLOCK, BLOCK)), scale[..., None].int() - 127).flatten(-2)


def _rows(s, begin, count, total):
    """Each row's page and slot, for `count` tokens of each request from position `begin` on."""
    req = torch.repeat_interleave(torch.arange(s["R"], device=DEV), count, output_size=total)
    ends = count.cumsum(0)
    where = torch.arange(total, device=DEV) - (ends - count)[req] + begin[req]
    return s["tables"][req, where // PAGE].long(), where % PAGE, where


def _plain_read(s):
    page, slot, _ = _rows(s, s["begin"], s["count"], s["rows"])
    for name in ("k", "v"):
        pool = s[name + "_pages"]
        codes, scales = pool[..., :PAGE * D // 2].unflatten(-1, (PAGE, D // 2)), pool[..., PAGE * D // 2:].unflatten(-1, (PAGE, D // BLOCK))
        s[name + "_out"].copy_(_values(codes[page, :, slot], scales[page, :, slot]))


def _plain_quant(s):
    page, slot, _ = _rows(s, s["P"], s["C"], s["T"])
    for name in ("k", "v"):
        pool = s[name + "_pages"]
        code, scale = _quantised(s[name].float())
        pool[..., :PAGE * D // 2].unflatten(-1, (PAGE, D // 2))[page, :, slot] = code[..., 0::2] + 16 * code[..., 1::2]
        pool[..., PAGE * D // 2:].unflatten(-1, (PAGE, D // BLOCK))[page, :, slot] = scale
    _plain_read(s)


def _groups(P, C, hq):
    """Requests of one chunk length each, so many at once as their scores allow."""
    groups = []
    for r in sorted(range(len(P)), key=lambda r: (C[r], P[r])):
        g = groups[-1] if groups else None
        if g and C[g[0]] == C[r] and (len(g) + 1) * C[r] * hq * (P[r] + C[r]) <= MOST_SCORES:
            g.append(r)
        else:
            groups.append([r])
    return [(torch.tensor(g, device=DEV), C[g[0]], max(P[r] for r in g) + C[g[0]]) for g in groups]


def _plain_attn(s):
    hq, hkv = s["case"]["hq"], s["case"]["hkv"]
    for g, c, most in s["groups"]:
        n, table = g.numel(), s["tables"][g, :-(-most // PAGE)].long()

        def values(pool):
            held = pool[table]                                                         # [n][pages][hkv][1088]
            x = _values(held[..., :PAGE * D // 2].unflatten(-1, (PAGE, D // 2)), held[..., PAGE * D // 2:].unflatten(-1, (PAGE, D // BLOCK)))
            return x.transpose(1, 2).reshape(n, hkv, -1, D)

        rows = s["cu"][g][:, None] + torch.arange(c, device=DEV)                       # [n][c]
        q = s["q"][rows].float().view(n, c, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, D)
        scores = (SCALE * q) @ values(s["k_pages"]).transpose(-1, -2)
        seen = torch.arange(scores.shape[-1], device=DEV) <= (s["P"][g][:, None] + torch.arange(c, device=DEV))[..., None]   # [n][c][keys]
        scores = scores.view(n, hkv, hq // hkv, c, -1).masked_fill_(~seen[:, None, None], -math.inf)
        w = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
        out = (w.flatten(2, 3) @ values(s["v_pages"])).view(n, hkv, hq // hkv, c, D) / w.sum(-1, keepdim=True)
        s["out"][rows] = out.permute(0, 3, 1, 2, 4).reshape(n, c, hq, D).to(torch.bfloat16)


def _plain_norm(s):
    rot, adjacent = s["case"]["rot"], s["case"]["layout"] == "adjacent"
    page, slot, where = _rows(s, s["P"], s["C"], s["T"])
    angle = where.double()[:, None] * s["inv_freq"].double()                           # [T][pairs]
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)

    def turned(x, weight):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * (weight.float() + s["case"]["offset"])
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., :rot // 2], x[..., rot // 2:rot])
        y = [a * cos - b * sin, b * cos + a * sin]
        return torch.cat([torch.stack(y, -1).flatten(-2) if adjacent else torch.cat(y, -1), x[..., rot:]], -1).to(torch.bfloat16)

    s["q_out"].copy_(turned(s["q"], s["q_weight"]))
    k, v = turned(s["k"], s["k_weight"]), s["v"]
    if s["case"]["kv"] == "none":
        s["k_out"].copy_(k)
        return
    if s["case"]["kv"] == "fp8":
        k, v = ((x.float() * (1 / c).unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn) for x, c in ((k, s["k_scale"]), (v, s["v_scale"])))
    whole = torch.uint8 if s["case"]["kv"] == "fp8" else torch.bfloat16
    s["k_pages"].view(whole)[page, :, slot] = k.view(whole)
    s["v_pages"].view(whole)[page, :, slot] = v.view(whole)


# ---- the definitions in 64 bits ----

def _meaning(held):
    """The values of one head's rows of a page run [..., 1088], in 64 bits, from the bits of the codes."""
    byte = held[..., :PAGE * D // 2].long()
    code = torch.stack([byte % 16, byte // 16], -1).flatten(-2)
    sign, exponent, mantissa = 1 - 2 * (code // 8), code // 2 % 4, code % 2
    x = sign * torch.where(exponent == 0, mantissa / 2, (2 + mantissa) * 2.0 ** (exponent.double() - 2))
    power = 2.0 ** (held[..., PAGE * D // 2:].double() - 127)
    return x.unflatten(-1, (PAGE, D)) * power.unflatten(-1, (PAGE, D // BLOCK)).repeat_interleave(BLOCK, -1)


def _nearest(x):
    """Each value's nearest one in its block's grid, in 64 bits; of two equally near the one with the even code."""
    x = x.double().unflatten(-1, (D // BLOCK, BLOCK))
    unit = 2.0 ** (torch.floor(torch.log2(x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -123))).clamp(max=127) - 2)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    away = (x.abs()[..., None] / unit[..., None] - grid).abs() + 1e-6 * (torch.arange(8, device=DEV) % 2)
    return (torch.copysign(grid[away.argmin(-1)], x) * unit).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    P, C = lengths(case)
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    if op == "quant":
        return {n: torch.cat([_nearest(x) for x in s[n].split(4096)]) for n in ("k", "v")}
    if op == "read":
        cached = lambda pool, r: _meaning(pool[s["tables"][r, :-(-P[r] // PAGE)].long()]).transpose(1, 2).flatten(0, 1)[:P[r]]  # noqa: E731
        return {n: torch.cat([cached(s[n + "_pages"], r) for r in range(len(P))]) for n in ("k", "v")}
    if op == "attn":
        out, G = torch.empty((s["T"], hq, D), dtype=torch.float64, device=DEV), hq // hkv
        for r, (p, c) in enumerate(zip(P, C)):
            at, table = sum(C[:r]), s["tables"][r, :-(-(p + c) // PAGE)].long()
            hidden = torch.arange(p + c, device=DEV) > p + torch.arange(c, device=DEV)[:, None]
            for h in range(hkv):
                k, v = (_meaning(s[n][table, h]).flatten(0, 1)[:p + c] for n in ("k_pages", "v_pages"))
                q = s["q"][at:at + c, h * G:(h + 1) * G].double().transpose(0, 1)      # [G][c][128]
                scores = (q @ k.T / math.sqrt(D)).masked_fill(hidden, -math.inf)
                out[at:at + c, h * G:(h + 1) * G] = (torch.softmax(scores, -1) @ v).transpose(0, 1)
        return {"out": out}
    where = torch.cat([p + torch.arange(c, dtype=torch.float64) for p, c in zip(P, C)]).to(DEV)
    rot, half, adjacent = case["rot"], case["rot"] // 2, case["layout"] == "adjacent"

    def normed(x, weight):
        x = x.double()
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + s["eps"]) * (weight.double() + case["offset"])
        y = x.clone()
        for i in range(half):
            angle = where * float(s["inv_freq"][i])
            c, d = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
            y[:, :, a] = x[:, :, a] * c - x[:, :, b] * d
            y[:, :, b] = x[:, :, a] * d + x[:, :, b] * c
        return y

    q, k = normed(s["q"], s["q_weight"]), normed(s["k"], s["k_weight"])
    if case["kv"] == "none":
        return {"q": q, "k": k}
    pools = {"k_pages": k, "v_pages": s["v"].double()}
    for name, x in pools.items():
        pool = s[name].double()
        if case["kv"] == "fp8":
            x = (x / s[name[0] + "_scale"].double()[:, None]).clamp(-448, 448)
        at = 0
        for r in range(s["R"]):
            pos = P[r] + torch.arange(C[r], device=DEV)
            pool[s["tables"][r][pos // PAGE].long(), :, pos % PAGE] = x[at:at + C[r]]
            at += C[r]
        pools[name] = pool
    return {"q": q, **pools}
