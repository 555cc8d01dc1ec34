"""Rotary positions, the append that rotates on the way, and linear attention with a decay: the calls
over the range in which a serving program makes them, each also in a plain form of elementary torch
operations.

"append": a step's queries, keys and values come out of the projection, one row of Hq + 2 Hkv heads a
token.  Queries and keys are rotated by their positions, keys and values go into their pages.
"rope": queries and keys of a layer without pages (a linear attention layer) are rotated.
"linear": linear attention of a varlen batch over states that are kept in slots: state in, chunk
processed, state out.

`own` picks the framework's calls; otherwise the plain form runs, in 32 bits (angles in 64) whatever
the inputs' type, rounded at the end.  Keys for e4m3 pages are first rounded to bf16, as the separate
calls round them; such pages come back as float8 values, without their head's scale.
"""
import math
import random

import torch

own = False

DEV = "cuda"
D, PAGE = 128, 16
SCALE = D ** -0.5
BLOCK = 256          # tokens of a block in the plain form of linear attention


def _case(name, op, **kw):
    case = dict(op=op, reqs=1, p_lo=0, p_hi=0, c_lo=1, c_hi=1, c_mode="uniform", lens=1, hq=32, hkv=8)
    if op != "linear":
        case.update(rot=128, layout="halves", axes=1, cyclic=False)
    if op == "append":
        case["kv"] = "bf16"
    case.update(kw)
    return dict(name=name, **case)


def listed():
    return [
        # the smallest step of a decoding request: one row, so latency and nothing else
        _case("append_one", "append", p_lo=2047, p_hi=2047),
        # a decode batch at ragged contexts, 70B-like heads, e4m3 pages
        _case("append_decode_fp8", "append", reqs=64, p_lo=1, p_hi=16384, hq=64, kv="fp8", lens=2),
        # a streamed chunk on 8192 cached tokens
        _case("append_chunk", "append", p_lo=8192, p_hi=8192, c_lo=512, c_hi=512),
        # a full mixed step of text, images and video: three position axes in turn over the pairs,
        # chunks from one token to 2048
        _case("append_mixed_axes", "append", reqs=64, p_lo=0, p_hi=32768, c_lo=1, c_hi=2048, c_mode="lognormal", lens=4,
              axes=3, cyclic=True),
        # a linear layer's queries and keys for a decode batch, a quarter of the dims rotated
        _case("rope_decode", "rope", reqs=8, p_lo=1, p_hi=8192, hkv=32, rot=32, lens=3),
        # the same for a prompt of images: adjacent pairs, three axes in blocks, odd lengths
        _case("rope_prompt_axes", "rope", reqs=3, c_lo=1000, c_hi=3001, hkv=32, layout="adjacent", axes=3, lens=5),
        # one decoding request: its states are read, advanced by a token and written
        _case("linear_one", "linear", p_lo=500, p_hi=500, hkv=32),
        # a decode batch: 64 requests' states
        _case("linear_decode", "linear", reqs=64, p_lo=1, p_hi=8192, hkv=32, lens=6),
        # a streamed chunk that goes on from its request's state
        _case("linear_chunk", "linear", p_lo=8192, p_hi=8192, c_lo=512, c_hi=512, hkv=32),
        # several requests' chunks, ragged, four query heads to a key head
        _case("linear_batch8", "linear", reqs=8, p_lo=0, p_hi=8192, c_lo=389, c_hi=1024, lens=7),
        # a full mixed step: chunks from one token to 2048
        _case("linear_mixed", "linear", reqs=48, p_lo=0, p_hi=32768, c_lo=1, c_hi=2048, c_mode="lognormal", hkv=32, lens=4),
        # a long prompt at once
        _case("linear_prompt", "linear", c_lo=32768, c_hi=32768, hkv=32),
    ]


MAX_BYTES, MAX_TOKENS = 1.08e9, 32768   # about the largest listed case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "append", "rope", "linear", "linear"])
        kind = rng.choice(["decode", "stream", "batch", "mixed"])
        kw = dict(lens=rng.randrange(1 << 20))
        if op == "append":
            kw["hq"], kw["hkv"] = rng.choice([(8, 2), (16, 4), (32, 8), (64, 8), (8, 1)])
            kw["kv"] = rng.choice(["bf16", "bf16", "fp8"])
        else:
            kw["hq"], kw["hkv"] = rng.choice([(8, 8), (16, 16), (32, 32), (64, 64), (32, 8), (16, 2)])
        if op != "linear":
            kw.update(rot=rng.choice([128, 128, 64, 96, 32, 16]), layout=rng.choice(["halves", "halves", "adjacent"]),
                      axes=rng.choice([1, 1, 2, 3]), cyclic=rng.random() < 0.5)
        if kind == "decode":
            hi = _log_int(rng, 64, 32768)
            kw.update(reqs=_log_int(rng, 1, 96), p_lo=max(1, hi // 16), p_hi=hi, c_lo=1, c_hi=rng.choice([1, 1, 4]))
        elif kind == "stream":
            p, c = rng.choice([0, _log_int(rng, 16, 131072)]), _log_int(rng, 2, 16384)
            kw.update(p_lo=p, p_hi=p, c_lo=c, c_hi=c)
        elif kind == "batch":
            kw.update(reqs=rng.randint(2, 16), p_lo=0, p_hi=_log_int(rng, 64, 32768), c_lo=_log_int(rng, 3, 512), c_hi=1024)
        else:
            kw.update(reqs=rng.randint(8, 64), p_lo=0, p_hi=_log_int(rng, 512, 32768), c_lo=1, c_hi=2048, c_mode="lognormal")
        case = _case("", op, **kw)
        del case["name"]
        if work(case)["bytes"] <= MAX_BYTES and sum(lengths(case)[1]) <= MAX_TOKENS:
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
    if case["op"] == "linear":
        states = hq * D * D * 4 * (len(C) + sum(p > 0 for p in P))    # written; read where there is one
        return {"bytes": T * row * (2 * hq + 2 * hkv) + states, "flops": 4 * T * hq * D * D}
    rotated = {"bytes": 2 * T * row * (hq + hkv) + 4 * T * case["axes"], "flops": 3 * T * (hq + hkv) * case["rot"]}
    if case["op"] == "append":
        rotated["bytes"] += T * hkv * (row + (0 if case["kv"] == "bf16" else -2 * D) + row)
    return rotated


def _pair_axes(case):
    """The position axis of each rotated pair: a quarter of them the first axis, the others shared out."""
    pairs, n = case["rot"] // 2, case["axes"]
    rest = [] if n == 1 else [(pairs * 3 // 4) // (n - 1)] * (n - 1)
    if case["cyclic"]:
        return [i % n if i % n and i // n < rest[i % n - 1] else 0 for i in range(pairs)]
    return [0] * (pairs - sum(rest)) + [a + 1 for a, m in enumerate(rest) for _ in range(m)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    P, C = lengths(case)
    T, R, hq, hkv = sum(C), len(P), case["hq"], case["hkv"]
    s = dict(case=case, T=T, R=R)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)  # noqa: E731
    s["P"], s["C"], s["cu"] = ints(P), ints(C), ints([sum(C[:r]) for r in range(R + 1)])

    # one projected row a token: queries, keys, values side by side
    qkv = normal(T, hq + 2 * hkv, D)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    s["q_out"] = torch.empty((T, hq, D), dtype=torch.bfloat16, device=DEV)

    # append writes the pages of the new tokens; the cached tokens' pages before them are one shared page
    first = [p // PAGE for p in P]
    last = [(p + c - 1) // PAGE if c else f - 1 for p, c, f in zip(P, C, first)]
    pages = 1 + sum(b - a + 1 for a, b in zip(first, last))
    tables = torch.zeros((R, max(last) + 1), dtype=torch.int32)
    if case["op"] == "append":
        order = iter((1 + torch.randperm(pages - 1, generator=torch.Generator().manual_seed(seed))).tolist())
        for r in range(R):
            tables[r, first[r]:last[r] + 1] = torch.tensor([next(order) for _ in range(first[r], last[r] + 1)], dtype=torch.int32)
    s["tables"] = tables.to(DEV)

    if case["op"] != "linear":
        pairs, axes = case["rot"] // 2, _pair_axes(case)
        s["inv_freq"] = (10000.0 ** -(torch.arange(pairs, dtype=torch.float64) / pairs)).float().to(DEV)
        s["pair_axes"] = torch.tensor(axes, device=DEV)
        s["positions"] = None
        if case["axes"] > 1:   # images and frames of 24 x 32 patches, from a first position on
            i = torch.arange(T, dtype=torch.int32, device=DEV) + torch.randint(0, 4096, (1,), generator=gen, device=DEV, dtype=torch.int32)
            s["positions"] = torch.stack([i // 768, i // 32 % 24 + i // 768, i % 32 + i // 768][:case["axes"]]).contiguous()
    if case["op"] == "append":
        shape = (pages, hkv, PAGE, D)
        if case["kv"] == "fp8":
            s["k_scale"], s["v_scale"] = (0.01 + 0.01 * torch.rand(hkv, generator=gen, device=DEV) for _ in range(2))
            s["k_pages"], s["v_pages"] = (torch.empty(shape, device=DEV).normal_(0, 50, generator=gen).to(torch.float8_e4m3fn) for _ in range(2))
        else:
            s["k_pages"], s["v_pages"] = normal(*shape), normal(*shape)
    if case["op"] == "rope":
        s["k_out"] = torch.empty((T, hkv, D), dtype=torch.bfloat16, device=DEV)
    if case["op"] == "linear":
        # slot r holds request r's state, slot R + r gets the state after the chunk
        s["states"] = torch.empty((2 * R, hq, D, D), device=DEV).normal_(0, 4, generator=gen)
        s["slot_in"] = ints([r if P[r] else -1 for r in range(R)])
        s["slot_out"] = ints(list(range(R, 2 * R)))
        s["log_decay"] = -(2.0 ** (-8.0 * (torch.arange(hq, dtype=torch.float64) + 1) / hq)).float().to(DEV)

    if own:   # the framework's objects for the same tensors
        import paper_2604_16395_amd as s2l
        s["batch"] = s2l.Batch(P, C, tables.numpy())
        if case["op"] == "linear":
            s["state"] = s2l.LinearState(s["states"], s["log_decay"], s["slot_in"], s["slot_out"])
            s["ws"] = torch.empty(s2l.s2l_linear_attn_workspace_bytes(s["batch"], hq), dtype=torch.uint8, device=DEV)
        else:
            s["rope"] = s2l.Rope(s["inv_freq"], positions=s["positions"], pair_axes=axes, adjacent=case["layout"] == "adjacent")
        if case["op"] == "append":
            fp8 = case["kv"] == "fp8"
            pools = [s[n].view(torch.uint8) if fp8 else s[n] for n in ("k_pages", "v_pages")]
            s["cache"] = s2l.PagedKVCache(*pools, *([s["k_scale"], s["v_scale"]] if fp8 else []))
    return s


def run(s):
    if own:
        import paper_2604_16395_amd as s2l
        if s["case"]["op"] == "append":
            s2l.s2l_rope_kv_append(s["cache"], s["batch"], s["rope"], s["q"], s["q_out"], s["k"], s["v"])
            return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
        if s["case"]["op"] == "rope":
            s2l.s2l_rope_qk(s["batch"], s["rope"], s["q"], s["q_out"], s["k"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        s2l.s2l_linear_attn(s["state"], s["batch"], s["q"], s["k"], s["v"], SCALE, s["q_out"], s["ws"])
        return {"out": s["q_out"], "states": s["states"]}
    return {"append": _plain_append, "rope": _plain_rope, "linear": _plain_linear}[s["case"]["op"]](s)


# ---- the plain forms ----

def _rows(s):
    """Each row's request, and its position in that request's sequence."""
    req = torch.repeat_interleave(torch.arange(s["R"], device=DEV), s["C"], output_size=s["T"])
    return req, torch.arange(s["T"], device=DEV) - s["cu"][req] + s["P"][req]


def _cos_sin(s, where):
    pos = where.expand(s["case"]["axes"], -1) if s["positions"] is None else s["positions"]
    angle = pos.double()[s["pair_axes"]].t() * s["inv_freq"].double()          # [T][pairs]
    return angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)


def _rotate(s, x, cos, sin):
    rot, x = s["case"]["rot"], x.float()
    if s["case"]["layout"] == "adjacent":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1).to(torch.bfloat16)


def _plain_append(s):
    req, where = _rows(s)
    cos, sin = _cos_sin(s, where)
    s["q_out"].copy_(_rotate(s, s["q"], cos, sin))
    k, v = _rotate(s, s["k"], cos, sin), s["v"]
    if s["case"]["kv"] == "fp8":
        k, v = ((x.float() * (1 / c).unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn) for x, c in ((k, s["k_scale"]), (v, s["v_scale"])))
    page, slot = s["tables"][req, where // PAGE].long(), where % PAGE
    whole = torch.uint8 if s["case"]["kv"] == "fp8" else torch.bfloat16
    s["k_pages"].view(whole)[page, :, slot] = k.view(whole)
    s["v_pages"].view(whole)[page, :, slot] = v.view(whole)
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_rope(s):
    cos, sin = _cos_sin(s, _rows(s)[1])
    s["q_out"].copy_(_rotate(s, s["q"], cos, sin))
    s["k_out"].copy_(_rotate(s, s["k"], cos, sin))
    return {"q": s["q_out"], "k": s["k_out"]}


def _plain_linear(s):
    """Blocks of the padded batch: each block's own product under the decay, the states at the blocks'
    starts as one product with the powers of the decay between blocks."""
    R, T, hq, C, cu = s["R"], s["T"], s["case"]["hq"], s["C"].long(), s["cu"].long()
    longest = max(lengths(s["case"])[1])
    B = min(BLOCK, longest)
    n = -(-longest // B)
    i = torch.arange(n * B, device=DEV)
    valid = i < C[:, None]                                                     # [R][n B]
    row = (cu[:-1, None] + i).clamp(max=T - 1)
    blocks = lambda x: (x[row].float() * valid[..., None, None]).view(R, n, B, x.shape[1], D).transpose(2, 3)  # noqa: E731
    shared = lambda x: x.repeat_interleave(hq // x.shape[2], 2)  # noqa: E731
    q, k, v = blocks(s["q"]), shared(blocks(s["k"])), shared(blocks(s["v"]))   # [R][n][H][B][D]

    g = s["log_decay"].double()
    t = torch.arange(B, device=DEV)
    gap = (t[:, None] - t).double()
    within = torch.where(gap >= 0, torch.exp(gap.clamp(min=0) * g[:, None, None]), 0.0).float()       # [H][B][B]
    out = ((q @ k.transpose(-1, -2)) * within) @ v

    # tokens from each row to the end of its block's valid part, and of each block
    size = (C[:, None] - B * torch.arange(n, device=DEV)).clamp(0, B)          # [R][n]
    ahead = (size[..., None] - 1 - t).clamp(min=0).double()
    fade = torch.exp(ahead[:, :, None] * g[:, None]).float()                   # [R][n][H][B]
    own_part = (k * fade[..., None]).transpose(-1, -2) @ v                     # [R][n][H][D][D]
    begin = torch.where((s["slot_in"] >= 0)[:, None, None, None], s["states"][s["slot_in"].clamp(min=0).long()], 0.0)
    parts = torch.cat([begin[:, None], own_part], 1)                           # [R][n + 1][H][D][D]
    ends = torch.cat([torch.zeros((R, 1), device=DEV, dtype=torch.long), size.cumsum(1)], 1)          # tokens up to here
    dist = (ends[:, None, :, None] - ends[:, None, None]).clamp(min=0).double()                       # [R][1][n + 1][n + 1]
    carry = torch.exp(dist * g[:, None, None]).tril().float()                  # [R][H][n + 1][n + 1]
    states = (carry @ parts.transpose(1, 2).reshape(R, hq, n + 1, D * D)).view(R, hq, n + 1, D, D)

    since = torch.exp((t + 1).double() * g[:, None]).float()                   # [H][B]
    out = SCALE * (out + (q @ states[:, :, :-1].transpose(1, 2)) * since[..., None])
    s["q_out"].copy_(out.transpose(2, 3).reshape(R, n * B, hq, D)[valid].to(torch.bfloat16))
    s["states"][s["slot_out"].long()] = states[:, :, -1]
    return {"out": s["q_out"], "states": s["states"]}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    P, C = lengths(case)

    def recurrence():
        """Token after token: the state fades, takes in the outer product, and is read."""
        hq, hkv = s["case"]["hq"], s["case"]["hkv"]
        head = torch.arange(hq, device=DEV) * hkv // hq
        decay = torch.exp(s["log_decay"].double())[:, None, None]
        order = sorted(range(s["R"]), key=lambda r: -C[r])                          # longest first: the live ones lead
        S = torch.stack([s["states"][r].double() if P[r] else torch.zeros((hq, D, D), dtype=torch.float64, device=DEV) for r in order])
        begin = s["cu"][:-1].long()[torch.tensor(order, device=DEV)]
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        out = torch.zeros((s["T"], hq, D), dtype=torch.float64, device=DEV)
        live = s["R"]
        for i in range(max(C)):
            while C[order[live - 1]] <= i:
                live -= 1
            rows = begin[:live] + i
            S[:live].mul_(decay).addcmul_(k[rows][:, head].unsqueeze(-1), v[rows][:, head].unsqueeze(-2))
            out[rows] = SCALE * (q[rows].unsqueeze(-2) @ S[:live]).squeeze(-2)
        states = s["states"].double()
        states[s["R"] + torch.tensor(order, device=DEV)] = S
        return {"out": out, "states": states}

    if case["op"] == "linear":
        return recurrence()
    where = torch.cat([p + torch.arange(c, dtype=torch.float64) for p, c in zip(P, C)]).to(DEV)
    rot, half, adjacent = case["rot"], case["rot"] // 2, case["layout"] == "adjacent"

    def turn(x):
        x = x.double()
        y = x.clone()
        for i, axis in enumerate(_pair_axes(case)):
            angle = (where if s["positions"] is None else s["positions"][axis].double()) * float(s["inv_freq"][i])
            c, d = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
            y[:, :, a] = x[:, :, a] * c - x[:, :, b] * d
            y[:, :, b] = x[:, :, a] * d + x[:, :, b] * c
        return y

    if case["op"] == "rope":
        return {"q": turn(s["q"]), "k": turn(s["k"])}
    pools = {"k_pages": turn(s["k"]), "v_pages": s["v"].double()}
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
    return {"q": turn(s["q"]), **pools}
