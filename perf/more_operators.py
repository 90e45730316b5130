"""The operators of attention over paged caches and of normed queries and keys, as cases that can be timed and compared.

    norm       the RMS norm of every head of queries and keys and the rotation behind it, in one pass, and the gradient of both
    cache      keys and values of new tokens written into pages, in 16 bits or in e4m3 with a power of two per row of a head, and read back
    attn       attention of new tokens, one or a chunk of a sequence, over the sequence's pages: every earlier key, or a window of
               them and the first ones

listed() names the cases, draw() gives further ones of the same ranges, prepare() makes what the caller has in hand,
run() is one pass (`own`: through the package's entry points, else in plain torch operations in 32 bits), work() the
bytes and operations that a pass cannot do without, exact() the same results in 64 bits.
"""
import math

import torch

own = False   # whether run() calls the package
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
F32, F64, I32, I64, U8 = torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8
LIMIT = {torch.bfloat16: 1.875 * 2.0 ** 127, torch.float16: 1.875 * 2.0 ** 15}   # the most that a row in e4m3 stands for
EPS = 1e-6


# ---- the cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # queries and keys of one new token of eight sequences, in the projection's rows: latency
        dict(name="norm_tokens", kind="norm", dtype="fp16", N=8, Hq=32, Hk=8, E=128, axes="64 0 0", halves=True, grad=False, packed=8),
        # queries and keys of an image model (text and a grid)
        dict(name="norm_image", kind="norm", dtype="bf16", N=4608, Hq=24, Hk=24, E=128, axes="8 28 28", halves=False, grad=False, packed=24),
        # of a clip, to heads of rows, as the column-sparse kernels take them
        dict(name="norm_clip", kind="norm", dtype="bf16", N=18000, Hq=40, Hk=40, E=128, axes="22 21 21", halves=False, grad=False, packed=0),
        # the gradient for one ragged prompt of a text model
        dict(name="norm_text_gradient", kind="norm", dtype="fp16", N=333, Hq=32, Hk=8, E=128, axes="64 0 0", halves=True, grad=True, packed=8),
        # the gradient for a clip
        dict(name="norm_clip_gradient", kind="norm", dtype="bf16", N=18000, Hq=40, Hk=40, E=128, axes="22 21 21", halves=False, grad=True, packed=0),
        # one new token of sixteen sequences to its place, and back: latency
        dict(name="cache_tokens", kind="cache", dtype="bf16", format="e4m3", T=16, held=30000, H=8, E=128, page=64, write=True, packed=32),
        # a batch of prompts into pages and back
        dict(name="cache_prompts", kind="cache", dtype="fp16", format="e4m3", T=16383, held=40000, H=8, E=128, page=16, write=True, packed=32),
        # a long sequence's keys and values out of its pages, as attention over whole tensors takes them
        dict(name="cache_read_back", kind="cache", dtype="bf16", format="e4m3", T=75600, held=80000, H=24, E=128, page=128, write=False, packed=0),
        # one new token of sixteen sequences over pages in 8 bits
        dict(name="paged_tokens", kind="attn", dtype="bf16", format="e4m3", q="1" + 15 * " 1",
             k="32011 30000 27999 25001 21017 17000 15999 12345 9000 8191 5000 4097 2048 777 65 1", Hq=32, Hk=8, E=128, page=64, window=0, sinks=0),
        # new tokens that see a window and the first four
        dict(name="paged_tokens_window", kind="attn", dtype="fp16", format="fp16", q="1 2 1 1 5 1 1 1", k="20001 17000 9999 8192 4500 4100 3000 129", Hq=40, Hk=8, E=128,
             page=16, window=4096, sinks=4),
        # chunks of prompts behind what the pages hold already
        dict(name="paged_chunks", kind="attn", dtype="bf16", format="bf16", q="1024 700 512 33", k="16384 9001 3000 1000", Hq=32, Hk=8, E=128, page=128, window=0, sinks=0),
        # chunks over pages in 8 bits, narrow heads, a window and sixteen first tokens
        dict(name="paged_chunks_window", kind="attn", dtype="bf16", format="e4m3", q="2048 1500 999", k="30000 12001 999", Hq=24, Hk=8, E=64, page=32, window=1024, sinks=16),
    ]


def _text(values):
    return " ".join(map(str, values))


def _list(text):
    return [int(n) for n in text.split()]


def _log_int(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / multiple)) * multiple))


_LARGEST_BYTES, _LARGEST_SCORES = 1.1e9, 3e9   # of a drawn case: no more than of the largest listed ones


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "cache", "attn", "attn", "attn"])
        case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16"]))
        if kind == "norm":
            E = rng.choice([64, 96, 128, 128, 256])
            P = rng.choice([E // 2, E // 2, E // 2, E // 4])   # or a part of the head
            whole = rng.random() < 0.3   # one axis
            t = P if whole else 8 * rng.randint(0, P // 16)
            h = 0 if whole else (P - t) // 2
            Hk = rng.choice([1, 2, 4, 8, 8, 24, 40])
            case.update(N=_log_int(rng, 1, 18000), Hq=Hk * rng.choice([1, 1, 4, 5]), Hk=Hk, E=E, axes=_text([t, h, P - t - h]), halves=rng.random() < 0.4,
                        grad=rng.random() < 0.5, packed=rng.choice([0, 0, rng.randint(1, 40)]))
        elif kind == "cache":
            T = _log_int(rng, 1, 75600)
            case.update(format=rng.choice(["e4m3", "e4m3", case["dtype"]]), T=T, held=T + _log_int(rng, 1, 40000), H=rng.choice([1, 2, 8, 8, 24]), E=rng.choice([64, 128, 128]),
                        page=rng.choice([16, 32, 64, 128, 256]), write=rng.random() < 0.6, packed=rng.choice([0, rng.randint(1, 40)]))
        else:
            tokens = rng.random() < 0.5   # a few queries a sequence
            S = _log_int(rng, 1, 64) if tokens else _log_int(rng, 1, 8)
            longest = _log_int(rng, 16, 32768)
            k = [longest] + [rng.randint(0, longest) for _ in range(S - 1)]
            few = rng.choice([1, 1, 1, 2, 5]) if tokens else _log_int(rng, 8, 4096)
            q = [min(n, few if tokens else rng.randint(1, few)) for n in k]
            Hk = rng.choice([1, 2, 4, 8, 8, 12])
            some = rng.random() < 0.5
            case.update(format=rng.choice(["e4m3", case["dtype"]]), q=_text(q), k=_text(k), Hq=Hk * rng.choice([1, 2, 4, 5]), Hk=Hk, E=rng.choice([64, 128, 128]),
                        page=rng.choice([16, 32, 64, 128, 256]), window=_log_int(rng, 1, longest) if some else 0, sinks=rng.choice([0, 4, 64]) if some else 0)
            if S * case["Hq"] * max(q) * longest > _LARGEST_SCORES:
                continue
        if work(case)["bytes"] <= _LARGEST_BYTES:
            return case


# ---- what the caller has in hand ---------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 16 + 7)
    return g


def _randn(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=F32) * scale).to(dtype)


def _ints(values, dtype=I32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def prepare(case, seed):
    return {"norm": _prepare_norm, "cache": _prepare_cache, "attn": _prepare_attn}[case["kind"]](case, seed)


def _prepare_norm(case, seed):
    """Rows of heads.  `packed`: queries and keys lie in front of the values' `packed` heads in the projection's result; else the
    result goes to heads of rows."""
    g, t = _gen(seed), DTYPES[case["dtype"]]
    N, H, E, axes = case["N"], case["Hq"] + case["Hk"], case["E"], _list(case["axes"])
    x = _randn((N, H + case["packed"], E), t, g, 1.5)
    if axes[1]:   # a grid of patches behind the text's tokens, which all stand at the grid's origin
        side = max(1, int((N / 4) ** 0.5))
        at = (torch.arange(N, device=DEV) - N // 9).clamp(min=0)
        pos = torch.stack([at // (side * side), at // side % side, at % side], 1)
    else:         # single tokens somewhere in long texts
        pos = torch.randint(0, 100000, (N, 1), generator=g, device=DEV).expand(N, 3)
    freqs = torch.cat([10000.0 ** (-torch.arange(n, dtype=F64, device=DEV) / max(n, 1)) for n in axes])
    result = lambda: torch.empty((N, H, E), dtype=t, device=DEV) if case["packed"] else torch.empty((H, N, E), dtype=t, device=DEV).transpose(0, 1)   # noqa: E731
    weights = (torch.randn((2, E), generator=g, device=DEV) * 0.2 + 1).to(t)
    grad = result().copy_(_randn((N, H, E), t, g)) if case["grad"] else None
    return dict(case=case, axes=axes, x=x[:, :H], pos=pos.to(I32).contiguous(), freqs=freqs, out=result(), w=weights, grad=grad, dw=torch.empty((2, E), dtype=F32, device=DEV))


def _power(k):
    """2^k, k from -126 to 127, exactly (a library's powers need not be)."""
    return ((k + 127) << 23).view(F32)


def _e4m3(x):
    """Rows of e4m3 and the exponents of their powers of two, as bytes: x is about code * 2^(byte - 127)."""
    most = x.abs().amax(-1, keepdim=True).float()
    fraction, exponent = torch.frexp(most)                                   # 0.5 <= fraction < 1
    k = (exponent - 9 + (fraction > 0.875).int()).clamp(-126, 127)
    k = torch.where(most > 0, k, 0)
    return (x.float() * _power(-k)).to(torch.float8_e4m3fn), (k + 127).to(U8)[..., 0]


def _pages(case, count, g):
    """Caches of so many pages with earlier tokens' keys and values in every place."""
    t, H, E, page = DTYPES[case["dtype"]], case.get("H") or case["Hk"], case["E"], case["page"]
    k, v = _randn((count, page, H, E), t, g), _randn((count, page, H, E), t, g)
    if case["format"] != "e4m3":
        return dict(k=k, v=v, k_scales=None, v_scales=None)
    (k, k_scales), (v, v_scales) = _e4m3(k), _e4m3(v)
    # a page's exponents of one head lie side by side
    rows = lambda s: s.transpose(1, 2).contiguous().transpose(1, 2)   # noqa: E731
    return dict(k=k, v=v, k_scales=rows(k_scales), v_scales=rows(v_scales))


def _prepare_cache(case, seed):
    """New tokens' keys and values as the projection leaves them behind `packed` heads of queries, and their places in the pages: in
    runs of a page, the pages anywhere."""
    g, t = _gen(seed), DTYPES[case["dtype"]]
    T, H, E, page = case["T"], case["H"], case["E"], case["page"]
    count = -(-case["held"] // page)
    order = torch.randperm(count, generator=g, device=DEV)
    at = torch.arange(T, device=DEV) if T > 64 else torch.randperm(case["held"], generator=g, device=DEV)[:T]
    rows = (order[at // page] * page + at % page).to(I64)
    qkv = _randn((T, case["packed"] + 2 * H, E), t, g) if case["write"] else None
    return dict(case=case, pages=_pages(case, count, g), rows=rows, new=qkv, k=torch.empty((T, H, E), dtype=t, device=DEV), v=torch.empty((T, H, E), dtype=t, device=DEV))


def _prepare_attn(case, seed):
    """Queries one sequence behind the other, and the sequences' pages, anywhere among all; where a sequence has no page the table
    names none."""
    g, t = _gen(seed), DTYPES[case["dtype"]]
    nq, nk, page = _list(case["q"]), _list(case["k"]), case["page"]
    S, Hq, E = len(nq), case["Hq"], case["E"]
    need = [-(-n // page) for n in nk]
    order, table, used = torch.randperm(sum(need) + 3, generator=g, device=DEV).to(I32), torch.full((S, max(need)), -1, dtype=I32, device=DEV), 0
    for s, n in enumerate(need):
        table[s, :n] = order[used:used + n]
        used += n
    at_q = [sum(nq[:s]) for s in range(S + 1)]
    owner = torch.repeat_interleave(torch.arange(S, device=DEV), torch.tensor(nq, device=DEV))
    return dict(case=case, longest=(max(nq), max(nk)), scale=1 / math.sqrt(E), q=_randn((at_q[-1], Hq, E), t, g), pages=_pages(case, used + 3, g), table=table, cu_q=_ints(at_q),
                k_len=_ints(nk), q_len=_ints(nq), owner=owner, row=torch.arange(at_q[-1], device=DEV) - _ints(at_q)[owner], out=torch.empty((at_q[-1], Hq, E), dtype=t, device=DEV))


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    return {"norm": _norm, "cache": _cache, "attn": _attn}[state["case"]["kind"]](state)


def _handle(s):
    """The pages as a program holds them, made once."""
    import paper_2506_03275_amd as cm
    if "handle" not in s:
        s["handle"] = cm.Pages(s["pages"]["k"], s["pages"]["v"], s["pages"]["k_scales"], s["pages"]["v_scales"])
    return s["handle"]


def _turned(s, x, sign):
    """The pairs of x [N, H, E], 32 bits, turned; angles in 64 bits."""
    case, pairs = s["case"], sum(s["axes"])
    axis = torch.tensor([0] * s["axes"][0] + [1] * s["axes"][1] + [2] * s["axes"][2], device=DEV)
    angle = s["pos"].double()[:, axis] * s["freqs"]                        # [N, pairs]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None] * sign
    a, b = (x[..., :pairs], x[..., pairs:2 * pairs]) if case["halves"] else (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2])
    turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -2 if case["halves"] else -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * pairs:]], -1)


def _norm(s):
    case, x, w = s["case"], s["x"], s["w"]
    Hq, Hk = case["Hq"], case["Hk"]
    if own:
        import paper_2506_03275_amd as cm
        if not case["grad"]:
            cm.norm_rope(x, w[0], w[1], Hq, s["pos"], s["freqs"], s["out"], s["axes"], EPS, halves=case["halves"])
            return s["out"]
        if "ws" not in s:   # made once, as a program keeps it
            s["ws"] = torch.empty(max(16, cm.norm_rope_grad_workspace_bytes(case["N"], Hq + Hk, case["E"])), dtype=U8, device=DEV)
        cm.norm_rope_grad(s["grad"], x, w[0], w[1], Hq, s["pos"], s["freqs"], s["out"], s["dw"][0], s["dw"][1], s["axes"], EPS, halves=case["halves"], ws=s["ws"])
        return dict(dx=s["out"], dw=s["dw"])
    f = x.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    per_head = torch.cat([w[:1].expand(Hq, -1), w[1:].expand(Hk, -1)]).float()
    if not case["grad"]:
        s["out"].copy_(_turned(s, f * r * per_head, 1.0))
        return s["out"]
    g, n = _turned(s, s["grad"].float(), -1.0), f * r
    gn = g * n
    s["out"].copy_(r * (g * per_head - n * (gn * per_head).mean(-1, keepdim=True)))
    by_head = gn.sum(0, dtype=F64)
    s["dw"].copy_(torch.stack([by_head[:Hq].sum(0), by_head[Hq:].sum(0)]))
    return dict(dx=s["out"], dw=s["dw"])


def _cache(s):
    case, p, H = s["case"], s["pages"], s["case"]["H"]
    new = None if s["new"] is None else (s["new"][:, case["packed"]:case["packed"] + H], s["new"][:, case["packed"] + H:])
    if own:
        import paper_2506_03275_amd as cm
        if new:
            cm.cache_write(new[0], new[1], s["rows"], _handle(s))
        cm.cache_read(_handle(s), s["rows"], s["k"], s["v"])
        return dict(k=s["k"], v=s["v"])
    page, place = s["rows"] // case["page"], s["rows"] % case["page"]
    if new and case["format"] != "e4m3":
        p["k"][page, place], p["v"][page, place] = new
    elif new:
        both = torch.stack(new).float().clamp(-LIMIT[new[0].dtype], LIMIT[new[0].dtype])
        codes, scales = _e4m3(both)
        p["k"].view(U8)[page, place], p["v"].view(U8)[page, place] = codes.view(U8)
        p["k_scales"][page, place], p["v_scales"][page, place] = scales
    s["k"].copy_(_values(p["k"], p["k_scales"], page, place))
    s["v"].copy_(_values(p["v"], p["v_scales"], page, place))
    return dict(k=s["k"], v=s["v"])


def _values(held, scales, page, place):
    """Rows of the pages in 32 bits."""
    if scales is None:
        return held[page, place].float()
    codes = held.view(U8)[page, place].view(torch.float8_e4m3fn).float()
    return codes * _power(scales[page, place].int()[..., None] - 127)


def _attn(s):
    case, p, table = s["case"], s["pages"], s["table"]
    nq, nk = s["longest"]
    S, Hq, Hk, E, page = table.shape[0], case["Hq"], case["Hk"], case["E"], case["page"]
    if own:
        import paper_2506_03275_amd as cm
        if "ws" not in s:   # made once, as a program keeps it
            s["ws"] = torch.empty(max(16, cm.attn_paged_workspace_bytes(S, Hq, Hk, E, nq, nk, case["window"], case["sinks"])), dtype=U8, device=DEV)
        cm.attn_paged(s["q"], _handle(s), table, s["cu_q"], s["k_len"], s["out"], nq, nk, True, s["scale"], case["window"], case["sinks"], ws=s["ws"])
        return s["out"]
    i, j = torch.arange(nq, device=DEV), torch.arange(nk, device=DEV)
    at_q = (s["cu_q"][:S, None] + i).clamp(max=s["q"].shape[0] - 1)         # padded to the longest sequence
    at_k = table[:, j // page].clamp(min=0).long()
    q = s["q"][at_q].view(S, nq, Hk, Hq // Hk, E).permute(0, 2, 3, 1, 4).float().reshape(S, Hk, -1, E)
    k, v = (_values(p[n], p[n + "_scales"], at_k, (j % page).expand(S, -1)).permute(0, 2, 1, 3) for n in "kv")
    place = i + (s["k_len"] - s["q_len"])[:, None]                           # [S, nq], of each query among the keys
    hidden = j > place[..., None]                                            # [S, nq, nk]
    if case["window"]:
        hidden |= (j <= place[..., None] - case["window"]) & (j >= case["sinks"])
    v = v.masked_fill((j >= s["k_len"][:, None])[:, None, :, None], 0)
    w = (q @ k.transpose(2, 3)).view(S, Hk, Hq // Hk, nq, nk)
    w *= s["scale"]
    w.masked_fill_(hidden[:, None, None], -math.inf)
    w -= w.amax(-1, keepdim=True).clamp(min=-1e30)
    w.exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.view(S, Hk, -1, nk) @ v).view(S, Hk, Hq // Hk, nq, E) / total.clamp(min=1e-30)
    s["out"].copy_(o[s["owner"], :, :, s["row"]].reshape(-1, Hq, E))
    return s["out"]


# ---- bytes and operations ------------------------------------------------------------------------------------------------

def _seen(case):
    """Of each sequence: its keys that some query sees, and its pairs of a query and a key that it sees."""
    for a, b in zip(_list(case["q"]), _list(case["k"])):
        w, first = case["window"] or b + 1, min(case["sinks"], b)
        pairs = 0
        for place in range(b - a, b):
            low = max(0, place + 1 - w)
            pairs += place + 1 - low + min(first, low)
        low = max(0, b - a + 1 - w)
        yield a, b - low + min(first, low) if a else 0, pairs


def work(case):
    E = case["E"]
    if case["kind"] == "norm":
        rows, pairs = case["N"] * (case["Hq"] + case["Hk"]), sum(_list(case["axes"]))
        small = 12 * case["N"] + 8 * pairs + 4 * E
        if case["grad"]:
            return dict(bytes=6 * rows * E + small + 8 * E, flops=rows * (13 * E + 6 * pairs))
        return dict(bytes=4 * rows * E + small, flops=rows * (4 * E + 6 * pairs))
    held = E + 1 if case["format"] == "e4m3" else 2 * E   # bytes of a row of a head in the pages
    if case["kind"] == "cache":
        rows = 2 * case["T"] * case["H"]
        return dict(bytes=rows * (2 * E + held) * (2 if case["write"] else 1) + 8 * case["T"], flops=rows * E)
    queries, keys, pairs = (sum(n) for n in zip(*_seen(case)))
    return dict(bytes=4 * E * case["Hq"] * queries + 2 * held * case["Hk"] * keys, flops=4 * E * case["Hq"] * pairs)


# ---- in 64 bits ----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    return {"norm": _exact_norm, "cache": _exact_cache, "attn": _exact_attn}[case["kind"]](prepare(case, seed))


def _exact_norm(s):
    """A pair as a complex number; a few heads at a time."""
    case, P = s["case"], sum(s["axes"])
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(s["axes"], device=DEV))
    angle = s["pos"].double().index_select(1, axis) * s["freqs"]
    turn = torch.polar(torch.ones_like(angle), angle)
    first, second = (slice(0, P), slice(P, 2 * P)) if case["halves"] else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))

    def turned(y, by):
        z = torch.complex(y[:, first].contiguous(), y[:, second].contiguous()) * by
        y = y.clone()
        y[:, first], y[:, second] = z.real, z.imag
        return y
    out, dw = torch.empty(s["x"].shape, dtype=F64, device=DEV), torch.zeros(s["dw"].shape, dtype=F64, device=DEV)
    for h in range(case["Hq"] + case["Hk"]):
        x, which = s["x"][:, h].double(), int(h >= case["Hq"])
        w, length = s["w"][which].double(), torch.sqrt((x * x).sum(1, keepdim=True) / case["E"] + EPS)
        unit = x / length
        if not case["grad"]:
            out[:, h] = turned(unit * w, turn)
            continue
        g = turned(s["grad"][:, h].double(), turn.conj())
        dw[which] += (g * unit).sum(0)
        g = g * w
        out[:, h] = (g - unit * (g * unit).mean(1, keepdim=True)) / length
    return dict(dx=out, dw=dw) if case["grad"] else out


def _nearest_e4m3(x):
    """What rows of values become in e4m3 under their power of two, by arithmetic: 4 significant bits, steps of 2^-9 at least."""
    most = x.abs().amax(-1, keepdim=True)
    k = torch.floor(torch.log2(most.clamp(min=2.0 ** -150))) - 8
    k = torch.where(most * torch.exp2(-k) > 448, k + 1, k).clamp(min=-126)
    y = x * torch.exp2(-k)
    step = torch.exp2((torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))) - 3).clamp(min=-9))
    return torch.round(y / step) * step * torch.exp2(k)


def _exact_cache(s):
    case, p, H, got = s["case"], s["pages"], s["case"]["H"], {}
    for i, name in enumerate("kv"):
        if s["new"] is None:
            rows = p[name].flatten(0, 1).view(U8 if case["format"] == "e4m3" else p[name].dtype)[s["rows"]]
            got[name] = rows.view(p[name].dtype).double()
            if case["format"] == "e4m3":
                got[name] *= torch.exp2(p[name + "_scales"].flatten(0, 1)[s["rows"]].double() - 127)[..., None]
        else:
            x = s["new"][:, case["packed"] + i * H:][:, :H].double()
            got[name] = _nearest_e4m3(x.clamp(-LIMIT[s["new"].dtype], LIMIT[s["new"].dtype])) if case["format"] == "e4m3" else x
    return got


def _exact_attn(s):
    """A sequence and a head at a time."""
    case, p = s["case"], s["pages"]
    G, page = case["Hq"] // case["Hk"], case["page"]
    out = torch.zeros(s["out"].shape, dtype=F64, device=DEV)
    for n, (nq, nk) in enumerate(zip(_list(case["q"]), _list(case["k"]))):
        if not nq or not nk:
            continue
        q0, mine = int(s["cu_q"][n]), s["table"][n, :-(-nk // page)].long()
        held = {}
        for name in "kv":
            x = p[name].view(U8 if case["format"] == "e4m3" else p[name].dtype)[mine].view(p[name].dtype).double()
            if case["format"] == "e4m3":
                x = x * torch.exp2(p[name + "_scales"][mine].double() - 127)[..., None]
            held[name] = x.flatten(0, 1)[:nk]
        hide = torch.zeros((nq, nk), dtype=F64, device=DEV)
        hide.masked_fill_(torch.ones_like(hide, dtype=torch.bool).triu(1 + nk - nq), -math.inf)
        if case["window"]:
            far = torch.ones_like(hide, dtype=torch.bool).tril(nk - nq - case["window"])
            far[:, :case["sinks"]] = False
            hide.masked_fill_(far, -math.inf)
        for h in range(case["Hq"]):
            scores = torch.mm(s["q"][q0:q0 + nq, h].double(), held["k"][:, h // G].t().contiguous()) * s["scale"] + hide
            out[q0:q0 + nq, h] = torch.mm(torch.exp(scores - torch.logsumexp(scores, 1, keepdim=True)), held["v"][:, h // G].contiguous())
    return out
