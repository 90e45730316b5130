"""The norm of queries and keys with rotary positions, and its gradient, against their definitions in 64 bits, against differences, and what they
refuse.

Tolerances.  u = 2^-24, half a step of 32 bits.  A sum of E squares of one sign passes E / 8 + 8 roundings at most, and half of its relative
error is the norm's; a reciprocal root is off by 2 u more, the products by 3 u: r w x is off by d = ((E / 8 + 8) / 2 + 8) u of itself.  Sines and cosines of a turn
given in 32 bits: 4e-6 of the pair's magnitude, in which d is lost twice over for E <= 512; a result is rounded once, eps / 2 of its value.  The gradient
has two such factors: with a = r (|g w| + |n| mean |g w n|), g by rotation off by 4e-6 of its pair, dx is off by 1.2e-5 + 4 d of a, pair by pair or
by the mean, and rounded once.  The weights' gradients sum R rows' products, each off by 8e-6 + 2 d, in 32 bits in chains of at most 64 + R / 64 roundings."""
import ctypes
import math

import pytest
import torch

DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16]
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def cm():
    import paper_2506_03275_amd as cm
    cm.load()
    return cm


def _turn(y, pos, freqs, axes, halves, sign):
    """The pairs of y [tokens, heads, E] in 64 bits, turned."""
    P = sum(axes)
    if P == 0:
        return y.clone()
    axis = torch.tensor(sum(([i] * n for i, n in enumerate(axes)), []), device=y.device)
    angle = (pos.double()[:, axis] * freqs * sign)[:, None]
    out = y.clone()
    a, b = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    out[..., a], out[..., b] = y[..., a] * angle.cos() - y[..., b] * angle.sin(), y[..., a] * angle.sin() + y[..., b] * angle.cos()
    return out


def _pairs(size, axes, halves):
    """Each element's pair's magnitude: |a| + |b|, itself where it has no partner."""
    P = sum(axes)
    out = size.clone()
    a, b = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    out[..., a], out[..., b] = size[..., a] + size[..., b], size[..., a] + size[..., b]
    return out


def _weights(wq, wk, q_heads, heads, E):
    rows = [wq.double().expand(q_heads, E)] if q_heads else []
    return torch.cat(rows + ([wk.double().expand(heads - q_heads, E)] if q_heads < heads else []))


def _d(E):
    return ((E / 8 + 8) / 2 + 8) * 2.0 ** -24


def norm_rope_reference(x, wq, wk, q_heads, pos, freqs, axes, eps, halves):
    info = torch.finfo(x.dtype)
    f = x.double()
    E = x.shape[-1]
    y = f / torch.sqrt(f.square().mean(-1, keepdim=True) + eps) * _weights(wq, wk, q_heads, x.shape[1], E)
    out = _turn(y, pos, freqs, axes, halves, 1)
    return out, info.eps / 2 * out.abs() * 1.01 + (4e-6 + 2 * _d(E)) * _pairs(y.abs(), axes, halves) + info.tiny * info.eps


def norm_rope_grad_reference(grad, x, wq, wk, q_heads, pos, freqs, axes, eps, halves):
    """dx, dq_weight, dk_weight and how far they may be off."""
    info = torch.finfo(x.dtype)
    f, heads, E = x.double(), x.shape[1], x.shape[2]
    r = 1 / torch.sqrt(f.square().mean(-1, keepdim=True) + eps)
    n, w = f * r, _weights(wq, wk, q_heads, heads, E)
    g = _turn(grad.double(), pos, freqs, axes, halves, -1)
    dx = r * (g * w - n * (g * w * n).mean(-1, keepdim=True))
    size = _pairs(g.abs(), axes, halves)                       # of g's pair, which its error goes by
    a = r * (size * w.abs() + n.abs() * (size * w.abs() * n.abs()).mean(-1, keepdim=True))
    off = info.eps / 2 * dx.abs() * 1.01 + (1.2e-5 + 4 * _d(E)) * a + info.tiny * info.eps
    both, slack = [], []
    for heads_of in (slice(0, q_heads), slice(q_heads, heads)):
        R = x.shape[0] * len(range(*heads_of.indices(heads)))
        both.append((g * n)[:, heads_of].sum((0, 1)))
        slack.append((8e-6 + 2 * _d(E) + (64 + R / 64) * 2.0 ** -24) * (size * n.abs())[:, heads_of].sum((0, 1)) + 1e-30)
    return dx, both, off, slack


def _inputs(cm, tokens, heads, E, axes, dtype, seed, layout="rows", scale=1.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *shape: torch.randn(shape, generator=g, device=DEV)   # noqa: E731
    def rows(values=None):
        if layout == "rows":
            t = torch.full((tokens, heads, E), math.nan, dtype=dtype, device=DEV)
        elif layout == "projection":   # other heads behind them
            t = torch.full((tokens, heads + 3, E), math.nan, dtype=dtype, device=DEV)[:, :heads]
        else:
            t = torch.full((heads, tokens, E), math.nan, dtype=dtype, device=DEV).transpose(0, 1)
        return t if values is None else t.copy_(values)
    x = rows((r(tokens, heads, E) * scale).to(dtype))
    wq, wk = (r(E) * 0.3 + 1).to(dtype), (r(E) * 0.3 - 0.5).to(dtype)
    pos = torch.randint(-3000, 100000, (tokens, 3), generator=g, device=DEV, dtype=torch.int32)
    return x, wq, wk, pos, cm.rope_frequencies(axes) if sum(axes) else None, rows, r


SIZES = [(1, 1, 1, 64, (32, 0, 0)), (1, 40, 32, 128, (64, 0, 0)), (8, 40, 32, 128, (64, 0, 0)), (5, 3, 0, 64, (8, 8, 16)), (333, 7, 7, 128, (16, 24, 24)),
         (77, 24, 12, 128, (8, 28, 28)), (257, 48, 24, 128, (22, 21, 21)), (64, 5, 4, 256, (40, 44, 44)), (100, 2, 1, 80, (0, 16, 16)), (33, 65, 60, 8, (4, 0, 0)),
         (17, 9, 5, 512, (128, 64, 64)), (200, 100, 37, 96, (16, 0, 16)), (3, 1000, 999, 64, (8, 12, 12)), (50, 6, 3, 24, (0, 0, 0)), (19, 4, 2, 136, (0, 24, 0)),
         (40, 3, 1, 320, (80, 0, 72)), (2100, 70, 50, 128, (16, 24, 24)), (12011, 90, 45, 128, (22, 21, 21))]   # the last two past the L2s, past every cache


@gpu
@pytest.mark.parametrize("tokens,heads,q_heads,E,axes", SIZES, ids=lambda v: str(v).replace(" ", ""))
@pytest.mark.parametrize("halves", [False, True])
def test_norm_rope(cm, tokens, heads, q_heads, E, axes, halves):
    if halves and sum(axes) % 8:
        pytest.skip("halves of a multiple of eight pairs")
    for dtype in TYPES if tokens < 10000 else TYPES[:1]:
        for layout, to in (("rows", "heads"), ("projection", "rows"), ("heads", "projection")):
            x, wq, wk, pos, freqs, rows, _ = _inputs(cm, tokens, heads, E, axes, dtype, tokens + heads, layout)
            layout = to
            out = _inputs(cm, tokens, heads, E, axes, dtype, 0, to)[5]()
            p = pos if sum(axes) else None
            cm.norm_rope(x, wq, wk, q_heads, p, freqs, out, axes, 1e-6, halves)
            want, off = norm_rope_reference(x, wq, wk, q_heads, pos, freqs, axes, 1e-6, halves)
            assert bool(((out.double() - want).abs() <= off).all()), (dtype, layout, float(((out.double() - want).abs() / off).nan_to_num(1e9).max()))
            cm.norm_rope(x, wq, wk, q_heads, p, freqs, x, axes, 1e-6, halves)   # in place
            assert torch.equal(x, out)
            if tokens * heads > 100000:
                break


@gpu
@pytest.mark.parametrize("tokens,heads,q_heads,E,axes", SIZES, ids=lambda v: str(v).replace(" ", ""))
@pytest.mark.parametrize("halves", [False, True])
def test_gradient(cm, tokens, heads, q_heads, E, axes, halves):
    if halves and sum(axes) % 8:
        pytest.skip("halves of a multiple of eight pairs")
    for dtype in TYPES if tokens < 10000 else TYPES[:1]:
        for layout in ("rows", "projection", "heads"):
            x, wq, wk, pos, freqs, rows, r = _inputs(cm, tokens, heads, E, axes, dtype, tokens + heads, layout)
            grad, dx = rows(r(tokens, heads, E).to(dtype)), rows()
            dq, dk = torch.full((2, E), math.nan, device=DEV)
            ws = torch.full((cm.norm_rope_grad_workspace_bytes(tokens, heads, E),), 255, dtype=torch.uint8, device=DEV)
            p = pos if sum(axes) else None
            call = lambda to: cm.norm_rope_grad(grad, x, wq, wk, q_heads, p, freqs, to, dq if q_heads else None, dk if q_heads < heads else None, axes, 1e-6, halves, ws)   # noqa: E731
            call(dx)
            want, weights, off, slack = norm_rope_grad_reference(grad, x, wq, wk, q_heads, pos, freqs, axes, 1e-6, halves)
            assert bool(((dx.double() - want).abs() <= off).all()), (dtype, layout, float(((dx.double() - want).abs() / off).nan_to_num(1e9).max()))
            for got, exact, most, some in ((dq, weights[0], slack[0], q_heads > 0), (dk, weights[1], slack[1], q_heads < heads)):
                assert bool(((got.double() - exact).abs() <= most).all()) if some else bool(got.isnan().all())
            before = dq.clone(), dk.clone()
            call(grad)                                          # in the place of the gradient that came in; the same bits again
            assert torch.equal(grad, dx) and all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(before, (dq, dk)))
            if tokens * heads > 100000:
                break


@gpu
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("tokens,heads", [(1, 40), (8, 40), (333, 48), (4608, 48), (12011, 90)])
def test_what_the_order_of_the_weights_sums_goes_by(cm, tokens, heads, halves):
    """Sizes, halves and which of dx's strides is the larger: where x and grad lie, what is between dx's rows and the alignment of a row change no bit of
    the weights' gradients, and nothing changes dx.  Each of dx's two orders is compared with 64 bits (test_gradient has one for the largest size)."""
    axes, E, got = (16, 24, 24), 128, {}
    for order, layouts in (("rows", ("rows", "projection", "rows of 136")), ("heads", ("heads", "heads of 136"))):
        for to, source in zip(layouts, ("rows", "heads", "projection")):
            x, wq, wk, pos, freqs, rows, r = _inputs(cm, tokens, heads, E, axes, torch.bfloat16, 11, source)
            grad, dw = rows(r(tokens, heads, E).to(torch.bfloat16)), torch.full((2, E), math.nan, device=DEV)
            wide = to.endswith("136")
            dx = torch.empty((heads, tokens, 136), dtype=x.dtype, device=DEV).transpose(0, 1)[..., 8:] if wide and order == "heads" else (
                torch.empty((tokens, heads, 136), dtype=x.dtype, device=DEV)[..., 8:] if wide else _inputs(cm, tokens, heads, E, axes, x.dtype, 0, to)[5]())
            ws = torch.full((cm.norm_rope_grad_workspace_bytes(tokens, heads, E),), 255, dtype=torch.uint8, device=DEV)
            cm.norm_rope_grad(grad, x, wq, wk, heads // 2, pos, freqs, dx, dw[0], dw[1], axes, 1e-6, halves, ws)
            if order not in got:
                want, weights, off, slack = norm_rope_grad_reference(grad, x, wq, wk, heads // 2, pos, freqs, axes, 1e-6, halves)
                assert bool(((dx.double() - want).abs() <= off).all()), order
                assert all(bool(((d.double() - exact).abs() <= most).all()) for d, exact, most in zip(dw, weights, slack)), order
                got[order] = dw
            got["dx"] = got.get("dx", dx)
            assert torch.equal(dx, got["dx"]) and torch.equal(dw, got[order]), to


@gpu
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("heads,E", [(40, 128), (100, 64), (5, 128)])
def test_one_token_is_summed_as_the_first_of_two(cm, heads, E, halves):
    """A token alone has no stride that could tell rows from heads of rows: its rows' sums are those of a second one behind it whose gradient is zero."""
    axes, dw = (E // 2, 0, 0), []
    x, wq, wk, pos, freqs, rows, r = _inputs(cm, 2, heads, E, axes, torch.bfloat16, 4)
    grad = rows(r(2, heads, E).to(torch.bfloat16))
    grad[1] = 0
    ws = torch.empty(cm.norm_rope_grad_workspace_bytes(2, heads, E), dtype=torch.uint8, device=DEV)
    for n in (2, 1):
        dx = torch.empty((n, heads, E), dtype=torch.bfloat16, device=DEV)
        dw.append((dx[0], torch.empty((2, E), device=DEV)))
        cm.norm_rope_grad(grad[:n], x[:n], wq, wk, heads // 2, pos[:n], freqs, dx, dw[-1][1][0], dw[-1][1][1], axes, 1e-6, halves, ws)
    assert torch.equal(dw[0][0], dw[1][0]) and torch.equal(dw[0][1], dw[1][1])


@gpu
@pytest.mark.parametrize("halves", [False, True])
def test_gradient_against_differences(cm, halves):
    """The loss sum(c out) over single steps of x and of a weight: differences of the definition in 64 bits against the kernel's gradients."""
    axes, dtype, eps = (8, 16, 8), torch.float16, 1e-3
    x, wq, wk, pos, freqs, rows, r = _inputs(cm, 9, 4, 80, axes, dtype, 3)
    grad, dx, dw = r(9, 4, 80).to(dtype), rows(), torch.empty((2, 80), device=DEV)
    ws = torch.empty(cm.norm_rope_grad_workspace_bytes(9, 4, 80), dtype=torch.uint8, device=DEV)
    cm.norm_rope_grad(grad, x, wq, wk, 3, pos, freqs, dx, dw[0], dw[1], axes, eps, halves, ws)

    def loss(x, wq, wk):
        f = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * torch.cat([wq.expand(3, 80), wk.expand(1, 80)])
        return (_turn(f, pos, freqs, axes, halves, 1) * grad.double()).sum().item()
    at, h = (x.double(), wq.double(), wk.double()), 1e-6
    for which, index in ((0, (0, 0, 0)), (0, (4, 2, 31)), (0, (8, 3, 79)), (0, (3, 1, 64)), (1, (0,)), (1, (63,)), (2, (5,)), (2, (79,))):
        up, down = [t.clone() for t in at], [t.clone() for t in at]
        up[which][index] += h
        down[which][index] -= h
        slope = (loss(*up) - loss(*down)) / (2 * h)
        got = float((dx, dw[0], dw[1])[which][index])
        # third derivatives of order one times h^2, and differences of sums of some hundreds in 64 bits over h: 1e-7; then the kernel's own rounding
        assert abs(got - slope) <= 1e-4 * max(1.0, abs(slope)) + (2.0 ** -11 * abs(slope) if which == 0 else 0.0), (which, index, got, slope)


@gpu
@pytest.mark.parametrize("halves", [False, True])
def test_rows_of_zeros_and_of_extremes(cm, halves):
    """A row of zeros stays one; squares that pass 32 bits' range, an infinity, a NaN: each in its own row."""
    axes = (16, 8, 8)
    x, wq, wk, pos, freqs, rows, r = _inputs(cm, 6, 3, 64, axes, torch.bfloat16, 5)
    x[0] = 0
    x[1] = 3e38
    x[2, :, ::2] = -2e30
    x[3, 1, 7] = math.inf
    x[4, 2, 9] = math.nan
    out = rows()
    cm.norm_rope(x, wq, wk, 2, pos, freqs, out, axes, 1e-6, halves)
    want, off = norm_rope_reference(x, wq, wk, 2, pos, freqs, axes, 1e-6, halves)
    assert torch.equal(out[0], torch.zeros_like(out[0]))
    fine = want.isfinite()
    assert bool(((out.double() - want).abs() <= off)[fine].all()) and torch.equal(out.isnan(), want.isnan())
    grad, dx, dw = r(6, 3, 64).to(torch.bfloat16), rows(), torch.empty((2, 64), device=DEV)
    ws = torch.empty(cm.norm_rope_grad_workspace_bytes(6, 3, 64), dtype=torch.uint8, device=DEV)
    for at in (slice(0, 3), slice(5, 6)):                        # (a NaN would be in the sums)
        cm.norm_rope_grad(grad[at], x[at], wq, wk, 2, pos[at], freqs, dx[at], dw[0], dw[1], axes, 1e-6, halves, ws)
        want, weights, off, slack = norm_rope_grad_reference(grad[at], x[at], wq, wk, 2, pos[at], freqs, axes, 1e-6, halves)
        assert bool(((dx[at].double() - want).abs() <= off).all())
        assert all(bool(((got.double() - exact).abs() <= most).all()) for got, exact, most in zip(dw, weights, slack))


@gpu
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("size,eps", [(2.0 ** 61, 1e37), (1.2e18, 3.4e38), (3e19, 3e38), (1.0, 3.4e38), (2.0 ** 61, 1e-6)])
def test_squares_beyond_32_bits_beside_an_eps_of_their_size(cm, size, eps, halves):
    """The sum of a row's squares, or their mean and eps together, pass 32 bits' range (1.2e18: the latter alone): eps counts all the same."""
    axes = (16, 8, 8)
    x, wq, wk, pos, freqs, rows, r = _inputs(cm, 6, 3, 64, axes, torch.bfloat16, 7)
    x.copy_(torch.where(x < 0, -size, size) * (1 + 0.1 * torch.rand(x.shape, device=DEV)))
    x[4] = r(3, 64)                                             # (a row as any)
    out = rows()
    cm.norm_rope(x, wq, wk, 2, pos, freqs, out, axes, eps, halves)
    want, off = norm_rope_reference(x, wq, wk, 2, pos, freqs, axes, eps, halves)
    assert bool(((out.double() - want).abs() <= off).all())
    grad, dx, dw = r(6, 3, 64).to(torch.bfloat16), rows(), torch.empty((2, 64), device=DEV)
    ws = torch.empty(cm.norm_rope_grad_workspace_bytes(6, 3, 64), dtype=torch.uint8, device=DEV)
    cm.norm_rope_grad(grad, x, wq, wk, 2, pos, freqs, dx, dw[0], dw[1], axes, eps, halves, ws)
    want, weights, off, slack = norm_rope_grad_reference(grad, x, wq, wk, 2, pos, freqs, axes, eps, halves)
    assert bool(((dx.double() - want).abs() <= off).all())
    assert all(bool(((got.double() - exact).abs() <= most).all()) for got, exact, most in zip(dw, weights, slack))


@gpu
def test_one_weight_alone(cm):
    """Where no head has a weight there need not be one."""
    x, w, other, pos, freqs, rows, r = _inputs(cm, 20, 3, 64, (32, 0, 0), torch.bfloat16, 2)
    a, b = rows(), rows()
    cm.norm_rope(x, w, None, 3, pos, freqs, a, (32, 0, 0))
    cm.norm_rope(x, None, w, 0, pos, freqs, b, (32, 0, 0))
    want, off = norm_rope_reference(x, w, other, 3, pos, freqs, (32, 0, 0), 1e-6, False)
    assert torch.equal(a, b) and bool(((a.double() - want).abs() <= off).all())


@gpu
def test_what_lies_between_the_rows_stays(cm):
    x, wq, wk, pos, freqs, _, r = _inputs(cm, 50, 6, 128, (64, 0, 0), torch.float16, 1, "projection")
    held = torch.full((50, 10, 136), 7.0, dtype=torch.float16, device=DEV)
    out = held[:, 2:8, :128]
    cm.norm_rope(x, wq, wk, 4, pos, freqs, out, (64, 0, 0), halves=True)
    rest = held.clone()
    rest[:, 2:8, :128] = 7.0
    assert torch.equal(rest, torch.full_like(held, 7.0)) and not bool((out == 7.0).all())


@gpu
def test_on_another_stream_and_in_graphs(cm):
    """Both calls captured, two graphs with workspaces of their own, replayed by turns with new inputs."""
    axes, calls = (16, 24, 24), []
    for seed, tokens in ((1, 300), (2, 77)):
        x, wq, wk, pos, freqs, rows, r = _inputs(cm, tokens, 12, 128, axes, torch.bfloat16, seed)
        state = dict(x=x, out=rows(), grad=rows(r(tokens, 12, 128).to(torch.bfloat16)), dx=rows(), dw=torch.zeros((2, 128), device=DEV),
                     ws=torch.empty(cm.norm_rope_grad_workspace_bytes(tokens, 12, 128), dtype=torch.uint8, device=DEV))

        def run(s=state, wq=wq, wk=wk, pos=pos, freqs=freqs):
            cm.norm_rope(s["x"], wq, wk, 8, pos, freqs, s["out"], axes)
            cm.norm_rope_grad(s["grad"], s["x"], wq, wk, 8, pos, freqs, s["dx"], s["dw"][0], s["dw"][1], axes, ws=s["ws"])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        calls.append((state, run, graph, r))
    for turn in range(3):
        for state, run, graph, r in calls:
            state["x"].copy_(r(*state["x"].shape))
            graph.replay()
            torch.cuda.synchronize()
            got = [state[n].clone() for n in ("out", "dx", "dw")]
            run()
            assert all(torch.equal(a, state[n]) for a, n in zip(got, ("out", "dx", "dw"))) and bool(got[2].isfinite().all())


def test_refuses(cm):
    """Before any launch; the addresses are never read."""
    lib, P = cm.load(), ctypes.c_void_p
    a, b = P(0x1000), P(0x1008)
    ok = [a, 256, 64, a, a, 2, a, a, a, 256, 64, 10, 4, 64, 16, 8, 8, 1e-6, 0, 0, None]
    f = lambda **at: lib.chipmunk_norm_rope(*[at.get("_" + str(i), v) for i, v in enumerate(ok)])   # noqa: E731
    for i in (0, 3, 4, 6, 7, 8):
        assert f(**{f"_{i}": None}) == -1
    assert f(_0=b) == f(_8=b) == f(_3=b) == f(_6=P(0x1002)) == f(_7=P(0x1004)) == -3
    assert f(_1=60, _2=60) == f(_1=32) == f(_9=-256) == -2           # rows overlap
    assert f(_1=260, _9=256) == f(_1=257) == -3
    assert f(_11=0) == f(_12=0) == f(_13=0) == f(_5=5) == f(_5=-1) == f(_12=70000) == f(_14=-8) == f(_14=100) == -2
    assert f(_13=68, _1=288, _2=72, _9=288, _10=72) == f(_14=14, _15=8, _16=8) == f(_19=2) == -4
    assert f(_14=4, _18=1) == -4                                     # halves of 20 pairs
    for eps in (0.0, -1.0, math.nan, math.inf, 1e-39):
        assert f(_17=eps) == -2
    size = lib.chipmunk_norm_rope_grad_workspace_bytes
    assert size(10, 4, 64) == 40 * 2 * 64 * 4 and size(0, 4, 64) == size(10, 0, 64) == size(10, 4, 60) == size(10, 4, 520) == 0
    assert size(10 ** 6, 40, 128) == 2048 * 2 * 128 * 4
    ok_grad = [a, 256, 64] + ok[:8] + [a, 256, 64, a, a] + ok[11:20] + [a, 1 << 20, None]
    h = lambda **at: lib.chipmunk_norm_rope_grad(*[at.get("_" + str(i), v) for i, v in enumerate(ok_grad)])   # noqa: E731
    for i in (0, 3, 6, 7, 9, 10, 11, 14, 15):
        assert h(**{f"_{i}": None}) == -1, i
    assert h(_25=None) == h(_26=100) == -5 and h(_25=b) == h(_0=b) == h(_14=P(0x1002)) == -3 and h(_1=32) == -2


def test_functions_refuse(cm):
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)   # noqa: E731
    with pytest.raises(ValueError, match="must live on the GPU"):
        cm.norm_rope(t(4, 2, 64), t(64), t(64), 1, t(4, 3, dtype=torch.int32), t(32, dtype=torch.float64), t(4, 2, 64), (32, 0, 0))
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        cm.norm_rope(t(4, 2, 64, dtype=torch.float32), t(64), t(64), 1, None, None, t(4, 2, 64), (0, 0, 0))


@gpu
def test_functions_refuse_on_the_gpu(cm):
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device=DEV)   # noqa: E731
    x, w, pos, freqs = t(4, 2, 64), t(64), t(4, 3, dtype=torch.int32), t(32, dtype=torch.float64)
    good = [x, w, w, 1, pos, freqs, t(4, 2, 64), (32, 0, 0)]
    cm.norm_rope(*good)
    for i, bad, error in ((0, t(4, 2, 64, dtype=torch.float16), TypeError), (1, t(32), ValueError), (2, t(64, dtype=torch.float32), TypeError), (3, 2 ** 40, ValueError),
                          (4, t(3, 3, dtype=torch.int32), ValueError), (5, t(31, dtype=torch.float64), ValueError), (6, t(4, 2, 128)[..., ::2], ValueError),
                          (6, t(4, 3, 64), ValueError), (3, 3, cm.ChipmunkError), (1, None, cm.ChipmunkError)):
        with pytest.raises(error):
            cm.norm_rope(*good[:i], bad, *good[i + 1:])
    dw, ws = t(2, 64, dtype=torch.float32), t(1 << 16, dtype=torch.uint8)
    good = [x, x, w, w, 1, pos, freqs, t(4, 2, 64), dw[0], dw[1], (32, 0, 0), 1e-6, False, ws]
    cm.norm_rope_grad(*good)
    for i, bad, error in ((0, t(4, 2, 64, dtype=torch.float16), TypeError), (0, t(4, 3, 64), ValueError), (8, t(63, dtype=torch.float32), ValueError), (9, w, TypeError),
                          (13, ws[:64], cm.ChipmunkError), (13, None, cm.ChipmunkError), (8, None, cm.ChipmunkError)):
        with pytest.raises(error):
            cm.norm_rope_grad(*good[:i], bad, *good[i + 1:])
