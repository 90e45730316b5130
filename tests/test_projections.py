"""The linear layer and rotary positions against their definitions in 64 bits, and what they refuse.

Tolerances.  A result is rounded once, to half a step of its type, eps / 2 of its value (eps: torch.finfo).  Before that a sum of D
products in 32 bits: eight products are added with one rounding, so a sum has passed through D / 8 + 8 of them at most, each 2^-24
of what has been added in magnitude; an activation (slope below 1.13) hands that on and adds a few units of 32 bits of its own,
2e-6 (1 + |y|).  Sines and cosines of a turn given in 32 bits: 4e-6 of the pair's magnitude."""
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


def _randn(shape, dtype, seed, scale=1.0, device=DEV):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=device) * scale).to(dtype)


def _spread(t, columns, fill):
    """The same values as the first columns of wider rows."""
    wide = torch.full((t.shape[0], t.shape[1] + columns), fill, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide, wide[:, :t.shape[1]]


def _activation(y, act):
    return {0: lambda: 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5))), 1: lambda: 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))),
            2: lambda: y, 3: lambda: y / (1 + torch.exp(-y))}[act]()


def linear_reference(x, w, bias, residual, act):
    """The result in 64 bits and how far the kernel's may be from it."""
    x64, w64 = x.double(), w.double()
    y = x64 @ w64.t()
    magnitude = x64.abs() @ w64.abs().t()
    if bias is not None:
        y, magnitude = y + bias.double(), magnitude + bias.double().abs()
    off = 1.13 * (x.shape[1] / 8 + 8) * 2.0 ** -24 * magnitude + (0 if act == 2 else 2e-6 * (1 + y.abs()))
    out = _activation(y, act)
    if residual is not None:
        out = out + residual.double()
        off = off + 2.0 ** -24 * out.abs()
    info = torch.finfo(x.dtype)
    return out, off * (1 + info.eps) + info.eps / 2 * out.abs() + info.tiny * info.eps


def _check_linear(cm, N, D, F, dtype, act, bias=True, residual=True, seed=0, spread=0, alias=False):
    x, w = _randn((N, D), dtype, seed), _randn((F, D), dtype, seed + 1, 1 / math.sqrt(D))
    b = _randn((F,), dtype, seed + 2) if bias else None
    r = _randn((N, F), dtype, seed + 3) if residual else None
    want, off = linear_reference(x, w, b, r, act)
    out = torch.full((N, F), math.nan, dtype=dtype, device=DEV)
    frame = None
    if spread:
        _, x = _spread(x, spread, math.nan)          # behind a row's end is nothing that may be read into a result
        frame, out = _spread(out, spread, 7.0)
        if residual:
            _, r = _spread(r, spread + 8, math.nan)
    if alias:
        out.copy_(r)
        r = out
    cm.linear(x, w, b, r, out, act)
    assert bool(((out.double() - want).abs() <= off).all()), float(((out.double() - want).abs() / off).max())
    if frame is not None:
        assert bool((frame[:, F:] == 7.0).all())
    again = torch.empty_like(out)
    if not alias:
        cm.linear(x, w, b, r, again, act)
        assert torch.equal(out, again)


SIZES = [(1, 8, 8), (1, 264, 72), (2, 256, 5120), (3, 4096, 1000), (5, 72, 16), (15, 1032, 520), (16, 640, 136), (17, 2056, 264), (31, 512, 2048),
         (33, 4104, 88), (64, 1024, 1024), (65, 64, 64), (100, 5120, 24), (127, 576, 392), (200, 8, 640), (255, 1536, 768), (256, 256, 256),
         (257, 320, 2056), (500, 3000, 1288), (1000, 128, 5000), (2049, 1000, 2000), (4608, 640, 1920)]
MORE_SIZES = [(100, 1040, 13392), (380, 392, 10880), (900, 4360, 2544), (450, 200, 10880), (2100, 968, 8200), (1500, 1016, 3000), (513, 72, 12296), (33, 8200, 264),
              (130, 5056, 640), (77, 1544, 1000), (300, 2056, 1000), (45, 640, 3496), (601, 1096, 520), (289, 4104, 1000), (33, 72, 24)]


@gpu
@pytest.mark.parametrize("N,D,F", SIZES + MORE_SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear(cm, N, D, F, dtype):
    seed = N + D + F
    _check_linear(cm, N, D, F, dtype, seed // 8 % 4, bias=seed % 3 != 0, residual=seed % 5 != 0, seed=seed)


# one row in the last tile of 64 or 128, whose contraction has an odd number of steps, the last one cut: two teams of waves, the second with
# a step less
LONE_ROWS = [(257, 3488, 1856), (193, 4400, 2512), (385, 3728, 1976), (513, 936, 2224), (385, 5560, 2960)]


def test_lone_rows_take_two_teams(cm):
    form = cm.load().chipmunk_internal_linear_form
    assert {form(*size) for size in LONE_ROWS} == {1, 2}
    assert all(N % (64, 128)[form(N, D, F) - 1] == 1 and D % 64 and -(-D // 64) % 2 for N, D, F in LONE_ROWS)


@gpu
@pytest.mark.parametrize("N,D,F", LONE_ROWS)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_a_lone_row_and_a_cut_step(cm, N, D, F, dtype):
    """Of a tile's only row nothing behind the contraction's end gets into a result: NaN stand there."""
    x, w = _randn((N, D), dtype, N), _randn((F, D), dtype, D, 1 / math.sqrt(D))
    frame = torch.full((N * D + 4096,), math.nan, dtype=dtype, device=DEV)
    frame[:N * D] = x.view(-1)
    want, off = linear_reference(x, w, None, None, 2)
    out = torch.full((N, F), math.nan, dtype=dtype, device=DEV)
    cm.linear(frame[:N * D].view(N, D), w, None, None, out)
    assert bool(((out.double() - want).abs() <= off).all())


@gpu
@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("N", [1, 40, 300])
def test_linear_what_follows_the_product(cm, act, bias, residual, N):
    for dtype in TYPES:
        _check_linear(cm, N, 136, 328, dtype, act, bias, residual, seed=act)


@gpu
@pytest.mark.parametrize("N,D,F", [(1, 520, 264), (7, 1032, 40), (50, 72, 136), (130, 200, 1032), (700, 1096, 520), (1500, 328, 2056)])
def test_linear_rows_with_gaps(cm, N, D, F):
    """Rows further apart than they are long: nothing between them is read into a result or written."""
    for dtype in TYPES:
        _check_linear(cm, N, D, F, dtype, 2, seed=N, spread=24)
        _check_linear(cm, N, D, F, dtype, 1, seed=N, spread=24, alias=True)


@gpu
@pytest.mark.parametrize("N", [1, 100, 3000])
def test_linear_infinite_and_nan(cm, N):
    """A row or a column that holds one is the only one that shows it."""
    x, w = _randn((N, 264), torch.bfloat16, 1), _randn((136, 264), torch.bfloat16, 2)
    clean = torch.empty((N, 136), dtype=torch.bfloat16, device=DEV)
    cm.linear(x, w, None, None, clean)
    x[N // 2, 263], w[77, 0] = math.nan, math.inf
    out = torch.empty_like(clean)
    cm.linear(x, w, None, None, out)
    rows, columns = torch.arange(N, device=DEV) != N // 2, torch.arange(136, device=DEV) != 77
    assert torch.equal(out[rows][:, columns], clean[rows][:, columns])
    assert bool(out[N // 2].isnan().all()) and not bool(out[:, 77].isfinite().any())


@gpu
@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [1, 12, 40, 300, 3000])
def test_linear_activations_of_anything(cm, N, act, dtype):
    """Infinities, NaN and values where an exponential over- or underflows, as the formulas in 64 bits have them: the product is zero, so that
    the bias goes through the activation as it is."""
    most = float(torch.finfo(dtype).max)
    values = [math.inf, -math.inf, math.nan, most, -most, most / 2, -most / 2, 1000.0, -1000.0, 88.0, -88.0, -103.0, 30.0, -30.0, -31.0, 14.0, -14.0, -13.0, 5.0, -5.0, 1.0, -1.0, 0.0, 2.0 ** -14]
    bias = torch.tensor(values * 11, dtype=dtype, device=DEV)
    x, w = torch.zeros((N, 72), dtype=dtype, device=DEV), _randn((len(bias), 72), dtype, 3)
    out = torch.zeros((N, len(bias)), dtype=dtype, device=DEV)
    cm.linear(x, w, bias, None, out, act)
    want = _activation(bias.double(), act).expand(N, -1)
    finite = want.isfinite()
    assert torch.equal(out.isnan(), want.isnan()) and bool((out[want.isinf()].double() == want[want.isinf()]).all())
    # as linear_reference has it, without the product: a few units of 32 bits, and the rounding
    info = torch.finfo(dtype)
    off = (2e-6 * (1 + want.abs()) if act != 2 else 0) + info.eps / 2 * want.abs() + info.tiny * info.eps
    assert bool(((out.double() - want).abs() <= off)[finite].all())


@gpu
def test_linear_overflow_is_infinite(cm):
    for dtype, large in ((torch.float16, 200.0), (torch.bfloat16, 1e19)):
        x, w = torch.full((3, 64), large, dtype=dtype, device=DEV), torch.full((16, 64), large, dtype=dtype, device=DEV)
        out = torch.empty((3, 16), dtype=dtype, device=DEV)
        cm.linear(x, w, None, None, out)
        assert bool((out == math.inf).all())
        if dtype is torch.float16:   # finite in 32 bits
            cm.linear(-x, w, None, None, out, cm.ACT_GELU_TANH)
            assert bool((out == 0).all())


@gpu
def test_linear_on_another_stream_and_in_a_graph(cm):
    x, w, r = _randn((300, 512), torch.bfloat16, 1), _randn((640, 512), torch.bfloat16, 2, 0.05), _randn((300, 640), torch.bfloat16, 3)
    want = torch.empty((300, 640), dtype=torch.bfloat16, device=DEV)
    cm.linear(x, w, None, r, want)
    out, side = torch.zeros_like(want), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cm.linear(x, w, None, r, out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cm.linear(x, w, None, r, out)
    for seed in range(3):
        x.copy_(_randn((300, 512), torch.bfloat16, 10 + seed))
        cm.linear(x, w, None, r, want)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@gpu
def test_linear_beyond_32_bits(cm):
    """Rows whose distance in bytes passes 2^32, in x and in out."""
    N, D, F = 4200, 64, 72
    ld = (1 << 19) + 8
    wide = torch.empty((N, ld), dtype=torch.bfloat16, device=DEV)
    x, out = wide[:, :D], wide[:, D:D + F]
    x.copy_(_randn((N, D), torch.bfloat16, 4))
    w = _randn((F, D), torch.bfloat16, 5, 0.1)
    cm.linear(x, w, None, None, out)
    want, off = linear_reference(x.contiguous(), w, None, None, 2)
    assert bool(((out.double() - want).abs() <= off).all())


@gpu
@pytest.mark.parametrize("N,D,F", [(30000, 64, 5120), (30000, 512, 5120), (120, 136, 1130048), (190, 264, 720064)])
def test_linear_results_past_the_caches(cm, N, D, F):
    """Larger than the last-level cache: of whole lines, and the same in rows that are not."""
    x, w, bias, residual = _randn((N, D), torch.bfloat16, 1), _randn((F, D), torch.bfloat16, 2, 0.1), _randn((F,), torch.bfloat16, 3), _randn((N, F), torch.bfloat16, 4)
    out = torch.full((N, F), math.nan, dtype=torch.bfloat16, device=DEV)
    cm.linear(x, w, bias, residual, out)
    for rows in (slice(0, 10), slice(N - 10, N)):
        want, off = linear_reference(x[rows], w, bias, residual[rows], 2)
        assert bool(((out[rows].double() - want).abs() <= off).all())
    assert not bool(out.isnan().any())
    frame, inside = _spread(out, 8, 7.0)
    inside.fill_(math.nan)
    cm.linear(x, w, bias, residual, inside)
    assert torch.equal(inside, out) and bool((frame[:, F:] == 7.0).all())


def test_every_form_of_tiles_is_reached(cm):
    """From one row to thousands; the sizes of test_linear take each form."""
    form = cm.load().chipmunk_internal_linear_form
    assert form(1, 4096, 4096) == form(16, 64, 30720) == 11 and form(400, 4096, 4096) < 7 <= form(17, 4096, 1024) < 11
    assert {form(N, D, F) for N, D, F in SIZES + MORE_SIZES} == set(range(12))
    # a result so long that one launch does not cover it with small tiles has larger ones
    sizes = [(64, 64), (64, 64), (64, 128), (128, 128), (128, 128), (128, 192), (256, 256), (16, 16), (16, 32), (32, 32), (64, 32)]
    for N, F in ((2 ** 29, 8), (2 ** 30 - 256, 8), (8, 2 ** 29), (16, 2 ** 30 - 256)):
        columns, rows = sizes[form(N, 8, F)]
        assert -(-N // rows) * -(-F // columns) < 2 ** 22


def test_no_accumulator_is_touched_before_its_product_has_landed(tmp_path):
    """The widest tiles' products are inline assembly (see the module of the same check)."""
    import os
    import re
    import subprocess

    from paper_2506_03275_amd import build
    from test_compiled_products import _faults
    out = tmp_path / "linear.s"
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--offload-device-only", "-S", os.path.join(build.CSRC, "linear.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    text = out.read_text()
    kernels = re.findall(r"^(_ZN\w*linear_wide_kernel\w*):(.*?)^\s*\.size\s+\1,", text, re.S | re.M)
    assert len(kernels) == 4   # two types, a whole or a cut last step
    for name, body in kernels:
        lines = [line.split(";")[0].strip() for line in body.split("\n")]
        assert not _faults([line for line in lines if line and not re.match(r"\.(?!L)", line)]), name
    # nothing lies in scratch memory
    spills = dict(re.findall(r"\.name:\s+(_ZN\w*linear_\w+_kernel\w*).*?\.vgpr_spill_count:\s*(\d+)", text, re.S))
    assert len(spills) >= 20 and set(spills.values()) == {"0"}, spills


# ---- rotary positions ---------------------------------------------------------------------------------------------------

def rope_reference(x, pos, freqs, axes, halves, inverse):
    P = sum(axes)
    axis = torch.tensor(sum(([i] * n for i, n in enumerate(axes)), []), device=x.device)
    angle = (pos.double()[:, axis] * freqs * (-1 if inverse else 1))[:, None]
    out = x.double().clone()
    a, b = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    xa, xb = x.double()[..., a], x.double()[..., b]
    out[..., a], out[..., b] = xa * angle.cos() - xb * angle.sin(), xa * angle.sin() + xb * angle.cos()
    info = torch.finfo(x.dtype)
    off = info.eps / 2 * out.abs() + info.tiny * info.eps
    for half in (a, b):
        off[..., half] += 4e-6 * (1 + info.eps) * (xa.abs() + xb.abs())
    off[..., 2 * P:] = 0
    return out, off


def _positions(n, seed, most):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(-most, most + 1, (n, 3), generator=g, dtype=torch.int64)
    pos[0] = 0
    return pos.clamp(-2 ** 31, 2 ** 31 - 1).to(torch.int32).to(DEV)


ROPES = [(1, 1, 64, (32, 0, 0)), (1, 40, 128, (64, 0, 0)), (8, 40, 128, (64, 0, 0)), (5, 3, 64, (8, 8, 16)), (333, 7, 128, (16, 24, 24)), (77, 24, 128, (8, 28, 28)),
         (1000, 48, 128, (22, 21, 21)), (64, 5, 256, (40, 44, 44)), (100, 2, 80, (0, 16, 16)), (33, 65, 8, (4, 0, 0)), (17, 9, 512, (128, 64, 64)),
         (200, 100, 96, (16, 0, 16)), (3, 1000, 64, (8, 12, 12)), (2100, 70, 128, (16, 24, 24)), (20011, 53, 128, (22, 21, 21))]   # the last two past the L2s, past every cache


@gpu
@pytest.mark.parametrize("tokens,heads,E,axes", ROPES)
@pytest.mark.parametrize("halves", [False, True])
def test_rope(cm, tokens, heads, E, axes, halves):
    if sum(axes) % 8 and halves:
        axes = (sum(axes) // 8 * 8 or 8, 0, 0)
        if 2 * sum(axes) > E:
            pytest.skip("no eight pairs in so short a head")
    freqs = cm.rope_frequencies(axes)
    pos = _positions(tokens, tokens, 100000)
    for dtype in TYPES:
        x = _randn((tokens, heads, E), dtype, E)
        for inverse in (False, True):
            want, off = rope_reference(x, pos, freqs, axes, halves, inverse)
            out = torch.full_like(x, math.nan)
            cm.rope(x, pos, freqs, out, axes, halves, inverse)
            assert bool(((out.double() - want).abs() <= off).all()), float(((out.double() - want).abs() / off.clamp(min=1e-30)).max())
            by_head = torch.full((heads, tokens, E), math.nan, dtype=dtype, device=DEV)      # to heads of rows, and from there in place
            cm.rope(x, pos, freqs, by_head.transpose(0, 1), axes, halves, inverse)
            assert torch.equal(by_head.transpose(0, 1), out)
            by_head.copy_(x.transpose(0, 1))
            cm.rope(by_head.transpose(0, 1), pos, freqs, by_head.transpose(0, 1), axes, halves, inverse)
            assert torch.equal(by_head.transpose(0, 1), out)


@gpu
def test_rope_inside_wider_rows(cm):
    """Queries and keys of a projection's result, in place: the values behind them stay."""
    rows = _randn((50, 5 + 2, 64), torch.bfloat16, 3)
    before, x = rows.clone(), rows[:, :5]
    pos, axes = _positions(50, 1, 300), (8, 8, 8)
    freqs = cm.rope_frequencies(axes)
    want, off = rope_reference(x.clone(), pos, freqs, axes, False, False)
    cm.rope(x, pos, freqs, x, axes)
    assert bool(((x.double() - want).abs() <= off).all()) and torch.equal(rows[:, 5:], before[:, 5:])
    assert torch.equal(x[..., 48:], before[:, :5, 48:])                                       # behind the pairs


@gpu
def test_rope_results_beyond_32_bits(cm):
    """Results further apart than an offset of 32 bits reaches, of whole lines and not, and one larger than the last-level cache."""
    heads, E, axes = 3, 128, (64, 0, 0)
    freqs = cm.rope_frequencies(axes)
    wide = torch.empty((18, 1 << 26), dtype=torch.bfloat16, device=DEV)
    for at in (0, 8):
        out, x, pos = wide[:, at:at + heads * E].unflatten(1, (heads, E)), _randn((18, heads, E), torch.bfloat16, at), _positions(18, at, 1000)
        for halves in (False, True):
            want, off = rope_reference(x, pos, freqs, axes, halves, False)
            cm.rope(x, pos, freqs, out, axes, halves)
            assert bool(((out.double() - want).abs() <= off).all())
    x, pos = _randn((23000, 48, E), torch.bfloat16, 1), _positions(23000, 1, 1000)
    out = torch.empty_like(x)
    cm.rope(x, pos, freqs, out, axes)
    for rows in (slice(0, 200), slice(22900, 23000)):
        want, off = rope_reference(x[rows], pos[rows], freqs, axes, False, False)
        assert bool(((out[rows].double() - want).abs() <= off).all())


@gpu
@pytest.mark.parametrize("most", [0, 1, 2 ** 20, 2 ** 31])
def test_rope_far_positions(cm, most):
    """The angle of a far position keeps its precision: 2^31 positions at one radian each."""
    pos, axes = _positions(40, 5, most), (16, 8, 8)
    freqs = cm.rope_frequencies(axes)
    x = _randn((40, 4, 64), torch.float16, 6)
    want, off = rope_reference(x, pos, freqs, axes, True, False)
    out = torch.empty_like(x)
    cm.rope(x, pos, freqs, out, axes, halves=True)
    assert bool(((out.double() - want).abs() <= off).all())
    if most == 0:
        assert torch.equal(out, x)


@gpu
def test_rope_inverse_is_the_gradient(cm):
    """<turn(x), y> = <x, turn back(y)>, and a difference of the turn along a direction is the turn of the direction."""
    axes = (8, 12, 12)
    pos, freqs = _positions(30, 2, 500), cm.rope_frequencies(axes)
    x, y = _randn((30, 6, 64), torch.float16, 7), _randn((30, 6, 64), torch.float16, 8)
    turned, back = torch.empty_like(x), torch.empty_like(y)
    cm.rope(x, pos, freqs, turned, axes)
    cm.rope(y, pos, freqs, back, axes, inverse=True)
    # of 11520 products, each off by half a step of one factor: their sum at most by the sum of them
    left, right = (turned.double() * y.double()).sum(), (x.double() * back.double()).sum()
    bound = (2.0 ** -11 + 4e-6) * ((turned.double() * y.double()).abs().sum() + (x.double() * back.double()).abs().sum())
    assert abs(float(left - right)) <= float(bound)
    want, off = rope_reference(x, pos, freqs, axes, False, False)
    other, off_other = rope_reference(y, pos, freqs, axes, False, False)
    moved, h = torch.empty_like(x), 2.0 ** -2
    step = (x.double() + h * y.double()).to(torch.float16)
    cm.rope(step, pos, freqs, moved, axes)
    along, off_along = rope_reference(step, pos, freqs, axes, False, False)
    assert bool((((moved.double() - turned.double()) - (along - want)).abs() <= off + off_along).all())


@gpu
def test_rope_over_voxel_ordered_positions(cm):
    """Positions go through the token reorder like the tokens (rows of three int32), and turning commutes with it."""
    T, H, W, voxel, E, axes = 3, 6, 8, (2, 2, 4), 64, (8, 12, 12)
    n = 5 + T * H * W
    grid = torch.stack(torch.meshgrid(torch.arange(T), torch.arange(H), torch.arange(W), indexing="ij"), -1).view(-1, 3)
    pos = torch.cat([torch.zeros(5, 3, dtype=torch.int64), grid]).to(torch.int32).to(DEV)[None]
    x = _randn((1, n, 2, E), torch.bfloat16, 11)
    pos2, x2, turned, turned2, moved = torch.empty_like(pos), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    freqs = cm.rope_frequencies(axes)
    cm.voxel_reorder(pos, pos2, None, None, 5, T, H, W, 0, *voxel)
    cm.voxel_reorder(x, x2, None, None, 5, T, H, W, 0, *voxel)
    cm.rope(x[0], pos[0], freqs, turned[0], axes)
    cm.rope(x2[0], pos2[0], freqs, turned2[0], axes)
    cm.voxel_reorder(turned, moved, None, None, 5, T, H, W, 0, *voxel)
    assert torch.equal(moved, turned2) and not torch.equal(x2, turned2)


# ---- refusals (no GPU) ----------------------------------------------------------------------------------------------------

def test_linear_refuses(cm):
    f, a = cm.load().chipmunk_linear, ctypes.c_void_p(0x1000)

    def call(x=a, ldx=64, w=a, bias=a, residual=a, ldr=128, out=a, ldo=128, N=4, D=64, F=128, act=2, dtype=0):
        return f(x, ldx, w, bias, residual, ldr, out, ldo, N, D, F, act, dtype, None)
    for missing in ("x", "w", "out"):
        assert call(**{missing: None}) == -1
    for wrong in (dict(N=0), dict(N=-1), dict(D=0), dict(F=0), dict(ldx=56), dict(ldo=120), dict(ldr=120), dict(ldx=1 << 22), dict(ldo=1 << 22),
                  dict(ldr=1 << 22), dict(D=1 << 20, ldx=1 << 20), dict(N=2 ** 31 - 1, F=1 << 20, ldo=1 << 20, ldr=1 << 20)):
        assert call(**wrong) == -2, wrong
    for wrong in (dict(D=60), dict(F=124), dict(act=4), dict(act=-1), dict(dtype=2), dict(dtype=-1)):
        assert call(**wrong) == -4, wrong
    for wrong in (dict(x=ctypes.c_void_p(0x1008)), dict(w=ctypes.c_void_p(0x1002)), dict(bias=ctypes.c_void_p(0x1008)), dict(residual=ctypes.c_void_p(0x1004)),
                  dict(out=ctypes.c_void_p(0x1008)), dict(ldx=68), dict(ldo=132), dict(ldr=132)):
        assert call(**wrong) == -3, wrong


def test_rope_refuses(cm):
    f, a = cm.load().chipmunk_rope, ctypes.c_void_p(0x1000)

    def call(x=a, xt=256, xh=64, pos=a, freqs=a, out=a, ot=256, oh=64, tokens=3, heads=4, E=64, axes=(16, 8, 8), halves=0, inverse=0, dtype=0):
        return f(x, xt, xh, pos, freqs, out, ot, oh, tokens, heads, E, *axes, halves, inverse, dtype, None)
    for missing in ("x", "pos", "freqs", "out"):
        assert call(**{missing: None}) == -1
    for wrong in (dict(tokens=0), dict(heads=0), dict(E=0), dict(axes=(0, 0, 0)), dict(axes=(-4, 8, 8)), dict(axes=(16, 16, 4)), dict(xt=192), dict(oh=56),
                  dict(xt=64, xh=128), dict(xt=-256), dict(heads=65537, xt=1 << 23, ot=1 << 23), dict(axes=(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1))):
        assert call(**wrong) == -2, wrong
    for wrong in (dict(E=60, axes=(16, 8, 4)), dict(E=520, xh=520, xt=2080, oh=520, ot=2080), dict(axes=(3, 0, 0)), dict(axes=(16, 8, 4), halves=1), dict(dtype=2)):
        assert call(**wrong) == -4, wrong
    for wrong in (dict(x=ctypes.c_void_p(0x1008)), dict(out=ctypes.c_void_p(0x1008)), dict(pos=ctypes.c_void_p(0x1002)), dict(freqs=ctypes.c_void_p(0x1004)),
                  dict(xt=260), dict(oh=68, ot=300)):
        assert call(**wrong) == -3, wrong


def test_functions_refuse(cm):
    bf = torch.bfloat16
    x, w, out = torch.zeros(4, 64, dtype=bf), torch.zeros(16, 64, dtype=bf), torch.zeros(4, 16, dtype=bf)
    for args, error in (((x.float(), w, None, None, out), TypeError), ((x, w.half(), None, None, out), ValueError), ((x, w, None, None, out), ValueError),
                        ((x[0], w, None, None, out), ValueError), ((None, w, None, None, out), TypeError)):
        with pytest.raises(error):
            cm.linear(*args)
    h, pos, f = torch.zeros(4, 2, 64, dtype=bf), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    for args, error in (((h.float(), pos, f, h, (32, 0, 0)), TypeError), ((h, pos, f, h, (32, 0, 0)), ValueError), ((h[0], pos, f, h, (32, 0, 0)), ValueError)):
        with pytest.raises(error):
            cm.rope(*args)


@gpu
def test_functions_refuse_on_the_gpu(cm):
    bf = torch.bfloat16
    x, w, out = torch.zeros(4, 64, dtype=bf, device=DEV), torch.zeros(16, 64, dtype=bf, device=DEV), torch.zeros(4, 16, dtype=bf, device=DEV)
    b = torch.zeros(16, dtype=bf, device=DEV)
    wrong = [(x, w.half(), None, None, out), (x, w[:, :32], None, None, out), (x.t(), w, None, None, out), (x, w, b[:8], None, out), (x, w, None, out[:2], out),
             (x, w, None, None, out[:, :8]), (x, w, None, None, out.t()), (x[:, ::2], w[:, :32].contiguous(), None, None, out), (x, w, None, None, out.cpu())]
    for args in wrong:
        with pytest.raises((TypeError, ValueError)):
            cm.linear(*args)
    with pytest.raises(cm.ChipmunkError):
        cm.linear(x, w, None, None, out, 9)
    with pytest.raises(cm.ChipmunkError):
        cm.linear(x[:, 4:], torch.zeros(16, 60, dtype=bf, device=DEV), None, None, out)
    h, pos, f = torch.zeros(4, 2, 64, dtype=bf, device=DEV), torch.zeros(4, 3, dtype=torch.int32, device=DEV), torch.zeros(32, dtype=torch.float64, device=DEV)
    wrong = [(h, pos.long(), f, h, (32, 0, 0)), (h, pos[:3], f, h, (32, 0, 0)), (h, pos, f.float(), h, (32, 0, 0)), (h, pos, f, h, (16, 0, 0)), (h, pos, f, h[:2], (32, 0, 0)),
             (h, pos, f, h.half(), (32, 0, 0)), (h[..., ::2], pos, f[:16], h[..., ::2], (16, 0, 0))]
    for args in wrong:
        with pytest.raises((TypeError, ValueError)):
            cm.rope(*args)
