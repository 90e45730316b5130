"""The compiled binding's functions for tensors with strides (projections, rotary positions, packed attention) against the Python
functions that they stand in front of: the same results, the same refusals."""
import math

import pytest
import torch

from test_binding import _wrong


@pytest.fixture(scope="module")
def cm():
    import paper_2506_03275_amd as cm
    cm.load()
    return cm


def _calls(dev, dtype=torch.bfloat16):
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    r = lambda *shape: torch.randn(shape, generator=g, device=dev).to(dtype)   # noqa: E731
    i32 = lambda *values: torch.tensor(values, dtype=torch.int32, device=dev)  # noqa: E731
    rows = r(40, 6, 64)
    return dict(
        linear=[r(40, 144)[:, 8:72], r(24, 64), r(24), r(40, 24), r(40, 24), 1],
        rope=[rows[:, :4], torch.arange(120, dtype=torch.int32, device=dev).view(40, 3), torch.linspace(1, 0.1, 32, dtype=torch.float64, device=dev), r(4, 40, 64).transpose(0, 1),
              [16, 8, 8], False, True],
        attn_packed=[rows[:, :4], rows[:, 4:5], rows[:, 5:], i32(0, 30, 40), i32(0, 25, 40), r(40, 4, 64), 30, 40, True, 1 / math.sqrt(64), i32(20, 10),
                     torch.zeros(1 << 20, dtype=torch.uint8, device=dev)])


NAMES = list(_calls("cpu"))


def _outcome(cm, fast, name, args):
    out = {"linear": 4, "rope": 3, "attn_packed": 5}[name]
    if isinstance(args[out], torch.Tensor) and args[out].device.type == "cuda" and type(args[out]) is torch.Tensor:
        args = args[:out] + [args[out].clone(memory_format=torch.preserve_format)] + args[out + 1:]
    before, cm._fast = cm._fast, fast
    try:
        getattr(cm, name)(*args)
    except Exception as e:   # noqa: BLE001
        return type(e).__name__, str(e)
    finally:
        cm._fast = before
    return args[out]


@pytest.mark.parametrize("name", NAMES)
def test_what_is_wrong_raises_what_it_raised(cm, name):
    native = cm._fast
    assert native.__name__.endswith("_native")
    args = _calls("cpu")[name]
    assert getattr(native, name)(*args) is None and getattr(native, name)(*args[:-1]) is None and getattr(native, name)() is None
    for i, bad in _wrong(args):
        assert getattr(native, name)(*bad) is None, i
        got = _outcome(cm, native, name, bad)
        assert isinstance(got, tuple) and got == _outcome(cm, cm._Python(), name, bad), i


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", NAMES)
def test_the_binding_does_what_the_python_functions_do(cm, name, dtype):
    native = cm._fast
    args = _calls("cuda", dtype)[name]
    optional = {"linear": (2, 3), "rope": (), "attn_packed": (10, 11)}[name]
    for plain in [args] + [args[:i] + [None] + args[i + 1:] for i in optional]:
        assert getattr(native, name)(*plain) == 0
        got, want = _outcome(cm, native, name, plain), _outcome(cm, cm._Python(), name, plain)
        assert isinstance(got, torch.Tensor) and torch.equal(got, want)
    refused = 0
    for i, bad in _wrong(args):   # whatever is refused is refused before anything is launched
        got, want = _outcome(cm, native, name, bad), _outcome(cm, cm._Python(), name, bad)
        assert type(got) is type(want) and (got == want if isinstance(got, tuple) else torch.equal(got, want)), (i, got, want)
        refused += isinstance(got, tuple)
    assert refused >= 4 * len(args)


def test_sizes_beyond_32_bits_are_refused(cm):
    """Not cut to what 32 bits hold, in which more than 2^32 rows would be a few.  (Tensors without memory: the sizes are looked at first.)"""
    bf, far = torch.bfloat16, 2 ** 32 + 8
    e = lambda *shape, dtype=bf: torch.empty(shape, dtype=dtype, device="meta")   # noqa: E731
    cu, heads = e(2, dtype=torch.int32), e(8, 1, 64)
    for fast in (cm._fast, cm._Python()):
        before, cm._fast = cm._fast, fast
        try:
            for name, args in (("linear", (e(far, 64), e(16, 64), None, None, e(far, 16))),
                               ("rope", (e(far, 1, 64), e(far, 3, dtype=torch.int32), e(32, dtype=torch.float64), e(far, 1, 64), (32, 0, 0))),
                               ("attn_packed", (e(far, 1, 64), heads, heads, cu, cu, e(far, 1, 64), 1, 1, True, 0.1))):
                with pytest.raises(ValueError, match="2\\^31"):
                    getattr(cm, name)(*args)
        finally:
            cm._fast = before
    for i in range(6):
        with pytest.raises(ValueError, match="32 bits"):
            cm.attn_packed_workspace_bytes(*[far if n == i else 64 for n in range(6)])


@pytest.mark.gpu
def test_numbers_beyond_32_bits_are_refused(cm):
    far = 2 ** 32
    linear, rope, attn = (_calls("cuda")[name] for name in ("linear", "rope", "attn_packed"))
    wrong = [("linear", linear[:5] + [far + 1]), ("rope", rope[:4] + [[far + 16, 8, 8 - far], False, True])]
    wrong += [("attn_packed", attn[:i] + [far + attn[i]] + attn[i + 1:]) for i in (6, 7)]
    for name, args in wrong:
        for fast in (cm._fast, cm._Python()):
            got = _outcome(cm, fast, name, args)
            assert isinstance(got, tuple) and got[0] == "ValueError" and "32 bits" in got[1], (name, got)
    many = lambda t: t[:1].expand(far + 8, *t.shape[1:])   # noqa: E731
    for name, args in (("linear", linear[:1] + [many(linear[1])] + linear[2:]), ("attn_packed", attn[:1] + [many(attn[1]), many(attn[2])] + attn[3:])):
        for fast in (cm._fast, cm._Python()):
            got = _outcome(cm, fast, name, args)
            assert isinstance(got, tuple) and got[0] == "ValueError" and "2^31" in got[1], (name, got)


@pytest.mark.gpu
def test_a_workspace_may_be_larger(cm):
    args = _calls("cuda")["attn_packed"]
    large = args[:11] + [torch.empty(2 ** 31 + 64, dtype=torch.uint8, device="cuda")]
    assert torch.equal(_outcome(cm, cm._fast, "attn_packed", large), _outcome(cm, cm._fast, "attn_packed", args))
