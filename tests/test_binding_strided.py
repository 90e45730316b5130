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
