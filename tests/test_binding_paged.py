"""The compiled binding's functions for normed queries and keys, paged caches and attention over them against the Python functions that they
stand in front of: the same results, the same refusals."""
import math
import types

import pytest
import torch

from test_binding import _wrong

E4M3 = torch.float8_e4m3fn
OUT = dict(norm_rope=(6,), norm_rope_grad=(7, 8, 9), cache_write=(), cache_read=(2, 3), attn_paged=(5,))


@pytest.fixture(scope="module")
def cm():
    import paper_2506_03275_amd as cm
    cm.load()
    return cm


def _calls(cm, dev, dtype=torch.bfloat16):
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    r = lambda *shape: torch.randn(shape, generator=g, device=dev).to(dtype)   # noqa: E731
    i32 = lambda *values: torch.tensor(values, dtype=torch.int32, device=dev)  # noqa: E731
    qkv, f32 = r(40, 6, 64), lambda *shape: torch.zeros(shape, device=dev)     # noqa: E731
    pos, freqs = torch.arange(120, dtype=torch.int32, device=dev).view(40, 3), torch.linspace(1, 0.1, 32, dtype=torch.float64, device=dev)
    rows, ws = torch.arange(40, device=dev) * 2, torch.zeros(1 << 20, dtype=torch.uint8, device=dev)
    if dev == "cuda":
        scales = [torch.full((5, 16, 1), 127, dtype=torch.uint8, device=dev) for _ in "kv"]
        pages = cm.Pages(r(5, 16, 1, 64).to(E4M3), r(5, 16, 1, 64).to(E4M3), *scales)
    else:
        pages = types.SimpleNamespace(_plain=(4096, 0, 1, 64))
    return dict(
        norm_rope=[qkv[:, :5], r(64), r(64), 4, pos, freqs, r(5, 40, 64).transpose(0, 1), [16, 8, 8], 1e-6, True],
        norm_rope_grad=[r(40, 5, 64), qkv[:, :5], r(64), r(64), 4, pos, freqs, r(5, 40, 64).transpose(0, 1), f32(64), f32(64), (16, 8, 8), 1e-5, False, ws],
        cache_write=[qkv[:, 4:5], qkv[:, 5:], rows, pages],
        cache_read=[pages, rows, r(40, 1, 64), r(40, 1, 64)],
        attn_paged=[qkv[:, :4], pages, i32(4, 0, 2, 1, 3).view(1, 5), i32(0, 40), i32(70), r(40, 4, 64), 40, 80, True, 1 / math.sqrt(64), 30, 2, ws])


NAMES = list(OUT)


def _native_args(args):
    """What the Python functions hand over: of pages what these say of themselves."""
    return [getattr(a, "_plain", a) if not isinstance(a, torch.Tensor) else a for a in args]


def _outcome(cm, fast, name, args):
    args = list(args)
    for i in OUT[name]:
        if type(args[i]) is torch.Tensor and args[i].device.type == "cuda":
            args[i] = args[i].clone(memory_format=torch.preserve_format)
    before, cm._fast = cm._fast, fast
    try:
        getattr(cm, name)(*args)
    except Exception as e:   # noqa: BLE001
        return type(e).__name__, str(e)
    finally:
        cm._fast = before
    if name == "cache_write":
        pages = args[3]
        return [pages.k.view(torch.uint8).clone(), pages.v_scales.clone()]
    return [args[i] for i in OUT[name] if args[i] is not None]


def _same(got, want):
    if isinstance(got, tuple) or isinstance(want, tuple):
        return got == want
    return len(got) == len(want) and all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_what_is_wrong_raises_what_it_raised(cm, name):
    native = cm._fast
    assert native.__name__.endswith("_native")
    args = _calls(cm, "cpu")[name]
    plain = _native_args(args)
    assert getattr(native, name)(*plain) is None and getattr(native, name)(*plain[:-1]) is None and getattr(native, name)() is None
    for i, bad in _wrong(args):
        assert getattr(native, name)(*_native_args(bad)) is None, i
        got = _outcome(cm, native, name, bad)
        assert isinstance(got, tuple) and got == _outcome(cm, cm._Python(), name, bad), i


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", NAMES)
def test_the_binding_does_what_the_python_functions_do(cm, name, dtype):
    native = cm._fast
    args = _calls(cm, "cuda", dtype)[name]
    if name == "norm_rope":
        args[6].fill_(0)
    assert getattr(native, name)(*_native_args(args)) == 0
    got, want = _outcome(cm, native, name, args), _outcome(cm, cm._Python(), name, args)
    assert isinstance(got, list) and _same(got, want)
    refused = 0
    for i, bad in _wrong(args):   # whatever is refused is refused before anything is launched
        if name.startswith("cache") and isinstance(bad[i], torch.Tensor) and bad[i].dtype == torch.int64 and bad[i].is_cuda and bad[i].numel():
            bad[i] = bad[i] % 80  # (still rows, none twice)
            if len(set(bad[i].flatten().tolist())) < bad[i].numel():
                continue
        got, want = _outcome(cm, native, name, bad), _outcome(cm, cm._Python(), name, bad)
        assert _same(got, want), (i, got, want)
        refused += isinstance(got, tuple)
    assert refused >= 4 * len(args)


@pytest.mark.gpu
def test_pages_of_another_device_are_refused(cm):
    args = _calls(cm, "cuda")["cache_write"]
    args[3].device, args[3]._plain = 1, (args[3]._address, 1, 1, 64)
    for fast in (cm._fast, cm._Python()):
        got = _outcome(cm, fast, "cache_write", args)
        assert got == ("ValueError", "pages: must live on the current device")


def test_sizes_beyond_32_bits_are_refused(cm):
    """Not cut to what 32 bits hold.  (Tensors without memory: the sizes are looked at first.)"""
    bf, far = torch.bfloat16, 2 ** 32 + 8
    e = lambda *shape, dtype=bf: torch.empty(shape, dtype=dtype, device="meta")   # noqa: E731
    for fast in (cm._fast, cm._Python()):
        before, cm._fast = cm._fast, fast
        try:
            for name, args in (("norm_rope", (e(far, 1, 64), e(64), e(64), 1, None, None, e(far, 1, 64), (0, 0, 0))), ("cache_write", (e(far, 1, 64), e(far, 1, 64), e(far, dtype=torch.int64), None)),
                               ("attn_paged", (e(far, 1, 64), None, e(1, 4, dtype=torch.int32), e(2, dtype=torch.int32), e(1, dtype=torch.int32), e(far, 1, 64), 1, 1, True, 0.1))):
                with pytest.raises(ValueError, match="2\\^31"):
                    getattr(cm, name)(*args)
        finally:
            cm._fast = before
    for i in range(8):
        with pytest.raises(ValueError, match="32 bits"):
            cm.attn_paged_workspace_bytes(*[far if n == i else 64 for n in range(8)])
    for i in range(3):
        with pytest.raises(ValueError, match="32 bits"):
            cm.norm_rope_grad_workspace_bytes(*[far if n == i else 64 for n in range(3)])
