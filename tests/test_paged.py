"""Paged caches: what is written and read back, bit by bit, and attention over the pages against its definition in 64 bits; and what they refuse.

Tolerance of attention: that of attention over packed sequences (test_attn_packed.py), on the rows that the pages stand for."""
import ctypes
import math

import pytest
import torch

from test_attn_packed import _starts

DEV = "cuda"
TYPES = [torch.bfloat16, torch.float16]
E4M3 = torch.float8_e4m3fn
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def cm():
    import paper_2506_03275_amd as cm
    cm.load()
    return cm


# ---- writing and reading ------------------------------------------------------------------------------------------------

def _power(k):
    """2^k in 64 bits, exactly (library powers need not be)."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def in_codes(x):
    """Rows of x in e4m3: codes (as bytes), scales.  By the definition, in 64 bits, on any device."""
    emax = 127 if x.dtype == torch.bfloat16 else 15
    f = x.double()
    finite = f.isfinite()
    f = torch.where(finite, f.clamp(-1.875 * 2.0 ** emax, 1.875 * 2.0 ** emax), 0.0)
    most = f.abs().amax(-1, keepdim=True)
    fraction, exponent = torch.frexp(most)                    # most = fraction 2^exponent, 0.5 <= fraction < 1
    k = torch.where(most > 0, (exponent - 9 + (fraction > 0.875).int()).clamp(min=-126), 0)
    y = f * _power(-k)
    step = _power((torch.frexp(y)[1] - 4).clamp(min=-9))   # of four significant bits; 2^-9 at least
    y = torch.round(y / step) * step                          # (to even; both exact)
    codes = y.float().to(E4M3).view(torch.uint8)
    negative = x.double().signbit()
    codes = torch.where(y == 0, negative.to(torch.uint8) * 128, codes)
    return torch.where(finite, codes, 0x7f), (k + 127).to(torch.uint8)[..., 0]


def of_codes(codes, scales, dtype):
    """The rows that codes (bytes) stand for."""
    return (codes.view(E4M3).double() * _power(scales.int()[..., None] - 127)).to(dtype)


def make_pages(cm, pages, page, H, E, fmt, layout="plain", fill=None):
    """Pages of zeros (or bytes `fill`).  layouts: plain; heads: a page's rows of one head side by side; both: k and v in one tensor, page by page."""
    def held(width, dtype, lay):
        if lay == "heads":
            return [torch.zeros((pages, H, page, width), dtype=dtype, device=DEV).transpose(1, 2) for _ in "kv"]
        if lay == "both":
            t = torch.zeros((pages, 2, page, H, width), dtype=dtype, device=DEV)
            return [t[:, 0], t[:, 1]]
        return [torch.zeros((pages, page, H, width), dtype=dtype, device=DEV) for _ in "kv"]
    k, v = held(E, torch.uint8 if fmt == E4M3 else fmt, layout)
    if fill is not None:
        k.fill_(fill), v.fill_(fill)
    if fmt != E4M3:
        return cm.Pages(k, v)
    ks, vs = (t[..., 0] for t in held(1, torch.uint8, "heads" if layout == "plain" else "plain"))
    ks.fill_(127), vs.fill_(127)
    return cm.Pages(k.view(E4M3), v.view(E4M3), ks, vs)


def _flat(pages):
    """Codes or elements and scales of all rows: [rows, H, E], [rows, H]."""
    b = lambda t: (t.view(torch.uint8) if t.dtype == E4M3 else t).reshape(-1, *t.shape[2:])   # noqa: E731
    return b(pages.k), b(pages.v), None if pages.k_scales is None else b(pages.k_scales), None if pages.v_scales is None else b(pages.v_scales)


def _values(shape, dtype, seed, kind):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if kind == "bits":     # any bits, infinities and NaN among them
        return torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int16).view(dtype)
    if kind == "wide":     # rows of every magnitude that the type has
        power = torch.randint(-24 if dtype == torch.float16 else -133, 16 if dtype == torch.float16 else 128, shape[:-1], generator=g, device=DEV)
        return ((torch.rand(shape, generator=g, device=DEV, dtype=torch.float64) * 2 - 1) * _power(power[..., None])).to(dtype)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


@gpu
@pytest.mark.parametrize("kind", ["normal", "wide", "bits"])
@pytest.mark.parametrize("E", [64, 128])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,page,layout", [(1, 1, 16, "plain"), (7, 3, 16, "heads"), (300, 8, 64, "plain"), (1000, 2, 32, "both"), (129, 5, 256, "heads")])
def test_codes(cm, kind, E, dtype, T, H, page, layout):
    x = _values((T, 3 * H + 1, E), dtype, T + E, kind)
    k, v = x[:, H:2 * H], x[:, 2 * H:3 * H]
    pages = make_pages(cm, -(-T // page) + 2, page, H, E, E4M3, layout, fill=0x55)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    rows = torch.randperm(pages.rows(), generator=g, device=DEV)[:T]
    cm.cache_write(k, v, rows, pages)
    kc, vc, ks, vs = _flat(pages)
    for got, scale, values in ((kc, ks, k), (vc, vs, v)):
        codes, scales = in_codes(values)
        same = got[rows] == codes
        same |= ((got[rows] & 0x7f) == 0x7f) & ((codes & 0x7f) == 0x7f)     # a NaN has either sign
        assert bool(same.all()) and torch.equal(scale[rows], scales)
    untouched = torch.ones(pages.rows(), dtype=torch.bool, device=DEV)
    untouched[rows] = False
    assert bool((kc[untouched] == 0x55).all() and (vc[untouched] == 0x55).all() and (ks[untouched] == 127).all())
    for to in (torch.float16, torch.bfloat16):
        out = torch.full((2, H, T, E), 3.0, dtype=to, device=DEV).transpose(1, 2)
        cm.cache_read(pages, rows, out[0], out[1])
        for got, codes, scales in ((out[0], kc, ks), (out[1], vc, vs)):
            want = of_codes(codes[rows], scales[rows], to)
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
        if to == dtype:
            fine = torch.isfinite(k)
            size = k.double().abs().nan_to_num(posinf=0).amax(-1, keepdim=True)
            info = torch.finfo(dtype)
            # half a step of four significant bits, or of the least ones of the row's power; the clamp at the type's end; and of the type itself
            off = torch.maximum(2.0 ** -4 * k.double().abs(), 2.0 ** -10 * 2.0 ** -7 * size) + info.tiny * info.eps + 2.0 ** -136
            assert bool(((out[0].double() - k.double()).abs() <= off)[fine].all()) and bool(out[0].isnan()[~fine].all())


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["plain", "heads", "both"])
def test_elements(cm, dtype, layout):
    """Pages of the element type hold bit by bit what was written."""
    x = _values((77, 9, 128), dtype, 3, "bits")
    pages = make_pages(cm, 9, 16, 3, 128, dtype, layout, fill=5.0)
    rows = torch.arange(77, device=DEV) + 40
    cm.cache_write(x[:, 3:6], x[:, 6:], rows, pages)
    k, v, _, _ = _flat(pages)
    bits = lambda t: t.contiguous().view(torch.int16)   # noqa: E731
    assert torch.equal(bits(k[40:117]), bits(x[:, 3:6])) and torch.equal(bits(v[40:117]), bits(x[:, 6:])) and bool((k[:40] == 5).all() and (v[117:] == 5).all())
    out = torch.zeros((2, 77, 3, 128), dtype=dtype, device=DEV)
    cm.cache_read(pages, rows, out[0], out[1])
    assert torch.equal(bits(out[0]), bits(x[:, 3:6])) and torch.equal(bits(out[1]), bits(x[:, 6:]))


@gpu
@pytest.mark.parametrize("fmt", [E4M3, torch.bfloat16])
def test_rows_outside_are_left_alone(cm, fmt):
    """Negative rows and those behind the last page: nothing is written for them, and nothing read; a row may be read twice."""
    x = _values((6, 4, 64), torch.bfloat16, 1, "normal")
    pages = make_pages(cm, 2, 16, 2, 64, fmt, fill=9)
    rows = torch.tensor([-1, 31, 32, -2 ** 62, 2 ** 40 + 3, 0], device=DEV)
    cm.cache_write(x[:, :2], x[:, 2:], rows, pages)
    k = _flat(pages)[0]
    assert bool((k[1:31] == 9).all()) and not bool((k[[0, 31]] == 9).all())
    out = torch.full((2, 6, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    cm.cache_read(pages, torch.tensor([31, -1, 32, 31, 2 ** 62, 0], device=DEV), out[0], out[1])
    assert torch.equal(out[:, 0], out[:, 3]) and bool((out[:, [1, 2, 4]] == 7).all()) and not bool((out[:, [0, 5]] == 7).all())


# ---- attention ----------------------------------------------------------------------------------------------------------

def reference(q, k, v, causal, scale, window=0, sinks=0):
    """One sequence: q [n_q, Hq, E], k, v [n_k, Hk, E] -> the result in 64 bits and how far the kernel's may be from it."""
    (nq, Hq, E), (nk, Hk, _) = q.shape, k.shape
    info = torch.finfo(q.dtype)
    out, off = torch.zeros(nq, Hq, E, dtype=torch.float64, device=q.device), torch.zeros(nq, Hq, E, dtype=torch.float64, device=q.device)
    if nk == 0:
        return out, off
    j, at = torch.arange(nk, device=q.device), torch.arange(nq, device=q.device)[:, None] + (nk - nq)
    seen = (j <= at) if causal else torch.ones((nq, nk), dtype=torch.bool, device=q.device)
    if window:
        seen = seen & ((j > at - window) | (j < sinks))
    for h in range(Hq):
        qh, kh, vh = q[:, h].double(), k[:, h // (Hq // Hk)].double(), v[:, h // (Hq // Hk)].double()
        s = (qh @ kh.t() * scale).masked_fill(~seen, -math.inf)
        m = s.amax(1, keepdim=True).clamp(min=-1e300)
        p = torch.exp(s - m)
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        out[:, h] = p @ vh
        A = p @ vh.abs()
        d = 2.0 ** -24 * ((E / 8 + 10) * (qh.abs() @ kh.abs().t()) * scale + 2 * s.abs() + 8).masked_fill(~seen, 0).amax(1, keepdim=True)
        off[:, h] = info.eps / 2 * (A + 2 * out[:, h].abs()) * 1.02 + 2 * d * A + info.tiny * info.eps
        if q.dtype == torch.float16:
            off[:, h] += 2.0 ** -25 * nk * vh.abs().amax()
    return out, off


class Batch:
    """Sequences in pages, in any order; every place that no sequence has in use is NaN, and so are the scales' there."""

    def __init__(self, cm, nq, nk, Hq, Hk, E, dtype, fmt, page, seed=0, layout="plain", size=1.0, spare=2):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.cm, self.nq, self.nk, self.Hq, self.Hk, self.E, self.dtype = cm, nq, nk, Hq, Hk, E, dtype
        need = [-(-n // page) for n in nk]
        count = sum(need) + spare
        order = torch.randperm(count, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(nk), max(max(need), 1) + 1), -7, dtype=torch.int32, device=DEV)   # (a column more than is needed)
        used, rows = 0, []
        for s, n in enumerate(need):
            self.table[s, :n] = order[used:used + n]
            used += n
            j = torch.arange(nk[s], device=DEV)
            rows.append(self.table[s, j // page].long() * page + j % page)
        self.rows = rows
        self.pages = make_pages(cm, count, page, Hk, E, fmt, layout, fill=0x7f if fmt == E4M3 else math.nan)
        kv = (torch.randn((2, sum(nk), Hk, E), generator=g, device=DEV) * size).to(dtype)
        if sum(nk):
            cm.cache_write(kv[0], kv[1], torch.cat(rows), self.pages)
        self.q = (torch.randn((max(sum(nq), 1), Hq, E), generator=g, device=DEV) * size).to(dtype)
        self.cu = torch.tensor(_starts(nq), dtype=torch.int32, device=DEV)
        self.k_len = torch.tensor(nk, dtype=torch.int32, device=DEV)

    def held(self, s):
        """The keys and values that sequence s has, as its pages stand for them."""
        out = torch.empty((2, len(self.rows[s]), self.Hk, self.E), dtype=self.dtype, device=DEV)
        if len(self.rows[s]):
            self.cm.cache_read(self.pages, self.rows[s], out[0], out[1])
        return out

    def run(self, causal=True, scale=None, window=0, sinks=0, out=None, max_q=None, max_k=None, q=None):
        cm, scale = self.cm, scale or 1 / math.sqrt(self.E)
        max_q, max_k = max_q or max(max(self.nq), 1), max_k or max(max(self.nk), 1)
        bytes = cm.attn_paged_workspace_bytes(len(self.nq), self.Hq, self.Hk, self.E, max_q, max_k, window, sinks)
        ws = torch.full((max(16, bytes),), 255, dtype=torch.uint8, device=DEV)
        q = self.q if q is None else q
        out = torch.full(q.shape, math.nan, dtype=self.dtype, device=DEV) if out is None else out
        cm.attn_paged(q, self.pages, self.table, self.cu, self.k_len, out, max_q, max_k, causal, scale, window, sinks, ws=ws)
        return out

    def check(self, causal=True, scale=None, window=0, sinks=0, **more):
        out = self.run(causal, scale, window, sinks, **more)
        at = _starts(self.nq)
        for s, n in enumerate(self.nq):
            k, v = self.held(s)
            want, off = reference(self.q[at[s]:at[s] + n], k, v, causal, scale or 1 / math.sqrt(self.E), window, sinks)
            got = out[at[s]:at[s] + n].double()
            assert bool(((got - want).abs() <= off).all()), (s, n, self.nk[s], float(((got - want).abs() / off.clamp(min=1e-30)).nan_to_num(1e9).max()))
        total = sum(self.nq)
        assert torch.equal(self.run(causal, scale, window, sinks, **more)[:total], out[:total])
        return out


LENGTHS = [([1], [1]), ([1], [31]), ([1], [33]), ([5], [70]), ([64], [64]), ([200], [200]), ([1, 1, 1], [1, 4000, 129]), ([17, 3], [200, 3]), ([150], [1000]),
           ([64, 0, 9], [64, 30, 0]), ([300, 2], [100, 1]), ([4, 4, 4, 4], [4, 5, 600, 0]), ([1] * 40, list(range(0, 2000, 50))), ([130, 1, 33], [129, 900, 31]), ([8], [5000]),
           ([700], [2500]), ([1], [9001]), ([40, 17], [6000, 5100]), ([100], [7001])]


@gpu
@pytest.mark.parametrize("nq,nk", LENGTHS, ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("fmt", ["elements", "codes"])
@pytest.mark.parametrize("causal", [False, True])
def test_sequences(cm, nq, nk, fmt, causal):
    for i, (dtype, (Hq, Hk), E, page) in enumerate(((torch.bfloat16, (8, 2), 128, 16), (torch.float16, (4, 4), 64, 64), (torch.float16, (5, 1), 128, 256), (torch.bfloat16, (6, 2), 64, 32))):
        Batch(cm, nq, nk, Hq, Hk, E, dtype, dtype if fmt == "elements" else E4M3, page, seed=max(nk) + i, layout=("plain", "heads", "both", "plain")[i]).check(causal)


@gpu
@pytest.mark.parametrize("nq,nk", LENGTHS, ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 2), (64, 4), (100, 0), (129, 64), (1000, 1), (40, 300), (3000, 65)])
def test_windows(cm, nq, nk, window, sinks):
    for i, (dtype, (Hq, Hk), E, page, fmt) in enumerate(((torch.bfloat16, (8, 2), 128, 16, E4M3), (torch.float16, (4, 4), 64, 64, torch.float16), (torch.bfloat16, (3, 1), 128, 32, torch.bfloat16))):
        Batch(cm, nq, nk, Hq, Hk, E, dtype, fmt, page, seed=max(nk) + i).check(True, None, window, sinks)


# one batch for each form of whole sequences, of elements and of codes: 0 and 1: 16 and 32 rows of a key head, 2 and 3: 64 and 128 of a head
FORMS = [(128, 0, 0, 1, 1, [43, 6, 20, 32]), (128, 0, 1, 2, 2, [2761]), (128, 0, 2, 40, 8, [62, 7, 17, 17, 1, 2]), (128, 0, 3, 40, 8, [179, 95, 62, 175, 174, 169]),
         (128, 1, 0, 1, 1, [101]), (128, 1, 1, 2, 2, [2338]), (128, 1, 2, 40, 8, [127, 2, 122, 10, 85, 23]), (128, 1, 3, 40, 8, [97, 50, 87, 42, 79, 86]),
         (64, 0, 0, 1, 1, [101]), (64, 0, 1, 8, 8, [1572, 6]), (64, 0, 2, 1, 1, [38, 20, 35, 8]), (64, 0, 3, 32, 8, [1937, 1884]),
         (64, 1, 0, 1, 1, [101]), (64, 1, 1, 8, 8, [1482, 105, 5, 25]), (64, 1, 2, 1, 1, [30, 7, 6, 14, 29, 15]), (64, 1, 3, 40, 8, [360, 138, 194, 64, 228, 37])]
# and of more than 32 rows of a key head over keys in parts: E, codes, keys of a part, Hq, Hk, nq, nk
DIVIDED = [(128, 0, 512, 1, 1, [37], [5314]), (128, 0, 1536, 4, 4, [88, 1, 0, 80], [7550, 1537, 3, 7000]), (128, 1, 512, 1, 1, [33], [2251]), (128, 1, 768, 4, 4, [65, 64, 1, 60], [3689, 3600, 769, 768]),
           (64, 0, 768, 2, 2, [65, 2, 3, 65, 0, 9], [5758, 5000, 1, 300, 70, 769]), (64, 1, 1024, 20, 4, [181], [3011]), (64, 1, 512, 1, 1, [35], [2251])]
# and 64 or 128 rows of a head over keys in parts: E, codes, ten times the further parts and the form, Hq, Hk, nq, nk
ROWS_DIVIDED = [(128, 0, 52, 8, 1, [300, 7], [6000, 4097]), (128, 1, 53, 8, 1, [300, 1, 0, 299], [6100, 1024, 70, 1025]), (64, 0, 112, 16, 2, [200], [9001]), (64, 1, 113, 16, 2, [200, 150], [9000, 5000]),
                (128, 1, 152, 8, 1, [130], [40000]), (64, 0, 152, 9, 1, [129], [20011]), (128, 0, 72, 8, 8, [33, 1, 0, 20, 33, 7], [5404, 5000, 3, 1025, 40, 7]),
                (64, 1, 112, 4, 4, [130, 9, 1, 2], [8589, 1024, 1025, 3000])]


def _form(cm, E, Hq, Hk, nq, nk, codes, window=0, sinks=0, causal=1):
    Tq = len(nq) * max(nq) if nk is not nq else sum(nq)
    return cm.load().chipmunk_internal_attn_paged_form(len(nq), Tq, Hq, Hk, E, max(nq), max(nk), causal, window, sinks, codes)


def test_the_forms_are_what_the_batches_take(cm):
    for E, codes, form, Hq, Hk, lengths in FORMS:
        assert _form(cm, E, Hq, Hk, lengths, lengths, codes) == form == _form(cm, E, Hq, Hk, lengths, lengths, codes, 150, 70)
    for E, codes, keys, Hq, Hk, nq, nk in DIVIDED:
        assert _form(cm, E, Hq, Hk, nq, nk, codes) == keys and max(nq) * Hq // Hk > 32
    for E, codes, form, Hq, Hk, nq, nk in ROWS_DIVIDED:
        assert _form(cm, E, Hq, Hk, nq, nk, codes) == form


@gpu
@pytest.mark.parametrize("E,codes,form,Hq,Hk,lengths", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 70)])
def test_every_form(cm, E, codes, form, Hq, Hk, lengths, window, sinks):
    for dtype in TYPES:
        Batch(cm, lengths, lengths, Hq, Hk, E, dtype, E4M3 if codes else dtype, 64, seed=form).check(True, None, window, sinks)


@gpu
@pytest.mark.parametrize("E,codes,keys,Hq,Hk,nq,nk", DIVIDED)
def test_many_rows_over_divided_keys(cm, E, codes, keys, Hq, Hk, nq, nk):
    for dtype in TYPES:
        b = Batch(cm, nq, nk, Hq, Hk, E, dtype, E4M3 if codes else dtype, 32, seed=keys)
        q = torch.zeros((len(nq) * max(nq), Hq, E), dtype=dtype, device=DEV)      # (the tensor's rows are as many as the limit says)
        q[:b.q.shape[0]] = b.q
        b.q = q
        for window, sinks in ((0, 0), (2000, 40)):
            b.check(True, None, window, sinks)
        b.check(False)


@gpu
@pytest.mark.parametrize("E,codes,form,Hq,Hk,nq,nk", ROWS_DIVIDED)
def test_rows_over_divided_keys(cm, E, codes, form, Hq, Hk, nq, nk):
    for dtype in TYPES:
        b = Batch(cm, nq, nk, Hq, Hk, E, dtype, E4M3 if codes else dtype, 64, seed=form)
        q = torch.zeros((len(nq) * max(nq), Hq, E), dtype=dtype, device=DEV)
        q[:b.q.shape[0]] = b.q
        b.q = q
        for window, sinks in ((0, 0), (max(nk) - 1500, 100), (3000, 0)):
            b.check(True, None, window, sinks)
        b.check(False)


@gpu
def test_large_batches(cm):
    """More workgroups than stand on the card at a time."""
    lengths = [2003, 1, 1201, 701, 0, 700]
    for E, dtype, fmt in ((128, torch.bfloat16, E4M3), (64, torch.float16, E4M3), (128, torch.float16, torch.float16), (64, torch.bfloat16, torch.bfloat16)):
        b = Batch(cm, lengths, lengths, 40, 40, E, dtype, fmt, 64, seed=E)
        at = _starts(lengths)
        for window, sinks in ((0, 0), (150, 70)):
            out = b.run(True, None, window, sinks)
            assert not bool(out.isnan().any()) and torch.equal(b.run(True, None, window, sinks), out)
            for s, n in enumerate(lengths):
                k, v = b.held(s)
                for h in (0, 21, 39):
                    want, off = reference(b.q[at[s]:at[s] + n, h:h + 1], k[:, h:h + 1], v[:, h:h + 1], True, E ** -0.5, window, sinks)
                    assert bool(((out[at[s]:at[s] + n, h:h + 1].double() - want).abs() <= off).all()), (s, n, h)


@gpu
@pytest.mark.parametrize("E", [64, 128])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nq,nk", [([1, 2], [3000, 70]), ([300], [900]), ([2000], [2000])])
def test_codes_give_what_their_elements_give(cm, E, dtype, nq, nk):
    """Bit by bit: the same call over pages that hold the elements for which the codes stand."""
    b = Batch(cm, nq, nk, 8, 2, E, dtype, E4M3, 32, seed=E)
    want = b.run(True, None, 400, 5)
    plain = make_pages(cm, b.pages.k.shape[0], 32, 2, E, dtype)
    for s in range(len(nk)):
        cm.cache_write(*b.held(s), b.rows[s], plain)
    b.pages = plain
    assert torch.equal(b.run(True, None, 400, 5), want)


@gpu
@pytest.mark.parametrize("nq,nk", [([1], [400]), ([5], [400]), ([200], [300]), ([3, 9], [5000, 100])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (37, 0), (100, 40)])
@pytest.mark.parametrize("kind", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("fmt", ["elements", "codes"])
def test_hidden_keys_have_no_influence(cm, nq, nk, window, sinks, kind, fmt):
    """A key and a value that hold an infinity or a NaN reach the queries that see them and no other.  (In codes either is a NaN.)"""
    for dtype, E in ((torch.bfloat16, 128), (torch.float16, 64)):
        b = Batch(cm, nq, nk, 4, 2, E, dtype, E4M3 if fmt == "codes" else dtype, 16, seed=5)
        clean = b.run(True, 0.1, window, sinks)
        place = torch.arange(nq[0], device=DEV) + nk[0] - nq[0]
        held = b.held(0)
        for at in (3, nk[0] - 150, nk[0] - 1):
            sees = (place >= at) & (torch.tensor(at < sinks or not window, device=DEV) | (at > place - window))
            for which in (0, 1):
                spoiled = held.clone()
                spoiled[which, at, :, 5] = kind
                b.cm.cache_write(spoiled[0, at:at + 1], spoiled[1, at:at + 1], b.rows[0][at:at + 1], b.pages)
                out = b.run(True, 0.1, window, sinks)
                b.cm.cache_write(held[0, at:at + 1], held[1, at:at + 1], b.rows[0][at:at + 1], b.pages)
                assert torch.equal(out[:nq[0]][~sees], clean[:nq[0]][~sees]) and torch.equal(out[nq[0]:], clean[nq[0]:])
                if which == 1:
                    others = [e for e in range(E) if e != 5]
                    if fmt == "elements":
                        assert torch.equal(out[..., others], clean[..., others])
                    seen = out[:nq[0]][sees][..., 5]
                    assert bool(seen.isnan().all() if math.isnan(kind) or fmt == "codes" else (seen == kind).all())
                elif math.isnan(kind):
                    assert bool(out[:nq[0]][sees].isnan().all())
        assert torch.equal(b.run(True, 0.1, window, sinks), clean)


@gpu
def test_rows_of_no_sequence_stay(cm):
    b = Batch(cm, [5, 0, 70], [40, 3, 70], 4, 2, 64, torch.bfloat16, E4M3, 16)
    want = b.check()
    q = torch.cat([b.q, torch.full((9, 4, 64), math.nan, dtype=torch.bfloat16, device=DEV)])
    out = b.run(out=torch.full((84, 4, 64), 3.0, dtype=torch.bfloat16, device=DEV), q=q)
    assert torch.equal(out[:75], want) and bool((out[75:] == 3).all())


@gpu
@pytest.mark.parametrize("nq,nk", [([1, 2], [700, 30]), ([90], [500])])
def test_limits_far_above_the_lengths(cm, nq, nk):
    b = Batch(cm, nq, nk, 8, 2, 128, torch.bfloat16, E4M3, 16)
    for window, sinks in ((0, 0), (50, 3), (2 ** 31 - 1, 2 ** 31 - 1)):
        for max_q, max_k in ((None, 2 ** 31 - 1), (4096, 100000), (2 ** 31 - 1, 2 ** 31 - 1)):
            b.check(True, None, window, sinks, max_q=max_q, max_k=max_k)


@gpu
def test_bad_pages_and_lengths_stay_inside(cm):
    """Pages that there are not read as zeros; lengths and starts beyond the tensors are cut."""
    b = Batch(cm, [3, 70], [200, 90], 4, 2, 128, torch.bfloat16, torch.bfloat16, 16)
    clean = b.run()
    for bad in (-1, b.pages.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        page, rows = b.table[0, 2].clone(), b.rows[0][32:48]
        b.table[0, 2] = bad
        got = b.run()
        b.table[0, 2] = page
        held = b.held(0)
        zeros = torch.zeros((16, 2, 128), dtype=torch.bfloat16, device=DEV)
        cm.cache_write(zeros, zeros, rows, b.pages)
        assert torch.equal(b.run(), got) and torch.equal(got[3:], clean[3:])
        cm.cache_write(held[0, 32:48], held[1, 32:48], rows, b.pages)
    for k_len, cu in (([2 ** 31 - 1, -5], [0, 3, 73]), ([200, 90], [0, 3, 2 ** 31 - 1]), ([200, 90], [-9, 2 ** 30, -1])):
        b.k_len.copy_(torch.tensor(k_len)), b.cu.copy_(torch.tensor(cu))
        b.run(), b.run(max_q=2 ** 31 - 1, max_k=2 ** 31 - 1), b.run(window=20, sinks=2)
    b.k_len.copy_(torch.tensor([200, 90])), b.cu.copy_(torch.tensor([0, 3, 73]))
    assert torch.equal(b.run(), clean)


@gpu
@pytest.mark.parametrize("fmt", ["elements", "codes"])
@pytest.mark.parametrize("nq", [1, 70])
def test_offsets_beyond_32_bits(cm, fmt, nq):
    """Pages that lie more than 2^32 elements from the first."""
    dtype, H, E, page = torch.bfloat16, 4, 128, 16
    b = Batch(cm, [nq], [100], 8, H, E, dtype, E4M3 if fmt == "codes" else dtype, page)
    far = (1 << 32) // (H * E * page) + 9
    pages = make_pages(cm, far + 8, page, H, E, E4M3 if fmt == "codes" else dtype)
    want, held = b.run(), b.held(0)
    for i in range(7):
        b.table[0, i] = far + 6 - i if i != 3 else 0
    j = torch.arange(100, device=DEV)
    b.rows, b.pages = [b.table[0, j // page].long() * page + j % page], pages
    cm.cache_write(held[0], held[1], b.rows[0], pages)
    assert torch.equal(b.held(0), held) and torch.equal(b.run(), want)


@gpu
def test_a_sequence_longer_than_the_table_in_lds(cm):
    """Parts of the table come and go: 4096 keys of it are at hand at a time."""
    for nq, nk, Hq, Hk in ((300, 13001, 4, 2), (2, 40000, 4, 2), (65, 9000, 64, 1)):
        for fmt, dtype, E in ((E4M3, torch.bfloat16, 128), (torch.float16, torch.float16, 64)):
            for window, sinks in ((0, 0), (8500, 5)):
                Batch(cm, [nq], [nk], Hq, Hk, E, dtype, fmt, 16).check(True, None, window, sinks)


@gpu
def test_shared_pages(cm):
    """Two sequences may have the same first pages."""
    b = Batch(cm, [1, 1], [100, 96], 4, 2, 64, torch.bfloat16, E4M3, 32)
    b.table[1, :3] = b.table[0, :3]
    b.rows[1] = b.rows[0][:96]
    b.check()


@gpu
def test_on_another_stream_and_in_graphs(cm):
    """Writing, attention and reading captured together, two graphs with workspaces of their own, replayed by turns with new inputs and lengths."""
    calls = []
    for seed, nq, nk in ((1, [1, 1, 2], [5000, 30, 700]), (2, [90, 1], [200, 3000])):
        b = Batch(cm, nq, nk, 8, 2, 128, torch.bfloat16, E4M3, 32, seed=seed)
        T = sum(nq)
        state = dict(new=torch.randn((2, T, 2, 128), device=DEV).to(torch.bfloat16), rows=torch.cat([r[len(r) - n:] for r, n in zip(b.rows, nq)]), out=torch.zeros_like(b.q),
                     back=torch.zeros((2, T, 2, 128), dtype=torch.bfloat16, device=DEV),
                     ws=torch.empty(max(16, cm.attn_paged_workspace_bytes(len(nq), 8, 2, 128, max(nq), 8192, 2500, 4)), dtype=torch.uint8, device=DEV))

        def run(b=b, s=state, most=max(nq)):
            cm.cache_write(s["new"][0], s["new"][1], s["rows"], b.pages)
            cm.attn_paged(b.q, b.pages, b.table, b.cu, b.k_len, s["out"], most, 8192, True, 0.1, 2500, 4, s["ws"])
            cm.cache_read(b.pages, s["rows"], s["back"][0], s["back"][1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        calls.append((b, state, run, graph))
    for turn in range(3):
        for b, s, run, graph in calls:
            b.q.copy_(torch.randn(b.q.shape, device=DEV))
            s["new"].copy_(torch.randn(s["new"].shape, device=DEV))
            b.k_len.sub_(turn)
            graph.replay()
            torch.cuda.synchronize()
            got = s["out"].clone(), s["back"].clone()
            run()
            assert torch.equal(got[0], s["out"]) and torch.equal(got[1], s["back"]) and bool(got[0].isfinite().all())


@gpu
@pytest.mark.parametrize("fmt", ["elements", "codes"])
@pytest.mark.parametrize("E,nq,nk,Hq,Hk", [(64, [70], [70], 2, 1), (64, [1], [9001], 8, 1), (128, [100], [7001], 8, 1), (128, [300], [300], 40, 8)])
def test_the_largest_and_smallest_scales(cm, fmt, E, nq, nk, Hq, Hk):
    """The largest score alone, but for rows whose two largest are closer than what 32 bits tell apart (2^-24 of sums of 128 products); or all keys alike."""
    b = Batch(cm, nq, nk, Hq, Hk, E, torch.bfloat16, E4M3 if fmt == "codes" else torch.bfloat16, 32, seed=3)
    out = b.run(False, 2.0 ** 127)
    k, v = b.held(0)
    for h in range(0, Hq, 7):
        two = (b.q[:, h].double() @ k[:, h // (Hq // Hk)].double().t()).topk(2, -1)
        clear = two.values[:, 0] - two.values[:, 1] > 1e-3
        assert torch.equal(out[clear, h], v[two.indices[clear, 0], h // (Hq // Hk)]) and bool(clear.any())
    b.check(False, 2.0 ** -140)


@gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 70)])
def test_minus_infinite_scores(cm, window, sinks):
    """A key whose score is minus infinity has no weight, also where it stands in front of all others, and where the window begins."""
    b = Batch(cm, [70, 1], [170, 300], 2, 1, 64, torch.bfloat16, torch.bfloat16, 16, seed=9)
    b.q.abs_().clamp_(min=0.1)
    at = _starts(b.nq)
    for s, n in ((0, 20), (1, 200)):
        kv = b.held(s)
        kv[0, :n, :, 3] = -math.inf
        cm.cache_write(kv[0], kv[1], b.rows[s], b.pages)
    out = b.run(True, 0.1, window, sinks)
    for s, n in ((0, 20), (1, 200)):
        k, v = b.held(s)
        k[:n, :, 3] = 0                                             # (the same without those keys, which are hidden below)
        q = b.q[at[s]:at[s + 1]]
        j, place = torch.arange(b.nk[s], device=DEV), torch.arange(b.nq[s], device=DEV)[:, None] + b.nk[s] - b.nq[s]
        seen = (j <= place) & (j >= n) & ((j > place - window) | (j < sinks) if window else True)
        for h in range(2):
            sc = (q[:, h].double() @ k[:, 0].double().t() * 0.1).masked_fill(~seen, -math.inf)
            w = torch.softmax(sc, 1)
            want, size = w @ v[:, 0].double(), w @ v[:, 0].double().abs()
            off = 2.0 ** -8 * (size + 2 * want.abs()) * 1.02 + 1e-4 * size      # (32-bit scores of 64 products: below 1e-4 here)
            assert bool(((out[at[s]:at[s + 1], h].double() - want).abs() <= off).all())


@gpu
def test_heads_of_rows_and_other_strides(cm):
    """[heads, rows, E] and rows inside wider ones, and an output with gaps that stay; a table with columns behind it."""
    for nq, nk in (([130, 40], [130, 40]), ([1, 3], [300, 77])):
        b = Batch(cm, nq, nk, 4, 2, 128, torch.bfloat16, E4M3, 16, seed=2)
        want, q = b.run(), b.q
        b.q = q.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(b.run(out=torch.empty_like(b.q)), want)
        wide = torch.full((q.shape[0], 6, 136), 3.0, dtype=q.dtype, device=DEV)
        b.run(out=wide[:, 1:5, :128])
        assert torch.equal(wide[:, 1:5, :128], want) and bool((wide[:, [0, 5]] == 3).all()) and bool((wide[..., 128:] == 3).all())
        table = torch.full((2, 100), 2 ** 30, dtype=torch.int32, device=DEV)
        table[:, 7:7 + b.table.shape[1]] = b.table
        b.table = table[:, 7:7 + b.table.shape[1]]
        assert torch.equal(b.run(), want)


@gpu
def test_scales_of_other_writers(cm):
    """Every scale byte with every code: rows come back as the formula has it, 255 as NaN, rounded to the elements' type."""
    pages = make_pages(cm, 16, 16, 4, 64, E4M3)
    pages.k.view(torch.uint8).copy_(torch.arange(256, dtype=torch.uint8, device=DEV).view(4, 64).expand(16, 16, 4, 64))
    pages.k_scales.copy_(torch.arange(256, dtype=torch.uint8, device=DEV).view(16, 16, 1).expand(16, 16, 4))
    for dtype in TYPES:
        out = torch.zeros((2, 256, 4, 64), dtype=dtype, device=DEV)
        cm.cache_read(pages, torch.arange(256, device=DEV), out[0], out[1])
        codes, _, scales, _ = _flat(pages)
        want = of_codes(codes, scales, torch.float32).to(dtype)      # (2^128 is infinite in 32 bits: of byte 255)
        got, want = out[0][:255], want[:255]
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0)) and bool(out[0][255].isnan().all())


def test_the_workspace_of_any_limit_is_bounded(cm):
    """Up to the largest limits, and as many parts as the limits' plan has; without it the call is refused before anything is launched."""
    of, most = cm.attn_paged_workspace_bytes, 2 ** 31 - 1
    for S, Hq, Hk, max_q in ((1, 8, 8, 1), (32, 32, 8, 1), (1, 64, 1, 16), (512, 32, 8, 1), (4096, 32, 8, 1), (2, 8, 8, 1024), (65536, 8, 8, 5), (most, most, most, 1)):
        for max_k in (300, 5001, 131072, 2 ** 24, most):
            for window, sinks in ((0, 0), (1, 0), (4096, 4), (most, most)):
                assert 0 <= of(S, Hq, Hk, 128, max_q, max_k, window, sinks) <= 2 ** 17 * 64 * 130 * 4
    assert of(32, 32, 8, 128, 1, most) >= of(32, 32, 8, 128, 1, 131072) > of(32, 32, 8, 128, 1, 131072, 4096, 4) > 0
    assert of(1, 8, 8, 128, most, most) == 0


@gpu
def test_a_batch_of_none(cm):
    b = Batch(cm, [0, 0], [50, 0], 4, 2, 64, torch.bfloat16, E4M3, 16)
    out = b.run()
    assert bool(out.isnan().all())


# ---- refusals -----------------------------------------------------------------------------------------------------------

def _struct(cm, **at):
    s = cm._PagesStruct(0x1000, 0x2000, 0x3001, 0x4003, 16 * 2 * 64, 2 * 64, 64, 32, 1, 16, 10, 16, 2, 64, 2)
    for name, value in at.items():
        setattr(s, name, value)
    return s


def test_refuses(cm):
    """Before any launch; the addresses are never read."""
    lib, P = cm.load(), ctypes.c_void_p
    a, b, ok = P(0x1000), P(0x1008), ctypes.byref(_struct(cm))
    w = lambda pages=ok, k=a, kt=128, kh=64, v=a, vt=128, vh=64, rows=a, tokens=5, dtype=0: lib.chipmunk_cache_write(k, kt, kh, v, vt, vh, rows, pages, tokens, dtype, None)   # noqa: E731
    r = lambda pages=ok, k=a, kt=128, kh=64, v=a, vt=128, vh=64, rows=a, tokens=5, dtype=0: lib.chipmunk_cache_read(pages, rows, k, kt, kh, v, vt, vh, tokens, dtype, None)    # noqa: E731
    at = lambda pages=ok, q=a, qt=256, qh=64, table=a, row=9, width=9, out=a, ot=256, oh=64, cu=a, k_len=a, S=3, Tq=7, Hq=4, max_q=1, max_k=99, causal=1, window=0, sinks=0, scale=0.1, dtype=0, ws=None, n=0: (   # noqa: E731
        lib.chipmunk_attn_paged(q, qt, qh, pages, table, row, width, out, ot, oh, cu, k_len, S, Tq, Hq, max_q, max_k, causal, window, sinks, scale, dtype, ws, n, None))
    for f in (w, r):
        assert f(None) == f(k=None) == f(v=None) == f(rows=None) == -1
        assert f(tokens=0) == f(kt=100) == f(kh=60) == f(vt=-128) == -2 and f(tokens=2 ** 31 - 1) == -2
        assert f(k=b) == f(v=b) == f(rows=P(0x1004)) == f(kt=132) == f(vh=68, vt=136) == -3 and f(dtype=2) == -4
    for f in (w, r, at):
        for wrong, status in ((dict(k=None), -1), (dict(v=None), -1), (dict(k_scales=None), -1), (dict(v_scales=None), -1), (dict(pages=0), -2), (dict(heads=0), -2), (dict(E=96), -4),
                              (dict(page_size=24), -4), (dict(page_size=8), -4), (dict(page_size=1 << 17), -4), (dict(page_size=0), -2), (dict(format=1), -4), (dict(format=3), -4),
                              (dict(page_size=1 << 16, pages=1 << 15, page_stride=1 << 40, scale_page_stride=1 << 40), -2), (dict(token_stride=64), -2), (dict(head_stride=0), -2),
                              (dict(page_stride=1024), -2), (dict(scale_token_stride=0), -2), (dict(scale_head_stride=8), -2), (dict(k=0x1008), -3), (dict(page_stride=2056), -3),
                              (dict(token_stride=1 << 24, page_stride=1 << 30), -2), (dict(page_stride=1 << 62), -2)):
            assert f(ctypes.byref(_struct(cm, **wrong))) == status, wrong
    assert at(None) == at(q=None) == at(table=None) == at(out=None) == at(cu=None) == at(k_len=None) == -1
    assert at(S=0) == at(Tq=0) == at(Hq=3) == at(Hq=0) == at(max_q=0) == at(max_k=0) == at(width=0) == at(window=-1) == at(sinks=-1) == at(window=5, causal=0) == -2
    assert at(scale=0.0) == at(scale=math.nan) == at(scale=math.inf) == at(scale=2.0 ** 127 * 1.5) == at(qt=32) == at(row=8) == at(oh=32) == at(qt=1 << 24) == -2
    assert at(row=1 << 27, width=(1 << 26) + 1) == -2                     # sequences of more than 2^30 keys
    assert at(q=b) == at(out=b) == at(table=P(0x1001)) == at(cu=P(0x1002)) == at(k_len=P(0x1003)) == at(qt=260) == at(ws=b) == -3
    size = lib.chipmunk_attn_paged_workspace_bytes
    assert size(1, 8, 2, 128, 1, 100000, 0, 0) > 0 and at(S=1, max_k=100000, row=10000, width=10000) == -5
    assert size(0, 8, 2, 128, 1, 100, 0, 0) == size(1, 8, 3, 128, 1, 100, 0, 0) == size(1, 8, 2, 96, 1, 100, 0, 0) == size(1, 8, 2, 128, 0, 100, 0, 0) == size(1, 8, 2, 128, 1, 100, -1, 0) == 0
    assert size(4, 32, 8, 128, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1) < 2 ** 33


def test_functions_refuse(cm):
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)   # noqa: E731
    with pytest.raises(ValueError, match="must live on the GPU"):
        cm.Pages(t(2, 16, 2, 64), t(2, 16, 2, 64))
    with pytest.raises(TypeError, match="bfloat16, float16 or float8"):
        cm.Pages(t(2, 16, 2, 64, dtype=torch.float32), t(2, 16, 2, 64))
    with pytest.raises(ValueError, match="go with float8"):
        cm.Pages(t(2, 16, 2, 64).to(E4M3), t(2, 16, 2, 64).to(E4M3))
    for call in (lambda: cm.cache_write(t(4, 2, 64), t(4, 2, 64), t(4, dtype=torch.int64), None), lambda: cm.cache_read(None, t(4, dtype=torch.int64), t(4, 2, 64), t(4, 2, 64)),
                 lambda: cm.attn_paged(t(4, 2, 64), None, t(1, 4, dtype=torch.int32), t(2, dtype=torch.int32), t(1, dtype=torch.int32), t(4, 2, 64), 4, 4, True, 0.1)):
        with pytest.raises((TypeError, ValueError)):
            call()


@gpu
def test_functions_refuse_on_the_gpu(cm):
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device=DEV)   # noqa: E731
    i32, i64, u8 = (lambda *shape, d=d: t(*shape, dtype=d) for d in (torch.int32, torch.int64, torch.uint8))
    code = lambda *shape: t(*shape).to(E4M3)   # noqa: E731
    for bad, error in (((t(2, 16, 2, 64), t(2, 16, 2, 128)), ValueError), ((t(2, 16, 2, 64), t(2, 2, 16, 64).transpose(1, 2)), ValueError), ((t(2, 16, 2, 64), t(2, 16, 2, 64).half()), TypeError),
                       ((t(2, 16, 2, 64), t(2, 16, 2, 64), u8(2, 16, 2), u8(2, 16, 2)), ValueError), ((code(2, 16, 2, 64), code(2, 16, 2, 64), u8(2, 16, 2)), ValueError),
                       ((code(2, 16, 2, 64), code(2, 16, 2, 64), u8(2, 16, 2), u8(2, 16, 3)), ValueError), ((code(2, 16, 2, 64), code(2, 16, 2, 64), i32(2, 16, 2), u8(2, 16, 2)), TypeError),
                       ((t(16, 2, 64), t(16, 2, 64)), ValueError), ((t(2, 16, 2, 128)[..., ::2], t(2, 16, 2, 128)[..., ::2]), ValueError)):
        with pytest.raises(error):
            cm.Pages(*bad)
    pages = cm.Pages(t(3, 16, 2, 64), t(3, 16, 2, 64))
    good = [t(5, 2, 64), t(5, 2, 64), torch.arange(5, device=DEV), pages]
    cm.cache_write(*good)
    for i, bad, error in ((0, t(5, 3, 64), ValueError), (1, t(5, 2, 64).half(), TypeError), (1, t(4, 2, 64), ValueError), (2, i32(5), TypeError), (2, i64(4), ValueError), (3, None, TypeError),
                          (0, t(5, 2, 128)[..., ::2], ValueError)):
        with pytest.raises(error):
            cm.cache_write(*good[:i], bad, *good[i + 1:])
        with pytest.raises(error):
            other = good[:i] + [bad] + good[i + 1:]
            cm.cache_read(other[3], other[2], other[0], other[1])
    with pytest.raises(cm.ChipmunkError):                                 # elements of another type than the pages'
        cm.cache_write(t(5, 2, 64).half(), t(5, 2, 64).half(), good[2], pages)
    good = [t(4, 4, 64), pages, i32(2, 3), torch.tensor([0, 1, 4], dtype=torch.int32, device=DEV), i32(2), t(4, 4, 64), 3, 48, True, 0.1, 0, 0, None]
    cm.attn_paged(*good)
    for i, bad, error in ((0, t(4, 4, 128), ValueError), (1, None, TypeError), (1, 3, TypeError), (2, i32(3, 3), ValueError), (2, i64(2, 3), TypeError), (3, i32(2), ValueError), (4, i32(3), ValueError),
                          (5, t(3, 4, 64), ValueError), (6, 0, cm.ChipmunkError), (6, 2 ** 40, ValueError), (7, -1, cm.ChipmunkError), (9, 0.0, cm.ChipmunkError), (10, -1, cm.ChipmunkError),
                          (11, 2 ** 33, ValueError), (0, t(4, 3, 64), ValueError), (12, t(4), TypeError)):
        with pytest.raises(error):
            cm.attn_paged(*good[:i], bad, *good[i + 1:])
