"""Attention over packed sequences against its definition in 64 bits, and what it refuses.

Tolerance.  With w_j the weights of a row and A = sum_j w_j |v_j|: a weight is rounded to the element type, by half a step, eps / 2
of its value at most, in the products with v and in their sum alike, so the row moves by eps / 2 (A + |out|); the result is rounded
once, eps / 2 |out|.  A score is a sum of E products in 32 bits that pass E / 8 + 8 roundings at most, and is read off by an
exponential as far from one: together d = 2^-24 ((E / 8 + 10) sum |q k| scale + 2 |score| + 8), which moves the row by 2 d A.  In fp16
a weight below 2^-14 of the largest is rounded in steps of 2^-24, so n_k of them add 2^-25 n_k max |v| at most."""
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


def _starts(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def reference(q, k, v, causal, scale):
    """One sequence: q [n_q, Hq, E], k, v [n_k, Hk, E] -> the result in 64 bits and how far the kernel's may be from it."""
    (nq, Hq, E), (nk, Hk, _) = q.shape, k.shape
    info = torch.finfo(q.dtype)
    out, off = torch.zeros(nq, Hq, E, dtype=torch.float64, device=q.device), torch.zeros(nq, Hq, E, dtype=torch.float64, device=q.device)
    if nk == 0:
        return out, off
    seen = torch.arange(nk, device=q.device) <= (torch.arange(nq, device=q.device)[:, None] + (nk - nq if causal else nk))
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


def _inputs(nq, nk, Hq, Hk, E, dtype, seed, slot=0, scale=1.0, packed=False):
    """q, k, v of the sequences one behind the other, k and v in slots of so many rows; what belongs to no sequence is NaN."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    at_q, at_k = _starts(nq), [i * slot for i in range(len(nk) + 1)] if slot else _starts(nk)
    r = lambda n, H: (torch.randn((max(n, 1), H, E), generator=g, device=DEV) * scale).to(dtype)   # noqa: E731
    if packed:   # side by side, as a projection leaves them
        rows = r(at_q[-1], Hq + 2 * Hk)
        q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:]
    else:
        q, k, v = r(at_q[-1], Hq), r(at_k[-1], Hk), r(at_k[-1], Hk)
    if slot:
        for s, n in enumerate(nk):
            k[at_k[s] + n:at_k[s + 1]] = math.nan
            v[at_k[s] + n:at_k[s + 1]] = math.nan
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)   # noqa: E731
    return q, k, v, i32(at_q), i32(at_k), i32(nk) if slot else None


def _run(cm, q, k, v, cu_q, cu_k, k_len, nq, nk, causal, scale, out=None, max_q=None, max_k=None):
    S, (_, Hq, E), Hk = len(nq), q.shape, k.shape[1]
    max_q, max_k = max_q or max(max(nq), 1), max_k or max(max(nk), 1)
    ws = torch.full((max(16, cm.attn_packed_workspace_bytes(S, Hq, Hk, E, max_q, max_k)),), 255, dtype=torch.uint8, device=DEV)
    if out is None:
        out = torch.full((q.shape[0], Hq, E), math.nan, dtype=q.dtype, device=DEV)
    cm.attn_packed(q, k, v, cu_q, cu_k, out, max_q, max_k, causal, scale, k_len=k_len, ws=ws)
    return out


def _check(cm, nq, nk, Hq, Hk, E, dtype, causal, seed=0, slot=0, scale=None, size=1.0, packed=False, **more):
    scale = scale or 1 / math.sqrt(E)
    q, k, v, cu_q, cu_k, k_len = _inputs(nq, nk, Hq, Hk, E, dtype, seed, slot, size, packed)
    out = _run(cm, q, k, v, cu_q, cu_k, k_len, nq, nk, causal, scale, **more)
    for s, (a, b) in enumerate(zip(nq, nk)):
        q0, k0 = int(cu_q[s]), int(cu_k[s])
        want, off = reference(q[q0:q0 + a], k[k0:k0 + b], v[k0:k0 + b], causal, scale)
        got = out[q0:q0 + a].double()
        assert bool(((got - want).abs() <= off).all()), (s, a, b, float(((got - want).abs() / off.clamp(min=1e-30)).nan_to_num(1e9).max()))
    again = _run(cm, q, k, v, cu_q, cu_k, k_len, nq, nk, causal, scale, **more)
    assert torch.equal(again[:sum(nq)], out[:sum(nq)])                     # no order of anything is left to chance
    return out


PROMPTS = [[1], [2], [63], [64], [65], [127], [128], [129], [191], [192], [193], [300], [1000], [2500], [77, 31, 1, 64, 0, 77, 12, 50], [0, 0, 5, 0],
           [513, 200, 1, 640, 64], [129] * 9, [1] * 130, [700] + [3] * 70 + [400]]


@gpu
@pytest.mark.parametrize("lengths", PROMPTS, ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("E", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_prompts(cm, lengths, E, causal):
    for dtype in TYPES:
        _check(cm, lengths, lengths, 4, 2, E, dtype, causal, seed=len(lengths), packed=True)


@gpu
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (2, 1), (3, 3), (5, 1), (6, 6), (8, 8), (16, 8), (20, 4), (24, 24), (10, 2), (12, 3), (64, 8), (40, 40)])
@pytest.mark.parametrize("causal", [False, True])
def test_heads(cm, Hq, Hk, causal):
    _check(cm, [260, 7, 130], [260, 7, 130], Hq, Hk, 64, torch.bfloat16, causal)
    _check(cm, [1, 1, 2], [260, 7, 130], Hq, Hk, 128, torch.float16, causal)


# one batch for each form that takes whole tiles of queries: rows of a tile / 64 + 1
FORMS = [(64, False, 3, 40, 40, [701, 0, 700, 129, 301, 1, 64, 700]), (64, False, 4, 32, 8, [4003, 1, 0, 70]), (64, True, 2, 40, 40, [130, 60, 0, 1]),
         (64, True, 3, 40, 40, [1201, 701, 1, 1201, 33, 701, 0, 701, 701]), (64, True, 4, 64, 8, [8003, 1, 0, 70]), (128, False, 2, 40, 40, [130, 60, 0, 1]),
         (128, False, 3, 32, 8, [301, 301, 0, 301, 301, 1]), (128, False, 4, 64, 8, [1503, 1, 64, 0]), (128, True, 3, 40, 40, [301, 1, 301, 301, 301, 0]),
         (128, True, 4, 32, 8, [4003, 0, 1, 31])]


def test_the_forms_are_what_the_batches_take(cm):
    form = cm.load().chipmunk_internal_attn_packed_form
    for E, causal, want, Hq, Hk, lengths in FORMS:
        assert form(len(lengths), sum(lengths), Hq, Hk, E, max(lengths), max(lengths), causal) == want


@gpu
@pytest.mark.parametrize("E,causal,form,Hq,Hk,lengths", FORMS)
def test_large_batches(cm, E, causal, form, Hq, Hk, lengths):
    for dtype in TYPES:
        q, k, v, cu_q, cu_k, _ = _inputs(lengths, lengths, Hq, Hk, E, dtype, form, packed=True)
        out = _run(cm, q, k, v, cu_q, cu_k, None, lengths, lengths, causal, E ** -0.5)
        assert not bool(out.isnan().any())
        for s, n in enumerate(lengths):
            rows = slice(int(cu_q[s]), int(cu_q[s]) + n)
            for h in (0, Hq // 2 + 1, Hq - 1):
                g = h // (Hq // Hk)
                want, off = reference(q[rows, h:h + 1], k[rows, g:g + 1], v[rows, g:g + 1], causal, E ** -0.5)
                got = out[rows, h:h + 1].double()
                assert bool(((got - want).abs() <= off).all()), (s, n, h)
        again = _run(cm, q, k, v, cu_q, cu_k, None, lengths, lengths, causal, E ** -0.5)
        assert torch.equal(again, out)


# one long prompt among many short sequences, S, Tq, Hq, Hk, E, max_q: forms that cut every sequence like the longest launch workgroups by the
# million, or more than a launch holds
RAGGED = [(1024, 5119, 128, 8, 128, 4096), (4096, 5119, 64, 8, 64, 1024), (484, 6913, 8, 1, 64, 6430), (1000, 8194, 96, 12, 128, 2639), (447, 5085, 8, 8, 64, 2676),
          (20000, 40000, 64, 8, 128, 20001)]


def test_one_long_sequence_among_many_short_ones_is_not_cut_a_million_times(cm):
    form = cm.load().chipmunk_internal_attn_packed_form
    for S, Tq, Hq, Hk, E, most in RAGGED:
        for causal in (False, True):
            taken = form(S, Tq, Hq, Hk, E, most, most, causal)
            rows = (16, 32, 64, 128, 192)[taken]
            workgroups = S * Hk * -(-most * (Hq // Hk) // rows) if taken < 2 else (S if most <= rows else Tq // rows + S) * Hq
            assert workgroups < 2 ** 24
            # the queries that there are, cut by themselves, and one more tile a sequence and head
            assert workgroups <= 2 * (Tq // 64 + S) * Hq, (S, Tq, Hq, Hk, E, most, taken, workgroups)


@gpu
@pytest.mark.parametrize("S,Hq,Hk,E,most,at", [(1024, 128, 8, 128, 4096, 0), (4096, 64, 8, 64, 1024, 4095), (447, 8, 8, 64, 2676, 200)])
def test_one_long_sequence_among_many_short_ones(cm, S, Hq, Hk, E, most, at):
    lengths = [1] * S
    lengths[at] = most
    q, k, v, cu_q, cu_k, _ = _inputs(lengths, lengths, Hq, Hk, E, torch.bfloat16, S, packed=True)
    out = _run(cm, q, k, v, cu_q, cu_k, None, lengths, lengths, True, E ** -0.5)
    rows = slice(at, at + most)
    for h in (0, Hq - 1):
        g = h // (Hq // Hk)
        want, off = reference(q[rows, h:h + 1], k[rows, g:g + 1], v[rows, g:g + 1], True, E ** -0.5)
        assert bool(((out[rows, h:h + 1].double() - want).abs() <= off).all())
    # a token that sees itself alone takes its value as it is
    alone = torch.ones(out.shape[0], dtype=torch.bool, device=DEV)
    alone[rows] = False
    assert torch.equal(out[alone], v[alone].repeat_interleave(Hq // Hk, 1))


CONTINUED = [([5], [70]), ([1], [1]), ([1], [64]), ([1], [65]), ([1, 1, 1], [1, 4000, 129]), ([17, 3], [200, 3]), ([150], [1000]), ([64, 0, 9], [64, 30, 0]),
             ([300, 2], [100, 1]), ([200], [1]), ([4, 4, 4, 4], [4, 5, 600, 0]), ([1] * 40, list(range(0, 2000, 50))), ([130, 1, 33], [129, 900, 31]), ([8], [5000]), ([1], [9001])]


@gpu
@pytest.mark.parametrize("nq,nk", CONTINUED, ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("slot", [False, True])
def test_more_or_fewer_keys_than_queries(cm, nq, nk, causal, slot):
    """Caches with room, NaN behind what is in use; a causal query that sees no key gets zero."""
    for dtype, (Hq, Hk), E in ((torch.bfloat16, (8, 2), 128), (torch.float16, (4, 4), 64)):
        _check(cm, nq, nk, Hq, Hk, E, dtype, causal, seed=max(nk), slot=max(nk) + 3 if slot else 0)


@gpu
@pytest.mark.parametrize("nq", [1, 2, 3, 5, 8, 16, 17, 40])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 16])
def test_few_queries(cm, nq, G):
    _check(cm, [nq, nq, 1], [700, nq, 2111], 2 * G, 2, 128, torch.bfloat16, True, seed=G, slot=2200)
    _check(cm, [nq, nq, 1], [700, nq, 2111], 2 * G, 2, 64, torch.float16, True, seed=G)


# more than 32 rows of a key head over keys in parts, whose blocks of 16 rows and tiles of 64 go to the workspace and are joined: nq, nk, Hq, Hk
DIVIDED = [([40, 17], [6000, 5100], 16, 2), ([100], [7001], 8, 1), ([64, 0, 3], [5003, 4790, 4800], 32, 2), ([5, 200], [3000, 5900], 5, 1), ([33], [4097], 1, 1), ([9, 9, 1], [4400, 8, 4000], 16, 4)]
FAR = [(8, 1, 200000), (3, 3, 140001)]   # one token over more than 64 parts: Hq, Hk, n_k


def test_the_batches_are_divided(cm):
    form = cm.load().chipmunk_internal_attn_packed_form
    for nq, nk, Hq, Hk in DIVIDED:
        keys = form(len(nq), sum(nq), Hq, Hk, 128, max(nq), max(nk), 1)
        assert 32 < max(nq) * (Hq // Hk) <= 1024 and 256 <= keys < max(nk)
    assert all(form(1, 1, Hq, Hk, 128, 1, nk, 1) >= 256 and -(-nk // form(1, 1, Hq, Hk, 128, 1, nk, 1)) > 64 for Hq, Hk, nk in FAR)


@gpu
@pytest.mark.parametrize("nq,nk,Hq,Hk", DIVIDED)
@pytest.mark.parametrize("causal", [False, True])
def test_many_rows_over_divided_keys(cm, nq, nk, Hq, Hk, causal):
    for dtype, E in ((torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 64), (torch.float16, 128)):
        for slot in (0, max(nk) + 3):
            _check(cm, nq, nk, Hq, Hk, E, dtype, causal, seed=E + max(nq), slot=slot)


@gpu
@pytest.mark.parametrize("Hq,Hk,nk", FAR)
@pytest.mark.parametrize("sign", [-1.0, 0.0, 1.0])
def test_a_token_over_more_than_64_parts(cm, Hq, Hk, nk, sign):
    """Scores that rise or fall from the first part to the last, so that a later round of the joining raises what it holds, or does not."""
    for dtype, E in ((torch.bfloat16, 128), (torch.float16, 64)):
        q, k, v, cu_q, cu_k, _ = _inputs([1], [nk], Hq, Hk, E, dtype, 11)
        q.fill_(0.5)
        k.copy_((k.float() * 0.1 + sign * torch.linspace(-10, 10, nk, device=DEV)[:, None, None] / math.sqrt(E)).to(dtype))
        out = _run(cm, q, k, v, cu_q, cu_k, None, [1], [nk], True, 1 / math.sqrt(E))
        want, off = reference(q, k, v, True, 1 / math.sqrt(E))
        assert bool(((out.double() - want).abs() <= off).all())


@gpu
@pytest.mark.parametrize("nq,nk,Hq,Hk", [([5], [6000], 4, 2), ([1, 2], [200000, 300], 8, 1), ([100], [7000], 8, 1), ([40, 17], [6000, 5100], 16, 2)])
@pytest.mark.parametrize("kind", [math.nan, math.inf, -math.inf])
def test_hidden_keys_of_divided_sequences(cm, nq, nk, Hq, Hk, kind):
    """As test_hidden_keys_have_no_influence, with the key in the first, a middle or the last part."""
    for dtype, E in ((torch.bfloat16, 128), (torch.float16, 64)):
        q, k, v, cu_q, cu_k, _ = _inputs(nq, nk, Hq, Hk, E, dtype, 6)
        clean = _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1)
        for at in (3, nk[0] // 2, nk[0] - nq[0] // 2 - 1):
            sees = (torch.arange(nq[0], device=DEV) + nk[0] - nq[0]) >= at
            for spoiled in (k, v):
                before = spoiled[at].clone()
                spoiled[at, :, 5] = kind
                out = _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1)
                spoiled[at] = before
                assert torch.equal(out[:nq[0]][~sees], clean[:nq[0]][~sees]) and torch.equal(out[nq[0]:], clean[nq[0]:])
                if spoiled is v:
                    others = [e for e in range(E) if e != 5]
                    assert torch.equal(out[..., others], clean[..., others])
                    seen = out[:nq[0]][sees][..., 5]
                    assert bool(seen.isnan().all() if math.isnan(kind) else (seen == kind).all())
                elif math.isnan(kind):
                    assert bool(out[:nq[0]][sees].isnan().all())


@gpu
@pytest.mark.parametrize("scale,size", [(3.0, 1.0), (1e-4, 1.0), (0.125, 30.0), (1.0, 0.01)])
@pytest.mark.parametrize("E", [64, 128])
def test_peaked_and_flat_rows(cm, scale, size, E):
    """Scores into the hundreds, where one key has all the weight, and rows of equal weights."""
    for dtype in TYPES:
        _check(cm, [400, 1], [400, 1500], 2, 1, E, dtype, True, scale=scale, size=size)


@gpu
@pytest.mark.parametrize("E", [64, 128])
@pytest.mark.parametrize("nq,nk", [([500, 300], [500, 300]), ([1, 1], [900, 300]), ([6, 3], [900, 300])])
def test_rising_and_falling_scores(cm, E, nq, nk):
    """The largest score last: the reference rises with every tile; first: it never does.  Far below zero all of them."""
    for sign in (1.0, -1.0):
        for shift in (0.0, -40.0):
            q, k, v, cu_q, cu_k, _ = _inputs(nq, nk, 2, 2, E, torch.bfloat16, 3)
            q.fill_(0.5)
            ramp = torch.cat([torch.linspace(0, 20, n) for n in nk]).to(DEV)
            k.copy_((k.float() * 0.01 + sign * ramp[:, None, None] * 0.1 + shift).to(k.dtype))
            out = _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.25)
            for s in range(2):
                a, b = slice(int(cu_q[s]), int(cu_q[s + 1])), slice(int(cu_k[s]), int(cu_k[s + 1]))
                want, off = reference(q[a], k[b], v[b], True, 0.25)
                assert bool(((out[a].double() - want).abs() <= off).all())


@gpu
@pytest.mark.parametrize("nq,nk,at", [([200], [200], 150), ([200], [200], 64), ([300], [300], 0), ([5], [400], 397), ([1], [400], 399), ([3, 9], [100, 100], 98), ([64], [64], 63)])
@pytest.mark.parametrize("kind", [math.nan, math.inf, -math.inf])
def test_hidden_keys_have_no_influence(cm, nq, nk, at, kind):
    """A key and value that hold an infinity or a NaN reach the queries that see them and no other."""
    for dtype, E in ((torch.bfloat16, 128), (torch.float16, 64)):
        q, k, v, cu_q, cu_k, _ = _inputs(nq, nk, 4, 2, E, dtype, 5)
        clean = _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1)
        row = int(cu_k[0]) + at
        sees = (torch.arange(nq[0], device=DEV) + nk[0] - nq[0]) >= at
        for spoiled in (k, v):
            before = spoiled[row].clone()
            spoiled[row, :, 5] = kind
            out = _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1)
            spoiled[row] = before
            assert torch.equal(out[:nq[0]][~sees], clean[:nq[0]][~sees]) and torch.equal(out[nq[0]:], clean[nq[0]:])
            if spoiled is v:
                others = [e for e in range(E) if e != 5]
                assert torch.equal(out[..., others], clean[..., others])
                seen = out[:nq[0]][sees][..., 5]
                assert bool(seen.isnan().all() if math.isnan(kind) else (seen == kind).all())
            elif math.isnan(kind):
                assert bool(out[:nq[0]][sees].isnan().all())


@gpu
def test_minus_infinite_scores(cm):
    """A key whose score is minus infinity has no weight, also where it stands in front of all others."""
    q, k, v, cu_q, cu_k, _ = _inputs([70, 1], [70, 300], 2, 1, 64, torch.bfloat16, 9)
    q.abs_().clamp_(min=0.1)
    for s, n in ((0, 20), (1, 200)):
        k[int(cu_k[s]):int(cu_k[s]) + n, :, 3] = -math.inf
    out = _run(cm, q, k, v, cu_q, cu_k, None, [70, 1], [70, 300], False, 0.1)
    for s, n in ((0, 20), (1, 200)):
        a, b = slice(int(cu_q[s]), int(cu_q[s + 1])), slice(int(cu_k[s]) + n, int(cu_k[s + 1]))
        want, off = reference(q[a], k[b], v[b], False, 0.1)
        assert bool(((out[a].double() - want).abs() <= off).all())


@gpu
def test_rows_of_no_sequence_stay(cm):
    nq, nk = [30, 70], [30, 70]
    q, k, v, cu_q, cu_k, _ = _inputs(nq, nk, 2, 2, 64, torch.bfloat16, 1)
    grown = [torch.cat([t[:9], t, t[:40]]) for t in (q, k, v)]
    out = torch.full_like(grown[0], 7.0)
    _run(cm, *grown, cu_q + 9, cu_k + 9, None, nq, nk, True, 0.1, out=out)
    assert bool((out[:9] == 7).all()) and bool((out[109:] == 7).all())
    assert torch.equal(out[9:109], _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1))


@gpu
def test_longer_limits_than_needed(cm):
    """max_q and max_k are upper limits: another limit is another way to divide the work, within the tolerance of either."""
    for nq, nk in (([3, 1], [500, 2000]), ([100, 60], [100, 60])):
        for more in (1, 10, 100):
            _check(cm, nq, nk, 4, 2, 64, torch.float16, True, max_q=max(nq) * more, max_k=max(nk) * more)


def test_the_workspace_of_any_limit_is_bounded(cm):
    """Up to the largest limits, and as many parts as the limits' plan has; without it the call is refused before anything is launched."""
    of = cm.attn_packed_workspace_bytes
    for S, Hq, Hk, max_q in ((1, 8, 8, 1), (32, 32, 8, 1), (1, 64, 1, 16), (512, 32, 8, 1), (4096, 32, 8, 1), (2, 8, 8, 1024), (65536, 8, 8, 5), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 1)):
        for max_k in (5001, 131072, 2 ** 24, 2 ** 31 - 1):
            assert 0 <= of(S, Hq, Hk, 128, max_q, max_k) <= 2 ** 17 * 64 * 130 * 4
    assert of(32, 32, 8, 128, 1, 2 ** 31 - 1) >= of(32, 32, 8, 128, 1, 131072) > 0
    assert of(1, 8, 8, 128, 2 ** 31 - 1, 2 ** 31 - 1) == 0
    a = ctypes.c_void_p(0x1000)
    for max_k in (20000, 2 ** 31 - 1):
        assert cm.load().chipmunk_attn_packed(a, 4096, 128, a, 1024, 128, a, 1024, 128, a, 4096, 128, a, a, a, 32, 32, 640000, 32, 8, 128, 1, max_k, 1, 0.1, 0, None, 0, None) == -5


@gpu
@pytest.mark.parametrize("nq,nk,Hq,Hk", [([1] * 31 + [2], [1, 0, 70] + [900] * 28 + [4100], 32, 8), ([1], [9001], 8, 1), ([40, 17], [6000, 5100], 16, 2), ([100, 60], [100, 60], 4, 2)])
def test_limits_far_above_the_lengths(cm, nq, nk, Hq, Hk):
    for max_q, max_k in ((None, 2 ** 31 - 1), (None, 2 ** 22), (2 ** 31 - 1, 2 ** 31 - 1)):
        _check(cm, nq, nk, Hq, Hk, 128, torch.bfloat16, True, seed=len(nq), max_q=max_q, max_k=max_k)


@gpu
def test_heads_of_rows_and_other_strides(cm):
    """[heads, rows, E] and rows inside wider ones, and an output with gaps that stay."""
    for nq, nk in (([130, 40], [130, 40]), ([1, 3], [300, 77])):
        q, k, v, cu_q, cu_k, _ = _inputs(nq, nk, 4, 2, 128, torch.bfloat16, 2)
        want = _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1)
        by_head = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
        assert torch.equal(_run(cm, *by_head, cu_q, cu_k, None, nq, nk, True, 0.1, out=torch.empty_like(by_head[0])), want)
        wide = torch.full((q.shape[0], 6, 136), 3.0, dtype=q.dtype, device=DEV)
        _run(cm, q, k, v, cu_q, cu_k, None, nq, nk, True, 0.1, out=wide[:, 1:5, :128])
        assert torch.equal(wide[:, 1:5, :128], want) and bool((wide[:, [0, 5]] == 3).all()) and bool((wide[..., 128:] == 3).all())


@gpu
@pytest.mark.parametrize("nq", [1, 70])
def test_offsets_beyond_32_bits(cm, nq):
    """A head whose keys span more than 2^32 bytes."""
    E, nk, stride = 64, 2300, 1 << 20
    rows = torch.zeros((nk * stride + 4 * E,), dtype=torch.bfloat16, device=DEV)
    q, k, v, cu_q, cu_k, _ = _inputs([nq], [nk], 2, 1, E, torch.bfloat16, 4)
    far_k, far_v = (rows[i * E:].as_strided((nk, 1, E), (stride, E, 1)) for i in range(2))
    far_k.copy_(k)
    far_v.copy_(v)
    assert torch.equal(_run(cm, q, far_k, far_v, cu_q, cu_k, None, [nq], [nk], True, 0.1), _run(cm, q, k, v, cu_q, cu_k, None, [nq], [nk], True, 0.1))


@gpu
def test_on_another_stream_and_in_graphs(cm):
    """Two captured graphs with a workspace each, replayed by turns."""
    calls = []
    for nq, nk in (([1, 2, 1], [3000, 900, 20]), ([1, 1], [50, 2500])):
        q, k, v, cu_q, cu_k, _ = _inputs(nq, nk, 8, 2, 128, torch.bfloat16, len(nq))
        ws = torch.empty(max(16, cm.attn_packed_workspace_bytes(len(nq), 8, 2, 128, 2, 3000)), dtype=torch.uint8, device=DEV)
        calls.append((q, k, v, cu_q, cu_k, torch.zeros_like(q), ws))
    graphs = []
    for q, k, v, cu_q, cu_k, out, ws in calls:
        cm.attn_packed(q, k, v, cu_q, cu_k, out, 2, 3000, True, 0.1, ws=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cm.attn_packed(q, k, v, cu_q, cu_k, out, 2, 3000, True, 0.1, ws=ws)
        graphs.append(graph)
    for turn in range(3):
        for (q, k, v, cu_q, cu_k, out, ws), graph in zip(calls, graphs):
            k.mul_(0.9)
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for q, k, v, cu_q, cu_k, out, ws in calls:
            want, side = torch.empty_like(out), torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                cm.attn_packed(q, k, v, cu_q, cu_k, want, 2, 3000, True, 0.1, ws=torch.empty_like(ws))
            side.synchronize()
            assert torch.equal(out, want)


@gpu
def test_bad_starts_stay_inside(cm):
    """Entries outside the tensors, and descending ones: some result, and nothing outside the tensors is read or written."""
    q, k, v, cu_q, cu_k, _ = _inputs([40, 40], [40, 40], 2, 1, 64, torch.bfloat16, 1)
    frame = torch.full((120, 2, 64), 5.0, dtype=q.dtype, device=DEV)
    for bad in ([-7, 30, 90], [50, 20, 10], [0, 2 ** 31 - 1, -2 ** 31], [79, 80, 81]):
        starts = torch.tensor(bad, dtype=torch.int32, device=DEV)
        for lens in (None, torch.tensor([1000, -3], dtype=torch.int32, device=DEV)):
            cm.attn_packed(q, k, v, starts, starts, frame[20:100], 80, 80, True, 0.1, k_len=lens)
            cm.attn_packed(q, k, v, starts, starts, frame[20:100], 1, 80, True, 0.1, k_len=lens, ws=torch.empty(1 << 20, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert bool((frame[:20] == 5).all()) and bool((frame[100:] == 5).all())


@gpu
def test_the_largest_and_smallest_scales(cm):
    """The largest score alone, or all keys alike."""
    q, k, v, cu_q, cu_k, _ = _inputs([70], [70], 2, 1, 64, torch.bfloat16, 2)
    scores = (q.double().transpose(0, 1) @ k.double().permute(1, 2, 0))
    first = scores.argmax(-1)                                                        # [heads, queries]
    out = _run(cm, q, k, v, cu_q, cu_k, None, [70], [70], False, 2.0 ** 127)
    assert torch.equal(out, v[:, 0][first].transpose(0, 1))
    out = _run(cm, q, k, v, cu_q, cu_k, None, [70], [70], False, 2.0 ** -140)
    want, off = reference(q, k, v, False, 2.0 ** -140)
    assert bool(((out.double() - want).abs() <= off).all())


@gpu
@pytest.mark.parametrize("n,nk,Hq,Hk", [(130, 130, 40, 40), (1, 9001, 8, 1), (100, 7001, 8, 1), (1503, 1503, 64, 8)])
def test_the_largest_scale_in_every_form(cm, n, nk, Hq, Hk):
    """The largest score alone, but for rows whose two largest are closer than what 32 bits tell apart (2^-24 of sums of 64 products)."""
    q, k, v, cu_q, cu_k, _ = _inputs([n], [nk], Hq, Hk, 64, torch.bfloat16, 3)
    out = _run(cm, q, k, v, cu_q, cu_k, None, [n], [nk], False, 2.0 ** 127)
    for h in range(0, Hq, 7):
        two = (q[:, h].double() @ k[:, h // (Hq // Hk)].double().t()).topk(2, -1)
        clear = two.values[:, 0] - two.values[:, 1] > 1e-3
        assert torch.equal(out[clear, h], v[two.indices[clear, 0], h // (Hq // Hk)]) and bool(clear.any())


# ---- refusals (no GPU) ------------------------------------------------------------------------------------------------------

def test_refuses_a_scale_that_overflows(cm):
    a = ctypes.c_void_p(0x1000)
    for scale in (2.0 ** 128 / 1.44, 3.4e38):
        assert cm.load().chipmunk_attn_packed(a, 512, 64, a, 256, 64, a, 256, 64, a, 512, 64, a, a, None, 2, 100, 100, 8, 4, 64, 100, 100, 1, scale, 0, a, 1 << 30, None) == -2


def test_refuses(cm):
    f, a = cm.load().chipmunk_attn_packed, ctypes.c_void_p(0x1000)

    def call(q=a, qt=512, qh=64, k=a, kt=256, kh=64, v=a, vt=256, vh=64, out=a, ot=512, oh=64, cu_q=a, cu_k=a, k_len=a, S=2, Tq=100, Tk=100, Hq=8, Hk=4, E=64,
             max_q=100, max_k=100, causal=1, scale=0.1, dtype=0, ws=a, ws_bytes=1 << 30):
        return f(q, qt, qh, k, kt, kh, v, vt, vh, out, ot, oh, cu_q, cu_k, k_len, S, Tq, Tk, Hq, Hk, E, max_q, max_k, causal, scale, dtype, ws, ws_bytes, None)
    for missing in ("q", "k", "v", "out", "cu_q", "cu_k"):
        assert call(**{missing: None}) == -1
    for wrong in (dict(S=0), dict(Tq=0), dict(Tk=0), dict(Hq=0), dict(Hk=0), dict(Hq=9), dict(Hq=2), dict(max_q=0), dict(max_k=-1), dict(scale=0.0), dict(scale=-1.0),
                  dict(scale=math.nan), dict(scale=math.inf), dict(qt=56), dict(kt=0), dict(vt=-256), dict(ot=1 << 24), dict(kt=1 << 24), dict(qh=56), dict(vh=0),
                  dict(S=1 << 22, Hq=64, qt=4096, ot=4096, max_q=1 << 20, Tq=1 << 30)):
        assert call(**wrong) == -2, wrong
    for wrong in (dict(E=96), dict(E=256), dict(dtype=2), dict(dtype=-1)):
        assert call(**wrong) == -4, wrong
    for wrong in (dict(q=ctypes.c_void_p(0x1008)), dict(k=ctypes.c_void_p(0x1004)), dict(v=ctypes.c_void_p(0x1002)), dict(out=ctypes.c_void_p(0x1008)),
                  dict(cu_q=ctypes.c_void_p(0x1002)), dict(k_len=ctypes.c_void_p(0x1001)), dict(qt=516), dict(oh=68), dict(kh=68)):
        assert call(**wrong) == -3, wrong


def test_function_refuses(cm):
    bf, i32 = torch.bfloat16, torch.int32
    q, k, cu = torch.zeros(4, 2, 64, dtype=bf), torch.zeros(4, 1, 64, dtype=bf), torch.zeros(2, dtype=i32)
    for args, error in (((q.float(), k, k, cu, cu, q, 4, 4, True, 0.1), TypeError), ((q, k, k, cu, cu, q, 4, 4, True, 0.1), ValueError), ((q, k.half(), k, cu, cu, q, 4, 4, True, 0.1), (TypeError, ValueError))):
        with pytest.raises(error):
            cm.attn_packed(*args)


@gpu
def test_function_refuses_on_the_gpu(cm):
    bf, i32 = torch.bfloat16, torch.int32
    q, k, cu = torch.zeros(4, 2, 64, dtype=bf, device=DEV), torch.zeros(4, 1, 64, dtype=bf, device=DEV), torch.tensor([0, 4], dtype=i32, device=DEV)
    wrong = [(q, k.half(), k, cu, cu, q), (q, k, k[:3], cu, cu, q), (q, k[..., :32], k[..., :32], cu, cu, q), (q, k, k, cu.long(), cu, q), (q, k, k, cu, cu[:1], q),
             (q, k, k, cu, cu, q[:3]), (q[0], k, k, cu, cu, q), (q, k, k, cu.cpu(), cu, q), (q, k, k, cu, cu, q.half()), (q[..., ::2], k, k, cu, cu, q)]
    for args in wrong:
        with pytest.raises((TypeError, ValueError)):
            cm.attn_packed(*args, 4, 4, True, 0.1)
    with pytest.raises((TypeError, ValueError)):
        cm.attn_packed(q, k, k, cu, cu, torch.empty_like(q), 4, 4, True, 0.1, k_len=cu)
    for scale in (0.0, math.nan):
        with pytest.raises(cm.ChipmunkError):
            cm.attn_packed(q, k, k, cu, cu, torch.empty_like(q), 4, 4, True, scale)
