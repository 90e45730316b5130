"""The projections, normed queries and keys, paged caches and attention over them together, as stack.PagedAttentionLayer runs them: prompts of
different lengths, then chunks and single tokens over the pages, each stage against its definition in 64 bits on what the stage before left;
and the whole step captured and replayed."""
import math

import pytest
import torch

from test_attn_packed import _starts
from test_norm_rope import norm_rope_reference
from test_paged import E4M3, in_codes, of_codes
from test_paged import reference as attention_reference
from test_projections import linear_reference

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _layer(dtype, D, heads, kv_heads, E, fmt, page, count, **more):
    import paper_2506_03275_amd as cm
    from paper_2506_03275_amd import stack
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    r = lambda *shape, scale=1.0: (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)   # noqa: E731
    rows = (heads + 2 * kv_heads) * E
    axes = (E // 8, E // 8, E // 4)
    pages = stack.empty_pages(count, page, kv_heads, E, fmt)
    for t in (pages.k, pages.v):
        t.view(torch.uint8).fill_(0xff)    # NaN: what no token has reached must not matter
    return stack.PagedAttentionLayer(r(rows, D, scale=1 / math.sqrt(D)), r(rows, scale=0.1), r(D, heads * E, scale=1 / math.sqrt(heads * E)), None, heads, 1 + r(E, scale=0.2),
                                     1 + r(E, scale=0.2), cm.rope_frequencies(axes), axes, pages, **more), r


class Sequences:
    """Pages given out as the sequences grow."""

    def __init__(self, layer, S, most):
        self.page, self.free, self.held, self.most = layer.pages.k.shape[1], list(range(layer.pages.k.shape[0] - 1, -1, -1)), [0] * S, most
        self.table = torch.full((S, -(-most // self.page)), -1, dtype=torch.int32, device=DEV)

    def grow(self, new, padding=0):
        """cu_q, rows, k_len, table of a step that brings so many new tokens to each."""
        rows = []
        for s, n in enumerate(new):
            for i in range(self.held[s], self.held[s] + n):
                if i % self.page == 0:
                    self.table[s, i // self.page] = self.free.pop()
                rows.append(int(self.table[s, i // self.page]) * self.page + i % self.page)
            self.held[s] += n
        t = lambda x, dtype: torch.tensor(x, dtype=dtype, device=DEV)   # noqa: E731
        return t(_starts(new), torch.int32), t(rows + [-1] * padding, torch.int64), t(self.held, torch.int32), self.table

    def rows(self, s):
        i = torch.arange(self.held[s], device=DEV)
        return self.table[s, i // self.page].long() * self.page + i % self.page


def _close(got, want, off):
    return bool(((got.double() - want).abs() <= off).all())


@pytest.mark.parametrize("dtype,D,heads,kv_heads,E,fmt,page,more", [
    (torch.bfloat16, 256, 8, 2, 64, E4M3, 16, dict(halves=True)), (torch.float16, 384, 3, 3, 128, torch.float16, 64, dict(causal=False)),
    (torch.bfloat16, 512, 4, 1, 128, E4M3, 32, dict(window=50, sinks=4)), (torch.float16, 256, 4, 2, 64, E4M3, 32, dict(window=33))])
def test_prompts_then_tokens(dtype, D, heads, kv_heads, E, fmt, page, more):
    import paper_2506_03275_amd as cm
    prompts = [70, 0, 1, 133, 64]
    layer, r = _layer(dtype, D, heads, kv_heads, E, fmt, page, 60, **more)
    sequences = Sequences(layer, len(prompts), 200)
    for new in (prompts, [1, 1, 1, 1, 0], [1, 40, 1, 0, 9], [1] * 5):
        tokens = sum(new)
        x = r(tokens, D)
        pos = torch.randint(0, 60, (tokens, 3), dtype=torch.int32, device=DEV)
        cu, rows, k_len, table = sequences.grow(new)
        buffers = layer.buffers(tokens, len(new), max(new), 200)
        out = layer.step(x, pos, cu, rows, k_len, table, buffers)
        # the projections, by the operator alone and then by definition
        plain = torch.empty_like(buffers["qkv"])
        cm.linear(x, layer.w_qkv, layer.b_qkv, None, plain.view(tokens, -1))
        want, off = linear_reference(x, layer.w_qkv, layer.b_qkv, None, cm.ACT_NONE)
        assert _close(plain.view(tokens, -1), want, off)
        want, off = norm_rope_reference(plain[:, :heads + kv_heads], layer.q_norm, layer.k_norm, heads, pos, layer.freqs, layer.axes, layer.eps, layer.halves)
        qkv = buffers["qkv"]
        assert _close(qkv[:, :heads + kv_heads], want, off) and torch.equal(qkv[:, heads + kv_heads:], plain[:, heads + kv_heads:])
        # the new tokens' rows of the pages
        back = torch.empty((2, tokens, kv_heads, E), dtype=dtype, device=DEV)
        cm.cache_read(layer.pages, rows, back[0], back[1])
        for got, values in zip(back, (qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:])):
            assert torch.equal(got, of_codes(*in_codes(values), dtype) if fmt == E4M3 else values)
        for s, n in enumerate(new):
            a, mine = slice(int(cu[s]), int(cu[s + 1])), sequences.rows(s)
            kv = torch.empty((2, len(mine), kv_heads, E), dtype=dtype, device=DEV)
            if len(mine):
                cm.cache_read(layer.pages, mine, kv[0], kv[1])
            want, off = attention_reference(qkv[a, :heads], kv[0], kv[1], layer.causal, layer.scale, layer.window, layer.sinks)
            assert _close(buffers["att"][a], want, off)
        want, off = linear_reference(buffers["att"].view(tokens, -1), layer.w_out, None, x, cm.ACT_NONE)
        assert _close(out, want, off)


def test_captured_steps():
    """Two captured steps of different sequences, each with buffers of its own, replayed by turns with new inputs."""
    D, heads, kv_heads, E = 256, 8, 2, 64
    layer, r = _layer(torch.bfloat16, D, heads, kv_heads, E, E4M3, 32, 70)
    sequences = Sequences(layer, 3, 1600)
    layer.step(r(1807, D), torch.zeros((1807, 3), dtype=torch.int32, device=DEV), *sequences.grow([1500, 300, 7]), layer.buffers(1807, 3, 1500, 1600))
    calls = []
    for new in ([1, 1, 1], [0, 2, 1]):
        n = sum(new)
        x, pos = r(n, D), torch.randint(0, 50, (n, 3), dtype=torch.int32, device=DEV)
        cu, rows, k_len, table = sequences.grow(new)
        calls.append([x, pos, cu, rows, k_len, table.clone(), layer.buffers(n, 3, 2, 1600)])
    graphs = []
    for call in calls:
        layer.step(*call)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.step(*call)
        graphs.append(graph)
    for turn in range(3):
        for call, graph in zip(calls, graphs):
            call[0].copy_(r(*call[0].shape))
            call[-1]["out"].zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = call[-1]["out"].clone()
            assert torch.equal(layer.step(*call[:-1], layer.buffers(call[0].shape[0], 3, 2, 1600)), got) and bool(got.isfinite().all())


@pytest.mark.parametrize("fmt", [E4M3, torch.bfloat16])
def test_a_padded_batch(fmt):
    """Tokens behind the last sequence, whatever they hold, change nothing of the others, nor of the pages."""
    D, heads, kv_heads, E, real, padded = 256, 4, 2, 64, 71, 96
    layer, r = _layer(torch.bfloat16, D, heads, kv_heads, E, fmt, 16, 20)
    cu, rows, k_len, table = Sequences(layer, 3, 64).grow([40, 0, 31], padded - real)
    x, pos = r(padded, D), torch.randint(0, 50, (padded, 3), dtype=torch.int32, device=DEV)
    results = []
    for fill in (0.0, 5.0, math.nan):
        layer.pages.k.view(torch.uint8).fill_(0xff)
        layer.pages.v.view(torch.uint8).fill_(0xff)
        x[real:] = fill
        buffers = layer.buffers(padded, 3, 64, 64)
        buffers["att"].fill_(math.nan)
        results.append((layer.step(x, pos, cu, rows, k_len, table, buffers)[:real].clone(), layer.pages.k.view(torch.uint8).clone()))
    assert bool(results[0][0].isfinite().all()) and all(torch.equal(a[0], results[0][0]) and torch.equal(a[1], results[0][1]) for a in results[1:])
