"""The projections, rotary positions and packed attention together, as stack.AttentionLayer runs them: prompts of different lengths,
then single tokens over the caches, each stage against its definition in 64 bits on what the stage before left; and the whole step
captured and replayed."""
import math

import pytest
import torch

from test_attn_packed import reference as attention_reference
from test_projections import linear_reference, rope_reference

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _layer(dtype, D, heads, kv_heads, E, slots, slot_tokens, causal, halves=False):
    import paper_2506_03275_amd as cm
    from paper_2506_03275_amd import stack
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    r = lambda *shape, scale=1.0: (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)   # noqa: E731
    rows = (heads + 2 * kv_heads) * E
    axes = (E // 8, E // 8, E // 4)
    return stack.AttentionLayer(r(rows, D, scale=1 / math.sqrt(D)), r(rows, scale=0.1), r(D, heads * E, scale=1 / math.sqrt(heads * E)), None, heads, kv_heads,
                                cm.rope_frequencies(axes), axes, slots, slot_tokens, causal, halves), r


def _batch(new, held, slot_tokens):
    """cu_q, rows, k_len of slots that get so many new tokens behind those that they hold."""
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    rows = [s * slot_tokens + held[s] + i for s in range(len(new)) for i in range(new[s])]
    t = lambda x, dtype: torch.tensor(x, dtype=dtype, device=DEV)   # noqa: E731
    return t(cu, torch.int32), t(rows, torch.int64), t([a + b for a, b in zip(new, held)], torch.int32)


def _close(got, want, off):
    return bool(((got.double() - want).abs() <= off).all())


@pytest.mark.parametrize("dtype,D,heads,kv_heads,E,causal,halves", [(torch.bfloat16, 256, 8, 2, 64, True, True), (torch.float16, 384, 3, 3, 128, False, False),
                                                                   (torch.bfloat16, 512, 4, 1, 128, True, False)])
def test_prompts_then_tokens(dtype, D, heads, kv_heads, E, causal, halves):
    import paper_2506_03275_amd as cm
    prompts, slot = [70, 0, 1, 133, 64], 200
    layer, r = _layer(dtype, D, heads, kv_heads, E, len(prompts), slot, causal, halves)
    layer.k_cache.fill_(math.nan)      # what no token has reached must not matter
    layer.v_cache.fill_(math.nan)
    held = [0] * len(prompts)
    for new in (prompts, [1, 1, 1, 1, 0], [1, 5, 1, 0, 1], [1] * 5):
        tokens = sum(new)
        x = r(tokens, D)
        pos = torch.randint(0, 60, (tokens, 3), dtype=torch.int32, device=DEV)
        cu, rows, k_len = _batch(new, held, slot)
        buffers = layer.buffers(tokens, max(new), slot)
        out = layer.step(x, pos, cu, rows, k_len, buffers)
        held = [a + b for a, b in zip(new, held)]
        # the projections as the caches and the queries' buffer hold them, by the operator alone and then by definition
        plain = torch.empty_like(buffers["qkv"])
        cm.linear(x, layer.w_qkv, layer.b_qkv, None, plain.view(tokens, -1))
        want, off = linear_reference(x, layer.w_qkv, layer.b_qkv, None, cm.ACT_NONE)
        assert _close(plain.view(tokens, -1), want, off)
        turned, off = rope_reference(plain[:, :heads + kv_heads], pos, layer.freqs, layer.axes, halves, False)
        qkv = buffers["qkv"]
        assert _close(qkv[:, :heads + kv_heads], turned, off) and torch.equal(qkv[:, heads + kv_heads:], plain[:, heads + kv_heads:])
        assert torch.equal(layer.k_cache[rows], qkv[:, heads:heads + kv_heads]) and torch.equal(layer.v_cache[rows], qkv[:, heads + kv_heads:])
        for s, n in enumerate(new):
            a, b = slice(int(cu[s]), int(cu[s + 1])), slice(s * slot, s * slot + held[s])
            want, off = attention_reference(qkv[a, :heads], layer.k_cache[b], layer.v_cache[b], causal, layer.scale)
            assert _close(buffers["att"][a], want, off)
        want, off = linear_reference(buffers["att"].view(tokens, -1), layer.w_out, None, x, cm.ACT_NONE)
        assert _close(out, want, off)


def test_tokens_are_what_a_prompt_is():
    """A sequence in one step and the same one token by token: the same keys and values, and results within what either may be off."""
    D, heads, kv_heads, E, n = 256, 4, 2, 64, 40
    layer, r = _layer(torch.float16, D, heads, kv_heads, E, 2, 64, True)
    x, pos = r(n, D), torch.randint(0, 50, (n, 3), dtype=torch.int32, device=DEV)
    cu, rows, k_len = _batch([n, 0], [0, 0], 64)
    whole = layer.buffers(n, n, 64)
    layer.step(x, pos, cu, rows, k_len, whole)
    keys, one = layer.k_cache[:n].clone(), layer.buffers(1, 1, 64)
    for i in range(n):
        cu, rows, k_len = _batch([0, 1], [n, i], 64)
        layer.step(x[i:i + 1], pos[i:i + 1], cu, rows, k_len, one)
        # the projection's sums are made in another order for one row: its rounding may fall on the next value, one step
        eps = torch.finfo(torch.float16).eps
        step = eps * keys[i].double().abs().clamp(min=1) + 1e-6
        assert _close(layer.k_cache[64 + i], keys[i].double(), 2 * step)
        a = attention_reference(one["qkv"][:, :heads], layer.k_cache[64:64 + i + 1], layer.v_cache[64:64 + i + 1], True, layer.scale)
        assert _close(one["att"], *a)


def test_captured_steps():
    """Two captured steps of different sequences, each with buffers of its own, replayed by turns with new inputs."""
    D, heads, kv_heads, E, slot = 256, 8, 2, 64, 1600
    layer, r = _layer(torch.bfloat16, D, heads, kv_heads, E, 3, slot, True)
    cu, rows, k_len = _batch([1500, 300, 7], [0, 0, 0], slot)
    layer.step(r(1807, D), torch.zeros((1807, 3), dtype=torch.int32, device=DEV), cu, rows, k_len, layer.buffers(1807, 1500, slot))
    calls = []
    for new, held in (([1, 1, 1], [1500, 300, 7]), ([0, 2, 1], [1501, 301, 8])):
        n = sum(new)
        x, pos = r(n, D), torch.randint(0, 50, (n, 3), dtype=torch.int32, device=DEV)
        calls.append([x, pos, *_batch(new, held, slot), layer.buffers(n, 2, slot)])
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
            assert torch.equal(layer.step(*call[:-1], layer.buffers(call[0].shape[0], 2, slot)), got) and bool(got.isfinite().all())


def test_a_padded_batch():
    """Tokens behind the last sequence, whatever they hold, change nothing of the others."""
    D, heads, kv_heads, E, slot, real, padded = 256, 4, 2, 64, 200, 71, 96
    layer, r = _layer(torch.bfloat16, D, heads, kv_heads, E, 3, slot, True)
    new = [40, 0, 31]
    cu, rows, k_len = _batch(new, [0, 0, 0], slot)
    x, pos = r(padded, D), torch.randint(0, 50, (padded, 3), dtype=torch.int32, device=DEV)
    free = torch.arange(3 * slot - (padded - real), 3 * slot, device=DEV)       # the last slot's end
    results = []
    for fill in (0.0, 5.0, math.nan):
        layer.k_cache.fill_(math.nan)
        layer.v_cache.fill_(math.nan)
        x[real:] = fill
        buffers = layer.buffers(padded, 64, slot)
        buffers["att"].fill_(math.nan)
        results.append(layer.step(x, pos, cu, torch.cat([rows, free]), k_len, buffers)[:real].clone())
    assert bool(results[0].isfinite().all()) and all(torch.equal(a, results[0]) for a in results[1:])
