"""The example's attention block: prompts and decode steps on one cache."""
import importlib.util
import math
import os

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16


def example():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_decode_steps_continue_a_prompt():
    """Three prompts, then steps of all of them together: what a step gives is what the same tokens give as the end of a longer prompt,
    which attends to the same INT4 vectors.  (The linear layers' kernels for one and for many tokens add in other orders, which moves a
    4-bit code now and then, by one step: a few in a hundred of an output's rms at most.)"""
    ex = example()
    heads, kv_heads, D = 8, 2, 128
    prompts, steps = [70, 1, 33], 5
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = [torch.randn((p + steps, 2, heads * D), generator=g, device="cuda").to(BF16) for p in prompts]
    make = lambda: ex.AttentionBlock(heads, kv_heads, D, ex.Cache(16, kv_heads, D, 16, 128))  # noqa: E731
    one, two = make(), make()
    seqs = [one.cache.new() for _ in prompts]
    for s, p in zip(seqs, prompts):
        one(x[s][:p, 0].contiguous(), x[s][:p, 1].contiguous(), [s], p)
    ys = []
    for t in range(steps):
        now = torch.stack([x[s][prompts[s] + t] for s in seqs])
        y, stream = one(now[:, 0].contiguous(), now[:, 1].contiguous(), seqs, 1)
        assert torch.equal(stream, (now[:, 0].float() + now[:, 1].float()).to(BF16))
        ys.append(y)
    assert one.cache.lengths == [p + steps for p in prompts]
    for s, p in zip(seqs, prompts):
        two.cache.new()
        y, _ = two(x[s][:, 0].contiguous(), x[s][:, 1].contiguous(), [s], p + steps)
        got, want = torch.stack([v[s] for v in ys]).float(), y[p:].float()
        assert (got - want).norm() <= 0.05 * want.norm()


def test_block_against_unquantised_arithmetic():
    """The whole block against fp64 without any quantisation.  Five quantisers of 4 bits on Gaussian data (weights and activations of two
    layers, keys and values), each with a relative error of about a tenth: the sum of their squares is under a quarter of the output's."""
    ex = example()
    heads, kv_heads, D, T = 8, 4, 128, 60
    block = ex.AttentionBlock(heads, kv_heads, D, ex.Cache(8, kv_heads, D, 16, 64))
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x, r = (torch.randn((T, heads * D), generator=g, device="cuda").to(BF16) for _ in range(2))
    y, _ = block(x, r, [block.cache.new()], T)
    h, n = ref.add_rms_norm(x, r, block.norm, block.eps)
    qkv = (n @ ref.f64(block.w_qkv).t()).view(T, heads + 2 * kv_heads, D)
    positions = torch.arange(T)
    q = ref.turn(qkv[:, :heads], block.cos_sin, positions, False, True, torch.float64)
    k = ref.turn(qkv[:, heads:heads + kv_heads], block.cos_sin, positions, False, True, torch.float64).repeat_interleave(heads // kv_heads, 1)
    v = qkv[:, heads + kv_heads:].repeat_interleave(heads // kv_heads, 1)
    s = torch.einsum("thd,uhd->htu", q, k) / math.sqrt(D)
    s = s.masked_fill(torch.ones(T, T).tril() == 0, -math.inf)
    o = torch.einsum("htu,uhd->thd", s.softmax(-1), v).reshape(T, heads * D)
    want = o @ ref.f64(block.w_out).t()
    assert (ref.f64(y) - want).norm() <= 0.5 * want.norm()


def test_cache_books():
    ex = example()
    cache = ex.Cache(3, 1, 64, 16, 40, "cpu")
    s = cache.new()
    at, slots = cache.grow(s, 17)
    assert at == list(range(17)) and len(set(slots)) == 17 and len(cache.free) == 1
    t = cache.new()
    cache.grow(t, 1)
    with pytest.raises(MemoryError):
        cache.grow(t, 16)
    with pytest.raises(ValueError):
        cache.grow(s, 40)
