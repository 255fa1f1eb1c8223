"""The example that runs the attention step's operators together: prompts and single
tokens over a paged cache against the same tokens as whole packed prompts, and one
prompt against a plain 64-bit attention of the same projections."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import attn_plain
from paper_2607_08779_gb300 import inputs, sss

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_step.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("attention_step", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


# The two ways round q, k, v, p and the attention's output to bf16 (2^-8 each at most,
# of values that a projection of random signs averages) from products that differ by
# 2^-11 (the batched and the tiled products' operands): less than 8 x 2^-8 in all.
TOL = 8 * 2.0 ** -8


@pytest.mark.parametrize("layer,q,prompts,steps,page", [
    ("small", 4, (40, 3, 129), 4, 16), ("small", 2, (1,), 20, 32), ("small", 3, (300, 17), 2, 64),
    ("llama3_8b", 4, (130, 20), 3, 16), ("qwen3_32b", 4, (64, 33, 5), 2, 128),
])
def test_steps_give_what_whole_prompts_give(example, layer, q, prompts, steps, page):
    diff, status = example.run(layer, q, prompts, steps, page)
    assert status == 0
    assert diff <= TOL


def test_a_prompt_against_64_bits(example):
    heads, kv_heads, dim, hidden, norm = example.LAYERS["small"]
    n = 150
    net = example.AttentionLayer(heads, kv_heads, dim, hidden, norm, 4, 16, 16, 256)
    x = inputs.normal_bf16_cuda((n, hidden), 3)
    q, k, v = (t.cpu().numpy().reshape(n, -1, dim) for t in net.project(x))
    cos, sin = net.rope.cos.cpu().numpy(), net.rope.sin.cpu().numpy()
    pos = np.arange(n)
    turn = lambda t, w: attn_plain.norm_rope(t, w.cpu().numpy(), cos, sin, pos, dim, True, 1e-6)[0]  # noqa: E731
    qr, kr = turn(q, net.rope.q_norm), turn(k, net.rope.k_norm)
    want = np.zeros((n, heads, dim))
    for h in range(heads):
        s = qr[:, h] @ kr[:, h // (heads // kv_heads)].T * dim ** -0.5
        s[np.triu_indices(n, 1)] = -np.inf
        p = np.exp(s - s.max(1, keepdims=True))
        want[:, h] = p @ v[:, h // (heads // kv_heads)].astype(np.float64) / p.sum(1, keepdims=True)
    want = net.output(torch.from_numpy(want).to(torch.bfloat16).cuda())
    got = net.whole(x, [n], None)
    assert float((got - want).abs().max() / want.abs().max()) <= TOL
