"""examples/shared_prompt_decode.py: the block's steps, eager and replayed, against the same block in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("shared_prompt_decode", os.path.join(ROOT, "examples", "shared_prompt_decode.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _hadamard(d):
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < d:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)))
    return h / math.sqrt(d)


def _in_64_bits(block, x_prompt, x_steps):
    """Outputs of every step, from the definition: no cache, every sequence's keys one after the other."""
    w, alpha, rope = block.w_qkv.cpu().double(), block.alpha.cpu().double(), block.rope.cpu().double()
    heads, keys, n = block.heads, block.key_heads, block.head_dim
    H = _hadamard(block.d)

    def project(x, position):
        y = (x.cpu().double() @ w).to(torch.bfloat16).double().view(-1, heads + 2 * keys, n)     # the product is rounded to bfloat16
        c, s = rope[position, :, 0][:, None], rope[position, :, 1][:, None]
        a, b = y[:, :heads + keys, :n // 2], y[:, :heads + keys, n // 2:]
        turned = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
        return turned[:, :heads], turned[:, heads:], y[:, heads + keys:]

    P = x_prompt.shape[0]
    _, kp, vp = project(x_prompt, torch.arange(P))
    k, v = kp[:, None].expand(-1, block.sequences, -1, -1), vp[:, None].expand(-1, block.sequences, -1, -1)      # [tokens, sequences, keys, n]
    out = []
    for t, x in enumerate(x_steps):
        q, kt, vt = project(x, torch.full((block.sequences,), P + t))
        k, v = torch.cat((k, kt[None])), torch.cat((v, vt[None]))
        q = q.view(block.sequences, keys, heads // keys, n)
        p = torch.softmax(torch.einsum("bhgd,tbhd->bhgt", q, k) / math.sqrt(n), dim=-1)
        a = torch.einsum("bhgt,tbhd->bhgd", p, v).reshape(block.sequences, -1)
        out.append(x.cpu().double() + alpha * (a @ H))
    return out


@pytest.mark.gpu
def test_steps_in_64_bits_and_replayed():
    example = _example()
    small = dict(sequences=5, prompt=75, tokens=9, heads=8, key_heads=2, head_dim=64)
    block, x_prompt, x_steps, eager, _ = example.run(**small, graph=False)
    replayed = example.run(**small, graph=True)[3]
    assert all(torch.equal(a, b) for a, b in zip(eager, replayed))
    # roundings to bfloat16 on the way, half a step (2^-8) each: q and k twice, the weights, v and the attention's output, the result.  A score
    # is of the size of 1, so that q's and k's four move a weight by about 4 * 2^-8 at most, and the others are one each.
    for got, want in zip(eager, _in_64_bits(block, x_prompt, x_steps)):
        off = (got.cpu().double() - want).abs()
        assert float((off - 2.0 ** -8 * want.abs()).max()) <= 8 * 2.0 ** -8
