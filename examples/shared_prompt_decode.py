"""Several answers to one prompt, token by token: an attention block with the Walsh-Hadamard output layer, served from a paged cache.

    python examples/shared_prompt_decode.py [--sequences 64] [--prompt 4096] [--tokens 64] [--heads 32] [--key-heads 8] [--head-dim 128]

The prompt's keys and values are computed once and lie in pages that all sequences name as their prefix; every sequence then
grows by a token a step.  A step of a layer is

    q, k, v = x W_qkv                                   a library product
    q       = wht_attention_append(...)                 k rotated into the cache, v beside it, q rotated
    a       = wht_attention_paged(...)                  over the prefix and the sequence's own pages
    x, sums = wht_affine_forward_residual_stats(...)    x + alpha (.) (H a) + beta, in place of a dense output projection

captured into a HIP graph once and replayed: lengths live on the GPU, and a step raises them.  Weights are random, the tokens' embeddings
as well: this shows the calls and what they take, not a language model.
"""
import argparse
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2603_08343_amd as wht


class Block:
    """One attention block: d = heads * head_dim, a fused projection, a paged cache, the Hadamard output layer."""

    def __init__(self, heads, key_heads, head_dim, sequences, prompt, tokens, page=64, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.key_heads, self.head_dim, self.d = heads, key_heads, head_dim, heads * head_dim
        self.sequences, self.prompt, self.page, self.dtype, self.device = sequences, prompt, page, dtype, device
        width = (heads + 2 * key_heads) * head_dim
        self.w_qkv = (torch.randn(self.d, width, generator=g, device=device) / self.d ** 0.5).to(dtype)
        self.alpha = torch.empty(self.d, device=device).uniform_(0.5, 1.5, generator=g)
        self.beta = torch.zeros(self.d, device=device)
        # pages: the prompt's, then room for `tokens` of every sequence
        front, own = -(-prompt // page), -(-tokens // page)
        shape = (front + sequences * own, key_heads, page, head_dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        numbers = torch.arange(shape[0], dtype=torch.int32, device=device)
        self.prefix_table, self.table = numbers[:front], numbers[front:].view(sequences, own)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.rope = wht.wht_attention_rope_table(prompt + tokens, head_dim, device=device)

    def _attend(self, x, table, lengths, q_starts, position, prefix_length, max_q):
        """x [T, d] -> x + alpha (.) (H attention(x)) + beta, and the sum of its squares; T new tokens go into the cache."""
        h, k = self.heads, self.key_heads
        qkv = (x @ self.w_qkv).view(x.shape[0], h + 2 * k, self.head_dim)
        q = wht.wht_attention_append(qkv[:, :h], qkv[:, h:h + k], qkv[:, h + k:], self.k_pages, self.v_pages, table, lengths, self.rope,
                                     q_starts=q_starts, position=position)
        a = wht.wht_attention_paged(q, self.k_pages, self.v_pages, table, lengths, q_starts=q_starts, prefix_table=self.prefix_table,
                                    prefix_length=prefix_length, max_q=max_q)
        return wht.wht_affine_forward_residual_stats(a.view(x.shape), self.alpha, self.beta, x)

    def read_prompt(self, x):
        """The prompt's tokens x [prompt, d], as the one sequence whose pages are the prefix."""
        n = torch.tensor([x.shape[0]], dtype=torch.int32, device=self.device)
        starts = torch.tensor([0, x.shape[0]], dtype=torch.int32, device=self.device)
        return self._attend(x, self.prefix_table.view(1, -1), n, starts, 0, 0, x.shape[0])

    def step(self, x):
        """One new token of every sequence, x [sequences, d]."""
        self.lengths.add_(1)
        return self._attend(x, self.table, self.lengths, None, self.prompt, self.prompt, 1)


def run(sequences=64, prompt=4096, tokens=64, heads=32, key_heads=8, head_dim=128, graph=True, seed=0):
    """Returns (block, prompt embeddings, embeddings of every step, outputs of every step, microseconds a step)."""
    block = Block(heads, key_heads, head_dim, sequences, prompt, tokens, seed=seed)
    g = torch.Generator(device=block.device).manual_seed(seed + 1)
    x_prompt = torch.randn(prompt, block.d, generator=g, device=block.device).to(block.dtype)
    x_steps = torch.randn(tokens, sequences, block.d, generator=g, device=block.device).to(block.dtype)
    block.read_prompt(x_prompt)
    x = x_steps[0].clone()
    step = lambda: block.step(x)                                                # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                                  # libraries load, memory is found
    torch.cuda.current_stream().wait_stream(side)
    block.lengths.zero_()
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            result = step()
    outputs = []
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for t in range(tokens):
        x.copy_(x_steps[t])
        if graph:
            captured.replay()
        else:
            result = step()
        outputs.append(result[0].clone())
    end.record()
    torch.cuda.synchronize()
    return block, x_prompt, x_steps, outputs, begin.elapsed_time(end) * 1e3 / tokens


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("sequences", 64), ("prompt", 4096), ("tokens", 64), ("heads", 32), ("key-heads", 8), ("head-dim", 128)):
        ap.add_argument("--" + name, type=int, default=value)
    a = vars(ap.parse_args())
    for graph in (False, True):
        us = run(**a, graph=graph)[-1]
        print(f"{'replayed graph' if graph else 'eager calls':15s} {us:8.1f} us a step, {a['sequences'] / us * 1e6:10.0f} tokens/s and layer")


if __name__ == "__main__":
    main()
