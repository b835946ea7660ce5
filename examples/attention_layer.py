"""The attention of one decoder layer, as a serving program runs it: W4A8 projections with a 4-bit cache of keys and values.

    python3 examples/attention_layer.py [--heads 32 --kv-heads 8 --prompts 700,133,260 --steps 16]

Prompts of different lengths are packed and go through

    quantise -> qkv projection -> norm and rotation -> attention over the prompts -> quantise -> output projection,

their keys and values into the cache; then every sequence takes a token at a time:

    quantise -> qkv projection -> rotation, cache write -> attention over the cache -> quantise -> output projection,

captured once as a HIP graph and replayed.  What the steps return is compared with the same tokens run as part of a prompt, which
reads their keys and values unquantised.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2509_01229_amd import api  # noqa: E402
from paper_2509_01229_amd import workloads as WL  # noqa: E402

HEAD_DIM, PAGE, GROUP = 128, 64, 64


class Linear:
    """A W4A8 linear layer: FP16 in, FP16 out."""

    def __init__(self, N, K, seed):
        self.N, self.K = N, K
        W = WL.make_weights(N, K, sigma=K ** -0.5, seed=seed)
        self.codes, self.gparams, self.scales = (torch.from_numpy(t).cuda() for t in api.liquidquant_pack_weights(W, GROUP))

    def __call__(self, x):
        return api.w4a8_gemm(*api.w4a8_quantize_activations(x), self.codes, self.gparams, self.scales, self.N, self.K, GROUP)


class PagedCache:
    """The 4-bit cache and who has which of its pages."""

    def __init__(self, sequences, longest, kv_heads):
        self.width = -(-longest // PAGE)
        self.cache = api.kv4_cache(sequences * self.width, PAGE, kv_heads, HEAD_DIM)
        # (a serving program hands pages out as sequences grow; here each has its own from the start, in any order)
        self.table = torch.randperm(sequences * self.width, device="cuda").to(torch.int32).view(sequences, self.width)

    def slots(self, sequence, position):
        """Places of tokens: two int tensors of the same length."""
        return (self.table[sequence, position // PAGE] * PAGE + position % PAGE).to(torch.int32)


class AttentionLayer:
    def __init__(self, heads, kv_heads, longest, seed=0):
        self.heads, self.kv_heads, self.hidden = heads, kv_heads, heads * HEAD_DIM
        self.qkv = Linear((heads + 2 * kv_heads) * HEAD_DIM, self.hidden, seed)
        self.out = Linear(self.hidden, self.hidden, seed + 1)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.q_norm, self.k_norm = (1.0 + 0.1 * torch.randn(HEAD_DIM, generator=gen, device="cuda") for _ in range(2))
        self.rope = torch.from_numpy(api.attn_rope_table(longest, HEAD_DIM)).cuda()

    def _project(self, x):
        return self.qkv(x).view(-1, self.heads + 2 * self.kv_heads, HEAD_DIM).split((self.heads, self.kv_heads, self.kv_heads), 1)

    def prompts(self, x, starts, positions, slots=None, cache=None):
        """Packed prompts x [tokens, hidden]; where there is a cache, their keys and values go into its slots."""
        q, k, v = self._project(x)
        q, k = api.attn_qk_norm_rope(q, k, positions, self.rope, q_norm=self.q_norm, k_norm=self.k_norm)
        if cache is not None:
            api.kv4_write(k, v, slots, cache)
        return self.out(api.attn_prompt(q, k, v, starts).view(-1, self.hidden))

    def step(self, x, positions, slots, cache, table, context):
        """One token for each sequence, x [sequences, hidden]."""
        q, k, v = self._project(x)
        q = api.kv4_append(q, k, v, positions, self.rope, slots, cache, q_norm=self.q_norm, k_norm=self.k_norm)
        return self.out(api.kv4_attention(q, cache, table, context).view(-1, self.hidden))


def run(heads=32, kv_heads=8, lengths=(700, 133, 260), steps=16, seed=0):
    """(result of the steps, of the same tokens as part of prompts): [sequences, steps, hidden] each."""
    longest = max(lengths) + steps
    layer = AttentionLayer(heads, kv_heads, longest, seed)
    pages = PagedCache(len(lengths), longest, kv_heads)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    xs = [torch.randn((n + steps, layer.hidden), generator=gen, device="cuda").half() for n in lengths]

    def packed(lens):
        sequence = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
        position = torch.cat([torch.arange(n, device="cuda") for n in lens])
        starts = torch.tensor([0, *lens], device="cuda").cumsum(0).to(torch.int32)
        return sequence, position, starts

    # the prompts
    sequence, position, starts = packed(lengths)
    layer.prompts(torch.cat([x[:n] for x, n in zip(xs, lengths)]), starts, position.to(torch.int32), pages.slots(sequence, position), pages.cache)

    # the steps, from a graph
    each = torch.arange(len(lengths), device="cuda")
    lens = torch.tensor(lengths, device="cuda")
    x = torch.empty((len(lengths), layer.hidden), dtype=torch.float16, device="cuda")
    positions, slots, context = (torch.empty(len(lengths), dtype=torch.int32, device="cuda") for _ in range(3))

    def feed(i):
        x.copy_(torch.stack([s[n + i] for s, n in zip(xs, lengths)]))
        positions.copy_(lens + i)
        slots.copy_(pages.slots(each, lens + i))
        context.copy_(lens + i + 1)

    feed(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(x, positions, slots, pages.cache, pages.table, context)  # (makes the stream's workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = layer.step(x, positions, slots, pages.cache, pages.table, context)
    got = []
    for i in range(steps):
        feed(i)
        graph.replay()
        got.append(y.clone())
    got = torch.stack(got, 1)

    # the same tokens as the ends of longer prompts
    sequence, position, starts = packed([n + steps for n in lengths])
    whole = layer.prompts(torch.cat(xs), starts, position.to(torch.int32))
    want = torch.stack([whole[int(s) + n: int(s) + n + steps] for s, n in zip(starts, lengths)])
    torch.cuda.synchronize()
    return got, want


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--prompts", default="700,133,260", help="lengths of the prompts")
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    got, want = run(a.heads, a.kv_heads, [int(n) for n in a.prompts.split(",")], a.steps)
    off = float((got.float() - want.float()).norm() / want.float().norm())
    print(f"{got.shape[0]} sequences, {got.shape[1]} steps each: {100 * off:.1f}% off the same tokens with unquantised keys and values")


if __name__ == "__main__":
    main()
