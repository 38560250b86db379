"""Decoder blocks over a hybrid batch: attention to a paged key/value cache in front of the MoE layer.

A small stack with random weights serves prompts of different lengths and decodes from all of them:

    python examples/decoder_blocks.py [--dtype bf16|f32] [--kv-format fp8] [--chunk 64] [--steps 8]

Every pass is one batch of rows, decode rows first.  A layer appends its new keys and values to its pages (moe_kv_append), attends to
everything the sequences hold (moe_paged_attention) and runs the expert layer (moe_group_forward); the projections around them
are plain matrix products.  One batch struct serves all layers of a pass, and its tensors live as long as the server.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_08055_amd import binding  # noqa: E402


class Stack:
    def __init__(self, layers=2, H=256, heads=8, kv_heads=2, dim=64, E=16, K=4, I=192, page=16, max_seqs=8, max_tokens=1024,
                 max_rows=1024, window=0, dtype=torch.float32, kv_format="", device="cuda:0", seed=0):
        g = torch.Generator().manual_seed(seed)

        def weight(*shape, std=0.05):
            return (torch.randn(*shape, generator=g) * std).to(dtype).to(device)

        self.H, self.heads, self.kv_heads, self.dim, self.page, self.window = H, heads, kv_heads, dim, page, window
        self.dtype, self.device, self.max_seqs = dtype, device, max_seqs
        self.layers = [{"w_qkv": weight(H, (heads + 2 * kv_heads) * dim), "w_o": weight(heads * dim, H),
                        "sinks": weight(heads, std=1.0).float(),
                        "moe": {"w_router": weight(E, H), "w_gate_up": weight(E, 2 * I, H), "w_down": weight(E, H, I)}}
                       for _ in range(layers)]
        self.kv = binding.KVContext(heads, kv_heads, dim, page, dtype, kv_format=kv_format, device=device)
        self.moe = binding.Context(H, E, K, I, dtype, max_tokens=max_rows, residual=True, device=device)
        # the cache: pages of every layer, one page table for all of them
        per_seq = -(-max_tokens // page)
        self.n_pages = max_seqs * per_seq
        for layer in self.layers:
            shape = (self.n_pages, kv_heads, page, dim)
            pages = [torch.zeros(shape, device=device).to(self.kv.page_dtype) for _ in range(2)]
            scales = [torch.zeros(shape[:3], dtype=torch.uint8, device=device) for _ in range(2)] if self.kv.fp8 else []
            layer["pages"] = self.kv.pack_pages(*pages, *scales)
            layer["moe_packed"] = self.moe.pack_layers([layer["moe"]])
        self.free = list(range(self.n_pages))
        self.table = torch.full((max_seqs, per_seq), -1, dtype=torch.int32)
        self.lens = [0] * max_seqs
        self.offsets_dev = torch.zeros(max_seqs + 1, dtype=torch.int32, device=device)
        self.lens_dev = torch.zeros(max_seqs, dtype=torch.int32, device=device)
        self.table_dev = self.table.to(device)
        self.batch = self.kv.pack_batch(self.offsets_dev, self.lens_dev, self.table_dev)

    def step(self, new):
        """One pass: new[s] are the rows [n_s, H] of sequence s (or None).  The rows' hidden states, in the order of the sequences."""
        rows = [x.shape[0] if x is not None else 0 for x in new] + [0] * (self.max_seqs - len(new))
        for s, n in enumerate(rows):
            have = -(-self.lens[s] // self.page)
            self.lens[s] += n
            for i in range(have, -(-self.lens[s] // self.page)):
                self.table[s, i] = self.free.pop()
        self.offsets_dev.copy_(torch.tensor([0] + rows).cumsum(0))
        self.lens_dev.copy_(torch.tensor(self.lens))
        self.table_dev.copy_(self.table)
        x = torch.cat([r for r in new if r is not None])
        q_end, k_end = self.heads * self.dim, (self.heads + self.kv_heads) * self.dim
        for layer in self.layers:
            qkv = x @ layer["w_qkv"]
            q = qkv[:, :q_end].unflatten(1, (self.heads, self.dim))
            k = qkv[:, q_end:k_end].unflatten(1, (self.kv_heads, self.dim))
            v = qkv[:, k_end:].unflatten(1, (self.kv_heads, self.dim))
            self.kv.moe_kv_append(k, v, layer["pages"], self.batch)
            a = self.kv.moe_paged_attention(q, layer["pages"], self.batch, window=self.window, sinks=layer["sinks"])
            x = x + a.flatten(1) @ layer["w_o"]
            x = self.moe.moe_group_forward(None, x.contiguous(), None, packed=layer["moe_packed"])[0]
        return x.split([n for n in rows if n])

    def release(self, s):
        """Gives a sequence's pages back."""
        self.free += [int(p) for p in self.table[s] if p >= 0]
        self.table[s] = -1
        self.lens[s] = 0


def serve(stack, prompts, steps, chunk=0):
    """Prefills the prompts (each in chunks of `chunk` rows; 0: whole) and decodes `steps` tokens from each: the next row of a sequence is
    its last hidden state, scaled to unit size, as a stand-in for sampling and embedding.  Returns every sequence's hidden states."""
    left = [p for p in prompts]
    got = [[] for _ in prompts]
    while any(len(g) < len(p) + steps for g, p in zip(got, prompts)):
        new, who = [], []
        for s, p in enumerate(prompts):
            if left[s].shape[0] > 0:
                n = min(chunk or left[s].shape[0], left[s].shape[0])
                new.append(left[s][:n])
                left[s] = left[s][n:]
            elif len(got[s]) < len(p) + steps:
                last = got[s][-1].float()
                new.append((last / last.square().mean().sqrt()).to(p.dtype)[None])
            else:
                new.append(None)
                continue
            who.append(s)
        for s, out in zip(who, stack.step(new)):
            got[s] += list(out)
    return [torch.stack(g) for g in got]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--kv-format", choices=("", "fp8"), default="")
    ap.add_argument("--chunk", type=int, default=64)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randn(n, 256, generator=g).to(dtype).cuda() for n in (1, 37, 200, 90)]
    runs = {}
    serve(Stack(dtype=dtype, kv_format=a.kv_format), prompts, a.steps, a.chunk)      # loads the kernels
    for name, chunk in (("whole prompts", 0), (f"chunks of {a.chunk}", a.chunk)):
        stack = Stack(dtype=dtype, kv_format=a.kv_format)
        start, end = torch.cuda.Event(True), torch.cuda.Event(True)
        start.record()
        runs[name] = torch.cat(serve(stack, prompts, a.steps, chunk)).float()
        end.record()
        end.synchronize()
        print(f"{name}: {runs[name].shape[0]} rows in {start.elapsed_time(end):.2f} ms")
    x, y = runs.values()
    print(f"relative difference of the two: {float((x - y).norm() / y.norm()):.2e}")


if __name__ == "__main__":
    main()
