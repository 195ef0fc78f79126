"""Decoding with whole layers: the compressed products and every operator around
them.

A small random-weight decoder.  Per layer

    residual's addition and norm -> QKV product -> rotation by position, new keys
    and values into the paged cache -> attention -> output product
    -> residual's addition and norm -> gate and up product -> gated activation
    -> down product

The middle layers' linears are QTEA-compressed (fp16 activations); the first
layer's feed-forward part and the LM head stay outside that format, in 4 bits
with 8-bit activations straight from the norm and the gate.

Run:  python examples/decode.py [--format e4m3] [--tokens 16]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_00224_amd as q  # noqa: E402

HIDDEN, HEADS, KV_HEADS, DIM, INNER, LAYERS, VOCAB, PAGE, EPS = 256, 8, 2, 64, 512, 2, 1000, 16, 1e-5


def ternary_parts(gen, N, K):
    """A random matrix's ternary codes, scales and residual on 2 % of its columns."""
    dev = "cuda"
    n = max(1, K // 50)
    uni = lambda shape, lo, hi: (lo + (hi - lo) * torch.rand(shape, generator=gen, device=dev)).half()  # noqa: E731
    return (torch.randint(-1, 2, (N, K), generator=gen, device=dev, dtype=torch.int8), uni((N,), 0.05, 0.1), uni((K,), 0.8, 1.2),
            torch.randperm(K, generator=gen, device=dev)[:n].sort().values.int(),
            (0.05 * torch.randn((n, N // 4), generator=gen, device=dev)).half(), torch.randint(0, 4, (n, N // 4), generator=gen, device=dev, dtype=torch.uint8))


class Ternary:
    """A compressed matrix: fp16 rows in, fp32 out, 16 rows at a time."""

    eight_bits = False

    def __init__(self, gen, N, K):
        self.parts = ternary_parts(gen, N, K)
        self.m, self.N, self.K = q.pack_matrix(*self.parts), N, K
        self.ws = q.new_workspace(self.m.desc, q.QTEA_MAX_BATCH)

    def __call__(self, x, scale=None):
        y = torch.empty((x.shape[0], self.N), device="cuda")
        for i in range(0, x.shape[0], q.QTEA_MAX_BATCH):
            rows = x[i:i + q.QTEA_MAX_BATCH]
            q.qtea_gemm_lowbatch(self.m.desc, self.m.packed, rows, rows.shape[0], y[i:i + rows.shape[0]], self.ws)
        return y


class FourBit:
    """A matrix of 4-bit codes: 8-bit rows in, fp32 out, 64 rows at a time."""

    eight_bits = True

    def __init__(self, gen, N, K):
        self.W = torch.randn((N, K), generator=gen, device="cuda") * K ** -0.5
        self.m, self.N, self.K = q.pack_matrix_w4(self.W), N, K

    def __call__(self, x, scale):
        y = torch.empty((x.shape[0], self.N), device="cuda")
        for i in range(0, x.shape[0], q.QTEA_W4_MAX_BATCH):
            rows = slice(i, i + q.QTEA_W4_MAX_BATCH)
            q.qtea_w4_gemm_lowbatch(self.m, x[rows], y[rows], x_scale=scale[rows])
        return y


def rows_for(linear, n):
    """Room for n rows of the type that a linear takes: values, or codes and scales."""
    if not linear.eight_bits:
        return torch.empty((n, linear.K), dtype=torch.float16, device="cuda"), None
    return torch.empty((n, linear.K), dtype=torch.uint8, device="cuda"), torch.empty((n, linear.K // 32), dtype=torch.uint8, device="cuda")


class Decoder:
    """`seqs` sequences of up to `most` tokens; cached keys and values in `fmt`."""

    def __init__(self, fmt, seqs, most, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        norm = lambda: 0.5 + torch.rand(HIDDEN, generator=gen, device="cuda")  # noqa: E731
        self.embed = torch.randn((VOCAB, HIDDEN), generator=gen, device="cuda")
        self.layers = []
        for i in range(LAYERS):
            ffn = FourBit if i == 0 else Ternary
            self.layers.append((norm(), Ternary(gen, (HEADS + 2 * KV_HEADS) * DIM, HIDDEN), Ternary(gen, HIDDEN, HEADS * DIM),
                                norm(), ffn(gen, 2 * INNER, HIDDEN), ffn(gen, HIDDEN, INNER)))
        self.last, self.head = norm(), FourBit(gen, VOCAB, HIDDEN)
        self.freq = 10000.0 ** (-2.0 * torch.arange(DIM // 2, device="cuda") / DIM)
        pages = -(-most // PAGE)
        self.caches = [q.new_kv_cache(fmt, seqs * pages, PAGE, KV_HEADS, DIM) for _ in range(LAYERS)]
        self.table = torch.randperm(seqs * pages, generator=gen, device="cuda").int().view(seqs, pages)
        self.attention_ws = q.new_attention_workspace(HEADS, DIM)
        self.rows = torch.bfloat16 if fmt == "bf16" else torch.float16  # what the attention takes

    def logits(self, tokens, q_start, kv_len):
        """Of each of the new tokens [rows]."""
        n = len(tokens)
        residual = self.embed[tokens.long()]
        add = torch.zeros_like(residual)  # what the last product gave
        for (norm1, qkv, out, norm2, gate_up, down), cache in zip(self.layers, self.caches):
            x, scale = rows_for(qkv, n)
            q.qtea_rms_norm(add, norm1, x, residual=residual, eps=EPS, out_scale=scale)
            y = qkv(x, scale).view(n, HEADS + 2 * KV_HEADS, DIM)
            rows = torch.empty((n, HEADS, DIM), dtype=self.rows, device="cuda")
            q.qtea_kv_append_rotated(cache, y[:, :HEADS], y[:, HEADS:HEADS + KV_HEADS], y[:, HEADS + KV_HEADS:], q_start, kv_len, self.table, self.freq, rows)
            attended = torch.empty_like(rows)
            q.qtea_paged_attention(cache, rows, q_start, kv_len, self.table, attended, self.attention_ws)
            add = out(attended.view(n, HEADS * DIM).half())
            x, scale = rows_for(gate_up, n)
            q.qtea_rms_norm(add, norm2, x, residual=residual, eps=EPS, out_scale=scale)
            y = gate_up(x, scale)
            x, scale = rows_for(down, n)
            q.qtea_silu_mul(y[:, :INNER], y[:, INNER:], x, out_scale=scale)
            add = down(x, scale)
        x, scale = rows_for(self.head, n)
        q.qtea_rms_norm(add, self.last, x, residual=residual, eps=EPS, out_scale=scale)
        return self.head(x, scale)


def generate(fmt, prompts, count, seed=0):
    """`count` greedy tokens after each prompt."""
    model = Decoder(fmt, len(prompts), max(map(len, prompts)) + count, seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    sizes = [len(p) for p in prompts]
    starts = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    kv_len = i32(sizes)
    last = model.logits(i32([t for p in prompts for t in p]), i32(starts), kv_len)[[s - 1 for s in starts[1:]]]
    got = []
    one = torch.arange(len(prompts) + 1, dtype=torch.int32, device="cuda")
    for _ in range(count):
        token = last.argmax(-1).int()
        got.append(token)
        kv_len = kv_len + 1
        last = model.logits(token, one, kv_len)
    return torch.stack(got, 1).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", default="e4m3", choices=sorted(q.KV_FORMATS))
    ap.add_argument("--tokens", type=int, default=16)
    args = ap.parse_args()
    prompts = [[1, 2, 3, 4, 5], [6, 7], [8, 9, 10, 11, 12, 13]]
    for p, g in zip(prompts, generate(args.format, prompts, args.tokens)):
        print(f"prompt {p}: {g}")


if __name__ == "__main__":
    main()
