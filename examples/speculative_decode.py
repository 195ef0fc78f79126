"""Speculative decoding with the library's products and serving operators.

A small random-weight decoder (attention layers only) whose linears are
QTEA-compressed.  Each step verifies a few drafted tokens per sequence in one
pass, as many rows as the low-batch product takes:

    drafts from a bigram table
    -> per layer: QKV product, new keys and values into the paged cache,
       attention of the new rows over it, output product
    -> LM head product, probabilities
    -> verification: accepted drafts and the next token

Run:  python examples/speculative_decode.py [--format e4m3] [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_00224_amd as q  # noqa: E402

HIDDEN, HEADS, KV_HEADS, DIM, LAYERS, VOCAB, PAGE = 256, 8, 2, 64, 2, 1000, 16


def packed(gen, N, K):
    """A random compressed matrix: ternary codes, scales, 2 % salient columns."""
    dev = "cuda"
    n = max(1, K // 50)
    uni = lambda shape, lo, hi: (lo + (hi - lo) * torch.rand(shape, generator=gen, device=dev)).half()  # noqa: E731
    return q.pack_matrix(torch.randint(-1, 2, (N, K), generator=gen, device=dev, dtype=torch.int8), uni((N,), 0.05, 0.1), uni((K,), 0.8, 1.2),
                         torch.randperm(K, generator=gen, device=dev)[:n].sort().values.int(),
                         (0.05 * torch.randn((n, N // 4), generator=gen, device=dev)).half(),
                         torch.randint(0, 4, (n, N // 4), generator=gen, device=dev, dtype=torch.uint8))


class Decoder:
    """`seqs` sequences of up to `most` tokens; cached keys and values in `fmt`."""

    def __init__(self, fmt, seqs, most, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.embed = torch.randn((VOCAB, HIDDEN), generator=gen, device="cuda")
        self.bigram = torch.softmax(3 * torch.randn((VOCAB, VOCAB), generator=gen, device="cuda"), -1)
        self.layers = [(packed(gen, (HEADS + 2 * KV_HEADS) * DIM, HIDDEN), packed(gen, HIDDEN, HEADS * DIM)) for _ in range(LAYERS)]
        self.head = packed(gen, VOCAB, HIDDEN)
        pages = -(-most // PAGE)
        self.caches = [q.new_kv_cache(fmt, seqs * pages, PAGE, KV_HEADS, DIM) for _ in range(LAYERS)]
        self.table = torch.randperm(seqs * pages, generator=gen, device="cuda").int().view(seqs, pages)
        self.attention_ws = q.new_attention_workspace(HEADS, DIM)
        self.verify_ws = q.new_verify_workspace(seqs)
        # one workspace for all products: they run one after another
        mats = [m for pair in self.layers for m in pair] + [self.head]
        self.ws = torch.zeros(max(q.qtea_workspace_bytes(m.desc, b) for m in mats for b in range(1, q.QTEA_MAX_BATCH + 1)), dtype=torch.uint8, device="cuda")

    def product(self, m, x):
        """y = x W^T (fp16 in, fp32 out), 16 rows at a time."""
        x = x.half().contiguous()
        y = torch.empty((x.shape[0], m.N), device="cuda")
        for i in range(0, x.shape[0], q.QTEA_MAX_BATCH):
            rows = x[i:i + q.QTEA_MAX_BATCH]
            q.qtea_gemm_lowbatch(m.desc, m.packed, rows, rows.shape[0], y[i:i + rows.shape[0]], self.ws)
        return y

    def probabilities(self, tokens, q_start, kv_len, temperature):
        """The target's distribution after each of the new tokens [rows]."""
        x = self.embed[tokens.long()]
        for (qkv, out), cache in zip(self.layers, self.caches):
            y = self.product(qkv, torch.nn.functional.rms_norm(x, (HIDDEN,))).view(-1, HEADS + 2 * KV_HEADS, DIM)
            q.qtea_kv_append(cache, y[:, HEADS:HEADS + KV_HEADS], y[:, HEADS + KV_HEADS:], q_start, kv_len, self.table)
            rows = y[:, :HEADS].half()
            attended = torch.empty_like(rows)
            q.qtea_paged_attention(cache, rows, q_start, kv_len, self.table, attended, self.attention_ws)
            x = x + self.product(out, attended.view(-1, HEADS * DIM))
        logits = self.product(self.head, torch.nn.functional.rms_norm(x, (HIDDEN,)))
        if temperature == 0:  # greedy: all mass on the largest
            return torch.nn.functional.one_hot(logits.argmax(-1), VOCAB).float()
        return torch.softmax(logits / temperature, -1)

    def step(self, last, kv_len, drafts, gen, temperature):
        """One step for all sequences: `last` their newest tokens (not cached
        yet), kv_len their cached lengths.  Returns (accepted, tokens)."""
        n = len(last)
        tokens, rows_q = [last], []
        for _ in range(drafts):  # the draft model, one token after the other
            rows_q.append(self.bigram[tokens[-1].long()])
            tokens.append(torch.multinomial(rows_q[-1], 1, generator=gen).flatten().int())
        fed = torch.stack(tokens, 1)  # [seqs][1 + drafts]
        q_start = torch.arange(0, n * (drafts + 1) + 1, drafts + 1, device="cuda", dtype=torch.int32)
        target = self.probabilities(fed.flatten(), q_start, kv_len + drafts + 1, temperature)
        accepted = torch.empty(n, dtype=torch.int32, device="cuda")
        out = torch.empty((n, drafts + 1), dtype=torch.int32, device="cuda")
        draft = torch.stack(rows_q, 1).flatten(0, 1) if drafts else target[:0]
        u = torch.rand(n * (drafts + 1), generator=gen, device="cuda")
        q.qtea_verify_draft(target, draft, fed[:, 1:].flatten().contiguous(), q_start, u[n:].contiguous(), u[:n].contiguous(), accepted, out,
                            self.verify_ws)
        return accepted, out


def generate(fmt, prompts, steps, drafts, temperature, seed=0):
    """Tokens of each sequence after `steps` verification steps."""
    n = len(prompts)
    model = Decoder(fmt, n, max(map(len, prompts)) + steps * (drafts + 1) + drafts + 1, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    # the prompts but their last tokens, all sequences packed together
    sizes = [len(p) - 1 for p in prompts]
    kv_len = i32(sizes)
    if sum(sizes):
        starts = [0]
        for k in sizes:
            starts.append(starts[-1] + k)
        model.probabilities(i32([t for p in prompts for t in p[:-1]]), i32(starts), kv_len, 1.0)
    got = [list(p) for p in prompts]
    for _ in range(steps):
        accepted, out = model.step(i32([g[-1] for g in got]), kv_len, drafts, gen, temperature)
        for s, (a, row) in enumerate(zip(accepted.tolist(), out.tolist())):
            got[s] += row[:a + 1]
        # what was written for rejected drafts is past the length and will be written over
        kv_len = kv_len + accepted + 1
    return got


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", default="e4m3", choices=sorted(q.KV_FORMATS))
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=3, choices=range(0, 5))
    ap.add_argument("--temperature", type=float, default=1.0)
    args = ap.parse_args()
    prompts = [[1, 2, 3, 4, 5], [6, 7], [8, 9, 10, 11, 12, 13]]
    for p, g in zip(prompts, generate(args.format, prompts, args.steps, args.drafts, args.temperature)):
        print(f"prompt {p}: {len(g) - len(p)} tokens in {args.steps} steps: {g[len(p):]}")


if __name__ == "__main__":
    main()
