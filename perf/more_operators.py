"""The operators of a decoder layer around its products and attention, as
cases to time.

  norm     qtea_rms_norm: the residual's addition and the root-mean-square
           norm of the sum, into 16 or 32 bits, or E4M3 codes in blocks of 32
           channels that share a power of two;
  gate     qtea_silu_mul: the gated activation between a feed-forward part's
           products, into the same;
  rotate   qtea_kv_append_rotated: queries and keys rotated by their
           positions, keys and values written to the paged cache;
  product  qtea_w4_gemm_lowbatch: a few rows by a matrix of E2M1 codes in
           blocks of 32 with a power of two each, for the layers that stay
           outside the ternary format.

Sizes are those of the 8B- and 14B-shaped decoders of synth/workloads.py, of
the example's decoder and of perf/operators.py, and generic ones.

`own` chooses between the framework's kernels and the plain forms: elementary
torch operations in 32 bits, angles in 64.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1 + 1 / 32, "": 0}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# per format: the largest code's value as a fraction of the power of two above
# it, that power, and the range of a block's exponent
FORMAT = {"e4m3": (0.875, 9, -15, 7), "e2m1": (0.75, 3, -23, 13)}
EPS = 1e-5


def listed():
    return [
        # a decoding batch between two products: the one's fp32 output joins
        # the fp32 residual, the next takes fp16
        {"name": "norm_tokens_f16", "kind": "norm", "rows": 16, "heads": 1, "dim": 4096, "x": "f32", "residual": "f32", "out": "f16", "weight": "f32"},
        # a prompt's rows, into 8 bits for a product with 4-bit weights
        {"name": "norm_prompt_e4m3", "kind": "norm", "rows": 8192, "heads": 1, "dim": 5120, "x": "bf16", "residual": "bf16", "out": "e4m3", "weight": "bf16"},
        # each query head's own norm, in a fused projection's output (14B heads)
        {"name": "norm_heads_bf16", "kind": "norm", "rows": 3001, "heads": 40, "dim": 128, "x": "bf16", "residual": "", "out": "bf16", "weight": "bf16"},
        # the two halves of a decoding batch's gate_up product
        {"name": "gate_tokens_f16", "kind": "gate", "rows": 16, "dim": 14336, "x": "f32", "out": "f16"},
        # a prompt's, into 8 bits
        {"name": "gate_prompt_e4m3", "kind": "gate", "rows": 4099, "dim": 17408, "x": "bf16", "out": "e4m3"},
        # the newest token of sixteen sequences, straight from the products' fp32 output
        {"name": "rotate_tokens_e4m3", "kind": "rotate", "fmt": "e4m3", "src": "f32", "out": "f16", "seqs": 16, "new": 1, "ctx": 4000, "heads": 32, "kvh": 8, "dim": 128, "page": 64, "rot": 128, "interleaved": False},
        # prompts of four sequences
        {"name": "rotate_prompts_e4m3", "kind": "rotate", "fmt": "e4m3", "src": "f16", "out": "f16", "seqs": 4, "new": 6000, "ctx": 6000, "heads": 32, "kvh": 8, "dim": 128, "page": 64, "rot": 128, "interleaved": False},
        # ragged chunks of very long sequences, part of each head rotated
        {"name": "rotate_chunks_bf16", "kind": "rotate", "fmt": "bf16", "src": "bf16", "out": "bf16", "seqs": 5, "new": 777, "ctx": 300001, "heads": 15, "kvh": 5, "dim": 96, "page": 32, "rot": 32, "interleaved": True},
        # the example's vocabulary: where latency counts
        {"name": "product_small_f16", "kind": "product", "N": 1000, "K": 256, "batch": 3, "x": "f16", "y": "f32"},
        # the LM head over one token
        {"name": "product_head_token_f16", "kind": "product", "N": 128257, "K": 4096, "batch": 1, "x": "f16", "y": "f32"},
        # a layer kept in 4 bits, a decoding batch in 8 bits
        {"name": "product_gate_up_e4m3", "kind": "product", "N": 28672, "K": 4096, "batch": 16, "x": "e4m3", "y": "bf16"},
        # the LM head over the drafted tokens of a batch
        {"name": "product_head_drafts_bf16", "kind": "product", "N": 32000, "K": 5120, "batch": 40, "x": "bf16", "y": "f32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "norm", "gate", "gate", "rotate", "rotate", "rotate", "product", "product", "product", "product"))
    if kind == "norm":
        heads = rng.choice((1, 1, 1, rng.randint(2, 48)))
        dim = _log_int(rng, 64, 16384) if heads == 1 else rng.choice((64, 96, 128, 256))
        out = rng.choice(("f16", "bf16", "f32", "e4m3"))
        if out == "e4m3":
            dim = -(-dim // 32) * 32
        return {"kind": kind, "rows": _log_int(rng, 1, 8192 * 5120 // (heads * dim)), "heads": heads, "dim": dim, "x": rng.choice(("f16", "bf16", "f32")),
                "residual": rng.choice(("f16", "bf16", "f32")) if heads == 1 else "", "out": out, "weight": rng.choice(("f16", "bf16", "f32"))}
    if kind == "gate":
        out = rng.choice(("f16", "bf16", "f32", "e4m3"))
        dim = _log_int(rng, 64, 28672)
        if out == "e4m3":
            dim = -(-dim // 32) * 32
        return {"kind": kind, "rows": _log_int(rng, 1, 4099 * 17408 // dim // 2), "dim": dim, "x": rng.choice(("f16", "bf16", "f32")), "out": out}
    if kind == "rotate":
        group, kvh, dim = rng.choice(((1, 4, 64), (4, 8, 128), (4, 8, 128), (5, 8, 128), (8, 8, 128), (3, 5, 96), (16, 1, 256), (2, 4, 160)))
        fmt = rng.choice(("f16", "bf16", "e4m3", "e4m3"))
        seqs = rng.randint(1, 16)
        new = _log_int(rng, 1, 24000 * 32 * 128 // (seqs * group * kvh * dim) // 2)
        return {"kind": kind, "fmt": fmt, "src": rng.choice(("f16", "bf16", "f32")), "out": fmt if fmt != "e4m3" else rng.choice(("f16", "bf16")), "seqs": seqs,
                "new": new, "ctx": new + _log_int(rng, 1, 500000), "heads": group * kvh, "kvh": kvh, "dim": dim, "page": rng.choice((16, 32, 64, 128, 256)),
                "rot": rng.choice((dim, dim, dim, 32)), "interleaved": rng.random() < 0.4}
    x, K = rng.choice(("f16", "bf16", "e4m3")), _log_int(rng, 64, 28672)
    if x == "e4m3":
        K = -(-K // 32) * 32
    return {"kind": kind, "N": _log_int(rng, 100, min(128257, 128257 * 4096 // K)), "K": K, "batch": rng.choice((1, 1, 2, 4, 8, 16, rng.randint(1, 16), rng.randint(17, 64))),
            "x": x, "y": rng.choice(("f32", "f32", "bf16", "f16"))}


# -- what a case's sequences are -------------------------------------------------
def _lengths(case):
    """(tokens so far, new tokens among them) of each sequence: the first has
    the case's own sizes, the others are shorter."""
    r = random.Random("%d %d %d" % (case["seqs"], case["new"], case["ctx"]))
    got = [(case["ctx"], case["new"])]
    for _ in range(case["seqs"] - 1):
        n = r.randint((case["new"] + 1) // 2, case["new"])
        old = case["ctx"] - case["new"]
        got.append((n + r.randint(old // 4, old), n))
    return got


# -- blocks of 32 that share a power of two, plainly --------------------------------
def _encode(x, fmt):
    """x [..., 32 n] fp32 as (codes, scale bytes): per block the smallest power
    of two (within the format's range) under which no code saturates, and x over
    it rounded to the nearest code, ties to even."""
    top, above, low, high = FORMAT[fmt]
    b = x.reshape(*x.shape[:-1], -1, 32)
    amax = b.abs().amax(-1)
    mant, power = torch.frexp(amax)
    e = torch.where(mant > top, power - above + 1, power - above)
    e = torch.where(amax == 0, torch.full_like(e, low), e).clamp(low, high)
    limit = top * 2.0 ** above
    y = torch.ldexp(b, -e.unsqueeze(-1)).clamp(-limit, limit).reshape(x.shape)
    scale = (e + 127).to(torch.uint8)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn), scale
    a = y.abs()
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, 2 + torch.round(a), 4 + torch.round(a / 2)))
    code = code.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _decode(codes, scale, dt=torch.float32):
    """The values that codes (E4M3 values, or bytes of two E2M1) and scale bytes stand for."""
    if codes.dtype == torch.float8_e4m3fn:
        y = codes.to(dt)
    else:
        table = torch.tensor([(a, b) for b in E2M1 + tuple(-v for v in E2M1) for a in E2M1 + tuple(-v for v in E2M1)], dtype=dt, device=codes.device)
        y = table[codes.long()].flatten(-2)
    unit = torch.ldexp(torch.ones((), dtype=dt, device=codes.device), scale.int() - 127)
    return (y.reshape(*y.shape[:-1], -1, 32) * unit.unsqueeze(-1)).reshape(y.shape)


def _scales(t):
    """Scale bytes as the powers of two that they are."""
    return t.view(torch.float8_e8m0fnu)


# -- inputs ----------------------------------------------------------------------------
def _values(gen, *shape):
    """Activations: normal, with channels of different strength."""
    x = torch.randn(shape, generator=gen, device=DEV)
    return x.mul_(0.25 + 1.5 * torch.rand(shape[-1:], generator=gen, device=DEV))


def _room(shape, kind):
    """An output of that type (8 bits: codes and scales)."""
    if kind != "e4m3":
        return torch.empty(shape, dtype=TYPES[kind], device=DEV), None
    return torch.empty(shape, dtype=torch.uint8, device=DEV), torch.empty((*shape[:-1], shape[-1] // 32), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = {"case": case}
    if case["kind"] == "norm":
        rows, heads, dim = case["rows"], case["heads"], case["dim"]
        if heads == 1:
            s["x"] = _values(gen, rows, dim).to(TYPES[case["x"]])
            shape = (rows, dim)
        else:  # the query heads of a fused projection's output: two heads more than the norm takes
            s["x"] = _values(gen, rows, heads + 2, dim).to(TYPES[case["x"]])[:, :heads]
            shape = (rows, heads, dim)
        s["weight"] = (0.5 + torch.rand(dim, generator=gen, device=DEV)).to(TYPES[case["weight"]])
        s["residual"] = (4 * _values(gen, *shape)).to(TYPES[case["residual"]]) if case["residual"] else None
        s["out"], s["out_scale"] = _room(shape, case["out"])
    elif case["kind"] == "gate":
        both = (2 * _values(gen, case["rows"], 2 * case["dim"])).to(TYPES[case["x"]])  # columns of one fused product
        s["gate"], s["up"] = both[:, :case["dim"]], both[:, case["dim"]:]
        s["out"], s["out_scale"] = _room((case["rows"], case["dim"]), case["out"])
    elif case["kind"] == "rotate":
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        lens, page = _lengths(case), case["page"]
        rows, H, V, D = sum(n for _, n in lens), case["heads"], case["kvh"], case["dim"]
        fused = _values(gen, rows, H + 2 * V, D).to(TYPES[case["src"]])
        s["q"], s["k"], s["v"] = fused[:, :H], fused[:, H:H + V], fused[:, H + V:]
        s["q_out"] = torch.empty((rows, H, D), dtype=TYPES[case["out"]], device=DEV)
        # pages for the positions that are written (what lies far behind a
        # window has been given back)
        first = [(c - n) // page for c, n in lens]
        need = [(c - 1) // page + 1 - f for (c, _), f in zip(lens, first)]
        order = torch.randperm(sum(need) + 3, generator=gen, device=DEV).int()
        table = torch.full((len(lens), max(f + k for f, k in zip(first, need))), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, (f, k) in enumerate(zip(first, need)):
            table[i, f:f + k] = order[at:at + k]
            at += k
        starts = [0]
        for _, n in lens:
            starts.append(starts[-1] + n)
        s.update(q_start=ints(starts), kv_len=ints([c for c, _ in lens]), page_table=table)
        s["freq"] = (500000.0 ** (-2.0 * torch.arange(case["rot"] // 2, dtype=torch.float64) / case["rot"])).float().to(DEV)
        shape = (sum(need) + 3, V, page, D)
        quant = case["fmt"] == "e4m3"
        for w in ("pool_k", "pool_v"):
            s[w] = torch.zeros(shape, dtype=torch.uint8 if quant else TYPES[case["fmt"]], device=DEV)
            s[w + "_scale"] = torch.full((*shape[:3], D // 32), 127, dtype=torch.uint8, device=DEV) if quant else None
    else:
        N, K, B = case["N"], case["K"], case["batch"]
        W = torch.zeros((N, -(-K // 32) * 32), device=DEV)
        W[:, :K] = torch.randn((N, K), generator=gen, device=DEV).mul_(K ** -0.5)
        s["codes"], s["scale"] = _encode(W, "e2m1")
        x = _values(gen, B, K)
        s["x"], s["x_scale"] = _encode(x, "e4m3") if case["x"] == "e4m3" else (x.to(TYPES[case["x"]]), None)
        s["y"] = torch.empty((B, N), dtype=TYPES[case["y"]], device=DEV)
    return s


# -- one pass ----------------------------------------------------------------------------
def run(s):
    return _kernels(s) if own else _plain(s)


def _kernels(s):
    import paper_2609_00224_amd as q

    case = s["case"]
    if case["kind"] == "norm":
        q.qtea_rms_norm(s["x"], s["weight"], s["out"], residual=s["residual"], eps=EPS, out_scale=s["out_scale"])
        return _dense(s)
    if case["kind"] == "gate":
        q.qtea_silu_mul(s["gate"], s["up"], s["out"], out_scale=s["out_scale"])
        return _dense(s)
    if case["kind"] == "rotate":
        if "program" not in s:  # a serving program's cache object
            s["program"] = q.KvCache(case["fmt"], s["pool_k"], s["pool_v"], s["pool_k_scale"], s["pool_v_scale"])
        q.qtea_kv_append_rotated(s["program"], s["q"], s["k"], s["v"], s["q_start"], s["kv_len"], s["page_table"], s["freq"], s["q_out"],
                                 interleaved=case["interleaved"])
        return _state(s)
    if "program" not in s:  # the weights, laid out once (their values are fp16 values)
        s["program"] = q.pack_matrix_w4(_decode(s["codes"], s["scale"], torch.float16)[:, :case["K"]])
        if case["x"] == "e4m3":
            s["x"] = s["x"].view(torch.uint8)
    q.qtea_w4_gemm_lowbatch(s["program"], s["x"], s["y"], x_scale=s["x_scale"])
    return {"y": s["y"]}


def _dense(s):
    got = {"out": s["out"]}
    if s["out_scale"] is not None:
        got = {"out": s["out"].view(torch.float8_e4m3fn), "scale": _scales(s["out_scale"])}
    if s.get("residual") is not None:
        got["residual"] = s["residual"]
    return got


def _state(s):
    """Rotated queries and the pools."""
    got = {"q": s["q_out"], "k": s["pool_k"], "v": s["pool_v"]}
    if s["case"]["fmt"] == "e4m3":
        got.update(k=s["pool_k"].view(torch.float8_e4m3fn), v=s["pool_v"].view(torch.float8_e4m3fn), k_scale=_scales(s["pool_k_scale"]), v_scale=_scales(s["pool_v_scale"]))
    return got


def _plain(s):
    case = s["case"]
    if case["kind"] == "norm":
        t = s["x"].float()
        if s["residual"] is not None:
            t = t + s["residual"].float()
            s["residual"].copy_(t)
        y = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
        return _plain_store(s, y)
    if case["kind"] == "gate":
        g = s["gate"].float()
        return _plain_store(s, g / (1 + torch.exp(-g)) * s["up"].float())
    if case["kind"] == "rotate":
        return _plain_rotate(s)
    x = s["x"].float() if s["x_scale"] is None else _decode(s["x"].view(torch.float8_e4m3fn), s["x_scale"])
    s["y"].copy_(x @ _decode(s["codes"], s["scale"])[:, :case["K"]].T)
    return {"y": s["y"]}


def _plain_store(s, y):
    if s["out_scale"] is None:
        s["out"].copy_(y)
    else:
        codes, scale = _encode(y, "e4m3")
        s["out"].copy_(codes.view(torch.uint8))
        s["out_scale"].copy_(scale)
    return _dense(s)


def _plain_rotate(s):
    case = s["case"]
    page, R = case["page"], case["rot"]
    r = torch.arange(s["q"].shape[0], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["q_start"], r, right=True) - 1
    pos = s["kv_len"][seq] - s["q_start"][seq + 1] + r
    pg, off = s["page_table"][seq, (pos // page).long()].long(), (pos % page).long()
    angle = pos.double()[:, None] * s["freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(x):
        y = x.float()
        if case["interleaved"]:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((turned, y[..., R:]), -1)

    s["q_out"].copy_(rotated(s["q"]))
    k, v = rotated(s["k"]), s["v"].float()
    if case["fmt"] == "e4m3":
        (k, ks), (v, vs) = _encode(k, "e4m3"), _encode(v, "e4m3")
        k, v = k.view(torch.uint8), v.view(torch.uint8)
        s["pool_k_scale"][pg, :, off], s["pool_v_scale"][pg, :, off] = ks, vs
    s["pool_k"][pg, :, off], s["pool_v"][pg, :, off] = k.to(s["pool_k"].dtype), v.to(s["pool_v"].dtype)
    return _state(s)


# -- floors ---------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "norm":
        n = case["rows"] * case["heads"] * case["dim"]
        return {"bytes": n * (SIZE[case["x"]] + 2 * SIZE[case["residual"]] + SIZE[case["out"]]) + case["dim"] * SIZE[case["weight"]], "flops": 5.0 * n}
    if case["kind"] == "gate":
        n = case["rows"] * case["dim"]
        return {"bytes": n * (2 * SIZE[case["x"]] + SIZE[case["out"]]), "flops": 5.0 * n}
    if case["kind"] == "rotate":
        lens = _lengths(case)
        rows = sum(n for _, n in lens)
        q, kv = rows * case["heads"] * case["dim"], 2 * rows * case["kvh"] * case["dim"]
        return {"bytes": q * (SIZE[case["src"]] + SIZE[case["out"]]) + kv * (SIZE[case["src"]] + SIZE[case["fmt"]]) + 2 * case["rot"] + 4 * (3 * len(lens) + 1),
                "flops": 3.0 * (q + kv / 2) * case["rot"] / case["dim"]}
    N, K, B = case["N"], case["K"], case["batch"]
    return {"bytes": N * K * 0.5 + N * (-(-K // 32)) + B * K * SIZE[case["x"]] + B * N * SIZE[case["y"]], "flops": 2.0 * B * N * K}


# -- the definitions in 64 bits ----------------------------------------------------------------
def _exact_blocks(x):
    """x [..., 32 n] fp64 in E4M3 blocks: (code values, units), each value the
    nearest of the ladder in units of its block, the even code on a tie."""
    steps = torch.tensor(([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])[:127], dtype=torch.float64, device=DEV)
    units = 2.0 ** torch.arange(-15, 8, dtype=torch.float64, device=DEV)
    b = x.reshape(*x.shape[:-1], -1, 32)
    unit = units[torch.searchsorted(units * steps[-1], b.abs().amax(-1).contiguous()).clamp(max=len(units) - 1)]
    a = (b.abs() / unit.unsqueeze(-1)).clamp(max=float(steps[-1]))
    mid = (steps[1:] + steps[:-1]) / 2
    lo, hi = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    return (torch.sign(b) * steps[torch.where(lo % 2 == 0, lo, hi)]).reshape(x.shape), unit


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "gate"):
        if case["kind"] == "norm":
            t = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
            y = t / (((t ** 2).sum(-1, keepdim=True) / case["dim"] + EPS) ** 0.5) * s["weight"].double()
        else:
            g = s["gate"].double()
            y = g * torch.sigmoid(g) * s["up"].double()
        got = {"out": y}
        if case["out"] == "e4m3":
            got["out"], got["scale"] = _exact_blocks(y)
        if s.get("residual") is not None:
            got["residual"] = t
        return got
    if case["kind"] == "product":
        values = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
        values = torch.cat((values, -values))
        W = torch.empty((case["N"], s["codes"].shape[1] * 2), dtype=torch.float64, device=DEV)
        W[:, 0::2], W[:, 1::2] = values[(s["codes"] & 15).long()], values[(s["codes"] >> 4).long()]
        W *= (2.0 ** (s["scale"].double() - 127)).repeat_interleave(32, 1)
        x = s["x"].double()
        if s["x_scale"] is not None:
            x = x * (2.0 ** (s["x_scale"].double() - 127)).repeat_interleave(32, 1)
        return {"y": x @ W[:, :case["K"]].T}
    lens, page, D, R = _lengths(case), case["page"], case["dim"], case["rot"]
    start = s["q_start"].tolist()
    quant = case["fmt"] == "e4m3"
    got = {"q": torch.empty((start[-1], case["heads"], D), dtype=torch.float64, device=DEV)}
    for w in ("k", "v"):
        got[w] = torch.zeros(s["pool_" + w].shape, dtype=torch.float64, device=DEV)
        if quant:
            got[w + "_scale"] = torch.ones(s["pool_" + w + "_scale"].shape, dtype=torch.float64, device=DEV)
    i = torch.arange(R // 2, device=DEV)
    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
    for n, (c, new) in enumerate(lens):
        rows = slice(start[n], start[n + 1])
        t = torch.arange(c - new, c, device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), t.double()[:, None] * s["freq"].double())[:, None]
        pg, off = s["page_table"][n].long()[t // page], t % page
        for w in ("q", "k", "v"):
            x = s[w][rows].double()
            if w != "v":
                z = torch.complex(x[..., a], x[..., b]) * turn
                x[..., a], x[..., b] = z.real, z.imag
            if w == "q":
                got["q"][rows] = x
            elif quant:
                code, unit = _exact_blocks(x)
                got[w][pg, :, off], got[w + "_scale"][pg, :, off] = code, unit
            else:
                got[w][pg, :, off] = x
    return got
