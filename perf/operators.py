"""The serving operators around the compressed products, as cases to time.

Four operators, each through the Python binding's entry points, over one
paged key/value cache:

  append   qtea_kv_append: new tokens' keys and values go to their sequences'
           pages, in 16 bits or quantized to blocks of 32 channels that share
           a power of two (E4M3 or E2M1 codes);
  refresh  the same and qtea_kv_read of the rows just written, which gives
           the values that the 8 or 4 bits stand for;
  read     qtea_kv_read: sequences of the cache as dense 16-bit rows;
  attn     qtea_paged_attention: causal attention of each sequence's newest
           tokens (one of them, a few drafted ones, a chunk of a prompt) over
           its pages, with grouped heads and an optional window;
  verify   qtea_verify_draft: drafted tokens against the target's
           probabilities, with given uniform numbers.

Head counts are those of the 8B-, 14B- and 70B-shaped decoders of
synth/workloads.py (32, 40 and 64 query heads over 8 key/value heads of 128
channels) and generic ones.  The sequences of a case have lengths of their
own, up to the case's, and their pages lie in the pool in a random order.

`own` chooses between the framework's kernels and the plain forms: elementary
torch operations in 32 bits, over all sequences at once (padded to the
longest).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
SOURCE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
WIDE = ("f16", "bf16")  # cache formats that hold 16-bit values as they are
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# per quantized format: the largest code's value as a fraction of the power
# of two above it, that power, and the range of a block's exponent (every
# value is then an fp16 value)
FORMAT = {"e4m3": (0.875, 9, -15, 7), "e2m1": (0.75, 3, -23, 13)}
FIXED = 2.0 ** 38  # a probability's unit in qtea_verify_draft


def listed():
    return [
        # the newest token of sixteen sequences (the largest batch of the
        # compressed products), straight from the products' fp32 output
        {"name": "append_tokens_e4m3", "kind": "append", "fmt": "e4m3", "src": "f32", "seqs": 16, "new": 1, "ctx": 2000, "kvh": 8, "dim": 128, "page": 64},
        # prompts of four sequences, quantized as they are written
        {"name": "append_prompts_e4m3", "kind": "append", "fmt": "e4m3", "src": "f16", "seqs": 4, "new": 8192, "ctx": 8192, "kvh": 8, "dim": 128, "page": 64},
        # ragged chunks in 4 bits, and the values that later steps will see
        {"name": "refresh_chunks_e2m1", "kind": "refresh", "fmt": "e2m1", "src": "bf16", "seqs": 7, "new": 999, "ctx": 5000, "kvh": 8, "dim": 128, "page": 32},
        # whole sequences fetched from an 8-bit cache
        {"name": "read_sequences_e4m3", "kind": "read", "fmt": "e4m3", "src": "f16", "seqs": 8, "new": 6000, "ctx": 6000, "kvh": 8, "dim": 128, "page": 64},
        # one token of one short conversation: where latency counts
        {"name": "attn_token_short_f16", "kind": "attn", "fmt": "f16", "src": "f16", "seqs": 1, "new": 1, "ctx": 700, "heads": 32, "kvh": 8, "dim": 128, "page": 16, "window": 0},
        # a full decoding batch over ragged histories in 8 bits
        {"name": "attn_tokens_e4m3", "kind": "attn", "fmt": "e4m3", "src": "f16", "seqs": 16, "new": 1, "ctx": 16000, "heads": 32, "kvh": 8, "dim": 128, "page": 64, "window": 0},
        # one token over a very long history in 4 bits, 70B heads
        {"name": "attn_token_long_e2m1", "kind": "attn", "fmt": "e2m1", "src": "f16", "seqs": 1, "new": 1, "ctx": 260001, "heads": 64, "kvh": 8, "dim": 128, "page": 128, "window": 0},
        # drafted tokens of four sequences, 14B heads (five to a group)
        {"name": "attn_drafts_bf16", "kind": "attn", "fmt": "bf16", "src": "bf16", "seqs": 4, "new": 6, "ctx": 9001, "heads": 40, "kvh": 8, "dim": 128, "page": 64, "window": 0},
        # a chunk of a long prompt over the part already cached
        {"name": "attn_chunk_e4m3", "kind": "attn", "fmt": "e4m3", "src": "f16", "seqs": 1, "new": 2048, "ctx": 12345, "heads": 32, "kvh": 8, "dim": 128, "page": 64, "window": 0},
        # whole prompts of different lengths, small heads, a sliding window
        {"name": "attn_prompts_bf16", "kind": "attn", "fmt": "bf16", "src": "bf16", "seqs": 6, "new": 4000, "ctx": 4000, "heads": 16, "kvh": 4, "dim": 64, "page": 16, "window": 1024},
        # one sequence's drafts
        {"name": "verify_one", "kind": "verify", "src": "f32", "seqs": 1, "drafts": 4, "vocab": 32000},
        # a batch of sequences, ragged drafts, a large odd vocabulary
        {"name": "verify_batch", "kind": "verify", "src": "f32", "seqs": 48, "drafts": 7, "vocab": 128257},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "refresh", "read", "attn", "attn", "attn", "attn", "attn", "verify", "verify"))
    if kind == "verify":
        return {"kind": kind, "src": rng.choice(("f32", "f32", "bf16", "f16")), "seqs": _log_int(rng, 1, 48),
                "drafts": rng.randint(1, 7), "vocab": _log_int(rng, 1000, 128257)}
    fmt = rng.choice(("f16", "bf16", "e4m3", "e4m3", "e2m1", "e2m1"))
    page = rng.choice((16, 32, 64, 128, 256))
    if kind != "attn":
        if kind == "append" and fmt == "e2m1":
            fmt = "e4m3"  # (4-bit codes come back as values: the other kinds)
        seqs, kvh, dim = rng.randint(1, 16), rng.choice((1, 2, 4, 5, 8)), rng.choice((64, 96, 128, 256))
        new = _log_int(rng, 1, 32768 * 8 * 128 // (seqs * kvh * dim) // 2)
        return {"kind": kind, "fmt": fmt, "src": fmt if fmt in WIDE else rng.choice(("f16", "bf16", "f32")), "seqs": seqs, "new": new,
                "ctx": new + rng.randint(0, 2000), "kvh": kvh, "dim": dim, "page": page}
    group, kvh, dim = rng.choice(((1, 4, 64), (4, 8, 128), (4, 8, 128), (5, 8, 128), (8, 8, 128), (3, 5, 96), (16, 1, 256), (2, 4, 256)))
    new = rng.choice((1, 1, 1, rng.randint(2, 16), rng.randint(2, 16), _log_int(rng, 17, 1500)))
    seqs = rng.randint(1, 16) if new <= 16 else rng.randint(1, 4)
    # (as many cached values as the largest listed batch, at most, and as many
    # products as the largest listed chunk)
    most = min(60000, 16 * 16000 * 8 * 128 // (seqs * kvh * dim)) if new <= 16 else min(12000, 2048 * 11000 * 32 * 128 // (seqs * new * group * kvh * dim))
    return {"kind": kind, "fmt": fmt, "src": fmt if fmt in WIDE else rng.choice(("f16", "bf16")), "seqs": seqs, "new": new,
            "ctx": new + _log_int(rng, 1, max(2, most - new)), "heads": group * kvh, "kvh": kvh, "dim": dim, "page": page,
            "window": rng.choice((0, 0, 0, 500, 2000))}


# -- what a case's sequences are -------------------------------------------
def _lengths(case):
    """(cached tokens, new tokens among them) of each sequence: the first has
    the case's own sizes, the others are shorter."""
    r = random.Random("%d %d %d" % (case["seqs"], case["new"], case["ctx"]))
    got = [(case["ctx"], case["new"])]
    for _ in range(case["seqs"] - 1):
        n = r.randint((case["new"] + 1) // 2, case["new"])
        old = case["ctx"] - case["new"]
        got.append((n + r.randint(old // 4, old), n))
    return got


def _drafts(case):
    r = random.Random("%d %d" % (case["seqs"], case["drafts"]))
    return [case["drafts"]] + [r.randint(0, case["drafts"]) for _ in range(case["seqs"] - 1)]


def _starts(counts):
    got = [0]
    for n in counts:
        got.append(got[-1] + n)
    return got


def _row_bytes(fmt, dim):
    """Bytes of one token's key (or value) of one head in the cache."""
    return {"f16": 2 * dim, "bf16": 2 * dim, "e4m3": dim + dim // 32, "e2m1": dim // 2 + dim // 32}[fmt]


# -- the cache format, plainly ----------------------------------------------
def _encode(x, fmt):
    """x [..., dim] fp32 as (codes, scales): per block of 32 channels the
    smallest power of two (within the format's range) under which no code
    saturates, and x over it rounded to the nearest code, ties to even."""
    if fmt in WIDE:
        return x.to(SOURCE[fmt]), None
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
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scale
    a = y.abs()
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, 2 + torch.round(a), 4 + torch.round(a / 2)))
    code = code.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _decode(codes, scale, fmt):
    """The values of _encode's result, fp32."""
    if fmt in WIDE:
        return codes.float()
    if fmt == "e4m3":
        y = codes.view(torch.float8_e4m3fn).float()
    else:
        nib = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
        y = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)[nib]
    b = y.reshape(*y.shape[:-1], -1, 32)
    return torch.ldexp(b, (scale.int() - 127).unsqueeze(-1)).reshape(y.shape)


# -- inputs ------------------------------------------------------------------
def _values(gen, *shape):
    """Keys or values: normal, with channels of different strength."""
    x = torch.randn(shape, generator=gen, device=DEV)
    return x.mul_(0.5 + torch.rand(shape[-2:], generator=gen, device=DEV))


def _pool(gen, pages, case):
    """A pool of cached keys or values, and its scales: pages with earlier
    contents, a slab of pages at a time."""
    fmt, shape = case["fmt"], (case["kvh"], case["page"], case["dim"])
    codes = scale = None
    slab = max(1, (1 << 26) // (shape[0] * shape[1] * shape[2]))
    strength = 0.5 + torch.rand((shape[0], 1, shape[2]), generator=gen, device=DEV)
    for p in range(0, pages, slab):
        c, s = _encode(torch.randn((min(slab, pages - p), *shape), generator=gen, device=DEV).mul_(strength), fmt)
        if codes is None:
            codes = torch.empty((pages, *c.shape[1:]), dtype=c.dtype, device=DEV)
            scale = None if s is None else torch.empty((pages, *s.shape[1:]), dtype=s.dtype, device=DEV)
        codes[p:p + slab] = c
        if s is not None:
            scale[p:p + slab] = s
    return codes, scale


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = {"case": case}
    if case["kind"] == "verify":
        n = _drafts(case)
        rows, V = sum(n), case["vocab"]
        # the draft model's distribution is the target's, blurred
        target = torch.empty((rows + len(n), V), dtype=SOURCE[case["src"]], device=DEV)
        draft = torch.empty((rows, V), dtype=SOURCE[case["src"]], device=DEV)
        tokens = torch.empty(rows, dtype=torch.int32, device=DEV)
        at = 0
        for i, k in enumerate(n):
            logits = 3.0 * torch.randn((k + 1, V), generator=gen, device=DEV)
            target[at + i:at + i + k + 1] = torch.softmax(logits, -1)
            blur = torch.softmax(logits[:k] + 0.5 * torch.randn((k, V), generator=gen, device=DEV), -1)
            draft[at:at + k] = blur
            if k:
                tokens[at:at + k] = torch.multinomial(blur, 1, generator=gen).flatten().int()
            at += k
        s.update(target=target, draft=draft, tokens=tokens, q_start=ints(_starts([k + 1 for k in n])),
                 u_accept=torch.rand(rows, generator=gen, device=DEV), u_sample=torch.rand(len(n), generator=gen, device=DEV),
                 n_accepted=torch.empty(len(n), dtype=torch.int32, device=DEV),
                 out_tokens=torch.empty((len(n), case["drafts"] + 1), dtype=torch.int32, device=DEV))
        return s
    lens = _lengths(case)
    need = [-(-c // case["page"]) for c, _ in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    s["k"], s["k_scale"] = _pool(gen, pages, case)
    s["v"], s["v_scale"] = _pool(gen, pages, case)
    s.update(q_start=ints(_starts([n for _, n in lens])), kv_len=ints([c for c, _ in lens]), page_table=table)
    rows = sum(n for _, n in lens)
    src = SOURCE[case["src"]]
    if case["kind"] == "attn":
        s["q"] = _values(gen, rows, case["heads"], case["dim"]).to(src)
        s["out"] = torch.empty_like(s["q"])
    if case["kind"] in ("append", "refresh"):
        # columns of one fused projection's output
        both = _values(gen, rows, 2 * case["kvh"], case["dim"]).to(src)
        s["new_k"], s["new_v"] = both[:, :case["kvh"]], both[:, case["kvh"]:]
    if case["kind"] in ("refresh", "read"):
        dense = (rows, case["kvh"], case["dim"])
        to = torch.bfloat16 if case["src"] == "bf16" else torch.float16
        s["dense_k"], s["dense_v"] = (torch.empty(dense, dtype=to, device=DEV) for _ in range(2))
    return s


# -- one pass ------------------------------------------------------------------
def run(s):
    return _kernels(s) if own else _plain(s)


def _kernels(s):
    import paper_2609_00224_amd as q

    case = s["case"]
    kind = case["kind"]
    if "program" not in s:  # what a serving program makes once: its cache object and its workspace
        if kind == "verify":
            s["program"] = q.new_verify_workspace(case["seqs"], DEV)
        else:
            s["program"] = (q.KvCache(case["fmt"], s["k"], s["v"], s["k_scale"], s["v_scale"]),
                            q.new_attention_workspace(case["heads"], case["dim"], DEV) if kind == "attn" else None)
    if kind == "verify":
        q.qtea_verify_draft(s["target"], s["draft"], s["tokens"], s["q_start"], s["u_accept"], s["u_sample"],
                            s["n_accepted"], s["out_tokens"], s["program"])
        return {"accepted": s["n_accepted"], "tokens": s["out_tokens"]}
    cache, ws = s["program"]
    if kind == "attn":
        q.qtea_paged_attention(cache, s["q"], s["q_start"], s["kv_len"], s["page_table"], s["out"], ws, window=case["window"])
        return {"out": s["out"]}
    if kind != "read":
        q.qtea_kv_append(cache, s["new_k"], s["new_v"], s["q_start"], s["kv_len"], s["page_table"])
    if kind == "append":
        return _state(s)
    q.qtea_kv_read(cache, s["q_start"], s["kv_len"], s["page_table"], s["dense_k"], s["dense_v"])
    return {"k": s["dense_k"], "v": s["dense_v"]}


def _state(s):
    """The cache after an append (E4M3 codes as their values)."""
    if s["case"]["fmt"] == "e4m3":
        return {"k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return {"k": s["k"], "v": s["v"]}


def _places(s, rows):
    """(page, offset) of every new row."""
    page = s["case"]["page"]
    r = torch.arange(rows, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["q_start"], r, right=True) - 1
    pos = s["kv_len"][seq] - s["q_start"][seq + 1] + r
    return s["page_table"][seq, (pos // page).long()].long(), (pos % page).long()


def _plain(s):
    kind, fmt = s["case"]["kind"], s["case"]["fmt"] if "fmt" in s["case"] else None
    if kind == "verify":
        return _plain_verify(s)
    if kind == "attn":
        return _plain_attention(s)
    pg, off = _places(s, (s["new_k"] if kind != "read" else s["dense_k"]).shape[0])
    if kind != "read":
        k, ks = _encode(s["new_k"].float(), fmt)
        v, vs = _encode(s["new_v"].float(), fmt)
        s["k"][pg, :, off], s["v"][pg, :, off] = k, v
        if ks is not None:
            s["k_scale"][pg, :, off], s["v_scale"][pg, :, off] = ks, vs
    if kind == "append":
        return _state(s)
    scales = (None, None) if fmt in WIDE else (s["k_scale"][pg, :, off], s["v_scale"][pg, :, off])
    s["dense_k"].copy_(_decode(s["k"][pg, :, off], scales[0], fmt))
    s["dense_v"].copy_(_decode(s["v"][pg, :, off], scales[1], fmt))
    return {"k": s["dense_k"], "v": s["dense_v"]}


def _gather(codes, scale, table, length, fmt):
    """A pool's rows of all sequences, [seqs][kv heads][longest][dim] fp32,
    zero past a sequence's end."""
    at = table.clamp(min=0).long()
    x = _decode(codes[at], None if scale is None else scale[at], fmt)  # [seqs][pages][heads][page][dim]
    x = x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], x.shape[2], -1, x.shape[4])
    t = torch.arange(x.shape[2], device=DEV)
    return torch.where((t < length[:, None])[:, None, :, None], x, 0.0)


def _plain_attention(s):
    case = s["case"]
    H, G, D = case["kvh"], case["heads"] // case["kvh"], case["dim"]
    n = s["q_start"][1:] - s["q_start"][:-1]
    S, T = case["seqs"], case["new"]
    k = _gather(s["k"], s["k_scale"], s["page_table"], s["kv_len"], case["fmt"])
    v = _gather(s["v"], s["v_scale"], s["page_table"], s["kv_len"], case["fmt"])
    i = torch.arange(T, device=DEV)
    row = (s["q_start"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1).long()  # [S][T]
    q = s["q"][row].float().reshape(S, T, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * T, D)
    score = torch.matmul(q, k.transpose(2, 3)).mul_(D ** -0.5).reshape(S, H, G, T, -1)
    pos = (s["kv_len"] - n)[:, None] + i  # [S][T]
    t = torch.arange(k.shape[2], device=DEV)
    seen = t <= pos[..., None]
    if case["window"]:
        seen &= t > pos[..., None] - case["window"]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(S, H, G * T, -1), v).reshape(S, H, G, T, D) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(S, T, H * G, D).to(s["q"].dtype)
    s["out"].copy_(o[i < n[:, None]])
    return {"out": s["out"]}


def _fixed(p):
    """Probabilities in whole units of 2^-38 (floor)."""
    return torch.floor(torch.nan_to_num(p.float()).clamp(0.0, 1.0) * FIXED).long()


def _plain_verify(s):
    case = s["case"]
    S, K, V = case["seqs"], case["drafts"], case["vocab"]
    start = s["q_start"][:-1].long()
    n = s["q_start"][1:].long() - start - 1
    at = start - torch.arange(S, device=DEV)  # first draft row
    i = torch.arange(K, device=DEV)
    valid = i < n[:, None]
    d = (at[:, None] + i).clamp(max=s["draft"].shape[0] - 1)
    t = (start[:, None] + i).clamp(max=s["target"].shape[0] - 1)
    x = s["tokens"][d].long()
    u = torch.floor(s["u_accept"] * 2.0 ** 24).long()[d]
    ok = (u * _fixed(s["draft"][d, x]) < (_fixed(s["target"][t, x]) << 24)) & valid
    acc = ok.long().cumprod(1).sum(1)
    p = _fixed(s["target"][start + acc])
    dr = (at + acc).clamp(max=s["draft"].shape[0] - 1)
    w = (p - torch.where((acc < n)[:, None], _fixed(s["draft"][dr]), 0)).clamp(min=0)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p)
    total = w.sum(1)
    r = (torch.floor(s["u_sample"] * 2.0 ** 24).long() * total) >> 24
    token = (w.cumsum(1) <= r[:, None]).sum(1)
    token = torch.where(total > 0, token, -1)
    j = torch.arange(K + 1, device=DEV)
    padded = torch.cat((x, x[:, :1]), 1)
    out = torch.where(j < acc[:, None], padded, torch.where(j == acc[:, None], token[:, None], -1))
    s["n_accepted"].copy_(acc)
    s["out_tokens"].copy_(out)
    return {"accepted": s["n_accepted"], "tokens": s["out_tokens"]}


# -- floors ----------------------------------------------------------------------
def work(case):
    if case["kind"] == "verify":
        # a target row each, the draft's row where one is rejected (about one
        # draft in five is), and two values per draft
        n = _drafts(case)
        size = 4 if case["src"] == "f32" else 2
        rows = sum(1 + (1 - 0.8 ** k) for k in n)
        return {"bytes": rows * case["vocab"] * size + sum(n) * (2 * size + 8) + 4 * case["seqs"] * (case["drafts"] + 4),
                "flops": 3.0 * rows * case["vocab"]}
    lens = _lengths(case)
    rows = sum(n for _, n in lens)
    cached = 2 * case["kvh"] * _row_bytes(case["fmt"], case["dim"])  # of one token
    meta = 4 * (2 * len(lens) + 1)
    if case["kind"] == "attn":
        win = case["window"] or case["ctx"]
        read = sum(min(c, n + win - 1) for c, n in lens)
        pairs = sum(min(c - n + i + 1, win) for c, n in lens for i in range(n))
        qo = 2 * rows * case["heads"] * case["dim"] * 2
        return {"bytes": float(read * cached + qo + meta + 4 * (read // case["page"])), "flops": 4.0 * pairs * case["heads"] * case["dim"]}
    per = 2 * case["kvh"] * case["dim"]  # values of one token
    size = 4 if case["src"] == "f32" else 2
    moved = {"append": per * size + cached, "refresh": per * size + cached + 2 * per, "read": cached + 2 * per}[case["kind"]]
    return {"bytes": float(rows * moved + meta), "flops": float(3 * rows * per)}


# -- the definitions in 64 bits -----------------------------------------------------
def _ladder(fmt):
    """A quantized format's non-negative code values, ascending."""
    if fmt == "e2m1":
        return list(E2M1)
    return [m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127]


def _exact_quantized(x, fmt):
    """x [..., dim] fp64: (code values, block units), each value the nearest
    of the ladder in units of its block, the even code on a tie."""
    steps = torch.tensor(_ladder(fmt), dtype=torch.float64, device=DEV)
    top, above, low, high = FORMAT[fmt]
    b = x.reshape(*x.shape[:-1], -1, 32)
    units = 2.0 ** torch.arange(low, high + 1, dtype=torch.float64, device=DEV)
    pick = torch.searchsorted(units * steps[-1], b.abs().amax(-1).contiguous()).clamp(max=len(units) - 1)
    unit = units[pick].unsqueeze(-1)
    a = (b.abs() / unit).clamp(max=float(steps[-1]))
    mid = (steps[1:] + steps[:-1]) / 2
    lo, hi = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    code = torch.where(lo % 2 == 0, lo, hi)
    return (torch.sign(b) * steps[code]).reshape(x.shape), unit


def _exact_rows(s, case, which):
    """The new rows' quantized values (in units of their blocks) and units, or the rows themselves."""
    x = s[which].double()
    if case["fmt"] in WIDE:
        return x, None
    return _exact_quantized(x, case["fmt"])


def exact(case, seed):
    if case["kind"] == "verify":
        return None  # whole numbers
    s = prepare(case, seed)
    lens, page = _lengths(case), case["page"]
    start = s["q_start"].tolist()
    where = []  # (page, offset) of each new row
    for i, (c, n) in enumerate(lens):
        t = torch.arange(c - n, c, device=DEV)
        where.append((s["page_table"][i].long()[t // page], t % page))

    def values(codes, scale):
        if scale is None:
            return codes.double()
        if case["fmt"] == "e4m3":
            y = torch.tensor(_ladder("e4m3") + [math.nan], dtype=torch.float64, device=DEV)[(codes & 127).long()] * (1 - 2 * (codes >> 7).double())
        else:
            flat = torch.empty((*codes.shape[:-1], codes.shape[-1] * 2), dtype=torch.uint8, device=DEV)
            flat[..., 0::2], flat[..., 1::2] = codes & 15, codes >> 4
            y = torch.tensor(E2M1, dtype=torch.float64, device=DEV)[(flat & 7).long()] * (1 - 2 * (flat >> 3).double())
        return (y.reshape(*y.shape[:-1], -1, 32) * 2.0 ** (scale.double() - 127).unsqueeze(-1)).reshape(y.shape)

    if case["kind"] == "append":
        got = {}
        for which in ("k", "v"):
            x, _ = _exact_rows(s, case, "new_" + which)
            pool = s[which].view(torch.float8_e4m3fn).double() if case["fmt"] == "e4m3" else s[which].double()
            for i, (pg, off) in enumerate(where):
                pool[pg, :, off] = x[start[i]:start[i + 1]]
            got[which] = pool
        return {**got, "k_scale": None, "v_scale": None} if case["fmt"] == "e4m3" else got
    if case["kind"] == "refresh":
        got = {}
        for which in ("k", "v"):
            x, unit = _exact_rows(s, case, "new_" + which)
            got[which] = x if unit is None else (x.reshape(*x.shape[:-1], -1, 32) * unit).reshape(x.shape)
        return got
    if case["kind"] == "read":
        return {w: torch.cat([values(s[w][pg, :, off], None if s[w + "_scale"] is None else s[w + "_scale"][pg, :, off]) for pg, off in where]) for w in ("k", "v")}
    H, G, D = case["kvh"], case["heads"] // case["kvh"], case["dim"]
    out = torch.zeros((start[-1], case["heads"], D), dtype=torch.float64, device=DEV)
    for i, (c, n) in enumerate(lens):
        t = torch.arange(c, device=DEV)
        pg = s["page_table"][i].long()[t // page]
        pos = torch.arange(c - n, c, device=DEV)
        hidden = t[None] > pos[:, None]
        if case["window"]:
            hidden |= t[None] <= pos[:, None] - case["window"]
        for h in range(H):
            k, v = (values(s[w][pg, h, t % page], None if s[w + "_scale"] is None else s[w + "_scale"][pg, h, t % page]) for w in ("k", "v"))
            for g in range(G):
                a = (s["q"][start[i]:start[i + 1], h * G + g].double() @ k.T) / math.sqrt(D)
                out[start[i]:start[i + 1], h * G + g] = torch.softmax(a.masked_fill(hidden, -math.inf), -1) @ v
    return {"out": out}
