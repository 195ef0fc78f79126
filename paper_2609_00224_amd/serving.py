"""Serving operators of libqtea.so (include/qtea_serve.h): a paged key/value
cache in 16, 8 or 4 bits with the rotation of queries and keys by their
positions, causal attention of a batch's newest tokens over it, and the
verification of drafted tokens.

As the rest of the binding, these functions marshal arguments only; every
step runs in the kernels of ``csrc/kv_cache.hip``, ``csrc/paged_attn.hip`` and
``csrc/verify.hip``.  They are exported by the package itself, which imports
this module when the first of them is asked for.
"""
from __future__ import annotations

import ctypes

import torch

import paper_2609_00224_amd as _q
from paper_2609_00224_amd import KV_FORMATS, QTEA_BF16, QTEA_F16, QTEA_F32, QTEA_KV_BLOCK, QteaKvBatch, QteaKvCache

_i64 = ctypes.c_int64

_TYPES = {torch.float16: QTEA_F16, torch.bfloat16: QTEA_BF16, torch.float32: QTEA_F32}
_I32, _F32 = torch.int32, torch.float32


def _int(n):
    """A count as the C int that it is passed as: past its range the largest one,
    which the entry points refuse."""
    return min(n, 0x7fffffff)


def _type(t, what):
    got = _TYPES.get(t.dtype)
    if got is None:
        raise ValueError(f"{what}: fp16, bf16 or fp32, got {t.dtype}")
    return got


def _stream(stream, device):
    """The handle of `stream`, or of the device's current one (asked for
    without making a torch.cuda.Stream of it, which takes 2.5 us)."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _call(name, device, stream, *args):
    """The entry point on tensors of `device`, which is the current device for
    the call: a kernel is launched, and its workgroups counted, there."""
    fn = getattr(_q.load(), name)
    if torch.cuda.device_count() < 2 or torch.cuda.current_device() == device:
        rc = fn(*args, _stream(stream, device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream(stream, device))
    _q._check(rc, name)


class KvCache:
    """A paged cache's pools: k and v [n_pages][n_heads][page_size][head_dim]
    (fp16 or bf16; uint8 E4M3 codes; uint8 pairs of E2M1 codes, head_dim / 2
    bytes), with k_scale and v_scale uint8 [n_pages][n_heads][page_size]
    [head_dim / 32] for the quantized formats."""

    def __init__(self, fmt, k, v, k_scale=None, v_scale=None):
        if fmt not in KV_FORMATS:
            raise ValueError(f"cache format {fmt!r}: one of {', '.join(KV_FORMATS)}")
        want = {"f16": torch.float16, "bf16": torch.bfloat16}.get(fmt, torch.uint8)
        quant = want == torch.uint8
        tensors = (k, v, k_scale, v_scale) if quant else (k, v)
        if any(t is None for t in tensors) or (not quant and (k_scale is not None or v_scale is not None)):
            raise ValueError("quantized caches have k_scale and v_scale, 16-bit ones do not")
        if k.dim() != 4 or k.shape != v.shape or k.dtype != want or v.dtype != want:
            raise ValueError(f"k and v: {want}, [pages][heads][page size][channels]")
        self.fmt, self.k, self.v, self.k_scale, self.v_scale = fmt, k, v, k_scale, v_scale
        self.n_pages, self.n_heads, self.page_size, row = k.shape
        self.head_dim = 2 * row if fmt == "e2m1" else row
        if quant and not all(t.dtype == torch.uint8 and tuple(t.shape) == (*k.shape[:3], self.head_dim // QTEA_KV_BLOCK) for t in (k_scale, v_scale)):
            raise ValueError("k_scale and v_scale: uint8, [pages][heads][page size][channels / 32]")
        for t in tensors:
            if not t.is_contiguous():
                raise ValueError("qtea entry points take contiguous tensors")
            if not t.is_cuda or t.device != k.device:
                raise ValueError("qtea entry points take device tensors, a cache's of one device")
        self.device_index = k.get_device()
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.desc = QteaKvCache(ptr(k), ptr(v), ptr(k_scale), ptr(v_scale), self.n_pages, KV_FORMATS[fmt], self.n_heads,
                                self.head_dim, self.page_size)


def new_kv_cache(fmt, n_pages, page_size, n_heads, head_dim, device="cuda") -> KvCache:
    """A cache of zeros."""
    if fmt not in KV_FORMATS:
        raise ValueError(f"cache format {fmt!r}: one of {', '.join(KV_FORMATS)}")
    shape = (n_pages, n_heads, page_size)
    if fmt in ("f16", "bf16"):
        dt = torch.float16 if fmt == "f16" else torch.bfloat16
        return KvCache(fmt, *(torch.zeros((*shape, head_dim), dtype=dt, device=device) for _ in range(2)))
    row = head_dim // 2 if fmt == "e2m1" else head_dim
    new = lambda n: torch.zeros((*shape, n), dtype=torch.uint8, device=device)  # noqa: E731
    return KvCache(fmt, new(row), new(row), new(head_dim // QTEA_KV_BLOCK), new(head_dim // QTEA_KV_BLOCK))


def _batch(cache, rows, q_start, kv_len, page_table):
    if q_start.dtype is not _I32 or kv_len.dtype is not _I32 or page_table.dtype is not _I32:
        raise ValueError("q_start, kv_len and page_table are int32")
    n, table = kv_len.numel(), page_table.shape
    if q_start.numel() != n + 1 or len(table) != 2 or table[0] != n:
        raise ValueError("q_start has one entry more than kv_len, page_table one row per entry of it")
    if not (q_start.is_contiguous() and kv_len.is_contiguous() and page_table.is_contiguous()):
        raise ValueError("qtea entry points take contiguous tensors")
    if not (q_start.get_device() == kv_len.get_device() == page_table.get_device() == cache.device_index):
        raise ValueError("qtea entry points take tensors of the cache's device")
    return QteaKvBatch(q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), rows, n, table[1])


def _rows(cache, t, heads, what):
    """A dense operand [tokens][heads][channels]: the stride of its tokens (of
    one token it is not used, whatever the view has)."""
    shape, stride, dim = t.shape, t.stride(), cache.head_dim
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{what}: [tokens][{heads}][{dim}], got {list(shape)}")
    if stride[2] != 1 or (stride[1] != dim and heads > 1):
        raise ValueError(f"{what}: a token's heads and channels are contiguous")
    if t.get_device() != cache.device_index:
        raise ValueError(f"{what}: a tensor of the cache's device")
    return heads * dim if shape[0] <= 1 else stride[0]


def _dense(name, cache, k, v, q_start, kv_len, page_table, stream):
    ks, vs = _rows(cache, k, cache.n_heads, "k"), _rows(cache, v, cache.n_heads, "v")
    if k.dtype != v.dtype or k.shape[0] != v.shape[0]:
        raise ValueError("k and v: one type, one number of tokens")
    b = _batch(cache, k.shape[0], q_start, kv_len, page_table)
    if k.shape[0] == 0:
        return
    _call(name, cache.device_index, stream, cache.desc, b, k.data_ptr(), v.data_ptr(), _type(k, "k and v"), ks, vs)


def qtea_kv_append(cache: KvCache, k, v, q_start, kv_len, page_table, stream=None):
    """Write the batch's new keys and values, [tokens][n_heads][head_dim]
    (fp16, bf16 or fp32; a token's part contiguous, tokens any stride), at
    their sequences' ends (kv_len already counts them)."""
    _dense("qtea_kv_append", cache, k, v, q_start, kv_len, page_table, stream)


def qtea_kv_append_rotated(cache: KvCache, Q, k, v, q_start, kv_len, page_table, freq, q_out, interleaved: bool = False, stream=None):
    """qtea_kv_append with queries and keys turned by their positions on the
    way: Q [tokens][n_q_heads][head_dim] (of k's type) goes to q_out (the same
    shape, fp16, bf16 or fp32; Q itself for in place), k to the cache, v as it
    is.  freq: fp32 [rot_dim / 2], the angle of a pair per position; pairs are
    channels i and i + rot_dim / 2, or interleaved 2i and 2i + 1; channels from
    rot_dim on are not turned.  Q and q_out may be None: keys and values only."""
    ks, vs = _rows(cache, k, cache.n_heads, "k"), _rows(cache, v, cache.n_heads, "v")
    n = k.shape[0]
    if k.dtype != v.dtype or v.shape[0] != n:
        raise ValueError("k and v: one type, one number of tokens")
    if freq.dtype is not _F32 or not freq.is_contiguous() or freq.get_device() != cache.device_index:
        raise ValueError("freq: contiguous fp32 of the cache's device")
    heads = qs = os_ = kind = 0
    if (Q is None) != (q_out is None):
        raise ValueError("Q and q_out come together")
    if Q is not None:
        heads = Q.shape[1] if Q.dim() == 3 else 0
        qs, os_, kind = _rows(cache, Q, heads, "Q"), _rows(cache, q_out, heads, "q_out"), _type(q_out, "q_out")
        if Q.dtype != k.dtype or Q.shape[0] != n or q_out.shape[0] != n or heads == 0:
            raise ValueError("Q, k and v: one type; Q, q_out, k and v: one number of tokens")
    b = _batch(cache, n, q_start, kv_len, page_table)
    if n == 0:
        return
    _call("qtea_kv_append_rotated", cache.device_index, stream, cache.desc, b, None if Q is None else Q.data_ptr(), k.data_ptr(), v.data_ptr(),
          _type(k, "k and v"), qs, ks, vs, _int(heads), freq.data_ptr(), _int(2 * freq.numel()), bool(interleaved), None if Q is None else q_out.data_ptr(), kind, os_)


def qtea_kv_read(cache: KvCache, q_start, kv_len, page_table, k, v, stream=None):
    """Read the batch's rows (each sequence's last q_start[s+1] - q_start[s]
    positions) into k and v, [tokens][n_heads][head_dim]."""
    _dense("qtea_kv_read", cache, k, v, q_start, kv_len, page_table, stream)


def qtea_attention_workspace_bytes(n_q_heads: int, head_dim: int) -> int:
    q, out = _q, _i64(0)
    q._check(q.load().qtea_attention_workspace_bytes(int(n_q_heads), int(head_dim), ctypes.byref(out)), "qtea_attention_workspace_bytes")
    return out.value


def new_attention_workspace(n_q_heads: int, head_dim: int, device="cuda"):
    """A zero-filled workspace for qtea_paged_attention on `device`."""
    with torch.cuda.device(device):
        return torch.zeros(qtea_attention_workspace_bytes(n_q_heads, head_dim), dtype=torch.uint8, device=device)


def qtea_paged_attention(cache: KvCache, Q, q_start, kv_len, page_table, out, workspace, scale=None, window: int = 0, stream=None):
    """Causal attention of the batch's new tokens, Q [tokens][n_q_heads]
    [head_dim] (fp16 or bf16), over the cache that already holds them, into
    `out` (as Q).  scale: 1 / sqrt(head_dim) unless given; window: positions a
    row sees, 0 for all (a number past the C type's is passed as its largest)."""
    if Q.dim() != 3 or Q.shape != out.shape or Q.dtype != out.dtype:
        raise ValueError("Q and out: one type, one shape [tokens][heads][channels]")
    heads = Q.shape[1]
    qs, os_ = _rows(cache, Q, heads, "Q"), _rows(cache, out, heads, "out")
    b = _batch(cache, Q.shape[0], q_start, kv_len, page_table)
    if workspace.get_device() != cache.device_index or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous tensor of the cache's device")
    if Q.shape[0] == 0:
        return
    _call("qtea_paged_attention", cache.device_index, stream, cache.desc, b, Q.data_ptr(), out.data_ptr(), _type(Q, "Q and out"), heads, qs, os_,
          cache.head_dim ** -0.5 if scale is None else scale, max(-1, min(window, 0x7fffffff)), workspace.data_ptr(),
          workspace.numel() * workspace.element_size())


def qtea_verify_workspace_bytes(n_seq: int) -> int:
    q, out = _q, _i64(0)
    q._check(q.load().qtea_verify_workspace_bytes(int(n_seq), ctypes.byref(out)), "qtea_verify_workspace_bytes")
    return out.value


def new_verify_workspace(n_seq: int, device="cuda"):
    """A zero-filled workspace for qtea_verify_draft."""
    return torch.zeros(qtea_verify_workspace_bytes(n_seq), dtype=torch.uint8, device=device)


def qtea_verify_draft(target, draft, tokens, q_start, u_accept, u_sample, n_accepted, out_tokens, workspace, stream=None):
    """Which drafted tokens each sequence keeps, and its next token.

    target [rows][vocab] and draft [drafts][vocab] (fp16, bf16 or fp32
    probabilities; draft may be None: deterministic drafts), tokens int32 and
    u_accept fp32 [drafts], q_start int32 [n_seq + 1] over the target's rows,
    u_sample fp32 [n_seq]; outputs n_accepted int32 [n_seq] and out_tokens
    int32 [n_seq][max_draft + 1]."""
    n_seq, n_drafts = u_sample.numel(), tokens.numel()
    if target.dim() != 2 or (target.stride(1) != 1 and target.shape[1] > 1):
        raise ValueError("target: [rows][vocab], a row contiguous")
    vocab = target.shape[1]
    if draft is not None and (draft.dim() != 2 or tuple(draft.shape) != (n_drafts, vocab) or draft.dtype != target.dtype or (draft.stride(1) != 1 and vocab > 1 and n_drafts > 0)):
        raise ValueError("draft: a row of the target's type and vocabulary for each drafted token")
    if (tokens.dtype is not _I32 or q_start.dtype is not _I32 or n_accepted.dtype is not _I32 or out_tokens.dtype is not _I32
            or u_accept.dtype is not _F32 or u_sample.dtype is not _F32):
        raise ValueError("tokens, q_start, n_accepted and out_tokens are int32, u_accept and u_sample fp32")
    if q_start.numel() != n_seq + 1 or n_accepted.numel() != n_seq or u_accept.numel() != n_drafts or out_tokens.dim() != 2 or out_tokens.shape[0] != n_seq or out_tokens.shape[1] < 1:
        raise ValueError("one u_sample, n_accepted and row of out_tokens per sequence, one u_accept per draft, one q_start more than sequences")
    dev = target.get_device()
    if dev < 0 or (draft is not None and draft.get_device() != dev):
        raise ValueError("qtea entry points take device tensors, one call's of one device")
    for t in (tokens, q_start, u_accept, u_sample, n_accepted, out_tokens, workspace):
        if not t.is_contiguous():
            raise ValueError("qtea entry points take contiguous tensors")
        if t.get_device() != dev:
            raise ValueError("qtea entry points take device tensors, one call's of one device")
    if n_seq == 0:
        return
    one = lambda t: max(t.stride(0), vocab) if t.shape[0] <= 1 else t.stride(0)  # noqa: E731
    _call("qtea_verify_draft", dev, stream, target.data_ptr(), None if draft is None else draft.data_ptr() or None, _type(target, "target"), vocab,
          one(target), 0 if draft is None else one(draft), tokens.data_ptr(), q_start.data_ptr(), u_accept.data_ptr(), u_sample.data_ptr(),
          n_seq, target.shape[0], n_drafts, out_tokens.shape[1] - 1, n_accepted.data_ptr(), out_tokens.data_ptr(), workspace.data_ptr(),
          workspace.numel() * workspace.element_size())
