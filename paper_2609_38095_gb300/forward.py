"""Python binding of include/zo_forward.h: the operators of a forward point,
between the weights that a step perturbs and the loss table that its
preconditioner reads. As in zo.py, every numeric step runs in the library's
CUDA kernels; this module checks arguments, turns torch tensors into pointers
and strides and passes the current torch stream.

A decoder layer of a forward point over packed documents:

    table = zo.forward.rotary_table(positions_in_all, head_dim, base=1e6)       # once per model
    spans = zo.forward.document_spans(starts, tokens=T)                         # once per batch
    q, k = zo.forward.rotate_heads(q, k, table=table, positions=pos, q_weight=wq, k_weight=wk)
    out = zo.forward.attention(q, k, v, spans)
    ...
    zo.forward.token_loss(logits, targets, out=losses[probe, 0:1])              # an entry of the loss table

and of an answer's next token, over a paged cache (pages, page_size, kv_heads, head_dim):

    q, _, _ = zo.forward.rotate_heads(q, k, v, k_out=k_cache, v_out=v_cache, slots=slots, ...)
    out = zo.forward.decode_attention(q, k_cache, v_cache, pages, lengths)

The method has no backward pass: a tensor that asks for a gradient is refused
where torch would record one.
"""
import ctypes

import torch

from . import zo as _zo
from .zo import DTYPE_CODE

EXPORTS = ["zo_rotary_table", "zo_document_spans", "zo_rotate_heads", "zo_attention", "zo_attention_decode",
           "zo_token_loss_workspace_size", "zo_token_loss"]
MAX_HEAD_DIM = 256
MAX_HEADS = 1024
LAYOUTS = {"half": 0, "interleaved": 1}
INDEX_BYTES = {torch.int32: 4, torch.int64: 8}
LOSS_MEAN, LOSS_ADD, LOSS_F32 = 1, 2, 4

_signed = False


def _lib():
    global _signed
    L = _zo._lib()
    if not _signed:
        vp, i32, i64, f32, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double
        sig = {
            "zo_rotary_table": ([vp, i64, i32, f64, f64, i64, f64, f64, f64, vp], ctypes.c_int),
            "zo_document_spans": ([vp, vp, vp, i32, vp, i64, vp], ctypes.c_int),
            "zo_rotate_heads": ([vp, i32, i64, i32, i32, vp, i64, i32, i32, vp, vp, i32, i64, i64, f32, vp], ctypes.c_int),
            "zo_attention": ([vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, vp, f32, f32, vp, vp, vp], ctypes.c_int),
            "zo_attention_decode": ([vp, vp, vp, vp, i64, i32, i32, i32, i32, vp, i64, i64, i64, i32, vp, f32, f32, vp, vp,
                                     vp], ctypes.c_int),
            "zo_token_loss_workspace_size": ([i64], i64),
            "zo_token_loss": ([vp, i64, i64, i64, i32, vp, i32, i32, vp, vp, vp, i64, vp], ctypes.c_int),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        _signed = True
    return L


def _rows(t, what, dim, like=None):
    """Checks a tensor of heads: on the device of `like` and of its type, `dim` dimensions, heads contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dim() != dim:
        raise ValueError(f"{what} must have {dim} dimensions, got {t.dim()}")
    if like is None:
        if t.dtype not in DTYPE_CODE:
            raise TypeError(f"unsupported dtype {t.dtype}")
    elif t.dtype != like.dtype:
        raise TypeError(f"{what} must be {like.dtype}, got {t.dtype}")
    elif t.device != like.device:
        raise ValueError(f"{what} is on {t.device}, expected {like.device}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: the elements of a head must be contiguous")
    if t.requires_grad and torch.is_grad_enabled():
        raise RuntimeError(f"{what} asks for a gradient, which this operator does not have")
    return t


def _flat(t, what, dtypes, device, dim=1):
    """Checks a contiguous tensor of numbers beside the heads."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")
    if t.dim() != dim or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous, with {dim} dimension{'s' if dim > 1 else ''}")
    return t


def _stride(t, i):
    """The stride of dimension i; 0 where only its first element exists."""
    return t.stride(i) if t.shape[i] > 1 else 0


def rotary_table(rows, rotary_dim, base=10000.0, scale=1.0, original=0, low=1.0, high=32.0, magnitude=1.0, device=None):
    """Cosines and sines of positions 0 .. rows - 1, float32 (rows, rotary_dim): cosines of the rotary_dim / 2
    frequencies, then sines (zo_rotary_table). scale > 1 stretches the positions that the model was made for, by parts
    where `original` names that context's length."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    if device.type != "cuda":
        raise ValueError("the table must live on a CUDA device")
    table = torch.empty(rows, rotary_dim, dtype=torch.float32, device=device)
    _zo._launch("zo_rotary_table", _zo._index(device), _lib().zo_rotary_table, table.data_ptr(), rows, rotary_dim, base,
                scale, original, low, high, magnitude)
    return table


def document_spans(q_starts, k_starts=None, prefix=None, *, tokens):
    """int32 (3, tokens): for each packed query row its first key, the end of its keys and its own key
    (zo_document_spans). q_starts and k_starts (q_starts by default): int32, one more than there are documents."""
    _flat(q_starts, "q_starts", (torch.int32,), q_starts.device)
    dev, docs = q_starts.device, q_starts.numel() - 1
    if docs < 0:
        raise ValueError("q_starts must have one element more than there are documents")
    k_starts = q_starts if k_starts is None else _flat(k_starts, "k_starts", (torch.int32,), dev)
    if k_starts.numel() != docs + 1 or (prefix is not None and _flat(prefix, "prefix", (torch.int32,), dev).numel() != docs):
        raise ValueError("k_starts must have as many elements as q_starts, prefix one less")
    spans = torch.empty(3, tokens, dtype=torch.int32, device=dev)
    _zo._launch("zo_document_spans", _zo._index(dev), _lib().zo_document_spans, q_starts.data_ptr(), k_starts.data_ptr(),
                prefix.data_ptr() if prefix is not None else None, docs, spans.data_ptr(), tokens)
    return spans


def rotate_heads(q, k=None, v=None, *, table, positions, q_weight=None, k_weight=None, eps=1e-6, layout="half",
                 q_out=None, k_out=None, v_out=None, slots=None):
    """Norms (where a weight is given) and rotation of q (tokens, heads, head_dim) and k (tokens, kv_heads, head_dim);
    v is copied (zo_rotate_heads). Returns what was written, one tensor per tensor given: q alone, (q, k) or (q, k, v);
    new tensors where no *_out is given. With slots (one per token) k and v go to rows of a cache, k_out and v_out:
    (rows, kv_heads, head_dim) or (pages, page_size, kv_heads, head_dim). q_out may be q, and k_out k."""
    _rows(q, "q", 3)
    dev, dtype, (tokens, _, dim) = q.device, q.dtype, q.shape
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
    _flat(table, "table", (torch.float32,), dev, 2)
    _flat(positions, "positions", INDEX_BYTES, dev)
    if positions.numel() != tokens:
        raise ValueError("positions must have one element per token")
    if v is not None and k is None:
        raise ValueError("v needs k")
    if slots is not None:
        if k is None or k_out is None or (v is None) != (v_out is None):
            raise ValueError("slots need k and the cache that it goes to, and v both or neither")
        _flat(slots, "slots", (positions.dtype,), dev)
        if slots.numel() != tokens:
            raise ValueError("slots must have one element per token")
    words, made = [], []
    n_slots = page_size = 1
    for what, x, weight, out, rotate in (("q", q, q_weight, q_out, 1), ("k", k, k_weight, k_out, 1), ("v", v, None, v_out, 0)):
        if x is None:
            if out is not None or weight is not None:
                raise ValueError(f"an output or weight is given for {what}, but not {what}")
            continue
        if what != "q":
            _rows(x, what, 3, q)
            if x.shape[0] != tokens or x.shape[2] != dim:
                raise ValueError(f"{what} must have q's tokens and head size")
        if weight is not None:
            _flat(weight, f"{what}_weight", DTYPE_CODE, dev)
            if weight.numel() != dim:
                raise ValueError(f"{what}_weight must have one element per element of a head")
            if weight.requires_grad and torch.is_grad_enabled():
                raise RuntimeError(f"{what}_weight asks for a gradient, which this operator does not have")
        by_slot = slots is not None and what != "q"
        if out is None:
            out = torch.empty(x.shape, dtype=dtype, device=dev)
        paged = by_slot and out.dim() == 4
        _rows(out, f"{what}_out", 4 if paged else 3, q)
        if out.shape[-2:] != x.shape[-2:] or (not by_slot and out.shape[0] != tokens):
            raise ValueError(f"{what}_out must have {what}'s heads and, without slots, tokens")
        if by_slot:
            size = (out.shape[0] * out.shape[1], out.shape[1]) if paged else (out.shape[0], max(out.shape[0], 1))
            if what == "k":
                n_slots, page_size = size
            elif size != (n_slots, page_size):
                raise ValueError("k_out and v_out must have the same rows")
        words += [x.data_ptr(), _stride(x, 0), _stride(x, 1), out.data_ptr(), _stride(out, 0) if paged else 0,
                  _stride(out, -3), _stride(out, -2), weight.data_ptr() if weight is not None else 0,
                  (DTYPE_CODE[weight.dtype] if weight is not None else 0) | x.shape[1] << 32,
                  rotate | (2 if by_slot else 0)]
        made.append(out)
    arr = (ctypes.c_int64 * len(words))(*words)
    _zo._launch("zo_rotate_heads", _zo._index(dev), _lib().zo_rotate_heads, ctypes.addressof(arr), len(made), tokens, dim,
                DTYPE_CODE[dtype], table.data_ptr(), table.shape[0], table.shape[1], LAYOUTS[layout], positions.data_ptr(),
                slots.data_ptr() if slots is not None else None, INDEX_BYTES[positions.dtype], n_slots, max(page_size, 1),
                eps)
    return made[0] if len(made) == 1 else tuple(made)


def _shared(q, k, v, out, scale, slopes, dim):
    """Checks that attention and decode_attention share; returns (out, scale)."""
    _rows(k, "k", dim, q)
    _rows(v, "v", dim, q)
    if k.shape != v.shape or k.shape[-1] != q.shape[2]:
        raise ValueError("k and v must have the same shape and q's head size")
    if k.shape[-2] == 0 or q.shape[1] % k.shape[-2]:
        raise ValueError("the key-value heads must divide the query heads")
    if slopes is not None and _flat(slopes, "slopes", (torch.float32,), q.device).numel() != q.shape[1]:
        raise ValueError("slopes must have one element per query head")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif _rows(out, "out", 3, q).shape != q.shape:
        raise ValueError("out must have q's shape")
    return out, q.shape[2] ** -0.5 if scale is None else scale


def attention(q, k, v, spans, *, scale=None, softcap=0.0, slopes=None, out=None, with_lse=False):
    """Attention of q (tokens, heads, head_dim) over k and v (keys, kv_heads, head_dim), each row over the keys of its
    span (zo_attention). spans: document_spans, or any int32 (3, tokens) of first key, end and own key. softcap: scores
    are softcap * tanh(score / softcap); slopes: float32 (heads), a bias of -slope * distance. Returns out, or (out,
    lse) with lse float32 (heads, tokens)."""
    _rows(q, "q", 3)
    out, scale = _shared(q, k, v, out, scale, slopes, 3)
    tokens, heads, dim = q.shape
    if _flat(spans, "spans", (torch.int32,), q.device, 2).shape != (3, tokens):
        raise ValueError("spans must have shape (3, tokens)")
    lse = torch.empty(heads, tokens, dtype=torch.float32, device=q.device) if with_lse else None
    arr = (ctypes.c_int64 * 12)(q.data_ptr(), _stride(q, 0), _stride(q, 1), k.data_ptr(), _stride(k, 0), _stride(k, 1),
                                v.data_ptr(), _stride(v, 0), _stride(v, 1), out.data_ptr(), _stride(out, 0), _stride(out, 1))
    at = ctypes.addressof(arr)
    _zo._launch("zo_attention", _zo._index(q.device), _lib().zo_attention, at, at + 24, at + 48, at + 72, tokens,
                k.shape[0], heads, k.shape[1], dim, DTYPE_CODE[q.dtype], spans.data_ptr(), scale, softcap,
                slopes.data_ptr() if slopes is not None else None, lse.data_ptr() if with_lse else None)
    return (out, lse) if with_lse else out


def decode_attention(q, k_cache, v_cache, pages, lengths, *, scale=None, softcap=0.0, slopes=None, out=None, with_lse=False):
    """Attention of one new token per sequence, q (batch, heads, head_dim), over the first lengths[b] keys of each
    sequence, its own the last (zo_attention_decode). k_cache, v_cache: (pages, page_size, kv_heads, head_dim); pages:
    int32 (batch, pages of the longest); lengths: int32 (batch). Returns out, or (out, lse) with lse float32 (batch,
    heads)."""
    _rows(q, "q", 3)
    out, scale = _shared(q, k_cache, v_cache, out, scale, slopes, 4)
    batch, heads, dim = q.shape
    if not isinstance(pages, torch.Tensor) or pages.dtype != torch.int32 or pages.device != q.device:
        raise TypeError("pages must be an int32 tensor on q's device")
    if pages.dim() != 2 or pages.shape[0] != batch or (pages.shape[1] > 1 and pages.stride(1) != 1):
        raise ValueError("pages must have one row per sequence, contiguous")
    if _flat(lengths, "lengths", (torch.int32,), q.device).numel() != batch:
        raise ValueError("lengths must have one element per sequence")
    n_pages, page_size, kv_heads = k_cache.shape[:3]
    if page_size < 1:
        raise ValueError("a page must hold at least one row")
    lse = torch.empty(batch, heads, dtype=torch.float32, device=q.device) if with_lse else None
    k, v = k_cache, v_cache
    arr = (ctypes.c_int64 * 14)(q.data_ptr(), _stride(q, 0), _stride(q, 1), k.data_ptr(), _stride(k, 0), _stride(k, 1),
                                _stride(k, 2), v.data_ptr(), _stride(v, 0), _stride(v, 1), _stride(v, 2), out.data_ptr(),
                                _stride(out, 0), _stride(out, 1))
    at = ctypes.addressof(arr)
    _zo._launch("zo_attention_decode", _zo._index(q.device), _lib().zo_attention_decode, at, at + 24, at + 56, at + 88, batch,
                heads, kv_heads, dim, DTYPE_CODE[q.dtype], pages.data_ptr(), _stride(pages, 0), pages.shape[1], n_pages,
                page_size, lengths.data_ptr(), scale, softcap, slopes.data_ptr() if slopes is not None else None,
                lse.data_ptr() if with_lse else None)
    return (out, lse) if with_lse else out


def token_loss(logits, targets, *, mean=False, add=False, out=None, dtype=torch.float64, with_nll=False):
    """-log p of the targets under logits (tokens, vocab), summed over the tokens whose target is not negative, or their
    mean (zo_token_loss). Returns a one-element tensor: `out` (for instance losses[k, 0:1] of a step's loss table; added
    to what is there with add), or a new one of `dtype` (float64 or float32). with_nll: also each token's, float32."""
    _rows(logits, "logits", 2)
    dev, (tokens, vocab) = logits.device, logits.shape
    _flat(targets, "targets", INDEX_BYTES, dev)
    if targets.numel() != tokens:
        raise ValueError("targets must have one element per token")
    if out is None:
        if add:
            raise ValueError("add needs out")
        out = torch.empty(1, dtype=dtype, device=dev)
    if _flat(out, "out", (torch.float64, torch.float32), dev).numel() != 1:
        raise ValueError("out must have one element")
    nll = torch.empty(tokens, dtype=torch.float32, device=dev) if with_nll else None
    work = torch.empty(max(tokens, 1), dtype=torch.float64, device=dev)
    flags = (LOSS_MEAN if mean else 0) | (LOSS_ADD if add else 0) | (LOSS_F32 if out.dtype == torch.float32 else 0)
    _zo._launch("zo_token_loss", _zo._index(dev), _lib().zo_token_loss, logits.data_ptr(), _stride(logits, 0), tokens, vocab,
                DTYPE_CODE[logits.dtype], targets.data_ptr(), INDEX_BYTES[targets.dtype], flags, out.data_ptr(),
                nll.data_ptr() if with_nll else None, work.data_ptr(), work.numel() * 8)
    return (out, nll) if with_nll else out
