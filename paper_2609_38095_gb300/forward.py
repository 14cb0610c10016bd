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
from struct import Struct

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
        for name in ("rotate_heads", "attention", "attention_decode", "token_loss"):
            sig["zo_internal_" + name] = ([ctypes.c_char_p, vp], ctypes.c_int)
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        _signed = True
    return L


# A call's arguments travel in one block; the checks of the calls below are one
# expression each, and the functions named _refuse_* say what was wrong. (On the
# GB300's host cores an attribute of a tensor costs 0.1 us and a Python call 0.3,
# of 10 to 15 us that a call takes in all.)
_ROTATE = [None] + [Struct(f"13qfxxxx{10 * n}q") for n in (1, 2, 3)]
_ATTENTION = Struct("21qff")
_DECODE = Struct("27qff")
_LOSS = Struct("12q")
_grad = torch.is_grad_enabled
_empty = torch.empty



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
    if t.requires_grad and _grad():
        raise RuntimeError(f"{what} asks for a gradient, which this operator does not have")
    return t


def _flat(t, what, dtypes, device, dim=1, n=None):
    """Checks a contiguous tensor of numbers beside the heads, of n elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")
    if t.dim() != dim or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous, with {dim} dimension{'s' if dim > 1 else ''}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{what} must have {n} elements, got {t.numel()}")
    if t.requires_grad and _grad():
        raise RuntimeError(f"{what} asks for a gradient, which this operator does not have")
    return t


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
    k_starts = q_starts if k_starts is None else _flat(k_starts, "k_starts", (torch.int32,), dev, n=docs + 1)
    if prefix is not None:
        _flat(prefix, "prefix", (torch.int32,), dev, n=docs)
    spans = torch.empty(3, tokens, dtype=torch.int32, device=dev)
    _zo._launch("zo_document_spans", _zo._index(dev), _lib().zo_document_spans, q_starts.data_ptr(), k_starts.data_ptr(),
                prefix.data_ptr() if prefix is not None else None, docs, spans.data_ptr(), tokens)
    return spans


def _refuse_part(what, q, x, weight, out, by_slot):
    _rows(x, what, 3, None if what == "q" else q)
    if x.shape[0] != q.shape[0] or x.shape[2] != q.shape[2]:
        raise ValueError(f"{what} must have q's tokens and head size")
    if weight is not None:
        _flat(weight, f"{what}_weight", DTYPE_CODE, q.device, n=q.shape[2])
    _rows(out, f"{what}_out", 4 if by_slot and out.dim() == 4 else 3, q)
    raise ValueError(f"{what}_out must have {what}'s heads and, without slots, tokens")


def _part(what, q, idx, dtype, tokens, dim, x, weight, out, flags):
    """The output of one of rotate_heads's tensors, its words of the argument block, and its rows and rows per page."""
    shape = x.shape
    if out is None:
        out = _empty(shape, dtype=dtype, device=x.device)
    made, steps, by_slot = out.shape, out.stride(), flags & 2
    strides = x.stride()
    if not (len(shape) == 3 and x.dtype == dtype == out.dtype and x.get_device() == idx == out.get_device()
            and shape[0] == tokens and shape[2] == dim and (strides[2] == 1 or dim == 1) and (steps[-1] == 1 or dim == 1)
            and made[-2:] == shape[1:] and (len(made) == 3 or (by_slot and len(made) == 4)) and (by_slot or made[0] == tokens)
            and (weight is None or (weight.numel() == dim and weight.dtype in DTYPE_CODE and weight.get_device() == idx
                                    and weight.dim() == 1 and weight.is_contiguous()))
            and not (_grad() and (x.requires_grad or out.requires_grad or (weight is not None and weight.requires_grad)))):
        _refuse_part(what, q, x, weight, out, by_slot)
    if len(made) == 4:
        page, rows, per_page = steps[0], made[0] * made[1], made[1]
    else:
        page, rows, per_page = 0, made[0], made[0]
    kind = shape[1] << 32
    if weight is not None:
        kind |= DTYPE_CODE[weight.dtype]
    return out, (x.data_ptr(), strides[0], strides[1], out.data_ptr(), page, steps[-3], steps[-2],
                 0 if weight is None else weight.data_ptr(), kind, flags), rows, per_page


def rotate_heads(q, k=None, v=None, *, table, positions, q_weight=None, k_weight=None, eps=1e-6, layout="half",
                 q_out=None, k_out=None, v_out=None, slots=None):
    """Norms (where a weight is given) and rotation of q (tokens, heads, head_dim) and k (tokens, kv_heads, head_dim);
    v is copied (zo_rotate_heads). Returns what was written, one tensor per tensor given: q alone, (q, k) or (q, k, v);
    new tensors where no *_out is given. With slots (one per token) k and v go to rows of a cache, k_out and v_out:
    (rows, kv_heads, head_dim) or (pages, page_size, kv_heads, head_dim). q_out may be q, and k_out k."""
    shape, idx, index = q.shape, q.get_device(), positions.dtype
    if not (idx >= 0 and len(shape) == 3 and q.dtype in DTYPE_CODE):
        _rows(q, "q", 3)
    tokens, _, dim = shape
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
    size = table.shape
    if not (len(size) == 2 and table.dtype is torch.float32 and table.is_contiguous() and table.get_device() == idx
            and index in INDEX_BYTES and positions.get_device() == idx and positions.shape == shape[:1]
            and positions.is_contiguous()):
        _flat(table, "table", (torch.float32,), q.device, 2)
        _flat(positions, "positions", INDEX_BYTES, q.device, n=tokens)
    by_slot, rows, per_page = 0, 1, 1
    if slots is not None:
        if k is None or k_out is None or (v is None) != (v_out is None):
            raise ValueError("slots need k and the cache that it goes to, and v both or neither")
        _flat(slots, "slots", (index,), q.device, n=tokens)
        by_slot = 2
    if (k is None and (v is not None or k_out is not None or k_weight is not None)) or (v is None and v_out is not None):
        raise ValueError("an output, weight or v is given for a tensor that is not")
    out, words, _, _ = _part("q", q, idx, q.dtype, tokens, dim, q, q_weight, q_out, 1)
    made = (out,)
    if k is not None:
        out, more, rows, per_page = _part("k", q, idx, q.dtype, tokens, dim, k, k_weight, k_out, 1 | by_slot)
        made, words = made + (out,), words + more
    if v is not None:
        out, more, *same = _part("v", q, idx, q.dtype, tokens, dim, v, None, v_out, by_slot)
        made, words = made + (out,), words + more
        if by_slot and same != [rows, per_page]:
            raise ValueError("k_out and v_out must have the same rows")
    block = _ROTATE[len(made)].pack(len(made), tokens, dim, DTYPE_CODE[q.dtype], table.data_ptr(), size[0], size[1],
                                    LAYOUTS[layout], positions.data_ptr(), 0 if slots is None else slots.data_ptr(),
                                    INDEX_BYTES[index], rows, per_page or 1, eps, *words)
    _zo._launch("zo_rotate_heads", idx, _lib().zo_internal_rotate_heads, block)
    return made[0] if len(made) == 1 else made


def _refuse_attention(q, k, v, out, slopes, dim):
    """Says why attention's or decode_attention's tensors of heads are none that it takes."""
    _rows(q, "q", 3)
    _rows(k, "k", dim, q)
    _rows(v, "v", dim, q)
    if k.shape != v.shape or k.shape[-1] != q.shape[2]:
        raise ValueError("k and v must have the same shape and q's head size")
    if k.shape[-2] == 0 or q.shape[1] % k.shape[-2]:
        raise ValueError("the key-value heads must divide the query heads")
    if slopes is not None:
        _flat(slopes, "slopes", (torch.float32,), q.device, n=q.shape[1])
    if out is not None and _rows(out, "out", 3, q).shape != q.shape:
        raise ValueError("out must have q's shape")


def _beside(shape, dtype, idx, slopes, out):
    """Whether slopes and out, where given, fit queries of that shape."""
    return (slopes is None or (slopes.dtype is torch.float32 and slopes.get_device() == idx and slopes.shape == shape[1:2]
                               and slopes.is_contiguous() and not (_grad() and slopes.requires_grad))) and (
        out is None or (out.shape == shape and out.dtype == dtype and out.get_device() == idx
                        and (out.stride(2) == 1 or shape[2] == 1) and not (_grad() and out.requires_grad)))


def attention(q, k, v, spans, *, scale=None, softcap=0.0, slopes=None, out=None, with_lse=False):
    """Attention of q (tokens, heads, head_dim) over k and v (keys, kv_heads, head_dim), each row over the keys of its
    span (zo_attention). spans: document_spans, or any int32 (3, tokens) of first key, end and own key. softcap: scores
    are softcap * tanh(score / softcap); slopes: float32 (heads), a bias of -slope * distance. Returns out, or (out,
    lse) with lse float32 (heads, tokens)."""
    shape, size, dtype, idx = q.shape, k.shape, q.dtype, q.get_device()
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    if not (idx >= 0 and len(shape) == 3 == len(size) and v.shape == size and size[2] == shape[2] and dtype in DTYPE_CODE
            and k.dtype == dtype == v.dtype and k.get_device() == idx == v.get_device() and size[1] > 0
            and shape[1] % size[1] == 0 and (qs[2] == 1 == ks[2] == vs[2] or shape[2] == 1) and _beside(shape, dtype, idx, slopes, out)
            and not (_grad() and (q.requires_grad or k.requires_grad or v.requires_grad))):
        _refuse_attention(q, k, v, out, slopes, 3)
    tokens, heads, dim = shape
    if not (spans.dtype is torch.int32 and spans.get_device() == idx and spans.shape == (3, tokens) and spans.is_contiguous()):
        _flat(spans, "spans", (torch.int32,), q.device, 2)
        raise ValueError("spans must have shape (3, tokens)")
    if out is None:
        out = _empty(shape, dtype=dtype, device=q.device)
    os = out.stride()
    lse = _empty((heads, tokens), dtype=torch.float32, device=q.device) if with_lse else None
    block = _ATTENTION.pack(q.data_ptr(), qs[0], qs[1], k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], out.data_ptr(),
                            os[0], os[1], tokens, size[0], heads, size[1], dim, DTYPE_CODE[dtype], spans.data_ptr(),
                            0 if slopes is None else slopes.data_ptr(), lse.data_ptr() if with_lse else 0,
                            dim ** -0.5 if scale is None else scale, softcap)
    _zo._launch("zo_attention", idx, _lib().zo_internal_attention, block)
    return (out, lse) if with_lse else out


def decode_attention(q, k_cache, v_cache, pages, lengths, *, scale=None, softcap=0.0, slopes=None, out=None, with_lse=False):
    """Attention of one new token per sequence, q (batch, heads, head_dim), over the first lengths[b] keys of each
    sequence, its own the last (zo_attention_decode). k_cache, v_cache: (pages, page_size, kv_heads, head_dim); pages:
    int32 (batch, pages of the longest); lengths: int32 (batch). Returns out, or (out, lse) with lse float32 (batch,
    heads)."""
    shape, size, dtype, idx = q.shape, k_cache.shape, q.dtype, q.get_device()
    qs, ks, vs = q.stride(), k_cache.stride(), v_cache.stride()
    if not (idx >= 0 and len(shape) == 3 and len(size) == 4 and v_cache.shape == size and size[3] == shape[2]
            and dtype in DTYPE_CODE and k_cache.dtype == dtype == v_cache.dtype
            and k_cache.get_device() == idx == v_cache.get_device() and size[2] > 0 and shape[1] % size[2] == 0
            and (qs[2] == 1 == ks[3] == vs[3] or shape[2] == 1) and _beside(shape, dtype, idx, slopes, out)
            and not (_grad() and (q.requires_grad or k_cache.requires_grad or v_cache.requires_grad))):
        _refuse_attention(q, k_cache, v_cache, out, slopes, 4)
    batch, heads, dim = shape
    table, steps = pages.shape, pages.stride()
    if not (pages.dtype is torch.int32 and pages.get_device() == idx and len(table) == 2 and table[0] == batch
            and (steps[1] == 1 or table[1] <= 1)):
        raise ValueError("pages must be an int32 tensor on q's device with a contiguous row per sequence")
    if not (lengths.dtype is torch.int32 and lengths.get_device() == idx and lengths.shape == shape[:1]
            and lengths.is_contiguous()):
        _flat(lengths, "lengths", (torch.int32,), q.device, n=batch)
    n_pages, page_size, kv_heads, _ = size
    if page_size < 1:
        raise ValueError("a page must hold at least one row")
    if out is None:
        out = _empty(shape, dtype=dtype, device=q.device)
    os = out.stride()
    lse = _empty((batch, heads), dtype=torch.float32, device=q.device) if with_lse else None
    block = _DECODE.pack(q.data_ptr(), qs[0], qs[1], out.data_ptr(), os[0], os[1], k_cache.data_ptr(), ks[0], ks[1], ks[2],
                         v_cache.data_ptr(), vs[0], vs[1], vs[2], batch, heads, kv_heads, dim, DTYPE_CODE[dtype],
                         pages.data_ptr(), steps[0], table[1], n_pages, page_size, lengths.data_ptr(),
                         0 if slopes is None else slopes.data_ptr(), lse.data_ptr() if with_lse else 0,
                         dim ** -0.5 if scale is None else scale, softcap)
    _zo._launch("zo_attention_decode", idx, _lib().zo_internal_attention_decode, block)
    return (out, lse) if with_lse else out


def token_loss(logits, targets, *, mean=False, add=False, out=None, dtype=torch.float64, with_nll=False):
    """-log p of the targets under logits (tokens, vocab), summed over the tokens whose target is not negative, or their
    mean (zo_token_loss). Returns a one-element tensor: `out` (for instance losses[k, 0:1] of a step's loss table; added
    to what is there with add), or a new one of `dtype` (float64 or float32). with_nll: also each token's, float32."""
    shape, idx, kind, strides = logits.shape, logits.get_device(), targets.dtype, logits.stride()
    if not (idx >= 0 and len(shape) == 2 and logits.dtype in DTYPE_CODE and (strides[1] == 1 or shape[1] == 1)
            and not (logits.requires_grad and _grad())):
        _rows(logits, "logits", 2)
    tokens, vocab = shape
    if not (kind in INDEX_BYTES and targets.get_device() == idx and targets.shape == shape[:1] and targets.is_contiguous()):
        _flat(targets, "targets", INDEX_BYTES, logits.device, n=tokens)
    if out is None:
        if add:
            raise ValueError("add needs out")
        out = _empty(1, dtype=dtype, device=logits.device)
    single = out.dtype is torch.float32
    if not ((single or out.dtype is torch.float64) and out.get_device() == idx and out.shape == (1,)):
        _flat(out, "out", (torch.float64, torch.float32), logits.device, n=1)
    nll = _empty(tokens, dtype=torch.float32, device=logits.device) if with_nll else None
    work = _empty(tokens or 1, dtype=torch.float64, device=logits.device)
    flags = (LOSS_MEAN if mean else 0) | (LOSS_ADD if add else 0) | (LOSS_F32 if single else 0)
    block = _LOSS.pack(logits.data_ptr(), strides[0] if tokens > 1 else 0, tokens, vocab, DTYPE_CODE[logits.dtype],
                       targets.data_ptr(), INDEX_BYTES[kind], flags, out.data_ptr(), nll.data_ptr() if with_nll else 0,
                       work.data_ptr(), 8 * (tokens or 1))
    _zo._launch("zo_token_loss", idx, _lib().zo_internal_token_loss, block)
    return (out, nll) if with_nll else out
