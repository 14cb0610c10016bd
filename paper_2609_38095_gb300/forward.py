"""Python binding of include/zo_forward.h: the operators of a forward point,
between the weights that a step perturbs and the loss table that its
preconditioner reads. As in zo.py, every numeric step runs in the library's
CUDA kernels; arguments are checked, and tensors turned into pointers and
strides, by the compiled module _binding (csrc/zo_binding.cpp).

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
where torch would record one, and a tensor with a tangent of forward mode is.
"""
import ctypes
import importlib.machinery
import importlib.util
import os

import torch

from . import zo as _zo

EXPORTS = ["zo_rotary_table", "zo_document_spans", "zo_rotate_heads", "zo_attention", "zo_attention_decode",
           "zo_token_loss_workspace_size", "zo_token_loss"]
MAX_HEAD_DIM = 256
MAX_HEADS = 1024
LAYOUTS = {"half": False, "interleaved": True}
BINDING_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_binding.so")

_L = None
_B = None


def _lib():
    """The library, with this header's signatures."""
    global _L
    if _L is None:
        L = _zo._lib()
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
        _L = L
    return _L


def _binding():
    """The compiled module, bound to the library."""
    global _B
    if _B is None:
        if not os.path.exists(BINDING_PATH):
            raise RuntimeError(f"{BINDING_PATH} is not built; run paper_2609_38095_gb300.build.build_binding()")
        loader = importlib.machinery.ExtensionFileLoader(__package__ + "._binding", BINDING_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader(loader.name, loader))
        loader.exec_module(module)
        module.bind(*(ctypes.cast(getattr(_lib(), "zo_" + n), ctypes.c_void_p).value
                      for n in ("rotate_heads", "attention", "attention_decode", "token_loss")))
        _B = module
    return _B


def _made(what, result):
    """What a call of the binding returned, or the error that its status is."""
    if type(result) is int:
        raise _zo.ZoError(what, result)
    return result


def _flat(t, what, dtypes, device=None, n=None):
    """Checks a contiguous vector of numbers, of n elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")
    if t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{what} must be contiguous, with one dimension" + (f" and {n} elements" if n is not None else ""))
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
    _flat(q_starts, "q_starts", (torch.int32,))
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


def rotate_heads(q, k=None, v=None, *, table, positions, q_weight=None, k_weight=None, eps=1e-6, layout="half",
                 q_out=None, k_out=None, v_out=None, slots=None):
    """Norms (where a weight is given) and rotation of q (tokens, heads, head_dim) and k (tokens, kv_heads, head_dim);
    v is copied (zo_rotate_heads). Returns what was written, one tensor per tensor given: q alone, (q, k) or (q, k, v);
    new tensors where no *_out is given. With slots (one per token) k and v go to rows of a cache, k_out and v_out:
    (rows, kv_heads, head_dim) or (pages, page_size, kv_heads, head_dim). q_out may be q, and k_out k; outputs overlap
    nothing else."""
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}")
    return _made("zo_rotate_heads", (_B or _binding()).rotate_heads(q, k, v, table, positions, q_weight, k_weight, eps,
                                                                    LAYOUTS[layout], q_out, k_out, v_out, slots))


def attention(q, k, v, spans, *, scale=None, softcap=0.0, slopes=None, out=None, with_lse=False):
    """Attention of q (tokens, heads, head_dim) over k and v (keys, kv_heads, head_dim), each row over the keys of its
    span (zo_attention). spans: document_spans, or any int32 (3, tokens) of first key, end and own key. softcap: scores
    are softcap * tanh(score / softcap); slopes: float32 (heads), a bias of -slope * distance. Returns out, or (out,
    lse) with lse float32 (heads, tokens). An `out` of the caller's overlaps no input."""
    return _made("zo_attention", (_B or _binding()).attention(q, k, v, spans, scale, softcap, slopes, out, with_lse))


def decode_attention(q, k_cache, v_cache, pages, lengths, *, scale=None, softcap=0.0, slopes=None, out=None, with_lse=False):
    """Attention of one new token per sequence, q (batch, heads, head_dim), over the first lengths[b] keys of each
    sequence, its own the last (zo_attention_decode). k_cache, v_cache: (pages, page_size, kv_heads, head_dim); pages:
    int32 (batch, pages of the longest); lengths: int32 (batch). Returns out, or (out, lse) with lse float32 (batch,
    heads). An `out` of the caller's may be q, and overlaps nothing else."""
    return _made("zo_attention_decode", (_B or _binding()).decode_attention(q, k_cache, v_cache, pages, lengths, scale, softcap,
                                                                            slopes, out, with_lse))


def token_loss(logits, targets, *, mean=False, add=False, out=None, dtype=torch.float64, with_nll=False):
    """-log p of the targets under logits (tokens, vocab), summed over the tokens whose target is not negative, or their
    mean (zo_token_loss). Returns a one-element tensor: `out` (for instance losses[k, 0:1] of a step's loss table; added
    to what is there with add), or a new one of `dtype` (float64 or float32). with_nll: also each token's, float32."""
    if dtype is not torch.float64 and dtype is not torch.float32:
        raise ValueError("dtype must be torch.float64 or torch.float32")
    return _made("zo_token_loss", (_B or _binding()).token_loss(logits, targets, mean, add, out, dtype is torch.float32, with_nll))
