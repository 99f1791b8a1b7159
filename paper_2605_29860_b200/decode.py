"""Binding of the operators around the decode step: key/value cache, attention over shared prompts, sampling from given
random numbers.  Same names as the C ABI, argument marshalling only (see ``espo.h``)."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import binding as _b

ESPO_E4M3 = 2
ESPO_DEV_BAD_PAGE, ESPO_DEV_CACHE_FULL = 32, 64
ESPO_ROPE_PLAIN, ESPO_ROPE_LINEAR, ESPO_ROPE_BY_PARTS = 0, 1, 2

_CODES = {torch.float32: _b.ESPO_F32, torch.bfloat16: _b.ESPO_BF16}


# (a decode step's calls take microseconds: the device is asked for without torch's lazy initialisation in between; a torch
# built without CUDA lacks that function, and the rest of the package works there)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _ptr(t: Optional[torch.Tensor], name: str, dtype, shape=None):
    """Address of a contiguous CUDA tensor of the given type on the current device (None stays None)."""
    if t is None:
        return None
    if t.dtype != dtype or not t.is_contiguous() or (shape is not None and t.shape != shape):
        want = f" of shape {shape}" if shape is not None else ""
        raise ValueError(f"{name} must be a contiguous {dtype} tensor{want}, got {t.dtype} {tuple(t.shape)}")
    _on_device(t, name)
    return t.data_ptr()


def _on_device(t: torch.Tensor, name: str) -> None:
    device = t.get_device()
    if device < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    if device != _current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{_current_device()}")


def _rows(t: torch.Tensor, name: str, dtype, n: int, heads: int, dim: int):
    """(address, stride) of an [n, heads, dim] tensor whose rows may lie apart (a slice of a wider projection)."""
    if t.dtype != dtype or t.shape != (n, heads, dim):
        raise ValueError(f"{name} must be a {dtype} tensor of shape {(n, heads, dim)}, got {t.dtype} {tuple(t.shape)}")
    row, head, step = t.stride()
    if step != 1 or (heads > 1 and head != dim):
        raise ValueError(f"{name}: only the stride between rows may differ from a contiguous tensor's")
    _on_device(t, name)
    return t.data_ptr(), row if n > 1 else heads * dim


def _word(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if t.element_size() != 4 or t.numel() < 1:
        raise ValueError("status_out must hold one 32-bit word")
    _on_device(t, "status_out")
    return t.data_ptr()


def _structs_here(*structs) -> None:
    """The structures' tensors lie on the current device (theirs is that of their construction)."""
    for x in structs:
        if x is not None and x.tensors[0].get_device() != _current_device():
            raise ValueError(f"{type(x).__name__} is on {x.tensors[0].device}, the current device is cuda:{_current_device()}")


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(_current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class espo_kv_cache(C.Structure):
    """A paged cache over the caller's tensors: k, v [n_pages, n_kv_heads, page_size, head_dim] bfloat16, or
    float8_e4m3fn with uint8 exponents k_exp, v_exp [n_pages, n_kv_heads, page_size]."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("reserved", C.c_int32)]

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: Optional[torch.Tensor] = None,
                 v_exp: Optional[torch.Tensor] = None):
        if k.dim() != 4:
            raise ValueError("k must be [n_pages, n_kv_heads, page_size, head_dim]")
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise ValueError(f"a cache holds bfloat16 or float8_e4m3fn, got {k.dtype}")
        e4m3 = k.dtype == torch.float8_e4m3fn
        if e4m3 != (k_exp is not None) or e4m3 != (v_exp is not None):
            raise ValueError("a float8_e4m3fn cache needs k_exp and v_exp, a bfloat16 one has none")
        shape = tuple(k.shape)
        super().__init__(_ptr(k, "k", k.dtype), _ptr(v, "v", k.dtype, shape), _ptr(k_exp, "k_exp", torch.uint8, shape[:3]),
                         _ptr(v_exp, "v_exp", torch.uint8, shape[:3]), shape[0], shape[2], shape[1], shape[3],
                         ESPO_E4M3 if e4m3 else _b.ESPO_BF16, 0)
        self.tensors = (k, v, k_exp, v_exp)      # kept alive as long as their addresses are


class espo_rope(C.Structure):
    """Rotary embedding from inv_freq (float64 [rot_dim / 2]); ``espo_rope_frequencies`` computes the table."""
    _fields_ = [("inv_freq", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("mscale", C.c_float),
                ("reserved", C.c_int32)]

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, mscale: float = 1.0):
        super().__init__(_ptr(inv_freq, "inv_freq", torch.float64), 2 * inv_freq.numel(), int(bool(interleaved)), mscale, 0)
        self.tensors = (inv_freq,)


class espo_sequences(C.Structure):
    """The batch's sequences by trajectory slot: page tables and lengths of the slots' own tokens and of the prefixes their
    groups share, and the status array that says which slots take part."""
    _fields_ = [("pages", C.c_void_p), ("length", C.c_void_p), ("status", C.c_void_p), ("group", C.c_void_p),
                ("prefix_pages", C.c_void_p), ("prefix_length", C.c_void_p), ("max_pages", C.c_int32),
                ("capacity", C.c_int32), ("max_prefix_pages", C.c_int32), ("n_groups", C.c_int32)]

    def __init__(self, pages: torch.Tensor, length: torch.Tensor, status: Optional[torch.Tensor] = None,
                 group: Optional[torch.Tensor] = None, prefix_pages: Optional[torch.Tensor] = None,
                 prefix_length: Optional[torch.Tensor] = None):
        n = length.numel()
        if pages.dim() != 2 or pages.shape[0] != n:
            raise ValueError("pages must be [capacity, max_pages] with one row per entry of length")
        if status is not None and status.numel() < n:
            raise ValueError("status is shorter than length")
        if (group is None) != (prefix_pages is None) or (group is None) != (prefix_length is None):
            raise ValueError("group, prefix_pages and prefix_length go together")
        n_groups = max_prefix = 0
        if group is not None:
            n_groups = prefix_length.numel()
            if prefix_pages.dim() != 2 or prefix_pages.shape[0] != n_groups:
                raise ValueError("prefix_pages must be [n_groups, max_prefix_pages] with one row per entry of prefix_length")
            max_prefix = prefix_pages.shape[1]
        i32 = torch.int32
        super().__init__(_ptr(pages, "pages", i32), _ptr(length, "length", i32), _ptr(status, "status", torch.uint8),
                         _ptr(group, "group", i32, (n,)), _ptr(prefix_pages, "prefix_pages", i32),
                         _ptr(prefix_length, "prefix_length", i32), pages.shape[1], n, max_prefix, n_groups)
        self.tensors = (pages, length, status, group, prefix_pages, prefix_length)


_lib = None


def _ops():
    global _lib
    if _lib is None:
        L = _b.lib()
        vp, i32, i64, f32, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double
        cache, rope, seqs = C.POINTER(espo_kv_cache), C.POINTER(espo_rope), C.POINTER(espo_sequences)
        L.espo_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp, C.POINTER(f32)]
        L.espo_kv_append.argtypes = [cache, rope, vp, i64, vp, i64, i32, vp, vp, i32, vp, i64, i32, vp, i64, vp, vp]
        L.espo_kv_append_rows.argtypes = [cache, rope, vp, i64, vp, i64, i32, seqs, vp, i32, vp, i64, i32, vp, i64, vp, vp]
        L.espo_kv_gather.argtypes = [cache, vp, i32, vp, vp, i32, vp, vp]
        L.espo_attention_workspace.argtypes = [cache, i32, i32, C.POINTER(i64)]
        L.espo_attention.argtypes = [cache, seqs, vp, i64, i32, vp, i32, f32, vp, i64, vp, i64, vp, vp]
        L.espo_sample.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, i64, vp, vp]
        L.espo_sample_workspace.argtypes = [i32, i32, C.POINTER(i64)]
        for n in ("espo_rope_frequencies", "espo_kv_append", "espo_kv_append_rows", "espo_kv_gather",
                  "espo_attention_workspace", "espo_attention", "espo_sample", "espo_sample_workspace"):
            getattr(L, n).restype = C.c_int
        _lib = L
    return _lib


def espo_rope_frequencies(rot_dim: int, theta: float = 10000.0, kind: int = ESPO_ROPE_PLAIN, factor: float = 1.0,
                          original_length: float = 4096.0, fast_turns: float = 32.0, slow_turns: float = 1.0):
    """(float64 CPU tensor [rot_dim / 2], mscale) of a rotary embedding, optionally stretched for long contexts."""
    out = torch.empty(max(int(rot_dim) // 2, 1), dtype=torch.float64)
    mscale = C.c_float(1.0)
    _b._check(_ops().espo_rope_frequencies(kind, theta, rot_dim, factor, original_length, fast_turns, slow_turns,
                                           out.data_ptr(), C.byref(mscale)), "espo_rope_frequencies")
    return out, mscale.value


def _append_args(cache, key, value, rope, q, q_out):
    if key.dtype not in _CODES:
        raise ValueError(f"key must be float32 or bfloat16, got {key.dtype}")
    _structs_here(cache, rope)
    n, h, d = key.shape[0], cache.n_kv_heads, cache.head_dim
    kp, ks = _rows(key, "key", key.dtype, n, h, d)
    vp, vs = _rows(value, "value", key.dtype, n, h, d)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    qp = op = None
    qs = os_ = hq = 0
    if q is not None:
        hq = q.shape[1]
        qp, qs = _rows(q, "q", key.dtype, n, hq, d)
        op, os_ = _rows(q_out, "q_out", key.dtype, n, hq, d)
    return n, (cache, rope, kp, ks, vp, vs, _CODES[key.dtype]), (qp, qs, hq, op, os_)


def espo_kv_append(cache: espo_kv_cache, key: torch.Tensor, value: torch.Tensor, cache_slots: torch.Tensor,
                   positions: Optional[torch.Tensor] = None, rope: Optional[espo_rope] = None,
                   q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                   status_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rotates and writes n tokens' keys and values [n, n_kv_heads, head_dim] to the given cache slots, and rotates q
    [n, n_q_heads, head_dim] into q_out; see ``espo.h``."""
    n, head, tail = _append_args(cache, key, value, rope, q, q_out)
    if rope is not None and positions is None:
        raise ValueError("a rotation needs positions")
    _b._check(_ops().espo_kv_append(*head, _ptr(cache_slots, "cache_slots", torch.int32, (n,)),
                                    _ptr(positions, "positions", torch.int32, (n,)), n, *tail, _word(status_out),
                                    _stream(stream)), "espo_kv_append")


def espo_kv_append_rows(cache: espo_kv_cache, key: torch.Tensor, value: torch.Tensor, sequences: espo_sequences,
                        row_ids: Optional[torch.Tensor] = None, rope: Optional[espo_rope] = None,
                        q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                        status_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """The decode form: row i is the next token of its trajectory slot, whose length grows by one on the device."""
    _structs_here(sequences)
    n, head, tail = _append_args(cache, key, value, rope, q, q_out)
    if row_ids is not None and row_ids.numel() < n:
        raise ValueError("row_ids is shorter than the rows")
    _b._check(_ops().espo_kv_append_rows(*head, sequences, _ptr(row_ids, "row_ids", torch.int32), n, *tail,
                                         _word(status_out), _stream(stream)), "espo_kv_append_rows")


def espo_kv_gather(cache: espo_kv_cache, cache_slots: torch.Tensor, k_out: Optional[torch.Tensor] = None,
                   v_out: Optional[torch.Tensor] = None, status_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Reads cache slots back into k_out, v_out [n, n_kv_heads, head_dim] (float32 or bfloat16); see ``espo.h``."""
    _structs_here(cache)
    some = k_out if k_out is not None else v_out
    if some is None:
        raise ValueError("k_out or v_out is needed")
    if some.dtype not in _CODES:
        raise ValueError(f"k_out and v_out must be float32 or bfloat16, got {some.dtype}")
    n = cache_slots.numel()
    shape = (n, cache.n_kv_heads, cache.head_dim)
    _b._check(_ops().espo_kv_gather(cache, _ptr(cache_slots, "cache_slots", torch.int32), n,
                                    _ptr(k_out, "k_out", some.dtype, shape), _ptr(v_out, "v_out", some.dtype, shape),
                                    _CODES[some.dtype], _word(status_out), _stream(stream)), "espo_kv_gather")


def espo_attention_workspace(cache: espo_kv_cache, n_rows: int, n_q_heads: int) -> torch.Tensor:
    """A workspace for ``espo_attention`` calls of up to n_rows rows.  Calls that share one must not overlap."""
    size = C.c_int64(0)
    _b._check(_ops().espo_attention_workspace(cache, n_rows, n_q_heads, C.byref(size)), "espo_attention_workspace")
    return torch.empty(size.value, dtype=torch.uint8, device="cuda")


def espo_attention(cache: espo_kv_cache, sequences: espo_sequences, q: torch.Tensor, out: torch.Tensor,
                   workspace: torch.Tensor, scale: float, row_ids: Optional[torch.Tensor] = None,
                   status_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """One query token per row, q and out [n_rows, n_q_heads, head_dim] bfloat16, over the row's group's prefix and its
    own tokens; see ``espo.h``."""
    _structs_here(cache, sequences)
    n, h, d = q.shape
    qp, qs = _rows(q, "q", torch.bfloat16, n, h, d)
    op, os_ = _rows(out, "out", torch.bfloat16, n, h, cache.head_dim)
    if d != cache.head_dim:
        raise ValueError(f"q has {d} dims per head, the cache {cache.head_dim}")
    if row_ids is not None and row_ids.numel() < n:
        raise ValueError("row_ids is shorter than the rows")
    _b._check(_ops().espo_attention(cache, sequences, qp, qs, h, _ptr(row_ids, "row_ids", torch.int32), n, scale,
                                    op, os_, _ptr(workspace, "workspace", torch.uint8), workspace.numel(),
                                    _word(status_out), _stream(stream)), "espo_attention")


def espo_sample_workspace(n_rows: int, V: int) -> torch.Tensor:
    """A workspace for ``espo_sample`` calls of up to n_rows rows of V ids.  Calls that share one must not overlap."""
    size = C.c_int64(0)
    _b._check(_ops().espo_sample_workspace(n_rows, V, C.byref(size)), "espo_sample_workspace")
    return torch.empty(size.value, dtype=torch.uint8, device="cuda")


def espo_sample(logits: torch.Tensor, u: torch.Tensor, tokens_out: torch.Tensor, logp_out: Optional[torch.Tensor] = None,
                temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
                top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
                row_ids: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                status_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """One token per row of logits [n_rows, V] from the random numbers u, every row with its own parameters; see
    ``espo.h``.  Without a workspace (``espo_sample_workspace``) one is taken from torch's allocator on the call's stream."""
    if logits.dim() != 2 or logits.dtype not in _CODES:
        raise ValueError(f"logits must be a float32 or bfloat16 matrix, got {logits.dtype} {tuple(logits.shape)}")
    if logits.shape[1] > 1 and logits.stride(1) != 1:
        raise ValueError("logits must have unit stride along the vocabulary")
    _on_device(logits, "logits")
    n, v = logits.shape
    if row_ids is not None and row_ids.numel() < n:
        raise ValueError("row_ids is shorter than the rows")
    if status is not None and row_ids is None and status.numel() < n:
        raise ValueError("status is shorter than the rows")
    f32, i32 = torch.float32, torch.int32
    raw = _stream(stream)
    if workspace is None:
        if stream is None:
            workspace = espo_sample_workspace(n, v)
        else:
            with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(raw)):
                workspace = espo_sample_workspace(n, v)
    _b._check(_ops().espo_sample(logits.data_ptr(), _CODES[logits.dtype], logits.stride(0) if n > 1 else v, n, v,
                                 _ptr(u, "u", f32, (n,)), _ptr(temperature, "temperature", f32, (n,)),
                                 _ptr(top_k, "top_k", i32, (n,)), _ptr(top_p, "top_p", f32, (n,)),
                                 _ptr(min_p, "min_p", f32, (n,)), _ptr(row_ids, "row_ids", i32),
                                 _ptr(status, "status", torch.uint8), status.numel() if status is not None else 0,
                                 _ptr(tokens_out, "tokens_out", i32, (n,)), _ptr(logp_out, "logp_out", f32, (n,)),
                                 _ptr(workspace, "workspace", torch.uint8), workspace.numel(), _word(status_out), raw),
              "espo_sample")
