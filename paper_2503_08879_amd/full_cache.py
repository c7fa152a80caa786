"""ctypes binding of the operators on the full cache (include/sagekv_cache.h): rotary positions, new tokens into a dense
or paged cache, attention over it.  Argument marshalling only, as in `binding`; every step runs in the library's kernels.

The descriptor makers check shapes, element types and strides once; the calls check that what they are given lies on the
current GPU and has the types of the descriptor, since a wrong pointer is not an error there but a fault.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import PagedKV, _check, _dtype_of, _stream, lib

ROTARY_HALF, ROTARY_PAIRS = 0, 1
SCALING_NONE, SCALING_LINEAR, SCALING_PARTS, SCALING_YARN = 0, 1, 2, 3

EXPORTS = ("sagekvc_rotary_frequencies", "sagekvc_rotary", "sagekvc_write", "sagekvc_attn_workspace_bytes", "sagekvc_attn")

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class RotaryMap(ctypes.Structure):
    _fields_ = [("rotary_dim", _i32), ("layout", _i32), ("transpose", _i32), ("amplitude", ctypes.c_float), ("inv_freq", _vp)]


class RotaryScaling(ctypes.Structure):
    _fields_ = [("kind", _i32), ("factor", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double),
                ("original_len", ctypes.c_double)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("n_tokens", _i64), ("n_heads", _i32), ("head_dim", _i32), ("dtype", _i32),
                ("x_stride_token", _i64), ("x_stride_head", _i64), ("out_stride_token", _i64), ("out_stride_head", _i64)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("n_problems", _i32), ("n_q_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32), ("capacity", _i64),
                ("k_stride_problem", _i64), ("k_stride_head", _i64), ("k_stride_token", _i64),
                ("v_stride_problem", _i64), ("v_stride_head", _i64), ("v_stride_token", _i64)]


class NewTokens(ctypes.Structure):
    _fields_ = [("n_tokens", _i64), ("q_stride_token", _i64), ("q_stride_head", _i64), ("k_stride_token", _i64), ("k_stride_head", _i64),
                ("v_stride_token", _i64), ("v_stride_head", _i64), ("q_out_stride_token", _i64), ("q_out_stride_head", _i64)]


_functions = {}


def _fn(name):
    """The library's function, with its argument types."""
    f = getattr(lib(), name)
    f.restype = ctypes.c_size_t if name.endswith("_bytes") else ctypes.c_int
    f.argtypes = {
        "sagekvc_rotary_frequencies": [_i32, ctypes.c_double, _vp, _vp, _vp],
        "sagekvc_rotary": [_vp] * 6,
        "sagekvc_write": [_vp] * 14,
        "sagekvc_attn_workspace_bytes": [_vp],
        "sagekvc_attn": [_vp] * 6 + [_i32] * 3 + [_vp] * 3 + [ctypes.c_size_t, _vp],
    }[name]
    _functions[name] = f
    return f


# The checks below are most of what a call costs on the host (a single token's launch takes 3 us on the GPU and was 8.5 on the host with a function call per
# tensor and byref per descriptor, 6 as it is).
_types = {}


def _begin(desc):
    """(element type of the descriptor, number of the current GPU)."""
    if not _types:
        import torch

        device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device) if torch.cuda.is_available() else lambda: None
        _types.update({binding.BF16: torch.bfloat16, binding.F32: torch.float32, "int": torch.int32, "device": device})
    return _types[desc.dtype], _types["device"]()


def _at(tensors, dtype, device):
    """Addresses of tensors of one element type on one GPU; None stays None."""
    got = []
    for t in tensors:
        if t is None:
            got.append(None)
            continue
        if t.dtype is not dtype or t.get_device() != device:
            raise ValueError(f"expected a tensor of {dtype} on GPU {device}, got {t.dtype} on {t.device}")
        got.append(t.data_ptr())
    return got


def _ints(t, n, device):
    """Address of an int32 tensor of at least n elements without gaps on that GPU; None stays None."""
    if t is None:
        return None
    if t.dtype is not _types["int"] or t.get_device() != device or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"expected {n} contiguous int32 values on GPU {device}, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


def _place(struct):
    """Address of a descriptor (ctypes.byref makes an object per call)."""
    return None if struct is None else ctypes.addressof(struct)


# ---------------------------------------------------------------------------------------- rotary positions
def sagekvc_rotary_frequencies(rotary_dim: int, base: float, kind: int = SCALING_NONE, factor: float = 1.0, low: float = 1.0,
                               high: float = 32.0, original_len: float = 1.0):
    """(frequencies as a list of rotary_dim / 2 floats, amplitude); host only.  See the header for the scalings."""
    freq, amplitude = (ctypes.c_double * max(1, rotary_dim // 2))(), ctypes.c_float()
    scaling = RotaryScaling(kind, factor, low, high, original_len)
    _check(_fn("sagekvc_rotary_frequencies")(rotary_dim, base, ctypes.byref(scaling), freq, ctypes.byref(amplitude)),
           "sagekvc_rotary_frequencies")
    return list(freq), amplitude.value


def rotary(inv_freq, layout: int = ROTARY_HALF, amplitude: float = 1.0, transpose: bool = False) -> RotaryMap:
    """A rotation by inv_freq, float64 [rotary_dim / 2] on the GPU, radians per position (kept alive by the result)."""
    import torch

    if inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or not inv_freq.is_cuda:
        raise ValueError("inv_freq: a contiguous float64 vector on the GPU is expected")
    m = RotaryMap(2 * inv_freq.numel(), layout, int(transpose), amplitude, inv_freq.data_ptr())
    m.tensor = inv_freq
    return m


def _step(t, i):
    """Stride of axis i; of one that has a single entry torch gives any number: 0."""
    return t.stride(i) if t.shape[i] > 1 else 0


def _rows(t, what):
    """(tokens, heads, head_dim, token stride, head stride) of t [n, heads, head_dim]."""
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError(f"{what}: [tokens, heads, head_dim] with a unit inner stride is expected")
    return (*t.shape, _step(t, 0), _step(t, 1))


def rotary_desc(x, out) -> RotaryDesc:
    """Descriptor for x and out [n, heads, head_dim], any strides with a unit inner stride."""
    n, h, d, *steps = _rows(x, "x")
    if _rows(out, "out")[:3] != (n, h, d) or out.dtype != x.dtype:
        raise ValueError("out: x's shape and element type are expected")
    return RotaryDesc(n, h, d, _dtype_of(x), *steps, *_rows(out, "out")[3:])


def sagekvc_rotary(desc: RotaryDesc, rot: RotaryMap, x, positions, out) -> None:
    """out = x's heads rotated by positions (int32 [n]); out may be x."""
    dt, dev = _begin(desc)
    x, out = _at((x, out), dt, dev)
    f = _functions.get("sagekvc_rotary") or _fn("sagekvc_rotary")
    code = f(_place(desc), _place(rot), x, _ints(positions, desc.n_tokens, dev), out, _stream())
    if code:
        _check(code, "sagekvc_rotary")


# ---------------------------------------------------------------------------------------- the full cache
def _same_cache(K, V):
    if K.dim() != 4 or V.shape != K.shape or V.dtype != K.dtype or K.stride(3) != 1 or V.stride(3) != 1:
        raise ValueError("K, V: two 4-dimensional tensors of one shape and element type with unit inner strides are expected")


def cache_desc(K, V, n_q_heads: int) -> CacheDesc:
    """Descriptor of a dense cache K, V [P, Hkv, capacity, d] (any strides with a unit inner stride)."""
    _same_cache(K, V)
    P, Hkv, capacity, d = K.shape
    steps = [_step(t, i) if i < 2 or capacity > 1 else d for t in (K, V) for i in range(3)]
    return CacheDesc(P, n_q_heads, Hkv, d, _dtype_of(K), capacity, *steps)


def paged_cache_desc(K_pool, V_pool, block_table, n_q_heads: int, capacity: int | None = None):
    """Descriptors of a paged cache: pools [n_pages, Hkv, page_size, d] (any strides with a unit inner stride), block_table
    int32 [P, pages per problem]; capacity defaults to what the table has entries for.  Returns (CacheDesc, PagedKV)."""
    import torch

    _same_cache(K_pool, V_pool)
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.stride(1) != 1 or not block_table.is_cuda:
        raise ValueError("block_table: int32 [problems, pages] with a unit inner stride on the GPU is expected")
    n_pages, Hkv, page, d = K_pool.shape
    P, per = block_table.shape
    capacity = per * page if capacity is None else capacity
    if not 0 < capacity <= per * page:
        raise ValueError("capacity: more tokens than the block table has entries for")
    desc = CacheDesc(P, n_q_heads, Hkv, d, _dtype_of(K_pool), capacity, 0, _step(K_pool, 1), K_pool.stride(2), 0, _step(V_pool, 1),
                     V_pool.stride(2))
    # (the table is kept alive by the description)
    pitch = block_table.stride(0) if P > 1 else per
    pages = PagedKV(block_table.data_ptr(), pitch, page, n_pages, _step(K_pool, 0), _step(V_pool, 0))
    pages.tensor = block_table
    return desc, pages


def new_tokens(q, k_new, v_new, q_out) -> NewTokens:
    """Strides of packed new tokens: q, q_out [n, Hq, d] (both None: no queries), k_new, v_new [n, Hkv, d]."""
    n, hkv, d, kt, kh = _rows(k_new, "k_new")
    vs = _rows(v_new, "v_new")
    if vs[:3] != (n, hkv, d) or v_new.dtype != k_new.dtype or (q is None) != (q_out is None):
        raise ValueError("k_new and v_new of one shape and element type, and q_out with q, are expected")
    qs = [0, 0, 0, 0]
    if q is not None:
        a, b = _rows(q, "q"), _rows(q_out, "q_out")
        if a[:3] != b[:3] or a[0] != n or a[2] != d or q.dtype != k_new.dtype or q_out.dtype != q.dtype:
            raise ValueError("q and q_out: as many tokens, head_dim and element type as k_new are expected")
        qs = [a[3], a[4], b[3], b[4]]
    t = NewTokens(n, qs[0], qs[1], kt, kh, vs[3], vs[4], qs[2], qs[3])
    t.heads = (q.shape[1] if q is not None else 0, hkv)
    return t


def sagekvc_write(desc: CacheDesc, pages, tokens: NewTokens, rot, q, k_new, v_new, token_offsets, seq_lens, positions, q_out, K, V) -> None:
    """New tokens into the cache, keys and queries rotated on the way.  token_offsets int32 [P + 1] or None (one token per problem); seq_lens
    int32 [P], the lengths with the new tokens; positions int32 [n] or None (the places); rot None: no rotation; pages None: dense."""
    heads = getattr(tokens, "heads", None)  # (strides filled in by hand know of none)
    if heads is not None and heads != (desc.n_q_heads if q is not None else 0, desc.n_kv_heads):
        raise ValueError(f"new tokens of {heads} heads for a cache of {desc.n_q_heads} and {desc.n_kv_heads}")
    dt, dev = _begin(desc)
    q, k_new, v_new, q_out, K, V = _at((q, k_new, v_new, q_out, K, V), dt, dev)
    P = desc.n_problems
    f = _functions.get("sagekvc_write") or _fn("sagekvc_write")
    code = f(_place(desc), _place(pages), _place(tokens), _place(rot), q, k_new, v_new, _ints(token_offsets, P + 1, dev), _ints(seq_lens, P, dev),
             _ints(positions, tokens.n_tokens, dev), q_out, K, V, _stream())
    if code:
        _check(code, "sagekvc_write")


def sagekvc_attn_workspace_bytes(desc: CacheDesc) -> int:
    return _fn("sagekvc_attn_workspace_bytes")(ctypes.byref(desc))


def sagekvc_attn(desc: CacheDesc, pages, q, K, V, seq_lens, max_len: int, n_sink: int, n_recent: int, out, lse, workspace) -> None:
    """Attention of one new token per problem, q [P, Hq, d], over the first seq_lens[p] (int32 [P], at most max_len) tokens of the full cache; n_recent > 0:
    over the first n_sink and the last n_recent of them.  out float32 [P, Hq, d]; lse float32 [P, Hq] or None."""
    dt, dev = _begin(desc)
    P, heads = desc.n_problems, desc.n_problems * desc.n_q_heads
    size = heads * desc.head_dim
    if q.numel() != size or out.numel() != size or (lse is not None and (lse.numel() != heads or not lse.is_contiguous())) or not (
            q.is_contiguous() and out.is_contiguous() and workspace.is_contiguous()):
        raise ValueError("q and out: [problems, heads, head_dim], lse: [problems, heads], contiguous, are expected, and a contiguous workspace")
    q, K, V = _at((q, K, V), dt, dev)
    out, lse = _at((out, lse), _types[binding.F32], dev)
    at, = _at((workspace,), workspace.dtype, dev)
    f = _functions.get("sagekvc_attn") or _fn("sagekvc_attn")
    code = f(_place(desc), _place(pages), q, K, V, _ints(seq_lens, P, dev), max_len, n_sink, n_recent, out, lse, at,
             workspace.numel() * workspace.element_size(), _stream())
    if code:
        _check(code, "sagekvc_attn")
