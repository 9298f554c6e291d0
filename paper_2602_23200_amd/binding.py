"""ctypes binding of libinnerq.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; this module turns
torch tensors into device pointers, keeps the caller-owned cache buffers alive
and raises on any non-zero status.  There is no CPU fallback: if the library is
not built, importing it here fails.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libinnerq.so")

SYM, ASYM, HYBRID = 0, 1, 2
KIND_INNER, KIND_OUTER, KIND_FP16 = 0, 1, 2
(BUF_K_CODES, BUF_K_SCALES, BUF_K_ZEROS, BUF_V_CODES, BUF_V_SCALES, BUF_V_ZEROS,
 BUF_K_SINK, BUF_V_SINK, BUF_K_RECENT, BUF_V_RECENT, BUF_COUNT) = range(11)
BUFFER_NAMES = ("k_codes", "k_scales", "k_zeros", "v_codes", "v_scales", "v_zeros",
                "k_sink", "v_sink", "k_recent", "v_recent")

OK, E_NULL, E_ARG, E_UNSUPPORTED, E_CAPACITY, E_ALIGN, E_WORKSPACE, E_HIP = 0, -1, -2, -3, -4, -5, -6, -7


class innerq_config_t(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("bits", C.c_int32), ("group", C.c_int32),
                ("w_sink", C.c_int32), ("w_recent", C.c_int32), ("k_mode", C.c_int32),
                ("v_mode", C.c_int32), ("sym_denominator", C.c_int32), ("kind", C.c_int32),
                ("capacity_tokens", C.c_int64), ("v_bits", C.c_int32), ("sparse_zeros", C.c_int32),
                ("page_pool_pages", C.c_int64)]


class innerq_cache_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in BUFFER_NAMES] + [("n_tokens", C.c_int64), ("store_ahead_tokens", C.c_int64),
                                                           ("page_table", C.c_void_p)]


class innerq_strides_t(C.Structure):
    _fields_ = [("batch", C.c_int64), ("head", C.c_int64), ("token", C.c_int64)]


class innerq_rotation_t(C.Structure):
    _fields_ = [("cos_table", C.c_void_p), ("sin_table", C.c_void_p), ("table_positions", C.c_int64),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("n_axes", C.c_int32), ("pair_axis", C.c_uint8 * 64)]


class InnerQError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib() -> C.CDLL:
    """Load libinnerq.so (built by __graft_entry__.build / paper_2602_23200_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2602_23200_amd.build`")
        L = C.CDLL(LIB_PATH)
        cfgp, cachep = C.POINTER(innerq_config_t), C.POINTER(innerq_cache_t)
        L.innerq_validate_config.argtypes = [cfgp]
        L.innerq_validate_config.restype = C.c_int
        L.innerq_buffer_bytes.argtypes = [cfgp, C.c_int]
        L.innerq_buffer_bytes.restype = C.c_size_t
        L.innerq_workspace_bytes.argtypes = [cfgp]
        L.innerq_workspace_bytes.restype = C.c_size_t
        L.innerq_status_string.argtypes = [C.c_int]
        L.innerq_status_string.restype = C.c_char_p
        L.innerq_partition.argtypes = [cfgp, C.c_int, C.c_int64] + [C.POINTER(C.c_int64)] * 3
        L.innerq_partition.restype = C.c_int
        L.innerq_calibrate_key_norm.argtypes = [cfgp, C.c_void_p, C.c_int64, C.c_int, C.c_void_p,
                                                C.c_void_p, C.c_void_p]
        L.innerq_calibrate_key_norm.restype = C.c_int
        L.innerq_quantize_append.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_int64,
                                             C.c_void_p, C.c_void_p]
        L.innerq_quantize_append.restype = C.c_int
        L.innerq_prefill.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_void_p,
                                     C.c_void_p, C.c_void_p]
        L.innerq_prefill.restype = C.c_int
        L.innerq_decode_attention.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                              C.c_void_p, C.c_size_t, C.c_void_p]
        L.innerq_decode_attention.restype = C.c_int
        L.innerq_decode_attention_static.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                                     C.c_void_p]
        L.innerq_decode_attention_static.restype = C.c_int
        L.innerq_quantize_ahead.argtypes = [cfgp, cachep, C.c_void_p]
        L.innerq_quantize_ahead.restype = C.c_int
        L.innerq_decode_attention_next.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                   C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.innerq_decode_attention_next.restype = C.c_int
        L.innerq_decode_step.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.innerq_decode_step.restype = C.c_int
        L.innerq_decode_step_ragged.argtypes = [cfgp, cachep, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                                C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_size_t,
                                                C.c_void_p]
        L.innerq_decode_step_ragged.restype = C.c_int
        L.innerq_append_deferred.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_void_p]
        L.innerq_append_deferred.restype = C.c_int
        rotp, strp = C.POINTER(innerq_rotation_t), C.POINTER(innerq_strides_t)
        L.innerq_rotate.argtypes = [cfgp, rotp, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, strp, C.c_void_p, strp,
                                    C.c_int32, C.c_int64, C.c_void_p]
        L.innerq_rotate.restype = C.c_int
        L.innerq_append_rotated.argtypes = [cfgp, cachep, rotp, C.c_void_p, C.c_void_p, strp, C.c_void_p, strp, C.c_int64, C.c_void_p,
                                            C.c_void_p]
        L.innerq_append_rotated.restype = C.c_int
        L.innerq_append_rotated_ragged.argtypes = [cfgp, cachep, rotp, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, strp, C.c_void_p,
                                                   strp, C.c_int64, C.c_void_p, C.c_void_p]
        L.innerq_append_rotated_ragged.restype = C.c_int
        L.innerq_chunk_workspace_bytes.argtypes = [cfgp, C.c_int64]
        L.innerq_chunk_workspace_bytes.restype = C.c_size_t
        L.innerq_chunk_attention.argtypes = [cfgp, cachep, C.c_void_p, strp, C.c_void_p, strp, C.c_void_p, strp, C.c_int64, C.c_void_p,
                                             C.c_void_p, strp, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.innerq_chunk_attention.restype = C.c_int
        L.innerq_chunk_attention_ragged.argtypes = [cfgp, cachep, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, strp, C.c_void_p, strp,
                                                    C.c_void_p, strp, C.c_int64, C.c_void_p, C.c_void_p, strp, C.c_int, C.c_void_p,
                                                    C.c_size_t, C.c_void_p]
        L.innerq_chunk_attention_ragged.restype = C.c_int
        L.innerq_profile_next_attention.argtypes = [C.c_void_p, C.c_void_p]
        L.innerq_profile_next_attention.restype = C.c_int
        L.innerq_select_inner_kernel.argtypes = [C.c_int]
        L.innerq_select_inner_kernel.restype = C.c_int
        L.innerq_stream_read_probe.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.innerq_stream_read_probe.restype = C.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().innerq_status_string(status).decode()


def make_config(batch, n_q_heads, n_kv_heads, head_dim, bits, group, w_sink, w_recent,
                k_mode=HYBRID, v_mode=HYBRID, sym_denominator=0, kind=KIND_INNER,
                capacity_tokens=0, v_bits=0, sparse_zeros=0, page_pool_pages=0) -> innerq_config_t:
    return innerq_config_t(batch, n_q_heads, n_kv_heads, head_dim, bits, group, w_sink, w_recent,
                           k_mode, v_mode, sym_denominator, kind, capacity_tokens, v_bits, sparse_zeros, page_pool_pages)


def innerq_validate_config(cfg: innerq_config_t) -> int:
    return lib().innerq_validate_config(C.byref(cfg))


def innerq_buffer_bytes(cfg: innerq_config_t, which: int) -> int:
    return lib().innerq_buffer_bytes(C.byref(cfg), which)


def innerq_workspace_bytes(cfg: innerq_config_t) -> int:
    return lib().innerq_workspace_bytes(C.byref(cfg))


def innerq_partition(cfg: innerq_config_t, which: int, n_tokens: int):
    a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
    st = lib().innerq_partition(C.byref(cfg), which, n_tokens, C.byref(a), C.byref(b), C.byref(c))
    if st != OK:
        raise InnerQError(st, "innerq_partition")
    return a.value, b.value, c.value


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    """Handle of `stream`, or of the current stream of the current device (looked up without making a Stream object of it:
    torch.cuda.current_stream() takes 2.4 us of the 8.3 that a decode step called from Python keeps the host, this 0.1)."""
    import torch
    if stream is not None:
        return stream.cuda_stream or None
    try:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None
    except AttributeError:                                # (private names: where a torch does not have them)
        return torch.cuda.current_stream().cuda_stream or None


@dataclass
class Cache:
    """Caller-owned cache buffers (torch uint8 tensors on the GPU) plus the C struct that points at them."""
    cfg: innerq_config_t
    buffers: dict
    c: innerq_cache_t

    @property
    def n_tokens(self) -> int:
        return self.c.n_tokens

    def view(self, name: str, dtype, shape):
        return self.buffers[name].view(dtype).view(*shape)


def allocate_cache(cfg: innerq_config_t, device="cuda", page_table=None) -> Cache:
    """Allocate every buffer the configuration needs, sized by innerq_buffer_bytes, zero-filled.
    page_table: for a paged store (cfg.page_pool_pages > 0), the caller's int32 [B, capacity_tokens / 64]
    tensor on the device; the cache keeps a reference to it."""
    import torch
    st = innerq_validate_config(cfg)
    if st != OK:
        raise InnerQError(st, "allocate_cache")
    bufs, c = {}, innerq_cache_t()
    for i, name in enumerate(BUFFER_NAMES):
        n = innerq_buffer_bytes(cfg, i)
        bufs[name] = torch.zeros(n, dtype=torch.uint8, device=device) if n else None
        setattr(c, name, _ptr(bufs[name]))
    c.n_tokens = 0
    c.store_ahead_tokens = 0
    if cfg.page_pool_pages > 0:
        assert page_table is not None and page_table.dtype == torch.int32 and page_table.is_contiguous()
        assert tuple(page_table.shape) == (cfg.batch, cfg.capacity_tokens // 64)
        bufs["page_table"] = page_table
        c.page_table = _ptr(page_table)
    return Cache(cfg, bufs, c)


def allocate_workspace(cfg: innerq_config_t, device="cuda"):
    import torch
    return torch.empty(innerq_workspace_bytes(cfg), dtype=torch.uint8, device=device)


def innerq_calibrate_key_norm(cfg: innerq_config_t, k, per_head: bool = False, stream=None):
    """k: fp16 CUDA tensor [B, Hk, N, d] -> (norm, inv_norm) fp32 [Hk, d]."""
    import torch
    assert k.dtype == torch.float16 and k.is_contiguous() and k.is_cuda
    norm = torch.empty(cfg.n_kv_heads, cfg.head_dim, dtype=torch.float32, device=k.device)
    inv = torch.empty_like(norm)
    st = lib().innerq_calibrate_key_norm(C.byref(cfg), k.data_ptr(), k.shape[2], int(per_head),
                                         norm.data_ptr(), inv.data_ptr(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_calibrate_key_norm")
    return norm, inv


def innerq_quantize_append(cache: Cache, k_new, v_new, k_inv_norm=None, stream=None) -> None:
    """k_new, v_new: fp16 CUDA tensors [B, Hk, T, d]."""
    import torch
    for t in (k_new, v_new):
        assert t.dtype == torch.float16 and t.is_contiguous() and t.is_cuda
    assert k_new.shape == v_new.shape
    st = lib().innerq_quantize_append(C.byref(cache.cfg), C.byref(cache.c), k_new.data_ptr(), v_new.data_ptr(),
                                      k_new.shape[2], _ptr(k_inv_norm), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_quantize_append")


def innerq_prefill(cache: Cache, k, v, per_head: bool = False, stream=None):
    """Calibrate the key factors over the prompt k and append the prompt (k divided by them) to the empty cache:
    k, v fp16 CUDA tensors [B, Hk, N, d] -> (norm, inv_norm) fp32 [Hk, d]."""
    import torch
    for t in (k, v):
        assert t.dtype == torch.float16 and t.is_contiguous() and t.is_cuda
    assert k.shape == v.shape
    norm = torch.empty(cache.cfg.n_kv_heads, cache.cfg.head_dim, dtype=torch.float32, device=k.device)
    inv = torch.empty_like(norm)
    st = lib().innerq_prefill(C.byref(cache.cfg), C.byref(cache.c), k.data_ptr(), v.data_ptr(), k.shape[2],
                              int(per_head), norm.data_ptr(), inv.data_ptr(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_prefill")
    return norm, inv


def innerq_decode_attention(cache: Cache, q, workspace, out=None, q_scale=None, stream=None):
    """q: fp16 CUDA tensor [B, Hq, d] -> out [B, Hq, d] (fp32 unless an fp16 `out` is passed)."""
    import torch
    assert q.dtype == torch.float16 and q.is_contiguous() and q.is_cuda
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    assert out.is_contiguous() and out.dtype in (torch.float32, torch.float16)
    st = lib().innerq_decode_attention(C.byref(cache.cfg), C.byref(cache.c), q.data_ptr(), _ptr(q_scale),
                                       out.data_ptr(), int(out.dtype == torch.float32), workspace.data_ptr(),
                                       workspace.numel() * workspace.element_size(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_decode_attention")
    return out


STATIC_WORKSPACE_BYTES = 32 << 20


def innerq_decode_attention_static(cache: Cache, q, out=None, q_scale=None, stream=None):
    """innerq_decode_attention with the split-K partials in the library's own static device array (no workspace)."""
    import torch
    assert q.dtype == torch.float16 and q.is_contiguous() and q.is_cuda
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    assert out.is_contiguous() and out.dtype in (torch.float32, torch.float16)
    st = lib().innerq_decode_attention_static(C.byref(cache.cfg), C.byref(cache.c), q.data_ptr(), _ptr(q_scale),
                                              out.data_ptr(), int(out.dtype == torch.float32), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_decode_attention_static")
    return out


def innerq_quantize_ahead(cache: Cache, stream=None) -> None:
    """Writes to the store what the next single-token append will evict (n_tokens unchanged)."""
    st = lib().innerq_quantize_ahead(C.byref(cache.cfg), C.byref(cache.c), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_quantize_ahead")


def innerq_decode_attention_next(cache: Cache, k_new, v_new, q, workspace, out=None, q_scale=None, stream=None):
    """Attention over the cache plus one token whose rows are k_new, v_new (fp16 [B, Hk, 1, d]), not yet appended."""
    import torch
    for t in (k_new, v_new, q):
        assert t.dtype == torch.float16 and t.is_contiguous() and t.is_cuda
    assert k_new.shape == v_new.shape and k_new.shape[2] == 1
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    assert out.is_contiguous() and out.dtype in (torch.float32, torch.float16)
    st = lib().innerq_decode_attention_next(C.byref(cache.cfg), C.byref(cache.c), k_new.data_ptr(), v_new.data_ptr(),
                                            q.data_ptr(), _ptr(q_scale), out.data_ptr(),
                                            int(out.dtype == torch.float32), workspace.data_ptr(),
                                            workspace.numel() * workspace.element_size(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_decode_attention_next")
    return out


def innerq_decode_step(cache: Cache, k_new, v_new, q, workspace, out=None, q_scale=None, stream=None):
    """innerq_decode_attention_next + innerq_append_deferred in one launch, or in two (merge and append share the second)."""
    import torch
    for t in (k_new, v_new, q):
        assert t.dtype == torch.float16 and t.is_contiguous() and t.is_cuda
    assert k_new.shape == v_new.shape and k_new.shape[2] == 1
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    assert out.is_contiguous() and out.dtype in (torch.float32, torch.float16)
    st = lib().innerq_decode_step(C.byref(cache.cfg), C.byref(cache.c), k_new.data_ptr(), v_new.data_ptr(),
                                  q.data_ptr(), _ptr(q_scale), out.data_ptr(), int(out.dtype == torch.float32),
                                  workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_decode_step")
    return out


def innerq_decode_step_ragged(cache: Cache, n_tokens_dev, max_tokens: int, k_new, v_new, q, workspace, out=None,
                              q_scale=None, stream=None):
    """innerq_decode_step with one token count per sequence in device memory (int32 CUDA tensor [B], advanced by
    the call); max_tokens bounds every count + 1."""
    import torch
    for t in (k_new, v_new, q):
        assert t.dtype == torch.float16 and t.is_contiguous() and t.is_cuda
    assert n_tokens_dev.dtype == torch.int32 and n_tokens_dev.is_cuda and n_tokens_dev.is_contiguous()
    assert k_new.shape == v_new.shape and k_new.shape[2] == 1
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    st = lib().innerq_decode_step_ragged(C.byref(cache.cfg), C.byref(cache.c), n_tokens_dev.data_ptr(), max_tokens,
                                         k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(), _ptr(q_scale),
                                         out.data_ptr(), int(out.dtype == torch.float32), workspace.data_ptr(),
                                         workspace.numel() * workspace.element_size(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_decode_step_ragged")
    return out


def sequence_view(cache: Cache, b: int) -> Cache:
    """Sequence b of a batched cache as a cache of its own (batch 1) over the same device memory: every buffer
    is laid out [B][...], so a sequence is one contiguous slice of each."""
    from dataclasses import replace as _replace
    cfg = innerq_config_t.from_buffer_copy(bytes(cache.cfg))
    assert cfg.page_pool_pages == 0, "the buffers of a paged store are pools, not per-sequence slices"
    B = cfg.batch
    cfg.batch = 1
    bufs, c = {}, innerq_cache_t()
    for name in BUFFER_NAMES:
        t = cache.buffers[name]
        bufs[name] = None if t is None else t.view(B, -1)[b]
        setattr(c, name, _ptr(bufs[name]))
    c.n_tokens = 0
    c.store_ahead_tokens = 0
    return Cache(cfg, bufs, c)


def innerq_append_deferred(cache: Cache, k_new, v_new, stream=None) -> None:
    """Copies the token k_new, v_new (fp16 [B, Hk, 1, d]) into its window and quantises one step ahead."""
    import torch
    for t in (k_new, v_new):
        assert t.dtype == torch.float16 and t.is_contiguous() and t.is_cuda
    assert k_new.shape == v_new.shape and k_new.shape[2] == 1
    st = lib().innerq_append_deferred(C.byref(cache.cfg), C.byref(cache.c), k_new.data_ptr(), v_new.data_ptr(),
                                      _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_append_deferred")


# ---- several new tokens of a sequence at once: rows [B, H, T, d] fp16 wherever they lie (a projection's output [B, T, H, d]
# transposed, say); channels contiguous, strides multiples of eight elements.

@dataclass
class Rotation:
    """Rotary positions: the caller's tables (kept alive here) and the C struct that names them."""
    c: innerq_rotation_t
    tables: tuple


def make_rotation(cos, sin, interleaved: bool = False, pair_axis=None) -> Rotation:
    """cos, sin: fp32 CUDA tensors [positions, rot_dim / 2]; pair_axis: the axis (0 to 2) of every pair, or None: one axis."""
    import torch
    for t in (cos, sin):
        assert t.dtype == torch.float32 and t.is_contiguous() and t.is_cuda and t.dim() == 2
    assert cos.shape == sin.shape and 1 <= cos.shape[1] <= 64
    axes = [0] * cos.shape[1] if pair_axis is None else [int(a) for a in pair_axis]
    assert len(axes) == cos.shape[1] and all(0 <= a <= 2 for a in axes)
    c = innerq_rotation_t(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(interleaved), max(axes) + 1)
    c.pair_axis[:len(axes)] = axes
    return Rotation(c, (cos, sin))


def _rows(t, cfg: innerq_config_t, heads: int, tokens: int, dtype=None):
    """Pointer and strides of rows [B, H, T, d]."""
    import torch
    shape, s = t.shape, t.stride()
    assert t.is_cuda and t.dtype == (dtype or torch.float16) and shape == (cfg.batch, heads, tokens, cfg.head_dim) and s[3] == 1
    if 1 in shape:                                         # (a dimension of one has no stride to speak of)
        s = [x if n > 1 else 0 for x, n in zip(s, shape)]
    return t.data_ptr(), C.byref(innerq_strides_t(s[0], s[1], s[2]))


def _positions(positions, rotation: Optional[Rotation], cfg: innerq_config_t, tokens: int) -> Optional[int]:
    import torch
    if positions is None or rotation is None:
        return None
    axes, shape = rotation.c.n_axes, positions.shape
    assert positions.is_cuda and positions.dtype == torch.int32 and positions.is_contiguous()
    assert shape == (axes, cfg.batch, tokens) or (axes == 1 and shape == (cfg.batch, tokens))
    return positions.data_ptr()


def _counts(t, cfg: innerq_config_t) -> Optional[int]:
    import torch
    if t is None:
        return None
    assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.shape == (cfg.batch,)
    return t.data_ptr()


def innerq_rotate(cfg: innerq_config_t, rotation: Rotation, x, out=None, positions=None, n_tokens: int = 0, n_tokens_dev=None,
                  t_new_dev=None, stream=None):
    """x [B, H, T, d] rotated into out (x itself for in place; a new tensor of x's layout if None).  positions int32 [axes, B, T], or
    None: token t stands at n_tokens (n_tokens_dev[b]) + t."""
    import torch
    if out is None:
        out = torch.empty_like(x)
    _, heads, T, _ = x.shape
    xp, xs = _rows(x, cfg, heads, T)
    yp, ys = _rows(out, cfg, heads, T)
    st = lib().innerq_rotate(C.byref(cfg), C.byref(rotation.c), _positions(positions, rotation, cfg, T), n_tokens,
                             _counts(n_tokens_dev, cfg), _counts(t_new_dev, cfg), xp, xs, yp, ys, heads, T, _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_rotate")
    return out


def _factors(f, cfg: innerq_config_t) -> Optional[int]:
    import torch
    if f is None:
        return None
    assert f.is_cuda and f.dtype == torch.float32 and f.is_contiguous() and tuple(f.shape) == (cfg.n_kv_heads, cfg.head_dim)
    return f.data_ptr()


def innerq_append_rotated(cache: Cache, k_new, v_new, rotation: Optional[Rotation] = None, positions=None, k_inv_norm=None,
                          stream=None) -> None:
    """innerq_quantize_append of k_new, v_new [B, Hk, T, d] where they lie, the keys rotated on their way in."""
    cfg, T = cache.cfg, k_new.shape[2]
    kp, ks = _rows(k_new, cfg, cfg.n_kv_heads, T)
    vp, vs = _rows(v_new, cfg, cfg.n_kv_heads, T)
    st = lib().innerq_append_rotated(C.byref(cfg), C.byref(cache.c), None if rotation is None else C.byref(rotation.c),
                                     _positions(positions, rotation, cfg, T), kp, ks, vp, vs, T, _factors(k_inv_norm, cfg), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_append_rotated")


def innerq_append_rotated_ragged(cache: Cache, n_tokens_dev, t_new_dev, k_new, v_new, rotation: Optional[Rotation] = None,
                                 positions=None, k_inv_norm=None, stream=None) -> None:
    """innerq_append_rotated with the counts of every sequence in device memory (int32 CUDA tensors [B]): n_tokens_dev cached,
    advanced by the call, t_new_dev new ones, at most T; every store is left one step ahead."""
    cfg, T = cache.cfg, k_new.shape[2]
    kp, ks = _rows(k_new, cfg, cfg.n_kv_heads, T)
    vp, vs = _rows(v_new, cfg, cfg.n_kv_heads, T)
    st = lib().innerq_append_rotated_ragged(C.byref(cfg), C.byref(cache.c), None if rotation is None else C.byref(rotation.c),
                                            _positions(positions, rotation, cfg, T), _counts(n_tokens_dev, cfg), _counts(t_new_dev, cfg),
                                            kp, ks, vp, vs, T, _factors(k_inv_norm, cfg), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_append_rotated_ragged")


def innerq_chunk_workspace_bytes(cfg: innerq_config_t, t_new: int) -> int:
    return lib().innerq_chunk_workspace_bytes(C.byref(cfg), t_new)


def allocate_chunk_workspace(cfg: innerq_config_t, t_new: int, device="cuda"):
    import torch
    return torch.empty(innerq_chunk_workspace_bytes(cfg, t_new), dtype=torch.uint8, device=device)


def _chunk_out(out, q):
    """The output rows: a new fp32 tensor [B, T, Hq, d] seen as [B, Hq, T, d] where none is given."""
    import torch
    if out is None:
        B, H, T, d = q.shape
        out = torch.empty(B, T, H, d, dtype=torch.float32, device=q.device).transpose(1, 2)
    assert out.dtype in (torch.float32, torch.float16)
    return out


def innerq_chunk_attention(cache: Cache, k_new, v_new, q, workspace, out=None, q_scale=None, stream=None):
    """q [B, Hq, T, d] attends to the cache and causally to the new rows k_new, v_new [B, Hk, T, d] (not appended by this call)
    -> out [B, Hq, T, d] (fp32 unless an fp16 `out` is passed)."""
    cfg, T = cache.cfg, q.shape[2]
    out = _chunk_out(out, q)
    kp, ks = _rows(k_new, cfg, cfg.n_kv_heads, T)
    vp, vs = _rows(v_new, cfg, cfg.n_kv_heads, T)
    qp, qs = _rows(q, cfg, cfg.n_q_heads, T)
    op, os_ = _rows(out, cfg, cfg.n_q_heads, T, out.dtype)
    st = lib().innerq_chunk_attention(C.byref(cfg), C.byref(cache.c), kp, ks, vp, vs, qp, qs, T, _factors(q_scale, cfg), op, os_,
                                      int(out.element_size() == 4), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                      _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_chunk_attention")
    return out


def innerq_chunk_attention_ragged(cache: Cache, n_tokens_dev, t_new_dev, max_tokens: int, k_new, v_new, q, workspace, out=None,
                                  q_scale=None, stream=None):
    """innerq_chunk_attention with the counts of every sequence in device memory (int32 CUDA tensors [B]): n_tokens_dev cached,
    t_new_dev new ones, at most T; max_tokens bounds their sum.  Rows of `out` beyond a sequence's new tokens are left as they were."""
    cfg, T = cache.cfg, q.shape[2]
    out = _chunk_out(out, q)
    kp, ks = _rows(k_new, cfg, cfg.n_kv_heads, T)
    vp, vs = _rows(v_new, cfg, cfg.n_kv_heads, T)
    qp, qs = _rows(q, cfg, cfg.n_q_heads, T)
    op, os_ = _rows(out, cfg, cfg.n_q_heads, T, out.dtype)
    st = lib().innerq_chunk_attention_ragged(C.byref(cfg), C.byref(cache.c), _counts(n_tokens_dev, cfg), _counts(t_new_dev, cfg), max_tokens,
                                             kp, ks, vp, vs, qp, qs, T, _factors(q_scale, cfg), op, os_, int(out.element_size() == 4),
                                             workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream))
    if st != OK:
        raise InnerQError(st, "innerq_chunk_attention_ragged")
    return out


def innerq_profile_next_attention(ev_start: Optional[int], ev_stop: Optional[int]) -> None:
    """ev_start / ev_stop: raw hipEvent_t handles (ints), or None to cancel."""
    lib().innerq_profile_next_attention(ev_start, ev_stop)


def innerq_select_inner_kernel(which: int) -> None:
    """0: the fp16 matrix form of the fused kernel everywhere (default); 1: the fp8 x fp4 kernel for 2-bit caches where it applies."""
    st = lib().innerq_select_inner_kernel(which)
    if st != OK:
        raise InnerQError(st, "innerq_select_inner_kernel")


def innerq_stream_read_probe(data, sink, ev_start: Optional[int] = None, ev_stop: Optional[int] = None,
                             stream=None) -> None:
    """Plain streaming read of the CUDA tensor `data` (byte count a multiple of 16); `sink`: >= 4 bytes."""
    st = lib().innerq_stream_read_probe(data.data_ptr(), data.numel() * data.element_size(), sink.data_ptr(),
                                        _stream(stream), ev_start, ev_stop)
    if st != OK:
        raise InnerQError(st, "innerq_stream_read_probe")
