"""ctypes binding of libtri (include/tri.h).

Argument marshalling only: every step of the layer runs in the HIP kernels of
libtri.so.  torch supplies device memory (``tensor.data_ptr()``) and the
current HIP stream.  Loading fails loudly if the library has not been built.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Dict, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtri.so")

TRI_OK, TRI_ERR_NULL, TRI_ERR_SHAPE, TRI_ERR_UNSUPPORTED = 0, -1, -2, -3
TRI_ERR_RANGE, TRI_ERR_ALIGN, TRI_ERR_WORKSPACE, TRI_ERR_HIP, TRI_ERR_ALIAS = -4, -5, -6, -7, -8
TRI_ERR_SCRATCH = -9
NOALLOC_SCRATCH_BYTES = 64 << 20
TRI_BF16, TRI_F32 = 0, 1
TRI_KV8_INT8, TRI_KV8_E4M3 = 0, 1
TRI_ROPE_HALF, TRI_ROPE_INTERLEAVED = 0, 1
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "turns": 3, "index": 4}  # tri_rope_scaling
TRI_F_QKV_BIAS, TRI_F_MOE, TRI_F_MOE_RENORM, TRI_F_QK_NORM, TRI_F_MROPE = 1, 2, 4, 8, 16


class LayerConfig(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("ffn_dim", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("expert_ffn_dim", ctypes.c_int32),
                ("rms_eps", ctypes.c_float), ("rope_base", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("mrope_section", ctypes.c_int32 * 3)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("attn_norm", "w_qkv", "b_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down",
                 "w_router", "q_norm", "k_norm")]


class KVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_slots", ctypes.c_int32),
                ("max_seq", ctypes.c_int32), ("block_table", ctypes.c_void_p),
                ("block_size", ctypes.c_int32), ("n_blocks", ctypes.c_int32)]


class KV8CacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "mass", "stamp")] + \
               [("n_slots", ctypes.c_int32), ("max_seq", ctypes.c_int32),
                ("block_table", ctypes.c_void_p)] + \
               [(n, ctypes.c_int32) for n in ("block_size", "n_blocks", "format", "scale_rows")]


class RopeConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("head_dim", "rotary_dim", "layout", "scaling",
                                              "original_len")] + \
               [(n, ctypes.c_float) for n in ("base", "factor", "low", "high", "magnitude")]


class RopeTable(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("head_dim", "rotary_dim", "layout")] + \
               [("magnitude", ctypes.c_float), ("turns", ctypes.c_double * 128)]


class BatchStruct(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
                ("max_q_len", ctypes.c_int32), ("max_ctx_len", ctypes.c_int32),
                ("cu_q", ctypes.c_void_p), ("ctx_len", ctypes.c_void_p),
                ("slot", ctypes.c_void_p), ("pos", ctypes.c_void_p)]


class WorkspaceMap(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("h", "q", "attn", "x1", "h2", "act", "perm", "y",
                                                "total")]


class Profile(ctypes.Structure):
    _fields_ = [("n_stages", ctypes.c_int32), ("name", ctypes.c_char_p * 16),
                ("launches", ctypes.c_int32 * 16), ("total_ms", ctypes.c_double * 16)]


class Work(ctypes.Structure):
    _fields_ = [("n_stages", ctypes.c_int32), ("name", ctypes.c_char_p * 16),
                ("runs", ctypes.c_int32 * 16), ("flops", ctypes.c_double * 16),
                ("bytes", ctypes.c_double * 16)]


class TriError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: tri status {status} ({status_string(status)})")


_lib: Optional[ctypes.CDLL] = None

_FUNCS = {
    "tri_workspace_size": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "tri_workspace_layout": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "tri_layer_prefill": (ctypes.c_int, [ctypes.c_void_p] * 4 + [ctypes.c_void_p] * 4
                          + [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "tri_layer_decode": (ctypes.c_int, [ctypes.c_void_p] * 4 + [ctypes.c_void_p] * 4
                         + [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "tri_layer_decode_noalloc": (ctypes.c_int, [ctypes.c_void_p] * 4 + [ctypes.c_void_p] * 4
                                 + [ctypes.c_void_p]),
    "tri_kvcache_append": (ctypes.c_int, [ctypes.c_void_p] * 6),
    "tri_moe_route": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_void_p]),
    "tri_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "tri_profile_enable": (ctypes.c_int, [ctypes.c_int32]),
    "tri_profile_read": (ctypes.c_int, [ctypes.c_void_p]),
    "tri_layer_work": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_void_p]),
    "tri_phase_intensity": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "tri_version": (ctypes.c_int32, []),
    "tri_linear_workspace_size": (ctypes.c_int, [ctypes.c_int32] * 3 + [ctypes.c_void_p]),
    "tri_linear": (ctypes.c_int, [ctypes.c_void_p] * 3 + [ctypes.c_int32] * 3
                   + [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "tri_rope_table_make": (ctypes.c_int, [ctypes.c_void_p] * 2),
    "tri_rope": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                ctypes.c_int64, ctypes.c_void_p] + [ctypes.c_int32] * 3
                 + [ctypes.c_void_p]),
    "tri_workspace_size_kv8": (ctypes.c_int, [ctypes.c_void_p] * 4),
    "tri_layer_prefill_kv8": (ctypes.c_int, [ctypes.c_void_p] * 9
                              + [ctypes.c_size_t, ctypes.c_void_p]),
    "tri_layer_decode_kv8": (ctypes.c_int, [ctypes.c_void_p] * 9
                             + [ctypes.c_size_t, ctypes.c_void_p]),
    "tri_kv8_append": (ctypes.c_int, [ctypes.c_void_p] * 5 + [ctypes.c_int64, ctypes.c_void_p]),
    "tri_kv8_attention_workspace_size": (ctypes.c_int, [ctypes.c_void_p] * 4),
    "tri_kv8_attention": (ctypes.c_int, [ctypes.c_void_p] * 4
                          + [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                             ctypes.c_void_p]),
    "tri_kv8_select_workspace_size": (ctypes.c_int, [ctypes.c_void_p] * 3
                                      + [ctypes.c_int32, ctypes.c_void_p]),
    "tri_kv8_select": (ctypes.c_int, [ctypes.c_void_p] * 3 + [ctypes.c_int32] * 3
                       + [ctypes.c_void_p] * 3 + [ctypes.c_size_t, ctypes.c_void_p]),
    "tri_kv8_move": (ctypes.c_int, [ctypes.c_void_p] * 4 + [ctypes.c_int32, ctypes.c_void_p]),
}


def lib() -> ctypes.CDLL:
    """The loaded libtri.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libtri.so not built at {LIB_PATH}; run "
                               "`python -m paper_2606_29629_amd.build` first")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _FUNCS.items():
            f = getattr(l, name)
            f.restype = res
            f.argtypes = args
        _lib = l
    return _lib


def status_string(s: int) -> str:
    return lib().tri_status_string(s).decode()


def _check(status: int, what: str) -> None:
    if status != TRI_OK:
        raise TriError(status, what)


def make_config(cfg, f32: bool = False) -> LayerConfig:
    """LayerConfig from any object with the layer's attribute names; f32
    selects the fp32 storage mode (TRI_F32: fp32 weights, activations and
    cache)."""
    flags = 0
    if getattr(cfg, "qkv_bias", False):
        flags |= TRI_F_QKV_BIAS
    if getattr(cfg, "qk_norm", False):
        flags |= TRI_F_QK_NORM
    sec = getattr(cfg, "mrope_section", None)
    if sec:
        flags |= TRI_F_MROPE
    n_exp = int(getattr(cfg, "n_experts", 0) or 0)
    if n_exp > 0:
        flags |= TRI_F_MOE
        if getattr(cfg, "moe_renorm", True):
            flags |= TRI_F_MOE_RENORM
    return LayerConfig(int(cfg.hidden), int(cfg.n_q_heads), int(cfg.n_kv_heads),
                       int(cfg.head_dim), int(getattr(cfg, "ffn_dim", 0) or 0), n_exp,
                       int(getattr(cfg, "top_k", 0) or 0),
                       int(getattr(cfg, "expert_ffn_dim", 0) or 0), float(cfg.rms_eps),
                       float(cfg.rope_base), TRI_F32 if f32 else TRI_BF16, flags,
                       (ctypes.c_int32 * 3)(*(sec or (0, 0, 0))))


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


class DeviceBatch:
    """A ragged batch: device int32 arrays plus the host scalars that size launches."""

    def __init__(self, slot: Sequence[int], ctx_len: Sequence[int], q_len: Sequence[int],
                 device="cuda", pos=None):
        """pos: the rotary positions (default ctx_len + i per token), or the
        three planes [3, n_tokens] of a TRI_F_MROPE layer."""
        import numpy as np
        import torch
        slot = np.asarray(slot, dtype=np.int32)
        ctx = np.asarray(ctx_len, dtype=np.int32)
        q = np.asarray(q_len, dtype=np.int32)
        cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
        if pos is not None:
            pos = np.ascontiguousarray(pos, dtype=np.int32).ravel()
        elif len(q):
            pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, q)]).astype(np.int32)
        else:
            pos = np.zeros(0, np.int32)
        self.n_seqs, self.n_tokens = int(len(q)), int(cu[-1])
        self.max_q_len = int(q.max()) if len(q) else 0
        self.max_ctx_len = int(ctx.max()) if len(ctx) else 0
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
        self.cu_q, self.ctx_len, self.slot, self.pos = dev(cu), dev(ctx), dev(slot), dev(pos)
        self.host = dict(slot=slot, ctx_len=ctx, q_len=q)

    def struct(self) -> BatchStruct:
        return BatchStruct(self.n_seqs, self.n_tokens, self.max_q_len, self.max_ctx_len,
                           _ptr(self.cu_q), _ptr(self.ctx_len), _ptr(self.slot), _ptr(self.pos))

    def advance(self) -> None:
        """In place: every sequence has appended its new tokens; next step is one token each."""
        import numpy as np
        h = self.host
        ctx = (h["ctx_len"] + h["q_len"]).astype(np.int32)
        self.__init__(h["slot"], ctx, np.ones_like(h["q_len"]), device=self.cu_q.device)


def weights_struct(w: Dict[str, object]) -> LayerWeights:
    return LayerWeights(*[_ptr(w.get(n)) for n in
                          ("attn_norm", "w_qkv", "b_qkv", "w_o", "mlp_norm", "w_gate_up",
                           "w_down", "w_router", "q_norm", "k_norm")])


def workspace_size(cfg: LayerConfig, batch: DeviceBatch, cache=None) -> int:
    """Workspace bytes of a layer call; cache: the KV8Cache of one on an 8-bit cache."""
    n = ctypes.c_size_t(0)
    b = batch.struct()
    if isinstance(cache, KV8Cache):
        _check(lib().tri_workspace_size_kv8(ctypes.byref(cfg), cache._ref, ctypes.byref(b),
                                            ctypes.byref(n)), "tri_workspace_size_kv8")
        return n.value
    _check(lib().tri_workspace_size(ctypes.byref(cfg), ctypes.byref(b), ctypes.byref(n)),
           "tri_workspace_size")
    return n.value


def workspace_layout(cfg: LayerConfig, batch: DeviceBatch) -> WorkspaceMap:
    m = WorkspaceMap()
    b = batch.struct()
    _check(lib().tri_workspace_layout(ctypes.byref(cfg), ctypes.byref(b), ctypes.byref(m)),
           "tri_workspace_layout")
    return m


class PagedCache:
    """A paged KV cache: K and V pools [n_blocks, Hkv, block_size, D] (bf16) and
    a device int32 block table [n_slots, max_seq / block_size]."""

    def __init__(self, k_pool, v_pool, block_table, max_seq: int):
        self.k, self.v, self.block_table = k_pool, v_pool, block_table
        self.n_slots = int(block_table.shape[0])
        self.max_seq = int(max_seq)
        self.block_size = int(k_pool.shape[2])
        self.n_blocks = int(k_pool.shape[0])

    def __getitem__(self, i):
        return (self.k, self.v)[i]


def kv_struct(cache) -> KVCache:
    """KVCache for a contiguous (k, v) pair [n_slots, Hkv, max_seq, D] or a PagedCache."""
    if isinstance(cache, PagedCache):
        return KVCache(_ptr(cache.k), _ptr(cache.v), cache.n_slots, cache.max_seq,
                       _ptr(cache.block_table), cache.block_size, cache.n_blocks)
    return KVCache(_ptr(cache[0]), _ptr(cache[1]), int(cache[0].shape[0]),
                   int(cache[0].shape[2]), None, 0, 0)


def _layer(fn_name, cfg, w, cache, batch, x, out, workspace, route_idx, route_w, stream):
    import torch
    if out is None:
        with _memory(stream, x.device):
            out = torch.empty_like(x)
    if isinstance(cache, KV8Cache):
        if (cfg.n_kv_heads, cfg.head_dim) != (cache.n_kv_heads, cache.head_dim):
            raise ValueError(f"{fn_name}: the cache has {cache.n_kv_heads} heads of {cache.head_dim}")
        _on_gpu(fn_name, stream, x, out, cache.k, batch.slot, workspace)
        fn_name, kc = fn_name + "_kv8", cache.struct()
    else:
        kc = kv_struct(cache)
    need = workspace_size(cfg, batch, cache)
    if workspace is None:
        workspace = _empty(stream, max(need, 1), torch.uint8, x.device)
    ws = weights_struct(w)
    b = batch.struct()
    st = getattr(lib(), fn_name)(ctypes.byref(cfg), ctypes.byref(ws), ctypes.byref(kc),
                                 ctypes.byref(b), _ptr(x), _ptr(out), _ptr(route_idx),
                                 _ptr(route_w), _ptr(workspace), workspace.numel(),
                                 _stream(stream))
    _check(st, fn_name)
    return out, workspace


def layer_prefill(cfg, w, cache, batch, x, out=None, workspace=None, route_idx=None,
                  route_w=None, stream=None):
    """One decoder layer over a ragged batch; returns (out, workspace).  cache: a (k, v)
    pair, a PagedCache or a KV8Cache."""
    return _layer("tri_layer_prefill", cfg, w, cache, batch, x, out, workspace, route_idx,
                  route_w, stream)


def layer_decode(cfg, w, cache, batch, x, out=None, workspace=None, route_idx=None,
                 route_w=None, stream=None):
    """One decode step (one new token per sequence); returns (out, workspace).  cache: as in
    layer_prefill."""
    return _layer("tri_layer_decode", cfg, w, cache, batch, x, out, workspace, route_idx,
                  route_w, stream)


def layer_decode_noalloc(cfg, w, cache, batch, x, out=None, route_idx=None, route_w=None,
                         stream=None):
    """One decode step on the library's fixed device scratch (no workspace;
    tri_layer_decode_noalloc); returns out."""
    import torch
    if out is None:
        with _memory(stream, x.device):
            out = torch.empty_like(x)
    ws = weights_struct(w)
    kc = kv_struct(cache)
    b = batch.struct()
    _check(lib().tri_layer_decode_noalloc(ctypes.byref(cfg), ctypes.byref(ws), ctypes.byref(kc),
                                          ctypes.byref(b), _ptr(x), _ptr(out), _ptr(route_idx),
                                          _ptr(route_w), _stream(stream)),
           "tri_layer_decode_noalloc")
    return out


def kvcache_append(cfg, cache, batch, k_new, v_new, stream=None) -> None:
    kc = kv_struct(cache)
    b = batch.struct()
    _check(lib().tri_kvcache_append(ctypes.byref(cfg), ctypes.byref(kc), ctypes.byref(b),
                                    _ptr(k_new), _ptr(v_new), _stream(stream)),
           "tri_kvcache_append")


def linear_workspace_size(M: int, N: int, K: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().tri_linear_workspace_size(int(M), int(N), int(K), ctypes.byref(n)),
           "tri_linear_workspace_size")
    return n.value


def linear(a, b, out=None, workspace=None, stream=None):
    """out = a @ b^T (bf16 [M, K] x bf16 [N, K] -> bf16 [M, N]) through tri_linear."""
    import torch
    M, K = a.shape
    N = b.shape[0]
    if out is None:
        out = _empty(stream, (M, N), torch.bfloat16, a.device)
    need = linear_workspace_size(M, N, K)
    if workspace is None and need:
        workspace = _empty(stream, need, torch.uint8, a.device)
    wb = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().tri_linear(_ptr(a), _ptr(b), _ptr(out), M, N, K, _ptr(workspace), wb,
                            _stream(stream)), "tri_linear")
    return out


def make_rope(head_dim: int, rotary_dim: Optional[int] = None, base: float = 1e6,
              interleaved: bool = False, scaling: str = "none", factor: float = 1.0,
              low: float = 1.0, high: float = 32.0, original_len: int = 0,
              magnitude: float = 1.0) -> RopeTable:
    """What rope() takes, formed once (tri_rope_config, tri_rope_table_make); scaling: a key
    of ROPE_SCALING."""
    if scaling not in ROPE_SCALING:
        raise ValueError(f"scaling {scaling!r}: one of {sorted(ROPE_SCALING)}")
    cfg = RopeConfig(int(head_dim), int(head_dim if rotary_dim is None else rotary_dim),
                     TRI_ROPE_INTERLEAVED if interleaved else TRI_ROPE_HALF,
                     ROPE_SCALING[scaling], int(original_len), float(base), float(factor),
                     float(low), float(high), float(magnitude))
    table = RopeTable()
    _check(lib().tri_rope_table_make(ctypes.byref(cfg), ctypes.byref(table)), "tri_rope_table_make")
    return table


def _rows(x, what: str, last: int) -> int:
    """Token stride of x [tokens, heads, last] whose heads are contiguous (of one token: any)."""
    if x.dim() == 3:
        n, heads, d = x.shape
        st = x.stride()
        if d == last and st[2] == 1 and (heads <= 1 or st[1] == last):
            return st[0] if n > 1 else heads * last
    raise ValueError(f"{what}: [tokens, heads, {last}] with contiguous heads expected")


def _on_gpu(what: str, stream, first, *others) -> Optional[int]:
    """The kernels follow plain addresses: every tensor of a call on the current GPU, and the
    stream too.  Returns the handle of `stream`, or of the current stream."""
    import torch
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{what}: tensors on {first.device} and {t.device}")
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{what}: tensors on {first.device}, not on the current GPU")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError(f"{what}: tensors on {first.device}, a stream of GPU {stream.device_index}")
    return getattr(stream, "cuda_stream", stream)


def _memory(stream, device):
    """A context in which torch allocates from the memory of the stream that a call runs on:
    what is freed when the call returns is not handed to another stream while the kernels
    still use it."""
    import torch
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream, device=device)
    return torch.cuda.stream(stream)


def _empty(stream, shape, dtype, device):
    """torch.empty from the memory of the call's stream."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _memory(stream, device):
        return torch.empty(shape, dtype=dtype, device=device)


def rope(table: RopeTable, x, pos, out=None, stream=None):
    """x [tokens, heads, head_dim] (bf16 or float32, tokens any stride apart) with its
    heads rotated to int32 positions pos [tokens] (tri_rope); out=x: in place."""
    import torch
    if out is None:
        out = _empty(stream, x.shape, x.dtype, x.device)
    f32 = x.dtype == torch.float32
    if not f32 and x.dtype != torch.bfloat16 or out.dtype != x.dtype:
        raise ValueError(f"rope: bf16 or float32 in and out, got {x.dtype} and {out.dtype}")
    xs, ys = _rows(x, "rope: x", table.head_dim), _rows(out, "rope: out", table.head_dim)
    n, heads, _ = x.shape
    if pos.dtype != torch.int32 or not pos.is_contiguous() or pos.numel() != n:
        raise ValueError("rope: pos is a contiguous int32 [tokens]")
    if out.shape != x.shape:
        raise ValueError(f"rope: out {tuple(out.shape)}, x {tuple(x.shape)}")
    stream = _on_gpu("rope", stream, x, pos, out)
    st = lib().tri_rope(ctypes.byref(table), x.data_ptr(), xs, out.data_ptr(), ys, pos.data_ptr(),
                        n, heads, f32, stream)
    if st:
        raise TriError(st, "tri_rope")
    return out


class KV8Cache:
    """An 8-bit KV cache (tri_kv8_cache): codes k, v [panels, Hkv, rows, D] (int8, or
    float8_e4m3fn), a float32 scale per head and scale_rows rows, optionally the rows'
    accumulated attention weight and their tokens' positions.  Contiguous (a panel is a slot),
    or paged with block_table [n_slots, max_seq / rows] and max_seq.

    The calls work on the tensors that the attributes k, v, k_scale, v_scale, mass, stamp and
    block_table name: one of them may be replaced by another of its shape and type (mass and
    stamp by None too, or set where there were none), as `cache.mass = cache.mass * 0.5` does.
    (A captured graph keeps those it was captured with.)  The other attributes are fixed."""

    _TENSORS = ("k", "v", "k_scale", "v_scale", "mass", "stamp", "block_table")

    def __init__(self, k, v, k_scale, v_scale, scale_rows: int, mass=None, stamp=None,
                 block_table=None, max_seq: Optional[int] = None):
        import torch
        formats = {torch.int8: TRI_KV8_INT8, torch.float8_e4m3fn: TRI_KV8_E4M3}
        if k.dtype not in formats or k.dim() != 4:
            raise ValueError("KV8Cache: k and v are int8 or float8_e4m3fn [panels, Hkv, rows, D]")
        panels, heads, rows, d = k.shape
        if block_table is None:
            if max_seq is not None and max_seq != rows:  # (a slot's rows lie max_seq apart)
                raise ValueError(f"KV8Cache: max_seq {max_seq} of a contiguous cache of {rows} rows")
        elif max_seq is None or block_table.dim() != 2 or block_table.shape[1] * rows != max_seq:
            raise ValueError("KV8Cache: block_table is int32 [n_slots, max_seq / rows]")
        paged = block_table is not None
        fixed = dict(scale_rows=int(scale_rows), head_dim=int(d), n_kv_heads=int(heads),
                     n_slots=int(block_table.shape[0]) if paged else int(panels),
                     max_seq=int(max_seq) if paged else int(rows))
        codes, scales = tuple(k.shape), (panels, heads, -(-rows // fixed["scale_rows"]))
        self.__dict__.update(fixed, _device=k.device, _kind={
            "k": (codes, k.dtype), "v": (codes, k.dtype), "k_scale": (scales, torch.float32),
            "v_scale": (scales, torch.float32), "mass": (codes[:3], torch.float32),
            "stamp": (codes[:3], torch.int32),
            "block_table": (tuple(block_table.shape), torch.int32) if paged else None})
        struct = KV8CacheStruct(n_slots=self.n_slots, max_seq=self.max_seq,
                                block_size=int(rows) if paged else 0, n_blocks=int(panels) if paged else 0,
                                format=formats[k.dtype], scale_rows=self.scale_rows)
        self.__dict__.update(_struct=struct, _ref=ctypes.byref(struct))
        for name, t in zip(self._TENSORS, (k, v, k_scale, v_scale, mass, stamp, block_table)):
            setattr(self, name, t)

    def __setattr__(self, name, t):
        if name not in self._TENSORS:
            raise AttributeError(f"KV8Cache: {name} cannot be set")
        kind = self._kind[name]
        if t is None:
            if kind is not None and name not in ("mass", "stamp"):
                raise ValueError(f"KV8Cache: {name} is {kind[1]} {kind[0]}")
        elif kind is None:
            raise ValueError(f"KV8Cache: {name} of a contiguous cache")
        else:
            if (tuple(t.shape), t.dtype) != kind:
                raise ValueError(f"KV8Cache: {name} is {kind[1]} {kind[0]}")
            if not t.is_contiguous():
                raise ValueError("KV8Cache: contiguous tensors expected")
            if t.device != self._device:
                raise ValueError("KV8Cache: tensors on one device expected")
        self.__dict__[name] = t
        setattr(self._struct, name, _ptr(t))

    def __delattr__(self, name):
        raise AttributeError(f"KV8Cache: {name} cannot be deleted")

    def __reduce__(self):  # (a copy has a struct of its own)
        return KV8Cache, (self.k, self.v, self.k_scale, self.v_scale, self.scale_rows, self.mass, self.stamp,
                          self.block_table, self.max_seq)

    @classmethod
    def empty(cls, cfg: LayerConfig, n_slots: int, max_seq: int, format: str = "int8",
              scale_rows: int = 32, mass: bool = False, stamp: bool = False, block_table=None,
              block_size: int = 0, n_blocks: int = 0, device="cuda"):
        """A cache without rows: contiguous, or paged with a block_table."""
        import torch
        dt = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}[format]
        paged = block_table is not None
        panels, rows = (n_blocks, block_size) if paged else (n_slots, max_seq)
        shape = panels, cfg.n_kv_heads, rows
        codes = [torch.zeros(*shape, cfg.head_dim, dtype=torch.uint8, device=device).view(dt)
                 for _ in range(2)]
        scales = [torch.ones(panels, cfg.n_kv_heads, -(-rows // scale_rows), device=device)
                  for _ in range(2)]
        return cls(*codes, *scales, scale_rows,
                   mass=torch.zeros(shape, device=device) if mass else None,
                   stamp=torch.zeros(shape, dtype=torch.int32, device=device) if stamp else None,
                   block_table=block_table, max_seq=max_seq if paged else None)

    def struct(self) -> KV8CacheStruct:
        return self._struct


def _kv8(what, cfg, cache, batch, stream, *tensors):
    """The first arguments of a call on an 8-bit cache, and its stream."""
    if cfg.n_kv_heads != cache.n_kv_heads or cfg.head_dim != cache.head_dim:
        raise ValueError(f"{what}: the cache has {cache.n_kv_heads} heads of {cache.head_dim}, "
                         f"the layer {cfg.n_kv_heads} of {cfg.head_dim}")
    return (ctypes.byref(cfg), cache._ref, ctypes.byref(batch.struct()),
            _on_gpu(what, stream, cache.k, batch.slot, *tensors))


def kv8_append(cfg, cache: KV8Cache, batch, k_new, v_new, stream=None) -> None:
    """The batch's new keys (rotated) and values [tokens, Hkv, D] (bf16, tokens any one
    stride apart) into the 8-bit cache (tri_kv8_append)."""
    import torch
    d = cfg.head_dim
    stride = _rows(k_new, "kv8_append: k_new", d)
    n, heads, _ = k_new.shape
    if n != batch.n_tokens or heads != cfg.n_kv_heads or v_new.shape != k_new.shape or \
            _rows(v_new, "kv8_append: v_new", d) != stride:
        raise ValueError(f"kv8_append: k_new and v_new are [{batch.n_tokens}, {cfg.n_kv_heads}, {d}] "
                         "with one token stride")
    if k_new.dtype != torch.bfloat16 or v_new.dtype != torch.bfloat16:
        raise ValueError("kv8_append: k_new and v_new are bf16")
    c, kv, b, stream = _kv8("kv8_append", cfg, cache, batch, stream, k_new, v_new)
    st = lib().tri_kv8_append(c, kv, b, k_new.data_ptr(), v_new.data_ptr(), stride, stream)
    if st:
        raise TriError(st, "tri_kv8_append")


def kv8_attention_workspace_size(cfg, cache: KV8Cache, batch) -> int:
    n = ctypes.c_size_t()
    _check(lib().tri_kv8_attention_workspace_size(
        ctypes.byref(cfg), cache._ref, ctypes.byref(batch.struct()), ctypes.byref(n)),
        "tri_kv8_attention_workspace_size")
    return n.value


def kv8_attention(cfg, cache: KV8Cache, batch, q, out=None, workspace=None, stream=None):
    """Causal attention of q [tokens, Hq, D] (bf16, tokens any stride apart) over the 8-bit
    cache, adding up cache.mass where it has one (tri_kv8_attention); returns (out, workspace)."""
    import torch
    stride = _rows(q, "kv8_attention: q", cfg.head_dim)
    n, heads, _ = q.shape
    if n != batch.n_tokens or heads != cfg.n_q_heads or q.dtype != torch.bfloat16:
        raise ValueError(f"kv8_attention: q is bf16 [{batch.n_tokens}, {cfg.n_q_heads}, {cfg.head_dim}]")
    if out is None:
        out = _empty(stream, q.shape, q.dtype, q.device)
    if out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise ValueError(f"kv8_attention: out is contiguous bf16 {tuple(q.shape)}")
    if workspace is None:
        workspace = _empty(stream, kv8_attention_workspace_size(cfg, cache, batch), torch.uint8, q.device)
    c, kv, b, stream = _kv8("kv8_attention", cfg, cache, batch, stream, q, out, workspace)
    st = lib().tri_kv8_attention(c, kv, b, q.data_ptr(), stride, out.data_ptr(), workspace.data_ptr(),
                                 workspace.nbytes, stream)
    if st:
        raise TriError(st, "tri_kv8_attention")
    return out, workspace


def kv8_select_workspace_size(cfg, cache: KV8Cache, batch, budget: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().tri_kv8_select_workspace_size(
        ctypes.byref(cfg), cache._ref, ctypes.byref(batch.struct()), int(budget), ctypes.byref(n)),
        "tri_kv8_select_workspace_size")
    return n.value


def _plan(what, plan, n_seqs: int, heads: int, budget: int) -> None:
    import torch
    if plan.dtype != torch.int32 or plan.shape != (n_seqs, heads, budget) or not plan.is_contiguous():
        raise ValueError(f"{what}: plan is a contiguous int32 {(n_seqs, heads, budget)}")


def kv8_select(cfg, cache: KV8Cache, batch, budget: int, n_first: int = 0, n_recent: int = 0,
               plan=None, new_len=None, workspace=None, stream=None):
    """Which rows of the batch's sequences (ctx_len + q_len each) stay within budget
    (tri_kv8_select); returns (plan [n_seqs, Hkv, budget], new_len [n_seqs]), int32."""
    import torch
    n = batch.n_seqs
    if plan is None:
        plan = _empty(stream, (n, cfg.n_kv_heads, budget), torch.int32, cache.k.device)
    if new_len is None:
        new_len = _empty(stream, n, torch.int32, cache.k.device)
    _plan("kv8_select", plan, n, cfg.n_kv_heads, budget)
    if new_len.dtype != torch.int32 or new_len.numel() != n or not new_len.is_contiguous():
        raise ValueError(f"kv8_select: new_len is a contiguous int32 [{n}]")
    if workspace is None and batch.max_ctx_len + batch.max_q_len > 16384:  # (else none is needed)
        workspace = _empty(stream, kv8_select_workspace_size(cfg, cache, batch, budget), torch.uint8,
                           plan.device)
    c, kv, b, stream = _kv8("kv8_select", cfg, cache, batch, stream, plan, new_len, workspace)
    st = lib().tri_kv8_select(c, kv, b, budget, n_first, n_recent, plan.data_ptr(),
                              new_len.data_ptr(), _ptr(workspace),
                              0 if workspace is None else workspace.nbytes, stream)
    if st:
        raise TriError(st, "tri_kv8_select")
    return plan, new_len


def kv8_move(cfg, cache: KV8Cache, batch, plan, stream=None) -> None:
    """Rows of the batch's sequences to the places of a kv8_select plan (tri_kv8_move)."""
    budget = plan.shape[-1] if plan.dim() else 0
    _plan("kv8_move", plan, batch.n_seqs, cfg.n_kv_heads, budget)
    c, kv, b, stream = _kv8("kv8_move", cfg, cache, batch, stream, plan)
    st = lib().tri_kv8_move(c, kv, b, plan.data_ptr(), budget, stream)
    if st:
        raise TriError(st, "tri_kv8_move")


def moe_route(cfg, h2_f32, w_router, idx, w, stream=None) -> None:
    _check(lib().tri_moe_route(ctypes.byref(cfg), _ptr(h2_f32), _ptr(w_router),
                               int(h2_f32.shape[0]), _ptr(idx), _ptr(w), _stream(stream)),
           "tri_moe_route")


def profile_enable(on: bool = True) -> None:
    """Start (and reset) or stop per-stage HIP-event timing inside the library."""
    _check(lib().tri_profile_enable(1 if on else 0), "tri_profile_enable")


def profile_read(raw: bool = False):
    """Per-stage launches and total milliseconds recorded since profile_enable(True)
    (the Profile struct itself if raw)."""
    p = Profile()
    _check(lib().tri_profile_read(ctypes.byref(p)), "tri_profile_read")
    if raw:
        return p
    return {p.name[i].decode(): {"launches": p.launches[i], "total_ms": p.total_ms[i]}
            for i in range(p.n_stages)}


def _i32_array(v) -> ctypes.Array:
    v = [int(a) for a in v]
    return (ctypes.c_int32 * max(len(v), 1))(*v)


def layer_work(cfg: LayerConfig, decode: bool, q_len: Sequence[int], ctx_len: Sequence[int],
               expert_rows: Optional[Sequence[int]] = None) -> Work:
    """Algorithmic flops and HBM bytes per stage of one layer call (tri_layer_work)."""
    if len(q_len) != len(ctx_len):
        raise ValueError("q_len and ctx_len differ in length")
    w = Work()
    er = None if expert_rows is None else _i32_array(expert_rows)
    _check(lib().tri_layer_work(ctypes.byref(cfg), 1 if decode else 0, len(q_len),
                                _i32_array(q_len), _i32_array(ctx_len), er, ctypes.byref(w)),
           "tri_layer_work")
    return w


def work_sum(works: Sequence[Work]) -> Work:
    """Stage-by-stage sum of the work of several calls."""
    out = Work()
    out.n_stages = works[0].n_stages
    for i in range(16):
        out.name[i] = works[0].name[i]
        out.runs[i] = int(any(w.runs[i] for w in works))
        out.flops[i] = sum(w.flops[i] for w in works)
        out.bytes[i] = sum(w.bytes[i] for w in works)
    return out


def work_dict(w: Work) -> Dict[str, Dict[str, float]]:
    return {w.name[i].decode(): {"flops": w.flops[i], "bytes": w.bytes[i]}
            for i in range(w.n_stages) if w.runs[i]}


def phase_intensity(work: Work, prof: Profile) -> float:
    """Time-weighted arithmetic intensity of a phase (tri_phase_intensity, Eq. 5)."""
    ai = ctypes.c_double()
    _check(lib().tri_phase_intensity(ctypes.byref(work), ctypes.byref(prof), ctypes.byref(ai)),
           "tri_phase_intensity")
    return ai.value
