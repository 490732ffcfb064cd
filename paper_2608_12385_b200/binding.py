"""Thin ctypes binding over the C ABI of include/dbt.h (argument marshalling only).

PyTorch supplies device memory and the CUDA stream; every step of the path runs inside
libdbt_b200.so.  Loading fails loudly when the library has not been built
(`python -m paper_2608_12385_b200.build`): there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import os
import struct

import torch

from .inputs import ModelConfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdbt_b200.so")

DBT_OK = 0
STATUS_NAMES = {0: "DBT_OK", 1: "DBT_ERR_INVALID_ARG", 2: "DBT_ERR_UNSUPPORTED", 3: "DBT_ERR_CAPACITY",
                4: "DBT_ERR_STATE", 5: "DBT_ERR_CUDA", 6: "DBT_ERR_DEVICE", 7: "DBT_ERR_TIMEOUT"}

EXPORTS = ["dbt_query_sizes", "dbt_create", "dbt_destroy", "dbt_set_page_table", "dbt_reset", "dbt_set_seq_lens",
           "dbt_seq_len", "dbt_prefill", "dbt_decode_step", "dbt_decode_step_primary_only", "dbt_decode_step_host",
           "dbt_decode_step_primary_only_host", "dbt_last_experts", "dbt_last_expert_union", "dbt_sync_status",
           "dbt_launch_count", "dbt_last_error", "dbt_version", "dbt_profile_begin", "dbt_profile_end", "dbt_op_gemm_tc",
           "dbt_op_gemm_tc_static", "dbt_kv_export", "dbt_kv_import", "dbt_prefill_boundary", "dbt_rope_frequencies",
           "dbt_op_rope", "dbt_op_rope_append", "dbt_op_attn_tree_workspace", "dbt_op_attn_tree", "dbt_op_sample",
           "dbt_op_tree_accept", "dbt_sample_last"]


class DbtError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class DbtConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)]
    _fields_ += [(n, C.c_int32) for n in ("d_model", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "d_ff",
                                         "vocab", "weight_dtype")]
    _fields_ += [("rope_base", C.c_float), ("rms_eps", C.c_float)]
    _fields_ += [(n, C.c_int32) for n in ("final_norm", "n_experts", "d_expert", "n_shared_experts", "k_primary",
                                         "k_branch", "router_mode", "moe_b_coupling", "compute_matched", "n_paths", "max_batch", "max_seq",
                                         "page_size", "num_pages")]


LAYER_FIELDS = ("attn_norm_g", "wq", "wk", "wv", "wo", "coup_a", "mlp_norm_g", "w_gate", "w_up", "w_down", "coup_b",
                "coup_c", "router", "exp_gate", "exp_up", "exp_down", "sh_gate", "sh_up", "sh_down", "gate_a", "gate_g")


class DbtLayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LAYER_FIELDS]


class DbtProfileEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("launches", C.c_int64), ("total_ms", C.c_double), ("bytes", C.c_double)]


class DbtWeights(C.Structure):
    _fields_ = [("embed_primary", C.c_void_p), ("embed_branch", C.c_void_p), ("embed_norm_g", C.c_void_p),
                ("final_norm_g", C.c_void_p), ("lm_head", C.c_void_p), ("layers", C.POINTER(DbtLayerWeights))]


_lib = None


def load_library():
    """dlopen libdbt_b200.so and declare the signatures.  Raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_12385_b200.build` "
                           "(there is no CPU or PyTorch fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i32p = C.c_void_p, C.c_int32, C.POINTER(C.c_int32)
    L.dbt_query_sizes.argtypes = [C.POINTER(DbtConfig), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    L.dbt_create.argtypes = [C.POINTER(DbtConfig), C.POINTER(DbtWeights), vp, vp, vp, C.POINTER(vp)]
    L.dbt_destroy.argtypes = [vp]
    L.dbt_destroy.restype = None
    L.dbt_set_page_table.argtypes = [vp, vp, i32, i32]
    L.dbt_reset.argtypes = [vp]
    L.dbt_set_seq_lens.argtypes = [vp, vp, i32]
    L.dbt_seq_len.argtypes = [vp, i32]
    L.dbt_seq_len.restype = i32
    L.dbt_prefill.argtypes = [vp, vp, i32, i32, vp]
    L.dbt_decode_step.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    L.dbt_prefill_boundary.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp]
    L.dbt_decode_step_primary_only.argtypes = [vp, vp, i32, vp, vp]
    L.dbt_decode_step_host.argtypes = [vp, vp, i32, vp, vp]
    L.dbt_decode_step_primary_only_host.argtypes = [vp, vp, i32, vp]
    L.dbt_last_experts.argtypes = [vp, C.POINTER(vp), i32p]
    L.dbt_last_expert_union.argtypes = [vp, vp]
    L.dbt_sync_status.argtypes = [vp, i32p, i32p]
    L.dbt_kv_export.argtypes = [vp, vp, i32, i32, vp, vp]
    L.dbt_kv_import.argtypes = [vp, vp, i32, i32, vp, vp]
    L.dbt_op_gemm_tc.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, C.c_size_t, vp, vp, i32p]
    L.dbt_op_gemm_tc_static.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, i32p]
    L.dbt_rope_frequencies.argtypes = [vp, vp, vp]
    L.dbt_op_rope.argtypes = [vp, vp, vp, vp, C.c_int64, i32, i32, i32, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_float, i32,
                              i32, i32, vp]
    L.dbt_op_rope_append.argtypes = [vp, vp]
    L.dbt_op_attn_tree_workspace.argtypes = [vp, C.POINTER(C.c_size_t)]
    L.dbt_op_attn_tree.argtypes = [vp, vp]
    L.dbt_op_sample.argtypes = [vp, i32, i32, i32, C.c_int64, vp, vp, vp, vp, vp, vp, vp, vp]
    L.dbt_op_tree_accept.argtypes = [vp, vp]
    L.dbt_sample_last.argtypes = [vp, vp, i32, vp, vp]
    L.dbt_profile_begin.argtypes = [vp]
    L.dbt_profile_end.argtypes = [vp, C.POINTER(DbtProfileEntry), i32, i32p]
    L.dbt_launch_count.argtypes = [vp]
    L.dbt_launch_count.restype = C.c_int64
    L.dbt_last_error.argtypes = [vp]
    L.dbt_last_error.restype = C.c_char_p
    L.dbt_version.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("dbt_destroy", "dbt_seq_len", "dbt_launch_count", "dbt_last_error", "dbt_version"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def make_config_struct(cfg: ModelConfig, max_batch: int, max_seq: int, num_pages: int) -> DbtConfig:
    return DbtConfig(struct_size=C.sizeof(DbtConfig), d_model=cfg.d_model, n_layers=cfg.n_layers,
                     n_q_heads=cfg.n_q_heads, n_kv_heads=cfg.n_kv_heads, head_dim=cfg.head_dim, d_ff=cfg.d_ff,
                     vocab=cfg.vocab, weight_dtype=0 if cfg.weight_dtype == "fp32" else 1, rope_base=cfg.rope_base,
                     rms_eps=cfg.rms_eps, final_norm=cfg.final_norm, n_experts=cfg.n_experts, d_expert=cfg.d_expert,
                     n_shared_experts=cfg.n_shared_experts, k_primary=cfg.k_primary, k_branch=cfg.k_branch,
                     router_mode=cfg.router_mode, moe_b_coupling=cfg.moe_b_coupling,
                     compute_matched=cfg.compute_matched, n_paths=cfg.n_paths, max_batch=max_batch,
                     max_seq=max_seq, page_size=cfg.page_size, num_pages=num_pages)


def query_sizes(cfg: ModelConfig, max_batch: int, max_seq: int, num_pages: int) -> tuple[int, int]:
    L = load_library()
    c = make_config_struct(cfg, max_batch, max_seq, num_pages)
    kv, ws = C.c_size_t(0), C.c_size_t(0)
    st = L.dbt_query_sizes(C.byref(c), C.byref(kv), C.byref(ws))
    if st != DBT_OK:
        raise DbtError(st, L.dbt_last_error(None).decode())
    return kv.value, ws.value


def op_gemm_tc(W: torch.Tensor, X: torch.Tensor, force_split: int = 0, scratch: torch.Tensor | None = None):
    """Y = X W^T on the tensor cores.  W bf16 [n_out, K], X bf16 [R, K] on the GPU.
    Returns (Y fp32 [R, n_out], split used)."""
    L = load_library()
    assert W.dtype == torch.bfloat16 and X.dtype == torch.bfloat16 and W.is_cuda and X.is_cuda
    n_out, K = W.shape
    R = X.shape[0]
    Y = torch.empty(R, n_out, dtype=torch.float32, device=W.device)
    if scratch is None:
        scratch = torch.empty(max(force_split, 16) * 256 * n_out if R > 128 else max(force_split, 16) * 128 * n_out,
                              dtype=torch.float32, device=W.device)
    status = torch.zeros(2, dtype=torch.int32, device=W.device)
    used = C.c_int32(0)
    st = L.dbt_op_gemm_tc(W.data_ptr(), X.data_ptr(), n_out, K, R, force_split, Y.data_ptr(), scratch.data_ptr(),
                          scratch.numel(), status.data_ptr(), torch.cuda.current_stream().cuda_stream, C.byref(used))
    if st != DBT_OK:
        raise DbtError(st, L.dbt_last_error(None).decode())
    torch.cuda.synchronize()
    code = status.cpu().tolist()
    if code[0] != 0:  # 3: a bounded device wait ran out (the codes of dbt_sync_status)
        raise DbtError(7 if code[0] == 3 else 6, f"device status {code}")
    return Y, used.value


def op_gemm_tc_static(W: torch.Tensor, X: torch.Tensor, force_split: int = 0, Y: torch.Tensor | None = None,
                      status: torch.Tensor | None = None):
    """Y = X W^T through the entry point that allocates no device memory: its split-K workspace
    is a fixed 8 MiB array inside the library.  Pass Y and status to make the call itself
    allocation-free on the Python side too.  Returns (Y, split used)."""
    L = load_library()
    assert W.dtype == torch.bfloat16 and X.dtype == torch.bfloat16 and W.is_cuda and X.is_cuda
    n_out, K = W.shape
    R = X.shape[0]
    if Y is None:
        Y = torch.empty(R, n_out, dtype=torch.float32, device=W.device)
    if status is None:
        status = torch.zeros(2, dtype=torch.int32, device=W.device)
    used = C.c_int32(0)
    st = L.dbt_op_gemm_tc_static(W.data_ptr(), X.data_ptr(), n_out, K, R, force_split, Y.data_ptr(), status.data_ptr(),
                                 torch.cuda.current_stream().cuda_stream, C.byref(used))
    if st != DBT_OK:
        raise DbtError(st, L.dbt_last_error(None).decode())
    torch.cuda.synchronize()
    code = status.cpu().tolist()
    if code[0] != 0:  # 3: a bounded device wait ran out (the codes of dbt_sync_status)
        raise DbtError(7 if code[0] == 3 else 6, f"device status {code}")
    return Y, used.value


# ---- operators for sampled and drafted tokens -----------------------------------------------------------------------
# The argument structures of include/dbt.h as `struct` formats (native alignment): packing one costs a microsecond, filling a
# ctypes structure several.
ROPE_SPEC_FORMAT = struct.Struct("@I3i5d")
ROPE_APPEND_FORMAT = struct.Struct("@I10if3P9q2P4PPP")
ATTN_TREE_FORMAT = struct.Struct("@I8if2P3qP4PPNP")
TREE_ACCEPT_FORMAT = struct.Struct("@I8i6PP4PP")
SAMPLING_FORMAT = struct.Struct("@Ii5P")
ROPE_KINDS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


_I32, _F32, _F64 = torch.int32, torch.float32, torch.float64
_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _need(cond, message: str):
    if not cond:
        raise DbtError(1, message)


# The checks stand in one condition each and call _refuse for the message: a call costs a microsecond per tensor otherwise.
def _refuse(**tensors):
    """Say which of name = (tensor, dtype, shape) is not a contiguous tensor of that type and shape (None passes)."""
    for name, (t, dtype, shape) in tensors.items():
        if t is not None and not (t.dtype is dtype and t.shape == shape and t.is_contiguous()):
            raise DbtError(1, f"{name}: contiguous {dtype} {tuple(shape)} expected, got {t.dtype} {tuple(t.shape)}")


def _dtype(t: torch.Tensor) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise DbtError(1, f"float32 or bfloat16 expected, got {t.dtype}")
    return dt


def _stream(dev: int, tensors) -> int:
    """The current stream of the device that all tensors are on."""
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise DbtError(1, "all tensors have to be on one GPU")
    if dev < 0:
        raise DbtError(1, "the tensors have to be on a GPU")
    return _current_stream(dev)


def _call(fn, dev: int, *args):
    """Call an entry with `dev` as the current device."""
    if dev == _current_device():
        st = fn(*args)
    else:
        with torch.cuda.device(dev):
            st = fn(*args)
    if st != DBT_OK:
        raise DbtError(st, load_library().dbt_last_error(None).decode())


def check_status(status: torch.Tensor):
    """Wait for a status word that operators were given, and raise what they recorded in it."""
    code = status.cpu().tolist()
    if code[0] != 0:
        raise DbtError(7 if code[0] == 3 else 6, f"device status {code}")


def _own_status(like: torch.Tensor) -> torch.Tensor:
    return torch.zeros(2, dtype=torch.int32, device=like.device)


def rope_frequencies(rot_dim: int, base: float = 10000.0, kind: str = "plain", factor: float = 1.0, trained_len: float = 0.0,
                     low: float = 1.0, high: float = 32.0) -> tuple[torch.Tensor, float]:
    """(angle per position of each of the rot_dim / 2 pairs, float64 on the CPU; factor on queries and keys) for
    contexts as trained ("plain") or longer: "linear", "base", "ramp", "bands" as include/dbt.h defines them."""
    L = load_library()
    _need(kind in ROPE_KINDS, f"kind: one of {sorted(ROPE_KINDS)}")
    freq = torch.empty(max(rot_dim // 2, 1), dtype=torch.float64)
    scale = C.c_float(1.0)
    spec = ROPE_SPEC_FORMAT.pack(ROPE_SPEC_FORMAT.size, ROPE_KINDS[kind], rot_dim, 0, base, factor, trained_len, low, high)
    st = L.dbt_rope_frequencies(spec, freq.data_ptr(), C.addressof(scale))
    if st != DBT_OK:
        raise DbtError(st, L.dbt_last_error(None).decode())
    return freq, scale.value


def op_rope(x: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, scale: float = 1.0, interleaved: bool = False,
            inverse: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [rows, heads, head_dim] with the first 2 * freq.numel() elements of every head rotated by positions [rows] (int32)
    times freq (float64, on x's device).  inverse: the transposed map, which is the gradient.  out may be x."""
    L = _lib or load_library()
    dt = _dtype(x)
    _need(x.dim() == 3, "x: [rows, heads, head_dim] expected")
    rows, heads, dim = x.shape
    xs = x.stride()
    if out is None:
        out = torch.empty((rows, heads, dim), dtype=x.dtype, device=x.device)
    ys = out.stride()
    if not (xs[2] == 1 and out.dtype is x.dtype and out.shape == x.shape and ys[2] == 1):
        raise DbtError(1, "x, out: the same shape and type with contiguous head_dim expected")
    if not (positions.dtype is _I32 and positions.shape == (rows,) and positions.is_contiguous() and freq.dtype is _F64 and freq.dim() == 1
            and freq.is_contiguous()):
        _refuse(positions=(positions, _I32, (rows,)), freq=(freq, _F64, (freq.numel(),)))
    dev = x.get_device()
    _call(L.dbt_op_rope, dev, x.data_ptr(), out.data_ptr(), positions.data_ptr(), freq.data_ptr(), rows, heads, dim, 2 * freq.numel(), xs[0], xs[1],
          ys[0], ys[1], scale, interleaved, inverse, dt, _stream(dev, (out, positions, freq)))
    return out


def _cache_shape(cache: torch.Tensor, dims: int, dtype):
    shape = cache.shape
    if not (len(shape) == dims and shape[-5] == 2 and shape[-2] == 16 and cache.dtype is dtype and cache.is_contiguous()):
        raise DbtError(1, "cache: contiguous [.., 2, pages, kv heads, 16, head_dim] of the activations' type expected")
    return shape[-4], shape[-3], shape[-1]


def op_rope_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, cache_layer: torch.Tensor,
                   page_table: torch.Tensor, seq_lens: torch.Tensor, counts: torch.Tensor | None = None, scale: float = 1.0,
                   interleaved: bool = False, out: torch.Tensor | None = None, status: torch.Tensor | None = None) -> torch.Tensor:
    """q [B, N, query heads, head_dim], k, v [B, N, kv heads, head_dim] (any strides but the last) of N nodes per sequence: q and k
    rotated by positions [B, N]; the keys and values go to cache positions seq_lens[b] + node of cache_layer [2, pages, kv heads, 16,
    head_dim], the rotated queries are returned.  counts [B]: nodes that count; rows behind them are left as they were.  With a status
    word of the caller's (int32 [2], zeros; see check_status) the call does not wait; without one it waits and raises what the device
    found."""
    L = _lib or load_library()
    dt, dtype = _dtype(q), q.dtype
    pages, nkv, dim = _cache_shape(cache_layer, 5, dtype)
    _need(q.dim() == 4 and page_table.dim() == 2, "q: [B, nodes, heads, head_dim], page_table: [B, pages per sequence] expected")
    B, N, nq, qd = q.shape
    pps = page_table.shape[1]
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    if not (qd == dim and qs[3] == 1 and k.shape == (B, N, nkv, dim) and k.dtype is dtype and ks[3] == 1 and v.shape == (B, N, nkv, dim)
            and v.dtype is dtype and vs[3] == 1):
        raise DbtError(1, "q, k, v: [B, nodes, heads, head_dim] of the cache's type, head_dim and number of heads, with contiguous head_dim expected")
    if out is None:
        out = torch.empty((B, N, nq, dim), dtype=dtype, device=q.device)
    own = status is None
    if own:
        status = _own_status(q)
    if not (out.shape == q.shape and out.dtype is dtype and out.is_contiguous() and positions.dtype is _I32 and positions.shape == (B, N)
            and positions.is_contiguous() and page_table.dtype is _I32 and page_table.shape[0] == B and page_table.is_contiguous()
            and seq_lens.dtype is _I32 and seq_lens.shape == (B,) and seq_lens.is_contiguous() and freq.dtype is _F64 and freq.dim() == 1
            and freq.is_contiguous() and status.dtype is _I32 and status.shape == (2,) and status.is_contiguous()
            and (counts is None or (counts.dtype is _I32 and counts.shape == (B,) and counts.is_contiguous()))):
        _refuse(out=(out, dtype, q.shape), positions=(positions, _I32, (B, N)), page_table=(page_table, _I32, (B, pps)), seq_lens=(seq_lens, _I32, (B,)),
                counts=(counts, _I32, (B,)), freq=(freq, _F64, (freq.numel(),)), status=(status, _I32, (2,)))
    dev = q.get_device()
    stream = _stream(dev, (k, v, out, cache_layer, positions, page_table, seq_lens, counts, freq, status))
    _call(L.dbt_op_rope_append, dev, ROPE_APPEND_FORMAT.pack(
        ROPE_APPEND_FORMAT.size, dt, B, N, nq, nkv, dim, 2 * freq.numel(), interleaved, pages, pps, scale, q.data_ptr(), k.data_ptr(), v.data_ptr(),
        qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], out.data_ptr(), cache_layer.data_ptr(), positions.data_ptr(),
        page_table.data_ptr(), seq_lens.data_ptr(), 0 if counts is None else counts.data_ptr(), freq.data_ptr(), status.data_ptr()), stream)
    if own:
        check_status(status)
    return out


def op_attn_tree(q: torch.Tensor, cache_layer: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor, parents: torch.Tensor,
                 counts: torch.Tensor | None = None, softmax_scale: float = 0.0, out: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None, status: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of the N drafted nodes of every sequence: q [B, N, query heads, head_dim]; node i sees the seq_lens[b] cached positions,
    itself and its ancestors by parents [B, N] (-1: a root), whose keys and values stand in the cache behind them.  workspace (uint8, at
    least attn_tree_workspace(...) bytes) is allocated when none is given.  status as in op_rope_append."""
    L = _lib or load_library()
    dt, dtype = _dtype(q), q.dtype
    pages, nkv, dim = _cache_shape(cache_layer, 5, dtype)
    _need(q.dim() == 4 and page_table.dim() == 2, "q: [B, nodes, heads, head_dim], page_table: [B, pages per sequence] expected")
    B, N, nq, qd = q.shape
    pps = page_table.shape[1]
    qs = q.stride()
    if qd != dim or qs[3] != 1:
        raise DbtError(1, "q: [B, nodes, heads, head_dim] of the cache's head_dim, contiguous in it, expected")
    dev = q.get_device()
    if out is None:
        out = torch.empty((B, N, nq, dim), dtype=dtype, device=q.device)
    own = status is None
    if own:
        status = _own_status(q)
    if workspace is None:
        workspace = torch.empty(_tree_workspace(dt, B, N, nq, nkv, dim, pages, pps, dev), dtype=torch.uint8, device=q.device)
    if not (out.shape == q.shape and out.dtype is dtype and out.is_contiguous() and page_table.dtype is _I32 and page_table.shape[0] == B
            and page_table.is_contiguous() and seq_lens.dtype is _I32 and seq_lens.shape == (B,) and seq_lens.is_contiguous()
            and parents.dtype is _I32 and parents.shape == (B, N) and parents.is_contiguous() and status.dtype is _I32 and status.shape == (2,) and status.is_contiguous()
            and workspace.is_contiguous() and (counts is None or (counts.dtype is _I32 and counts.shape == (B,) and counts.is_contiguous()))):
        _refuse(out=(out, dtype, q.shape), page_table=(page_table, _I32, (B, pps)), seq_lens=(seq_lens, _I32, (B,)), parents=(parents, _I32, (B, N)),
                counts=(counts, _I32, (B,)), status=(status, _I32, (2,)), workspace=(workspace, workspace.dtype, workspace.shape))
    stream = _stream(dev, (out, cache_layer, page_table, seq_lens, parents, counts, workspace, status))
    _call(L.dbt_op_attn_tree, dev, ATTN_TREE_FORMAT.pack(
        ATTN_TREE_FORMAT.size, dt, B, N, nq, nkv, dim, pages, pps, softmax_scale, q.data_ptr(), cache_layer.data_ptr(), qs[0], qs[1], qs[2],
        out.data_ptr(), page_table.data_ptr(), seq_lens.data_ptr(), 0 if counts is None else counts.data_ptr(), parents.data_ptr(),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), status.data_ptr()), stream)
    if own:
        check_status(status)
    return out


@functools.lru_cache(maxsize=256)
def _tree_workspace(dt: int, B: int, N: int, nq: int, nkv: int, dim: int, pages: int, pps: int, dev: int) -> int:
    """The size that the library asks for: a function of these numbers and of the device's SMs alone."""
    L = load_library()
    n = C.c_size_t(0)
    args = ATTN_TREE_FORMAT.pack(ATTN_TREE_FORMAT.size, dt, B, N, nq, nkv, dim, pages, pps, 0.0, *[0] * 13)
    with torch.cuda.device(dev) if dev >= 0 else contextlib.nullcontext():
        st = L.dbt_op_attn_tree_workspace(args, C.byref(n))
    if st != DBT_OK:
        raise DbtError(st, L.dbt_last_error(None).decode())
    return n.value


def attn_tree_workspace(q: torch.Tensor, cache_layer: torch.Tensor, page_table: torch.Tensor) -> int:
    """Bytes of workspace that op_attn_tree needs for tensors of these shapes."""
    B, N, nq, dim = q.shape
    return _tree_workspace(_dtype(q), B, N, nq, cache_layer.shape[2], dim, cache_layer.shape[1], page_table.shape[1], q.get_device())


def op_sample(logits: torch.Tensor, uniforms: torch.Tensor, temperature: torch.Tensor | None = None, top_k: torch.Tensor | None = None,
              top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """A token per row of logits [rows, vocab] from one number in [0, 1) a row (uniforms fp32 [rows]); temperature, top_p, min_p fp32 [rows]
    and top_k int32 [rows], each optional.  Returns (tokens int32 [rows], log of each token's share of what the filters leave)."""
    L = _lib or load_library()
    dt = _dtype(logits)
    _need(logits.dim() == 2, "logits: [rows, vocab] expected")
    R, V = logits.shape
    zs = logits.stride()
    one = (R,)
    if not (zs[1] == 1 and uniforms.dtype is _F32 and uniforms.shape == one and uniforms.is_contiguous()
            and (temperature is None or (temperature.dtype is _F32 and temperature.shape == one and temperature.is_contiguous()))
            and (top_k is None or (top_k.dtype is _I32 and top_k.shape == one and top_k.is_contiguous()))
            and (top_p is None or (top_p.dtype is _F32 and top_p.shape == one and top_p.is_contiguous()))
            and (min_p is None or (min_p.dtype is _F32 and min_p.shape == one and min_p.is_contiguous()))):
        _need(zs[1] == 1, "logits: contiguous rows expected")
        _refuse(uniforms=(uniforms, _F32, one), temperature=(temperature, _F32, one), top_k=(top_k, _I32, one), top_p=(top_p, _F32, one),
                min_p=(min_p, _F32, one))
    dev = logits.get_device()
    stream = _stream(dev, (uniforms, temperature, top_k, top_p, min_p))
    device = logits.device
    tokens, logprobs = torch.empty(R, dtype=_I32, device=device), torch.empty(R, dtype=_F32, device=device)
    _call(L.dbt_op_sample, dev, logits.data_ptr(), dt, R, V, zs[0] if R > 1 else V, uniforms.data_ptr(), _p(temperature), _p(top_k), _p(top_p), _p(min_p),
          tokens.data_ptr(), logprobs.data_ptr(), stream)
    return tokens, logprobs


def op_tree_accept(tokens: torch.Tensor, parents: torch.Tensor, sampled: torch.Tensor, pool: torch.Tensor, page_table: torch.Tensor,
                   seq_lens: torch.Tensor, counts: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """The walk from node 0 along the children whose token was sampled at their parent; the accepted nodes' rows of pool [layers, 2, pages,
    kv heads, 16, head_dim] are moved together behind the cached positions.  tokens, parents, sampled [B, N] int32.  Returns (path [B, N],
    accepted nodes [B], token sampled at the last of them [B], new lengths [B]), all int32.  status as in op_rope_append."""
    L = _lib or load_library()
    dt = _dtype(pool)
    pages, nkv, dim = _cache_shape(pool, 6, pool.dtype)
    _need(tokens.dim() == 2 and page_table.dim() == 2, "tokens: [B, nodes], page_table: [B, pages per sequence] expected")
    both = B, N = tokens.shape
    pps = page_table.shape[1]
    own = status is None
    if own:
        status = _own_status(tokens)
    if not (tokens.dtype is _I32 and tokens.is_contiguous() and parents.dtype is _I32 and parents.shape == both and parents.is_contiguous()
            and sampled.dtype is _I32 and sampled.shape == both and sampled.is_contiguous() and page_table.dtype is _I32
            and page_table.shape[0] == B and page_table.is_contiguous() and seq_lens.dtype is _I32 and seq_lens.shape == (B,)
            and seq_lens.is_contiguous() and status.dtype is _I32 and status.shape == (2,) and status.is_contiguous()
            and (counts is None or (counts.dtype is _I32 and counts.shape == (B,) and counts.is_contiguous()))):
        _refuse(tokens=(tokens, _I32, both), parents=(parents, _I32, both), sampled=(sampled, _I32, both), page_table=(page_table, _I32, (B, pps)),
                seq_lens=(seq_lens, _I32, (B,)), counts=(counts, _I32, (B,)), status=(status, _I32, (2,)))
    dev = tokens.get_device()
    stream = _stream(dev, (parents, sampled, pool, page_table, seq_lens, counts, status))
    device = tokens.device
    path = torch.empty(both, dtype=_I32, device=device)
    accepted, following, lens = torch.empty((3, B), dtype=_I32, device=device).unbind(0)
    first = accepted.data_ptr()
    _call(L.dbt_op_tree_accept, dev, TREE_ACCEPT_FORMAT.pack(
        TREE_ACCEPT_FORMAT.size, dt, B, N, pool.shape[0], nkv, dim, pages, pps, tokens.data_ptr(), parents.data_ptr(), sampled.data_ptr(),
        page_table.data_ptr(), seq_lens.data_ptr(), 0 if counts is None else counts.data_ptr(), pool.data_ptr(), path.data_ptr(), first,
        first + 4 * B, first + 8 * B, status.data_ptr()), stream)
    if own:
        check_status(status)
    return path, accepted, following, lens


def weights_to_device(weights: dict, device="cuda") -> dict:
    out = {k: v.to(device) for k, v in weights.items() if k != "layers"}
    out["layers"] = [{k: v.to(device) for k, v in lw.items()} for lw in weights["layers"]]
    return out


def _p(t):
    return None if t is None else t.data_ptr()


class Model:
    """A Decode-Branch model handle: owns (as torch tensors) the KV pool and the workspace
    the library borrows, and keeps the device weights alive.  Calls enqueue their work on `stream` (None: the default
    stream) and their results are written there; a caller on another stream waits for it before reading them."""

    def __init__(self, cfg: ModelConfig, weights_dev: dict, max_batch: int, max_seq: int,
                 num_pages: int | None = None, stream: torch.cuda.Stream | None = None):
        self.L = load_library()
        self.cfg, self.weights = cfg, weights_dev
        self.max_batch, self.max_seq = max_batch, max_seq
        self.pages_per_seq_max = (max_seq + cfg.page_size - 1) // cfg.page_size
        self.num_pages = num_pages if num_pages is not None else max_batch * self.pages_per_seq_max
        self.device = weights_dev["lm_head"].device
        self.stream = stream
        self._c = make_config_struct(cfg, max_batch, max_seq, self.num_pages)
        kv_bytes, ws_bytes = query_sizes(cfg, max_batch, max_seq, self.num_pages)
        self.kv_pool = torch.zeros(kv_bytes // cfg.elem_bytes, dtype=cfg.torch_dtype, device=self.device)
        self.workspace = torch.zeros(ws_bytes, dtype=torch.uint8, device=self.device)
        layers = (DbtLayerWeights * cfg.n_layers)()
        for l, lw in enumerate(weights_dev["layers"]):
            for name in LAYER_FIELDS:
                t = lw.get(name)
                if t is not None:
                    assert t.is_cuda and t.is_contiguous(), name
                setattr(layers[l], name, _p(t))
        self._layers = layers
        self._w = DbtWeights(embed_primary=_p(weights_dev["embed_primary"]), embed_branch=_p(weights_dev["embed_branch"]),
                             embed_norm_g=_p(weights_dev["embed_norm_g"]), final_norm_g=_p(weights_dev["final_norm_g"]),
                             lm_head=_p(weights_dev["lm_head"]), layers=layers)
        h = C.c_void_p(None)
        torch.cuda.synchronize(self.device)
        st = self.L.dbt_create(C.byref(self._c), C.byref(self._w), self.kv_pool.data_ptr(), self.workspace.data_ptr(),
                               stream.cuda_stream if stream is not None else None, C.byref(h))
        if st != DBT_OK:
            raise DbtError(st, self.L.dbt_last_error(None).decode())
        self._h = h
        self.page_table = self.default_page_table(max_batch)

    # -- plumbing -------------------------------------------------------------------------
    def _check(self, st: int):
        if st != DBT_OK:
            raise DbtError(st, self.L.dbt_last_error(self._h).decode())

    def _own_stream(self) -> torch.cuda.Stream:
        return self.stream if self.stream is not None else torch.cuda.default_stream(self.device)

    def _elsewhere(self) -> bool:
        """Whether the caller works on another stream than the model does."""
        return _current_stream(self.device.index) != (self.stream.cuda_stream if self.stream is not None else 0)

    def _empty(self, *shape, dtype) -> torch.Tensor:
        """Memory for a result that the library writes on the model's stream.  It comes from that stream's share of the allocator: from the
        current stream's, it could still be read by earlier work there, and be handed out again before the model's stream has written it."""
        if not self._elsewhere():
            return torch.empty(*shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self._own_stream()):
            t = torch.empty(*shape, dtype=dtype, device=self.device)
        t.record_stream(torch.cuda.current_stream(self.device))  # (the caller reads it there)
        return t

    def close(self):
        if getattr(self, "_h", None):
            torch.cuda.synchronize(self.device)
            self.L.dbt_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv_view(self) -> torch.Tensor:
        """The pool as [n_layers, 2, num_pages, n_kv_heads, page_size, head_dim]."""
        c = self.cfg
        return self.kv_pool.view(c.n_layers, 2, self.num_pages, c.n_kv_heads, c.page_size, c.head_dim)

    # -- state ----------------------------------------------------------------------------
    def reset(self):
        self._check(self.L.dbt_reset(self._h))

    def set_page_table(self, table: torch.Tensor):
        t = table.to(torch.int32).cpu().contiguous()
        self._check(self.L.dbt_set_page_table(self._h, t.data_ptr(), t.shape[0], t.shape[1]))
        self.page_table = t

    def set_seq_lens(self, lens):
        t = torch.as_tensor(lens, dtype=torch.int32).cpu().contiguous()
        self._check(self.L.dbt_set_seq_lens(self._h, t.data_ptr(), t.shape[0]))

    def seq_len(self, b: int) -> int:
        return self.L.dbt_seq_len(self._h, b)

    def default_page_table(self, batch: int) -> torch.Tensor:
        pps = min(self.pages_per_seq_max, self.num_pages // self.max_batch) \
            if self.max_batch * self.pages_per_seq_max > self.num_pages else self.pages_per_seq_max
        return (torch.arange(batch, dtype=torch.int32)[:, None] * pps + torch.arange(pps, dtype=torch.int32)[None, :])

    # -- the four calls of the problem statement -------------------------------------------
    def prefill(self, tokens_dev: torch.Tensor, want_logits: bool = False):
        assert tokens_dev.dtype == torch.int32 and tokens_dev.is_cuda and tokens_dev.is_contiguous()
        B, n = tokens_dev.shape
        out = self._empty(B, self.cfg.vocab, dtype=_F32) if want_logits else None
        self._check(self.L.dbt_prefill(self._h, tokens_dev.data_ptr(), B, n, _p(out)))
        return out

    def prefill_boundary(self, tokens_dev: torch.Tensor) -> dict:
        """The whole prompt [B, S] and the boundary evaluation at its last token (Section 4.4 items 1-2)."""
        assert tokens_dev.dtype == torch.int32 and tokens_dev.is_cuda and tokens_dev.is_contiguous()
        B, S = tokens_dev.shape
        V, K = self.cfg.vocab, self.cfg.n_paths
        out = {"next": self._empty(B, dtype=_I32), "z1": self._empty(B, V, dtype=_F32),
               "z2": self._empty(*((B, V) if K == 2 else (K - 1, B, V)), dtype=_F32), "alpha": self._empty(B, dtype=_F32)}
        self._check(self.L.dbt_prefill_boundary(self._h, tokens_dev.data_ptr(), B, S, _p(out["next"]), _p(out["z1"]),
                                                _p(out["z2"]), _p(out["alpha"])))
        return out

    def decode_step(self, tokens_dev: torch.Tensor, next_dev: torch.Tensor | None = None, z1=None, z2=None,
                    alpha=None):
        B = tokens_dev.shape[0]
        self._check(self.L.dbt_decode_step(self._h, tokens_dev.data_ptr(), B, _p(next_dev), _p(z1), _p(z2), _p(alpha)))

    def decode_step_primary_only(self, tokens_dev: torch.Tensor, next_dev: torch.Tensor | None = None, z1=None):
        B = tokens_dev.shape[0]
        self._check(self.L.dbt_decode_step_primary_only(self._h, tokens_dev.data_ptr(), B, _p(next_dev), _p(z1)))

    def sample_last(self, uniforms: torch.Tensor, temperature: torch.Tensor | None = None, top_k: torch.Tensor | None = None,
                    top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None, next_dev: torch.Tensor | None = None):
        """Tokens of the last step (any of the step calls, or prefill_boundary) drawn from its mixture by the rules of op_sample instead of
        picked: (tokens int32 [B], log of each token's share).  The tensors have to be ready on the model's stream, and the results are
        written there: another stream waits for it before it reads them."""
        B = uniforms.shape[0]
        given = (uniforms, temperature, top_k, top_p, min_p, next_dev)
        _refuse(uniforms=(uniforms, _F32, (B,)), temperature=(temperature, _F32, (B,)), top_k=(top_k, _I32, (B,)), top_p=(top_p, _F32, (B,)),
                min_p=(min_p, _F32, (B,)), next_dev=(next_dev, _I32, (B,)))
        _stream(self.device.index, given)
        if next_dev is None:
            next_dev = self._empty(B, dtype=_I32)
        logprobs = self._empty(B, dtype=_F32)
        if self._elsewhere():
            for t in given:
                if t is not None:  # the caller may drop it before the model's stream has read or written it
                    t.record_stream(self._own_stream())
        self._check(self.L.dbt_sample_last(self._h, SAMPLING_FORMAT.pack(SAMPLING_FORMAT.size, 0, uniforms.data_ptr(), _p(temperature) or 0, _p(top_k) or 0,
                                                                         _p(top_p) or 0, _p(min_p) or 0), B, next_dev.data_ptr(), logprobs.data_ptr()))
        return next_dev, logprobs

    def decode_step_host(self, tokens_host: torch.Tensor, next_host: torch.Tensor, alpha_host=None):
        self._check(self.L.dbt_decode_step_host(self._h, tokens_host.data_ptr(), tokens_host.shape[0],
                                                next_host.data_ptr(), _p(alpha_host)))

    def decode_step_primary_only_host(self, tokens_host: torch.Tensor, next_host: torch.Tensor):
        self._check(self.L.dbt_decode_step_primary_only_host(self._h, tokens_host.data_ptr(), tokens_host.shape[0],
                                                             next_host.data_ptr()))

    def decode_full(self, tokens_dev: torch.Tensor, grouped: bool = True) -> dict:
        """One step returning every output (test convenience).  The library replays a step as
        a CUDA graph keyed by its buffer addresses, so the buffers are kept and reused; the
        returned tensors are copies."""
        B, V = tokens_dev.shape[0], self.cfg.vocab
        cache = self.__dict__.setdefault("_full_bufs", {})
        buf = cache.get(B)
        if buf is None:
            buf = {"tok": torch.empty(B, dtype=torch.int32, device=self.device),
                   "next": torch.empty(B, dtype=torch.int32, device=self.device),
                   "z1": torch.empty(B, V, dtype=torch.float32, device=self.device),
                   "z2": torch.empty((B, V) if self.cfg.n_paths == 2 else (self.cfg.n_paths - 1, B, V),
                                     dtype=torch.float32, device=self.device),
                   "alpha": torch.empty(B, dtype=torch.float32, device=self.device)}
            cache[B] = buf
        buf["tok"].copy_(tokens_dev)
        if grouped:
            self.decode_step(buf["tok"], buf["next"], buf["z1"], buf["z2"], buf["alpha"])
            return {k: buf[k].clone() for k in ("next", "z1", "z2", "alpha")}
        self.decode_step_primary_only(buf["tok"], buf["next"], buf["z1"])
        return {k: buf[k].clone() for k in ("next", "z1")}

    # -- diagnostics ----------------------------------------------------------------------
    def last_experts(self, batch: int) -> torch.Tensor:
        """[n_layers, n_paths, batch, kmax] expert ids used by the last decode step."""
        ptr, km = C.c_void_p(None), C.c_int32(0)
        self._check(self.L.dbt_last_experts(self._h, C.byref(ptr), C.byref(km)))
        n = self.cfg.n_layers * self.cfg.n_paths * self.max_batch * km.value
        torch.cuda.synchronize(self.device)
        host = torch.empty(n, dtype=torch.int32)
        # the ids live inside the workspace tensor: locate them by address
        off = ptr.value - self.workspace.data_ptr()
        host.copy_(self.workspace[off:off + 4 * n].view(torch.int32).cpu())
        return host.view(self.cfg.n_layers, self.cfg.n_paths, self.max_batch, km.value)[:, :, :batch].contiguous()

    def last_expert_union(self) -> list[int]:
        buf = (C.c_int32 * self.cfg.n_layers)()
        self._check(self.L.dbt_last_expert_union(self._h, buf))
        return list(buf)

    def sync_status(self) -> tuple[int, int]:
        s, d = C.c_int32(0), C.c_int32(0)
        st = self.L.dbt_sync_status(self._h, C.byref(s), C.byref(d))
        if st not in (DBT_OK, 6, 7):
            self._check(st)
        return s.value, d.value

    def profile_begin(self):
        self._check(self.L.dbt_profile_begin(self._h))

    def profile_end(self) -> list[dict]:
        buf = (DbtProfileEntry * 64)()
        n = C.c_int32(0)
        self._check(self.L.dbt_profile_end(self._h, buf, 64, C.byref(n)))
        return [dict(name=buf[i].name.decode(), launches=buf[i].launches, total_ms=buf[i].total_ms,
                     bytes=buf[i].bytes) for i in range(n.value)]

    def launch_count(self) -> int:
        return self.L.dbt_launch_count(self._h)

    # -- the cache through the C ABI (dbt_kv_export / dbt_kv_import) ---------------------------
    def export_kv(self, batch: int, length: int, seq_ids=None):
        """K, V [n_layers, batch, length, kv_dim] of sequences `seq_ids` (default 0..batch-1) as CPU
        tensors of the model's storage type."""
        c = self.cfg
        k = torch.empty(c.n_layers, batch, length, c.kv_dim, dtype=c.torch_dtype)
        v = torch.empty_like(k)
        ids = None if seq_ids is None else torch.as_tensor(seq_ids, dtype=torch.int32).contiguous()
        assert ids is None or ids.numel() == batch
        self._check(self.L.dbt_kv_export(self._h, _p(ids), batch, length, k.data_ptr(), v.data_ptr()))
        return k, v

    def import_kv(self, k: torch.Tensor, v: torch.Tensor, seq_ids=None):
        """Load K, V [n_layers, B, T, kv_dim] (any float type; converted to the model's) into sequences
        `seq_ids` (default 0..B-1) and set their lengths to T."""
        c = self.cfg
        k = k.to("cpu", c.torch_dtype).contiguous()
        v = v.to("cpu", c.torch_dtype).contiguous()
        assert k.shape == v.shape and k.shape[0] == c.n_layers and k.shape[3] == c.kv_dim
        ids = None if seq_ids is None else torch.as_tensor(seq_ids, dtype=torch.int32).contiguous()
        assert ids is None or ids.numel() == k.shape[1]
        self._check(self.L.dbt_kv_import(self._h, _p(ids), k.shape[1], k.shape[2], k.data_ptr(), v.data_ptr()))

    # -- direct pool access for the benchmark's synthetic fills (the pool is the caller's memory) --
    def write_kv(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor | None = None):
        """Scatter contiguous K, V [L, B, T, kv_dim] into the paged pool and set the lengths."""
        B, T = k.shape[1], k.shape[2]
        pt = page_table if page_table is not None else self.page_table
        scatter_kv(self.kv_view(), k.to(self.device, self.cfg.torch_dtype), v.to(self.device, self.cfg.torch_dtype),
                   pt.to(self.device), self.cfg)
        self.set_seq_lens([T] * B)


def _page_slot(pt: torch.Tensor, T: int, page_size: int):
    pos = torch.arange(T, device=pt.device)
    pages = pt.long()[:, pos // page_size]                       # [B, T] physical page of each position
    slots = (pos % page_size)[None, :].expand(pt.shape[0], T)    # [B, T]
    return pages, slots


def scatter_kv(view: torch.Tensor, k: torch.Tensor, v: torch.Tensor, pt: torch.Tensor, cfg: ModelConfig):
    """view [L, 2, P, n_kv, page, dh]  <-  k, v [L, B, T, kv_dim] through page table pt [B, pages]."""
    Lyr, B, T, _ = k.shape
    pages, slots = _page_slot(pt[:B], T, cfg.page_size)
    for which, src in ((0, k), (1, v)):
        s = src.view(Lyr, B, T, cfg.n_kv_heads, cfg.head_dim).permute(1, 2, 0, 3, 4)  # [B, T, L, n_kv, dh]
        sub = view[:, which]                                                          # [L, P, n_kv, page, dh]
        sub[:, pages, :, slots, :] = s  # the two index tensors broadcast to [B, T] and move to the front
