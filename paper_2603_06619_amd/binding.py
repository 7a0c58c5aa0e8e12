"""ctypes binding of include/nat.h.  Argument marshalling only (an input whose rows are one and the same in memory is copied, see _rows)."""
import ctypes
import functools
import os

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libnat_hip.so"
_lib = None

FULL, URS, RPC, DET = 0, 1, 2, 3
DTYPE_F32, DTYPE_BF16 = 0, 1
KL_LOG_RATIO, KL_NONNEG = 0, 1
KV_BF16, KV_FP8 = 0, 1
DIAG_BAD_ID, DIAG_SHIFT_RANGE, DIAG_CLIPPED, DIAG_NONZERO_ADV, DIAG_WORDS = 0, 1, 2, 3, 4


class NatError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where} failed: {status_string(status)} ({status})")


class _CSelectParams(ctypes.Structure):
    _fields_ = [("scheme", ctypes.c_int32), ("min_cut", ctypes.c_int32), ("p", ctypes.c_double),
                ("trunc_frac", ctypes.c_double), ("seed", ctypes.c_uint64), ("step", ctypes.c_uint32),
                ("rollout_id_base", ctypes.c_int32), ("d_scheme_per_rollout", ctypes.c_void_p),
                ("d_drop_zero_adv", ctypes.c_void_p)]


class _CAttnParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "causal")] + \
               [("scale", ctypes.c_float)] + \
               [(n, ctypes.c_int64) for n in ("n_q", "n_k", "q_stride", "k_stride", "v_stride", "out_stride", "dout_stride",
                                              "dq_stride", "dk_stride", "dv_stride")]


class _CKvCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("d_k", "d_v", "d_k_exp", "d_v_exp")] + \
               [(n, ctypes.c_int32) for n in ("n_pages", "n_kv_heads", "page_size", "head_dim", "format")]


class SelectParams:
    """Selection parameters of nat_select / nat_compact (see nat_select_params in nat.h)."""

    def __init__(self, scheme, p=1.0, min_cut=1, trunc_frac=1.0, seed=0, step=0, rollout_id_base=0,
                 scheme_per_rollout=None, drop_zero_adv=None):
        self.scheme, self.p, self.min_cut, self.trunc_frac = scheme, p, min_cut, trunc_frac
        self.seed, self.step, self.rollout_id_base = seed, step, rollout_id_base
        self.scheme_per_rollout = scheme_per_rollout      # int32 device tensor [B] or None
        self.drop_zero_adv = drop_zero_adv                # float32 device tensor [B] of advantages or None

    def _c(self):
        spr = self.scheme_per_rollout
        if spr is not None:
            _check(spr, torch.int32, "scheme_per_rollout")
        return _CSelectParams(int(self.scheme), int(self.min_cut), float(self.p), float(self.trunc_frac),
                              int(self.seed) & (2 ** 64 - 1), int(self.step) & 0xFFFFFFFF, int(self.rollout_id_base),
                              spr.data_ptr() if spr is not None else None,
                              _check(self.drop_zero_adv, torch.float32, "drop_zero_adv").data_ptr()
                              if self.drop_zero_adv is not None else None)


def library_path():
    # NAT_HIP_LIBRARY selects another build of the same library (A/B timing of kernel variants)
    return os.environ.get("NAT_HIP_LIBRARY") or os.path.join(_PKG_DIR, _LIB_NAME)


def load_library():
    """Load the built library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with `python -m paper_2603_06619_amd.build`")
    lib = ctypes.CDLL(path)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    pp = ctypes.POINTER(_CSelectParams)
    lib.nat_status_string.restype = ctypes.c_char_p
    lib.nat_status_string.argtypes = [i32]
    lib.nat_mask_words.restype = i64
    lib.nat_mask_words.argtypes = [i64]
    lib.nat_advantage.restype = i32
    lib.nat_advantage.argtypes = [vp, i32, i32, f32, vp, vp]
    lib.nat_select.restype = i32
    lib.nat_select.argtypes = [pp, vp, i32, i64, vp, vp, vp]
    lib.nat_compact_workspace_bytes.restype = sz
    lib.nat_compact_workspace_bytes.argtypes = [i64]
    lib.nat_compact.restype = i32
    lib.nat_compact.argtypes = [pp, i32, vp, vp, i32, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32,
                                vp, vp, vp, vp, vp, sz, vp]
    lib.nat_compact_static.restype = i32
    lib.nat_compact_static.argtypes = [pp, i32, vp, vp, i32, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32,
                                       vp, vp, vp, vp, vp]
    lib.nat_select_schedule.restype = i32
    lib.nat_select_schedule.argtypes = [pp, vp, vp, i32, i64, vp, vp, vp, vp]
    lib.nat_select_poisson.restype = i32
    lib.nat_select_poisson.argtypes = [pp, vp, vp, i32, i64, vp, vp]
    lib.nat_compact_pi.restype = i32
    lib.nat_compact_pi.argtypes = [i32, vp, vp, vp, i32, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32,
                                   vp, vp, vp, vp, vp, sz, vp]
    lib.nat_prefix_pack.restype = i32
    lib.nat_prefix_pack.argtypes = [vp, vp, vp, i32, i32, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    for name in ("nat_loss_workspace_bytes", "nat_loss_workspace_min_bytes"):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = [i32, i32, i32, i32]
    lib.nat_loss_fwd_bwd.restype = i32
    lib.nat_loss_fwd_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, f32, f32, f32,
                                     vp, vp, vp, vp, i32, vp, sz, vp]
    lib.nat_loss_fwd_bwd_kl.restype = i32
    lib.nat_loss_fwd_bwd_kl.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, f32, f32, f32,
                                        vp, f32, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    for name in ("nat_logp_workspace_bytes", "nat_logp_workspace_min_bytes"):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = [i32, i32, i32, i32]
    lib.nat_logp_fwd.restype = i32
    lib.nat_logp_fwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    pa, pc = ctypes.POINTER(_CAttnParams), ctypes.POINTER(_CKvCache)
    lib.nat_attn_fwd.restype = i32
    lib.nat_attn_fwd.argtypes = [pa, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.nat_attn_fwd_workspace_bytes.restype = sz
    lib.nat_attn_fwd_workspace_bytes.argtypes = [pa]
    lib.nat_attn_fwd_split.restype = i32
    lib.nat_attn_fwd_split.argtypes = [pa, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.nat_attn_bwd_workspace_bytes.restype = sz
    lib.nat_attn_bwd_workspace_bytes.argtypes = [i64, i32]
    lib.nat_attn_bwd_workspace_full_bytes.restype = sz
    lib.nat_attn_bwd_workspace_full_bytes.argtypes = [pa]
    lib.nat_attn_bwd.restype = i32
    lib.nat_attn_bwd.argtypes = [pa, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.nat_kv_write.restype = i32
    lib.nat_kv_write.argtypes = [pc, vp, i64, vp, i64, vp, i64, vp]
    lib.nat_kv_read.restype = i32
    lib.nat_kv_read.argtypes = [pc, vp, i32, vp, i32, i64, vp, i64, vp, i64, vp]
    lib.nat_attn_decode_workspace_bytes.restype = sz
    lib.nat_attn_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i64]
    lib.nat_attn_decode.restype = i32
    lib.nat_attn_decode.argtypes = [pc, vp, i64, i32, i32, vp, i32, vp, f32, vp, i64, vp, vp, sz, vp]
    lib.nat_sample.restype = i32
    lib.nat_sample.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.nat_sample_workspace_bytes.restype = sz
    lib.nat_sample_workspace_bytes.argtypes = [i32, i32, i32]
    lib.nat_probe_mfma_scratch_bytes.restype = sz
    lib.nat_probe_mfma_scratch_bytes.argtypes = []
    lib.nat_probe_mfma_bf16.restype = i32
    lib.nat_probe_mfma_bf16.argtypes = [i32, i32, vp, ctypes.POINTER(ctypes.c_double), vp]
    lib.nat_probe_copy.restype = i32
    lib.nat_probe_copy.argtypes = [vp, vp, sz, vp]
    lib.nat_profile_num_classes.restype = i32
    lib.nat_profile_class_name.restype = ctypes.c_char_p
    lib.nat_profile_class_name.argtypes = [i32]
    lib.nat_profile_enable.restype = i32
    lib.nat_profile_enable.argtypes = [i32]
    lib.nat_profile_collect.restype = i32
    lib.nat_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64), i32]
    _lib = lib
    return lib


def status_string(status):
    return load_library().nat_status_string(int(status)).decode()


def _check(t, dtype, name):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous {dtype} tensor")
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    # hipStream_t of the current stream; torch.cuda.current_stream() builds a Stream object around it (2.8 us of host
    # time a call, five calls a step)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _raise(status, where):
    if status != 0:
        raise NatError(status, where)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return DTYPE_F32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    raise TypeError("hidden / W must be float32 or bfloat16")


def mask_words(N):
    return int(load_library().nat_mask_words(int(N)))


def compact_workspace_bytes(N):
    return int(load_library().nat_compact_workspace_bytes(int(N)))


def loss_workspace_bytes(N_k, H, V, dtype):
    return int(load_library().nat_loss_workspace_bytes(int(N_k), int(H), int(V), int(dtype)))


def loss_workspace_min_bytes(N_k, H, V, dtype):
    return int(load_library().nat_loss_workspace_min_bytes(int(N_k), int(H), int(V), int(dtype)))


def nat_advantage(rewards, P, G, eps_adv, adv_out):
    _check(rewards, torch.float32, "rewards")
    _check(adv_out, torch.float32, "adv_out")
    _raise(load_library().nat_advantage(_ptr(rewards), P, G, eps_adv, _ptr(adv_out), _stream()), "nat_advantage")


def nat_select(params, cu_seqlens, B, N, cut_len_out, mask_bits_out):
    _check(cu_seqlens, torch.int64, "cu_seqlens")
    _check(cut_len_out, torch.int32, "cut_len_out")
    _check(mask_bits_out, torch.int32, "mask_bits_out")
    c = params._c()
    _raise(load_library().nat_select(ctypes.byref(c), _ptr(cu_seqlens), B, N, _ptr(cut_len_out),
                                     _ptr(mask_bits_out), _stream()), "nat_select")


def _kept_cap(kept_cap, kept_idx):
    return int(kept_idx.numel() if kept_cap is None and kept_idx is not None else (kept_cap or 0))


def nat_compact(params, n_rollouts_global, mask_bits, cu_seqlens, B, N, kept_idx, kept_seq, kept_w, cu_kept,
                n_kept, h_n_kept, workspace, hidden=None, hidden_k=None, ids=None, ids_k=None,
                old_logp=None, old_logp_k=None, kept_cap=None):
    """kept_cap: capacity of the per-kept-token outputs; default: the length of kept_idx."""
    c = params._c()
    H = hidden.shape[1] if hidden is not None else 0
    dt = _dtype_code(hidden) if hidden is not None else DTYPE_F32
    _raise(load_library().nat_compact(
        ctypes.byref(c), n_rollouts_global, _ptr(mask_bits), _ptr(cu_seqlens), B, N, _kept_cap(kept_cap, kept_idx),
        _ptr(kept_idx), _ptr(kept_seq),
        _ptr(kept_w), _ptr(cu_kept), _ptr(n_kept), _ptr(h_n_kept), _ptr(hidden), _ptr(hidden_k), H, dt,
        _ptr(ids), _ptr(ids_k), _ptr(old_logp), _ptr(old_logp_k), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()), "nat_compact")


def nat_compact_static(params, n_rollouts_global, mask_bits, cu_seqlens, B, N, kept_idx, kept_seq, kept_w, cu_kept,
                       n_kept, h_n_kept, hidden=None, hidden_k=None, ids=None, ids_k=None,
                       old_logp=None, old_logp_k=None, kept_cap=None):
    """nat_compact without a workspace argument (the library's resident scratch); allocates nothing."""
    c = params._c()
    H = hidden.shape[1] if hidden is not None else 0
    dt = _dtype_code(hidden) if hidden is not None else DTYPE_F32
    _raise(load_library().nat_compact_static(
        ctypes.byref(c), n_rollouts_global, _ptr(mask_bits), _ptr(cu_seqlens), B, N, _kept_cap(kept_cap, kept_idx),
        _ptr(kept_idx), _ptr(kept_seq), _ptr(kept_w), _ptr(cu_kept), _ptr(n_kept), _ptr(h_n_kept), _ptr(hidden),
        _ptr(hidden_k), H, dt, _ptr(ids), _ptr(ids_k), _ptr(old_logp), _ptr(old_logp_k), _stream()),
        "nat_compact_static")


def nat_select_schedule(params, weights, cu_seqlens, B, N, cut_len_out, mask_bits_out, pi_out):
    _check(cu_seqlens, torch.int64, "cu_seqlens")
    _check(weights, torch.int32, "weights")          # the 32 bits are read as unsigned
    _check(cut_len_out, torch.int32, "cut_len_out")
    _check(mask_bits_out, torch.int32, "mask_bits_out")
    _check(pi_out, torch.float64, "pi_out")
    c = params._c()
    _raise(load_library().nat_select_schedule(ctypes.byref(c), _ptr(weights), _ptr(cu_seqlens), B, N,
                                              _ptr(cut_len_out), _ptr(mask_bits_out), _ptr(pi_out), _stream()),
           "nat_select_schedule")


def nat_select_poisson(params, pi, cu_seqlens, B, N, mask_bits_out):
    _check(cu_seqlens, torch.int64, "cu_seqlens")
    _check(pi, torch.float64, "pi")
    _check(mask_bits_out, torch.int32, "mask_bits_out")
    c = params._c()
    _raise(load_library().nat_select_poisson(ctypes.byref(c), _ptr(pi), _ptr(cu_seqlens), B, N,
                                             _ptr(mask_bits_out), _stream()), "nat_select_poisson")


def nat_compact_pi(n_rollouts_global, mask_bits, pi, cu_seqlens, B, N, kept_idx, kept_seq, kept_w, cu_kept,
                   n_kept, h_n_kept, workspace, hidden=None, hidden_k=None, ids=None, ids_k=None,
                   old_logp=None, old_logp_k=None, kept_cap=None):
    _check(pi, torch.float64, "pi")
    H = hidden.shape[1] if hidden is not None else 0
    dt = _dtype_code(hidden) if hidden is not None else DTYPE_F32
    _raise(load_library().nat_compact_pi(
        n_rollouts_global, _ptr(mask_bits), _ptr(pi), _ptr(cu_seqlens), B, N, _kept_cap(kept_cap, kept_idx),
        _ptr(kept_idx), _ptr(kept_seq),
        _ptr(kept_w), _ptr(cu_kept), _ptr(n_kept), _ptr(h_n_kept), _ptr(hidden), _ptr(hidden_k), H, dt,
        _ptr(ids), _ptr(ids_k), _ptr(old_logp), _ptr(old_logp_k), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()), "nat_compact_pi")


def nat_prefix_pack(prompt_len, cu_seqlens, cut_len, B, next_token_shift, rows_cap, kept_cap, cu_packed, cu_loss,
                    src_idx, position_ids, loss_row, totals, h_totals, input_ids=None, input_ids_packed=None):
    _check(cu_seqlens, torch.int64, "cu_seqlens")
    _check(cut_len, torch.int32, "cut_len")
    _raise(load_library().nat_prefix_pack(
        _ptr(prompt_len), _ptr(cu_seqlens), _ptr(cut_len), B, int(next_token_shift), int(rows_cap), int(kept_cap),
        _ptr(cu_packed), _ptr(cu_loss), _ptr(src_idx), _ptr(position_ids), _ptr(loss_row), _ptr(totals),
        _ptr(h_totals), _ptr(input_ids), _ptr(input_ids_packed), _stream()), "nat_prefix_pack")


def nat_loss_fwd_bwd(hidden_k, W, ids_k, old_logp_k, adv, kept_seq, kept_w, N_k, eps_lo, eps_hi, grad_scale,
                     loss_out, logp_out, dH_out, dW_out, accumulate_dw, workspace):
    V, H = W.shape
    _raise(load_library().nat_loss_fwd_bwd(
        _ptr(hidden_k), _ptr(W), _ptr(ids_k), _ptr(old_logp_k), _ptr(adv), _ptr(kept_seq), _ptr(kept_w),
        N_k, H, V, _dtype_code(W), eps_lo, eps_hi, grad_scale, _ptr(loss_out), _ptr(logp_out), _ptr(dH_out),
        _ptr(dW_out), int(accumulate_dw), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()), "nat_loss_fwd_bwd")


def nat_loss_fwd_bwd_kl(hidden_k, W, ids_k, old_logp_k, adv, kept_seq, kept_w, N_k, eps_lo, eps_hi, grad_scale,
                        ref_logp_k, beta_kl, kl_kind, loss_out, logp_out, kl_out, entropy_out, dH_out, dW_out,
                        accumulate_dw, workspace, diag_out=None):
    V, H = W.shape
    _raise(load_library().nat_loss_fwd_bwd_kl(
        _ptr(hidden_k), _ptr(W), _ptr(ids_k), _ptr(old_logp_k), _ptr(adv), _ptr(kept_seq), _ptr(kept_w),
        N_k, H, V, _dtype_code(W), eps_lo, eps_hi, grad_scale, _ptr(ref_logp_k), float(beta_kl), int(kl_kind),
        _ptr(loss_out), _ptr(logp_out), _ptr(kl_out), _ptr(entropy_out), _ptr(diag_out), _ptr(dH_out), _ptr(dW_out),
        int(accumulate_dw), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()),
        "nat_loss_fwd_bwd_kl")


def logp_workspace_bytes(N_k, H, V, dtype):
    return int(load_library().nat_logp_workspace_bytes(int(N_k), int(H), int(V), int(dtype)))


def logp_workspace_min_bytes(N_k, H, V, dtype):
    return int(load_library().nat_logp_workspace_min_bytes(int(N_k), int(H), int(V), int(dtype)))


def nat_logp_fwd(hidden_k, W, ids_k, N_k, logp_out, entropy_out, workspace, diag_out=None):
    V, H = W.shape
    _raise(load_library().nat_logp_fwd(
        _ptr(hidden_k), _ptr(W), _ptr(ids_k), N_k, H, V, _dtype_code(W), _ptr(logp_out), _ptr(entropy_out),
        _ptr(diag_out), _ptr(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()),
        "nat_logp_fwd")


_SHARED = -1


def _rows(t, name, shape=None, dtype=torch.bfloat16, is_input=False):
    """A [rows, heads, head_dim] tensor whose heads lie back to back; returns its row stride.  What the kernels need and the
    library cannot see (device, element type, extents) is checked here.  A stride of 0 (a tensor expanded along its rows: a gradient that is equal for all of them, one
    query for several sequences) would mean rows back to back to the library: _SHARED for an input, which the caller then gives rows of its own."""
    if t.dtype != dtype or t.dim() != 3 or not t.is_cuda:
        raise TypeError(f"{name}: expected a {dtype} device tensor [rows, heads, head_dim]")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.is_contiguous():
        return 0
    row, head, one = t.stride()
    n, heads, dim = t.shape
    if n == 0 or heads == 0 or dim == 0:
        return 0
    if is_input and n > 1 and row == 0:
        return _SHARED
    if (dim > 1 and one != 1) or (heads > 1 and head != dim):
        raise ValueError(f"{name}: the heads of a row must lie back to back")
    if n > 1 and row < heads * dim:
        raise ValueError(f"{name}: its rows overlap in memory")
    return row if n > 1 else 0


def _own_rows(tensors, strides):
    """Inputs and what _rows says of them, with rows of their own for those that share one."""
    if _SHARED not in strides:
        return tensors, strides
    return [t.contiguous() if r == _SHARED else t for t, r in zip(tensors, strides)], [max(r, 0) for r in strides]


def _vector(t, dtype, n, name):
    if t is None:
        return None
    if t.dtype != dtype or not t.is_cuda or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous {dtype} device tensor of {n} elements")
    return t.data_ptr()


def _attn_params(q, k, v, cu_q, cu_k, causal, scale):
    n_q, hq, dim = q.shape
    n_k, hkv, _ = k.shape
    n_seqs = max(cu_q.numel() - 1, 0)
    _vector(cu_q, torch.int32, n_seqs + 1, "cu_q")
    _vector(cu_k, torch.int32, n_seqs + 1, "cu_k")
    (q, k, v), strides = _own_rows((q, k, v), (_rows(q, "q", is_input=True), _rows(k, "k", (n_k, hkv, dim), is_input=True),
                                               _rows(v, "v", (n_k, hkv, dim), is_input=True)))
    return _CAttnParams(n_seqs, hq, hkv, dim, DTYPE_BF16, int(causal), float(scale), n_q, n_k, *strides), q, k, v


@functools.lru_cache(maxsize=256)
def attn_fwd_workspace_bytes(n_q, n_k, n_seqs, n_q_heads, n_kv_heads, head_dim, causal):
    p = _CAttnParams(int(n_seqs), int(n_q_heads), int(n_kv_heads), int(head_dim), DTYPE_BF16, int(causal), 1.0, int(n_q), int(n_k))
    return int(load_library().nat_attn_fwd_workspace_bytes(ctypes.byref(p)))


def nat_attn_fwd(q, k, v, cu_q, cu_k, causal, scale, out, lse, workspace=None):
    """q [n_q, q heads, D], k, v [n_k, kv heads, D] bf16 (any row stride); cu_q, cu_k int32 [n_seqs + 1]; out like q, lse float32
    [q heads, n_q].  With a workspace (attn_fwd_workspace_bytes) this is nat_attn_fwd_split."""
    p, q, k, v = _attn_params(q, k, v, cu_q, cu_k, causal, scale)
    p.out_stride = _rows(out, "out", q.shape)
    args = (ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_q), _ptr(cu_k), _ptr(out), _vector(lse, torch.float32, p.n_q_heads * p.n_q, "lse"))
    if workspace is None:
        _raise(load_library().nat_attn_fwd(*args, _stream()), "nat_attn_fwd")
    else:
        _raise(load_library().nat_attn_fwd_split(*args, _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()), "nat_attn_fwd_split")


def attn_bwd_workspace_bytes(n_q, n_q_heads):
    return int(load_library().nat_attn_bwd_workspace_bytes(int(n_q), int(n_q_heads)))


@functools.lru_cache(maxsize=256)
def attn_bwd_workspace_full_bytes(n_q, n_k, n_seqs, n_q_heads, n_kv_heads, head_dim, causal):
    p = _CAttnParams(int(n_seqs), int(n_q_heads), int(n_kv_heads), int(head_dim), DTYPE_BF16, int(causal), 1.0, int(n_q), int(n_k))
    return int(load_library().nat_attn_bwd_workspace_full_bytes(ctypes.byref(p)))


def nat_attn_bwd(q, k, v, out, lse, dout, cu_q, cu_k, causal, scale, dq, dk, dv, workspace):
    """The gradients of nat_attn_fwd; dq like q, dk and dv like k (any row stride)."""
    p, q, k, v = _attn_params(q, k, v, cu_q, cu_k, causal, scale)
    (out, dout), (p.out_stride, p.dout_stride) = _own_rows((out, dout), (_rows(out, "out", q.shape, is_input=True), _rows(dout, "dout", q.shape, is_input=True)))
    p.dq_stride, p.dk_stride, p.dv_stride = _rows(dq, "dq", q.shape), _rows(dk, "dk", k.shape), _rows(dv, "dv", k.shape)
    _raise(load_library().nat_attn_bwd(
        ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _vector(lse, torch.float32, p.n_q_heads * p.n_q, "lse"), _ptr(dout),
        _ptr(cu_q), _ptr(cu_k), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()), "nat_attn_bwd")


class KvCache:
    """The arrays of a paged cache: k, v [n_pages, kv heads, page_size, D] in bfloat16, or in float8_e4m3fn with the exponents
    k_exp, v_exp [n_pages, kv heads, page_size] uint8 (see nat_kv_cache in nat.h)."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        shape, dtype = k.shape, k.dtype
        fp8 = dtype == torch.float8_e4m3fn
        if len(shape) != 4 or not (fp8 or dtype == torch.bfloat16):
            raise TypeError("k: expected a bfloat16 or float8_e4m3fn tensor [n_pages, heads, page_size, head_dim]")
        if not (k.is_contiguous() and k.is_cuda):
            raise TypeError(f"k: expected a contiguous {dtype} device tensor {tuple(shape)}")
        if v.shape != shape or v.dtype != dtype or not v.is_contiguous() or not v.is_cuda:
            raise TypeError(f"v: expected a contiguous {dtype} device tensor {tuple(shape)}")
        if fp8:
            rows = shape[:3]
            for t in (k_exp, v_exp):
                if t is None or t.shape != rows or t.dtype != torch.uint8 or not t.is_contiguous() or not t.is_cuda:
                    raise TypeError(f"{'k_exp' if t is k_exp else 'v_exp'}: expected a contiguous uint8 device tensor {tuple(rows)}")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        n_pages, heads, page_size, dim = shape
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = n_pages, heads, page_size, dim
        self._c = _CKvCache(k.data_ptr(), v.data_ptr(), k_exp.data_ptr() if fp8 else None, v_exp.data_ptr() if fp8 else None,
                            n_pages, heads, page_size, dim, KV_FP8 if fp8 else KV_BF16)


def nat_kv_write(cache, k, v, slots):
    """k, v [rows, kv heads, D] bf16; slots int64 [rows], -1 for rows that are skipped."""
    n = k.shape[0]
    shape = (n, cache.n_kv_heads, cache.head_dim)
    (k, v), (k_stride, v_stride) = _own_rows((k, v), (_rows(k, "k", shape, is_input=True), _rows(v, "v", shape, is_input=True)))
    _raise(load_library().nat_kv_write(ctypes.byref(cache._c), _ptr(k), k_stride, _ptr(v), v_stride,
                                       _vector(slots, torch.int64, n, "slots"), n, _stream()), "nat_kv_write")


def _table(block_table, n_seqs):
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or not block_table.is_contiguous() or not block_table.is_cuda or \
            block_table.shape[0] != n_seqs:
        raise TypeError(f"block_table: expected a contiguous int32 device tensor [{n_seqs}, pages]")
    return block_table.shape[1]


def nat_kv_read(cache, block_table, cu_k, k, v):
    """block_table int32 [n_seqs, pages], cu_k int32 [n_seqs + 1]; k, v [rows, kv heads, D] bf16 out."""
    n_seqs = max(cu_k.numel() - 1, 0)
    shape = (k.shape[0], cache.n_kv_heads, cache.head_dim)
    width = _table(block_table, n_seqs)
    _raise(load_library().nat_kv_read(ctypes.byref(cache._c), _ptr(block_table), width, _vector(cu_k, torch.int32, n_seqs + 1, "cu_k"), n_seqs,
                                      k.shape[0], _ptr(k), _rows(k, "k", shape), _ptr(v), _rows(v, "v", shape), _stream()), "nat_kv_read")


@functools.lru_cache(maxsize=256)
def attn_decode_workspace_bytes(n_seqs, n_q_heads, n_kv_heads, head_dim, max_tokens):
    return int(load_library().nat_attn_decode_workspace_bytes(int(n_seqs), int(n_q_heads), int(n_kv_heads), int(head_dim), int(max_tokens)))


def nat_attn_decode(cache, q, block_table, seq_lens, scale, out, lse, workspace):
    """q [n_seqs, q heads, D] bf16, block_table int32 [n_seqs, pages], seq_lens int32 [n_seqs]; out like q, lse float32 [n_seqs, q heads]."""
    n_seqs, hq, _ = q.shape
    width = _table(block_table, n_seqs)
    shape = (n_seqs, hq, cache.head_dim)
    (q,), (q_stride,) = _own_rows((q,), (_rows(q, "q", shape, is_input=True),))
    _raise(load_library().nat_attn_decode(
        ctypes.byref(cache._c), _ptr(q), q_stride, n_seqs, hq, _ptr(block_table), width,
        _vector(seq_lens, torch.int32, n_seqs, "seq_lens"), float(scale), _ptr(out), _rows(out, "out", shape),
        _vector(lse, torch.float32, n_seqs * hq, "lse"), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()), "nat_attn_decode")


@functools.lru_cache(maxsize=256)
def sample_workspace_bytes(n_rows, V, dtype):
    return int(load_library().nat_sample_workspace_bytes(int(n_rows), int(V), int(dtype)))


def nat_sample(logits, random, temperature, top_k, top_p, min_p, ids_out, logp_out=None, logq_out=None, workspace=None):
    """logits [rows, V] float32 or bfloat16 (any row stride), random int32 [rows] (the 32 bits are read as unsigned); temperature,
    top_p, min_p float32 [rows] and top_k int32 [rows], each or None; ids int32, logp and logq float32 [rows] out."""
    if logits.dim() != 2 or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError("logits: expected a device tensor [rows, vocabulary] with its rows contiguous")
    n, V = logits.shape
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    row = logits.stride(0) if n > 1 else V
    if row < V:
        if row > 0:
            raise ValueError("logits: rows overlap in memory")
        logits, row = logits.contiguous(), V             # one row for all, which the library would read as rows back to back
    _raise(load_library().nat_sample(
        _ptr(logits), row, n, V, _dtype_code(logits), _vector(random, torch.int32, n, "random"),
        _vector(temperature, torch.float32, n, "temperature"), _vector(top_k, torch.int32, n, "top_k"),
        _vector(top_p, torch.float32, n, "top_p"), _vector(min_p, torch.float32, n, "min_p"),
        _vector(ids_out, torch.int32, n, "ids_out"), _vector(logp_out, torch.float32, n, "logp_out"),
        _vector(logq_out, torch.float32, n, "logq_out"), _ptr(workspace),
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream()), "nat_sample")


def probe_mfma_scratch_bytes():
    return int(load_library().nat_probe_mfma_scratch_bytes())


def nat_probe_mfma_bf16(random_operands, iters, scratch):
    """Launches the matrix-core probe on the current stream; returns the flops of the launch."""
    flops = ctypes.c_double(0.0)
    _raise(load_library().nat_probe_mfma_bf16(int(bool(random_operands)), int(iters), _ptr(scratch),
                                              ctypes.byref(flops), _stream()), "nat_probe_mfma_bf16")
    return flops.value


def nat_probe_copy(dst, src, nbytes):
    _raise(load_library().nat_probe_copy(_ptr(dst), _ptr(src), int(nbytes), _stream()), "nat_probe_copy")


def profile_enable(on):
    _raise(load_library().nat_profile_enable(int(bool(on))), "nat_profile_enable")


def profile_collect():
    """Returns {class name: (milliseconds, launches)} accumulated since the last call."""
    lib = load_library()
    n = lib.nat_profile_num_classes()
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _raise(lib.nat_profile_collect(ms, cnt, n), "nat_profile_collect")
    return {lib.nat_profile_class_name(i).decode(): (ms[i], cnt[i]) for i in range(n)}
