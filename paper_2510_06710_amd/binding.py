"""ctypes binding of libvla.so: the same entry points as include/vla.h, argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch appears here solely as the owner
of device memory (``tensor.data_ptr()``) and of the stream the work is enqueued on.  If the library
has not been built this module raises on first use -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libvla.so")

VLA_OK, VLA_EINVAL, VLA_ESHAPE, VLA_EWORKSPACE, VLA_EDTYPE, VLA_EHIP = 0, -1, -2, -3, -4, -5
VLA_DTYPE_F32, VLA_DTYPE_BF16 = 0, 1
VLA_MODE_AR, VLA_MODE_PARALLEL_CHUNK = 0, 1
VLA_ENTRY_PREFILL, VLA_ENTRY_DECODE, VLA_ENTRY_RECOMPUTE = 0, 1, 2
VLA_N_BINS = 256
VLA_SELECT_PAGES = 8192


class vla_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_heads", C.c_int32),
                ("ffn", C.c_int32), ("vocab", C.c_int32), ("n_bins", C.c_int32),
                ("dtype", C.c_int32), ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("max_batch", C.c_int32), ("max_seq", C.c_int32), ("value_dim", C.c_int32)]


class vla_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm",
                                          "w_gate", "w_up", "w_down")]


class vla_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("value_w", C.c_void_p), ("value_b", C.c_float),
                ("layers", C.POINTER(vla_layer_weights)), ("value_bias", C.c_void_p)]


class vla_lora_factor(C.Structure):
    _fields_ = [("a", C.c_void_p), ("b", C.c_void_p)]


class vla_lora_grad(C.Structure):
    _fields_ = [("da", C.c_void_p), ("db", C.c_void_p)]


LORA_PROJECTIONS = ("q", "k", "v", "o", "gate", "up", "down")


class vla_lora_layer(C.Structure):
    _fields_ = [(n, vla_lora_factor) for n in LORA_PROJECTIONS]


class vla_lora_layer_grads(C.Structure):
    _fields_ = [(n, vla_lora_grad) for n in LORA_PROJECTIONS]


class vla_placement(C.Structure):
    _fields_ = [("k", C.c_int32), ("n_gen", C.c_int32), ("n_sim", C.c_int32), ("time", C.c_double)]


class vla_paged_cache(C.Structure):
    keep, device = (), None          # (make_* puts the tensors and their GPU here: of plain addresses nothing is known)
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class vla_paged_batch(C.Structure):
    keep, device = (), None
    _fields_ = [("n_seq", C.c_int32), ("n_rows", C.c_int32), ("max_rows", C.c_int32), ("max_len", C.c_int32), ("table_stride", C.c_int32),
                ("row_start", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p)]


class vla_rotary(C.Structure):
    keep, device = (None, None, None), None
    _fields_ = [("inv_freq", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_float), ("eps", C.c_float),
                ("q_gain", C.c_void_p), ("k_gain", C.c_void_p)]


class vla_paged_mask(C.Structure):
    keep, device = (None, None), None
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("slopes", C.c_void_p), ("prefix_len", C.c_void_p), ("window", C.c_int32),
                ("shared_len", C.c_int32)]


class vla_paged_rows(C.Structure):
    keep, device = (), None
    _fields_ = [("position", C.c_void_p), ("seen", C.c_void_p), ("prefix_len", C.c_void_p), ("bounds", C.c_void_p), ("mass", C.c_void_p), ("mass_stride", C.c_int64),
                ("words", C.c_int32), ("n_select", C.c_int32), ("first", C.c_int32), ("recent", C.c_int32)]


class VlaError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libvla error {code}: {message}")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """Load libvla.so (built in-tree by ``paper_2510_06710_amd.build``); fails loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(f"{_LIB_PATH} is not built; run `python -m paper_2510_06710_amd.build`")
        # The device pointers and streams this library is handed belong to PyTorch's HIP runtime, so that runtime must
        # be the one in the process: loaded first, the library's own dependency on libamdhip64 resolves to it (loaded
        # the other way round, the system copy comes in first and the kernels then find no device).
        import torch  # noqa: F401
        L = C.CDLL(_LIB_PATH)
        vp, i32, f32, sz = C.c_void_p, C.c_int, C.c_float, C.c_size_t
        L.vla_version.restype = C.c_int
        L.vla_last_error.restype = C.c_char_p
        L.vla_create.argtypes = [C.POINTER(vla_config), C.POINTER(vla_weights), C.POINTER(vp)]
        L.vla_destroy.argtypes = [vp]
        L.vla_prepack_bytes.argtypes = [C.POINTER(vla_config)]
        L.vla_prepack_bytes.restype = sz
        L.vla_prepack.argtypes = [vp, vp, sz, vp]
        L.vla_kv_bytes.argtypes = [C.POINTER(vla_config), i32, i32]
        L.vla_kv_bytes.restype = sz
        L.vla_workspace_bytes.argtypes = [C.POINTER(vla_config), i32, i32, i32, i32]
        L.vla_workspace_bytes.restype = sz
        L.vla_prefill.argtypes = [vp, vp, vp, sz, vp, vp, i32, i32, i32, vp, vp, vp]
        L.vla_decode_actions.argtypes = [vp, vp, vp, sz, vp, i32, i32, i32, i32, vp, f32, vp, vp, vp, vp, vp, vp]
        L.vla_logprob_recompute.argtypes = [vp, vp, sz, vp, vp, vp, i32, i32, i32, i32, i32, vp, f32,
                                            vp, vp, vp, vp, vp]
        L.vla_backward_workspace_bytes.argtypes = [C.POINTER(vla_config), i32, i32, i32, i32]
        L.vla_backward_workspace_bytes.restype = sz
        L.vla_backward_keep_workspace_bytes.argtypes = [C.POINTER(vla_config), i32, i32, i32, i32]
        L.vla_backward_keep_workspace_bytes.restype = sz
        L.vla_logprob_backward.argtypes = [vp, vp, sz, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, f32, i32, f32, i32,
                                           C.POINTER(vla_lora_layer), C.POINTER(vla_lora_layer_grads), vp, vp]
        L.vla_debug_force_generic.argtypes = [i32]
        L.vla_profile_enable.argtypes = [i32]
        L.vla_profile_report.argtypes = [C.c_char_p, sz]
        L.vla_calibration_copy.argtypes = [vp, vp, sz, vp]
        L.vla_gae.argtypes = [vp, vp, vp, i32, i32, f32, f32, vp, vp, vp]
        L.vla_grpo_advantage.argtypes = [vp, i32, i32, vp, vp, vp]
        L.vla_policy_objective_workspace_bytes.argtypes = [i32]
        L.vla_policy_objective_workspace_bytes.restype = sz
        L.vla_policy_objective.argtypes = [vp, vp, vp, i32, vp, i32, i32, f32, f32, i32, vp, sz, vp, vp, vp, vp]
        L.vla_policy_objective_noalloc_max_traj.restype = C.c_int
        L.vla_policy_objective_noalloc.argtypes = [vp, vp, vp, i32, vp, i32, i32, f32, f32, i32, vp, vp, vp, vp]
        L.vla_logp_aggregate.argtypes = [vp, sz, i32, vp, vp]
        i64, cache, batch = C.c_int64, C.POINTER(vla_paged_cache), C.POINTER(vla_paged_batch)
        L.vla_paged_append.argtypes = [cache, batch, C.POINTER(vla_rotary), vp, vp, vp, i32, i32, i64, i64, i64, vp, i64, vp]
        L.vla_paged_attention_workspace_bytes.argtypes = [cache, batch, C.POINTER(vla_paged_mask), i32]
        L.vla_paged_attention_workspace_bytes.restype = sz
        L.vla_paged_attention.argtypes = [cache, batch, C.POINTER(vla_paged_mask), vp, i32, i64, vp, i64, vp, vp, sz, vp]
        L.vla_forward_paged_workspace_bytes.argtypes = [C.POINTER(vla_config), cache, batch, i32]
        L.vla_forward_paged_workspace_bytes.restype = sz
        L.vla_forward_paged.argtypes = [vp, cache, sz, batch, vp, vp, i32, vp, i32, vp, sz, vp, vp, vp, vp]
        L.vla_sample_logits_workspace_bytes.argtypes = [i32, i32]
        L.vla_sample_logits_workspace_bytes.restype = sz
        L.vla_sample_logits.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        mask = C.POINTER(vla_paged_mask)
        L.vla_paged_append_at.argtypes = [cache, batch, C.POINTER(vla_rotary), vp, vp, vp, vp, i32, i32, i64, i64, i64, vp, i64, vp]
        L.vla_paged_tree.argtypes = [cache, batch, vp, vp, i32, vp, vp]
        L.vla_paged_tree_attention.argtypes = [cache, batch, mask, vp, i32, vp, i32, i64, vp, i64, vp, vp, sz, vp]
        L.vla_paged_accept.argtypes = [cache, i32, sz, batch, vp, vp, vp, vp, vp, vp, vp, vp]
        L.vla_paged_bounds.argtypes = [cache, batch, vp, vp]
        L.vla_paged_select_workspace_bytes.argtypes = [cache, batch]
        L.vla_paged_select_workspace_bytes.restype = sz
        L.vla_paged_select.argtypes = [cache, batch, vp, vp, i32, i64, i32, i32, i32, vp, vp, sz, vp]
        L.vla_paged_sparse_attention_workspace_bytes.argtypes = [cache, batch, mask, i32, i32]
        L.vla_paged_sparse_attention_workspace_bytes.restype = sz
        L.vla_paged_sparse_attention.argtypes = [cache, batch, mask, vp, i32, vp, i32, i64, vp, i64, vp, vp, sz, vp]
        L.vla_paged_weights_workspace_bytes.argtypes = [cache, batch, mask, i32]
        L.vla_paged_weights_workspace_bytes.restype = sz
        L.vla_paged_weights.argtypes = [cache, batch, mask, vp, i32, i64, vp, vp, i64, vp, sz, vp]
        L.vla_paged_evict.argtypes = [cache, batch, vp, i64, i32, i32, i32, vp, i32, vp, vp, i64, vp, vp]
        rows = C.POINTER(vla_paged_rows)
        L.vla_forward_paged_rows_workspace_bytes.argtypes = [C.POINTER(vla_config), cache, batch, rows, i32]
        L.vla_forward_paged_rows_workspace_bytes.restype = sz
        L.vla_forward_paged_rows.argtypes = [vp, cache, sz, batch, rows, vp, vp, i32, i32, vp, sz, vp, vp]
        dp = C.POINTER(C.c_double)
        L.vla_pipeline_time.argtypes = [C.c_double, C.c_double, i32, i32, dp]
        L.vla_profile_lookup.argtypes = [dp, i32, C.c_double, dp]
        L.vla_auto_placement.argtypes = [dp, dp, i32, i32, i32, i32, C.POINTER(vla_placement),
                                         C.POINTER(vla_placement), i32, C.POINTER(C.c_int)]
        _lib = L
    return _lib


def vla_last_error() -> str:
    return lib().vla_last_error().decode()


def _check(rc: int) -> None:
    if rc != VLA_OK:
        raise VlaError(rc, vla_last_error())


def _ptr(t) -> Optional[int]:
    """Device (or host) address of a tensor, None for None."""
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    """Address of the given stream, or of the calling thread's current one, which PyTorch hands out without building a
    Stream object around it: 0.4 instead of 3 us of host time per call (an epoch's advantages and objectives, four calls of
    this module and 18 us of kernels: 55 -> 45 us)."""
    if stream is not None:
        return stream.cuda_stream or None
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw and device and torch.cuda.is_initialized():          # (no public interface: other versions may lack them)
        return raw(device()) or None
    return torch.cuda.current_stream().cuda_stream or None


def vla_version() -> int:
    return lib().vla_version()


def vla_kv_bytes(cfg: vla_config, B: int, max_pos: int) -> int:
    n = lib().vla_kv_bytes(C.byref(cfg), B, max_pos)
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_workspace_bytes(cfg: vla_config, entry: int, B: int, S: int, A: int) -> int:
    n = lib().vla_workspace_bytes(C.byref(cfg), entry, B, S, A)
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_create(cfg: vla_config, weights: vla_weights) -> int:
    out = C.c_void_p()
    _check(lib().vla_create(C.byref(cfg), C.byref(weights), C.byref(out)))
    return out.value


def vla_destroy(model: int) -> None:
    _check(lib().vla_destroy(model))


def vla_prepack_bytes(cfg: vla_config) -> int:
    return lib().vla_prepack_bytes(C.byref(cfg))


def vla_prepack(model: int, buffer, stream=None) -> None:
    nbytes = 0 if buffer is None else buffer.numel() * buffer.element_size()
    _check(lib().vla_prepack(model, _ptr(buffer), nbytes, _stream(stream)))


def vla_prefill(model, kv, ws, patch, ids, B, P, T, h_last, value=None, stream=None) -> None:
    _check(lib().vla_prefill(model, _ptr(kv), _ptr(ws), ws.numel() * ws.element_size(), _ptr(patch),
                             _ptr(ids), B, P, T, _ptr(h_last), _ptr(value), _stream(stream)))


def vla_decode_actions(model, kv, ws, h_last, B, S, A, mode, slot_embed, temperature, gumbel, bins,
                       logp, entropy, logits=None, stream=None) -> None:
    _check(lib().vla_decode_actions(model, _ptr(kv), _ptr(ws), ws.numel() * ws.element_size(),
                                    _ptr(h_last), B, S, A, mode, _ptr(slot_embed), temperature,
                                    _ptr(gumbel), _ptr(bins), _ptr(logp), _ptr(entropy), _ptr(logits),
                                    _stream(stream)))


def vla_logprob_recompute(model, ws, patch, ids, bins, N, P, T, A, mode, slot_embed, temperature,
                          logp, entropy, value=None, logits=None, stream=None) -> None:
    _check(lib().vla_logprob_recompute(model, _ptr(ws), ws.numel() * ws.element_size(), _ptr(patch),
                                       _ptr(ids), _ptr(bins), N, P, T, A, mode, _ptr(slot_embed),
                                       temperature, _ptr(logp), _ptr(entropy), _ptr(value),
                                       _ptr(logits), _stream(stream)))


def vla_backward_workspace_bytes(cfg: vla_config, N: int, S: int, A: int, rank: int) -> int:
    n = lib().vla_backward_workspace_bytes(C.byref(cfg), N, S, A, rank)
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_backward_keep_workspace_bytes(cfg: vla_config, N: int, S: int, A: int, rank: int) -> int:
    n = lib().vla_backward_keep_workspace_bytes(C.byref(cfg), N, S, A, rank)
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_logprob_backward(model, ws, patch, ids, bins, coef, N, P, T, A, mode, slot_embed, temperature, rank, scale,
                         keep_activations, lora, grads, logp=None, stream=None) -> None:
    """lora[l][p] = (a, b) and grads[l][p] = (da, db): device tensors per layer and projection name."""
    n_layers = len(lora)
    la = (vla_lora_layer * n_layers)()
    ga = (vla_lora_layer_grads * n_layers)()
    for l in range(n_layers):
        for p in LORA_PROJECTIONS:
            f, g = getattr(la[l], p), getattr(ga[l], p)
            f.a, f.b = lora[l][p][0].data_ptr(), lora[l][p][1].data_ptr()
            g.da, g.db = grads[l][p][0].data_ptr(), grads[l][p][1].data_ptr()
    _check(lib().vla_logprob_backward(model, _ptr(ws), ws.numel() * ws.element_size(), _ptr(patch), _ptr(ids), _ptr(bins),
                                      _ptr(coef), N, P, T, A, mode, _ptr(slot_embed), temperature, rank, scale, int(bool(keep_activations)), la, ga,
                                      _ptr(logp), _stream(stream)))


def vla_debug_force_generic(mask: int) -> None:
    _check(lib().vla_debug_force_generic(mask))


def vla_calibration_copy(dst, src, nbytes: int, stream=None) -> None:
    _check(lib().vla_calibration_copy(_ptr(dst), _ptr(src), nbytes, _stream(stream)))


def vla_gae(rewards, values, dones, n, T, gamma, lam, adv, returns=None, stream=None) -> None:
    _check(lib().vla_gae(_ptr(rewards), _ptr(values), _ptr(dones), n, T, gamma, lam, _ptr(adv), _ptr(returns),
                         _stream(stream)))


def vla_grpo_advantage(total_reward, n_groups, G, adv, keep=None, stream=None) -> None:
    _check(lib().vla_grpo_advantage(_ptr(total_reward), n_groups, G, _ptr(adv), _ptr(keep), _stream(stream)))


def vla_policy_objective_workspace_bytes(n_traj: int) -> int:
    return lib().vla_policy_objective_workspace_bytes(n_traj)


def vla_policy_objective(logp_new, logp_old, adv, adv_per_step, mask, n_traj, T, clip_low, clip_high,
                         per_trajectory, ws, objective, per_step=None, clip_frac=None, stream=None) -> None:
    _check(lib().vla_policy_objective(_ptr(logp_new), _ptr(logp_old), _ptr(adv), int(adv_per_step), _ptr(mask),
                                      n_traj, T, clip_low, clip_high, int(per_trajectory), _ptr(ws),
                                      ws.numel() * ws.element_size(), _ptr(objective), _ptr(per_step),
                                      _ptr(clip_frac), _stream(stream)))


def vla_policy_objective_noalloc_max_traj() -> int:
    return lib().vla_policy_objective_noalloc_max_traj()


def vla_policy_objective_noalloc(logp_new, logp_old, adv, adv_per_step, mask, n_traj, T, clip_low, clip_high,
                                 per_trajectory, objective, per_step=None, clip_frac=None, stream=None) -> None:
    _check(lib().vla_policy_objective_noalloc(_ptr(logp_new), _ptr(logp_old), _ptr(adv), int(adv_per_step),
                                              _ptr(mask), n_traj, T, clip_low, clip_high, int(per_trajectory),
                                              _ptr(objective), _ptr(per_step), _ptr(clip_frac), _stream(stream)))


def vla_logp_aggregate(logp, n_out, inner, out, stream=None) -> None:
    _check(lib().vla_logp_aggregate(_ptr(logp), n_out, inner, _ptr(out), _stream(stream)))


_codes = {}


def _known() -> dict:
    """torch's types: VLA_DTYPE_* of those that storage has, and by name."""
    if not _codes:
        import torch
        _codes.update({torch.float32: VLA_DTYPE_F32, torch.bfloat16: VLA_DTYPE_BF16, "float32": torch.float32, "int32": torch.int32,
                       "float64": torch.float64})
    return _codes


def _dtype(t) -> int:
    code = _known().get(t.dtype)
    if code is None:
        raise VlaError(VLA_EDTYPE, f"{t.dtype} is neither float32 nor bfloat16")
    return code


def _want(t, kind: str, name: str, shape=None):
    """An array argument the library reads as packed values of one type: another type, shape or layout would be read wrongly."""
    if t is None:
        return None
    if t.dtype is _codes.get(kind) and (shape is None or t.shape == shape) and t.is_contiguous():          # (a call has a dozen of these: half a microsecond each)
        return t.data_ptr()
    if t.dtype is not _known()[kind] or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise VlaError(VLA_EINVAL, f"{name}: contiguous {kind}{'' if shape is None else ' ' + str(list(shape))} wanted, "
                                   f"{t.dtype} {list(t.shape)} given")
    return t.data_ptr()


def _device_of(*tensors):
    """The GPU that tensors are on; None if there are none, -1 for host memory or several."""
    found = None
    for t in tensors:
        if t is not None:
            d = t.get_device()
            found = d if found is None or found == d else -1
    return found


def _on_current_device(what, structures, tensors):
    """The library launches on the current GPU: arrays of another one, or of the host, would be read from there."""
    import torch
    here = tensors[0].get_device()
    for s in structures:
        if s.device is not None and s.device != here:
            here = -1
    for t in tensors:
        if t is not None and t.get_device() != here:
            here = -1
    if here < 0 or here != torch.cuda.current_device():
        raise VlaError(VLA_EINVAL, f"{what}: the arrays are not all on the current GPU")


def _rows_of_heads(t, heads, dim, rows, name):
    """Address and row stride of a [rows, heads, dim] view whose heads are packed within a row."""
    shape = t.shape
    if len(shape) != 3 or shape[0] != rows or shape[2] != dim or (heads is not None and shape[1] != heads):
        raise VlaError(VLA_ESHAPE, f"{name} is {list(shape)}, wanted [{rows}, {'heads' if heads is None else heads}, {dim}]")
    row, head, one = t.stride()
    if (one != 1 or (head != dim and shape[1] > 1)) and dim > 1 and t.numel():
        raise VlaError(VLA_EINVAL, f"{name}: the heads of a row are not packed (strides {t.stride()})")
    return t.data_ptr(), row if rows > 1 else shape[1] * dim


def make_paged_cache(k, v) -> vla_paged_cache:
    """``k``, ``v``: device tensors [n_pages, n_kv_heads, page_size, head_dim]."""
    if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or not k.is_contiguous() or not v.is_contiguous():
        raise VlaError(VLA_ESHAPE, "k and v are contiguous [n_pages, n_kv_heads, page_size, head_dim] tensors of one type")
    n_pages, n_kv_heads, page_size, head_dim = k.shape
    c = vla_paged_cache(k.data_ptr(), v.data_ptr(), _dtype(k), n_pages, page_size, n_kv_heads, head_dim)
    c.keep, c.device = (k, v), _device_of(k, v)
    return c


def make_paged_batch(row_start, kv_len, page_table, n_rows: int, max_rows: int, max_len: int) -> vla_paged_batch:
    """``row_start`` [n_seq + 1], ``kv_len`` [n_seq], ``page_table`` [n_seq, entries]: int32 device tensors."""
    n_seq, table = kv_len.shape[0], page_table.shape
    if len(table) != 2:
        raise VlaError(VLA_ESHAPE, f"page_table is {list(table)}, wanted [n_seq, entries]")
    b = vla_paged_batch(n_seq, n_rows, max_rows, max_len, table[1], _want(row_start, "int32", "row_start", (n_seq + 1,)),
                        _want(kv_len, "int32", "kv_len", (n_seq,)), _want(page_table, "int32", "page_table", (n_seq, table[1])))
    b.keep, b.device = (row_start, kv_len, page_table), _device_of(row_start, kv_len, page_table)
    return b


def make_rotary(inv_freq=None, interleaved=False, scale=1.0, q_gain=None, k_gain=None, eps=1e-6) -> vla_rotary:
    """``inv_freq``: fp64 device tensor [rot_dim / 2], or None for no rotation."""
    r = vla_rotary(_want(inv_freq, "float64", "inv_freq"), 0 if inv_freq is None else 2 * inv_freq.numel(), int(bool(interleaved)), scale, eps,
                   _want(q_gain, "float32", "q_gain"), _want(k_gain, "float32", "k_gain"))
    r.keep, r.device = (inv_freq, q_gain, k_gain), _device_of(inv_freq, q_gain, k_gain)
    return r


def make_paged_mask(scale: float, softcap=0.0, slopes=None, prefix_len=None, window=0, shared_len=0) -> vla_paged_mask:
    m = vla_paged_mask(scale, softcap, _want(slopes, "float32", "slopes"), _want(prefix_len, "int32", "prefix_len"), window, shared_len)
    m.keep, m.device = (slopes, prefix_len), _device_of(slopes, prefix_len)
    return m


def _append_arguments(cache, batch, rotary, q, k, v, q_out, position=None):
    d, rows = cache.head_dim, batch.n_rows
    if (q is None) != (q_out is None):
        raise VlaError(VLA_EINVAL, "paged_append: q and q_out come together")
    _, q_gain, k_gain = rotary.keep
    if q_gain is not None or k_gain is not None:
        _want(q_gain, "float32", "q_gain", (d,)), _want(k_gain, "float32", "k_gain", (d,))
    kp, ks = _rows_of_heads(k, cache.n_kv_heads, d, rows, "k")
    vp_, vs = _rows_of_heads(v, cache.n_kv_heads, d, rows, "v")
    qp = qs = op = os_ = 0
    heads = cache.n_kv_heads
    if q is not None:
        qp, qs = _rows_of_heads(q, None, d, rows, "q")
        heads = q.shape[1]
        op, os_ = _rows_of_heads(q_out, heads, d, rows, "q_out")
        if _dtype(q_out) != cache.dtype:
            raise VlaError(VLA_EDTYPE, "paged_append: q_out has the cache's type")
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise VlaError(VLA_EDTYPE, "paged_append: q, k and v have one type")
    _on_current_device("paged_append", (cache, batch, rotary), (k, v, q, q_out, position))
    return qp or None, kp, vp_, _dtype(k), heads, qs, ks, vs, op or None, os_


def vla_paged_append(cache, batch, rotary, q, k, v, q_out=None, stream=None) -> None:
    """``q`` [n_rows, n_heads, head_dim] (or None with ``q_out``), ``k``, ``v`` [n_rows, n_kv_heads, head_dim]: views with packed heads."""
    arguments = _append_arguments(cache, batch, rotary, q, k, v, q_out)
    _check(lib().vla_paged_append(C.byref(cache), C.byref(batch), C.byref(rotary), *arguments, _stream(stream)))


def vla_paged_append_at(cache, batch, rotary, position, q, k, v, q_out=None, stream=None) -> None:
    """``position`` int32 [n_rows]: of the rotation; the rest as in vla_paged_append."""
    at = _want(position, "int32", "position", (batch.n_rows,))
    arguments = _append_arguments(cache, batch, rotary, q, k, v, q_out, position)
    _check(lib().vla_paged_append_at(C.byref(cache), C.byref(batch), C.byref(rotary), at, *arguments, _stream(stream)))


def vla_paged_attention_workspace_bytes(cache, batch, mask, n_heads: int) -> int:
    n = lib().vla_paged_attention_workspace_bytes(C.byref(cache), C.byref(batch), C.byref(mask), n_heads)
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_paged_attention(cache, batch, mask, q, out, lse=None, ws=None, stream=None) -> None:
    rows = batch.n_rows
    qp, qs = _rows_of_heads(q, None, cache.head_dim, rows, "q")
    heads = q.shape[1]
    op, os_ = _rows_of_heads(out, heads, cache.head_dim, rows, "out")
    if _dtype(q) != cache.dtype or _dtype(out) != cache.dtype:
        raise VlaError(VLA_EDTYPE, "paged_attention: q and out have the cache's type")
    _want(mask.keep[0], "float32", "slopes", (heads,))
    _want(mask.keep[1], "int32", "prefix_len", (batch.n_seq,))
    _on_current_device("paged_attention", (cache, batch, mask), (q, out, lse, ws))
    _check(lib().vla_paged_attention(C.byref(cache), C.byref(batch), C.byref(mask), qp, heads, qs, op, os_,
                                     _want(lse, "float32", "lse", (rows, heads)), _ptr(ws),
                                     0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)))


def vla_forward_paged_workspace_bytes(cfg: vla_config, cache, batch, shared_len: int = 0) -> int:
    n = lib().vla_forward_paged_workspace_bytes(C.byref(cfg), C.byref(cache), C.byref(batch), shared_len)
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_forward_paged(model, cache, layer_stride: int, batch, ids, ws, h_last, patch=None, prefix_len=None, shared_len=0, logits=None, value=None, stream=None) -> None:
    """``ids`` int32 [n_rows]; ``patch`` [n_patch, hidden] in the model's type: the rows that negative ids name."""
    n, hidden = batch.n_seq, cache.n_kv_heads * cache.head_dim
    if patch is not None and (not patch.is_contiguous() or patch.dim() != 2 or patch.shape[1] != hidden or _dtype(patch) != cache.dtype):
        raise VlaError(VLA_EINVAL, f"forward_paged: patch is not contiguous [n_patch, {hidden}] of the cache's type")
    if value is not None and value.shape[:1] != (n,):
        raise VlaError(VLA_EINVAL, f"forward_paged: value is {list(value.shape)}, wanted [{n}, value_dim]")
    arrays = (_want(ids, "int32", "ids", (batch.n_rows,)), _want(prefix_len, "int32", "prefix_len", (n,)), _want(h_last, "float32", "h_last", (n, hidden)),
              _want(logits, "float32", "logits", (n, VLA_N_BINS)), _want(value, "float32", "value"))
    _on_current_device("forward_paged", (cache, batch), (ids, patch, prefix_len, ws, h_last, logits, value))
    _check(lib().vla_forward_paged(model, C.byref(cache), layer_stride, C.byref(batch), arrays[0], _ptr(patch), 0 if patch is None else patch.shape[0],
                                   arrays[1], shared_len, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), *arrays[2:], _stream(stream)))


def vla_sample_logits_workspace_bytes(n: int, vocab: int) -> int:
    size = lib().vla_sample_logits_workspace_bytes(n, vocab)
    if size == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return size


def vla_sample_logits(logits, token, temperature=None, top_k=None, top_p=None, min_p=None, u=None, logp=None, logp_kept=None, n_kept=None,
                      ws=None, stream=None) -> None:
    """``logits`` [n, vocab] (rows may be apart); one value per row in everything else."""
    if logits.dim() != 2 or (logits.numel() and logits.shape[1] > 1 and logits.stride(1) != 1):
        raise VlaError(VLA_ESHAPE, f"logits: rows of consecutive values wanted, {list(logits.shape)} with strides {logits.stride()} given")
    n, vocab = logits.shape
    f = lambda t, name: _want(t, "float32", name, (n,))
    i = lambda t, name: _want(t, "int32", name, (n,))
    settings = f(temperature, "temperature"), i(top_k, "top_k"), f(top_p, "top_p"), f(min_p, "min_p"), f(u, "u")
    outputs = i(token, "token"), f(logp, "logp"), f(logp_kept, "logp_kept"), i(n_kept, "n_kept")
    code = _dtype(logits)
    _on_current_device("sample_logits", (), (logits, temperature, top_k, top_p, min_p, u, token, logp, logp_kept, n_kept, ws))
    _check(lib().vla_sample_logits(logits.data_ptr(), code, logits.stride(0) if n > 1 else vocab, n, vocab, *settings, *outputs, _ptr(ws),
                                   0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)))


def _ws(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


def _ints(t, name, *shape):
    if t is not None and t.dtype is _codes.get("int32") and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    return _want(t, "int32", name, shape)


def _positive(n: int) -> int:
    if n == 0:
        raise VlaError(VLA_EINVAL, vla_last_error())
    return n


def vla_paged_tree(cache, batch, parent, seen, position=None, stream=None) -> None:
    """``parent`` int32 [n_rows]; ``seen`` int32 [n_rows, words] out; ``position`` int32 [n_rows] out."""
    rows = batch.n_rows
    if seen.dim() != 2:
        raise VlaError(VLA_ESHAPE, f"seen is {list(seen.shape)}, wanted [{rows}, words]")
    arrays = _ints(parent, "parent", rows), _ints(seen, "seen", rows, seen.shape[1]), seen.shape[1], _ints(position, "position", rows)
    _on_current_device("paged_tree", (cache, batch), (parent, seen, position))
    _check(lib().vla_paged_tree(C.byref(cache), C.byref(batch), *arrays, _stream(stream)))


def _attended(what, cache, batch, mask, q, out):
    """Address, heads and stride of q, address and stride of out."""
    qp, qs = _rows_of_heads(q, None, cache.head_dim, batch.n_rows, "q")
    heads = q.shape[1]
    op, os_ = _rows_of_heads(out, heads, cache.head_dim, batch.n_rows, "out")
    if _dtype(q) != cache.dtype or _dtype(out) != cache.dtype:
        raise VlaError(VLA_EDTYPE, f"{what}: q and out have the cache's type")
    return qp, heads, qs, op, os_


def vla_paged_tree_attention(cache, batch, mask, seen, q, out, lse=None, ws=None, stream=None) -> None:
    """``seen`` int32 [n_rows, words] as vla_paged_tree gives it; ``ws`` of vla_paged_attention_workspace_bytes bytes."""
    rows = batch.n_rows
    arguments = _attended("paged_tree_attention", cache, batch, mask, q, out)
    if seen.dim() != 2:
        raise VlaError(VLA_ESHAPE, f"seen is {list(seen.shape)}, wanted [{rows}, words]")
    bits, sums = _ints(seen, "seen", rows, seen.shape[1]), _want(lse, "float32", "lse", (rows, arguments[1]))
    _on_current_device("paged_tree_attention", (cache, batch, mask), (q, out, seen, lse, ws))
    _check(lib().vla_paged_tree_attention(C.byref(cache), C.byref(batch), C.byref(mask), bits, seen.shape[1], *arguments, sums, *_ws(ws),
                                          _stream(stream)))


def _in_pools(what, cache, n_layers, layer_stride):
    for pool in cache.keep if n_layers > 1 else ():
        if (pool.storage_offset() + (n_layers - 1) * layer_stride + pool.numel()) * pool.element_size() > pool.untyped_storage().nbytes():
            raise VlaError(VLA_ESHAPE, f"{what}: {n_layers} layers {layer_stride} elements apart reach beyond the pools")


def vla_paged_accept(cache, n_layers: int, layer_stride: int, batch, parent, ids, chosen, path, n_accepted, next=None, new_len=None, stream=None) -> None:
    """``parent``, ``ids``, ``chosen`` int32 [n_rows]; ``path`` int32 [n_seq, max_rows] out; ``n_accepted``, ``next``, ``new_len`` int32 [n_seq] out."""
    rows, n = batch.n_rows, batch.n_seq
    arrays = (_ints(parent, "parent", rows), _ints(ids, "ids", rows), _ints(chosen, "chosen", rows), _ints(path, "path", n, batch.max_rows),
              _ints(n_accepted, "n_accepted", n), _ints(next, "next", n), _ints(new_len, "new_len", n))
    _in_pools("paged_accept", cache, n_layers, layer_stride)
    _on_current_device("paged_accept", (cache, batch), (n_accepted, parent, ids, chosen, path, next, new_len))
    _check(lib().vla_paged_accept(C.byref(cache), n_layers, layer_stride, C.byref(batch), *arrays, _stream(stream)))


def _bounds(cache, bounds):
    if _dtype(bounds) != cache.dtype or bounds.shape != (cache.n_pages, cache.n_kv_heads, 2, cache.head_dim) or not bounds.is_contiguous():
        raise VlaError(VLA_EINVAL, f"bounds: contiguous [n_pages, n_kv_heads, 2, head_dim] of the cache's type wanted, {bounds.dtype} {list(bounds.shape)} given")
    return bounds.data_ptr()


def vla_paged_bounds(cache, batch, bounds, stream=None) -> None:
    """``bounds`` [n_pages, n_kv_heads, 2, head_dim] in the cache's type: those of the pages that hold the batch's rows are written."""
    at = _bounds(cache, bounds)
    _on_current_device("paged_bounds", (cache, batch), (bounds,))
    _check(lib().vla_paged_bounds(C.byref(cache), C.byref(batch), at, _stream(stream)))


def vla_paged_select_workspace_bytes(cache, batch) -> int:
    return _positive(lib().vla_paged_select_workspace_bytes(C.byref(cache), C.byref(batch)))


def _selected(cache, batch, selected):
    if selected.dim() != 3:
        raise VlaError(VLA_ESHAPE, f"selected is {list(selected.shape)}, wanted [{batch.n_rows}, {cache.n_kv_heads}, n_select]")
    return _ints(selected, "selected", batch.n_rows, cache.n_kv_heads, selected.shape[2])


def vla_paged_select(cache, batch, bounds, q, selected, first=1, recent=1, ws=None, stream=None) -> None:
    """``selected`` int32 [n_rows, n_kv_heads, n_select] out."""
    qp, qs = _rows_of_heads(q, None, cache.head_dim, batch.n_rows, "q")
    if _dtype(q) != cache.dtype:
        raise VlaError(VLA_EDTYPE, "paged_select: q has the cache's type")
    at, out = _bounds(cache, bounds), _selected(cache, batch, selected)
    _on_current_device("paged_select", (cache, batch), (q, bounds, selected, ws))
    _check(lib().vla_paged_select(C.byref(cache), C.byref(batch), at, qp, q.shape[1], qs, selected.shape[2], first, recent, out, *_ws(ws), _stream(stream)))


def vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, n_heads: int, n_select: int) -> int:
    return _positive(lib().vla_paged_sparse_attention_workspace_bytes(C.byref(cache), C.byref(batch), C.byref(mask), n_heads, n_select))


def vla_paged_sparse_attention(cache, batch, mask, selected, q, out, lse=None, ws=None, stream=None) -> None:
    """``selected`` int32 [n_rows, n_kv_heads, n_select]: ascending numbers of pages within the row's sequence, then -1."""
    arguments = _attended("paged_sparse_attention", cache, batch, mask, q, out)
    pages, sums = _selected(cache, batch, selected), _want(lse, "float32", "lse", (batch.n_rows, arguments[1]))
    _on_current_device("paged_sparse_attention", (cache, batch, mask), (q, out, selected, lse, ws))
    _check(lib().vla_paged_sparse_attention(C.byref(cache), C.byref(batch), C.byref(mask), pages, selected.shape[2], *arguments, sums,
                                            *_ws(ws), _stream(stream)))


def vla_paged_weights_workspace_bytes(cache, batch, mask, n_heads: int) -> int:
    return _positive(lib().vla_paged_weights_workspace_bytes(C.byref(cache), C.byref(batch), C.byref(mask), n_heads))


def _mass(cache, batch, mass, name):
    if mass.dim() != 3:
        raise VlaError(VLA_ESHAPE, f"{name} is {list(mass.shape)}, wanted [{batch.n_seq}, {cache.n_kv_heads}, positions]")
    return _want(mass, "float32", name, (batch.n_seq, cache.n_kv_heads, mass.shape[2])), mass.shape[2]


def vla_paged_weights(cache, batch, mask, q, lse, mass, ws=None, stream=None) -> None:
    """``lse`` [n_rows, n_heads] of the attention under the same mask; ``mass`` fp32 [n_seq, n_kv_heads, positions] in and out."""
    qp, qs = _rows_of_heads(q, None, cache.head_dim, batch.n_rows, "q")
    heads = q.shape[1]
    if _dtype(q) != cache.dtype:
        raise VlaError(VLA_EDTYPE, "paged_weights: q has the cache's type")
    _want(mask.keep[0], "float32", "slopes", (heads,))
    _want(mask.keep[1], "int32", "prefix_len", (batch.n_seq,))
    arrays = _want(lse, "float32", "lse", (batch.n_rows, heads)), *_mass(cache, batch, mass, "mass")
    _on_current_device("paged_weights", (cache, batch, mask), (q, lse, mass, ws))
    _check(lib().vla_paged_weights(C.byref(cache), C.byref(batch), C.byref(mask), qp, heads, qs, *arrays, *_ws(ws), _stream(stream)))


def vla_paged_evict(cache, batch, mass, first: int, recent: int, to_table, kept, mass_out, new_len=None, stream=None) -> None:
    """``kept`` int32 [n_seq, n_kv_heads, keep] out; ``to_table`` int32 [n_seq, entries]; ``mass``, ``mass_out`` fp32 [n_seq, n_kv_heads, positions]."""
    n = batch.n_seq
    if kept.dim() != 3 or to_table.dim() != 2:
        raise VlaError(VLA_ESHAPE, f"kept is {list(kept.shape)}, wanted [{n}, {cache.n_kv_heads}, keep]; to_table is {list(to_table.shape)}, wanted [{n}, entries]")
    sums, out = _mass(cache, batch, mass, "mass"), _mass(cache, batch, mass_out, "mass_out")
    keep, entries = kept.shape[2], to_table.shape[1]
    pages, which, lens = _ints(to_table, "to_table", n, entries), _ints(kept, "kept", n, cache.n_kv_heads, keep), _ints(new_len, "new_len", n)
    _on_current_device("paged_evict", (cache, batch), (mass, to_table, kept, mass_out, new_len))
    _check(lib().vla_paged_evict(C.byref(cache), C.byref(batch), *sums, keep, first, recent, pages, entries, which, *out, lens, _stream(stream)))


def make_paged_rows(position=None, seen=None, prefix_len=None, bounds=None, n_select=0, first=1, recent=1, mass=None) -> vla_paged_rows:
    """``position`` int32 [n_rows], ``seen`` int32 [n_rows, words], ``prefix_len`` int32 [n_seq], ``bounds`` [n_layers, n_pages, n_kv_heads, 2, head_dim] in the cache's type,
    ``mass`` fp32 [n_layers, n_seq, n_kv_heads, positions]."""
    if (seen is not None and seen.dim() != 2) or (bounds is not None and bounds.dim() != 5) or (mass is not None and mass.dim() != 4):
        raise VlaError(VLA_ESHAPE, "paged_rows: seen is [n_rows, words], bounds [n_layers, n_pages, n_kv_heads, 2, head_dim], mass [n_layers, n_seq, n_kv_heads, positions]")
    if bounds is not None and not bounds.is_contiguous():
        raise VlaError(VLA_EINVAL, "paged_rows: bounds is not contiguous")
    r = vla_paged_rows(_want(position, "int32", "position"), _want(seen, "int32", "seen"), _want(prefix_len, "int32", "prefix_len"), _ptr(bounds), _want(mass, "float32", "mass"),
                       0 if mass is None else mass.shape[3], 0 if seen is None else seen.shape[1], n_select, first, recent)
    r.keep, r.device = (position, seen, prefix_len, bounds, mass), _device_of(position, seen, prefix_len, bounds, mass)
    return r


def vla_forward_paged_rows_workspace_bytes(cfg: vla_config, cache, batch, rows, shared_len: int = 0) -> int:
    return _positive(lib().vla_forward_paged_rows_workspace_bytes(C.byref(cfg), C.byref(cache), C.byref(batch), C.byref(rows), shared_len))


def vla_forward_paged_rows(model, cache, layer_stride: int, n_layers: int, batch, rows, ids, ws, logits, patch=None, shared_len=0, stream=None) -> None:
    """``ids`` int32 [n_rows]; ``logits`` fp32 [n_rows, 256] out; ``n_layers``: the model's, which bounds and mass have to have."""
    n, hidden = batch.n_rows, cache.n_kv_heads * cache.head_dim
    if patch is not None and (not patch.is_contiguous() or patch.dim() != 2 or patch.shape[1] != hidden or _dtype(patch) != cache.dtype):
        raise VlaError(VLA_EINVAL, f"forward_paged_rows: patch is not contiguous [n_patch, {hidden}] of the cache's type")
    if rows.keep:
        position, seen, prefix_len, bounds, mass = rows.keep
        _ints(position, "position", n), _ints(prefix_len, "prefix_len", batch.n_seq)
        if seen is not None and seen.shape[0] != n:
            raise VlaError(VLA_ESHAPE, f"forward_paged_rows: seen is {list(seen.shape)}, wanted [{n}, words]")
        if bounds is not None and (bounds.shape != (n_layers, cache.n_pages, cache.n_kv_heads, 2, cache.head_dim) or _dtype(bounds) != cache.dtype):
            raise VlaError(VLA_ESHAPE, f"forward_paged_rows: bounds is {bounds.dtype} {list(bounds.shape)}, wanted [{n_layers}, {cache.n_pages}, {cache.n_kv_heads}, 2, {cache.head_dim}] of the cache's type")
        if mass is not None and mass.shape[:3] != (n_layers, batch.n_seq, cache.n_kv_heads):
            raise VlaError(VLA_ESHAPE, f"forward_paged_rows: mass is {list(mass.shape)}, wanted [{n_layers}, {batch.n_seq}, {cache.n_kv_heads}, positions]")
    _in_pools("forward_paged_rows", cache, n_layers, layer_stride)
    arrays = _ints(ids, "ids", n), _want(logits, "float32", "logits", (n, VLA_N_BINS))
    _on_current_device("forward_paged_rows", (cache, batch, rows), (ids, patch, ws, logits))
    _check(lib().vla_forward_paged_rows(model, C.byref(cache), layer_stride, C.byref(batch), C.byref(rows), arrays[0], _ptr(patch), 0 if patch is None else patch.shape[0], shared_len,
                                        *_ws(ws), arrays[1], _stream(stream)))


def _doubles(values):
    return (C.c_double * len(values))(*[float(v) for v in values])


def vla_pipeline_time(t_gen: float, t_sim: float, k: int, m_chunks: int) -> float:
    out = C.c_double()
    _check(lib().vla_pipeline_time(t_gen, t_sim, k, m_chunks, C.byref(out)))
    return out.value


def vla_profile_lookup(profile, batch: float) -> float:
    out = C.c_double()
    _check(lib().vla_profile_lookup(_doubles(profile), len(profile), batch, C.byref(out)))
    return out.value


def vla_auto_placement(t_gen, t_sim, n_envs: int, n_gpus: int, m_chunks: int):
    """Returns (best, candidates), each candidate a (k, n_gen, n_sim, time) tuple."""
    if len(t_gen) != len(t_sim):
        raise ValueError("t_gen and t_sim must cover the same batch sizes")
    best = vla_placement()
    cap = n_gpus
    arr = (vla_placement * cap)()
    n = C.c_int()
    _check(lib().vla_auto_placement(_doubles(t_gen), _doubles(t_sim), len(t_gen), n_envs, n_gpus, m_chunks,
                                    C.byref(best), arr, cap, C.byref(n)))
    tup = lambda c: (c.k, c.n_gen, c.n_sim, c.time)
    return tup(best), [tup(arr[i]) for i in range(min(n.value, cap))]


def make_config(shape, max_batch: int, max_seq: int, value_dim: int = 1) -> vla_config:
    """``shape`` is any object with the decoder fields (n_layers, hidden, ..., dtype "f32"/"bf16")."""
    return vla_config(shape.n_layers, shape.hidden, shape.n_heads, shape.ffn, shape.vocab, shape.n_bins,
                      VLA_DTYPE_F32 if shape.dtype == "f32" else VLA_DTYPE_BF16, shape.rms_eps,
                      shape.rope_theta, max_batch, max_seq, value_dim)


class DeviceModel:
    """Keeps device weight tensors alive and owns the library's model handle.  ``layers`` is a list
    of dicts of device tensors with the nine per-layer names of ``vla_layer_weights``."""

    def __init__(self, cfg: vla_config, embed, lm_head, final_norm, layers, value_w=None, value_b=0.0,
                 value_bias=None):
        self.cfg = cfg
        self._keep = (embed, lm_head, final_norm, layers, value_w, value_bias)
        arr = (vla_layer_weights * len(layers))()
        for a, d in zip(arr, layers):
            for name, _ in vla_layer_weights._fields_:
                setattr(a, name, d[name].data_ptr())
        self._layers = arr
        w = vla_weights(embed.data_ptr(), lm_head.data_ptr(), final_norm.data_ptr(), _ptr(value_w),
                        float(value_b), arr, _ptr(value_bias))
        self.handle = vla_create(cfg, w)

    def close(self):
        if self.handle:
            vla_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
