"""ctypes binding of libfise.so: same names as the C ABI (include/fise.h).

Argument marshalling only: torch tensors are used as device buffers (data_ptr),
every step of the path runs in the library's kernels.  There is no fallback: if
the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("FISE_LIB", os.path.join(_HERE, "libfise.so"))

FISE_F32, FISE_BF16, FISE_E4M3 = 0, 1, 2
FISE_STATS_CACHED, FISE_STATS_FRESH = 0, 1
FISE_MAX_LEVELS = 8
_lib = None
_initialized = torch.cuda.is_initialized
_raw_stream, _device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))      # absent in a build of torch without GPUs

vp, i32, f32, sz, i64 = C.c_void_p, C.c_int, C.c_float, C.c_size_t, C.c_int64


class FiseError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"fise error {code}: {msg}")
        self.code = code


class fise_conv_args(C.Structure):
    _fields_ = [("x0", vp), ("x1", vp), ("C0", i32), ("C1", i32), ("B", i32), ("H", i32), ("W", i32),
                ("w", vp), ("bias", vp), ("Cout", i32), ("ksize", i32), ("stride", i32), ("upsample", i32),
                ("gn_mean", vp), ("gn_rstd", vp), ("gn_gamma", vp), ("gn_beta", vp), ("G", i32), ("gn_silu", i32),
                ("temb", vp), ("residual", vp), ("tile_idx", vp), ("n_active", i32), ("tile", i32),
                ("y_cache", vp), ("dtype", i32), ("tile_w", i32)]


class fise_resnet_args(C.Structure):
    _fields_ = [("x0", vp), ("x1", vp), ("C0", i32), ("C1", i32), ("B", i32), ("H", i32), ("W", i32), ("Cout", i32), ("G", i32),
                ("gn1_mean", vp), ("gn1_rstd", vp), ("gn1_gamma", vp), ("gn1_beta", vp), ("conv1_w", vp), ("conv1_b", vp),
                ("temb", vp), ("temb_stride", i32),
                ("gn2_mean", vp), ("gn2_rstd", vp), ("gn2_gamma", vp), ("gn2_beta", vp), ("conv2_w", vp), ("conv2_b", vp),
                ("sc_w", vp), ("sc_b", vp), ("tile_idx", vp), ("n_active", i32), ("tile", i32),
                ("h1_cache", vp), ("out_cache", vp), ("stats_fresh", i32)]


class fise_transformer_args(C.Structure):
    _fields_ = [("x", vp), ("B", i32), ("H", i32), ("W", i32), ("C", i32), ("G", i32), ("heads", i32),
                ("gn_mean", vp), ("gn_rstd", vp), ("gn_gamma", vp), ("gn_beta", vp), ("pin_w", vp), ("pin_b", vp),
                ("ln1_g", vp), ("ln1_b", vp), ("qkv_w", vp), ("o1_w", vp), ("o1_b", vp),
                ("ln2_g", vp), ("ln2_b", vp), ("q2_w", vp), ("o2_w", vp), ("o2_b", vp),
                ("K_ctx", vp), ("Vt_ctx", vp), ("n_ctx", i32), ("n_ctx_stride", i32),
                ("ln3_g", vp), ("ln3_b", vp), ("ff1_w", vp), ("ff1_b", vp), ("ff2_w", vp), ("ff2_b", vp),
                ("pout_w", vp), ("pout_b", vp), ("K_cache", vp), ("Vt_cache", vp), ("out_cache", vp),
                ("tile_idx", vp), ("n_active", i32), ("tile", i32), ("stats_fresh", i32)]


class fise_w4_linear_args(C.Structure):
    _fields_ = [("x", vp), ("x_dtype", i32), ("x_stride", i64), ("packed", vp), ("N", i32), ("K", i32), ("group", i32),
                ("bias", vp), ("bias_dtype", i32), ("residual", vp), ("residual_stride", i64),
                ("y", vp), ("y_dtype", i32), ("y_stride", i64), ("M", i32), ("silu_in", i32)]


class fise_gated_norm_args(C.Structure):
    _fields_ = [("x", vp), ("B", i32), ("H", i32), ("W", i32), ("C", i32), ("dtype", i32), ("h", vp), ("h_is_map", i32),
                ("post_norm", i32), ("post_w", vp), ("post_b", vp), ("gate", vp), ("res_scale", f32),
                ("pre_norm", i32), ("pre_w", vp), ("pre_b", vp), ("mod_scale", vp), ("mod_shift", vp), ("mod_stride", i64), ("eps", f32),
                ("tile_idx", vp), ("n_active", i32), ("tile", i32), ("r", vp), ("y", vp), ("y_is_map", i32)]


class fise_latent_attention_args(C.Structure):
    _fields_ = [("q", vp), ("cache", vp), ("kv_len", vp), ("w_uk", vp), ("w_uv", vp), ("out", vp),
                ("B", i32), ("M", i32), ("n_keys", i32), ("cache_tokens", i64),
                ("heads", i32), ("d", i32), ("dr", i32), ("dv", i32), ("r", i32),
                ("scale", f32), ("causal", i32), ("form", i32), ("dtype", i32)]


class fise_rotary_tensor(C.Structure):
    _fields_ = [("x", vp), ("y", vp), ("heads", i32), ("d", i32), ("start", i32), ("x_batch", i64), ("x_row", i64), ("x_head", i64),
                ("y_batch", i64), ("y_row", i64), ("y_head", i64), ("x_is_map", i32), ("y_is_map", i32)]


class fise_rotary_args(C.Structure):
    _fields_ = [("t", fise_rotary_tensor * 2), ("n_tensors", i32), ("dtype", i32), ("B", i32), ("M", i32),
                ("n_axes", i32), ("axis_dim", i32 * 4), ("theta", C.c_double * 4), ("offset", C.c_double * 4),
                ("pairing", i32), ("shared_freq", i32), ("inverse", i32), ("pos", vp), ("pos_is_float", i32), ("pos_B", i32),
                ("T", i32), ("H", i32), ("W", i32), ("tile_idx", vp), ("n_active", i32), ("tile", i32)]


class fise_fp8_linear_args(C.Structure):
    _fields_ = [("x", vp), ("x_dtype", i32), ("x_stride", i64), ("x_scale", vp), ("x_scale_stride", i64),
                ("w", vp), ("w_stride", i64), ("w_scale", vp), ("M", i32), ("N", i32), ("K", i32),
                ("bias", vp), ("bias_dtype", i32), ("residual", vp), ("residual_stride", i64), ("y", vp), ("y_dtype", i32), ("y_stride", i64)]


class fise_route_args(C.Structure):
    _fields_ = [("logits", vp), ("dtype", i32), ("stride", i64), ("T", i32), ("E", i32), ("k", i32), ("score", i32), ("bias", vp),
                ("groups", i32), ("top_groups", i32), ("group_top", i32), ("renormalize", i32), ("scale", f32),
                ("ids", vp), ("weights", vp), ("offsets", vp), ("slots", vp)]


class fise_expert_mlp_args(C.Structure):
    _fields_ = [("x", vp), ("x_dtype", i32), ("x_stride", i64), ("T", i32), ("K", i32), ("ids", vp), ("weights", vp), ("offsets", vp), ("slots", vp),
                ("k", i32), ("E", i32), ("I", i32), ("N", i32), ("w_in", vp), ("w_in_scale", vp), ("w_out", vp), ("w_out_scale", vp),
                ("residual", vp), ("residual_stride", i64), ("y", vp), ("y_dtype", i32), ("y_stride", i64)]


class fise_unet_desc(C.Structure):
    _fields_ = [("in_ch", i32), ("out_ch", i32), ("base", i32), ("n_levels", i32),
                ("mults", i32 * FISE_MAX_LEVELS), ("attn", i32 * FISE_MAX_LEVELS), ("layers", i32),
                ("heads", i32), ("ctx_dim", i32), ("n_ctx", i32), ("groups", i32), ("H", i32), ("W", i32), ("B", i32)]


_SIGS = {
    "fise_last_error": (C.c_char_p, []),
    "fise_version": (i32, []),
    "fise_mask_detect": (i32, [vp, vp, i32, i32, i32, i32, i32, f32, i32, vp, vp, vp, i32, vp, vp]),
    "fise_mask_from_pixels": (i32, [vp, i32, i32, i32, vp, vp, i32, vp, vp]),
    "fise_mask_downsample": (i32, [vp, i32, i32, vp, vp]),
    "fise_otsu_workspace_bytes": (sz, []),
    "fise_otsu_mask": (i32, [vp, i32, vp, vp, vp, vp]),
    "fise_diff_accumulate": (i32, [vp, vp, i32, i32, i32, i32, i32, vp, vp]),
    "fise_apsc_block_counts": (i32, [vp, i32, i32, vp, vp]),
    "fise_apsc_select": (i32, [C.POINTER(C.c_int32), i32, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i64)]),
    "fise_mask_from_pixels_rect": (i32, [vp, i32, i32, i32, i32, vp, vp, i32, vp, vp]),
    "fise_groupnorm_stats_workspace_bytes": (sz, [i32, i32, i32, i32]),
    "fise_groupnorm_stats": (i32, [vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp, vp]),
    "fise_groupnorm_stats_static_capacity_bytes": (sz, []),
    "fise_groupnorm_stats_static": (i32, [vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp]),
    "fise_masked_groupnorm_silu": (i32, [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, i32, i32, vp, vp]),
    "fise_masked_conv_workspace_bytes": (sz, [C.POINTER(fise_conv_args)]),
    "fise_masked_conv": (i32, [C.POINTER(fise_conv_args), vp, sz, vp]),
    "fise_masked_conv3x3": (i32, [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, i32, i32, vp, vp, vp, vp, i32,
                                  vp, vp, vp, vp, sz, vp]),
    "fise_attention_active_workspace_bytes": (sz, [i32, i32, i32, i32, i32]),
    "fise_attention_active": (i32, [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, vp, vp, sz, vp]),
    "fise_context_kv_workspace_bytes": (sz, [i32, i32, i32, i32]),
    "fise_context_kv": (i32, [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, sz, vp]),
    "fise_masked_attention_workspace_bytes": (sz, [i32, i32, i32, i32]),
    "fise_masked_attention_restricted_workspace_bytes": (sz, [i32, i32, i32, i32]),
    "fise_masked_attention_restricted": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, i32, i32, vp,
                                               vp, sz, vp]),
    "fise_masked_attention": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp,
                                    i32, i32, vp, i32, i32, vp, vp, sz, vp]),
    "fise_masked_resnet_block_workspace_bytes": (sz, [C.POINTER(fise_resnet_args)]),
    "fise_masked_resnet_block": (i32, [C.POINTER(fise_resnet_args), vp, sz, vp]),
    "fise_masked_transformer_block_workspace_bytes": (sz, [C.POINTER(fise_transformer_args)]),
    "fise_masked_transformer_block": (i32, [C.POINTER(fise_transformer_args), vp, sz, vp]),
    "fise_unet_create": (i32, [C.POINTER(fise_unet_desc), C.POINTER(vp)]),
    "fise_unet_destroy": (None, [vp]),
    "fise_unet_num_tensors": (i32, [vp, i32]),
    "fise_unet_tensor_info": (i32, [vp, i32, i32, C.c_char_p, C.POINTER(i64), C.POINTER(i64)]),
    "fise_unet_weight_elems": (i64, [vp]),
    "fise_unet_cache_bytes": (sz, [vp]),
    "fise_unet_ctxkv_bytes": (sz, [vp]),
    "fise_unet_workspace_bytes": (sz, [vp, i32, i32]),
    "fise_unet_refresh_derived_workspace_bytes": (sz, [vp]),
    "fise_unet_refresh_derived": (i32, [vp, vp, vp, vp, sz, vp]),
    "fise_unet_context_kv": (i32, [vp, vp, vp, vp, vp, sz, vp]),
    "fise_unet_cache_layout_get": (i32, [vp, vp]),
    "fise_unet_desc_get": (i32, [vp, vp]),
    "fise_unet_cache_move_workspace_bytes": (sz, [vp]),
    "fise_unet_cache_move_active": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp]),
    "fise_unet_cache_move_tile_rows": (i32, [vp, vp, vp, C.POINTER(i32), i32, i32, i32, i32, vp]),
    "fise_masked_unet_step": (i32, [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, C.POINTER(i32), vp, sz, vp]),
    "fise_w4_bytes": (sz, [i32, i32, i32]),
    "fise_w4_pack": (i32, [vp, i32, vp, i32, i32, i32, vp, vp]),
    "fise_w4_unpack": (i32, [vp, i32, i32, i32, vp, i32, vp]),
    "fise_w4_linear": (i32, [C.POINTER(fise_w4_linear_args), vp]),
    "fise_masked_gated_norm": (i32, [C.POINTER(fise_gated_norm_args), vp]),
    "fise_latent_attention_workspace_bytes": (sz, [C.POINTER(fise_latent_attention_args)]),
    "fise_latent_attention": (i32, [C.POINTER(fise_latent_attention_args), vp, sz, vp]),
    "fise_rotary": (i32, [C.POINTER(fise_rotary_args), vp]),
    "fise_fp8_quantize": (i32, [vp, i32, i64, i32, i32, i32, vp, i64, vp, i64, vp]),
    "fise_fp8_linear_workspace_bytes": (sz, [C.POINTER(fise_fp8_linear_args)]),
    "fise_fp8_linear": (i32, [C.POINTER(fise_fp8_linear_args), vp, sz, vp]),
    "fise_route_experts_workspace_bytes": (sz, [C.POINTER(fise_route_args)]),
    "fise_route_experts": (i32, [C.POINTER(fise_route_args), vp, sz, vp]),
    "fise_expert_mlp_workspace_bytes": (sz, [C.POINTER(fise_expert_mlp_args)]),
    "fise_expert_mlp": (i32, [C.POINTER(fise_expert_mlp_args), vp, sz, vp]),
    "fise_profile_enable": (i32, [i32]),
    "fise_profile_calibrate": (i32, [i32, vp]),
    "fise_calibrate_peaks": (i32, [vp, sz, C.POINTER(C.c_double), C.POINTER(C.c_double), vp]),
    "fise_profile_read": (i32, [i32, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(i32)]),
    "fise_unet_num_modules": (i32, [vp]),
    "fise_unet_module_name": (i32, [vp, i32, C.c_char_p]),
    "fise_masked_unet_modules": (i32, [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, C.POINTER(i32), i32, i32, vp, sz, vp]),
}
EXPORTS = tuple(_SIGS)


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2305_17423_amd.build` "
                                    "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _p(t):
    """Device (or host) address of a tensor, None -> NULL."""
    if t is None:
        return None
    try:
        return t.data_ptr()
    except AttributeError:                  # a bare number here would reach a kernel as an address
        raise TypeError(f"expected a tensor or None where a buffer is passed, got {type(t).__name__}") from None


def _dt(t):
    d = t.dtype
    if d is torch.bfloat16:
        return FISE_BF16
    if d is torch.float32:
        return FISE_F32
    raise TypeError(f"unsupported dtype {d}")


def _stream(stream):
    if stream is None:
        # the handle alone: the Stream object around it costs 2.9 us a call, more than the launch (a mask detection 6.9 -> 4 us), and
        # torch.cuda.current_device() twice the call that it ends in
        if _initialized():
            return _raw_stream(_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _ck(code):
    if code != 0:
        raise FiseError(code, lib().fise_last_error().decode())


def fise_last_error():
    return lib().fise_last_error().decode()


def fise_version():
    return lib().fise_version()


# --------------------------------------------------------------------------- masks
def fise_mask_detect(cached, fresh, threshold, tile, pix_mask, tile_mask, tile_idx, n_active, stream=None):
    B, H, W, Cc = cached.shape
    _ck(lib().fise_mask_detect(_p(cached), _p(fresh), _dt(cached), B, H, W, Cc, threshold, tile, _p(pix_mask),
                               _p(tile_mask), _p(tile_idx), tile_idx.numel(), _p(n_active), _stream(stream)))


def fise_mask_from_pixels(pix_mask, tile, tile_mask, tile_idx, n_active, stream=None):
    H, W = pix_mask.shape
    _ck(lib().fise_mask_from_pixels(_p(pix_mask), H, W, tile, _p(tile_mask), _p(tile_idx), tile_idx.numel(),
                                    _p(n_active), _stream(stream)))


def fise_mask_from_pixels_rect(pix_mask, tile_h, tile_w, tile_mask, tile_idx, n_active, stream=None):
    H, W = pix_mask.shape
    _ck(lib().fise_mask_from_pixels_rect(_p(pix_mask), H, W, tile_h, tile_w, _p(tile_mask), _p(tile_idx), tile_idx.numel(),
                                         _p(n_active), _stream(stream)))


def fise_mask_downsample(mask, out, stream=None):
    H, W = mask.shape
    _ck(lib().fise_mask_downsample(_p(mask), H, W, _p(out), _stream(stream)))


def fise_otsu_workspace_bytes():
    return lib().fise_otsu_workspace_bytes()


def fise_otsu_mask(diff, eps_out, pix_mask, workspace, stream=None):
    _ck(lib().fise_otsu_mask(_p(diff), diff.numel(), _p(eps_out), _p(pix_mask), _p(workspace), _stream(stream)))


def fise_diff_accumulate(cached, fresh, diff_acc, stream=None):
    B, H, W, Cc = cached.shape
    _ck(lib().fise_diff_accumulate(_p(cached), _p(fresh), _dt(cached), B, H, W, Cc, _p(diff_acc), _stream(stream)))


def fise_apsc_block_counts(pix_mask, counts, stream=None):
    H, W = pix_mask.shape
    _ck(lib().fise_apsc_block_counts(_p(pix_mask), H, W, _p(counts), _stream(stream)))


def fise_apsc_select(counts_host, kh=3, kw=3):
    """(h, w, cost) from the 25 block counts (a host sequence of ints)."""
    arr = (C.c_int32 * 25)(*[int(v) for v in counts_host])
    h, w, cost = i32(), i32(), i64()
    _ck(lib().fise_apsc_select(arr, kh, kw, C.byref(h), C.byref(w), C.byref(cost)))
    return h.value, w.value, cost.value


# --------------------------------------------------------------------------- normalisation
def fise_groupnorm_stats_workspace_bytes(B, H, W, Cc):
    return lib().fise_groupnorm_stats_workspace_bytes(B, H, W, Cc)


def fise_groupnorm_stats(x, x1, G, eps, mean, rstd, workspace, stream=None):
    B, H, W, C0 = x.shape
    C1 = 0 if x1 is None else x1.shape[-1]
    _ck(lib().fise_groupnorm_stats(_p(x), _p(x1), _dt(x), B, H, W, C0, C1, G, eps, _p(mean), _p(rstd), _p(workspace),
                                   _stream(stream)))


def fise_groupnorm_stats_static_capacity_bytes():
    return lib().fise_groupnorm_stats_static_capacity_bytes()


def fise_groupnorm_stats_static(x, x1, G, eps, mean, rstd, stream=None):
    B, H, W, C0 = x.shape
    C1 = 0 if x1 is None else x1.shape[-1]
    _ck(lib().fise_groupnorm_stats_static(_p(x), _p(x1), _dt(x), B, H, W, C0, C1, G, eps, _p(mean), _p(rstd), _stream(stream)))


def fise_masked_groupnorm_silu(x, mean, rstd, gamma, beta, G, tile_idx, n_active, tile, y_cache, stream=None):
    B, H, W, Cc = x.shape
    _ck(lib().fise_masked_groupnorm_silu(_p(x), _p(mean), _p(rstd), _p(gamma), _p(beta), _dt(x), B, H, W, Cc, G,
                                         _p(tile_idx), n_active, tile, _p(y_cache), _stream(stream)))


# --------------------------------------------------------------------------- convolution
def conv_args(x0, w, bias, tile_idx, n_active, tile, y_cache, x1=None, ksize=3, stride=1, upsample=0, gn=None,
              gn_silu=1, temb=None, residual=None, tile_w=0):
    B, H, W, C0 = x0.shape
    a = fise_conv_args()
    a.x0, a.x1, a.C0, a.C1 = _p(x0), _p(x1), C0, (0 if x1 is None else x1.shape[-1])
    a.B, a.H, a.W = B, H, W
    a.w, a.bias, a.Cout, a.ksize, a.stride, a.upsample = _p(w), _p(bias), w.shape[0], ksize, stride, upsample
    if gn is not None:
        a.gn_mean, a.gn_rstd, a.gn_gamma, a.gn_beta, a.G = _p(gn["mean"]), _p(gn["rstd"]), _p(gn["gamma"]), _p(gn["beta"]), gn["groups"]
    a.gn_silu = gn_silu
    a.temb, a.residual, a.tile_idx, a.n_active, a.tile = _p(temb), _p(residual), _p(tile_idx), n_active, tile
    a.y_cache, a.dtype, a.tile_w = _p(y_cache), _dt(x0), tile_w
    return a


def fise_masked_conv_workspace_bytes(args):
    return lib().fise_masked_conv_workspace_bytes(C.byref(args))


def fise_masked_conv(args, workspace=None, stream=None):
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_masked_conv(C.byref(args), _p(workspace), nbytes, _stream(stream)))


def fise_masked_conv3x3(x, w, bias, stride, tile_idx, n_active, tile, y_cache, gn=None, temb=None, residual=None,
                        workspace=None, stream=None):
    B, H, W, Cin = x.shape
    g = gn or {}
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_masked_conv3x3(_p(x), _p(w), _p(bias), _dt(x), B, H, W, Cin, w.shape[0], stride, _p(tile_idx),
                                  n_active, tile, _p(g.get("mean")), _p(g.get("rstd")), _p(g.get("gamma")),
                                  _p(g.get("beta")), g.get("groups", 0), _p(temb), _p(residual), _p(y_cache),
                                  _p(workspace), nbytes, _stream(stream)))


# --------------------------------------------------------------------------- attention
def fise_attention_active_workspace_bytes(B, M, n_keys, Cc, heads):
    return lib().fise_attention_active_workspace_bytes(B, M, n_keys, Cc, heads)


def fise_attention_active(q, K, Vt, heads, scale, out, n_keys=None, workspace=None, stream=None):
    B, M, Cc = q.shape
    n_keys = K.shape[1] if n_keys is None else n_keys
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_attention_active(_p(q), _p(K), _p(Vt), _dt(q), B, M, n_keys, Vt.shape[2], Cc, heads, scale, _p(out),
                                    _p(workspace), nbytes, _stream(stream)))


def fise_context_kv(ctx, Wk, Wv, K_ctx, Vt_ctx, stream=None):
    B, n_ctx, Dc = ctx.shape
    _ck(lib().fise_context_kv(_p(ctx), _p(Wk), _p(Wv), _dt(ctx), B, n_ctx, Dc, Wk.shape[0], Vt_ctx.shape[2], _p(K_ctx),
                              _p(Vt_ctx), None, 0, _stream(stream)))


def fise_masked_attention_restricted_workspace_bytes(B, Cc, n_active, tile):
    return lib().fise_masked_attention_restricted_workspace_bytes(B, Cc, n_active, tile)


def fise_masked_attention_restricted(x, ln_gamma, ln_beta, Wq, Wk, Wv, Wo, bo, heads, tile_idx, n_active, tile, y_cache,
                                     workspace, stream=None):
    B, H, W, Cc = x.shape
    _ck(lib().fise_masked_attention_restricted(_p(x), _p(ln_gamma), _p(ln_beta), _p(Wq), _p(Wk), _p(Wv), _p(Wo), _p(bo), _dt(x), B,
                                               H, W, Cc, heads, _p(tile_idx), n_active, tile, _p(y_cache), _p(workspace),
                                               workspace.numel() * workspace.element_size(), _stream(stream)))


def fise_masked_attention_workspace_bytes(B, Cc, n_active, tile):
    return lib().fise_masked_attention_workspace_bytes(B, Cc, n_active, tile)


def fise_masked_attention(x, ln_gamma, ln_beta, Wq, Wk, Wv, Wo, bo, heads, K_cache, Vt_cache, K_ctx, Vt_ctx, n_ctx,
                          tile_idx, n_active, tile, y_cache, workspace, stream=None):
    B, H, W, Cc = x.shape
    nstride = 0 if Vt_ctx is None else Vt_ctx.shape[2]
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_masked_attention(_p(x), _p(ln_gamma), _p(ln_beta), _p(Wq), _p(Wk), _p(Wv), _p(Wo), _p(bo), _dt(x), B,
                                    H, W, Cc, heads, _p(K_cache), _p(Vt_cache), _p(K_ctx), _p(Vt_ctx), n_ctx, nstride,
                                    _p(tile_idx), n_active, tile, _p(y_cache), _p(workspace), nbytes, _stream(stream)))


# --------------------------------------------------------------------------- modules
def fill_args(struct_type, keep, **kw):
    """A ctypes argument struct from keyword values; tensors become addresses and are appended
    to `keep` so they outlive the (asynchronous) call.  An int in a pointer field is taken as an
    address read from another argument struct."""
    a = struct_type()
    types = dict(struct_type._fields_)
    for k, v in kw.items():
        if types[k] is vp:
            if hasattr(v, "data_ptr"):
                keep.append(v)
            setattr(a, k, v if isinstance(v, int) else _p(v))
        else:
            setattr(a, k, int(v))
    return a


def fise_masked_resnet_block_workspace_bytes(args):
    return lib().fise_masked_resnet_block_workspace_bytes(C.byref(args))


def fise_masked_resnet_block(args, workspace, stream=None):
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_masked_resnet_block(C.byref(args), _p(workspace), nbytes, _stream(stream)))


def fise_masked_transformer_block_workspace_bytes(args):
    return lib().fise_masked_transformer_block_workspace_bytes(C.byref(args))


def fise_masked_transformer_block(args, workspace, stream=None):
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_masked_transformer_block(C.byref(args), _p(workspace), nbytes, _stream(stream)))


# --------------------------------------------------------------------------- transformer denoisers
_NOTHING = 256


def _pn(t):
    """Address of a tensor that an empty selection leaves without elements, and so without an address of its own: one that is not NULL, which the library takes for a
    missing buffer, and which nothing is read from or written to."""
    return _NOTHING if t is not None and t.numel() == 0 else _p(t)


def _like(name, t, shape, dtype):
    """A tensor of that shape and one of those types, contiguous in memory."""
    if tuple(t.shape) != tuple(shape) or t.dtype not in dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor {tuple(shape)} of {dtype}, got {tuple(t.shape)} of {t.dtype} with strides {t.stride()}")


def _rows_of(name, t, shape):
    """Distance between the rows of a two-dimensional tensor whose columns are neighbours."""
    if tuple(t.shape) != tuple(shape) or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}: expected rows {tuple(shape)} with neighbouring columns, got {tuple(t.shape)} with strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def fise_w4_bytes(N, K, group):
    n = lib().fise_w4_bytes(N, K, group)
    if n == 0:
        raise FiseError(-2, fise_last_error())
    return n


def _packed_size(packed, N, K, group):
    if not packed.is_contiguous() or packed.numel() * packed.element_size() < fise_w4_bytes(N, K, group):
        raise ValueError(f"packed weights of {N} x {K} in groups of {group} take {fise_w4_bytes(N, K, group)} bytes side by side")


def fise_w4_pack(w, packed, group, scale=None, stream=None):
    N, K = w.shape
    _like("w", w, (N, K), (torch.float32, torch.bfloat16))
    _packed_size(packed, N, K, group)
    if scale is not None:
        _like("scale", scale, (N, -(-K // group)), (torch.bfloat16,))
    _ck(lib().fise_w4_pack(_p(w), _dt(w), _p(scale), N, K, group, _p(packed), _stream(stream)))


def fise_w4_unpack(packed, w, group, stream=None):
    N, K = w.shape
    _like("w", w, (N, K), (torch.float32, torch.bfloat16))
    _packed_size(packed, N, K, group)
    _ck(lib().fise_w4_unpack(_p(packed), N, K, group, _p(w), _dt(w), _stream(stream)))


def w4_linear_args(x, packed, group, y, bias=None, residual=None, silu_in=False):
    """Arguments of fise_w4_linear for x [M, K] and y [M, N], rows any distance apart; they keep the tensors alive."""
    M, K = x.shape
    N = y.shape[1]
    _packed_size(packed, N, K, group)
    a = fise_w4_linear_args()
    a.x, a.x_dtype, a.x_stride = _pn(x), _dt(x), _rows_of("x", x, (M, K))
    if M == 1:
        a.x_stride = (K + 7) // 8 * 8
    a.packed, a.N, a.K, a.group = _p(packed), N, K, group
    if bias is not None:
        _like("bias", bias, (N,), (torch.float32, torch.bfloat16))
        a.bias, a.bias_dtype = _p(bias), _dt(bias)
    a.y, a.y_dtype, a.y_stride = _pn(y), _dt(y), _rows_of("y", y, (M, N))
    if residual is not None:
        if residual.dtype != y.dtype:
            raise ValueError(f"residual is {residual.dtype}, y {y.dtype}")
        a.residual, a.residual_stride = _pn(residual), _rows_of("residual", residual, (M, N))
    a.M, a.silu_in = M, int(bool(silu_in))
    a.keep = (x, packed, bias, residual, y)
    return a


def fise_w4_linear(args, stream=None):
    _ck(lib().fise_w4_linear(C.byref(args), _stream(stream)))


FISE_NORM_NONE, FISE_NORM_LAYER, FISE_NORM_RMS = 0, 1, 2
_NORMS = {"none": FISE_NORM_NONE, "layer": FISE_NORM_LAYER, "rms": FISE_NORM_RMS}


def gated_norm_args(x, h=None, post="none", post_w=None, post_b=None, gate=None, res_scale=1.0, pre="none", pre_w=None, pre_b=None,
                    mod_scale=None, mod_shift=None, eps=1e-5, tile_idx=None, n_active=0, tile=0, r=None, y=None):
    """Arguments of fise_masked_gated_norm; they keep the tensors alive.  x and r are maps [B, H, W, C]; h and y maps too, or compact rows [B, M, C].
    gate, mod_scale, mod_shift: float [B, C], with the same distance between their rows."""
    B, H, W, Cc = x.shape
    M = n_active * tile * tile if tile else H * W
    types = (x.dtype,)
    a = fise_gated_norm_args()
    _like("x", x, (B, H, W, Cc), (torch.float32, torch.bfloat16))
    a.x, a.B, a.H, a.W, a.C, a.dtype = _p(x), B, H, W, Cc, _dt(x)
    for name, t in (("h", h), ("y", y)):
        if t is not None:
            _like(name, t, (B, H, W, Cc) if t.dim() == 4 else (B, M, Cc), types)
            setattr(a, name, _pn(t))
            setattr(a, name + "_is_map", int(t.dim() == 4))
    if r is not None:
        _like("r", r, (B, H, W, Cc), types)
        a.r = _p(r)
    for name, t in (("post_w", post_w), ("post_b", post_b), ("pre_w", pre_w), ("pre_b", pre_b)):
        if t is not None:
            _like(name, t, (Cc,), types)
            setattr(a, name, _p(t))
    strides = set()
    for name, t in (("gate", gate), ("mod_scale", mod_scale), ("mod_shift", mod_shift)):
        if t is not None:
            if t.dtype != torch.float32:
                raise ValueError(f"{name}: float is what modulations are, got {t.dtype}")
            apart = _rows_of(name, t, (B, Cc))
            strides.add(apart if B > 1 else 0)
            setattr(a, name, _p(t))
    if len(strides) > 1:
        raise ValueError(f"gate, mod_scale and mod_shift: rows {sorted(strides)} apart, they share one distance")
    a.mod_stride = strides.pop() if strides else 0
    if tile_idx is not None and (tile_idx.dtype != torch.int32 or not tile_idx.is_contiguous() or tile_idx.numel() < n_active):
        raise ValueError(f"tile_idx: expected {n_active} int32 numbers")
    a.post_norm, a.pre_norm, a.res_scale, a.eps = _NORMS[post], _NORMS[pre], res_scale, eps
    a.tile_idx, a.n_active, a.tile = _p(tile_idx), n_active, tile
    a.keep = (x, h, post_w, post_b, gate, pre_w, pre_b, mod_scale, mod_shift, tile_idx, r, y)
    return a


def fise_masked_gated_norm(args, stream=None):
    _ck(lib().fise_masked_gated_norm(C.byref(args), _stream(stream)))


FISE_LATENT_AUTO, FISE_LATENT_ABSORBED, FISE_LATENT_EXPANDED = 0, 1, 2


def latent_attention_args(q, cache, w_uk, w_uv, out, scale, kv_len=None, n_keys=None, causal=False, form=FISE_LATENT_AUTO):
    """Arguments of fise_latent_attention; they keep the tensors alive.  q [B, M, heads, d + dr], cache [B, cache_tokens, r + dr] or a map
    [B, H, W, r + dr], w_uk [heads, d, r], w_uv [heads, dv, r], out [B, M, heads * dv]; kv_len: int32 [B] on the device."""
    B, M, heads, width = q.shape
    d, r = w_uk.shape[1:]
    dv, dr, bf = w_uv.shape[1], width - d, (torch.bfloat16,)
    tokens = cache.numel() // max(B * (r + dr), 1)
    for name, t, shape in (("q", q, (B, M, heads, d + dr)), ("w_uk", w_uk, (heads, d, r)), ("w_uv", w_uv, (heads, dv, r)), ("out", out, (B, M, heads * dv)),
                           ("cache", cache, (B, *cache.shape[1:-1], r + dr))):
        _like(name, t, shape, bf)
    if kv_len is not None:
        _like("kv_len", kv_len, (B,), (torch.int32,))
    a = fise_latent_attention_args()
    a.q, a.cache, a.kv_len, a.w_uk, a.w_uv, a.out = _pn(q), _pn(cache), _p(kv_len), _p(w_uk), _p(w_uv), _pn(out)
    a.B, a.M, a.n_keys, a.cache_tokens = B, M, tokens if n_keys is None else n_keys, tokens
    a.heads, a.d, a.dr, a.dv, a.r = heads, d, dr, dv, r
    a.scale, a.causal, a.form, a.dtype = scale, int(bool(causal)), form, FISE_BF16
    a.keep = (q, cache, kv_len, w_uk, w_uv, out)
    return a


def fise_latent_attention_workspace_bytes(args):
    return lib().fise_latent_attention_workspace_bytes(C.byref(args))


def fise_latent_attention(args, workspace, stream=None):
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace: its bytes must lie side by side")
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _ck(lib().fise_latent_attention(C.byref(args), _p(workspace), nbytes, _stream(stream)))


# --------------------------------------------------------------------------- transformer denoisers with experts
_CODES = (torch.uint8, torch.float8_e4m3fn)


def _one_device(args, *tensors):
    """The call's tensors, kept alive; all on one device, which is the current one when the call is made."""
    args.keep = tensors
    where = {t.device for t in tensors if t is not None}
    if len(where) > 1:
        raise ValueError(f"tensors of one call on {sorted(map(str, where))}")
    args.device = where.pop()


def _here(args, workspace=None):
    """Address and size of the workspace, once the call's tensors are known to be where it is made."""
    d = args.device
    if d.type != "cuda" or (workspace is not None and workspace.device != d):
        raise ValueError(f"tensors on {d}, workspace on {None if workspace is None else workspace.device}: a call works on one GPU")
    if d.index != (_device() if _initialized() else torch.cuda.current_device()):
        raise ValueError(f"tensors on {d}, which is not the current device")
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous():
        raise ValueError("workspace: its bytes must lie side by side")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


FISE_ROTARY_ADJACENT, FISE_ROTARY_HALVES, FISE_ROTARY_AXIS_HALVES = 0, 1, 2
_PAIRINGS = {"adjacent": FISE_ROTARY_ADJACENT, "halves": FISE_ROTARY_HALVES, "axis_halves": FISE_ROTARY_AXIS_HALVES}


def rotary_tensor(x, y=None, start=0, x_is_map=False, y_is_map=False):
    """One tensor of a fise_rotary call: x and y [B, rows, heads, d], neighbouring channels, any other strides; y None: in place.  The pairs begin at channel `start`."""
    return (x, x if y is None else y, start, bool(x_is_map), bool(x_is_map if y is None else y_is_map))


def rotary_args(tensors, axes, theta, pos=None, offset=None, grid=(0, 0, 0), tile_idx=None, n_active=0, tile=0, pairing="adjacent", shared_frequencies=False, inverse=False):
    """Arguments of fise_rotary for one or two rotary_tensor()s; they keep the tensors alive.  axes: channels of each; theta: one number or one an axis;
    pos: int32 or float [B or 1, M, axes], or None for the places on grid (T, H, W)."""
    if not 1 <= len(tensors) <= 2 or not 1 <= len(axes) <= 4:
        raise ValueError(f"{len(tensors)} tensors of {len(axes)} axes: 1 or 2 of 1 to 4")
    theta = [float(theta)] * len(axes) if isinstance(theta, (int, float)) else [float(v) for v in theta]
    offset = [0.0] * len(axes) if offset is None else [float(v) for v in offset]
    if len(theta) != len(axes) or len(offset) != len(axes):
        raise ValueError(f"{len(axes)} axes, theta for {len(theta)}, offsets for {len(offset)}")
    T, H, W = grid
    tokens = T * H * W
    B = tensors[0][0].shape[0]
    M = n_active * tile * tile if tile else tokens if pos is None else pos.shape[1]
    a = fise_rotary_args()
    for i, (x, y, start, x_map, y_map) in enumerate(tensors):
        if x.dim() != 4 or x.shape != (B, tokens if x_map else M, *x.shape[2:]) or y.shape != (B, tokens if y_map else M, *x.shape[2:]) or x.dtype != y.dtype or x.dtype != tensors[0][0].dtype:
            raise ValueError(f"tensor {i}: {tuple(x.shape)} of {x.dtype} to {tuple(y.shape)} of {y.dtype}, {B} elements of {M} rows (a map's: {tokens}) expected")
        t = a.t[i]
        for v in (x, y):
            if v.shape[3] > 1 and v.stride(3) != 1:
                raise ValueError(f"tensor {i}: channels must be neighbours, strides {v.stride()}")
        if any(y.shape[j] > 1 and y.stride(j) == 0 for j in range(3)):
            raise ValueError(f"tensor {i}: an output that repeats itself, strides {y.stride()}")
        t.x, t.y, t.heads, t.d, t.start, t.x_is_map, t.y_is_map = _pn(x), _pn(y), x.shape[2], x.shape[3], start, int(x_map), int(y_map)
        for side, v in (("x", x), ("y", y)):
            for n, name in enumerate(("_batch", "_row", "_head")):
                setattr(t, side + name, v.stride(n) if v.shape[n] > 1 else 0)      # (a stride that nothing steps by may be any number)
    if pos is not None:
        if pos.dtype not in (torch.int32, torch.float32) or pos.dim() != 3 or pos.shape[0] not in (1, B) or pos.shape[1:] != (M, len(axes)) or not pos.is_contiguous():
            raise ValueError(f"pos: expected contiguous int32 or float [{B} or 1, {M}, {len(axes)}], got {tuple(pos.shape)} of {pos.dtype} with strides {pos.stride()}")
        a.pos, a.pos_is_float, a.pos_B = _pn(pos), int(pos.dtype == torch.float32), pos.shape[0]
    if tile_idx is not None and (tile_idx.dtype != torch.int32 or not tile_idx.is_contiguous() or tile_idx.numel() < n_active):
        raise ValueError(f"tile_idx: expected {n_active} int32 numbers")
    a.n_tensors, a.dtype, a.B, a.M, a.n_axes = len(tensors), _dt(tensors[0][0]), B, M, len(axes)
    for j in range(len(axes)):
        a.axis_dim[j], a.theta[j], a.offset[j] = axes[j], theta[j], offset[j]
    a.pairing, a.shared_freq, a.inverse = _PAIRINGS[pairing], int(bool(shared_frequencies)), int(bool(inverse))
    a.T, a.H, a.W, a.tile_idx, a.n_active, a.tile = T, H, W, _p(tile_idx), n_active, tile
    _one_device(a, pos, tile_idx, *(v for t in tensors for v in t[:2]))
    return a


def fise_rotary(args, stream=None):
    _here(args)
    _ck(lib().fise_rotary(C.byref(args), _stream(stream)))


def fise_fp8_quantize(x, codes, scale, block_rows=1, stream=None):
    """x [M, K] -> codes [M, K] (uint8 or float8_e4m3fn) and scale [ceil(K / 128), M] (block_rows 1) or [ceil(M / 128), ceil(K / 128)] (block_rows 128)."""
    M, K = x.shape
    blocks = -(-K // 128)
    if codes.dtype not in _CODES:
        raise ValueError(f"codes: {codes.dtype}, expected one of {_CODES}")
    if scale.dtype != torch.float32:
        raise ValueError(f"scale: {scale.dtype}, expected float")
    a = fise_fp8_linear_args()
    _one_device(a, x, codes, scale)
    x_stride, code_stride = _rows_of("x", x, (M, K)), _rows_of("codes", codes, (M, K))
    scale_stride = _rows_of("scale", scale, (blocks, M) if block_rows == 1 else (-(-M // 128), blocks))
    if M == 1:
        x_stride = code_stride = -(-K // 16) * 16
    _here(a)
    _ck(lib().fise_fp8_quantize(_pn(x), _dt(x), x_stride, M, K, block_rows, _pn(codes), code_stride, _pn(scale), scale_stride, _stream(stream)))


def fp8_linear_args(x, w, w_scale, y, x_scale=None, bias=None, residual=None):
    """Arguments of fise_fp8_linear for x [M, K] (float, bf16, or codes with x_scale [ceil(K / 128), M]), w [N, K] codes with w_scale [ceil(N / 128), ceil(K / 128)] and
    y [M, N]; they keep the tensors alive."""
    M, K = x.shape
    N = w.shape[0]
    a = fise_fp8_linear_args()
    if w.dtype not in _CODES or (x_scale is not None and x.dtype not in _CODES):
        raise ValueError(f"codes: w {w.dtype}, x {x.dtype}, expected one of {_CODES}")
    a.x, a.x_dtype, a.x_stride = _pn(x), FISE_E4M3 if x_scale is not None else _dt(x), _rows_of("x", x, (M, K))
    if M == 1:
        a.x_stride = -(-K // 16) * 16
    if x_scale is not None:
        if x_scale.dtype != torch.float32:
            raise ValueError(f"x_scale: {x_scale.dtype}, expected float")
        a.x_scale, a.x_scale_stride = _pn(x_scale), _rows_of("x_scale", x_scale, (-(-K // 128), M))
    a.w, a.w_stride = _p(w), _rows_of("w", w, (N, K))
    if N == 1:
        a.w_stride = -(-K // 16) * 16
    _like("w_scale", w_scale, (-(-N // 128), -(-K // 128)), (torch.float32,))
    a.w_scale, a.M, a.N, a.K = _p(w_scale), M, N, K
    if bias is not None:
        _like("bias", bias, (N,), (torch.float32, torch.bfloat16))
        a.bias, a.bias_dtype = _p(bias), _dt(bias)
    a.y, a.y_dtype, a.y_stride = _pn(y), _dt(y), _rows_of("y", y, (M, N))
    if residual is not None:
        if residual.dtype != y.dtype:
            raise ValueError(f"residual is {residual.dtype}, y {y.dtype}")
        a.residual, a.residual_stride = _pn(residual), _rows_of("residual", residual, (M, N))
    _one_device(a, x, x_scale, w, w_scale, bias, residual, y)
    return a


def fise_fp8_linear_workspace_bytes(args):
    return lib().fise_fp8_linear_workspace_bytes(C.byref(args))


def fise_fp8_linear(args, workspace=None, stream=None):
    ws, nbytes = _here(args, workspace)
    _ck(lib().fise_fp8_linear(C.byref(args), ws, nbytes, _stream(stream)))


FISE_SCORE_SOFTMAX, FISE_SCORE_SIGMOID = 0, 1
_SCORES = {"softmax": FISE_SCORE_SOFTMAX, "sigmoid": FISE_SCORE_SIGMOID}


def route_args(logits, ids, weights, offsets=None, slots=None, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renormalize=True, scale=1.0):
    """Arguments of fise_route_experts for logits [T, E], ids int32 and weights float [T, k], offsets int32 [E + 1] and slots int32 [T * k]; they keep the tensors alive."""
    T, E = logits.shape
    k = ids.shape[1]
    a = fise_route_args()
    a.logits, a.dtype, a.stride = _pn(logits), _dt(logits), _rows_of("logits", logits, (T, E))
    _like("ids", ids, (T, k), (torch.int32,))
    _like("weights", weights, (T, k), (torch.float32,))
    if (offsets is None) != (slots is None):
        raise ValueError("offsets and slots are given together")
    if offsets is not None:
        _like("offsets", offsets, (E + 1,), (torch.int32,))
        _like("slots", slots, (T * k,), (torch.int32,))
        a.offsets, a.slots = _p(offsets), _pn(slots)
    if bias is not None:
        _like("bias", bias, (E,), (torch.float32,))
        a.bias = _p(bias)
    a.ids, a.weights = _pn(ids), _pn(weights)
    a.T, a.E, a.k, a.score, a.groups, a.top_groups, a.group_top = T, E, k, _SCORES[score], groups, top_groups, group_top
    a.renormalize, a.scale = int(bool(renormalize)), scale
    _one_device(a, logits, bias, ids, weights, offsets, slots)
    return a


def fise_route_experts_workspace_bytes(args):
    return lib().fise_route_experts_workspace_bytes(C.byref(args))


def fise_route_experts(args, workspace=None, stream=None):
    ws, nbytes = _here(args, workspace)
    _ck(lib().fise_route_experts(C.byref(args), ws, nbytes, _stream(stream)))


def expert_mlp_args(x, ids, weights, offsets, slots, w_in, w_in_scale, w_out, w_out_scale, y, residual=None):
    """Arguments of fise_expert_mlp for x [T, K], what fise_route_experts left, codes w_in [E, 2, I, K] and w_out [E, N, I] with their scales, y [T, N]; they keep the
    tensors alive."""
    T, K = x.shape
    E, _, I, _ = w_in.shape
    N, k = w_out.shape[1], ids.shape[1]
    blocks = lambda n: -(-n // 128)
    a = fise_expert_mlp_args()
    a.x, a.x_dtype, a.x_stride = _pn(x), _dt(x), _rows_of("x", x, (T, K))
    if T == 1:
        a.x_stride = -(-K // 8) * 8
    _like("ids", ids, (T, k), (torch.int32,))
    _like("weights", weights, (T, k), (torch.float32,))
    _like("offsets", offsets, (E + 1,), (torch.int32,))
    _like("slots", slots, (T * k,), (torch.int32,))
    _like("w_in", w_in, (E, 2, I, K), _CODES)
    _like("w_in_scale", w_in_scale, (E, 2, blocks(I), blocks(K)), (torch.float32,))
    _like("w_out", w_out, (E, N, I), _CODES)
    _like("w_out_scale", w_out_scale, (E, blocks(N), blocks(I)), (torch.float32,))
    a.ids, a.weights, a.offsets, a.slots = _pn(ids), _pn(weights), _p(offsets), _pn(slots)
    a.T, a.K, a.k, a.E, a.I, a.N = T, K, k, E, I, N
    a.w_in, a.w_in_scale, a.w_out, a.w_out_scale = _p(w_in), _p(w_in_scale), _p(w_out), _p(w_out_scale)
    a.y, a.y_dtype, a.y_stride = _pn(y), _dt(y), _rows_of("y", y, (T, N))
    if T == 1:
        a.y_stride = -(-N // 8) * 8
    if residual is not None:
        if residual.dtype != y.dtype:
            raise ValueError(f"residual is {residual.dtype}, y {y.dtype}")
        a.residual, a.residual_stride = _pn(residual), _rows_of("residual", residual, (T, N))
        if T == 1:
            a.residual_stride = a.y_stride
    _one_device(a, x, ids, weights, offsets, slots, w_in, w_in_scale, w_out, w_out_scale, residual, y)
    return a


def fise_expert_mlp_workspace_bytes(args):
    return lib().fise_expert_mlp_workspace_bytes(C.byref(args))


def fise_expert_mlp(args, workspace, stream=None):
    ws, nbytes = _here(args, workspace)
    _ck(lib().fise_expert_mlp(C.byref(args), ws, nbytes, _stream(stream)))


# --------------------------------------------------------------------------- UNet
def make_desc(d):
    s = fise_unet_desc()
    s.in_ch, s.out_ch, s.base, s.n_levels = d["in_ch"], d["out_ch"], d["base"], len(d["mults"])
    for i, m in enumerate(d["mults"]):
        s.mults[i] = m
        s.attn[i] = 1 if d["attn"][i] else 0
    s.layers, s.heads, s.ctx_dim, s.n_ctx, s.groups = d["layers"], d["heads"], d["ctx_dim"], d["n_ctx"], d["groups"]
    s.H, s.W, s.B = d["H"], d["W"], d["B"]
    return s


def fise_unet_create(desc):
    h = vp()
    s = make_desc(desc) if isinstance(desc, dict) else desc
    _ck(lib().fise_unet_create(C.byref(s), C.byref(h)))
    return h


def fise_unet_destroy(u):
    lib().fise_unet_destroy(u)


def fise_unet_desc_of(u):
    """The description a plan was made from, as the dict make_desc() takes."""
    s = fise_unet_desc()
    _ck(lib().fise_unet_desc_get(u, C.byref(s)))
    n = s.n_levels
    return dict(in_ch=s.in_ch, out_ch=s.out_ch, base=s.base, mults=tuple(s.mults[i] for i in range(n)),
                attn=tuple(bool(s.attn[i]) for i in range(n)), layers=s.layers, heads=s.heads, ctx_dim=s.ctx_dim,
                n_ctx=s.n_ctx, groups=s.groups, H=s.H, W=s.W, B=s.B)


def fise_unet_tensors(u, kind):
    """[(name, offset, numel)] of the flat weight (0), cache (1) or context-K/V (2) buffer."""
    out = []
    name = C.create_string_buffer(64)
    off, num = i64(), i64()
    for i in range(lib().fise_unet_num_tensors(u, kind)):
        _ck(lib().fise_unet_tensor_info(u, kind, i, name, C.byref(off), C.byref(num)))
        out.append((name.value.decode(), off.value, num.value))
    return out


def fise_unet_weight_elems(u):
    return lib().fise_unet_weight_elems(u)


def fise_unet_cache_bytes(u):
    return lib().fise_unet_cache_bytes(u)


def fise_unet_ctxkv_bytes(u):
    return lib().fise_unet_ctxkv_bytes(u)


def fise_unet_workspace_bytes(u, max_active_tiles, base_tile):
    return lib().fise_unet_workspace_bytes(u, max_active_tiles, base_tile)


def fise_unet_refresh_derived_workspace_bytes(u):
    return lib().fise_unet_refresh_derived_workspace_bytes(u)


def fise_unet_refresh_derived(u, weights, cache, workspace, stream=None):
    _ck(lib().fise_unet_refresh_derived(u, _p(weights), _p(cache), _p(workspace), workspace.numel() * workspace.element_size(),
                                        _stream(stream)))


FISE_MOVE_MAPS, FISE_MOVE_K, FISE_MOVE_VT = 1, 2, 4
_LAYOUT_FIELDS = ("maps_off", "maps_bytes", "kv_off", "kv_bytes", "small_off", "small_bytes", "derived_maps_off",
                  "derived_maps_bytes", "stored_bytes")


def fise_unet_cache_layout(u):
    """{field: bytes} of the contiguous tensor groups of a per-step cache buffer."""
    raw = (i64 * len(_LAYOUT_FIELDS))()
    _ck(lib().fise_unet_cache_layout_get(u, raw))
    return dict(zip(_LAYOUT_FIELDS, (int(v) for v in raw)))


def fise_unet_cache_move_workspace_bytes(u):
    return lib().fise_unet_cache_move_workspace_bytes(u)


def fise_unet_cache_move_active(u, src, dst, tile_idx, n_active, base_tile, halo, what, workspace, stream=None):
    """src / dst: cache-sized uint8 tensors in device memory or pinned host memory."""
    _ck(lib().fise_unet_cache_move_active(u, _p(src), _p(dst), _p(tile_idx), n_active, base_tile, halo, what, _p(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)))


def fise_unet_cache_move_tile_rows(u, src, dst, tile_rows, base_tile, halo, what, stream=None):
    """tile_rows: [(first, last), ...] rows of the base tile grid (host integers)."""
    flat = [int(v) for r in tile_rows for v in r]
    arr = (i32 * max(len(flat), 1))(*flat)
    _ck(lib().fise_unet_cache_move_tile_rows(u, _p(src), _p(dst), arr, len(flat) // 2, base_tile, halo, what, _stream(stream)))


def fise_unet_context_kv(u, weights, ctx, ctxkv, stream=None):
    _ck(lib().fise_unet_context_kv(u, _p(weights), _p(ctx), _p(ctxkv), None, 0, _stream(stream)))


def fise_masked_unet_step(u, weights, cache, latent, t_sin, ctxkv, tile_idx, n_active, base_tile, stats_mode,
                          level_dense, workspace, stream=None):
    ld = None
    if level_dense is not None:
        ld = (i32 * len(level_dense))(*[int(v) for v in level_dense])
    _ck(lib().fise_masked_unet_step(u, _p(weights), _p(cache), _p(latent), _p(t_sin), _p(ctxkv), _p(tile_idx), n_active,
                                    base_tile, stats_mode, ld, _p(workspace), workspace.numel() * workspace.element_size(),
                                    _stream(stream)))


def fise_unet_module_names(u):
    name = C.create_string_buffer(64)
    out = []
    for i in range(lib().fise_unet_num_modules(u)):
        _ck(lib().fise_unet_module_name(u, i, name))
        out.append(name.value.decode())
    return out


def fise_masked_unet_modules(u, weights, cache, latent, t_sin, ctxkv, tile_idx, n_active, base_tile, stats_mode,
                             level_dense, first_module, n_modules, workspace, stream=None):
    ld = None
    if level_dense is not None:
        ld = (i32 * len(level_dense))(*[int(v) for v in level_dense])
    _ck(lib().fise_masked_unet_modules(u, _p(weights), _p(cache), _p(latent), _p(t_sin), _p(ctxkv), _p(tile_idx), n_active,
                                       base_tile, stats_mode, ld, first_module, n_modules, _p(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)))


def fise_profile_enable(on):
    _ck(lib().fise_profile_enable(1 if on else 0))


def fise_profile_calibrate(n, stream=None):
    _ck(lib().fise_profile_calibrate(int(n), _stream(stream)))


def fise_calibrate_peaks(scratch, stream=None):
    """(copy GB/s, bf16 MFMA TFLOP/s) measured on the current device; `scratch` is overwritten."""
    gbs, tf = C.c_double(), C.c_double()
    _ck(lib().fise_calibrate_peaks(_p(scratch), scratch.numel() * scratch.element_size(), C.byref(gbs), C.byref(tf),
                                   _stream(stream)))
    return gbs.value, tf.value


def fise_profile_read(kind):
    """(total_ms, total_flops, total_bytes, launches) of the launches recorded for `kind`; -1 clears."""
    ms, fl, by, n = C.c_double(), C.c_double(), C.c_double(), i32()
    _ck(lib().fise_profile_read(kind, C.byref(ms), C.byref(fl), C.byref(by), C.byref(n)))
    return ms.value, fl.value, by.value, n.value
