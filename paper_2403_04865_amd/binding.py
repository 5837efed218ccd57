"""ctypes binding of libslide.so: same names as include/slide.h, argument marshalling only.

torch is used for device memory and streams; every step of the path runs in the library's
HIP kernels.  Missing library => ImportError-like failure at load (no fallback).
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    return os.path.join(_HERE, "libslide.so")


class SlideError(RuntimeError):
    CODES = {-1: "SLIDE_EINVAL", -2: "SLIDE_EARENA", -3: "SLIDE_EUNSUPPORTED", -4: "SLIDE_ESTATE", -5: "SLIDE_EHIP"}

    def __init__(self, code, what, hip=0):
        self.code = code
        super().__init__(f"{what}: {self.CODES.get(code, code)}" + (f" (hipError {hip})" if code == -5 else ""))


class _CConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("tile", "patch", "dim", "layers", "heads", "mlp_ratio", "mil_hidden",
                                         "n_classes", "dtype", "recompute")] + \
               [("ln_eps", C.c_float), ("checkpoint8", C.c_int32)]


@dataclass
class SlideConfig:
    tile: int
    patch: int
    dim: int
    layers: int
    heads: int
    mlp_ratio: int
    mil_hidden: int
    n_classes: int
    dtype: int = 0          # 0 float32, 1 bfloat16
    recompute: int = 0
    ln_eps: float = 1e-6
    checkpoint8: int = 0    # with recompute: block inputs in 8 bits


def config_from(shape, dtype: int, recompute: int = 0) -> SlideConfig:
    """SlideConfig from any object with the fields tile, patch, dim, layers, heads, mlp_ratio, mil_hidden, n_classes
    and ln_eps (such as a workload description of the input generators)."""
    return SlideConfig(shape.tile, shape.patch, shape.dim, shape.layers, shape.heads, shape.mlp_ratio, shape.mil_hidden,
                       shape.n_classes, dtype=dtype, recompute=recompute, ln_eps=shape.ln_eps)


_SYMS = {
    "slide_ctx_create": (C.c_int, [C.POINTER(_CConfig), C.POINTER(C.c_void_p)]),
    "slide_ctx_destroy": (None, [C.c_void_p]),
    "slide_param_count": (C.c_size_t, [C.c_void_p]),
    "slide_param_tensors": (C.c_int, [C.c_void_p]),
    "slide_param_name": (C.c_int, [C.c_void_p, C.c_int, C.c_char_p, C.c_size_t, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "slide_param_offset": (C.c_int, [C.c_void_p, C.c_char_p, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "slide_arena_bytes": (C.c_size_t, [C.c_void_p, C.c_int64]),
    "slide_pool_arena_bytes": (C.c_size_t, [C.c_void_p, C.c_int64]),
    "slide_bind": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t]),
    "encoder_fwd_tiles": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.c_void_p]),
    "encoder_bwd_tiles": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_void_p]),
    "mil_pool_fwd": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "mil_pool_fwd_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p]),
    "mil_pool_bwd": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int, C.c_void_p]),
    "slide_step_fwd": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "slide_step_bwd": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "slide_chunked_arena_bytes": (C.c_size_t, [C.c_void_p, C.c_int64, C.c_int64]),
    "slide_step_chunked": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "slide_features": (C.c_void_p, [C.c_void_p]),
    "slide_feature_grads": (C.c_void_p, [C.c_void_p]),
    "slide_last_hip_error": (C.c_int, []),
    "slide_prof_begin": (C.c_int, [C.c_void_p, C.c_int]),
    "slide_prof_end": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int), C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "slide_prof_family": (C.c_int, [C.c_void_p, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int), C.POINTER(C.c_double),
                                   C.POINTER(C.c_double)]),
    "slide_kernel_name": (C.c_char_p, [C.c_int]),
    "slide_calib_copy": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "slide_adamw_step": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_int64, C.c_float,
                                   C.c_float, C.c_float, C.c_float, C.c_float, C.c_void_p]),
}


class _CResNetConfig(C.Structure):
    _fields_ = [("tile", C.c_int32), ("block", C.c_int32), ("depths", C.c_int32 * 4), ("width", C.c_int32),
                ("mil_hidden", C.c_int32), ("n_classes", C.c_int32), ("bn_eps", C.c_float), ("norm_groups", C.c_int16),
                ("checkpoint8", C.c_int16)]


@dataclass
class ResNetConfig:
    tile: int
    block: int              # 0 basic, 1 bottleneck
    depths: tuple
    width: int
    mil_hidden: int
    n_classes: int
    bn_eps: float = 1e-5
    norm_groups: int = 0    # 0 batch normalisation, else groups of a group normalisation
    checkpoint8: int = 0    # with group normalisation: convolution outputs kept in 8 bits for the backward


def resnet_config_from(shape) -> ResNetConfig:
    """ResNetConfig from any object with the fields tile, block ("basic" / "bottleneck"), depths, width, mil_hidden,
    n_classes and bn_eps (such as a workload description of the input generators), and norm_groups and checkpoint8 where it has them."""
    return ResNetConfig(shape.tile, 0 if shape.block == "basic" else 1, tuple(shape.depths), shape.width,
                        shape.mil_hidden, shape.n_classes, shape.bn_eps, getattr(shape, "norm_groups", 0), getattr(shape, "checkpoint8", 0))


_P4 = [C.POINTER(C.c_double), C.POINTER(C.c_int), C.POINTER(C.c_double), C.POINTER(C.c_double)]
_SYMS.update({
    "resnet_ctx_create": (C.c_int, [C.POINTER(_CResNetConfig), C.POINTER(C.c_void_p)]),
    "resnet_ctx_destroy": (None, [C.c_void_p]),
    "resnet_param_count": (C.c_size_t, [C.c_void_p]),
    "resnet_param_tensors": (C.c_int, [C.c_void_p]),
    "resnet_param_name": (C.c_int, [C.c_void_p, C.c_int, C.c_char_p, C.c_size_t, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "resnet_feature_dim": (C.c_int, [C.c_void_p]),
    "resnet_arena_bytes": (C.c_size_t, [C.c_void_p, C.c_int64]),
    "resnet_bind": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t]),
    "resnet_encoder_fwd_tiles": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "resnet_encoder_bwd_tiles": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_void_p]),
    "resnet_slide_step_fwd": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "resnet_slide_step_bwd": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "resnet_features": (C.c_void_p, [C.c_void_p]),
    "resnet_feature_grads": (C.c_void_p, [C.c_void_p]),
    "resnet_saved_activations": (C.c_int, [C.c_void_p]),
    "resnet_saved_activation": (C.c_int, [C.c_void_p, C.c_int, C.POINTER(C.c_void_p), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "resnet_prof_begin": (C.c_int, [C.c_void_p, C.c_int]),
    "resnet_prof_end": (C.c_int, [C.c_void_p] + _P4),
    "resnet_prof_family": (C.c_int, [C.c_void_p, C.c_int] + _P4),
    "resnet_kernel_name": (C.c_char_p, [C.c_int]),
})


class _CAct8(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("ldc", C.c_int64), ("scales", C.c_void_p), ("lds", C.c_int64),
                ("rows", C.c_int64), ("cols", C.c_int64)]


class _CGroupNorm(C.Structure):
    _fields_ = [("n", C.c_int64), ("hw", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32), ("dtype", C.c_int32),
                ("act", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32)]


_VP, _I64, _A8P = C.c_void_p, C.c_int64, C.POINTER(_CAct8)
_SYMS.update({
    "slide_act8_pack": (C.c_int, [_VP, C.c_int, _I64, C.c_int, _A8P, _VP]),
    "slide_act8_unpack": (C.c_int, [_A8P, _VP, C.c_int, _I64, _VP]),
    "slide_act8_linear": (C.c_int, [_VP, C.c_int, _I64, _A8P, _A8P, _VP, C.c_int, _VP, _I64, _VP, _I64, _VP]),
    "slide_act8_wgrad_workspace_bytes": (C.c_size_t, [_I64, _I64, _I64]),
    "slide_act8_wgrad": (C.c_int, [_VP, C.c_int, _I64, _I64, _A8P, _VP, _I64, _VP, C.c_int, _VP, C.c_size_t, _VP]),
    "slide_group_norm_workspace_bytes": (C.c_size_t, [C.POINTER(_CGroupNorm)]),
    "slide_group_norm_fwd": (C.c_int, [C.POINTER(_CGroupNorm), _VP, _I64, _VP, _VP, _VP, _I64, _VP, _I64, _A8P, _VP, _VP, _VP,
                                       C.c_size_t, _VP]),
    "slide_group_norm_bwd": (C.c_int, [C.POINTER(_CGroupNorm), _VP, _I64, _VP, _I64, _A8P, _VP, _VP, _VP, _I64, _VP, _VP, _VP,
                                       _I64, _VP, _I64, _VP, _VP, C.c_int, _VP, C.c_size_t, _VP]),
})


_loaded = {}   # the file as it was -> the library with its functions declared (190 us to do again for every Act8Lib)


def load_cdll():
    p = lib_path()
    if not os.path.exists(p):
        raise OSError(f"{p} is not built: run `python -m paper_2403_04865_amd.build` (there is no fallback path)")
    # Device memory and streams come from torch, so the process must run on torch's HIP runtime: with the library
    # loaded first, its own dependency brings up a second runtime and every launch on torch's pointers fails
    # (hipErrorNoDevice).
    import torch  # noqa: F401
    at = os.stat(p)
    key = (p, at.st_dev, at.st_ino, at.st_mtime_ns, at.st_size)
    if key not in _loaded:
        lib = C.CDLL(p)
        for name, (res, args) in _SYMS.items():
            f = getattr(lib, name)
            f.restype = res
            f.argtypes = args
        _loaded[key] = lib
    return _loaded[key]


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return C.c_void_p(t)
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return C.c_void_p(stream)
    return C.c_void_p(stream.cuda_stream)


class SlideLib:
    """One slide_ctx.  Methods carry the C ABI's names and pass torch tensors' device pointers."""

    def __init__(self, cfg: SlideConfig):
        self.lib = load_cdll()
        self.cfg = cfg
        cc = _CConfig(cfg.tile, cfg.patch, cfg.dim, cfg.layers, cfg.heads, cfg.mlp_ratio, cfg.mil_hidden,
                      cfg.n_classes, cfg.dtype, cfg.recompute, cfg.ln_eps, cfg.checkpoint8)
        h = C.c_void_p()
        self._check(self.lib.slide_ctx_create(C.byref(cc), C.byref(h)), "slide_ctx_create")
        self.ctx = h
        self._keep = []

    def __del__(self):
        try:
            if getattr(self, "ctx", None):
                self.lib.slide_ctx_destroy(self.ctx)
                self.ctx = None
        except Exception:
            pass

    def _check(self, rc, what):
        if rc != 0:
            raise SlideError(rc, what, self.lib.slide_last_hip_error())

    # ---- layout queries
    def slide_param_count(self):
        return int(self.lib.slide_param_count(self.ctx))

    def param_layout(self):
        """[(name, offset, length)] in layout order."""
        out = []
        buf = C.create_string_buffer(64)
        off, ln = C.c_size_t(), C.c_size_t()
        for i in range(self.lib.slide_param_tensors(self.ctx)):
            self._check(self.lib.slide_param_name(self.ctx, i, buf, 64, C.byref(off), C.byref(ln)), "slide_param_name")
            out.append((buf.value.decode(), off.value, ln.value))
        return out

    def slide_param_offset(self, name):
        off, ln = C.c_size_t(), C.c_size_t()
        self._check(self.lib.slide_param_offset(self.ctx, name.encode(), C.byref(off), C.byref(ln)), "slide_param_offset")
        return off.value, ln.value

    def slide_arena_bytes(self, n_tiles):
        return int(self.lib.slide_arena_bytes(self.ctx, n_tiles))

    def slide_pool_arena_bytes(self, n):
        return int(self.lib.slide_pool_arena_bytes(self.ctx, n))

    # ---- calls
    def slide_bind(self, params, grads, arena):
        self._keep = [params, grads, arena]
        self._check(self.lib.slide_bind(self.ctx, _ptr(params), _ptr(grads), _ptr(arena), arena.numel() * arena.element_size()),
                    "slide_bind")

    def encoder_fwd_tiles(self, pixels, n_tiles, feats_out, save_for_bwd, stream=None):
        self._check(self.lib.encoder_fwd_tiles(self.ctx, _ptr(pixels), n_tiles, _ptr(feats_out), int(save_for_bwd),
                                               _stream(stream)), "encoder_fwd_tiles")

    def encoder_bwd_tiles(self, dfeats, n_tiles, accumulate, pixel_grad=None, stream=None):
        self._check(self.lib.encoder_bwd_tiles(self.ctx, _ptr(dfeats), n_tiles, int(accumulate), _ptr(pixel_grad),
                                               _stream(stream)), "encoder_bwd_tiles")

    def mil_pool_fwd(self, feats, N, label, loss=None, logits=None, alpha=None, stream=None):
        self._check(self.lib.mil_pool_fwd(self.ctx, _ptr(feats), N, label, _ptr(loss), _ptr(logits), _ptr(alpha),
                                          _stream(stream)), "mil_pool_fwd")

    def mil_pool_fwd_static(self, params, feats, N, label, loss=None, logits=None, alpha=None, stream=None):
        self._check(self.lib.mil_pool_fwd_static(self.ctx, _ptr(params), _ptr(feats), N, label, _ptr(loss), _ptr(logits),
                                                 _ptr(alpha), _stream(stream)), "mil_pool_fwd_static")

    def mil_pool_bwd(self, feats, N, label, dfeats_out, accumulate, stream=None):
        self._check(self.lib.mil_pool_bwd(self.ctx, _ptr(feats), N, label, _ptr(dfeats_out), int(accumulate),
                                          _stream(stream)), "mil_pool_bwd")

    def slide_step_fwd(self, pixels, N, label, loss=None, logits=None, alpha=None, stream=None):
        self._check(self.lib.slide_step_fwd(self.ctx, _ptr(pixels), N, label, _ptr(loss), _ptr(logits), _ptr(alpha),
                                            _stream(stream)), "slide_step_fwd")

    def slide_step_bwd(self, accumulate, pixel_grad=None, stream=None):
        self._check(self.lib.slide_step_bwd(self.ctx, int(accumulate), _ptr(pixel_grad), _stream(stream)), "slide_step_bwd")

    def slide_chunked_arena_bytes(self, N, chunk_tiles):
        return int(self.lib.slide_chunked_arena_bytes(self.ctx, N, chunk_tiles))

    def slide_step_chunked(self, pixels, N, chunk_tiles, label, accumulate, loss=None, logits=None, alpha=None,
                           pixel_grad=None, stream=None):
        self._check(self.lib.slide_step_chunked(self.ctx, _ptr(pixels), N, chunk_tiles, label, int(accumulate),
                                                _ptr(loss), _ptr(logits), _ptr(alpha), _ptr(pixel_grad),
                                                _stream(stream)), "slide_step_chunked")

    def slide_features(self):
        return self.lib.slide_features(self.ctx)

    def slide_feature_grads(self):
        return self.lib.slide_feature_grads(self.ctx)

    def slide_prof_begin(self, kernel_id):
        self._check(self.lib.slide_prof_begin(self.ctx, kernel_id), "slide_prof_begin")

    def slide_prof_end(self):
        ms, n, fl, by = C.c_double(), C.c_int(), C.c_double(), C.c_double()
        self._check(self.lib.slide_prof_end(self.ctx, C.byref(ms), C.byref(n), C.byref(fl), C.byref(by)), "slide_prof_end")
        return ms.value, n.value, fl.value, by.value

    def slide_prof_family(self, kernel_id):
        ms, n, fl, by = C.c_double(), C.c_int(), C.c_double(), C.c_double()
        self._check(self.lib.slide_prof_family(self.ctx, kernel_id, C.byref(ms), C.byref(n), C.byref(fl), C.byref(by)),
                    "slide_prof_family")
        return ms.value, n.value, fl.value, by.value

    def slide_adamw_step(self, params, grads, exp_avg, exp_avg_sq, count, step, lr, beta1=0.9, beta2=0.999, eps=1e-8,
                         weight_decay=0.01, stream=None):
        self._check(self.lib.slide_adamw_step(_ptr(params), _ptr(grads), _ptr(exp_avg), _ptr(exp_avg_sq),
                                              C.c_size_t(count), int(step), lr, beta1, beta2, eps, weight_decay,
                                              _stream(stream)), "slide_adamw_step")

    def slide_calib_copy(self, dst, src, nbytes, stream=None):
        self._check(self.lib.slide_calib_copy(_ptr(dst), _ptr(src), C.c_size_t(nbytes), _stream(stream)), "slide_calib_copy")

    def kernel_names(self):
        out, i = [], 0
        while True:
            s = self.lib.slide_kernel_name(i)
            if s is None:
                return out
            out.append(s.decode())
            i += 1


class ResNetLib:
    """One resnet_ctx (include/resnet.h).  Methods carry the C ABI's names and pass torch tensors' device pointers."""

    def __init__(self, cfg: ResNetConfig):
        self.lib = load_cdll()
        self.cfg = cfg
        for v in (cfg.norm_groups, cfg.checkpoint8):
            if not -2 ** 15 <= v < 2 ** 15:     # their 16 bits would hold another number
                raise SlideError(-1, "resnet_ctx_create")
        cc = _CResNetConfig(cfg.tile, cfg.block, (C.c_int32 * 4)(*cfg.depths), cfg.width, cfg.mil_hidden, cfg.n_classes,
                            cfg.bn_eps, cfg.norm_groups, cfg.checkpoint8)
        h = C.c_void_p()
        self._check(self.lib.resnet_ctx_create(C.byref(cc), C.byref(h)), "resnet_ctx_create")
        self.ctx = h
        self._keep = []

    def __del__(self):
        try:
            if getattr(self, "ctx", None):
                self.lib.resnet_ctx_destroy(self.ctx)
                self.ctx = None
        except Exception:
            pass

    def _check(self, rc, what):
        if rc != 0:
            raise SlideError(rc, what, self.lib.slide_last_hip_error())

    def resnet_param_count(self):
        return int(self.lib.resnet_param_count(self.ctx))

    def resnet_feature_dim(self):
        return int(self.lib.resnet_feature_dim(self.ctx))

    def param_layout(self):
        """[(name, offset, length)] in layout order."""
        out = []
        buf = C.create_string_buffer(64)
        off, ln = C.c_size_t(), C.c_size_t()
        for i in range(self.lib.resnet_param_tensors(self.ctx)):
            self._check(self.lib.resnet_param_name(self.ctx, i, buf, 64, C.byref(off), C.byref(ln)), "resnet_param_name")
            out.append((buf.value.decode(), off.value, ln.value))
        return out

    def resnet_arena_bytes(self, n_tiles):
        return int(self.lib.resnet_arena_bytes(self.ctx, n_tiles))

    def resnet_bind(self, params, grads, arena):
        self._keep = [params, grads, arena]
        self._check(self.lib.resnet_bind(self.ctx, _ptr(params), _ptr(grads), _ptr(arena),
                                         arena.numel() * arena.element_size()), "resnet_bind")

    def resnet_encoder_fwd_tiles(self, pixels, n_tiles, feats_out, stream=None):
        self._check(self.lib.resnet_encoder_fwd_tiles(self.ctx, _ptr(pixels), n_tiles, _ptr(feats_out), _stream(stream)),
                    "resnet_encoder_fwd_tiles")

    def resnet_encoder_bwd_tiles(self, dfeats, n_tiles, accumulate, stream=None):
        self._check(self.lib.resnet_encoder_bwd_tiles(self.ctx, _ptr(dfeats), n_tiles, int(accumulate), _stream(stream)),
                    "resnet_encoder_bwd_tiles")

    def resnet_slide_step_fwd(self, pixels, N, label, loss=None, logits=None, alpha=None, stream=None):
        self._check(self.lib.resnet_slide_step_fwd(self.ctx, _ptr(pixels), N, label, _ptr(loss), _ptr(logits), _ptr(alpha),
                                                   _stream(stream)), "resnet_slide_step_fwd")

    def resnet_slide_step_bwd(self, accumulate, stream=None):
        self._check(self.lib.resnet_slide_step_bwd(self.ctx, int(accumulate), _stream(stream)), "resnet_slide_step_bwd")

    def resnet_features(self):
        return self.lib.resnet_features(self.ctx)

    def resnet_feature_grads(self):
        return self.lib.resnet_feature_grads(self.ctx)

    def resnet_saved_activations(self):
        return int(self.lib.resnet_saved_activations(self.ctx))

    def resnet_saved_activation(self, index):
        """(device pointer, side, channels) of saved activation `index`."""
        p, side, ch = C.c_void_p(), C.c_int32(), C.c_int32()
        self._check(self.lib.resnet_saved_activation(self.ctx, index, C.byref(p), C.byref(side), C.byref(ch)),
                    "resnet_saved_activation")
        return p.value, side.value, ch.value

    def resnet_prof_begin(self, kernel_id):
        self._check(self.lib.resnet_prof_begin(self.ctx, kernel_id), "resnet_prof_begin")

    def resnet_prof_end(self):
        ms, n, fl, by = C.c_double(), C.c_int(), C.c_double(), C.c_double()
        self._check(self.lib.resnet_prof_end(self.ctx, C.byref(ms), C.byref(n), C.byref(fl), C.byref(by)), "resnet_prof_end")
        return ms.value, n.value, fl.value, by.value

    def resnet_prof_family(self, kernel_id):
        ms, n, fl, by = C.c_double(), C.c_int(), C.c_double(), C.c_double()
        self._check(self.lib.resnet_prof_family(self.ctx, kernel_id, C.byref(ms), C.byref(n), C.byref(fl), C.byref(by)),
                    "resnet_prof_family")
        return ms.value, n.value, fl.value, by.value

    def kernel_names(self):
        out, i = [], 0
        while True:
            s = self.lib.resnet_kernel_name(i)
            if s is None:
                return out
            out.append(s.decode())
            i += 1


ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


class Act8:
    """A matrix [rows, cols] in 8 bits (include/act8.h): codes [rows, >= cols] uint8, scales [rows, >= ceil(cols / 128)] uint8.  The calls write
    and read every row of codes up to the next multiple of 16 columns: a single row must have them, and the last of several rows' must lie in
    the tensor's memory."""

    def __init__(self, rows, cols, codes, scales):
        if codes.dim() != 2 or scales.dim() != 2 or codes.element_size() != 1 or scales.element_size() != 1:
            raise ValueError("codes and scales are matrices of bytes")
        if codes.shape[0] != rows or scales.shape[0] != rows or codes.shape[1] < cols or scales.shape[1] < -(-cols // 128):
            raise ValueError(f"codes {tuple(codes.shape)} or scales {tuple(scales.shape)} too small for {rows} x {cols}")
        if codes.stride(1) != 1 or scales.stride(1) != 1:
            raise ValueError("codes and scales: rows must be contiguous")
        if codes.device != scales.device:
            raise ValueError("codes and scales are on different devices")
        whole = -(-cols // 16) * 16
        if codes.shape[1] < whole and (rows == 1 or codes.storage_offset() + (rows - 1) * codes.stride(0) + whole > codes.untyped_storage().nbytes()):
            raise ValueError(f"codes {tuple(codes.shape)}: a row of {cols} takes {whole} bytes")
        self.rows, self.cols, self.codes, self.scales = rows, cols, codes, scales
        # (the stride that torch reports of a single row says nothing)
        self._c = _CAct8(codes.data_ptr(), codes.stride(0) if rows > 1 else whole, scales.data_ptr(),
                         scales.stride(0) if rows > 1 else max(scales.shape[1], 1), rows, cols)
        self._ref = C.byref(self._c)

    @staticmethod
    def empty(rows, cols, device="cuda"):
        import torch
        return Act8(rows, cols, torch.empty((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=device),
                    torch.empty((rows, -(-cols // 128)), dtype=torch.uint8, device=device))

    def get_device(self):
        return self.codes.get_device()


class Act8Lib:
    """The calls of include/act8.h on torch tensors, whose shapes, strides and types they take; no context.  A call runs on the
    tensors' device, on `stream` (default: that device's current stream)."""

    def __init__(self):
        import torch
        self.lib = load_cdll()
        self._torch = torch
        self._types = {torch.float32: 0, torch.bfloat16: 1}
        self._shapes = {}
        # the raw handle of a device's current stream, where this torch has it without building a Stream
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        self._entry = {n: getattr(self.lib, n) for n in ("slide_act8_pack", "slide_act8_unpack", "slide_act8_linear", "slide_act8_wgrad",
                                                         "slide_group_norm_fwd", "slide_group_norm_bwd")}

    # ---- marshalling
    def _type(self, t):
        try:
            return self._types[t.dtype]
        except KeyError:
            raise ValueError(f"float32 or bfloat16, not {t.dtype}") from None

    def _matrix(self, t, rows, cols, dtype, what):
        """(pointer, elements between rows) of a [rows, cols] matrix of dtype, or of tiles [n, hw, cols] whose rows lie at one stride.
        (None, 0) for None."""
        if t is None:
            return None, 0
        if t.dtype != dtype:
            raise ValueError(f"{what}: {t.dtype}, expected {dtype}")
        shape = t.shape
        if len(shape) in (2, 3) and shape[-1] == cols and t.numel() == rows * cols and t.is_contiguous():   # most of them
            return t.data_ptr(), cols
        stride = t.stride()
        if len(shape) == 2:
            have, last = shape
            ld = stride[0]
        elif len(shape) == 3:
            n, hw, last = shape
            if n > 1 and hw > 1 and stride[0] != hw * stride[1]:
                raise ValueError(f"{what}: tiles must follow one another at one row stride")
            have = n * hw
            ld = stride[1] if hw > 1 else stride[0]
        else:
            raise ValueError(f"{what}: a matrix, or tiles of rows")
        if have != rows or last != cols:
            raise ValueError(f"{what}: {tuple(shape)}, expected {rows} rows of {cols}")
        if last > 1 and stride[-1] != 1:
            raise ValueError(f"{what}: rows must be contiguous")
        return t.data_ptr(), ld if have > 1 else max(ld, cols)

    def _floats(self, t, n, what):
        if t is None:
            return None
        if t.dtype != self._torch.float32 or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{what}: {n} contiguous float32 values")
        return t.data_ptr()

    def _act(self, act):
        if isinstance(act, str):
            try:
                return ACTS[act]
            except KeyError:
                raise ValueError(f"activation {act!r}: one of {', '.join(ACTS)}") from None
        return int(act)

    def _call(self, what, first, others, args, stream):
        """Run the entry point on the device of `first`, which all of `others` must be on."""
        dev = first.get_device()
        if dev < 0:
            raise ValueError(f"{what}: tensors must be on the GPU")
        for t in others:
            if t is not None and t.get_device() != dev:
                raise ValueError(f"{what}: tensors on different devices")
        cuda = self._torch.cuda
        if stream is None:
            stream = self._raw_stream(dev)
        elif not isinstance(stream, int):
            if stream.device.index != dev:
                raise ValueError(f"{what}: a stream of {stream.device} for tensors on device {dev}")
            stream = stream.cuda_stream
        if dev != cuda.current_device():
            with cuda.device(dev):
                rc = self._entry[what](*args, stream)
        else:
            rc = self._entry[what](*args, stream)
        if rc != 0:
            raise SlideError(rc, what, self.lib.slide_last_hip_error())

    def _work(self, t):
        if t is None:
            return None, 0
        if not t.is_contiguous():
            raise ValueError("workspace: a contiguous tensor")
        return t.data_ptr(), t.numel() * t.element_size()

    # ---- calls
    def slide_act8_pack(self, x, out, transpose=False, stream=None):
        rows, cols = (out.cols, out.rows) if transpose else (out.rows, out.cols)
        p, ld = self._matrix(x, rows, cols, x.dtype, "x")
        self._call("slide_act8_pack", out, (x,), (p, self._type(x), ld, int(transpose), out._ref), stream)

    def slide_act8_unpack(self, a, y, stream=None):
        p, ld = self._matrix(y, a.rows, a.cols, y.dtype, "y")
        self._call("slide_act8_unpack", a, (y,), (a._ref, p, self._type(y), ld), stream)

    def slide_act8_linear(self, x, x8, w8, y, bias=None, act="none", residual=None, stream=None):
        """y = act(x8 w8^T + bias) + residual, with x packed into x8 first (x None: x8 holds its values)."""
        xp, ldx = (None, 0) if x is None else self._matrix(x, x8.rows, x8.cols, y.dtype, "x")
        rp, ldr = self._matrix(residual, x8.rows, w8.rows, y.dtype, "residual")
        yp, ldy = self._matrix(y, x8.rows, w8.rows, y.dtype, "y")
        self._call("slide_act8_linear", y, (x, x8, w8, bias, residual),
                   (xp, self._type(y), ldx, x8._ref, w8._ref, self._floats(bias, w8.rows, "bias"), self._act(act), rp, ldr, yp, ldy),
                   stream)

    def slide_act8_wgrad_workspace_bytes(self, rows, out, cin):
        return int(self.lib.slide_act8_wgrad_workspace_bytes(rows, out, cin))

    def slide_act8_wgrad(self, dy, x8, dW, db=None, accumulate=False, workspace=None, stream=None):
        out = dW.shape[0]
        p, ld = self._matrix(dy, x8.rows, out, dy.dtype, "dy")
        wp, ldw = self._matrix(dW, out, x8.cols, self._torch.float32, "dW")
        self._call("slide_act8_wgrad", dW, (dy, x8, db, workspace),
                   (p, self._type(dy), ld, out, x8._ref, wp, ldw, self._floats(db, out, "db"), int(accumulate), *self._work(workspace)),
                   stream)

    def _shape(self, *key):
        """The C description of a group norm, kept by its values: n, hw, channels, groups, dtype, act, eps."""
        s = self._shapes.get(key)
        if s is None:
            if len(self._shapes) > 256:
                self._shapes.clear()
            s = self._shapes[key] = C.pointer(_CGroupNorm(*key, 0))
        return s

    def slide_group_norm_workspace_bytes(self, n, hw, channels, groups, dtype):
        """For both directions of a group norm over [n, hw, channels]; 0 for a shape that is refused."""
        s = self._shape(n, hw, channels, groups, self._types.get(dtype, -1), 0, 1.0)
        return int(self.lib.slide_group_norm_workspace_bytes(s))

    def slide_group_norm_fwd(self, x, gamma, beta, groups, y, mean, rstd, eps=1e-5, act="none", residual=None, x8=None,
                             workspace=None, stream=None):
        """x, y, residual: [n, hw, channels]; mean, rstd: [n, groups]."""
        if x.dim() != 3:
            raise ValueError("x: [n, hw, channels]")
        n, hw, c = x.shape
        s = self._shape(n, hw, c, groups, self._type(x), self._act(act), eps)
        xp, ldx = self._matrix(x, n * hw, c, x.dtype, "x")
        rp, ldr = self._matrix(residual, n * hw, c, x.dtype, "residual")
        yp, ldy = self._matrix(y, n * hw, c, x.dtype, "y")
        self._call("slide_group_norm_fwd", x, (gamma, beta, residual, y, x8, mean, rstd, workspace),
                   (s, xp, ldx, self._floats(gamma, c, "gamma"), self._floats(beta, c, "beta"), rp, ldr, yp, ldy,
                    None if x8 is None else x8._ref, self._floats(mean, n * groups, "mean"), self._floats(rstd, n * groups, "rstd"),
                    *self._work(workspace)), stream)

    def slide_group_norm_bwd(self, dy, x, gamma, beta, mean, rstd, groups, dx, dgamma, dbeta, act="none", residual=None,
                             dresidual=None, accumulate=False, workspace=None, stream=None):
        """x: [n, hw, channels], or the Act8 that the forward left."""
        if dy.dim() != 3:
            raise ValueError("dy: [n, hw, channels]")
        n, hw, c = dy.shape
        t = dy.dtype
        s = self._shape(n, hw, c, groups, self._type(dy), self._act(act), 1.0)
        kept = isinstance(x, Act8)
        xp, ldx = (None, 0) if kept else self._matrix(x, n * hw, c, t, "x")
        m = self._matrix
        self._call("slide_group_norm_bwd", dy, (x, gamma, beta, residual, mean, rstd, dx, dresidual, dgamma, dbeta, workspace),
                   (s, *m(dy, n * hw, c, t, "dy"), xp, ldx, x._ref if kept else None, self._floats(gamma, c, "gamma"),
                    self._floats(beta, c, "beta"), *m(residual, n * hw, c, t, "residual"), self._floats(mean, n * groups, "mean"),
                    self._floats(rstd, n * groups, "rstd"), *m(dx, n * hw, c, t, "dx"), *m(dresidual, n * hw, c, t, "dresidual"),
                    self._floats(dgamma, c, "dgamma"), self._floats(dbeta, c, "dbeta"), int(accumulate), *self._work(workspace)),
                   stream)
