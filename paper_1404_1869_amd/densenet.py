"""ctypes binding of libdensenet.so: the C ABI of include/densenet.h, same names, argument marshalling
only.  Device memory comes from torch tensors and the stream from torch.cuda.current_stream(); every
step of the computation runs in the library's HIP kernels.  There is no fallback: if the library or a
GPU is missing the calls raise.

On top of the raw entry points, ``convnet_featpyramid`` mirrors the paper's interface
(``pyra = convnet_featpyramid(image)``, Sec. 3.5): image(s) in, per-scale conv5 maps plus geometry out.
"""
from __future__ import annotations

import bisect
import ctypes
import functools
import os
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdensenet.so")

DN_OK, DN_E_INVALID_ARG, DN_E_TOO_LARGE, DN_E_BUFFER_TOO_SMALL = 0, -1, -2, -3
DN_E_UNSUPPORTED, DN_E_HIP, DN_E_INTERNAL = -4, -5, -6
DN_F32, DN_F16, DN_BF16 = 0, 1, 2
DN_F8 = 3   # e4m3: 8-bit outputs, operands with scales for blocks, and optimiser states only
DN_PAD_ZERO, DN_PAD_RAMP = 0, 1
DN_MAX_SCALES, DN_MAX_PLANES_PER_IMAGE, DN_MAX_WARP_SIDE, DN_MAX_ASPECTS = 64, 64, 1024, 8
DN_MAX_BATCH_ITEMS = 65536
DN_STATIC_SCRATCH_BYTES = 64 << 20
DN_MAX_NORM_C = 32768
DN_SCALE_BLOCK, DN_MAX_TOP, DN_MAX_NS_STEPS, DN_NO_WORKSPACE = 128, 64, 16, 256
ADAMW_BLOCK = 256
DTYPES = {"f32": DN_F32, "f16": DN_F16, "bf16": DN_BF16}

EXPORTS = ("densenet_plan_pyramid", "densenet_build_pyramid", "densenet_pack_weights",
           "densenet_conv_features", "densenet_region_windows", "densenet_conv_layer",
           "densenet_lrn_pool", "densenet_maxpool", "densenet_layer_sizes", "densenet_warp_regions",
           "densenet_region_pool", "densenet_plan_batch", "densenet_build_batch",
           "densenet_region_windows_batch", "densenet_build_pyramid_noalloc", "densenet_rms_norm",
           "densenet_rms_norm_backward", "densenet_softmax_loss", "densenet_softmax_loss_backward",
           "densenet_adamw", "densenet_quantize_blocks", "densenet_block_product", "densenet_token_scores",
           "densenet_token_scores_backward", "densenet_muon", "densenet_profile_start", "densenet_profile_stop", "densenet_last_error")


class dn_pyramid_params(ctypes.Structure):
    _fields_ = [("n_scales", ctypes.c_int32), ("steps_per_octave", ctypes.c_int32),
                ("base_scale", ctypes.c_double), ("base_longest_side", ctypes.c_int32),
                ("pad", ctypes.c_int32), ("pad_mode", ctypes.c_int32), ("plane_h", ctypes.c_int32),
                ("plane_w", ctypes.c_int32), ("mean", ctypes.c_float * 3), ("n_aspects", ctypes.c_int32),
                ("aspects", ctypes.c_double * DN_MAX_ASPECTS)]


class dn_scale_geom(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("k", "h", "w", "plane", "y", "x", "rh", "rw", "r0",
                                              "r1", "c0", "c1", "aspect", "image")] + \
               [(n, ctypes.c_double) for n in ("s", "sy", "sx")]


class dn_plane_desc(ctypes.Structure):
    _fields_ = [("h", ctypes.c_int32), ("w", ctypes.c_int32), ("offset", ctypes.c_int64),
                ("pitch", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class dn_net_params(ctypes.Structure):
    _fields_ = [("lrn_alpha", ctypes.c_float), ("lrn_beta", ctypes.c_float),
                ("lrn_k", ctypes.c_float), ("lrn_n", ctypes.c_int32),
                ("lrn_before_pool", ctypes.c_int32), ("pool5", ctypes.c_int32)]


class dn_profile_entry(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


class dn_adamw_tensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("block", ctypes.c_int64)]


class dn_adamw_params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "grad_scale")] + \
               [("step", ctypes.c_int64), ("seed", ctypes.c_uint32), ("state_bits", ctypes.c_int32)]


class dn_muon_tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("p", "g", "copy", "m")] + [("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                                                                         ("rate", ctypes.c_double)]


class dn_muon_params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "momentum", "weight_decay", "grad_scale", "eps")] + \
               [("coefficients", ctypes.c_double * 3 * DN_MAX_NS_STEPS)] + \
               [(n, ctypes.c_int32) for n in ("steps", "nesterov", "parts", "reserved")]


class DenseNetError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"densenet error {status}: {msg}")
        self.status = status


_lib = None


def lib():
    """Load libdensenet.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run __graft_entry__.build() first")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        pp, pg, pd = ctypes.POINTER(dn_pyramid_params), ctypes.POINTER(dn_scale_geom), ctypes.POINTER(dn_plane_desc)
        pn = ctypes.POINTER(dn_net_params)
        psz, pi32, pi64 = ctypes.POINTER(sz), ctypes.POINTER(i32), ctypes.POINTER(i64)
        sig = {
            "densenet_plan_pyramid": [i32, i32, pp, pg, pd, i32, pi32, pi64],
            "densenet_build_pyramid": [P, i32, i32, i32, pp, i32, P, sz, psz, pg, pd, i32, pi32, pi64, P],
            "densenet_build_pyramid_noalloc": [P, i32, i32, i32, pp, i32, P, sz, psz, pg, pd, i32, pi32, pi64,
                                               P],
            "densenet_pack_weights": [P, P, i32, P, sz, psz, P],
            "densenet_conv_features": [P, pd, i32, i32, P, pn, P, sz, psz, P, sz, psz, pd, P, sz, psz,
                                       pd, P],
            "densenet_region_windows": [P, pd, i32, i32, pg, i32, i32, i32, P, P, i32, f32, i32, P, P,
                                        P, P],
            "densenet_region_pool": [P, pd, i32, i32, pg, i32, i32, i32, P, P, i32, f32, i32, P, P, P,
                                     P],
            "densenet_conv_layer": [i32, P, i32, i32, i32, i32, P, P, P],
            "densenet_lrn_pool": [P, i32, i32, i32, i32, i32, pn, P, P],
            "densenet_maxpool": [P, i32, i32, i32, i32, i32, P, P],
            "densenet_layer_sizes": [i32, i32, pi32],
            "densenet_warp_regions": [P, i32, i32, i32, P, P, i32, i32, i32, ctypes.POINTER(f32), i32, P,
                                      sz, psz, P],
            "densenet_plan_batch": [i32, i32, i32, pp, pg, pd, i32, pi32, pi64],
            "densenet_build_batch": [P, i32, i32, i32, pp, i32, pg, P, i32, P, sz, psz, P],
            "densenet_region_windows_batch": [P, pd, i32, i32, pg, P, i32, i32, i32, i32, P, P, i32, f32,
                                              i32, P, P, P, P],
            "densenet_rms_norm": [P, i64, P, i64, P, i64, i32, i32, f32, P, i64, P, i64, i32, i32, P, P],
            "densenet_rms_norm_backward": [P, i64, i32, P, i64, P, i64, P, i64, i32, i32, f32, P, i64, P, P,
                                           sz, psz, P],
            "densenet_softmax_loss": [P, i64, P, i64, P, i64, i32, i32, i32, P, P, P, sz, psz, P],
            "densenet_softmax_loss_backward": [P, i64, P, i64, P, P, P, f32, i64, i32, i32, i32, P, i64, P,
                                               i64, P, sz, psz, P],
            "densenet_adamw": [ctypes.POINTER(dn_adamw_tensor), i32, i32, i32, i32,
                               ctypes.POINTER(dn_adamw_params), P, P, P, P, i64, P],
            "densenet_quantize_blocks": [P, i64, i64, i32, i32, i32, P, i64, P, P, i64, P, P],
            "densenet_block_product": [P, i64, P, P, i64, P, i64, i32, i32, P, i64, i32, P, sz, psz, P],
            "densenet_token_scores": [P, i64, P, i64, i32, i32, f32, i32, P, P, P, P, P, P, sz, psz, P],
            "densenet_token_scores_backward": [P, i64, P, P, P, P, P, P, P, P, i64, i32, i32, f32, i32, P, i64, P],
            "densenet_muon": [ctypes.POINTER(dn_muon_tensor), i32, i32, i32, i32, ctypes.POINTER(dn_muon_params), P, sz, psz, P],
            "densenet_profile_start": [ctypes.c_char_p],
            "densenet_profile_stop": [ctypes.POINTER(dn_profile_entry), i32, pi32],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        L.densenet_last_error.argtypes = []
        L.densenet_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def last_error() -> str:
    return lib().densenet_last_error().decode()


def check(status: int):
    if status != DN_OK:
        raise DenseNetError(status, last_error())
    return status


# ------------------------------------------------------------------------------------------------
# torch plumbing: device memory and streams only
# ------------------------------------------------------------------------------------------------
def _torch():
    import torch
    return torch


def _stream():
    return ctypes.c_void_p(_torch().cuda.current_stream().cuda_stream)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA/HIP tensors"
    return ctypes.c_void_p(t.data_ptr())


def _tdtype(dt: int):
    torch = _torch()
    return {DN_F32: torch.float32, DN_F16: torch.float16, DN_BF16: torch.bfloat16}[dt]


def pyramid_params(n_scales, steps_per_octave, base_scale=1.0, base_longest_side=0, pad=0,
                   pad_mode=DN_PAD_ZERO, plane_h=0, plane_w=0, mean=(0.0, 0.0, 0.0), aspects=()):
    p = dn_pyramid_params()
    p.n_scales, p.steps_per_octave, p.base_scale = n_scales, steps_per_octave, base_scale
    p.base_longest_side, p.pad, p.pad_mode = base_longest_side, pad, pad_mode
    p.plane_h, p.plane_w = plane_h, plane_w
    p.mean = (ctypes.c_float * 3)(*mean)
    p.n_aspects = len(aspects)
    for i, r in enumerate(aspects):
        p.aspects[i] = float(r)
    return p


def n_entries(p: dn_pyramid_params) -> int:
    """Pyramid entries (scales x aspect ratios) of a recipe: the length of its geometry arrays."""
    return p.n_scales * max(1, p.n_aspects)


def params_for(w):
    """dn_pyramid_params of a configs.Workload."""
    return pyramid_params(w.n_scales, w.steps_per_octave, w.base_scale, w.base_longest_side, w.pad,
                          w.pad_mode, w.plane_h, w.plane_w, w.mean, w.aspects)


def net_params(alpha=1e-4, beta=0.75, k=1.0, n=5, lrn_before_pool=True, pool5=False):
    q = dn_net_params()
    q.lrn_alpha, q.lrn_beta, q.lrn_k, q.lrn_n = alpha, beta, k, n
    q.lrn_before_pool, q.pool5 = int(lrn_before_pool), int(pool5)
    return q


# ------------------------------------------------------------------------------------------------
# Entry points
# ------------------------------------------------------------------------------------------------
@dataclass
class PlanResult:
    geom: list            # dn_scale_geom per scale
    planes: list          # dn_plane_desc per plane of one image
    image_elems: int

    def geom_array(self) -> np.ndarray:
        """[K][13] int32: k, h, w, plane, y, x, rh, rw, r0, r1, c0, c1, aspect."""
        return np.array([[getattr(g, f) for f in ("k", "h", "w", "plane", "y", "x", "rh", "rw", "r0",
                                                   "r1", "c0", "c1", "aspect")] for g in self.geom],
                        np.int32)

    def scale_array(self) -> np.ndarray:
        return np.array([[g.s, g.sy, g.sx] for g in self.geom], np.float64)

    def image_descs(self, n_img: int) -> list:
        """Descriptors of the planes of n_img images built with this plan (image b's planes at
        b * image_elems), image-major, for densenet_conv_features."""
        out = []
        for b in range(n_img):
            for d in self.planes:
                q = dn_plane_desc()
                q.h, q.w, q.pitch, q.offset = d.h, d.w, d.pitch, b * self.image_elems + d.offset
                out.append(q)
        return out


def plane_view(planes, d: dn_plane_desc, base: int = 0):
    """[3][h][w] view of the plane that descriptor d places in the flat planes tensor (rows d.pitch
    elements apart), shifted by base elements."""
    pitch = d.pitch or d.w
    o = base + d.offset
    return planes[o:o + 3 * d.h * pitch].view(3, d.h, pitch)[:, :, :d.w]


def densenet_plan_pyramid(H: int, W: int, p: dn_pyramid_params) -> PlanResult:
    geom = (dn_scale_geom * n_entries(p))()
    planes = (dn_plane_desc * DN_MAX_PLANES_PER_IMAGE)()
    n = ctypes.c_int32()
    e = ctypes.c_int64()
    check(lib().densenet_plan_pyramid(H, W, ctypes.byref(p), geom, planes, DN_MAX_PLANES_PER_IMAGE,
                                      ctypes.byref(n), ctypes.byref(e)))
    return PlanResult(list(geom), list(planes[:n.value]), e.value)


def densenet_build_pyramid(images, p: dn_pyramid_params, dtype: int, out=None):
    """images: uint8 device tensor [n][3][H][W] (or [3][H][W]).  Returns (planes tensor, PlanResult)."""
    torch = _torch()
    if images.dim() == 3:
        images = images[None]
    n_img, _, H, W = images.shape
    geom = (dn_scale_geom * n_entries(p))()
    planes = (dn_plane_desc * DN_MAX_PLANES_PER_IMAGE)()
    n = ctypes.c_int32()
    e = ctypes.c_int64()
    need = ctypes.c_size_t()
    L = lib()
    check(L.densenet_build_pyramid(None, n_img, H, W, ctypes.byref(p), dtype, None, 0,
                                   ctypes.byref(need), geom, planes, DN_MAX_PLANES_PER_IMAGE,
                                   ctypes.byref(n), ctypes.byref(e), None))
    es = 4 if dtype == DN_F32 else 2
    if out is None:
        out = torch.empty(need.value // es, dtype=_tdtype(dtype), device=images.device)
    check(L.densenet_build_pyramid(_ptr(images), n_img, H, W, ctypes.byref(p), dtype, _ptr(out),
                                   out.numel() * out.element_size(), ctypes.byref(need), geom, planes,
                                   DN_MAX_PLANES_PER_IMAGE, ctypes.byref(n), ctypes.byref(e),
                                   _stream()))
    return out, PlanResult(list(geom), list(planes[:n.value]), e.value)


def densenet_build_pyramid_noalloc(images, p: dn_pyramid_params, dtype: int, out=None):
    """As densenet_build_pyramid, with the builder's staging in the library's static array: `out` (the
    planes only) is the only device buffer.  Returns (planes tensor, PlanResult)."""
    torch = _torch()
    if images.dim() == 3:
        images = images[None]
    n_img, _, H, W = images.shape
    geom = (dn_scale_geom * n_entries(p))()
    planes = (dn_plane_desc * DN_MAX_PLANES_PER_IMAGE)()
    n = ctypes.c_int32()
    e = ctypes.c_int64()
    need = ctypes.c_size_t()
    L = lib()
    check(L.densenet_build_pyramid_noalloc(None, n_img, H, W, ctypes.byref(p), dtype, None, 0,
                                           ctypes.byref(need), geom, planes, DN_MAX_PLANES_PER_IMAGE,
                                           ctypes.byref(n), ctypes.byref(e), None))
    es = 4 if dtype == DN_F32 else 2
    if out is None:
        out = torch.empty(need.value // es, dtype=_tdtype(dtype), device=images.device)
    check(L.densenet_build_pyramid_noalloc(_ptr(images), n_img, H, W, ctypes.byref(p), dtype, _ptr(out),
                                           out.numel() * out.element_size(), ctypes.byref(need), geom,
                                           planes, DN_MAX_PLANES_PER_IMAGE, ctypes.byref(n),
                                           ctypes.byref(e), _stream()))
    return out, PlanResult(list(geom), list(planes[:n.value]), e.value)


class BatchPlan:
    """Cross-image packing (Sec. 3.1 stitching over a whole batch): the plan of n_img images of H x W,
    its host geometry (entry e of image b at b * E + e) and a device copy of it for the kernels,
    uploaded once."""

    def __init__(self, n_img: int, H: int, W: int, p: dn_pyramid_params, device="cuda"):
        """device=None plans on the host only (no device copy)."""
        self.n_img, self.H, self.W, self.params = n_img, H, W, p
        self.E = n_entries(p)
        self.geom = (dn_scale_geom * (n_img * self.E))()
        n, e = ctypes.c_int32(), ctypes.c_int64()
        cap = n_img * self.E
        planes = (dn_plane_desc * cap)()
        check(lib().densenet_plan_batch(n_img, H, W, ctypes.byref(p), self.geom, planes, cap,
                                        ctypes.byref(n), ctypes.byref(e)))
        self.planes = list(planes[:n.value])
        self.total_elems = e.value
        self.d_geom = None
        if device is not None:
            raw = np.frombuffer(bytes(self.geom), np.uint8).copy()
            self.d_geom = _torch().from_numpy(raw).to(device)

    @property
    def n_planes(self) -> int:
        return len(self.planes)

    def entry(self, b: int, e: int) -> dn_scale_geom:
        return self.geom[b * self.E + e]

    def geom_array(self) -> np.ndarray:
        """[n_img * E][14] int32: k, h, w, plane, y, x, rh, rw, r0, r1, c0, c1, aspect, image."""
        return np.array([[getattr(g, f) for f in ("k", "h", "w", "plane", "y", "x", "rh", "rw", "r0",
                                                   "r1", "c0", "c1", "aspect", "image")]
                         for g in self.geom], np.int32)


def densenet_build_batch(images, plan: BatchPlan, dtype: int, out=None):
    """images: uint8 device tensor [n_img][3][H][W] -> the packed batch's planes (flat tensor; plane j
    at j * 3 * plane_h * pitch, followed by the builder's scratch; views: plane_view(out, plan.planes[j]))."""
    torch = _torch()
    n_img, _, H, W = images.shape
    assert (n_img, H, W) == (plan.n_img, plan.H, plan.W), "images do not match the plan"
    need = ctypes.c_size_t()
    L = lib()
    check(L.densenet_build_batch(None, n_img, H, W, ctypes.byref(plan.params), dtype, plan.geom, None,
                                 plan.n_planes, None, 0, ctypes.byref(need), None))
    es = 4 if dtype == DN_F32 else 2
    if out is None:
        out = torch.empty(need.value // es, dtype=_tdtype(dtype), device=images.device)
    check(L.densenet_build_batch(_ptr(images), n_img, H, W, ctypes.byref(plan.params), dtype, plan.geom,
                                 _ptr(plan.d_geom), plan.n_planes, _ptr(out),
                                 out.numel() * out.element_size(), ctypes.byref(need), _stream()))
    return out


def densenet_region_windows_batch(conv5, conv5_desc, dtype: int, plan: BatchPlan, boxes, box_img=None,
                                  target=227.0, S=6, pooled=False, want_idx=False, out=None, scale=None):
    """Region windows (pooled=False) or max-pooled bins (pooled=True) over a cross-image packed batch."""
    torch = _torch()
    n = boxes.shape[0]
    if out is None:
        out = torch.empty((n, 256 * S * S), dtype=torch.float32, device=boxes.device)
    if scale is None:
        scale = torch.empty(n, dtype=torch.int32, device=boxes.device)
    idx = torch.empty((n, S, S, 4 if pooled else 2), dtype=torch.int32, device=boxes.device) if want_idx \
        else None
    cd = (dn_plane_desc * len(conv5_desc))(*conv5_desc)
    check(lib().densenet_region_windows_batch(_ptr(conv5), cd, len(conv5_desc), dtype, plan.geom,
                                              _ptr(plan.d_geom), plan.n_img, plan.E, plan.params.pad,
                                              int(pooled), _ptr(boxes), _ptr(box_img), n, target, S,
                                              _ptr(out), _ptr(scale), _ptr(idx), _stream()))
    return out, scale, idx


def densenet_pack_weights(weights, dtype: int):
    """weights: [(w, b)] conv1..conv5 as fp32 device tensors (OIHW).  Returns the packed blob."""
    torch = _torch()
    ws = [w.contiguous().float() for w, _ in weights]
    bs = [b.contiguous().float() for _, b in weights]
    wp = (ctypes.c_void_p * 5)(*[w.data_ptr() for w in ws])
    bp = (ctypes.c_void_p * 5)(*[b.data_ptr() for b in bs])
    need = ctypes.c_size_t()
    L = lib()
    check(L.densenet_pack_weights(wp, bp, dtype, None, 0, ctypes.byref(need), None))
    blob = torch.empty(need.value, dtype=torch.uint8, device=ws[0].device)
    check(L.densenet_pack_weights(wp, bp, dtype, _ptr(blob), need.value, ctypes.byref(need),
                                  _stream()))
    return blob


class ConvFeatures:
    """Reusable buffers for densenet_conv_features over a fixed plane list."""

    def __init__(self, planes_desc, dtype: int, net: dn_net_params, device="cuda"):
        torch = _torch()
        self.n = len(planes_desc)
        self.pd = (dn_plane_desc * self.n)(*planes_desc)
        self.dtype, self.net = dtype, net
        self.c5d = (dn_plane_desc * self.n)()
        self.p5d = (dn_plane_desc * self.n)()
        ws, c5, p5 = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        check(lib().densenet_conv_features(None, self.pd, self.n, dtype, None, ctypes.byref(net), None,
                                           0, ctypes.byref(ws), None, 0, ctypes.byref(c5), self.c5d,
                                           None, 0, ctypes.byref(p5), self.p5d, None))
        es = 4 if dtype == DN_F32 else 2
        self.workspace = torch.empty(max(ws.value, 1), dtype=torch.uint8, device=device)
        self.conv5 = torch.empty(c5.value // es, dtype=_tdtype(dtype), device=device)
        self.pool5 = torch.empty(p5.value // es, dtype=_tdtype(dtype), device=device) if net.pool5 else None

    def __call__(self, planes_tensor, packed):
        check(lib().densenet_conv_features(
            _ptr(planes_tensor), self.pd, self.n, self.dtype, _ptr(packed), ctypes.byref(self.net),
            _ptr(self.workspace), self.workspace.numel(), ctypes.byref(ctypes.c_size_t()),
            _ptr(self.conv5), self.conv5.numel() * self.conv5.element_size(),
            ctypes.byref(ctypes.c_size_t()), self.c5d, _ptr(self.pool5),
            0 if self.pool5 is None else self.pool5.numel() * self.pool5.element_size(),
            ctypes.byref(ctypes.c_size_t()), self.p5d, _stream()))
        return self.conv5, self.pool5

    def conv5_maps(self):
        """Per-plane [Hc][Wc][256] views of the conv5 buffer."""
        return [self.conv5[d.offset:d.offset + d.h * d.w * 256].view(d.h, d.w, 256) for d in self.c5d]

    def pool5_maps(self):
        return [self.pool5[d.offset:d.offset + d.h * d.w * 256].view(d.h, d.w, 256) for d in self.p5d]


def densenet_conv_features(planes_tensor, planes_desc, dtype: int, packed, net: dn_net_params):
    cf = ConvFeatures(planes_desc, dtype, net, device=planes_tensor.device)
    cf(planes_tensor, packed)
    return cf


def _regions(fn, conv5, conv5_desc, dtype, plan, pad, planes_per_img, boxes, box_img, target, S, want_idx,
             out, scale, idx_width):
    torch = _torch()
    n = boxes.shape[0]
    if out is None:
        out = torch.empty((n, 256 * S * S), dtype=torch.float32, device=boxes.device)
    if scale is None:
        scale = torch.empty(n, dtype=torch.int32, device=boxes.device)
    idx = torch.empty((n, S, S, idx_width), dtype=torch.int32, device=boxes.device) if want_idx else None
    geom = (dn_scale_geom * len(plan.geom))(*plan.geom)
    cd = (dn_plane_desc * len(conv5_desc))(*conv5_desc)
    check(fn(_ptr(conv5), cd, len(conv5_desc), dtype, geom, len(plan.geom), pad, planes_per_img,
             _ptr(boxes), _ptr(box_img), n, target, S, _ptr(out), _ptr(scale), _ptr(idx), _stream()))
    return out, scale, idx


def densenet_region_windows(conv5, conv5_desc, dtype: int, plan: PlanResult, pad: int, planes_per_img,
                            boxes, box_img=None, target=227.0, S=6, want_idx=False, out=None,
                            scale=None):
    """Region windows (Sec. 4, crop after): bilinear samples at the S x S bin centres of each box."""
    return _regions(lib().densenet_region_windows, conv5, conv5_desc, dtype, plan, pad, planes_per_img,
                    boxes, box_img, target, S, want_idx, out, scale, 2)


def densenet_region_pool(conv5, conv5_desc, dtype: int, plan: PlanResult, pad: int, planes_per_img,
                         boxes, box_img=None, target=227.0, S=6, want_idx=False, out=None, scale=None):
    """Max-pooled region bins: per-channel max over the conv5 cells centred inside each of the S x S
    bins of each box (idx: first/last row, first/last column of each bin)."""
    return _regions(lib().densenet_region_pool, conv5, conv5_desc, dtype, plan, pad, planes_per_img,
                    boxes, box_img, target, S, want_idx, out, scale, 4)


def densenet_warp_regions(images, boxes, dtype: int, S=227, mean=(0.0, 0.0, 0.0), box_img=None, out=None,
                          pitch=0):
    """Crop-before windows (Sec. 3.4 per-window baseline, Sec. 4): uint8 images [n_img][3][H][W], boxes
    [n][4] fp32 -> [n][3][S][pitch or S] mean-centred windows in `dtype` (columns past S are 0)."""
    torch = _torch()
    if images.dim() == 3:
        images = images[None]
    n_img, _, H, W = images.shape
    n = boxes.shape[0]
    P = pitch or S
    if out is None:
        out = torch.empty((n, 3, S, P), dtype=_tdtype(dtype), device=boxes.device)
    m = (ctypes.c_float * 3)(*[float(v) for v in mean])
    check(lib().densenet_warp_regions(_ptr(images), n_img, H, W, _ptr(boxes), _ptr(box_img), n, S, pitch, m,
                                      dtype, _ptr(out), out.numel() * out.element_size(),
                                      ctypes.byref(ctypes.c_size_t()), _stream()))
    return out


class PerWindow:
    """The per-window baseline (Sec. 3.4): every box warped to S x S on its own, then the whole conv stack
    with pool5 on each window as an independent plane (one launch per layer over all windows).  The
    per-window descriptor is the window's pool5 map, [n][Hp][Wp][256] (6 x 6 x 256 at S = 227).
    Window rows are padded to a multiple of 8 elements (zeros past S) so that conv1 loads them straight
    into LDS; the padding never reaches a stored output."""

    def __init__(self, n: int, dtype: int, S=227, device="cuda", net=None):
        torch = _torch()
        self.n, self.S, self.dtype = n, S, dtype
        self.pitch = (S + 7) // 8 * 8
        net = net or net_params(pool5=True)
        net.pool5 = 1
        desc = []
        for i in range(n):
            q = dn_plane_desc()
            q.h, q.w, q.offset, q.pitch = S, S, i * 3 * S * self.pitch, self.pitch
            desc.append(q)
        self.windows = torch.empty((n, 3, S, self.pitch), dtype=_tdtype(dtype), device=device)
        self.conv = ConvFeatures(desc, dtype, net, device=device)
        hp = self.conv.p5d[0]
        self.pool5_shape = (n, hp.h, hp.w, 256)

    def __call__(self, images, boxes, packed, mean=(0.0, 0.0, 0.0), box_img=None):
        densenet_warp_regions(images, boxes, self.dtype, self.S, mean, box_img, out=self.windows,
                              pitch=self.pitch)
        self.conv(self.windows, packed)
        return self.conv.pool5[: self.pool5_shape[0] * self.pool5_shape[1] * self.pool5_shape[2] * 256].view(
            self.pool5_shape)


def densenet_conv_layer(layer: int, x, n: int, H: int, W: int, dtype: int, packed):
    torch = _torch()
    hw = layer_sizes(H, W, strict=False) if layer == 1 else None
    M = (96, 256, 384, 384, 256)[layer - 1]
    Ho, Wo = (hw[0] if layer == 1 else (H, W))
    out = torch.empty((n, Ho, Wo, M), dtype=_tdtype(dtype), device=x.device)
    check(lib().densenet_conv_layer(layer, _ptr(x), n, H, W, dtype, _ptr(packed), _ptr(out), _stream()))
    return out


def _pool_side(v):
    return (v - 2) // 2 + 1 if v >= 2 else 0


def densenet_lrn_pool(x, dtype: int, net: dn_net_params):
    torch = _torch()
    n, H, W, C = x.shape
    out = torch.empty((n, _pool_side(H), _pool_side(W), C), dtype=_tdtype(dtype), device=x.device)
    check(lib().densenet_lrn_pool(_ptr(x), n, H, W, C, dtype, ctypes.byref(net), _ptr(out), _stream()))
    return out


def densenet_maxpool(x, dtype: int):
    torch = _torch()
    n, H, W, C = x.shape
    out = torch.empty((n, _pool_side(H), _pool_side(W), C), dtype=_tdtype(dtype), device=x.device)
    check(lib().densenet_maxpool(_ptr(x), n, H, W, C, dtype, _ptr(out), _stream()))
    return out


def layer_sizes(H: int, W: int, strict=True):
    hw = (ctypes.c_int32 * 16)()
    st = lib().densenet_layer_sizes(H, W, hw)
    if strict:
        check(st)
    return [(hw[2 * i], hw[2 * i + 1]) for i in range(8)]


def profile_start(names=None):
    """Trace launches (all, or those named in `names`) with events on their own streams."""
    check(lib().densenet_profile_start(",".join(names).encode() if names else None))


def profile_stop():
    """Stop tracing; returns {name: (launches, total_ms)} (waits for the traced launches)."""
    out = (dn_profile_entry * 64)()
    n = ctypes.c_int32()
    check(lib().densenet_profile_stop(out, 64, ctypes.byref(n)))
    return {out[i].name.decode(): (out[i].launches, out[i].total_ms) for i in range(min(n.value, 64))}


# ------------------------------------------------------------------------------------------------
# The paper's interface: pyra = convnet_featpyramid(image)
# ------------------------------------------------------------------------------------------------
@dataclass
class Pyramid:
    feat: list            # per scale: [rows][cols][256] view of its plane's conv5 map
    scales: np.ndarray    # [K] scale factors s_k
    plan: PlanResult
    planes: object        # the stitched planes tensor
    conv: ConvFeatures
    n_img: int


def convnet_featpyramid(images, p: dn_pyramid_params, packed, dtype: int, net=None) -> Pyramid:
    """Image(s) (uint8 device tensor [n][3][H][W]) -> per-scale conv5 maps (views) + geometry."""
    if images.dim() == 3:
        images = images[None]
    net = net or net_params()
    planes, plan = densenet_build_pyramid(images, p, dtype)
    n_img = images.shape[0]
    cf = densenet_conv_features(planes, plan.image_descs(n_img), dtype, packed, net)
    maps = cf.conv5_maps()
    feat = []
    npl = len(plan.planes)
    for b in range(n_img):
        for g in plan.geom:
            feat.append(maps[b * npl + g.plane][g.r0:g.r1 + 1, g.c0:g.c1 + 1])
    return Pyramid(feat, np.array([g.s for g in plan.geom]), plan, planes, cf, n_img)


def convnet_featpyramid_batch(images, p: dn_pyramid_params, packed, dtype: int, net=None,
                              plan: BatchPlan | None = None) -> Pyramid:
    """A batch of images stitched together (cross-image packing) -> per-(image, scale) conv5 maps
    (views, image-major) + the batch plan."""
    net = net or net_params()
    n_img, _, H, W = images.shape
    plan = plan or BatchPlan(n_img, H, W, p, device=images.device)
    planes = densenet_build_batch(images, plan, dtype)
    cf = densenet_conv_features(planes, plan.planes, dtype, packed, net)
    maps = cf.conv5_maps()
    feat = [maps[g.plane][g.r0:g.r1 + 1, g.c0:g.c1 + 1] for g in plan.geom]
    return Pyramid(feat, np.array([plan.geom[e].s for e in range(plan.E)]), plan, planes, cf, n_img)


# ------------------------------------------------------------------------------------------------
# A head learned on region descriptors: norm, softmax loss, AdamW
# ------------------------------------------------------------------------------------------------
_TYPES = None


def _types():
    """torch dtype -> dn_dtype, and back."""
    global _TYPES
    if _TYPES is None:
        torch = _torch()
        codes = {torch.float32: DN_F32, torch.float16: DN_F16, torch.bfloat16: DN_BF16,
                 torch.float8_e4m3fn: DN_F8}
        _TYPES = codes, {c: t for t, c in codes.items()}
    return _TYPES


def _bad(msg):
    return DenseNetError(DN_E_INVALID_ARG, msg)


def _code(t, what):
    code = _types()[0].get(t.dtype, DN_F8)
    if code == DN_F8:
        raise DenseNetError(DN_E_UNSUPPORTED, f"{what}: fp32, fp16 or bf16 expected, not {t.dtype}")
    return code


def _rows(t, what, shape=None, dtype=None, device=None):
    """Checks a matrix of rows (elements of a row next to each other, rows any distance apart); returns its
    address and row stride."""
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise _bad(f"{what}: a matrix{'' if shape is None else f' of {shape[0]} x {shape[1]}'} expected, not "
                   f"{tuple(size)}")
    if dtype is not None and t.dtype != dtype:
        raise _bad(f"{what}: {dtype} expected, not {t.dtype}")
    if size[1] >= 1 << 31:  # (a C int would take the low 32 bits)
        raise DenseNetError(DN_E_TOO_LARGE, f"{what}: rows of {size[1]} values")
    if (t.device != device) if device is not None else not t.is_cuda:
        raise _bad(f"{what}: not on the operands' GPU")
    row, col = t.stride()
    if col != 1 and size[1] > 1:
        raise _bad(f"{what}: the elements of a row must be next to each other")
    return t.data_ptr(), row if size[0] > 1 else size[1]


def _vector(t, what, n, dtype, device):
    if t is None:
        return None
    if t.shape != (n,) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise _bad(f"{what}: {n} contiguous {dtype} values on the operands' GPU expected")
    return t.data_ptr()


def _on(device):
    """The device's current stream; the device has to be the current one (the library launches there)."""
    torch = _torch()
    if device.index != torch.cuda.current_device():
        raise _bad("the operands are not on the current GPU")
    # the stream's address without a Stream object around it, 2 us less in a call of 13
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream


@functools.lru_cache(maxsize=1024)
def _work_bytes(entry, *args):
    """The workspace that an entry point asks for: its size query, whose answer depends on sizes, strides and alignment."""
    need = ctypes.c_size_t()
    check(getattr(lib(), entry)(*args, None, 0, ctypes.byref(need), None))
    return need.value


def densenet_rms_norm(x, gamma=None, residual=None, eps=1e-6, out_dtype=None, block=0, out=None, sum_out=None,
                      scale=None):
    """Root-mean-square norm of the rows of s = x + residual.  x, residual: [n][C] (fp32, fp16 or bf16); gamma: fp32
    [C].  out_dtype: DN_F32, DN_F16, DN_BF16 or DN_F8 (x's own by default); with DN_F8 a scale for every `block` values
    of a row (0: the row).  Returns (y, s, scale): s is None without a residual or sum_out, scale without DN_F8."""
    torch = _torch()
    dt = _code(x, "x")
    xp, xs = _rows(x, "x")
    n, C = x.shape
    dev = x.device
    ydt = dt if out_dtype is None else out_dtype
    yt = _types()[1].get(ydt)
    if yt is None:
        raise DenseNetError(DN_E_UNSUPPORTED, f"out_dtype {ydt}")
    if block not in (0, 32, 64, 128) or (block and ydt != DN_F8):
        raise DenseNetError(DN_E_UNSUPPORTED, "block: 0, or 32, 64 or 128 with DN_F8")
    rp, rs = (None, 0) if residual is None else _rows(residual, "residual", (n, C), x.dtype, dev)
    if residual is not None and sum_out is None:
        sum_out = torch.empty((n, C), dtype=x.dtype, device=dev)
    sp, ss = (None, 0) if sum_out is None else _rows(sum_out, "sum_out", (n, C), x.dtype, dev)
    if out is None:
        out = torch.empty((n, C), dtype=yt, device=dev)
    yp, ys = _rows(out, "out", (n, C), yt, dev)
    kp = None
    if ydt == DN_F8:
        blocks = -(-C // block) if block else 1
        if scale is None:
            scale = torch.empty((n, blocks), dtype=torch.float32, device=dev)
        if tuple(scale.shape) != (n, blocks) or scale.dtype != torch.float32 or scale.device != dev or \
                not scale.is_contiguous():
            raise _bad(f"scale: contiguous fp32 [{n}][{blocks}] on the operands' GPU expected")
        kp = scale.data_ptr()
    elif scale is not None:
        raise _bad("scale belongs to an 8-bit output")
    check(lib().densenet_rms_norm(xp, xs, rp, rs, _vector(gamma, "gamma", C, torch.float32, dev), n, C, dt, eps, sp, ss,
                                  yp, ys, ydt, block, kp, _on(dev)))
    return out, sum_out, scale


def densenet_rms_norm_backward(dy, s, gamma=None, dsum=None, eps=1e-6, dx=None, dgamma=None):
    """Gradient of densenet_rms_norm at s (its second result, or x without a residual), from dy and from dsum, the
    gradient that reaches s past the norm.  Returns (dx, dgamma); dx is the residual's gradient too."""
    torch = _torch()
    dt, ddt = _code(s, "s"), _code(dy, "dy")
    sp, ss = _rows(s, "s")
    n, C = s.shape
    dev = s.device
    dp, ds = _rows(dy, "dy", (n, C), None, dev)
    ep, es = (None, 0) if dsum is None else _rows(dsum, "dsum", (n, C), s.dtype, dev)
    if dx is None:
        dx = torch.empty((n, C), dtype=s.dtype, device=dev)
    xp, xs = _rows(dx, "dx", (n, C), s.dtype, dev)
    if dgamma is None:
        dgamma = torch.empty(C, dtype=torch.float32, device=dev)
    gp = _vector(gamma, "gamma", C, torch.float32, dev)
    op = _vector(dgamma, "dgamma", C, torch.float32, dev)
    # (the size depends on n and C alone, after the checks of both)
    need = _work_bytes("densenet_rms_norm_backward", None, 0, ddt, None, 0, None, 0, None, n, C, dt, eps, None, 0, None)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    check(lib().densenet_rms_norm_backward(dp, ds, ddt, sp, ss, ep, es, gp, n, C, dt, eps, xp, xs, op, ws.data_ptr(), need, None,
                                           _on(dev)))
    return dx, dgamma


def _loss_operands(h, w, labels):
    torch = _torch()
    dt = _code(h, "h")
    hp, hs = _rows(h, "h")
    n, C = h.shape
    dev = h.device
    if w.dim() != 2:
        raise _bad("w: a matrix expected")
    V = w.shape[0]
    if V >= 1 << 31:
        raise DenseNetError(DN_E_TOO_LARGE, f"w: {V} words")
    wp, ws = _rows(w, "w", (V, C), h.dtype, dev)
    return (hp, hs, wp, ws, _vector(labels, "labels", n, torch.int64, dev)), n, C, V, dt, dev


def _any_address(ops):
    """h, w and labels as a size query sees them: addresses of the same alignment (to 16 bytes) in place of their own."""
    hp, hs, wp, ws, lp = ops
    return 4096 + hp % 16 if hp else None, hs, 4096 + wp % 16, ws, lp and 4096


def densenet_softmax_loss(h, w, labels, loss=None, lse=None):
    """Softmax cross entropy of the rows of h [n][C] over the words of w [V][C].  labels: int64 [n]; outside [0, V) a row
    is masked (loss 0).  Returns (loss [n], lse [n]) in fp32, not reduced."""
    torch = _torch()
    ops, n, C, V, dt, dev = _loss_operands(h, w, labels)
    loss = torch.empty(n, dtype=torch.float32, device=dev) if loss is None else loss
    lse = torch.empty(n, dtype=torch.float32, device=dev) if lse is None else lse
    at = _any_address(ops)
    need = _work_bytes("densenet_softmax_loss", *at, n, C, V, dt, None, None)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    check(lib().densenet_softmax_loss(*ops, n, C, V, dt, _vector(loss, "loss", n, torch.float32, dev),
                                      _vector(lse, "lse", n, torch.float32, dev), ws.data_ptr(), need, None, _on(dev)))
    return loss, lse


def densenet_softmax_loss_backward(h, w, labels, lse, dloss=None, scale=1.0, dh=None, dw=None):
    """Gradient of densenet_softmax_loss, from its lse: dloss, fp32 [n], or None for the mean over the unmasked rows,
    times scale.  Returns (dh, dw) in h's type."""
    torch = _torch()
    ops, n, C, V, dt, dev = _loss_operands(h, w, labels)
    dh = torch.empty((n, C), dtype=h.dtype, device=dev) if dh is None else dh
    dw = torch.empty((V, C), dtype=h.dtype, device=dev) if dw is None else dw
    at = _any_address(ops)
    need = _work_bytes("densenet_softmax_loss_backward", *at, None, None, 1.0, n, C, V, dt, None, 0, None, 0)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    check(lib().densenet_softmax_loss_backward(
        *ops, _vector(lse, "lse", n, torch.float32, dev), _vector(dloss, "dloss", n, torch.float32, dev), scale, n, C, V, dt,
        *_rows(dh, "dh", (n, C), h.dtype, dev), *_rows(dw, "dw", (V, C), h.dtype, dev), ws.data_ptr(), need, None, _on(dev)))
    return dh, dw


class AdamWPlan:
    """Tensors that step together: parameters (one type, updated in place), their gradients' buffers (one type), 16-bit
    copies of the parameters (optional; None entries allowed, and so is a parameter that is its own copy, as
    `p.to(torch.bfloat16)` gives of a bf16 one: nothing else is written for it; copies in fp32 are refused here), and the
    optimiser's states.  state_bits: 32, or 8 (DN_F8 codes with a scale per 256 values); states are made as zeros, or given (m, v, and m_scale, v_scale in 8 bits): tensor
    i's start at value ADAMW_BLOCK * blocks[i]."""

    def __init__(self, params, grads, m=None, v=None, m_scale=None, v_scale=None, copies=None, state_bits=None):
        torch = _torch()
        self.params, self.grads = list(params), list(grads)
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        if not self.params or len(self.grads) != len(self.params) or len(self.copies) != len(self.params):
            raise _bad("as many gradients (and copies) as parameters expected, one at least")
        self.device = self.params[0].device
        self.blocks, self.n_blocks = [], 0
        for p in self.params:
            self.blocks.append(self.n_blocks)
            self.n_blocks += -(-p.numel() // ADAMW_BLOCK)
        total = self.n_blocks * ADAMW_BLOCK
        if state_bits is None:
            state_bits = 8 if m is not None and m.dtype == torch.float8_e4m3fn else 32
        if state_bits not in (8, 32):
            raise DenseNetError(DN_E_UNSUPPORTED, "state_bits must be 8 or 32")
        self.state_bits = state_bits
        st = torch.float8_e4m3fn if state_bits == 8 else torch.float32

        def state(t, what, n, dtype):
            if t is None:
                return torch.zeros(n * dtype.itemsize, dtype=torch.uint8, device=self.device).view(dtype)
            _vector(t, what, n, dtype, self.device)
            return t

        self.m, self.v = state(m, "m", total, st), state(v, "v", total, st)
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale = state(m_scale, "m_scale", self.n_blocks, torch.float32)
            self.v_scale = state(v_scale, "v_scale", self.n_blocks, torch.float32)
        elif m_scale is not None or v_scale is not None:
            raise _bad("scales belong to 8-bit states")
        self.p_dtype = _code(self.params[0], "params")
        self.copies = [None if c is not None and (c.data_ptr(), c.dtype, c.shape, c.stride()) == (p.data_ptr(), p.dtype, p.shape, p.stride())
                       else c for c, p in zip(self.copies, self.params)]
        given = [c for c in self.copies if c is not None]
        self.copy_dtype = _code(given[0], "copies") if given else DN_BF16
        if self.copy_dtype not in (DN_F16, DN_BF16):
            raise DenseNetError(DN_E_UNSUPPORTED, "copies: bf16 or fp16")
        self.table = (dn_adamw_tensor * len(self.params))()
        for e, p, c, b in zip(self.table, self.params, self.copies, self.blocks):
            self._fits(p, "params", p, self.params[0])
            if c is not None:
                self._fits(c, "copies", p, given[0])
            e.p, e.copy, e.n, e.block = p.data_ptr(), None if c is None else c.data_ptr(), p.numel(), b
        self.set_grads(self.grads)

    def _fits(self, t, what, p, first):
        if t.dtype != first.dtype or t.numel() != p.numel() or t.device != self.device or not t.is_cuda or \
                not t.is_contiguous():
            raise _bad(f"{what}: contiguous tensors of one type on one GPU, as large as their parameters, expected")

    def set_grads(self, grads):
        """Takes the gradients of the following steps from other tensors."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise _bad("as many gradients as parameters expected")
        for g, p in zip(grads, self.params):
            self._fits(g, "grads", p, grads[0])
        self.grads, self.g_dtype = grads, _code(grads[0], "grads")
        for e, g in zip(self.table, grads):
            e.g = g.data_ptr()


def densenet_adamw(plan: AdamWPlan, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0,
                   seed=0):
    """One AdamW step (the `step`-th, from 1) over a plan's tensors.  seed: of the 8-bit states' rounding, another one
    every step."""
    k = dn_adamw_params(lr, beta1, beta2, eps, weight_decay, grad_scale, step, seed & 0xFFFFFFFF, plan.state_bits)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    check(lib().densenet_adamw(plan.table, len(plan.table), plan.p_dtype, plan.g_dtype, plan.copy_dtype, ctypes.byref(k),
                               ptr(plan.m), ptr(plan.v), ptr(plan.m_scale), ptr(plan.v_scale), plan.n_blocks,
                               _on(plan.device)))


# ------------------------------------------------------------------------------------------------
# A head in 8 bits
# ------------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _no_workspace(device):
    return _torch().empty(DN_NO_WORKSPACE, dtype=_torch().uint8, device=device)


def _workspace(need, device):
    """A call's workspace: one for all calls that leave it alone."""
    return _no_workspace(device) if need == DN_NO_WORKSPACE else _torch().empty(need, dtype=_torch().uint8, device=device)


def _codes(shape, device):
    """Codes in rows that start on 16 bytes, which products read as they lie."""
    torch = _torch()
    n, C = shape
    return torch.empty((n, -(-C // 16) * 16), dtype=torch.float8_e4m3fn, device=device)[:, :C]


def _scales(t, what, shape, device):
    torch = _torch()
    if t is None:
        return torch.empty(shape, dtype=torch.float32, device=device)
    if tuple(t.shape) != shape or t.dtype != torch.float32 or t.device != device or not t.is_contiguous():
        raise _bad(f"{what}: contiguous fp32 {list(shape)} on the operands' GPU expected")
    return t


def densenet_quantize_blocks(x, rows=1, codes=True, turned=False, out=None, scale=None, turned_out=None, turned_scale=None):
    """Rows of x [n][C] as e4m3 codes, x = code * scale, with a scale for every 128 values of a row (rows=1) or every square of
    128 x 128 (rows=128).  Returns (codes [n][C], scale, turned [C][n], turned_scale): with codes=False or turned=False None in
    place of those; turned is the same of x's transpose, from one reading.  New codes lie in rows that start on 16 bytes."""
    torch = _torch()
    dt = _code(x, "x")
    xp, xs = _rows(x, "x")
    n, C = x.shape
    dev = x.device
    if rows not in (1, DN_SCALE_BLOCK):
        raise DenseNetError(DN_E_UNSUPPORTED, f"rows: 1 or {DN_SCALE_BLOCK}")
    codes, turned = codes or out is not None, turned or turned_out is not None
    if not codes and not turned:
        raise _bad("codes, turned or both")
    if (not codes and scale is not None) or (not turned and turned_scale is not None):
        raise _bad("scales belong to codes that are asked for")
    if n >= 1 << 31:
        raise DenseNetError(DN_E_TOO_LARGE, f"x: {n} rows")
    up = lambda v: -(-v // DN_SCALE_BLOCK)  # noqa: E731
    cp, cs, kp, tp, ts, tkp = None, 0, None, None, 0, None
    f8 = torch.float8_e4m3fn
    if codes:
        out = _codes((n, C), dev) if out is None else out
        cp, cs = _rows(out, "out", (n, C), f8, dev)
        scale = _scales(scale, "scale", (n if rows == 1 else up(n), up(C)), dev)
        kp = scale.data_ptr()
    if turned:
        turned_out = _codes((C, n), dev) if turned_out is None else turned_out
        tp, ts = _rows(turned_out, "turned_out", (C, n), f8, dev)
        turned_scale = _scales(turned_scale, "turned_scale", (C if rows == 1 else up(C), up(n)), dev)
        tkp = turned_scale.data_ptr()
    if n:
        check(lib().densenet_quantize_blocks(xp, xs, n, C, dt, rows, cp, cs, kp, tp, ts, tkp, _on(dev)))
    return out, scale, turned_out, turned_scale


def densenet_block_product(a, a_scale, w, w_scale, out_dtype=DN_BF16, out=None):
    """y [n][V] = a w^T of e4m3 codes a [n][C] and w [V][C]: a_scale [n][ceil(C / 128)], a scale for every 128 values of a row;
    w_scale [ceil(V / 128)][ceil(C / 128)], one for every square of 128 x 128 (densenet_quantize_blocks with rows 1 and 128).
    out_dtype: DN_F32, summed in 32 bits all through, or DN_F16 or DN_BF16: of each eight products bits below 2^-13 of the largest
    one are left out, so that a sum of eight is off by up to 7 times that."""
    torch = _torch()
    f8 = torch.float8_e4m3fn
    ap, as_ = _rows(a, "a", None, f8)
    n, C = a.shape
    dev = a.device
    if w.dim() != 2:
        raise _bad("w: a matrix expected")
    V = w.shape[0]
    if V >= 1 << 31:
        raise DenseNetError(DN_E_TOO_LARGE, f"w: {V} rows")
    wp, ws_ = _rows(w, "w", (V, C), f8, dev)
    up = lambda v: -(-v // DN_SCALE_BLOCK)  # noqa: E731
    if a_scale is None or w_scale is None:
        raise _bad("codes need their scales")
    a_scale, w_scale = _scales(a_scale, "a_scale", (n, up(C)), dev), _scales(w_scale, "w_scale", (up(V), up(C)), dev)
    yt = _types()[1].get(out_dtype)
    if yt is None or out_dtype == DN_F8:
        raise DenseNetError(DN_E_UNSUPPORTED, f"out_dtype {out_dtype}")
    out = torch.empty((n, V), dtype=yt, device=dev) if out is None else out
    yp, ys = _rows(out, "out", (n, V), yt, dev)
    # (the size depends on the codes' alignment: addresses of the same one in place of their own)
    need = _work_bytes("densenet_block_product", 4096 + ap % 16 if ap else None, as_, None, 4096 + wp % 16, ws_, None, n, C, V, None, 0,
                       out_dtype)
    ws = _workspace(need, dev)
    check(lib().densenet_block_product(ap, as_, a_scale.data_ptr(), wp, ws_, w_scale.data_ptr(), n, C, V, yp, ys, out_dtype,
                                       ws.data_ptr(), need, None, _on(dev)))
    return out


def _top_buffers(ids, logp, n, top, dev, make):
    torch = _torch()
    if top == 0:
        if ids is not None or logp is not None:
            raise _bad("ids and their values belong to top > 0")
        return None, None
    for t, what, dtype in ((ids, "ids", torch.int64), (logp, "their values", torch.float32)):
        if t is not None and (tuple(t.shape) != (n, top) or t.dtype != dtype or t.device != dev or not t.is_contiguous()):
            raise _bad(f"{what}: contiguous {dtype} [{n}][{top}] on the operands' GPU expected")
    if make:
        ids = torch.empty((n, top), dtype=torch.int64, device=dev) if ids is None else ids
        logp = torch.empty((n, top), dtype=torch.float32, device=dev) if logp is None else logp
    return ids, logp


def densenet_token_scores(logits, tokens=None, top=0, scale=1.0, logp=None, entropy=None, lse=None, top_id=None, top_logp=None):
    """Log probability of each row's token, entropy, log of the sum of exponentials, and the `top` (up to 64) best alternatives of
    logits [n][V] times scale.  tokens: int64 [n], or None (then logp is 0 where given, else None); a token outside [0, V): logp 0.
    Of equal logits the lower index comes first; -infinity is no alternative (id -1).  Returns (logp, entropy, lse, top_id,
    top_logp), the last two None with top=0."""
    torch = _torch()
    dt = _code(logits, "logits")
    xp, xs = _rows(logits, "logits")
    n, V = logits.shape
    dev = logits.device
    if not 0 <= top <= DN_MAX_TOP:
        raise DenseNetError(DN_E_UNSUPPORTED, f"top: 0 .. {DN_MAX_TOP}")
    new = lambda t: torch.empty(n, dtype=torch.float32, device=dev) if t is None else t  # noqa: E731
    entropy, lse = new(entropy), new(lse)
    if tokens is not None:
        logp = new(logp)
    top_id, top_logp = _top_buffers(top_id, top_logp, n, top, dev, True)
    vec = lambda t, what: _vector(t, what, n, torch.float32, dev)  # noqa: E731
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    need = _work_bytes("densenet_token_scores", 4096, V, None, n, V, dt, 1.0, top, None, None, None, None, None)
    ws = _workspace(need, dev)
    check(lib().densenet_token_scores(xp, xs, _vector(tokens, "tokens", n, torch.int64, dev), n, V, dt, scale, top, vec(logp, "logp"),
                                      vec(entropy, "entropy"), vec(lse, "lse"), ptr(top_id), ptr(top_logp), ws.data_ptr(), need, None,
                                      _on(dev)))
    return logp, entropy, lse, top_id, top_logp


def densenet_token_scores_backward(logits, tokens, lse, entropy=None, dlogp=None, dentropy=None, dlse=None, top_id=None, dtop=None,
                                   scale=1.0, out=None):
    """Gradient of densenet_token_scores by the logits, from its results and from the gradients of each of them (None: 0; dtop
    [n][top] belongs to top_id's log probabilities).  Returns dlogits in the logits' type; out may be the logits themselves."""
    torch = _torch()
    dt = _code(logits, "logits")
    xp, xs = _rows(logits, "logits")
    n, V = logits.shape
    dev = logits.device
    top = 0 if dtop is None else dtop.shape[1] if dtop.dim() == 2 else -1
    if not 0 <= top <= DN_MAX_TOP:
        raise DenseNetError(DN_E_UNSUPPORTED, f"dtop: up to {DN_MAX_TOP} alternatives of each row")
    if top and top_id is None:
        raise _bad("dtop needs top_id")
    ids, vals = _top_buffers(top_id if top else None, dtop if top else None, n, top, dev, False)
    out = torch.empty((n, V), dtype=logits.dtype, device=dev) if out is None else out
    op, os_ = _rows(out, "out", (n, V), logits.dtype, dev)
    vec = lambda t, what: _vector(t, what, n, torch.float32, dev)  # noqa: E731
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    check(lib().densenet_token_scores_backward(
        xp, xs, _vector(tokens, "tokens", n, torch.int64, dev), vec(lse, "lse"), vec(entropy, "entropy"), vec(dlogp, "dlogp"),
        vec(dentropy, "dentropy"), vec(dlse, "dlse"), ptr(ids), ptr(vals), n, V, dt, scale, top, op, os_, _on(dev)))
    return out


class MuonPlan:
    """Matrices that step together by Muon: parameters (one type, updated in place), their gradients' buffers (one type), momentum
    (fp32, made as zeros if not given), 16-bit copies of the parameters (optional; None entries allowed, and so is a parameter that
    is its own copy, as `p.to(torch.bfloat16)` gives of a bf16 one: nothing else is written for it), and a rate for each that
    multiplies the learning rate (by default 0.2 sqrt(max(rows, cols)), which gives updates of AdamW's size).  parts: fp16 parts of
    a value in the products (0: 1 for bf16 parameters, else 2).  Nothing that is stepped may meet another tensor of the plan in
    memory."""

    def __init__(self, params, grads, momentum=None, copies=None, rates=None, parts=0):
        torch = _torch()
        self.params, self.parts = list(params), parts
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        if not self.params or len(self.copies) != len(self.params):
            raise _bad("as many copies as parameters expected, one at least")
        if parts not in (0, 1, 2):
            raise DenseNetError(DN_E_UNSUPPORTED, "parts: 0, 1 or 2")
        self.device = self.params[0].device
        self.p_dtype = _code(self.params[0], "params")
        self.copies = [None if c is not None and (c.data_ptr(), c.dtype, c.shape, c.stride()) == (p.data_ptr(), p.dtype, p.shape, p.stride())
                       else c for c, p in zip(self.copies, self.params)]
        given = [c for c in self.copies if c is not None]
        self.copy_dtype = _code(given[0], "copies") if given else DN_BF16
        if self.copy_dtype not in (DN_F16, DN_BF16):
            raise DenseNetError(DN_E_UNSUPPORTED, "copies: bf16 or fp16")
        if momentum is None:
            momentum = [torch.zeros(p.shape, dtype=torch.float32, device=self.device) for p in self.params]
        self.momentum = list(momentum)
        rates = [0.2 * max(p.shape) ** 0.5 if p.dim() == 2 else 0.0 for p in self.params] if rates is None else list(rates)
        if len(self.momentum) != len(self.params) or len(rates) != len(self.params):
            raise _bad("as much momentum and as many rates as parameters expected")
        self.work_bytes = {}  # of each number of parts, once it has been asked for
        self.table = (dn_muon_tensor * len(self.params))()
        for e, p, c, m, rate in zip(self.table, self.params, self.copies, self.momentum, rates):
            if p.dim() != 2 or p.numel() == 0:
                raise _bad("params: matrices expected")
            self._fits(p, "params", p, self.params[0].dtype)
            self._fits(m, "momentum", p, torch.float32)
            if c is not None:
                self._fits(c, "copies", p, given[0].dtype)
            e.p, e.copy, e.m = p.data_ptr(), None if c is None else c.data_ptr(), m.data_ptr()
            e.rows, e.cols, e.rate = p.shape[0], p.shape[1], rate
        self._held = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self.params + self.momentum + given)
        if any(end > at for (_, end), (at, _) in zip(self._held, self._held[1:])):
            raise _bad("two of the tensors that are stepped meet in memory")
        self.set_grads(grads)

    def _fits(self, t, what, p, dtype):
        if t.dtype != dtype or t.shape != p.shape or t.device != self.device or not t.is_cuda or not t.is_contiguous():
            raise _bad(f"{what}: contiguous tensors of one type on one GPU, of their parameters' shapes, expected")

    def set_grads(self, grads):
        """Takes the gradients of the following steps from other tensors."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise _bad("as many gradients as parameters expected")
        for g, p in zip(grads, self.params):
            self._fits(g, "grads", p, grads[0].dtype)
            at = bisect.bisect_left(self._held, (g.data_ptr() + g.numel() * g.element_size(), 0))
            if at and self._held[at - 1][1] > g.data_ptr():
                raise _bad("a gradient meets a tensor that is stepped in memory")
        self.grads, self.g_dtype = grads, _code(grads[0], "grads")
        for e, g in zip(self.table, grads):
            e.g = g.data_ptr()


#: The usual coefficients of a Newton-Schulz step, which bring singular values to between 0.7 and 1.2 in five of them.
NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def densenet_muon(plan: MuonPlan, lr, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5, coefficients=NS_COEFFICIENTS, eps=1e-7,
                  grad_scale=1.0):
    """One Muon step over a plan's matrices: p = p (1 - lr weight_decay) - lr rate X, X the update orthogonalised by `steps`
    Newton-Schulz steps.  coefficients: (a, b, c) of all steps, or one such triple for each; they have to keep the update's singular
    values, at most 1 at first, below 4."""
    if not 1 <= steps <= DN_MAX_NS_STEPS:
        raise DenseNetError(DN_E_UNSUPPORTED, f"steps: 1 .. {DN_MAX_NS_STEPS}")
    each = [tuple(c) for c in coefficients] if hasattr(coefficients[0], "__len__") else [tuple(coefficients)] * steps
    if len(each) != steps or any(len(c) != 3 for c in each):
        raise _bad("coefficients: (a, b, c), or as many of these as steps, expected")
    k = dn_muon_params(lr, momentum, weight_decay, grad_scale, eps)
    for i, c in enumerate(each):
        k.coefficients[i][:] = c
    k.steps, k.nesterov, k.parts = steps, int(nesterov), plan.parts
    on = _on(plan.device)
    args = (plan.table, len(plan.table), plan.p_dtype, plan.g_dtype, plan.copy_dtype, ctypes.byref(k))
    need = plan.work_bytes.get(plan.parts)
    if need is None:
        asked = ctypes.c_size_t()
        check(lib().densenet_muon(*args, None, 0, ctypes.byref(asked), None))
        need = plan.work_bytes[plan.parts] = asked.value
    ws = _workspace(need, plan.device)
    check(lib().densenet_muon(*args, ws.data_ptr(), need, None, on))
