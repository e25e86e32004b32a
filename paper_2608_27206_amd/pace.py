"""ctypes binding of libpace.so (include/pace.h): argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their
device pointers and torch's current HIP stream to the C ABI, and returns the
output tensors it allocated with torch.  All arithmetic happens in the HIP
kernels; if the library is missing this module raises instead of computing
anything itself.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# PACE_LIB_PATH selects another build of the same library (the host-sanitized one of the C ABI
# tests); by default the in-tree libpace.so.
LIB_PATH = os.environ.get("PACE_LIB_PATH") or os.path.join(_HERE, "libpace.so")

_lib = None

c_int, c_size, c_double, c_float, c_void = (ctypes.c_int, ctypes.c_size_t, ctypes.c_double,
                                            ctypes.c_float, ctypes.c_void_p)
c_ll = ctypes.c_longlong
c_int_p = ctypes.POINTER(ctypes.c_int)

# name -> (restype, argtypes)
_PROTOS = {
    "pace_last_error": (ctypes.c_char_p, []),
    "pace_version": (c_int, []),
    "pace_keep_count": (c_int, [c_double, c_int]),
    "pace_keep_from_density": (c_int, [c_double, c_double, c_double, c_int]),
    "pace_apc_target_size": (c_int, [c_double, c_int, c_int, c_double, c_double, c_int, c_int_p,
                                     c_int_p]),
    "pace_apc_density_workspace_size": (c_size, [c_int, c_int, c_int]),
    "pace_apc_density": (c_int, [c_void, c_int, c_int, c_int, c_double, c_float, c_float, c_void,
                                 c_void, c_void, c_size, c_void]),
    "pace_apc_density_features_workspace_size": (c_size, [c_int, c_int]),
    "pace_apc_density_features": (c_int, [c_void, c_int, c_int, c_double, c_float, c_float, c_void,
                                          c_void, c_void, c_size, c_void]),
    "pace_apc_downsample": (c_int, [c_void, c_int, c_int, c_void, c_int, c_int, c_void]),
    "pace_apc_pixel_features": (c_int, [c_void, c_int, c_int, c_int, c_int, c_void, c_void]),
    "pace_apc_pixel_density_workspace_size": (c_size, [c_int, c_int, c_int, c_int]),
    "pace_apc_pixel_density": (c_int, [c_void, c_int, c_int, c_int, c_int, c_double, c_float, c_float,
                                       c_void, c_void, c_void, c_size, c_void]),
    "pace_apc_preview_workspace_size": (c_size, [c_int, c_int, c_int, c_int]),
    "pace_apc_preview": (c_int, [c_void, c_int, c_int, c_int, c_void, c_void, c_int, c_int, c_void, c_void,
                                 c_void, c_size, c_void]),
    "pace_gemm_bf16": (c_int, [c_void, c_void, c_void, c_void, c_void, c_int, c_int, c_int, c_int, c_void]),
    "pace_vit_attention_workspace_size": (c_size, [c_int, c_int, c_int, c_int, c_int]),
    "pace_vit_attention": (c_int, [c_void, c_void, c_void, c_int, c_int, c_int, c_void, c_int, c_int,
                                   c_float, c_void, c_void, c_void, c_void, c_size, c_void]),
    "pace_vit_attention_mass": (c_int, [c_void, c_void, c_int, c_int, c_int, c_void, c_int, c_int,
                                        c_float, c_void, c_void, c_void]),
    "pace_prefill_attention_workspace_size": (c_size, [c_int, c_int]),
    "pace_prefill_attention_with_mass": (c_int, [c_void, c_void, c_void, c_int, c_int, c_int, c_int,
                                                 c_void, c_int, c_int, c_void, c_void, c_void, c_int, c_int,
                                                 c_void, c_void, c_int, c_float, c_void, c_void,
                                                 c_void, c_void, c_size, c_void]),
    "pace_ddae_select_workspace_size": (c_size, [c_int, c_int]),
    "pace_ddae_select_varlen": (c_int, [c_void, c_int, c_int, c_void, c_void, c_int, c_int, c_int_p,
                                        c_int_p, c_int, c_float, c_float, c_void, c_size, c_void,
                                        c_void, c_void, c_void, c_void, c_size, c_void]),
    "pace_ddae_select": (c_int, [c_void, c_int, c_int, c_void, c_void, c_int, c_int, c_int, c_float,
                                 c_float, c_int, c_void, c_size, c_void, c_void, c_void, c_void,
                                 c_void, c_size, c_void]),
    "pace_ddae_select_noalloc_max_bytes": (c_size, []),
    "pace_ddae_select_varlen_noalloc": (c_int, [c_void, c_int, c_int, c_void, c_void, c_int, c_int, c_int_p,
                                                c_int_p, c_int, c_float, c_float, c_void, c_size, c_void,
                                                c_void, c_void, c_void, c_void]),
    "pace_topk_gather": (c_int, [c_void, c_int, c_int, c_void, c_size, c_void, c_void, c_void, c_size,
                                 c_void]),
    "pace_gather_rows": (c_int, [c_void, c_int, c_size, c_void, c_int, c_void, c_void]),
    "pace_cache_append": (c_int, [c_void, c_ll, c_void, c_ll, c_void, c_ll, c_int, c_int, c_void, c_void, c_int, c_int,
                                  c_int, c_void, c_void, c_int, c_void, c_int, c_int_p, c_void, c_void, c_void,
                                  c_void]),
    "pace_cache_attention_workspace_size": (c_size, [c_int] * 10),
    "pace_cache_attention": (c_int, [c_void, c_int, c_int, c_void, c_void, c_int, c_int, c_void, c_int, c_void, c_int,
                                     c_int, c_int, c_float, c_void, c_void, c_void, c_size, c_void]),
    "pace_gemm_w4_workspace_size": (c_size, [c_int, c_int, c_int]),
    "pace_gemm_w4": (c_int, [c_void, c_void, c_void, c_void, c_void, c_void, c_void, c_int, c_int, c_int, c_int, c_int,
                             c_void, c_size, c_void]),
    "pace_quantize_fp8": (c_int, [c_void, c_ll, c_int, c_int, c_int, c_void, c_void, c_void]),
    "pace_rmsnorm": (c_int, [c_void, c_ll, c_void, c_ll, c_void, c_float, c_int, c_int, c_void, c_void, c_void, c_void, c_void]),
    "pace_gemm_fp8_workspace_size": (c_size, [c_int] * 5),
    "pace_gemm_fp8": (c_int, [c_void, c_void, c_ll, c_void, c_void, c_void, c_void, c_void, c_void, c_int, c_int, c_int, c_int,
                              c_int, c_void, c_size, c_void]),
}

EXPORTED = tuple(_PROTOS.keys())


class PaceError(RuntimeError):
    pass


def lib():
    """Load libpace.so (built by paper_2608_27206_amd.build); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise PaceError(f"{LIB_PATH} is missing: run `python -m paper_2608_27206_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _PROTOS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(st: int, what: str):
    if st != 0:
        msg = lib().pace_last_error().decode(errors="replace")
        raise PaceError(f"{what} failed with status {st}: {msg}")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise PaceError("tensor must live on the GPU")
    if not t.is_contiguous():
        raise PaceError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(1, int(nbytes)), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- host helpers
def keep_count(ratio: float, n: int) -> int:
    return int(lib().pace_keep_count(float(ratio), int(n)))


def keep_from_density(rho: float, n: int, ratio_lo: float = 0.05, ratio_hi: float = 0.25) -> int:
    return int(lib().pace_keep_from_density(float(rho), float(ratio_lo), float(ratio_hi), int(n)))


def apc_target_size(rho: float, H: int, W: int, min_pixels: float, max_pixels: float, snap: int):
    oh, ow = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().pace_apc_target_size(float(rho), H, W, float(min_pixels), float(max_pixels), snap,
                                      ctypes.byref(oh), ctypes.byref(ow)), "pace_apc_target_size")
    return oh.value, ow.value


# ---------------------------------------------------------------- APC
def apc_density(img: torch.Tensor, patch: int = 14, tail_frac: float = 0.10, alpha: float = 0.6,
                gamma: float = 1.5, d_out: Optional[torch.Tensor] = None,
                rho_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """img: uint8 [H, W, 3] on the GPU.  Returns (rho [3] = rho_g, rho_d, rho; d [N]); phi = 1 - rho_g."""
    H, W, _ = img.shape
    N = (H // patch) * (W // patch)
    dev = img.device
    if d_out is None:
        d_out = torch.empty(N, dtype=torch.float32, device=dev)
    if rho_out is None:
        rho_out = torch.empty(3, dtype=torch.float32, device=dev)
    need = lib().pace_apc_density_workspace_size(H, W, patch)
    if workspace is None:
        workspace = _ws(need, dev)
    _check(lib().pace_apc_density(_ptr(img), H, W, patch, float(tail_frac), float(alpha),
                                  float(gamma), _ptr(d_out), _ptr(rho_out), _ptr(workspace),
                                  workspace.numel(), _stream()), "pace_apc_density")
    return rho_out, d_out


def apc_density_features(feat: torch.Tensor, tail_frac: float = 0.10, alpha: float = 0.6,
                         gamma: float = 1.5, d_out: Optional[torch.Tensor] = None,
                         rho_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """feat: bf16 [N, D] preview embeddings on the GPU.  Returns (rho [3] = rho_g, rho_d, rho;
    d [N])."""
    if feat.dtype != torch.bfloat16 or feat.dim() != 2:
        raise PaceError("feat must be a 2-D bfloat16 tensor")
    N, D = feat.shape
    dev = feat.device
    if d_out is None:
        d_out = torch.empty(N, dtype=torch.float32, device=dev)
    if rho_out is None:
        rho_out = torch.empty(3, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _ws(lib().pace_apc_density_features_workspace_size(N, D), dev)
    _check(lib().pace_apc_density_features(_ptr(feat), N, D, float(tail_frac), float(alpha),
                                           float(gamma), _ptr(d_out), _ptr(rho_out), _ptr(workspace),
                                           workspace.numel(), _stream()), "pace_apc_density_features")
    return rho_out, d_out


PIXEL_STATISTICS = {"rgb": 0, "entropy": 1, "edges": 2, "laplacian": 3}


def pixel_feature_dim(kind: int, patch: int) -> int:
    return (6, 64, 8, patch * patch)[kind]


def apc_pixel_features(img: torch.Tensor, kind: int, patch: int = 14,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """img: uint8 [H, W, 3] on the GPU.  Returns fp32 [N, dim] pixel-statistic preview vectors."""
    if img.dtype != torch.uint8 or img.dim() != 3 or img.shape[2] != 3:
        raise PaceError("img must be a uint8 [H, W, 3] tensor")
    H, W, _ = img.shape
    if not 0 <= kind <= 3:
        raise PaceError(f"kind={kind} not in 0..3")
    N = (H // patch) * (W // patch)
    if out is None:
        out = torch.empty(N, pixel_feature_dim(kind, patch), dtype=torch.float32, device=img.device)
    _check(lib().pace_apc_pixel_features(_ptr(img), H, W, patch, kind, _ptr(out), _stream()),
           "pace_apc_pixel_features")
    return out


def apc_pixel_density(img: torch.Tensor, kind: int, patch: int = 14, tail_frac: float = 0.10,
                      alpha: float = 0.6, gamma: float = 1.5, d_out: Optional[torch.Tensor] = None,
                      rho_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """APC density with a pixel-statistic preview.  Returns (rho [3]: rho_g, rho_d, rho; d [N])."""
    if img.dtype != torch.uint8 or img.dim() != 3 or img.shape[2] != 3:
        raise PaceError("img must be a uint8 [H, W, 3] tensor")
    H, W, _ = img.shape
    N = (H // patch) * (W // patch)
    dev = img.device
    if d_out is None:
        d_out = torch.empty(max(N, 1), dtype=torch.float32, device=dev)
    if rho_out is None:
        rho_out = torch.empty(3, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _ws(lib().pace_apc_pixel_density_workspace_size(H, W, patch, kind), dev)
    _check(lib().pace_apc_pixel_density(_ptr(img), H, W, patch, kind, float(tail_frac), float(alpha),
                                        float(gamma), _ptr(d_out), _ptr(rho_out), _ptr(workspace),
                                        workspace.numel(), _stream()), "pace_apc_pixel_density")
    return rho_out, d_out


class PreviewWeights(ctypes.Structure):
    """Mirror of pace_preview_weights (include/pace.h)."""
    _fields_ = [("pe", c_void), ("g1", c_void), ("wq", c_void), ("wk", c_void), ("wv", c_void),
                ("bq", c_void), ("bk", c_void), ("bv", c_void), ("wo", c_void), ("bo", c_void),
                ("g2", c_void), ("wgu", c_void), ("bgu", c_void), ("wd", c_void), ("bd", c_void),
                ("dim", c_int), ("ffn", c_int)]


def preview_weights_to_device(w: dict, device) -> dict:
    """Device copies of preview-block weights in the layout pace_apc_preview reads: bf16 bit
    arrays (uint16) and fp32 vectors as given; the patch embedding zero-padded to a multiple of
    8 columns, the hidden units zero-padded to a multiple of 8, gate and up rows interleaved.
    (Marshalling only: zero padding and row order leave the block's function unchanged.)"""
    import numpy as np

    def bf(a):
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).to(device)

    def f32(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)

    D, kin = w["pe"].shape
    F = w["wg"].shape[0]
    kp = (kin + 7) // 8 * 8
    F8 = (F + 7) // 8 * 8
    pe = np.zeros((D, kp), np.uint16)
    pe[:, :kin] = w["pe"]
    wgu = np.zeros((2 * F8, D), np.uint16)
    wgu[0:2 * F:2] = w["wg"]
    wgu[1:2 * F:2] = w["wu"]
    bgu = np.zeros(2 * F8, np.float32)
    bgu[0:2 * F:2] = w["bg"]
    bgu[1:2 * F:2] = w["bu"]
    wd = np.zeros((D, F8), np.uint16)
    wd[:, :F] = w["wd"]
    out = {"pe": bf(pe), "wgu": bf(wgu), "bgu": f32(bgu), "wd": bf(wd), "dim": D, "ffn": F8}
    for k in ("wq", "wk", "wv", "wo"):
        out[k] = bf(w[k])
    for k in ("g1", "g2", "bq", "bk", "bv", "bo", "bd"):
        out[k] = f32(w[k])
    return out


def apc_preview(img: torch.Tensor, patch: int, token_patch: torch.Tensor, cu_windows: torch.Tensor,
                max_window: int, wdev: dict, out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The preview block's token embeddings, bf16 [N, D]; wdev from preview_weights_to_device."""
    H, W, _ = img.shape
    N = (H // patch) * (W // patch)
    D, F = wdev["dim"], wdev["ffn"]
    dev = img.device
    if out is None:
        out = torch.empty((N, D), dtype=torch.bfloat16, device=dev)
    if workspace is None:
        workspace = _ws(lib().pace_apc_preview_workspace_size(N, D, F, patch), dev)
    pw = PreviewWeights(*(_ptr(wdev[k]) for k in ("pe", "g1", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "bo",
                                                  "g2", "wgu", "bgu", "wd", "bd")), D, F)
    nwin = cu_windows.numel() - 1
    _check(lib().pace_apc_preview(_ptr(img), H, W, patch, _ptr(token_patch), _ptr(cu_windows), nwin,
                                  int(max_window), ctypes.byref(pw), _ptr(out), _ptr(workspace),
                                  workspace.numel(), _stream()), "pace_apc_preview")
    return out


def gemm_bf16(a: torch.Tensor, b: torch.Tensor, bias: Optional[torch.Tensor] = None,
              residual: Optional[torch.Tensor] = None, epilogue: int = 0,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """C = a b^T (+ bias, + residual, or SwiGLU of interleaved columns); a [M, K], b [N, K] bf16."""
    M, K = a.shape
    N = b.shape[0]
    if out is None:
        out = torch.empty((M, N // 2 if epilogue == 2 else N), dtype=torch.bfloat16, device=a.device)
    _check(lib().pace_gemm_bf16(_ptr(a), _ptr(b), _ptr(bias), _ptr(residual), _ptr(out), M, N, K, int(epilogue),
                                _stream()), "pace_gemm_bf16")
    return out


def apc_downsample(src: torch.Tensor, oH: int, oW: int, dst: Optional[torch.Tensor] = None):
    H, W, _ = src.shape
    if dst is None:
        dst = torch.empty((oH, oW, 3), dtype=torch.uint8, device=src.device)
    _check(lib().pace_apc_downsample(_ptr(src), H, W, _ptr(dst), oH, oW, _stream()),
           "pace_apc_downsample")
    return dst


# ---------------------------------------------------------------- attention
def vit_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                  max_seglen: int, scale: Optional[float] = None, want_lse: bool = True,
                  want_mass: bool = True, o: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, mass: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None):
    """q, k, v: bf16 [N, H, d]; cu_seqlens int32 [nseg+1].  Returns (o, lse or None, mass or None)."""
    N, H, d = q.shape
    dev = q.device
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    if o is None:
        o = torch.empty_like(q)
    if want_lse and lse is None:
        lse = torch.empty((H, N), dtype=torch.float32, device=dev)
    if want_mass and mass is None:
        mass = torch.empty((H, N), dtype=torch.float32, device=dev)
    if not want_lse:
        lse = None
    if not want_mass:
        mass = None
    nseg = cu_seqlens.numel() - 1
    if workspace is None:
        # the library needs a workspace for LSE scratch (mass without lse) and for the fp16 V^T
        # tiles of the long-segment kernel; the size says which applies
        need = lib().pace_vit_attention_workspace_size(N, H, d, nseg, int(max_seglen))
        lse_scratch = (N * H * 4 + 255) // 256 * 256
        if (mass is not None and lse is None) or need > lse_scratch:
            workspace = _ws(need, dev)
    _check(lib().pace_vit_attention(_ptr(q), _ptr(k), _ptr(v), N, H, d, _ptr(cu_seqlens),
                                    cu_seqlens.numel() - 1, int(max_seglen), float(scale), _ptr(o),
                                    _ptr(lse), _ptr(mass), _ptr(workspace),
                                    0 if workspace is None else workspace.numel(), _stream()),
           "pace_vit_attention")
    return o, lse, mass


def vit_attention_mass(q: torch.Tensor, k: torch.Tensor, cu_seqlens: torch.Tensor, max_seglen: int,
                       lse: torch.Tensor, scale: Optional[float] = None,
                       mass: Optional[torch.Tensor] = None):
    """Mass pass alone from a given LSE [H, N].  Returns mass fp32 [H, N]."""
    N, H, d = q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    if mass is None:
        mass = torch.empty((H, N), dtype=torch.float32, device=q.device)
    _check(lib().pace_vit_attention_mass(_ptr(q), _ptr(k), N, H, d, _ptr(cu_seqlens),
                                         cu_seqlens.numel() - 1, int(max_seglen), float(scale),
                                         _ptr(lse), _ptr(mass), _stream()), "pace_vit_attention_mass")
    return mass


def prefill_attention_with_mass(q, k, v, cu_seqlens, max_seqlen: int, vis_len, cu_vis,
                                nvis_total: int, max_vis_len: int, mq_start, mq_len,
                                max_mq_len: int, scale: Optional[float] = None, want_mass=True,
                                o=None, lse=None, mass=None, workspace=None, vis_start=None):
    """Causal GQA prefill.  q bf16 [Ntot, Hq, d]; k, v bf16 [Ntot, Hkv, d]; metadata int32 on the
    GPU (vis_start None: visual tokens first).  Returns (o, lse [Hq, Ntot], mass [Hq, nvis_total]
    or None)."""
    Ntot, Hq, d = q.shape
    Hkv = k.shape[1]
    dev = q.device
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((Hq, Ntot), dtype=torch.float32, device=dev)
    if want_mass and mass is None:
        mass = torch.empty((Hq, max(1, nvis_total)), dtype=torch.float32, device=dev)
    if not want_mass:
        mass = None
    _check(lib().pace_prefill_attention_with_mass(
        _ptr(q), _ptr(k), _ptr(v), Ntot, Hq, Hkv, d, _ptr(cu_seqlens), cu_seqlens.numel() - 1,
        int(max_seqlen), _ptr(vis_start), _ptr(vis_len), _ptr(cu_vis), int(nvis_total), int(max_vis_len),
        _ptr(mq_start), _ptr(mq_len), int(max_mq_len), float(scale), _ptr(o), _ptr(lse),
        _ptr(mass), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()),
        "pace_prefill_attention_with_mass")
    return o, lse, mass


# ---------------------------------------------------------------- DDAE
def ddae_select(vis_mass: torch.Tensor, merge: int, vis_perm: Optional[torch.Tensor],
                llm_mass: torch.Tensor, nv: Sequence[int], keep: Sequence[int], mode: int = 0,
                tau: float = 0.5, w_llm_fixed: float = 0.5, hidden: Optional[torch.Tensor] = None,
                idx_out=None, score_out=None, fuse_out=None, out=None, workspace=None):
    """Segmented DDAE selection.  vis_mass fp32 [Hv, sum(nv)*merge]; llm_mass fp32 [Hl, sum(nv)];
    nv, keep: host lists.  Returns (idx int32 [sum keep], scores fp32 [sum nv], fuse fp32 [B, 4],
    gathered rows or None)."""
    B = len(nv)
    dev = llm_mass.device
    nv_total = int(sum(nv))
    ktot = int(sum(keep))
    Hv = vis_mass.shape[0]
    Hl = llm_mass.shape[0]
    if idx_out is None:
        idx_out = torch.empty(max(1, ktot), dtype=torch.int32, device=dev)
    if score_out is None:
        score_out = torch.empty(nv_total, dtype=torch.float32, device=dev)
    if fuse_out is None:
        fuse_out = torch.empty((B, 4), dtype=torch.float32, device=dev)
    row_bytes = 0
    if hidden is not None:
        row_bytes = hidden[0].numel() * hidden.element_size()
        if out is None:
            out = torch.empty((max(1, ktot),) + tuple(hidden.shape[1:]), dtype=hidden.dtype, device=dev)
    if workspace is None:
        workspace = _ws(lib().pace_ddae_select_workspace_size(nv_total, B), dev)
    nv_a = (ctypes.c_int * B)(*[int(x) for x in nv])
    kp_a = (ctypes.c_int * B)(*[int(x) for x in keep])
    _check(lib().pace_ddae_select_varlen(
        _ptr(vis_mass), Hv, merge, _ptr(vis_perm), _ptr(llm_mass), Hl, B, nv_a, kp_a, int(mode),
        float(tau), float(w_llm_fixed), _ptr(hidden), row_bytes, _ptr(idx_out), _ptr(score_out),
        _ptr(fuse_out), _ptr(out), _ptr(workspace), workspace.numel(), _stream()),
        "pace_ddae_select_varlen")
    return idx_out[:ktot], score_out, fuse_out, (out[:ktot] if out is not None else None)


def ddae_select_noalloc(vis_mass: torch.Tensor, merge: int, vis_perm: Optional[torch.Tensor],
                        llm_mass: torch.Tensor, nv: Sequence[int], keep: Sequence[int], mode: int = 0,
                        tau: float = 0.5, w_llm_fixed: float = 0.5, hidden: Optional[torch.Tensor] = None,
                        idx_out=None, score_out=None, fuse_out=None, out=None):
    """pace_ddae_select_varlen_noalloc: ddae_select without a workspace (the library's static
    per-GPU scratch); outputs are the caller's tensors, allocated here only when not given."""
    B = len(nv)
    dev = llm_mass.device
    nv_total = int(sum(nv))
    ktot = int(sum(keep))
    if idx_out is None:
        idx_out = torch.empty(max(1, ktot), dtype=torch.int32, device=dev)
    if score_out is None:
        score_out = torch.empty(nv_total, dtype=torch.float32, device=dev)
    if fuse_out is None:
        fuse_out = torch.empty((B, 4), dtype=torch.float32, device=dev)
    row_bytes = 0
    if hidden is not None:
        row_bytes = hidden[0].numel() * hidden.element_size()
        if out is None:
            out = torch.empty((max(1, ktot),) + tuple(hidden.shape[1:]), dtype=hidden.dtype, device=dev)
    nv_a = (ctypes.c_int * B)(*[int(x) for x in nv])
    kp_a = (ctypes.c_int * B)(*[int(x) for x in keep])
    _check(lib().pace_ddae_select_varlen_noalloc(
        _ptr(vis_mass), vis_mass.shape[0], merge, _ptr(vis_perm), _ptr(llm_mass), llm_mass.shape[0], B, nv_a,
        kp_a, int(mode), float(tau), float(w_llm_fixed), _ptr(hidden), row_bytes, _ptr(idx_out),
        _ptr(score_out), _ptr(fuse_out), _ptr(out), _stream()), "pace_ddae_select_varlen_noalloc")
    return idx_out[:ktot], score_out, fuse_out, (out[:ktot] if out is not None else None)


def ddae_select_one(vis_mass, merge, vis_perm, llm_mass, K: int, mode=0, tau=0.5, w_llm_fixed=0.5,
                    hidden=None, workspace=None):
    """Single-image pace_ddae_select."""
    Nv = llm_mass.shape[1]
    dev = llm_mass.device
    idx = torch.empty(max(1, K), dtype=torch.int32, device=dev)
    sc = torch.empty(Nv, dtype=torch.float32, device=dev)
    fz = torch.empty(4, dtype=torch.float32, device=dev)
    out = None
    row_bytes = 0
    if hidden is not None:
        row_bytes = hidden[0].numel() * hidden.element_size()
        out = torch.empty((max(1, K),) + tuple(hidden.shape[1:]), dtype=hidden.dtype, device=dev)
    if workspace is None:
        workspace = _ws(lib().pace_ddae_select_workspace_size(Nv, 1), dev)
    _check(lib().pace_ddae_select(_ptr(vis_mass), vis_mass.shape[0], merge, _ptr(vis_perm),
                                  _ptr(llm_mass), llm_mass.shape[0], Nv, int(mode), float(tau),
                                  float(w_llm_fixed), int(K), _ptr(hidden), row_bytes, _ptr(idx),
                                  _ptr(sc), _ptr(fz), _ptr(out), _ptr(workspace), workspace.numel(),
                                  _stream()), "pace_ddae_select")
    return idx[:K], sc, fz, (out[:K] if out is not None else None)


def topk_gather(scores: torch.Tensor, K: int, hidden: Optional[torch.Tensor] = None):
    N = scores.numel()
    dev = scores.device
    idx = torch.empty(max(1, K), dtype=torch.int32, device=dev)
    out = None
    row_bytes = 0
    if hidden is not None:
        row_bytes = hidden[0].numel() * hidden.element_size()
        out = torch.empty((max(1, K),) + tuple(hidden.shape[1:]), dtype=hidden.dtype, device=dev)
    _check(lib().pace_topk_gather(_ptr(scores), N, int(K), _ptr(hidden), row_bytes, _ptr(idx),
                                  _ptr(out), None, 0, _stream()), "pace_topk_gather")
    return idx[:K], (out[:K] if out is not None else None)


def gather_rows(src: torch.Tensor, idx: torch.Tensor, out: Optional[torch.Tensor] = None):
    """out[r] = src[idx[r]] (whole rows, bit for bit); src [rows, ...] with 16-byte rows."""
    n = idx.numel()
    if out is None:
        out = torch.empty((n,) + tuple(src.shape[1:]), dtype=src.dtype, device=src.device)
    row_bytes = src[0].numel() * src.element_size() if src.shape[0] > 0 else 0
    _check(lib().pace_gather_rows(_ptr(src), src.shape[0], row_bytes, _ptr(idx), n, _ptr(out),
                                  _stream()), "pace_gather_rows")
    return out


# ---------------------------------------------------------------- decode over a pruned context
# A decode step makes many short calls, so these marshal with as few Python operations as the checks allow.
class _KvCacheStruct(ctypes.Structure):
    """Mirror of pace_kv_cache (include/pace.h)."""
    _fields_ = [("k", c_void), ("v", c_void), ("k_scale", c_void), ("v_scale", c_void), ("num_pages", c_int),
                ("heads", c_int), ("page", c_int), ("dim", c_int), ("bits", c_int)]


_INT3 = ctypes.c_int * 3
_BF16, _F32, _I32, _U8, _E4M3 = (torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn)


def _arg(t: Optional[torch.Tensor], dtype, shape: tuple, device: int, name: str):
    """The address of a contiguous tensor of this type and shape on GPU number `device`, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise PaceError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on GPU {device}, not {t.dtype} "
                        f"{list(t.shape)} (strides {t.stride()}) on {t.device}")
    return t.data_ptr()


def _rows_arg(t: torch.Tensor, heads: int, dim: int, n: int, device: int, name: str):
    """Address and row stride of bf16 rows [n, heads, dim] whose heads lie one after the other."""
    if t.dtype is not _BF16 or t.shape != (n, heads, dim) or t.get_device() != device:
        raise PaceError(f"{name} must be bfloat16 [{n}, {heads}, {dim}] on GPU {device}, not {t.dtype} {list(t.shape)} on "
                        f"{t.device}")
    row, head, one = t.stride()
    if one != 1 or (heads > 1 and head != dim):
        raise PaceError(f"{name}: the heads of a row must lie one after the other, strides are {t.stride()}")
    return t.data_ptr(), (row if n > 1 else heads * dim)


def _scratch(workspace: Optional[torch.Tensor], device: int):
    """Address and bytes of a workspace (uint8, 1-D)."""
    if workspace is None:
        return None, 0
    return _arg(workspace, _U8, (workspace.numel(),), device, "workspace"), workspace.numel()


def _gpu_of(t: torch.Tensor) -> int:
    device = t.get_device()
    if device < 0:
        raise PaceError("tensor must live on the GPU")
    return device


# the current stream's address without a Stream object around it, where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _call(name: str, device: int, *args):
    """A library call on the current stream of GPU number `device`, made current for it if it is not."""
    L = _lib or lib()
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            st = getattr(L, name)(*args, _raw_stream(device))
    else:
        st = getattr(L, name)(*args, _raw_stream(device))
    if st:
        _check(st, name)


class KvCache:
    """A paged cache over the caller's tensors: k, v [num_pages, heads, page, dim], bfloat16 or
    float8_e4m3fn; with the latter k_scale, v_scale fp32 [num_pages, heads]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        shape, dtype = k.shape, k.dtype
        if len(shape) != 4 or v.shape != shape or v.dtype is not dtype:
            raise PaceError("k and v must be [num_pages, heads, page, dim] of one shape and type")
        if dtype is not _BF16 and dtype is not _E4M3:
            raise PaceError(f"cache type {dtype} is not bfloat16 or float8_e4m3fn")
        bits = 16 if dtype is _BF16 else 8
        n, heads, page, dim = shape
        if bits == 16:
            k_scale = v_scale = None
        elif k_scale is None or v_scale is None or k_scale.shape != (n, heads) or v_scale.shape != (n, heads):
            raise PaceError("8-bit pages need float32 scales [num_pages, heads]")
        self.device = _gpu_of(k)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.heads, self.page, self.dim, self.bits = heads, page, dim, bits
        self.struct = _KvCacheStruct(_arg(k, dtype, shape, self.device, "k"), _arg(v, dtype, shape, self.device, "v"),
                                     _arg(k_scale, _F32, (n, heads), self.device, "k_scale"),
                                     _arg(v_scale, _F32, (n, heads), self.device, "v_scale"), n, heads, page, dim, bits)
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, num_pages: int, heads: int, page: int, dim: int, dtype=torch.bfloat16, device="cuda"):
        """A cache over newly allocated, uninitialised pages."""
        k, v = (torch.empty((num_pages, heads, page, dim), dtype=dtype, device=device) for _ in range(2))
        if dtype is _BF16:
            return cls(k, v)
        return cls(k, v, *(torch.empty((num_pages, heads), dtype=_F32, device=device) for _ in range(2)))


def cache_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, cache: KvCache, cu_new: torch.Tensor,
                 ctx_len: torch.Tensor, block_table: torch.Tensor, max_new: int,
                 positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
                 sections: Optional[Sequence[int]] = None, rows: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Rotates q and k by positions (int32 [n_src] or [axes, n_src]; None: no rotation) and appends k and v to the
    cache.  q, k, v: bf16 [n_src, heads, dim], rows of any stride (slices of a fused projection); rows int32 [n_new]:
    the source rows to take (a selection's kept indices).  Returns the rotated queries [n_new, Hq, dim], or None
    without q."""
    gpu, dim, n_src = cache.device, cache.dim, k.shape[0]
    if block_table.dim() != 2:
        raise PaceError("block_table must be [B, max_pages]")
    B, max_pages = block_table.shape
    n_new = n_src if rows is None else rows.numel()
    kp, ks = _rows_arg(k, cache.heads, dim, n_src, gpu, "k")
    vp, vs = _rows_arg(v, cache.heads, dim, n_src, gpu, "v")
    qp, qs, hq = None, 0, 0
    if q is None:
        q_out = None
    else:
        hq = q.shape[1] if q.dim() == 3 else 0
        qp, qs = _rows_arg(q, hq, dim, n_src, gpu, "q")
        if q_out is None:
            q_out = torch.empty((n_new, hq, dim), dtype=_BF16, device=q.device)
    if n_new == 0:
        return q_out
    axes, sec = 1, None
    if positions is not None:
        axes = 1 if positions.dim() == 1 else positions.shape[0]
        if axes == 3:
            if sections is None or len(sections) != 3:
                raise PaceError("three position axes need three sections")
            sec = _INT3(*sections)
    _call("pace_cache_append", gpu, qp, qs, kp, ks, vp, vs, n_src, hq, _arg(rows, _I32, (n_new,), gpu, "rows"),
          _arg(cu_new, _I32, (B + 1,), gpu, "cu_new"), B, n_new, max_new, _arg(ctx_len, _I32, (B,), gpu, "ctx_len"),
          _arg(block_table, _I32, (B, max_pages), gpu, "block_table"), max_pages,
          _arg(positions, _I32, (n_src,) if positions is not None and positions.dim() == 1 else (axes, n_src), gpu,
               "positions"), axes, sec, _arg(inv_freq, _F32, (dim // 2,), gpu, "inv_freq"), cache.ref,
          _arg(q_out, _BF16, (n_new, hq, dim), gpu, "q_out"))
    return q_out


def cache_attention(q: torch.Tensor, cache: KvCache, cu_q: torch.Tensor, seq_len: torch.Tensor,
                    block_table: torch.Tensor, max_q: int, max_len: int, scale: Optional[float] = None,
                    window: int = 0, sinks: int = 0, want_lse: bool = True, o: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Attention of q bf16 [n_q, Hq, dim] over a paged cache that holds its tokens already.  cu_q int32 [B + 1],
    seq_len int32 [B], block_table int32 [B, max_pages] on the GPU.  Returns (o, lse [Hq, n_q] or None)."""
    gpu, dim = cache.device, cache.dim
    if q.dim() != 3 or block_table.dim() != 2:
        raise PaceError("q must be [n_q, Hq, dim], block_table [B, max_pages]")
    n_q, hq, _ = q.shape
    B, max_pages = block_table.shape
    if o is None:
        o = torch.empty_like(q)
    if not want_lse:
        lse = None
    elif lse is None:
        lse = torch.empty((hq, n_q), dtype=_F32, device=q.device)
    if n_q == 0:
        return o, lse
    if workspace is None:
        need = (_lib or lib()).pace_cache_attention_workspace_size(n_q, hq, cache.heads, dim, cache.bits, B, max_q, max_len,
                                                                   window, sinks)
        if need:
            workspace = torch.empty(need, dtype=_U8, device=q.device)
    _call("pace_cache_attention", gpu, _arg(q, _BF16, (n_q, hq, dim), gpu, "q"), n_q, hq, cache.ref,
          _arg(cu_q, _I32, (B + 1,), gpu, "cu_q"), B, max_q, _arg(seq_len, _I32, (B,), gpu, "seq_len"), max_len,
          _arg(block_table, _I32, (B, max_pages), gpu, "block_table"), max_pages, window, sinks,
          dim ** -0.5 if scale is None else scale, _arg(o, _BF16, (n_q, hq, dim), gpu, "o"),
          _arg(lse, _F32, (hq, n_q), gpu, "lse"),
          *_scratch(workspace, gpu))
    return o, lse


def gemm_w4(x: torch.Tensor, w: torch.Tensor, scale: torch.Tensor, zero: Optional[torch.Tensor] = None,
            bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, epilogue: int = 0,
            out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """C = x W^T with 4-bit weights: x bf16 [M, K]; w uint8 [N, K / 2] (low half first); scale bf16 [N, K / group];
    zero uint8 like scale, or None (8); bias, residual and epilogue as in gemm_bf16."""
    gpu = _gpu_of(x)
    if x.dim() != 2 or scale.dim() != 2:
        raise PaceError("x and scale must be 2-D")
    M, K = x.shape
    N, groups = scale.shape
    if groups < 1 or K % groups:
        raise PaceError(f"K={K} is not a multiple of the {groups} groups")
    cols = N // 2 if epilogue == 2 else N
    if out is None:
        out = torch.empty((M, cols), dtype=_BF16, device=x.device)
    if workspace is None:
        need = (_lib or lib()).pace_gemm_w4_workspace_size(M, N, K)
        if need:
            workspace = torch.empty(need, dtype=_U8, device=x.device)
    _call("pace_gemm_w4", gpu, _arg(x, _BF16, (M, K), gpu, "x"), _arg(w, _U8, (N, K // 2), gpu, "w"),
          _arg(scale, _BF16, (N, groups), gpu, "scale"), _arg(zero, _U8, (N, groups), gpu, "zero"),
          _arg(bias, _F32, (N,), gpu, "bias"), _arg(residual, _BF16, (M, cols), gpu, "residual"),
          _arg(out, _BF16, (M, cols), gpu, "out"), M, N, K, K // groups, epilogue,
          *_scratch(workspace, gpu))
    return out


# ---------------------------------------------------------------- a layer in 8 bits
SUMS_AUTO, SUMS_FAST, SUMS_WIDE = 0, 1, 2            # PACE_SUMS_* of include/pace.h


def _matrix_arg(t: torch.Tensor, dtype, shape: tuple, device: int, name: str):
    """Address and row stride of a matrix whose rows are contiguous and may lie further apart."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or (shape[1] > 1 and t.stride(1) != 1):
        raise PaceError(f"{name} must be a {dtype} matrix {list(shape)} of contiguous rows on GPU {device}, not {t.dtype} "
                        f"{list(t.shape)} (strides {t.stride()}) on {t.device}")
    return t.data_ptr(), (t.stride(0) if shape[0] > 1 else shape[1])


def _output(t: Optional[torch.Tensor], like: torch.Tensor, dtype, shape: tuple, device: int, name: str):
    """The caller's output tensor, or a new one beside `like`, and its address."""
    if t is None:
        t = like.new_empty(shape, dtype=dtype)
        return t, t.data_ptr()
    return t, _arg(t, dtype, shape, device, name)


def quantize_fp8(x: torch.Tensor, rows: int = 1, out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
    """x bf16 [M, K] (rows of any stride) to e4m3 codes [M, K] with a scale for each 128 neighbouring values of a row (rows=1:
    scale fp32 [ceil(K / 128), M], what gemm_fp8 takes for x) or for each 128 x 128 (rows=128: [ceil(M / 128), ceil(K / 128)],
    what it takes for w).  Returns (codes, scale)."""
    gpu = _gpu_of(x)
    if x.dim() != 2:
        raise PaceError("x must be 2-D")
    M, K = x.shape
    kb = (K + 127) // 128
    shape = (kb, M) if rows == 1 else ((M + 127) // 128, kb)
    xp, xs = _matrix_arg(x, _BF16, (M, K), gpu, "x")
    out, op = _output(out, x, _E4M3, (M, K), gpu, "out")
    scale, sp = _output(scale, x, _F32, shape, gpu, "scale")
    _call("pace_quantize_fp8", gpu, xp, xs, M, K, rows, op, sp)
    return out, scale


def rmsnorm(x: torch.Tensor, gamma: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, bits: int = 16,
            out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None):
    """RMS norm of x bf16 [M, K], or of x + residual, times gamma fp32 [K]; x and residual may have rows of any stride.
    Returns (y, scale, sum): y bf16 and scale None (bits=16), or e4m3 codes and their scales fp32 [ceil(K / 128), M]
    (bits=8); sum bf16 = x + residual, None without a residual.  sum_out may be the residual itself."""
    gpu = _gpu_of(x)
    if x.dim() != 2:
        raise PaceError("x must be 2-D")
    if bits != 8 and bits != 16:
        raise PaceError(f"bits={bits} is not 8 or 16")
    M, K = x.shape
    kb = (K + 127) // 128
    xp, xs = _matrix_arg(x, _BF16, (M, K), gpu, "x")
    rp, rs, hp = None, 0, None
    if residual is None:
        if sum_out is not None:
            raise PaceError("sum_out is x + residual: it needs a residual")
    else:
        rp, rs = _matrix_arg(residual, _BF16, (M, K), gpu, "residual")
        sum_out, hp = _output(sum_out, x, _BF16, (M, K), gpu, "sum_out")
    if bits == 16:
        if scale is not None:
            raise PaceError("a 16-bit output has no scale")
        qp = sp = None
        out, yp = _output(out, x, _BF16, (M, K), gpu, "out")
    else:
        yp = None
        out, qp = _output(out, x, _E4M3, (M, K), gpu, "out")
        scale, sp = _output(scale, x, _F32, (kb, M), gpu, "scale")
    _call("pace_rmsnorm", gpu, xp, xs, rp, rs, _arg(gamma, _F32, (K,), gpu, "gamma"), eps, M, K, hp, yp, qp, sp)
    return out, scale, sum_out


def gemm_fp8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
             residual: Optional[torch.Tensor] = None, epilogue: int = 0, bits: int = 16, sums: int = SUMS_AUTO,
             out: Optional[torch.Tensor] = None, out_scale: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None):
    """C = x W^T of e4m3 codes x [M, K] with x_scale fp32 [ceil(K / 128), M] (rows of any stride: a slice of rows is x[a:b],
    x_scale[:, a:b]) and w [N, K] with w_scale fp32 [ceil(N / 128), ceil(K / 128)]; bias, residual and epilogue as in
    gemm_bf16.  Returns (C, None), or with bits=8 and SwiGLU (codes [M, N / 2], their scales [ceil(N / 256), M]), ready for
    the next product.  sums: SUMS_FAST adds the products of a block as the matrix cores do (8 at a time on a grid of 2^-13 of
    the largest), SUMS_WIDE in 32 bits at half the matrix rate; SUMS_AUTO is wide for bits=8 alone."""
    gpu = _gpu_of(x)
    if x.dim() != 2 or w.dim() != 2:
        raise PaceError("x and w must be 2-D")
    if bits != 8 and bits != 16:
        raise PaceError(f"bits={bits} is not 8 or 16")
    M, K = x.shape
    N = w.shape[0]
    kb = (K + 127) // 128
    cols = N // 2 if epilogue == 2 else N
    xsp, xss = _matrix_arg(x_scale, _F32, (kb, M), gpu, "x_scale")
    out, op = _output(out, x, _E4M3 if bits == 8 else _BF16, (M, cols), gpu, "out")
    if bits == 16:
        if out_scale is not None:
            raise PaceError("a 16-bit output has no out_scale")
        sp = None
    else:
        out_scale, sp = _output(out_scale, x, _F32, ((cols + 127) // 128, M), gpu, "out_scale")
    if workspace is None:
        need = (_lib or lib()).pace_gemm_fp8_workspace_size(M, N, K, bits, sums)
        if need:
            workspace = x.new_empty((need,), dtype=_U8)
    _call("pace_gemm_fp8", gpu, _arg(x, _E4M3, (M, K), gpu, "x"), xsp, xss, _arg(w, _E4M3, (N, K), gpu, "w"),
          _arg(w_scale, _F32, ((N + 127) // 128, kb), gpu, "w_scale"), _arg(bias, _F32, (N,), gpu, "bias"),
          _arg(residual, _BF16, (M, cols), gpu, "residual"), op, sp, M, N, K, epilogue, sums, *_scratch(workspace, gpu))
    return out, out_scale
