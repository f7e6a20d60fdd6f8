"""ctypes binding of libvvs.so: the same entry points as include/vvs.h, taking torch CUDA tensors.

Argument marshalling only - every step of the verify pass runs inside the HIP library.  PyTorch is
used for device memory and the current stream.  There is no fallback: importing this module on a
machine where the library has not been built raises."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# VVS_LIBRARY: another build of the same library (for comparing builds); default: the in-tree one
LIB_PATH = os.environ.get("VVS_LIBRARY") or os.path.join(_HERE, "libvvs.so")

VVS_OK, VVS_EINVAL, VVS_ESTATE, VVS_ESIZE, VVS_EHIP = 0, -1, -2, -3, -4
VVS_FP32, VVS_BF16 = 0, 1
VVS_STRICT, VVS_RELAXED = 0, 1
VVS_NORM_AUTO, VVS_NORM_SEPARATE = 0, 1
VVS_CACHE_SAME, VVS_CACHE_E4M3 = 0, 1
VVS_MAX_T = 64
VVS_QCACHE_BLOCK = 32
VVS_ROPE_MAX_AXES = 4
VVS_ROPE_OWN, VVS_ROPE_SHARED = 0, 1
VVS_ROPE_ADJACENT, VVS_ROPE_HALVES = 0, 1
VVS_K_GEMM, VVS_K_ATTENTION, VVS_K_ACCEPT, VVS_K_ELEMENTWISE, VVS_K_COMMIT = range(5)


class VvsConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "d_ff", "vocab", "logit_lo", "logit_hi",
                                         "grid_h", "grid_w", "prefix_len", "prefix_kind", "n_classes", "n_prompts",
                                         "max_nodes", "dtype")] + \
               [("cfg_scale", C.c_float), ("rms_eps", C.c_float), ("rope_base", C.c_float),
                ("relax_k", C.c_int32), ("relax_delta", C.c_float),
                ("feature_slots", C.c_int32), ("feature_pre_norm", C.c_int32), ("draft_input", C.c_int32),
                ("norm_mode", C.c_int32), ("cache_kind", C.c_int32)]


class VvsQCacheConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_rows", "n_heads", "n_kv_heads", "head_size", "capacity", "max_tokens", "dtype")]


class VvsRopeConfig(C.Structure):
    _fields_ = [("head_size", C.c_int32), ("n_axes", C.c_int32), ("pairs", C.c_int32 * VVS_ROPE_MAX_AXES), ("series", C.c_int32),
                ("pairing", C.c_int32), ("dtype", C.c_int32), ("base", C.c_float)]


class VvsError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"vvs status {status}: {msg}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2511_13587_amd.build); "
                          "there is no CPU or PyTorch fallback for the verify pass")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    sigs = {
        "vvs_query_sizes": (i32, [C.POINTER(VvsConfig), C.POINTER(sz), C.POINTER(sz), C.POINTER(sz)]),
        "vvs_create": (i32, [C.POINTER(VvsConfig), vp, vp, vp, C.POINTER(vp)]),
        "vvs_destroy": (None, [vp]),
        "vvs_last_error": (C.c_char_p, [vp]),
        "vvs_num_weight_tensors": (i32, [C.POINTER(VvsConfig)]),
        "vvs_load_weights": (i32, [vp, C.POINTER(vp), i32, vp]),
        "vvs_set_neighbors": (i32, [vp, vp]),
        "vvs_check_tree": (i32, [i32, vp, vp, vp, vp]),
        "vvs_plan_is_fused": (i32, [vp, i32]),
        "vvs_prefill": (i32, [vp, vp, vp, i32, vp, vp, vp, vp]),
        "vvs_verify": (i32, [vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]),
        "vvs_verify_post": (i32, [vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]),
        "vvs_read_features": (i32, [vp, vp, vp, vp]),
        "vvs_select_unverified": (i32, [i32, vp, vp, C.c_float, vp, C.POINTER(i32)]),
        "vvs_skip_uniform": (i32, [i32, i32]),
        "vvs_skip_dynamic": (i32, [C.c_float, C.c_float, i32]),
        "vvs_set_codebook": (i32, [vp, vp, i32]),
        "vvs_path_similarity": (i32, [vp, i32, vp, vp, vp, C.c_float, i32, vp, vp]),
        "vvs_draft": (i32, [vp, vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp]),
        "vvs_accept_from_logits": (i32, [vp, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]),
        "vvs_accept_from_logits_noalloc": (i32, [vp, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]),
        "vvs_kv_commit": (i32, [vp, vp]),
        "vvs_kv_evict": (i32, [vp, i32, i32, vp]),
        "vvs_read_state": (i32, [vp, vp, vp]),
        "vvs_set_state": (i32, [vp, vp, vp]),
        "vvs_timing_enable": (i32, [vp, i32]),
        "vvs_timing_read": (i32, [vp, i32, C.POINTER(i32), C.POINTER(C.c_float)]),
        "vvs_debug_logits": (i32, [vp, vp, vp, vp, vp]),
        "vvs_debug_kv": (i32, [vp, i32, i32, i32, vp, vp, vp]),
        "vvs_debug_gemm_scratch_bytes": (sz, [vp, i32, i32, i32]),
        "vvs_debug_gemm": (i32, [vp, i32, i32, i32, vp, vp, vp, vp, vp]),
        "vvs_debug_copy": (i32, [vp, vp, vp, sz, vp]),
        "vvs_qcache_query_sizes": (i32, [C.POINTER(VvsQCacheConfig), C.POINTER(sz), C.POINTER(sz)]),
        "vvs_qcache_create": (i32, [C.POINTER(VvsQCacheConfig), vp, vp, C.POINTER(vp)]),
        "vvs_qcache_destroy": (None, [vp]),
        "vvs_qcache_last_error": (C.c_char_p, [vp]),
        "vvs_qcache_append": (i32, [vp, i32, i32, vp, i32, vp, i32, vp, vp, i64, vp, i64, vp]),
        "vvs_qcache_attention": (i32, [vp, i32, vp, i32, vp, vp, vp, vp, i64, vp, i64, vp, i64, C.c_float, vp, vp, i32, vp, vp, vp]),
        "vvs_qcache_evict": (i32, [vp, i32, i32, vp, i32, i32, vp, vp, vp, vp, vp]),
        "vvs_qcache_read": (i32, [vp, i32, i32, vp, vp, i32, vp, vp, vp]),
        "vvs_rope_create": (i32, [C.POINTER(VvsRopeConfig), C.POINTER(vp)]),
        "vvs_rope_destroy": (None, [vp]),
        "vvs_rope_last_error": (C.c_char_p, [vp]),
        "vvs_rope_apply": (i32, [vp, i32, vp, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, i32, vp]),
        "vvs_debug_wait_limit": (i32, [vp, i32]),
        "vvs_debug_fill_probe": (i32, [vp, vp, sz, sz, i32, i32, i32, i32, vp, vp]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib, list(sigs)


lib, EXPORTS = _load()


def make_config(shape, max_nodes: Optional[int] = None, feature_slots: int = 5, feature_pre_norm: int = 0,
                draft_input: int = 0, norm_mode: int = 0, cache_kind: int = 0) -> VvsConfig:
    """vvs_config from a synth.Shape-like object."""
    return VvsConfig(shape.n_layers, shape.d_model, shape.n_heads, shape.d_ff, shape.vocab, shape.logit_lo,
                     shape.logit_hi, shape.grid_h, shape.grid_w, shape.prefix_len, shape.prefix_kind,
                     shape.n_classes, shape.n_prompts, shape.n_nodes if max_nodes is None else max_nodes,
                     shape.dtype, shape.cfg_scale, shape.rms_eps, shape.rope_base, shape.relax_k, shape.relax_delta,
                     feature_slots, feature_pre_norm, draft_input, norm_mode, cache_kind)


def vvs_query_sizes(cfg: VvsConfig):
    kv, ws, pw = C.c_size_t(), C.c_size_t(), C.c_size_t()
    st = lib.vvs_query_sizes(C.byref(cfg), C.byref(kv), C.byref(ws), C.byref(pw))
    if st != VVS_OK:
        raise VvsError(st, (lib.vvs_last_error(None) or b"").decode())
    return kv.value, ws.value, pw.value


def vvs_check_tree(n_nodes: int, parent: Optional[np.ndarray], mask: Optional[np.ndarray]):
    """Host-only topology check; returns (status, depth[T], parent[N])."""
    depth = np.zeros(max(n_nodes, 0) + 1, dtype=np.int32)
    pout = np.zeros(max(n_nodes, 1), dtype=np.int32)
    p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
    m = None if mask is None else np.ascontiguousarray(mask, dtype=np.uint8)
    st = lib.vvs_check_tree(n_nodes, None if p is None else p.ctypes.data, None if m is None else m.ctypes.data,
                            depth.ctypes.data, pout.ctypes.data)
    return st, depth, pout[:max(n_nodes, 0)]


def vvs_select_unverified(n_nodes: int, parent: Optional[np.ndarray], mask: Optional[np.ndarray], u: float):
    """Host-only: (status, kept node ids) of the uniformly drawn, truncated candidate path."""
    nodes = np.zeros(VVS_MAX_T, dtype=np.int32)
    kept = C.c_int32()
    p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
    m = None if mask is None else np.ascontiguousarray(mask, dtype=np.uint8)
    st = lib.vvs_select_unverified(n_nodes, None if p is None else p.ctypes.data, None if m is None else m.ctypes.data,
                                   float(u), nodes.ctypes.data, C.byref(kept))
    return st, nodes[:max(kept.value, 0)].copy()


def vvs_skip_uniform(step_index: int, interval: int) -> bool:
    return bool(lib.vvs_skip_uniform(step_index, interval))


def vvs_skip_dynamic(similarity: float, threshold: float, last_step_verified: bool) -> bool:
    return bool(lib.vvs_skip_dynamic(float(similarity), float(threshold), 1 if last_step_verified else 0))


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def to_device(a: np.ndarray, dtype: int) -> torch.Tensor:
    """Model-dtype host array (float32 values) -> device tensor (bf16 bits as int16, or float32)."""
    a = np.ascontiguousarray(a, dtype=np.float32)
    if dtype == VVS_BF16:
        u = a.view(np.uint32)
        bits = ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) >> np.uint32(16)).astype(np.uint16)
        return torch.from_numpy(bits.view(np.int16)).cuda()
    return torch.from_numpy(a).cuda()


class Context:
    """Owns the three device buffers and the vvs_ctx; methods mirror the C entry points."""

    def __init__(self, cfg: VvsConfig, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("libvvs needs a HIP device; there is no CPU path")
        self.cfg = cfg
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.kv_bytes, self.ws_bytes, self.pw_bytes = vvs_query_sizes(cfg)
        self.kv = torch.empty(self.kv_bytes, dtype=torch.uint8, device=self.device)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.pw = torch.empty(self.pw_bytes, dtype=torch.uint8, device=self.device)
        torch.cuda.synchronize()
        h = C.c_void_p()
        st = lib.vvs_create(C.byref(cfg), self.kv.data_ptr(), self.ws.data_ptr(), self.pw.data_ptr(), C.byref(h))
        if st != VVS_OK:
            raise VvsError(st, (lib.vvs_last_error(None) or b"").decode())
        self.h = h
        self.B = cfg.n_prompts
        self.R = 2 * cfg.n_prompts
        self.veff = cfg.logit_hi - cfg.logit_lo
        self._nbr = None
        self.last_T = 0

    def close(self):
        if getattr(self, "h", None):
            torch.cuda.synchronize()
            lib.vvs_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != VVS_OK:
            raise VvsError(st, (lib.vvs_last_error(self.h) or b"").decode())

    # -- weights -------------------------------------------------------------------------------
    def vvs_load_weights(self, tensors: Sequence[Optional[torch.Tensor]]):
        arr = (C.c_void_p * len(tensors))(*[_ptr(t) for t in tensors])
        self._check(lib.vvs_load_weights(self.h, arr, len(tensors), _stream()))

    def load_weights_from_host(self, weights: Dict[str, np.ndarray], names: Sequence[str]):
        """Uploads float32 host arrays in canonical order (converted to the model dtype) and packs."""
        dev = [to_device(weights[n], self.cfg.dtype) for n in names]
        self.vvs_load_weights(dev)
        torch.cuda.synchronize()
        del dev

    def vvs_set_neighbors(self, nbr: torch.Tensor):
        assert nbr.dtype == torch.int32
        self._nbr = nbr
        self._check(lib.vvs_set_neighbors(self.h, _ptr(nbr)))

    # -- the three calls of the hot path ---------------------------------------------------------
    def vvs_prefill(self, prefix_cond: torch.Tensor, prefix_uncond: Optional[torch.Tensor], forced: Optional[torch.Tensor],
                    uniform: torch.Tensor, first_token: torch.Tensor):
        n_forced = 0 if forced is None else int(forced.shape[1])
        self._check(lib.vvs_prefill(self.h, _ptr(prefix_cond), _ptr(prefix_uncond), n_forced, _ptr(forced),
                                    _ptr(uniform), _ptr(first_token), _stream()))
        self.last_T = 1

    def vvs_verify(self, n_nodes: int, parent: Optional[np.ndarray], tree_mask: Optional[np.ndarray],
                   draft_tokens: Optional[torch.Tensor], draft_probs: Optional[torch.Tensor], uniforms: torch.Tensor,
                   mode: int, accept_len: torch.Tensor, path: torch.Tensor, next_token: torch.Tensor):
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        self._check(lib.vvs_verify(self.h, n_nodes, None if p is None else p.ctypes.data,
                                   None if m is None else m.ctypes.data, _ptr(draft_tokens), _ptr(draft_probs),
                                   _ptr(uniforms), mode, _ptr(accept_len), _ptr(path), _ptr(next_token), _stream()))
        self.last_T = n_nodes + 1

    def vvs_verify_post(self, n_nodes: int, n_post: int, parent: Optional[np.ndarray], tree_mask: Optional[np.ndarray],
                        draft_tokens: Optional[torch.Tensor], draft_probs: Optional[torch.Tensor], uniforms: torch.Tensor,
                        mode: int, accept_len: torch.Tensor, path: torch.Tensor, next_token: torch.Tensor):
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        self._check(lib.vvs_verify_post(self.h, n_nodes, n_post, None if p is None else p.ctypes.data,
                                        None if m is None else m.ctypes.data, _ptr(draft_tokens), _ptr(draft_probs),
                                        _ptr(uniforms), mode, _ptr(accept_len), _ptr(path), _ptr(next_token), _stream()))
        self.last_T = n_nodes + 1

    def vvs_set_codebook(self, embed: torch.Tensor):
        assert embed.dtype == torch.float32 and embed.dim() == 2
        self._codebook = embed                      # kept by reference in the library
        self._check(lib.vvs_set_codebook(self.h, _ptr(embed), int(embed.shape[1])))

    def vvs_path_similarity(self, n_nodes: int, parent, tree_mask, draft_tokens: Optional[torch.Tensor], alpha: float, stride: int = 2):
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        out = torch.empty((self.B,), dtype=torch.float32, device=self.device)
        self._check(lib.vvs_path_similarity(self.h, n_nodes, None if p is None else p.ctypes.data,
                                            None if m is None else m.ctypes.data, _ptr(draft_tokens), float(alpha), int(stride),
                                            _ptr(out), _stream()))
        return out

    def vvs_read_features(self):
        """(features float32 [R, feature_slots, d] oldest first, count int32 [B])."""
        feats = torch.empty((self.R, self.cfg.feature_slots, self.cfg.d_model), dtype=torch.float32, device=self.device)
        count = torch.empty((self.B,), dtype=torch.int32, device=self.device)
        self._check(lib.vvs_read_features(self.h, _ptr(feats), _ptr(count), _stream()))
        return feats.cpu().numpy(), count.cpu().numpy()

    def vvs_draft(self, target: "Context", n_nodes: int, parent, tree_mask, n_ctx: int, recent_tokens: torch.Tensor,
                  n_unverified: int, given_tokens: Optional[torch.Tensor], draft_tokens: torch.Tensor, draft_probs: torch.Tensor):
        """self is the drafter context (draft_input = 1)."""
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        assert recent_tokens.dtype == torch.int32 and draft_tokens.dtype == torch.int32 and draft_probs.dtype == torch.float32
        self._check(lib.vvs_draft(self.h, target.h, n_nodes, None if p is None else p.ctypes.data,
                                  None if m is None else m.ctypes.data, n_ctx, _ptr(recent_tokens), n_unverified,
                                  _ptr(given_tokens), _ptr(draft_tokens), _ptr(draft_probs), _stream()))
        internal = 0 if p is None else len(set(int(v) for v in p if v > 0))
        self.last_T = n_ctx + (n_nodes - 1 if p is None else internal)

    def vvs_accept_from_logits(self, n_nodes: int, parent, tree_mask, raw_logits: torch.Tensor, draft_tokens, draft_probs,
                               uniforms, mode, accept_len, path, next_token):
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        self._check(lib.vvs_accept_from_logits(self.h, n_nodes, None if p is None else p.ctypes.data,
                                               None if m is None else m.ctypes.data, _ptr(raw_logits), _ptr(draft_tokens),
                                               _ptr(draft_probs), _ptr(uniforms), mode, _ptr(accept_len), _ptr(path),
                                               _ptr(next_token), _stream()))

    def vvs_accept_from_logits_noalloc(self, n_nodes: int, parent, tree_mask, raw_logits: torch.Tensor, draft_tokens, draft_probs,
                                       uniforms, mode, accept_len, path, next_token):
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        self._check(lib.vvs_accept_from_logits_noalloc(self.h, n_nodes, None if p is None else p.ctypes.data,
                                                       None if m is None else m.ctypes.data, _ptr(raw_logits), _ptr(draft_tokens),
                                                       _ptr(draft_probs), _ptr(uniforms), mode, _ptr(accept_len), _ptr(path),
                                                       _ptr(next_token), _stream()))

    def vvs_kv_commit(self):
        self._check(lib.vvs_kv_commit(self.h, _stream()))

    def vvs_kv_evict(self, keep: int, recent: int):
        self._check(lib.vvs_kv_evict(self.h, keep, recent, _stream()))

    # -- inspection ----------------------------------------------------------------------------
    def vvs_plan_is_fused(self, n_tokens: int) -> bool:
        return bool(lib.vvs_plan_is_fused(self.h, n_tokens))

    def vvs_read_state(self) -> np.ndarray:
        out = torch.empty((3, self.B), dtype=torch.int32, device=self.device)
        self._check(lib.vvs_read_state(self.h, _ptr(out), _stream()))
        return out.cpu().numpy()

    def vvs_set_state(self, state: torch.Tensor):
        assert state.dtype == torch.int32 and state.numel() == 3 * self.B
        self._check(lib.vvs_set_state(self.h, _ptr(state), _stream()))

    def vvs_timing_enable(self, on: bool):
        self._check(lib.vvs_timing_enable(self.h, 1 if on else 0))

    def vvs_timing_read(self, kernel_class: int):
        n, ms = C.c_int32(), C.c_float()
        self._check(lib.vvs_timing_read(self.h, kernel_class, C.byref(n), C.byref(ms)))
        return n.value, ms.value

    def vvs_debug_logits(self):
        T = self.last_T
        raw = torch.empty((self.R, T, self.veff), dtype=torch.float32, device=self.device)
        mixed = torch.empty((self.B, T, self.veff), dtype=torch.float32, device=self.device)
        probs = torch.empty((self.B, T, self.veff), dtype=torch.float32, device=self.device)
        self._check(lib.vvs_debug_logits(self.h, _ptr(raw), _ptr(mixed), _ptr(probs), _stream()))
        return raw, mixed, probs

    def vvs_debug_kv(self, layer: int, row: int, n_slots: int):
        d = self.cfg.d_model
        k = torch.empty((n_slots, d), dtype=torch.float32, device=self.device)
        v = torch.empty((n_slots, d), dtype=torch.float32, device=self.device)
        self._check(lib.vvs_debug_kv(self.h, layer, row, n_slots, _ptr(k), _ptr(v), _stream()))
        return k, v

    def vvs_debug_copy(self, dst: torch.Tensor, src: torch.Tensor):
        nbytes = src.numel() * src.element_size()
        assert dst.numel() * dst.element_size() == nbytes
        self._check(lib.vvs_debug_copy(self.h, _ptr(dst), _ptr(src), nbytes, _stream()))

    def vvs_debug_wait_limit(self, polls: int):
        self._check(lib.vvs_debug_wait_limit(self.h, int(polls)))

    def vvs_debug_fill_probe(self, src: torch.Tensor, reps: int, mode: int, n_workgroups: int, waves: int,
                             region_bytes: int = 0, wg_stride_bytes: int = 0) -> torch.Tensor:
        """region_bytes 0: the whole of src, read by every workgroup; else workgroup w reads region_bytes at w * wg_stride_bytes"""
        total = src.numel() * src.element_size()
        region = region_bytes or total
        assert (n_workgroups - 1) * wg_stride_bytes + region <= total
        sink = torch.zeros(n_workgroups, dtype=torch.int32, device=self.device)
        self._check(lib.vvs_debug_fill_probe(self.h, _ptr(src), region, wg_stride_bytes, reps, mode, n_workgroups, waves,
                                             _ptr(sink), _stream()))
        return sink

    def vvs_debug_gemm(self, a: torch.Tensor, w: torch.Tensor, m: int, n: int, k: int) -> torch.Tensor:
        nbytes = lib.vvs_debug_gemm_scratch_bytes(self.h, m, n, k)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        out = torch.empty((m, n), dtype=torch.float32, device=self.device)
        self._check(lib.vvs_debug_gemm(self.h, m, n, k, _ptr(a), _ptr(w), _ptr(scratch), _ptr(out), _stream()))
        torch.cuda.synchronize()
        return out


# ---------------------------------------------------------------------------------------------- operators beside a context
def _wrong(what: str, t: torch.Tensor, device: int, dtype: torch.dtype, shape):
    raise ValueError(f"{what}: wants a {dtype} tensor {list(shape)} on device {device}, got {t.dtype} {list(t.shape)} on {t.device}")


def _on(t: Optional[torch.Tensor], device: int, dtype: torch.dtype, shape, what: str):
    """Pointer of a contiguous tensor of the library's arguments (None stays None); device: its index, -1 for the host."""
    if t is None:
        return None
    if t.get_device() != device or t.dtype != dtype or t.shape != shape:
        _wrong(what, t, device, dtype, shape)
    if not t.is_contiguous():
        raise ValueError(f"{what}: wants a contiguous tensor, got strides {t.stride()}")
    return t.data_ptr()


def _per_token(t: Optional[torch.Tensor], device: int, dtype: torch.dtype, shape, what: str):
    """(pointer, elements from token to token) of a tensor [..., tokens, heads, size] that may be a part of a wider one: heads and dims contiguous, every
    dimension in front of them in steps of whole tokens."""
    if t is None:
        return None, 0
    if t.get_device() != device or t.dtype != dtype or t.shape != shape:
        _wrong(what, t, device, dtype, shape)
    heads, size = shape[-2], shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), heads * size
    strides = t.stride()
    token, n = None, 1                   # n: tokens below each dimension
    ok = (strides[-1] == 1 or size == 1) and (strides[-2] == size or heads == 1)
    for d in range(len(shape) - 3, -1, -1):
        if shape[d] > 1:
            if token is None:
                token = strides[d] // n
            ok = ok and strides[d] == token * n
        n *= shape[d]
    token = heads * size if token is None else token
    if not ok or token < heads * size:
        raise ValueError(f"{what}: strides {strides} of {list(shape)} are not those of tokens one after the other")
    return t.data_ptr(), token


def _apart(out: int, n_out: int, tensors, tokens: int, width: int):
    """Refuses an output at address `out`, of n_out elements of `width` bytes, that shares memory with one of tensors: (address or None, elements from token to token, elements of a token)."""
    for p, stride, per in tensors:
        if p is not None and p < out + n_out * width and out < p + ((tokens - 1) * stride + per) * width:
            raise ValueError("out: shares memory with q, k or v")


_raw_stream = torch._C._cuda_getCurrentRawStream     # (current_stream() makes a stream object each time: 1.5 us of a 5 us call)


class _Current:
    """Makes a device current for a call, where it is not already (torch.cuda.device does it always: 2 us)."""

    def __init__(self, index: int):
        self.index, self.was = index, []

    def __enter__(self):
        now = torch.cuda.current_device()
        self.was.append(now)
        if now != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        was = self.was.pop()
        if was != self.index:
            torch.cuda.set_device(was)


_TORCH_DTYPE = {VVS_FP32: torch.float32, VVS_BF16: torch.bfloat16}


class QCache:
    """A key/value cache in 8 bits: owns its two device buffers; methods mirror the C entry points (include/vvs.h).  Lengths, accumulated weights and positions
    are the caller's tensors; tensors may be bfloat16 or float32, as the cache's dtype says."""

    def __init__(self, n_layers: int, n_rows: int, n_heads: int, n_kv_heads: int, head_size: int, capacity: int, max_tokens: int, dtype: int,
                 device: str = "cuda:0"):
        self.cfg = VvsQCacheConfig(n_layers, n_rows, n_heads, n_kv_heads, head_size, capacity, max_tokens, dtype)
        self.cache_bytes, self.ws_bytes = vvs_qcache_query_sizes(self.cfg)
        if not torch.cuda.is_available():
            raise RuntimeError("libvvs needs a HIP device; there is no CPU path")
        self.device, self.dtype = torch.device(device), _TORCH_DTYPE[dtype]
        self.width = self.dtype.itemsize
        self.index = torch.cuda.current_device() if self.device.index is None else self.device.index
        with torch.cuda.device(self.index):
            self.cache = torch.empty(self.cache_bytes, dtype=torch.uint8, device=self.device)
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
            torch.cuda.synchronize()
            h = C.c_void_p()
            st = lib.vvs_qcache_create(C.byref(self.cfg), self.cache.data_ptr(), self.ws.data_ptr(), C.byref(h))
        if st != VVS_OK:
            raise VvsError(st, (lib.vvs_last_error(None) or b"").decode())
        self.h = h
        self.shape = (n_rows, n_heads, n_kv_heads, head_size, capacity)      # (a field of the ctypes structure is 0.1 us to read)

    def close(self):
        if getattr(self, "h", None):
            torch.cuda.synchronize(self.index)
            lib.vvs_qcache_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != VVS_OK:
            raise VvsError(st, (lib.vvs_qcache_last_error(self.h) or b"").decode())

    def _rows(self, t, what):
        return _on(t, self.index, torch.int32, self.shape[:1], what)

    def vvs_qcache_append(self, length: torch.Tensor, k: torch.Tensor, v: torch.Tensor, n_tokens: Optional[torch.Tensor] = None,
                          select: Optional[torch.Tensor] = None, layer: int = 0, n_layers: int = 1):
        """k, v [n_layers, rows, tokens, kv heads, size]; select int32 [rows, n]: the tokens taken; n_tokens int32 [rows]: how many of them."""
        rows, heads, kv, size, capacity = self.shape
        src = k.shape[2] if k.dim() == 5 else 0
        shape = (n_layers, rows, src, kv, size)
        kp, ks = _per_token(k, self.index, self.dtype, shape, "k")
        vp, vs = _per_token(v, self.index, self.dtype, shape, "v")
        n = src if select is None else int(select.shape[1])
        with _Current(self.index):
            self._check(lib.vvs_qcache_append(self.h, layer, n_layers, self._rows(length, "length"), n, self._rows(n_tokens, "n_tokens"), src,
                                              _on(select, self.index, torch.int32, (rows, n), "select"), kp, ks, vp, vs, _raw_stream(self.index)))

    def vvs_qcache_attention(self, length: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor], v: Optional[torch.Tensor], out: torch.Tensor,
                             n_tokens: Optional[torch.Tensor] = None, parent=None, tree_mask=None, scale: Optional[float] = None,
                             lse: Optional[torch.Tensor] = None, n_counted: int = 0, mass: Optional[torch.Tensor] = None,
                             block_mass: Optional[torch.Tensor] = None, layer: int = 0):
        """q [rows, tokens, heads, size]; k, v [rows, tokens, kv heads, size] or None; out like q, contiguous, in memory of its own (or q itself, contiguous,
        where no weights are counted).  scale: None = size ** -0.5."""
        rows, heads, kv, size, capacity = self.shape
        t = q.shape[1] if q.dim() == 4 else 0
        qp, qs = _per_token(q, self.index, self.dtype, (rows, t, heads, size), "q")
        kp, ks = _per_token(k, self.index, self.dtype, (rows, t, kv, size), "k")
        vp, vs = _per_token(v, self.index, self.dtype, (rows, t, kv, size), "v")
        p = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
        m = None if tree_mask is None else np.ascontiguousarray(tree_mask, dtype=np.uint8)
        op = _on(out, self.index, self.dtype, (rows, t, heads, size), "out")
        token = self.width * rows * t                        # bytes per element of a token
        end = op + token * heads * size
        if (qp < end and op < qp + token * qs) or (kp is not None and kp < end and op < kp + token * ks) or (vp is not None and vp < end and op < vp + token * vs):
            in_place = op == qp and qs == heads * size and n_counted == 0 and block_mass is None
            _apart(op, rows * t * heads * size, ((None if in_place else qp, qs, heads * size), (kp, ks, kv * size), (vp, vs, kv * size)), rows * t, self.width)
        if (p is not None and p.shape != (t - 1,)) or (m is not None and m.shape != (t, t)):
            raise ValueError("parent wants [tokens - 1] and tree_mask [tokens, tokens] entries")
        with _Current(self.index):
            self._check(lib.vvs_qcache_attention(
                self.h, layer, self._rows(length, "length"), t, self._rows(n_tokens, "n_tokens"), None if p is None else p.ctypes.data,
                None if m is None else m.ctypes.data, qp, qs, kp, ks, vp, vs, size ** -0.5 if scale is None else float(scale),
                op, _on(lse, self.index, torch.float32, (rows, t, heads), "lse"), n_counted,
                _on(mass, self.index, torch.float32, (rows, kv, capacity), "mass"),
                _on(block_mass, self.index, torch.float32, (rows, kv, t), "block_mass"), _raw_stream(self.index)))

    def vvs_qcache_evict(self, length: torch.Tensor, keep: int, recent: int, mass: torch.Tensor, mass_out: torch.Tensor,
                         pos: Optional[torch.Tensor] = None, pos_out: Optional[torch.Tensor] = None, layer: int = 0, n_layers: int = 1):
        """mass, mass_out float32, pos, pos_out int32 [n_layers, rows, kv heads, capacity]; an output may be its input."""
        rows, heads, kv, size, capacity = self.shape
        shape = (n_layers, rows, kv, capacity)
        with _Current(self.index):
            self._check(lib.vvs_qcache_evict(self.h, layer, n_layers, self._rows(length, "length"), keep, recent,
                                             _on(mass, self.index, torch.float32, shape, "mass"), _on(mass_out, self.index, torch.float32, shape, "mass_out"),
                                             _on(pos, self.index, torch.int32, shape, "pos"), _on(pos_out, self.index, torch.int32, shape, "pos_out"),
                                             _raw_stream(self.index)))

    def vvs_qcache_read(self, length: torch.Tensor, k: torch.Tensor, v: torch.Tensor, first: Optional[torch.Tensor] = None, layer: int = 0, n_layers: int = 1):
        """k, v [n_layers, rows, slots, kv heads, size] out."""
        rows, heads, kv, size, capacity = self.shape
        n = k.shape[2] if k.dim() == 5 else 0
        shape = (n_layers, rows, n, kv, size)
        with _Current(self.index):
            self._check(lib.vvs_qcache_read(self.h, layer, n_layers, self._rows(length, "length"), self._rows(first, "first"), n,
                                            _on(k, self.index, self.dtype, shape, "k"), _on(v, self.index, self.dtype, shape, "v"), _raw_stream(self.index)))


def vvs_qcache_query_sizes(cfg: VvsQCacheConfig):
    cache, ws = C.c_size_t(), C.c_size_t()
    st = lib.vvs_qcache_query_sizes(C.byref(cfg), C.byref(cache), C.byref(ws))
    if st != VVS_OK:
        raise VvsError(st, (lib.vvs_last_error(None) or b"").decode())
    return cache.value, ws.value


class Rope:
    """Rotary positions on several axes; pairs: rotated pairs of each axis.  Owns a host object only."""

    def __init__(self, head_size: int, pairs: Sequence[int], base: float, dtype: int, shared: bool = False, halves: bool = False):
        if not 1 <= len(pairs) <= VVS_ROPE_MAX_AXES:
            raise VvsError(VVS_ESIZE, "rope config: 1 to VVS_ROPE_MAX_AXES axes")
        self.cfg = VvsRopeConfig(head_size, len(pairs), (C.c_int32 * VVS_ROPE_MAX_AXES)(*pairs), VVS_ROPE_SHARED if shared else VVS_ROPE_OWN,
                                 VVS_ROPE_HALVES if halves else VVS_ROPE_ADJACENT, dtype, base)
        h = C.c_void_p()
        st = lib.vvs_rope_create(C.byref(self.cfg), C.byref(h))
        if st != VVS_OK:
            raise VvsError(st, (lib.vvs_last_error(None) or b"").decode())
        self.h, self.size, self.axes, self.dtype = h, head_size, len(pairs), _TORCH_DTYPE[dtype]

    def close(self):
        if getattr(self, "h", None):
            lib.vvs_rope_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def vvs_rope_apply(self, pos: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor, k_out: Optional[torch.Tensor],
                       inverse: bool = False):
        """pos int32 [..., axes]; q, k, q_out, k_out [..., heads, size] with the same leading dimensions; an output may be its input."""
        device, dtype, size = q.get_device(), self.dtype, self.size
        *lead, heads, _ = shape = tuple(q.shape)
        if device < 0 or not lead:
            raise ValueError("q: wants a tensor [..., heads, size] on a HIP device")
        n = 1
        for d in lead:
            n *= d
        qp, qs = _per_token(q, device, dtype, (*lead, heads, size), "q")
        op, os_ = _per_token(q_out, device, dtype, shape, "q_out")
        kv = 0 if k is None else k.shape[-2]
        kp, ks = _per_token(k, device, dtype, (*lead, kv, size), "k")
        kop, kos = _per_token(k_out, device, dtype, (*lead, kv, size), "k_out")
        with _Current(device):
            st = lib.vvs_rope_apply(self.h, n, _on(pos, device, torch.int32, (*lead, self.axes), "pos"), heads, qp, qs, op, os_, kv, kp, ks, kop, kos,
                                    1 if inverse else 0, _raw_stream(device))
        if st != VVS_OK:
            raise VvsError(st, (lib.vvs_rope_last_error(self.h) or b"").decode())
