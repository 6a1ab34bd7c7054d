"""Python binding of libautotensor (HIP, gfx950): argument marshalling only.

Every function has the name of the C entry point it calls (include/autotensor.h)
and does nothing but check argument types, pass raw device pointers and the
current HIP stream, and turn a non-OK status into an exception.  All of the
method's work runs in the library's HIP kernels.  PyTorch provides device
memory and streams.

The library must have been built (``python -m paper_1805_08166_amd.build`` or
``__graft_entry__.build()``); importing this package without it raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libautotensor.so")

AT_TMPL_GEMM = 0
AT_TMPL_CONV2D_NCHW = 1
AT_TMPL_GEMM_VT = 2
AT_TMPL_CONV2D_NCHW_VT = 3

STATUS = {0: "AT_OK", -1: "AT_E_INVALID", -2: "AT_E_UNSUPPORTED", -3: "AT_E_OOM", -4: "AT_E_HIP",
          -5: "AT_E_RANGE", -6: "AT_E_MISMATCH"}

# at_entry: {uint64 cfg; float score; uint32 flag}
ENTRY_DTYPE = np.dtype([("cfg", "<u8"), ("score", "<f4"), ("flag", "<u4")])

EXPORTED = [
    "at_space_create", "at_space_info", "at_spaceset_create", "at_space_destroy",
    "at_extract_features", "at_extract_features_full", "at_extract_features_onehot", "at_extract_relation_features", "at_space_errors", "at_ensemble_create", "at_ensemble_destroy",
    "at_trees_depth", "at_trees_pad", "at_ensemble_import",
    "at_gbt_predict", "at_gbt_predict_global_local", "at_chains_create", "at_chains_destroy", "at_chains_step",
    "at_sa_thresholds", "at_sa_run", "at_sa_run_traced", "at_sa_run_global_local", "at_chains_export", "at_sa_set_profiling",
    "at_sa_kernel_times", "at_chains_set_path", "at_chains_last_path", "at_chains_last_plan", "at_select_batch", "at_select_batch_noalloc", "at_last_error",
    "at_embed", "at_embed_grad_workspace", "at_embed_grad", "at_logprobs_workspace", "at_logprobs",
    "at_logprobs_grad", "at_orthogonalize_workspace", "at_orthogonalize",
]

# at_sa_path
AT_SA_PATH_AUTO = 0
AT_SA_PATH_TREES = 1
AT_SA_PATH_LOCAL = 2


class ATError(RuntimeError):
    def __init__(self, func: str, status: int, msg: str):
        super().__init__(f"{func} -> {STATUS.get(status, status)}: {msg}")
        self.status = status


def _load():
    from . import build as _build
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
    if _build.stale():
        raise ImportError(f"{LIB_PATH} was built from other sources than those under csrc/; "
                          "run __graft_entry__.build() again")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
    sig = {
        "at_space_create": [i32, vp, i32, vp],
        "at_space_info": [vp, vp, vp, vp, vp, vp],
        "at_spaceset_create": [vp, i32, vp, vp],
        "at_space_destroy": [vp],
        "at_extract_features": [vp, vp, i64, vp, vp],
        "at_extract_relation_features": [vp, vp, i64, vp, vp],
        "at_extract_features_full": [vp, vp, i64, vp, vp],
        "at_extract_features_onehot": [vp, vp, i64, vp, vp],
        "at_space_errors": [vp, vp],
        "at_ensemble_create": [i32, i32, i32, vp, vp, vp, vp],
        "at_ensemble_destroy": [vp],
        "at_trees_depth": [i32, vp, vp, vp, vp],
        "at_trees_pad": [i32, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp],
        "at_ensemble_import": [i32, vp, vp, vp, vp, vp, vp, i32, vp],
        "at_gbt_predict": [vp, vp, i64, vp, vp, vp],
        "at_gbt_predict_global_local": [vp, vp, vp, vp, i64, vp, vp],
        "at_chains_create": [vp, i64, i64, i32, u64, vp],
        "at_chains_destroy": [vp],
        "at_chains_step": [vp, vp],
        "at_sa_thresholds": [u64, i64, i64, u64, i32, vp],
        "at_sa_run": [vp, vp, vp, i32, vp, vp, vp],
        "at_sa_run_traced": [vp, vp, vp, i32, vp, vp, vp, vp],
        "at_sa_run_global_local": [vp, vp, vp, vp, i32, vp, vp, vp, vp],
        "at_chains_export": [vp, vp, vp, vp],
        "at_sa_set_profiling": [vp, i32],
        "at_sa_kernel_times": [vp, vp, vp, vp, vp],
        "at_chains_set_path": [vp, i32],
        "at_chains_last_path": [vp, vp],
        "at_chains_last_plan": [vp, vp],
        "at_select_batch": [vp, vp, i64, i32, i32, ctypes.c_float, i32, u64, vp, vp],
        "at_select_batch_noalloc": [vp, vp, i64, i32, i32, ctypes.c_float, i32, u64, vp, vp],
        "at_last_error": [],
        "at_embed": [vp, i32, i64, i64, i64, vp, i32, i64, f32, vp, i32, i64, vp],
        "at_embed_grad_workspace": [i64, i64, i64, vp],
        "at_embed_grad": [vp, i32, i64, vp, i32, i64, f32, i32, vp, i32, i64, i64, i64, vp, i64, vp],
        "at_logprobs_workspace": [i64, i64, i32, vp],
        "at_logprobs": [vp, i32, i64, i64, i64, vp, vp, i32, f32, i32, vp, vp, vp, vp, vp, vp, i64, vp],
        "at_logprobs_grad": [vp, i32, i64, i64, i64, vp, vp, i32, f32, vp, vp, vp, vp, vp, i64, vp],
        "at_orthogonalize_workspace": [i64, i64, i64, i32, vp],
        "at_orthogonalize": [vp, i32, i64, i64, i64, i64, i64, i32, f32, f32, f32, f32, f32, vp, i32, i64, i64, vp,
                             i64, vp],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    for name in ("at_space_destroy", "at_ensemble_destroy", "at_chains_destroy"):
        getattr(L, name).restype = None
    L.at_last_error.restype = ctypes.c_char_p
    return L


_lib = _load()


def lib():
    return _lib


def _check(func: str, st: int):
    if st != 0:
        raise ATError(func, st, _lib.at_last_error().decode())


def _np(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def _dev(t, dtype=None, name="tensor"):
    """Raw device pointer of a CUDA/HIP torch tensor (contiguous)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


class _Handle:
    _destroy = None

    def __init__(self, h):
        self.h = h

    def close(self):
        if self.h:
            getattr(_lib, self._destroy)(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Space(_Handle):
    _destroy = "at_space_destroy"

    def info(self):
        return at_space_info(self)


class Ensemble(_Handle):
    _destroy = "at_ensemble_destroy"


class Chains(_Handle):
    _destroy = "at_chains_destroy"


def at_space_create(tmpl: int, shape) -> Space:
    sh = np.ascontiguousarray(shape, dtype=np.int64)
    h = ctypes.c_void_p()
    _check("at_space_create", _lib.at_space_create(int(tmpl), _np(sh), len(sh), ctypes.byref(h)))
    sp = Space(h)
    sp.n_knobs, sp.knob_sizes, sp.n_loops, sp.n_features, sp.n_configs = at_space_info(sp)
    return sp


def at_space_info(space: Space):
    nk, nl, nf = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    nc = ctypes.c_uint64()
    sizes = np.zeros(16, dtype=np.int32)
    _check("at_space_info", _lib.at_space_info(space.h, ctypes.byref(nk), _np(sizes), ctypes.byref(nl),
                                               ctypes.byref(nf), ctypes.byref(nc)))
    return nk.value, sizes[: nk.value].copy(), nl.value, nf.value, nc.value


def at_spaceset_create(spaces, chain_offsets) -> Space:
    arr = (ctypes.c_void_p * len(spaces))(*[s.h.value for s in spaces])
    off = np.ascontiguousarray(chain_offsets, dtype=np.int64)
    if len(off) != len(spaces) + 1:
        raise ValueError("chain_offsets must have len(spaces) + 1 entries")
    h = ctypes.c_void_p()
    _check("at_spaceset_create", _lib.at_spaceset_create(arr, len(spaces), _np(off), ctypes.byref(h)))
    sp = Space(h)
    sp.n_knobs, sp.knob_sizes, sp.n_loops, sp.n_features, sp.n_configs = at_space_info(sp)
    sp.chain_offsets = off.copy()
    return sp


def at_extract_features(space: Space, cfgs, feats, stream=None):
    """cfgs: device uint64 [n] (torch.int64 storage); feats: device int32 [n, F]."""
    import torch
    n = cfgs.numel()
    if feats.shape != (n, space.n_features):
        raise ValueError("feats must be [n, n_features]")
    _check("at_extract_features", _lib.at_extract_features(
        space.h, _dev(cfgs, torch.int64, "cfgs"), n, _dev(feats, torch.int32, "feats"), _stream(stream)))


def at_extract_features_full(space: Space, cfgs, feats, stream=None):
    """Full Appendix A.2 rows (13 per loop: loop-context columns with
    bitlen(top-down) and bitlen(bottom-up) after the annotation).
    cfgs: device uint64 [n] (torch.int64 storage); feats: device int32
    [n, 13 * n_loops]."""
    import torch
    n = cfgs.numel()
    if feats.shape != (n, 13 * space.n_loops):
        raise ValueError("feats must be [n, 13 * n_loops]")
    _check("at_extract_features_full", _lib.at_extract_features_full(
        space.h, _dev(cfgs, torch.int64, "cfgs"), n, _dev(feats, torch.int32, "feats"), _stream(stream)))


ONEHOT_PER_LOOP = 24


def at_extract_features_onehot(space: Space, cfgs, feats, stream=None):
    """Appendix A.2 rows with a one-hot annotation (24 per loop: length,
    12 annotation columns, top-down, bottom-up, touch/reuse/stride per
    buffer).  cfgs: device uint64 [n] (torch.int64 storage); feats: device
    int32 [n, 24 * n_loops]."""
    import torch
    n = cfgs.numel()
    if feats.shape != (n, ONEHOT_PER_LOOP * space.n_loops):
        raise ValueError("feats must be [n, 24 * n_loops]")
    _check("at_extract_features_onehot", _lib.at_extract_features_onehot(
        space.h, _dev(cfgs, torch.int64, "cfgs"), n, _dev(feats, torch.int32, "feats"), _stream(stream)))


RELATION_FEATURES = 192


def at_extract_relation_features(space: Space, cfgs, feats, stream=None):
    """cfgs: device uint64 [n] (torch.int64 storage); feats: device int32 [n, 192]."""
    import torch
    n = cfgs.numel()
    if feats.shape != (n, RELATION_FEATURES):
        raise ValueError("feats must be [n, 192]")
    _check("at_extract_relation_features", _lib.at_extract_relation_features(
        space.h, _dev(cfgs, torch.int64, "cfgs"), n, _dev(feats, torch.int32, "feats"), _stream(stream)))


def at_space_errors(space: Space) -> int:
    v = ctypes.c_uint64()
    _check("at_space_errors", _lib.at_space_errors(space.h, ctypes.byref(v)))
    return v.value


def at_ensemble_create(fid, thr, leaf, n_features: int) -> Ensemble:
    """fid, thr: host uint8 [T, 2^d-1]; leaf: host float32 [T, 2^d]."""
    fid = np.ascontiguousarray(fid, dtype=np.uint8)
    thr = np.ascontiguousarray(thr, dtype=np.uint8)
    leaf = np.ascontiguousarray(leaf, dtype=np.float32)
    T, n_int = fid.shape
    depth = int(n_int + 1).bit_length() - 1
    if thr.shape != fid.shape or leaf.shape != (T, 1 << depth) or (1 << depth) - 1 != n_int:
        raise ValueError("inconsistent ensemble tables")
    h = ctypes.c_void_p()
    _check("at_ensemble_create", _lib.at_ensemble_create(T, depth, int(n_features), _np(fid), _np(thr), _np(leaf),
                                                         ctypes.byref(h)))
    e = Ensemble(h)
    e.n_trees, e.depth, e.n_features = T, depth, int(n_features)
    return e


def _node_lists(trees):
    keys = ("offsets", "left", "right", "feature", "threshold", "value")
    dt = (np.int32,) * 4 + (np.float32,) * 2
    arr = [np.ascontiguousarray(trees[k], dtype=d) for k, d in zip(keys, dt)]
    m = len(arr[1])
    if len(arr[0]) < 2 or any(len(a) != m for a in arr[1:]) or arr[0][0] < 0 or arr[0][-1] > m:
        raise ValueError("inconsistent node lists")
    return arr


def at_trees_depth(trees) -> int:
    """Level of the deepest leaf of node-list trees (dict of offsets, left,
    right, feature, threshold, value; host arrays)."""
    off, left, right, _, _, _ = _node_lists(trees)
    d = ctypes.c_int()
    _check("at_trees_depth", _lib.at_trees_depth(len(off) - 1, _np(off), _np(left), _np(right), ctypes.byref(d)))
    return d.value


def at_trees_pad(trees, n_features: int, depth: int):
    """Full-tree tables (fid, thr uint8 [T, 2^d-1], leaf float32 [T, 2^d]) of
    node-list trees, padded to `depth`."""
    off, left, right, feat, th, val = _node_lists(trees)
    T = len(off) - 1
    dd = depth if 1 <= depth <= 12 else 1      # the library rejects other depths
    fid = np.zeros((T, (1 << dd) - 1), np.uint8)
    thr = np.zeros((T, (1 << dd) - 1), np.uint8)
    leaf = np.zeros((T, 1 << dd), np.float32)
    _check("at_trees_pad", _lib.at_trees_pad(T, _np(off), _np(left), _np(right), _np(feat), _np(th), _np(val),
                                             int(n_features), int(depth), _np(fid), _np(thr), _np(leaf)))
    return fid, thr, leaf


def at_ensemble_import(trees, n_features: int) -> Ensemble:
    """Ensemble from node-list trees of any shape, padded on the host to the
    deepest leaf's depth."""
    off, left, right, feat, th, val = _node_lists(trees)
    T = len(off) - 1
    h = ctypes.c_void_p()
    _check("at_ensemble_import", _lib.at_ensemble_import(T, _np(off), _np(left), _np(right), _np(feat), _np(th),
                                                         _np(val), int(n_features), ctypes.byref(h)))
    e = Ensemble(h)
    e.n_trees, e.depth, e.n_features = T, max(1, at_trees_depth(trees)), int(n_features)
    return e


def at_gbt_predict(ens: Ensemble, feats, scores, leaves=None, stream=None):
    """feats: device int32 [n, F]; scores: device float32 [n]; leaves: device int16 [n, T] or None."""
    import torch
    n = feats.shape[0]
    if feats.dim() != 2 or feats.shape[1] != ens.n_features or scores.numel() != n:
        raise ValueError("shape mismatch")
    if leaves is not None and leaves.shape != (n, ens.n_trees):
        raise ValueError("leaves must be [n, n_trees]")
    _check("at_gbt_predict", _lib.at_gbt_predict(
        ens.h, _dev(feats, torch.int32, "feats"), n, _dev(scores, torch.float32, "scores"),
        _dev(leaves, torch.int16, "leaves"), _stream(stream)))


def at_gbt_predict_global_local(glob: Ensemble, feats_global, local: Ensemble, feats_local, scores, stream=None):
    """Eq. 4: scores = global(feats_global) + local(feats_local), device tensors."""
    import torch
    n = scores.numel()
    if feats_global.shape != (n, glob.n_features) or feats_local.shape != (n, local.n_features):
        raise ValueError("shape mismatch")
    _check("at_gbt_predict_global_local", _lib.at_gbt_predict_global_local(
        glob.h, _dev(feats_global, torch.int32, "feats_global"), local.h, _dev(feats_local, torch.int32, "feats_local"),
        n, _dev(scores, torch.float32, "scores"), _stream(stream)))


def at_chains_create(space: Space, chain0: int, n_chains: int, topk: int, seed: int) -> Chains:
    h = ctypes.c_void_p()
    _check("at_chains_create", _lib.at_chains_create(space.h, int(chain0), int(n_chains), int(topk), int(seed),
                                                     ctypes.byref(h)))
    c = Chains(h)
    c.chain0, c.n_chains, c.topk, c.seed = int(chain0), int(n_chains), int(topk), int(seed)
    return c


def at_chains_step(chains: Chains) -> int:
    v = ctypes.c_uint64()
    _check("at_chains_step", _lib.at_chains_step(chains.h, ctypes.byref(v)))
    return v.value


def at_chains_set_path(chains: Chains, path: int):
    _check("at_chains_set_path", _lib.at_chains_set_path(chains.h, int(path)))


def at_chains_last_path(chains: Chains) -> int:
    v = ctypes.c_int()
    _check("at_chains_last_path", _lib.at_chains_last_path(chains.h, ctypes.byref(v)))
    return v.value


PLAN_KEYS_LOCAL = ["chains_per_wg", "threads", "workgroups", "trees_per_chunk", "chunks", "gather", "lds_bytes",
                   "stream_bytes_per_step"]
PLAN_KEYS_TREES = ["trees_per_wg", "waves", "workgroups", "slices", "slice_blocks", "chain_workgroups",
                   "tile_quads", "v_bytes_per_step"]


def at_chains_last_plan(chains: Chains) -> dict:
    """Launch plan of the last run, keyed by the layout of the path it took
    (PLAN_KEYS_LOCAL or PLAN_KEYS_TREES), plus "path"."""
    v = np.zeros(8, np.int64)
    _check("at_chains_last_plan", _lib.at_chains_last_plan(chains.h, _np(v)))
    path = at_chains_last_path(chains)
    keys = PLAN_KEYS_TREES if path == AT_SA_PATH_TREES else PLAN_KEYS_LOCAL
    plan = dict(zip(keys, (int(x) for x in v)))
    plan["path"] = path
    return plan


def _select(name, space: Space, cand, pool, n_greedy, alpha, n_random, seed, out, stream):
    import torch
    n_cand = cand.numel() // 4 if cand is not None else 0
    if cand is not None and (cand.dtype != torch.int32 or cand.shape[-1] != 4 or not cand.is_contiguous()):
        raise ValueError("cand must be a contiguous int32 [..., 4] at_entry tensor")
    if out.shape != (n_greedy + n_random, 4):
        raise ValueError("out must be [n_greedy + n_random, 4] int32")
    _check(name, getattr(_lib, name)(
        space.h, _dev(cand, torch.int32, "cand") if n_cand else None, int(n_cand), int(pool), int(n_greedy),
        float(alpha), int(n_random), int(seed), _dev(out, torch.int32, "out"), _stream(stream)))


def at_select_batch(space: Space, cand, pool: int, n_greedy: int, alpha: float, n_random: int, seed: int, out,
                    stream=None):
    """cand: device int32 [..., 4] (at_entry, any leading shape); out: device
    int32 [n_greedy + n_random, 4] (at_entry)."""
    _select("at_select_batch", space, cand, pool, n_greedy, alpha, n_random, seed, out, stream)


def at_select_batch_noalloc(space: Space, cand, pool: int, n_greedy: int, alpha: float, n_random: int, seed: int,
                            out, stream=None):
    """at_select_batch without device allocation (the library's fixed
    per-device scratch; calls that overlap on one device race)."""
    _select("at_select_batch_noalloc", space, cand, pool, n_greedy, alpha, n_random, seed, out, stream)


def at_sa_thresholds(seed: int, chain0: int, n_chains: int, step_base: int, steps: int) -> np.ndarray:
    out = np.zeros((n_chains, steps), dtype=np.float32)
    _check("at_sa_thresholds", _lib.at_sa_thresholds(int(seed), int(chain0), int(n_chains), int(step_base),
                                                     int(steps), _np(out)))
    return out


def at_sa_run(space: Space, ens: Ensemble, chains: Chains, steps: int, thr, best, stream=None):
    """thr: device float32 [n_chains, steps]; best: device int32 [n_chains, topk, 4] (at_entry)."""
    import torch
    _check_sa(chains, steps, thr, best)
    _check("at_sa_run", _lib.at_sa_run(space.h, ens.h, chains.h, int(steps), _dev(thr, torch.float32, "thr"),
                                       _dev(best, torch.int32, "best"), _stream(stream)))


def at_sa_run_traced(space: Space, ens: Ensemble, chains: Chains, steps: int, thr, best, trace, stream=None):
    """as at_sa_run; trace: device int32 [n_chains, steps, 4] (at_entry)."""
    import torch
    _check_sa(chains, steps, thr, best)
    if trace.shape != (chains.n_chains, steps, 4):
        raise ValueError("trace must be [n_chains, steps, 4] int32")
    _check("at_sa_run_traced", _lib.at_sa_run_traced(
        space.h, ens.h, chains.h, int(steps), _dev(thr, torch.float32, "thr"), _dev(best, torch.int32, "best"),
        _dev(trace, torch.int32, "trace"), _stream(stream)))


def at_sa_run_global_local(space: Space, glob: Ensemble, local: Ensemble, chains: Chains, steps: int, thr, best,
                           trace=None, stream=None):
    """Annealing with Eq. 4's energy: glob over the 192 relation features
    plus local over the loop features.  thr: device float32 [n_chains,
    steps]; best: device int32 [n_chains, topk, 4]; trace: device int32
    [n_chains, steps, 4] or None."""
    import torch
    _check_sa(chains, steps, thr, best)
    if trace is not None and trace.shape != (chains.n_chains, steps, 4):
        raise ValueError("trace must be [n_chains, steps, 4] int32")
    _check("at_sa_run_global_local", _lib.at_sa_run_global_local(
        space.h, glob.h, local.h, chains.h, int(steps), _dev(thr, torch.float32, "thr"),
        _dev(best, torch.int32, "best"), _dev(trace, torch.int32, "trace"), _stream(stream)))


def _check_sa(chains, steps, thr, best):
    if thr is not None and thr.numel() != chains.n_chains * steps:
        raise ValueError("thr must hold n_chains * steps values")
    if best.shape != (chains.n_chains, chains.topk, 4):
        raise ValueError("best must be [n_chains, topk, 4] int32")


def at_chains_export(chains: Chains, cur_cfg=None, cur_score=None, stream=None):
    import torch
    _check("at_chains_export", _lib.at_chains_export(
        chains.h, _dev(cur_cfg, torch.int64, "cur_cfg"), _dev(cur_score, torch.float32, "cur_score"),
        _stream(stream)))


def at_sa_set_profiling(chains: Chains, enable: bool):
    _check("at_sa_set_profiling", _lib.at_sa_set_profiling(chains.h, 1 if enable else 0))


def at_sa_kernel_times(chains: Chains) -> dict:
    """Device time of the last profiled run's launches (waits for the run)."""
    tms, cms = ctypes.c_double(0), ctypes.c_double(0)
    tn, cn = ctypes.c_int64(0), ctypes.c_int64(0)
    _check("at_sa_kernel_times", _lib.at_sa_kernel_times(chains.h, ctypes.byref(tms), ctypes.byref(tn),
                                                         ctypes.byref(cms), ctypes.byref(cn)))
    return {"tree_ms": tms.value, "tree_launches": tn.value, "chain_ms": cms.value, "chain_launches": cn.value}


def entries(t) -> np.ndarray:
    """Host structured view (cfg, score, flag) of a device at_entry tensor [..., 4] int32."""
    a = t.detach().cpu().contiguous().numpy()
    return a.view(ENTRY_DTYPE).reshape(a.shape[:-1])


# --------------------------------------------------------------------------
# Operators of sequence models over schedule tokens.  Tensors with rows may have
# any row stride (a last stride of 1); vectors are contiguous.  Outputs are
# the caller's; a workspace may be given as a uint8 tensor (the *_workspace
# functions say how many bytes), else one is taken from torch's allocator on the
# call's stream.  Gradients are calls of their own: nothing is recorded for
# autograd, which is told that the outputs changed, so that it refuses to use
# what they overwrote.
# --------------------------------------------------------------------------
AT_F32, AT_BF16, AT_F16 = 0, 1, 2
AT_I32, AT_I64 = 0, 1
AT_FP16_PRODUCTS = 16
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


class _Torch:
    """What these bindings need of torch, looked up once: a call costs a few
    microseconds, which is what the smallest of these operators take."""

    def __init__(self):
        import torch
        self.torch = torch
        self.types = {torch.float32: AT_F32, torch.bfloat16: AT_BF16, torch.float16: AT_F16}
        self.itypes = {torch.int32: AT_I32, torch.int64: AT_I64}
        self.f32, self.i32 = torch.float32, torch.int32
        # the current stream's handle, without the object around it where torch has that
        self.stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
        self.written = torch.autograd.graph.increment_version


_torch_parts = None


def _T() -> _Torch:
    global _torch_parts
    if _torch_parts is None:
        _torch_parts = _Torch()
    return _torch_parts


def _type(t, name):
    c = _T().types.get(t.dtype)
    if c is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return c


def _rows(t, name, rows=None, cols=None):
    """(pointer, element type, row stride) of a device tensor [rows, cols]."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    sh = t.shape
    if len(sh) != 2 or (rows is not None and sh[0] != rows) or (cols is not None and sh[1] != cols):
        raise ValueError(f"{name} must be [{'n' if rows is None else rows}, {'n' if cols is None else cols}], "
                         f"got {list(sh)}")
    st = t.stride()
    if sh[1] > 1 and st[1] != 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), _type(t, name), (st[0] if sh[0] > 1 else max(st[0], sh[1]))


def _vec(t, n, dtype, name):
    """Pointer of a contiguous device tensor of n values, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n:
        raise ValueError(f"{name} must hold {n} values of {dtype}")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    return t.data_ptr()


def _tokens(t, n=None):
    """(pointer, token type, count) of an int32 or int64 device tensor."""
    ti = _T().itypes.get(t.dtype)
    if ti is None:
        raise ValueError(f"tokens must be int32 or int64, got {t.dtype}")
    m = t.numel()
    if n is not None and m != n:
        raise ValueError(f"tokens must hold {n} values")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tokens must be a contiguous device tensor")
    return t.data_ptr(), ti, m


def _one_device(*tensors) -> int:
    d = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != d:
            raise ValueError("tensors are on different devices")
    return d


def _call(func, device: int, stream, args, outs, workspace=None, need: int = 0):
    """Calls the library on `device`, with `stream` or the device's current one
    as the last argument; outs: the tensors that it writes; where the call takes a workspace (need >= 0, the bytes),
    its pointer and size come before the stream."""
    T = _T()
    torch = T.torch
    if torch.cuda.current_device() != device:
        with torch.cuda.device(device):
            return _call(func, device, stream, args, outs, workspace, need)
    if need >= 0:
        if workspace is None:
            if not need:
                args += (None, 0)
            elif stream is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
            else:   # torch's allocator ties memory to the stream it is taken on
                with torch.cuda.stream(stream):
                    workspace = torch.empty(need, dtype=torch.uint8, device=device)
        if workspace is not None:
            if workspace.get_device() != device:
                raise ValueError("workspace is on another device")
            args += (_vec(workspace, workspace.numel(), torch.uint8, "workspace"), workspace.numel())
    st = getattr(_lib, func)(*args, T.stream(device) if stream is None else stream.cuda_stream)
    if st:
        _check(func, st)
    T.written(outs)


@functools.lru_cache(maxsize=256)
def _bytes(func, *sizes) -> int:
    v = ctypes.c_int64()
    _check(func, getattr(_lib, func)(*sizes, ctypes.byref(v)))
    return v.value


def at_embed(weight, tokens, out, scale: float = 1.0, stream=None):
    """out[i, :] = scale * weight[tokens[i], :]; zeros for tokens outside
    [0, vocab).  weight: [vocab, dim]; tokens: int32 or int64 [n]; out: [n, dim];
    weight and out each float32, bfloat16 or float16."""
    tp, ti, n = _tokens(tokens)
    wp, wt, lw = _rows(weight, "weight")
    vocab, dim = weight.shape
    op, ot, lo = _rows(out, "out", n, dim)
    _call("at_embed", _one_device(weight, tokens, out), stream,
          (wp, wt, lw, vocab, dim, tp, ti, n, scale, op, ot, lo), out, need=-1)


def at_embed_grad_workspace(n: int, vocab: int, dim: int) -> int:
    return _bytes("at_embed_grad_workspace", n, vocab, dim)


def at_embed_grad(dout, tokens, dweight, scale: float = 1.0, accumulate: bool = False, workspace=None, stream=None):
    """dweight[v, :] = scale * the sum of dout[i, :] with tokens[i] == v, or
    added to dweight with accumulate.  dout: [n, dim]; tokens: int32 or int64
    [n]; dweight: [vocab, dim]."""
    tp, ti, n = _tokens(tokens)
    gp, gt, lg = _rows(dweight, "dweight")
    vocab, dim = dweight.shape
    dp, dt, ld = _rows(dout, "dout", n, dim)
    _call("at_embed_grad", _one_device(dout, tokens, dweight), stream,
          (dp, dt, ld, tp, ti, n, scale, 1 if accumulate else 0, gp, gt, lg, vocab, dim), dweight, workspace,
          _bytes("at_embed_grad_workspace", n, vocab, dim))


def at_logprobs_workspace(n: int, vocab: int, k: int) -> int:
    return _bytes("at_logprobs_workspace", n, vocab, k)


def at_logprobs(logits, tokens=None, logp=None, entropy=None, lse=None, top_logp=None, top_idx=None, valid=None,
                scale: float = 1.0, workspace=None, stream=None):
    """Log probabilities of tokens under softmax(scale * logits), entropies, log
    sums, and the k largest logits' columns and log probabilities.  logits:
    [n, vocab]; tokens: int32 or int64 [n] (negative: none) or None; valid:
    int32 [n], the columns that each row has, or None; logp, entropy, lse:
    float32 [n]; top_logp: float32 [n, k]; top_idx: int32 [n, k]; an output
    that is None is not computed."""
    T = _T()
    xp, xt, ld = _rows(logits, "logits")
    n, vocab = logits.shape
    tp, ti, _ = _tokens(tokens, n) if tokens is not None else (None, AT_I32, n)
    k = 0
    for t in (top_logp, top_idx):
        if t is not None:
            if t.dim() != 2 or t.shape[0] != n or (k and t.shape[1] != k):
                raise ValueError("top_logp and top_idx must be [n, k]")
            k = t.shape[1]
    _call("at_logprobs", _one_device(logits, tokens, logp, entropy, lse, top_logp, top_idx, valid), stream,
          (xp, xt, ld, n, vocab, _vec(valid, n, T.i32, "valid"), tp, ti, scale, k, _vec(logp, n, T.f32, "logp"),
           _vec(entropy, n, T.f32, "entropy"), _vec(lse, n, T.f32, "lse"), _vec(top_logp, n * k, T.f32, "top_logp"),
           _vec(top_idx, n * k, T.i32, "top_idx")),
          [t for t in (logp, entropy, lse, top_logp, top_idx) if t is not None], workspace,
          _bytes("at_logprobs_workspace", n, vocab, k))


def at_logprobs_grad(logits, tokens, lse, entropy, dlogp, dlogits, dentropy=None, valid=None, scale: float = 1.0,
                     stream=None):
    """Gradient of at_logprobs with respect to its logits, from those of logp and
    entropy (float32 [n], or None for zero) and the forward call's lse and
    entropy.  dlogits: [n, vocab] of the logits' type."""
    T = _T()
    xp, xt, ld = _rows(logits, "logits")
    n, vocab = logits.shape
    dp, dt, ldd = _rows(dlogits, "dlogits", n, vocab)
    if dt != xt:
        raise ValueError("dlogits must have the logits' type")
    tp, ti, _ = _tokens(tokens, n) if tokens is not None else (None, AT_I32, n)
    _call("at_logprobs_grad", _one_device(logits, tokens, lse, entropy, dlogp, dlogits, dentropy, valid), stream,
          (xp, xt, ld, n, vocab, _vec(valid, n, T.i32, "valid"), tp, ti, scale, _vec(lse, n, T.f32, "lse"),
           _vec(entropy, n, T.f32, "entropy"), _vec(dlogp, n, T.f32, "dlogp"), _vec(dentropy, n, T.f32, "dentropy"), dp,
           ldd), dlogits, need=-1)


def _matrices(t, name):
    """(pointer, matrix stride, row stride) of a device tensor [batch, rows, cols] or [rows, cols]."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be [rows, cols] or [batch, rows, cols]")
    sh, st = t.shape, t.stride()
    if sh[-1] > 1 and st[-1] != 1:
        raise ValueError(f"{name} must have contiguous rows")
    ld = st[-2] if sh[-2] > 1 else max(st[-2], sh[-1])
    return t.data_ptr(), (st[0] if len(sh) == 3 else 0), ld


def at_orthogonalize_workspace(batch: int, rows: int, cols: int, otype: int = AT_BF16) -> int:
    return _bytes("at_orthogonalize_workspace", batch, rows, cols, otype)


def at_orthogonalize(x, out, steps: int = 5, coef=NEWTON_SCHULZ, eps: float = 1e-7, scale: float = 1.0, workspace=None,
                     stream=None, fp16_products: bool = False):
    """Newton-Schulz steps on each matrix of x ([rows, cols] or [batch, rows,
    cols]; float32, bfloat16 or float16), normalised first, into out (bfloat16
    or float32, the same shape), times scale.  Products have fp32's accuracy;
    fp16_products rounds their operands to fp16 where the shorter side is above
    128: about 0.4 of the time for large matrices, bf16 results within 2.4e-3
    of their norm for 1.7e-3 (its workspace: otype | AT_FP16_PRODUCTS)."""
    if out.shape != x.shape:
        raise ValueError("out must have x's shape")
    xp, xb, ldx = _matrices(x, "x")
    op, ob, ldo = _matrices(out, "out")
    batch = x.shape[0] if x.dim() == 3 else 1
    rows, cols = x.shape[-2:]
    a, b, c = coef
    ot = _type(out, "out") | (AT_FP16_PRODUCTS if fp16_products else 0)
    _call("at_orthogonalize", _one_device(x, out), stream,
          (xp, _type(x, "x"), xb, ldx, batch, rows, cols, steps, a, b, c, eps, scale, op, ot, ob, ldo), out, workspace,
          _bytes("at_orthogonalize_workspace", batch, rows, cols, ot))
