"""Python binding of ``libcpes`` -- the gfx950 C-ABI library of the CoPES
parameter-space hot path (see ``include/cpes.h``).

Argument marshalling only: every step runs in the library's HIP kernels.
Tensors must live on the GPU; streams default to torch's current stream.
There is no CPU fallback: if ``libcpes.so`` is missing or fails to load, every
call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libcpes.so")

OK, ERR_INVALID_ARGUMENT, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, -1, -2, -3, -4
BF16, F32 = 0, 1
PART_CONTIGUOUS, PART_PERMUTATION = 0, 1
AUX_NONE, AUX_SNAPSHOT, AUX_MASTER, AUX_BACKUP = 0, 1, 2, 3
NORM_Z, NORM_RANK = 0, 1
SCALE_ALPHA_OVER_N_SIGMA, SCALE_ALPHA_OVER_N = 0, 1
SUB_ASCENDING = 1
MAX_MEMBERS, MAX_REWARDS, MAX_GROUPS, MAX_PERMUTATION_K, MAX_STEP_SUBSPACES = 256, 4096, 1024, 256, 32
MAX_HEAD_DIM, MAX_HEADS, MAX_ALTERNATIVES, MAX_SEQUENCES, MAX_TREE = 256, 65536, 64, 1 << 20, 256
PAGES_OK, PAGES_SHORT, PAGES_BAD_SEQUENCE = 0, 1, 2

EXPORTED = (
    "cpes_partition", "cpes_partition32", "cpes_partition_workspace_bytes", "cpes_partition_chunks",
    "cpes_partition_chunks_workspace_bytes", "cpes_partition_chunks_static", "cpes_perturb", "cpes_restore", "cpes_backup",
    "cpes_backup_to_host", "cpes_restore_from_host", "cpes_stage_master", "cpes_normalize_rewards",
    "cpes_update", "cpes_update_step", "cpes_update_step32", "cpes_pages_workspace_bytes", "cpes_pages_reserve",
    "cpes_pages_fork", "cpes_pages_free", "cpes_pages_copy", "cpes_pages_compact", "cpes_cache_append",
    "cpes_attend_workspace_bytes", "cpes_attend", "cpes_logprobs_workspace_bytes", "cpes_logprobs",
    "cpes_logprobs_backward", "cpes_pages_keep_workspace_bytes", "cpes_pages_keep", "cpes_attend_tree_workspace_bytes",
    "cpes_attend_tree", "cpes_tree_accept", "cpes_sample_workspace_bytes", "cpes_sample", "cpes_debug_philox", "cpes_debug_normals", "cpes_debug_bm_grid",
    "cpes_debug_prp", "cpes_rng_probe", "cpes_probe_map_copy", "cpes_probe_copy", "cpes_fill_normal",
    "cpes_last_error", "cpes_abi_version",
)


class CpesError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{message} (status {code})")
        self.code = code


class Subspace(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_int64), ("length", ctypes.c_int64), ("index", ctypes.c_void_p),
                ("chunk", ctypes.c_int64), ("index32", ctypes.c_void_p), ("noise_offset", ctypes.c_int64),
                ("flags", ctypes.c_int64)]


class Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("layers", ctypes.c_int32), ("pages", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Pool(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("sequences", ctypes.c_int32), ("width", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load ``libcpes.so`` (built by ``paper_2608_02391_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2608_02391_amd.build`")
    L = ctypes.CDLL(path)
    vp, i64, u64, i32, u32, f32 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int32,
                                   ctypes.c_uint32, ctypes.c_float)
    sp, kc, pp, size = ctypes.POINTER(Subspace), ctypes.POINTER(Cache), ctypes.POINTER(Pool), ctypes.c_size_t
    sig = {
        "cpes_partition": [i32, i64, i32, u64, vp, vp, vp, vp, ctypes.c_size_t, vp, vp],
        "cpes_partition32": [i64, i32, u64, vp, vp, vp, ctypes.c_size_t, vp, vp],
        "cpes_partition_workspace_bytes": [i32, i64, i32],
        "cpes_partition_chunks": [i64, i64, i32, u64, vp, vp, vp, vp, ctypes.c_size_t, vp, vp],
        "cpes_partition_chunks_workspace_bytes": [i64, i64, i32],
        "cpes_partition_chunks_static": [i64, i64, i32, u64, vp, vp, vp, vp, vp],
        "cpes_perturb": [vp, i64, i32, sp, f32, u64, i32, vp, i32, vp],
        "cpes_restore": [vp, i64, i32, sp, f32, u64, i32, vp, i32, vp],
        "cpes_backup": [vp, i64, i32, sp, vp, vp],
        "cpes_backup_to_host": [vp, i64, i32, sp, vp, vp],
        "cpes_restore_from_host": [vp, i64, i32, sp, vp, vp],
        "cpes_stage_master": [vp, i64, i32, sp, vp, vp],
        "cpes_normalize_rewards": [vp, i32, i32, vp, i32, vp, vp, vp],
        "cpes_update": [vp, i64, i32, sp, vp, i32, vp, vp, vp, f32, f32, i32, vp],
        "cpes_update_step": [vp, i64, i32, i32, vp, vp, i64, vp, i32, vp, vp, vp, vp, f32, vp, i32, vp],
        "cpes_update_step32": [vp, i64, i32, i32, vp, vp, i32, vp, vp, vp, vp, f32, vp, i32, vp],
        "cpes_pages_workspace_bytes": [i32],
        "cpes_pages_reserve": [pp, i32, vp, vp, vp, size, vp, vp],
        "cpes_pages_fork": [kc, pp, i32, vp, vp, vp, size, vp, vp],
        "cpes_pages_free": [pp, i32, vp, vp, vp],
        "cpes_pages_copy": [kc, i32, vp, vp, vp],
        "cpes_pages_compact": [kc, pp, pp, vp, size, vp, vp],
        "cpes_cache_append": [kc, i32, pp, i32, vp, vp, vp, vp, i64, i64, vp],
        "cpes_attend_workspace_bytes": [i32, i32, i32, i32],
        "cpes_attend": [kc, i32, pp, i32, vp, vp, i64, i64, i32, f32, i32, i32, vp, i64, i64, vp, vp, size, vp],
        "cpes_logprobs_workspace_bytes": [i32, i32, i32],
        "cpes_logprobs": [vp, i32, i32, i32, i64, f32, vp, vp, vp, vp, vp, i32, vp, vp, vp, size, vp],
        "cpes_logprobs_backward": [vp, i32, i32, i32, i64, f32, vp, vp, vp, vp, vp, vp, i64, vp],
        "cpes_pages_keep_workspace_bytes": [i32, i32],
        "cpes_pages_keep": [kc, pp, i32, vp, vp, i32, vp, vp, vp, size, vp, vp],
        "cpes_attend_tree_workspace_bytes": [i32, i32, i32, i32, i32, i32],
        "cpes_attend_tree": [kc, i32, pp, i32, vp, vp, i32, i32, vp, vp, i64, i64, i32, f32, i32, i32, vp, i64, i64, vp, vp,
                             size, vp],
        "cpes_tree_accept": [i32, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp],
        "cpes_sample_workspace_bytes": [i32, i32],
        "cpes_sample": [vp, i32, i32, i32, i64, f32, i32, f32, f32, vp, vp, vp, vp, size, vp],
        "cpes_debug_philox": [u64, u32, u64, i64, vp, vp],
        "cpes_debug_normals": [u64, i64, i64, vp, vp],
        "cpes_debug_bm_grid": [u32, i64, vp, vp, vp, vp],
        "cpes_debug_prp": [u64, i64, i32, i64, i64, vp, vp, vp],
        "cpes_rng_probe": [u64, i64, vp, vp],
        "cpes_probe_map_copy": [vp, i64, i32, sp, vp, i32, vp],
        "cpes_probe_copy": [vp, vp, i64, i32, vp],
        "cpes_fill_normal": [vp, i64, i32, u64, u32, f32, vp],
        "cpes_last_error": [],
        "cpes_abi_version": [],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    for name in sig:
        if name.endswith("_workspace_bytes"):
            getattr(L, name).restype = ctypes.c_size_t
    L.cpes_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


def last_error() -> str:
    return load().cpes_last_error().decode()


def _check(rc: int) -> None:
    if rc != OK:
        raise CpesError(rc, last_error())


# ----------------------------------------------------------- marshalling --

# A call costs the host about 4 us, 2.4 of them the launch, in front of a kernel
# that takes 3 us on 262,144 parameters, so a step of small calls is bound by the
# host: the module, the dtype codes and the stream getters are looked up once
# (this file's share of a call 2.1 -> 1.4 us with a side buffer, 1.6 -> 0.9 us
# without; a step of 18 such calls 95.7 -> 87.4 us).
_torch_module = None
_dtype_codes: dict = {}


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch

        _dtype_codes.update({torch.bfloat16: BF16, torch.float32: F32})
        _torch_module = torch
    return _torch_module


def _dtype_code(t, what: str = "weights") -> int:
    code = _dtype_codes.get(t.dtype)
    if code is None:
        _torch()                        # the table is empty before the first call
        code = _dtype_codes.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be bfloat16 or float32, not {t.dtype}")
    return code


def _dev_ptr(t, what: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _need(t, what: str, numel: int, dtype=None) -> None:
    """A device buffer the kernels will address: it must hold ``numel``
    elements (of ``dtype`` when given).  The C ABI takes bare pointers and
    cannot see sizes, so the binding checks them before any launch."""
    if t is None:
        return
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must have dtype {dtype}, not {t.dtype}")
    if t.numel() < numel:
        raise ValueError(f"{what} holds {t.numel()} elements, {numel} needed")


def _aux_need(w, s: "Subspace", aux, aux_mode: int, what: str = "aux") -> None:
    if aux is None:
        return
    if aux_mode == AUX_MASTER:
        _need(aux, what, s.length, _torch().float32)
    elif aux_mode == AUX_SNAPSHOT or aux_mode == AUX_BACKUP:
        _need(aux, what, s.length, w.dtype)


def _host_ptr(t, w, s: "Subspace", what: str) -> int:
    """A host backup: a CPU tensor of w's dtype holding at least s.length
    elements.  Whether it is pinned is checked by the library."""
    if t.is_cuda:
        raise ValueError(f"{what} must be a host tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if t.dtype != w.dtype:
        raise TypeError(f"{what} must have dtype {w.dtype}, not {t.dtype}")
    if t.numel() < s.length:
        raise ValueError(f"{what} holds {t.numel()} elements, {s.length} needed")
    return t.data_ptr()


_raw_stream = _get_device = None


def _current_stream() -> int:
    """torch's current stream on the current device, as a raw hipStream_t."""
    global _raw_stream, _get_device
    if _raw_stream is None:
        torch = _torch()
        raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is None or dev is None:
            return torch.cuda.current_stream().cuda_stream
        _get_device, _raw_stream = dev, raw
    return _raw_stream(_get_device())   # the same handle, without building a Stream object per call


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def subspace(offset: int, length: int, index=None, chunk: int = 0, noise_offset: int = 0,
             ascending: bool = False) -> Subspace:
    """Positions j < length at parameter offset + j, index[offset + j], or
    (chunk > 0) index[offset + j // chunk] * chunk + j % chunk; the map must
    hold the entries those positions read.  An int64 map
    goes to ``index``; a 32-bit map (torch.int32 or torch.uint32 holding the
    uint32 entries of cpes_partition32) goes to ``index32``.  Position j uses
    noise index noise_offset + j (a shard of a larger subspace).
    ascending=True sets CPES_SUB_ASCENDING: the element map is strictly
    ascending (a partition's own map), so bf16 perturbations and restores may
    rewrite whole 128-byte lines around its entries."""
    torch = _torch()
    idx64 = idx32 = None
    if index is not None:
        if length > 0:
            entries = offset + (-(-length // chunk) if chunk else length)
            _need(index, "index map", entries)
        if index.dtype == torch.int64:
            idx64 = _dev_ptr(index, "index map")
        elif index.dtype in (torch.int32, getattr(torch, "uint32", torch.int32)):
            idx32 = _dev_ptr(index, "index map")
        else:
            raise TypeError("index map must be int64, or 32-bit for a uint32 map")
    sub = Subspace(int(offset), int(length), idx64, int(chunk), idx32, int(noise_offset),
                   SUB_ASCENDING if ascending else 0)
    sub._index = index      # the descriptor holds a raw pointer: keep the map's storage alive with it
    return sub


# ------------------------------------------------------------- entry points --

def cpes_partition(mode: int, d: int, K: int, seed: int = 0, bounds: Optional[Sequence[int]] = None,
                   index=None, workspace=None, status=None, stream=None):
    """Returns the K+1 subspace offsets (host ints); PERMUTATION fills ``index``."""
    L = load()
    offsets = (ctypes.c_int64 * (K + 1))()
    b = None if bounds is None else (ctypes.c_int64 * (K + 1))(*[int(x) for x in bounds])
    if bounds is not None and len(bounds) != K + 1:
        raise ValueError(f"bounds needs K + 1 = {K + 1} entries, not {len(bounds)}")
    if mode == PART_PERMUTATION:
        _need(index, "index", d, _torch().int64)
    _need(status, "status", 1, _torch().int32)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(L.cpes_partition(mode, d, K, seed, b, offsets, _dev_ptr(index, "index"),
                            _dev_ptr(workspace, "workspace"), ws_bytes, _dev_ptr(status, "status"),
                            _stream(stream)))
    return [int(x) for x in offsets]


def cpes_partition32(d: int, K: int, seed: int, index, workspace, status=None, stream=None):
    """Permutation partition into a 32-bit map (d <= 2^32); returns the K+1 offsets."""
    L = load()
    offsets = (ctypes.c_int64 * (K + 1))()
    if index.element_size() != 4:
        raise TypeError("cpes_partition32 writes a 32-bit map")
    _need(index, "index", d)
    _need(status, "status", 1, _torch().int32)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(L.cpes_partition32(d, K, seed, offsets, _dev_ptr(index, "index"), _dev_ptr(workspace, "workspace"),
                              ws_bytes, _dev_ptr(status, "status"), _stream(stream)))
    return [int(x) for x in offsets]


def cpes_partition_workspace_bytes(mode: int, d: int, K: int) -> int:
    return int(load().cpes_partition_workspace_bytes(mode, d, K))


def cpes_partition_chunks(d: int, chunk: int, K: int, seed: int, chunks, workspace, status=None, stream=None):
    """Chunk-granular random partition; returns (list_offsets[K+1], lengths[K])."""
    L = load()
    offs = (ctypes.c_int64 * (K + 1))()
    lens = (ctypes.c_int64 * K)()
    _need(chunks, "chunks", -(-d // chunk) if chunk > 0 else 0, _torch().int64)
    _need(status, "status", 1, _torch().int32)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(L.cpes_partition_chunks(d, chunk, K, seed, offs, lens, _dev_ptr(chunks, "chunks"),
                                   _dev_ptr(workspace, "workspace"), ws_bytes, _dev_ptr(status, "status"),
                                   _stream(stream)))
    return [int(x) for x in offs], [int(x) for x in lens]


def cpes_partition_chunks_static(d: int, chunk: int, K: int, seed: int, chunks, status=None, stream=None):
    """cpes_partition_chunks on the library's own device scratch array (no
    workspace, no allocation); returns (list_offsets[K+1], lengths[K])."""
    L = load()
    offs = (ctypes.c_int64 * (K + 1))()
    lens = (ctypes.c_int64 * K)()
    _need(chunks, "chunks", -(-d // chunk) if chunk > 0 else 0, _torch().int64)
    _need(status, "status", 1, _torch().int32)
    _check(L.cpes_partition_chunks_static(d, chunk, K, seed, offs, lens, _dev_ptr(chunks, "chunks"),
                                          _dev_ptr(status, "status"), _stream(stream)))
    return [int(x) for x in offs], [int(x) for x in lens]


def cpes_partition_chunks_workspace_bytes(d: int, chunk: int, K: int) -> int:
    return int(load().cpes_partition_chunks_workspace_bytes(d, chunk, K))


def cpes_perturb(w, s: Subspace, sigma: float, seed: int, sign: int, aux=None, aux_mode: int = AUX_NONE,
                 stream=None) -> None:
    _aux_need(w, s, aux, aux_mode)
    _check((_lib or load()).cpes_perturb(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s), sigma, seed, sign,
                               _dev_ptr(aux, "aux"), aux_mode, _stream(stream)))


def cpes_restore(w, s: Subspace, sigma: float = 0.0, seed: int = 0, sign: int = 1, aux=None,
                 aux_mode: int = AUX_SNAPSHOT, stream=None) -> None:
    _aux_need(w, s, aux, aux_mode)
    _check((_lib or load()).cpes_restore(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s), sigma, seed, sign,
                               _dev_ptr(aux, "aux"), aux_mode, _stream(stream)))


def cpes_backup(w, s: Subspace, backup, stream=None) -> None:
    """backup[j] = w[p(j)] into a device tensor of w's dtype."""
    _need(backup, "backup", s.length, w.dtype)
    _check((_lib or load()).cpes_backup(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s),
                              _dev_ptr(backup, "backup"), _stream(stream)))


def cpes_backup_to_host(w, s: Subspace, backup, stream=None) -> None:
    """backup[j] = w[p(j)] into a pinned host tensor (``pin_memory=True``)."""
    _check((_lib or load()).cpes_backup_to_host(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s),
                                      _host_ptr(backup, w, s, "backup"), _stream(stream)))


def cpes_restore_from_host(w, s: Subspace, backup, stream=None) -> None:
    """w[p(j)] = backup[j] from a pinned host tensor."""
    _check((_lib or load()).cpes_restore_from_host(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s),
                                         _host_ptr(backup, w, s, "backup"), _stream(stream)))


def cpes_fill_normal(w, seed: int, domain: int = 1, stddev: float = 0.02, stream=None) -> None:
    """Fill the device tensor w with cast(stddev * z_j) from stream (seed, domain)."""
    _check((_lib or load()).cpes_fill_normal(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), seed, domain, stddev,
                                   _stream(stream)))


def cpes_stage_master(w, s: Subspace, master, stream=None) -> None:
    _need(master, "master", s.length, _torch().float32)
    _check((_lib or load()).cpes_stage_master(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s),
                                    _dev_ptr(master, "master"), _stream(stream)))


def cpes_normalize_rewards(r, out, mode: int = NORM_Z, group=None, n_groups: int = 1, status=None,
                           stream=None) -> None:
    torch = _torch()
    _need(r, "rewards", 0, torch.float32)
    _need(out, "out", r.numel(), torch.float32)
    _need(group, "group", r.numel(), torch.int32)
    _need(status, "status", 1, torch.int32)
    _check((_lib or load()).cpes_normalize_rewards(_dev_ptr(r, "rewards"), r.numel(), mode, _dev_ptr(group, "group"),
                                         n_groups, _dev_ptr(out, "out"), _dev_ptr(status, "status"),
                                         _stream(stream)))


def cpes_update(w, s: Subspace, seeds: Sequence[int], signs: Sequence[int], rnorm, alpha: float, sigma: float,
                scale_mode: int = SCALE_ALPHA_OVER_N_SIGMA, master=None, stream=None) -> None:
    n = len(seeds)
    if len(signs) != n:
        raise ValueError("seeds and signs differ in length")
    _need(rnorm, "rnorm", n, _torch().float32)
    _need(master, "master", s.length, _torch().float32)
    cs = (ctypes.c_uint64 * n)(*[int(x) & 0xFFFFFFFFFFFFFFFF for x in seeds])
    cg = (ctypes.c_int8 * n)(*[int(x) for x in signs])
    _check((_lib or load()).cpes_update(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s),
                              _dev_ptr(master, "master"), n, cs, cg, _dev_ptr(rnorm, "rnorm"), alpha, sigma,
                              scale_mode, _stream(stream)))


def cpes_update_step(w, offsets: Sequence[int], seeds: Sequence[int], signs: Sequence[int],
                     subspaces: Sequence[int], rnorm, alpha: float, sigmas: Sequence[float],
                     scale_mode: int = SCALE_ALPHA_OVER_N_SIGMA, index=None, chunk: int = 0,
                     lengths: Optional[Sequence[int]] = None, stream=None) -> None:
    """Update every subspace of a partition with its own members (one launch).
    ``index``: None (contiguous), an int64 map or chunk list, or a 32-bit map
    (cpes_partition32) that goes to cpes_update_step32."""
    K = len(offsets) - 1
    n = len(seeds)
    if not (len(signs) == len(subspaces) == n) or len(sigmas) != K:
        raise ValueError("inconsistent member or subspace arrays")
    co = (ctypes.c_int64 * (K + 1))(*[int(x) for x in offsets])
    cs = (ctypes.c_uint64 * n)(*[int(x) & 0xFFFFFFFFFFFFFFFF for x in seeds])
    cg = (ctypes.c_int8 * n)(*[int(x) for x in signs])
    ck = (ctypes.c_int32 * n)(*[int(x) for x in subspaces])
    csg = (ctypes.c_float * K)(*[float(x) for x in sigmas])
    torch = _torch()
    idx32 = index is not None and index.dtype in (torch.int32, getattr(torch, "uint32", torch.int32))
    if index is not None and index.dtype != torch.int64 and not idx32:
        raise TypeError("index map must be int64, or 32-bit for a uint32 map")
    if idx32 and chunk:
        raise ValueError("chunk lists are int64 maps")
    if lengths is not None and len(lengths) != K:
        raise ValueError(f"lengths needs K = {K} entries, not {len(lengths)}")
    _need(index, "index map", int(offsets[-1]))
    _need(rnorm, "rnorm", n, torch.float32)
    if idx32:
        _check((_lib or load()).cpes_update_step32(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), K, co, _dev_ptr(index, "index"),
                                         n, cs, cg, ck, _dev_ptr(rnorm, "rnorm"), alpha, csg, scale_mode,
                                         _stream(stream)))
        return
    cl = None if lengths is None else (ctypes.c_int64 * K)(*[int(x) for x in lengths])
    _check((_lib or load()).cpes_update_step(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), K, co, _dev_ptr(index, "index"),
                                   int(chunk), cl, n, cs, cg, ck, _dev_ptr(rnorm, "rnorm"), alpha, csg, scale_mode,
                                   _stream(stream)))


# ------------------------------------------------------ evaluating a member --

def _same_strides(a, b, shape) -> bool:
    """Whether two tensors of a shape lie alike: the stride of a dimension of one entry addresses nothing."""
    return a == b or all(x == y or n <= 1 for x, y, n in zip(a, b, shape))


def paged_cache(k, v) -> Cache:
    """A key-value cache in pages: k and v of shape [layers, pages, heads,
    page_size, head_dim], bfloat16 or float32, with the same strides and the
    last dimension contiguous (token-major pages are a transposed view)."""
    if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or not _same_strides(k.stride(), v.stride(), k.shape):
        raise ValueError("keys and values must be [layers, pages, heads, page_size, head_dim] of one shape, dtype and strides")
    if not (k.is_cuda and v.is_cuda):
        raise ValueError("keys and values must be GPU tensors")
    if k.stride(4) != 1 and k.shape[4] > 1:
        raise ValueError("the head dimension must be contiguous")
    st = k.stride()
    cache = Cache(k.data_ptr(), v.data_ptr(), st[0], st[1], st[2], st[3], *k.shape, _dtype_code(k, "keys and values"))
    cache._tensors = (k, v)     # the descriptor holds raw pointers: keep the storage alive with it
    cache._dtype = k.dtype
    return cache


def page_pool(table, lengths, page_size: int, refs=None) -> Pool:
    """The pages of sequences: ``table`` int32 [sequences, width] (rows may be
    further apart), ``lengths`` int32 [sequences], and for the calls that hand
    pages out or take them back ``refs`` int32 [pages]."""
    torch = _torch()
    if table.dim() != 2 or (table.stride(1) != 1 and table.shape[1] > 1):
        raise ValueError("the page table must be [sequences, width] with contiguous rows")
    if not table.is_cuda:
        raise ValueError("the page table must be a GPU tensor")
    for t, what, n in ((table, "page table", 0), (lengths, "lengths", table.shape[0]), (refs, "refs", 0)):
        _need(t, what, n, torch.int32)
    pool = Pool(table.data_ptr(), _dev_ptr(lengths, "lengths"), _dev_ptr(refs, "refs"),
                max(table.stride(0), table.shape[1]) if table.shape[0] == 1 else table.stride(0), table.shape[0],
                table.shape[1], 0 if refs is None else refs.numel(), int(page_size))
    pool._tensors = (table, lengths, refs)
    return pool


def _buffer(t, what: str, n: int, dtype) -> Optional[int]:
    """Device pointer of a contiguous tensor of at least n elements of ``dtype``, or None.
    One test for the usual case (0.4 us); what is wrong is found out behind it."""
    if t is None:
        return None
    if t.dtype is dtype and t.is_cuda and t.numel() >= n and t.is_contiguous():
        return t.data_ptr()
    _need(t, what, n, dtype)
    return _dev_ptr(t, what)


def _int32_list(t, what: str, n: int = 0) -> Optional[int]:
    """Device pointer of an int32 list (of n entries)."""
    return _buffer(t, what, n, _torch().int32)


def _floats(t, what: str, n: int) -> Optional[int]:
    """Device pointer of a float32 tensor of n elements at least, or None."""
    return _buffer(t, what, n, _torch().float32)


def _workspace(t):
    return (None, 0) if t is None else (_dev_ptr(t, "workspace"), t.numel() * t.element_size())


def _rows(t, what: str, shape, dtype):
    """(pointer, row stride, head stride) of a [rows, heads, dim] tensor whose rows and heads may be apart."""
    if t.dtype is not dtype:
        raise TypeError(f"{what} must have dtype {dtype}, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, {tuple(shape)} needed")
    st = t.stride()
    if st[2] != 1 and shape[2] > 1:
        raise ValueError(f"{what} must be contiguous in its last dimension")
    return t.data_ptr(), st[0], st[1]


def cpes_pages_workspace_bytes(pages: int) -> int:
    return int(load().cpes_pages_workspace_bytes(pages))


def cpes_pages_reserve(pool: Pool, seqs, new_lengths, workspace, status=None, stream=None) -> None:
    """Sequences seqs[i] grow to new_lengths[i] tokens (all or nothing; ``status``
    receives PAGES_OK, PAGES_SHORT or PAGES_BAD_SEQUENCE)."""
    n = seqs.numel()
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_pages_reserve(ctypes.byref(pool), n, _int32_list(seqs, "seqs"),
                                               _int32_list(new_lengths, "new_lengths", n), ws, size,
                                               _int32_list(status, "status", 1), _stream(stream)))


def cpes_pages_fork(cache: Cache, pool: Pool, parents, children, workspace, status=None, stream=None) -> None:
    """Empty sequences children[i] become copies of parents[i]: full pages are
    shared, a partly filled last page is copied in every layer."""
    n = children.numel()
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_pages_fork(ctypes.byref(cache), ctypes.byref(pool), n,
                                            _int32_list(parents, "parents", n), _int32_list(children, "children"), ws,
                                            size, _int32_list(status, "status", 1), _stream(stream)))


def cpes_pages_free(pool: Pool, seqs, status=None, stream=None) -> None:
    """Sequences seqs[i] give their pages up."""
    _check((_lib or load()).cpes_pages_free(ctypes.byref(pool), seqs.numel(), _int32_list(seqs, "seqs"),
                                            _int32_list(status, "status", 1), _stream(stream)))


def cpes_pages_copy(cache: Cache, src, dst, stream=None) -> None:
    """Page dst[i] of every layer becomes a copy of page src[i]."""
    n = dst.numel()
    _check((_lib or load()).cpes_pages_copy(ctypes.byref(cache), n, _int32_list(src, "src", n), _int32_list(dst, "dst"),
                                            _stream(stream)))


def cpes_pages_compact(cache: Cache, pool: Pool, packed: Pool, workspace, moved=None, stream=None) -> None:
    """The live pages move to the front of the cache; ``packed`` (``pool`` itself,
    or a pool of the same shape) receives table, lengths and reference counts."""
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_pages_compact(ctypes.byref(cache), ctypes.byref(pool), ctypes.byref(packed), ws, size,
                                               _int32_list(moved, "moved", 1), _stream(stream)))


def cpes_pages_keep_workspace_bytes(n: int, longest: int) -> int:
    return int(load().cpes_pages_keep_workspace_bytes(n, longest))


def _starts(t) -> int:
    """Rows of an int32 [rows + 1] list of where each row's tokens begin."""
    if t.numel() < 1:
        raise ValueError("starts must hold rows + 1 entries")
    return t.numel() - 1


def cpes_pages_keep(cache: Cache, pool: Pool, starts, kept, path, workspace, seqs=None, status=None, stream=None) -> None:
    """Of the drafted tokens starts[i] .. starts[i + 1] - 1 of sequences seqs[i] (None: i), the newest in the cache,
    the first kept[i] of path[i] ([n, longest], as cpes_tree_accept leaves them) stay and move together; the
    sequences' other pages are given back."""
    n = _starts(starts)
    if path.dim() != 2 or path.shape[0] != n:
        raise ValueError(f"path must be [{n}, longest]")
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_pages_keep(ctypes.byref(cache), ctypes.byref(pool), n, _int32_list(seqs, "seqs", n),
                                            _int32_list(starts, "starts"), path.shape[1], _int32_list(kept, "kept", n),
                                            _int32_list(path, "path"), ws, size, _int32_list(status, "status", 1),
                                            _stream(stream)))


def cpes_cache_append(cache: Cache, layer: int, pool: Pool, k_new, v_new, positions, seqs=None, stream=None) -> None:
    """Keys and values of new tokens ([tokens, heads, head_dim], rows may be apart)
    enter the pages of sequences seqs[i] (None: i) at positions[i]."""
    shape = (k_new.shape[0], cache.heads, cache.head_dim)
    k, row, head = _rows(k_new, "k_new", shape, cache._dtype)
    v, v_row, v_head = _rows(v_new, "v_new", shape, cache._dtype)
    if not _same_strides((row, head), (v_row, v_head), shape):
        raise ValueError("k_new and v_new must have the same strides")
    _check((_lib or load()).cpes_cache_append(ctypes.byref(cache), layer, ctypes.byref(pool), shape[0],
                                              _int32_list(seqs, "seqs", shape[0]),
                                              _int32_list(positions, "positions", shape[0]), k, v, row, head,
                                              _stream(stream)))


def cpes_attend_workspace_bytes(rows: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    return int(load().cpes_attend_workspace_bytes(rows, q_heads, kv_heads, head_dim))


def cpes_attend(cache: Cache, layer: int, pool: Pool, q, out, lse=None, seqs=None, scale: Optional[float] = None,
                window: int = 0, sinks: int = 0, workspace=None, stream=None) -> None:
    """Attention of the newest token of sequences seqs[r] (None: r) over the cache:
    q and out are [rows, q_heads, head_dim] (rows and heads may be apart), lse
    float32 [rows, q_heads]; scale defaults to head_dim ** -0.5."""
    shape, dtype = q.shape, cache._dtype
    if len(shape) != 3 or shape[2] != cache.head_dim:
        raise ValueError(f"q must be [rows, q_heads, {cache.head_dim}], not {tuple(shape)}")
    rows, heads, dim = shape
    qp, q_row, q_head = _rows(q, "q", shape, dtype)
    op, o_row, o_head = _rows(out, "out", shape, dtype)
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_attend(ctypes.byref(cache), layer, ctypes.byref(pool), rows,
                                        _int32_list(seqs, "seqs", rows), qp, q_row, q_head, heads,
                                        dim ** -0.5 if scale is None else scale, window, sinks, op, o_row,
                                        o_head, _floats(lse, "lse", rows * heads), ws, size, _stream(stream)))


def cpes_attend_tree_workspace_bytes(rows: int, tokens: int, longest: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    return int(load().cpes_attend_tree_workspace_bytes(rows, tokens, longest, q_heads, kv_heads, head_dim))


def cpes_attend_tree(cache: Cache, layer: int, pool: Pool, q, out, starts, longest: int, parents=None, lse=None, seqs=None,
                     scale: Optional[float] = None, window: int = 0, sinks: int = 0, workspace=None, stream=None) -> None:
    """Attention of the newest tokens of sequences seqs[r] (None: r) over the cache: tokens starts[r] .. starts[r + 1]
    - 1 (at most ``longest``) of q and out [tokens, q_heads, head_dim] (rows and heads may be apart) are a tree with
    ``parents`` (int32 [tokens], within the row; None: a chain).  lse is float32 [tokens, q_heads]; scale defaults to
    head_dim ** -0.5."""
    shape, dtype = q.shape, cache._dtype
    if len(shape) != 3 or shape[2] != cache.head_dim:
        raise ValueError(f"q must be [tokens, q_heads, {cache.head_dim}], not {tuple(shape)}")
    tokens, heads, dim = shape
    rows = _starts(starts)
    qp, q_row, q_head = _rows(q, "q", shape, dtype)
    op, o_row, o_head = _rows(out, "out", shape, dtype)
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_attend_tree(ctypes.byref(cache), layer, ctypes.byref(pool), rows,
                                             _int32_list(seqs, "seqs", rows), _int32_list(starts, "starts"), tokens, longest,
                                             _int32_list(parents, "parents", tokens), qp, q_row, q_head, heads,
                                             dim ** -0.5 if scale is None else scale, window, sinks, op, o_row, o_head,
                                             _floats(lse, "lse", tokens * heads), ws, size, _stream(stream)))


def cpes_tree_accept(starts, drafted, sampled, kept, path, next_tokens, parents=None, stream=None) -> None:
    """The walk down each row's tree along the sampled tokens: ``drafted`` and ``sampled`` int64 [tokens]; ``kept`` int32
    [rows], ``path`` int32 [rows, longest] and ``next_tokens`` int64 [rows] receive how many tokens stay, which, and
    the token behind them."""
    rows, tokens, int64 = _starts(starts), drafted.numel(), _torch().int64
    if path.dim() != 2 or path.shape[0] != rows:
        raise ValueError(f"path must be [{rows}, longest]")
    _check((_lib or load()).cpes_tree_accept(rows, _int32_list(starts, "starts"), tokens, path.shape[1],
                                             _int32_list(parents, "parents", tokens), _buffer(drafted, "drafted", 0, int64),
                                             _buffer(sampled, "sampled", tokens, int64), _int32_list(kept, "kept", rows),
                                             _int32_list(path, "path"), _buffer(next_tokens, "next_tokens", rows, int64),
                                             _stream(stream)))


def _logits(x, what: str = "logits"):
    """(pointer, rows, vocabulary, row stride) of a [rows, vocabulary] tensor whose rows may be apart."""
    shape, strides = x.shape, x.stride()
    if len(shape) != 2 or (strides[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what} must be [rows, vocabulary] with contiguous rows")
    if not x.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    rows, vocab = shape
    return x.data_ptr(), rows, vocab, strides[0] if rows > 1 else max(strides[0], vocab)


def cpes_logprobs_workspace_bytes(rows: int, vocab: int, top: int = 0) -> int:
    """Enough for any number of rows up to ``rows``: a batch keeps its workspace as its rows end."""
    return int(load().cpes_logprobs_workspace_bytes(rows, vocab, top))


def cpes_logprobs(logits, targets, logp, entropy=None, lse=None, stats=None, top_logp=None, top_ids=None,
                  scale: float = 1.0, workspace=None, stream=None) -> None:
    """Scores of tokens targets[r] (int64) under logits [rows, vocabulary] times
    ``scale``: float32 [rows] log probabilities, entropies and normalisers, the
    float32 [rows, 2] ``stats`` for cpes_logprobs_backward, and the most likely
    alternatives in float32 / int64 [rows, k] ``top_logp`` and ``top_ids``."""
    x, rows, vocab, stride = _logits(logits)
    int64 = _torch().int64
    top = 0
    if top_ids is not None or top_logp is not None:
        if top_ids is None or top_logp is None or top_ids.dim() != 2 or top_ids.shape[0] != rows or top_logp.shape != top_ids.shape:
            raise ValueError("top_logp and top_ids must both be [rows, k]")
        top = top_ids.shape[1]
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_logprobs(x, _dtype_code(logits, "logits"), rows, vocab, stride, scale,
                                          _buffer(targets, "targets", rows, int64), _floats(logp, "logp", rows),
                                          _floats(entropy, "entropy", rows), _floats(lse, "lse", rows),
                                          _floats(stats, "stats", 2 * rows), top, _floats(top_logp, "top_logp", rows * top),
                                          _buffer(top_ids, "top_ids", rows * top, int64), ws, size, _stream(stream)))


def cpes_logprobs_backward(logits, targets, stats, entropy, d_logp, d_entropy, d_logits, scale: float = 1.0,
                           stream=None) -> None:
    """d_logits (dtype of the logits, may be them) from the upstream gradients
    d_logp and d_entropy (float32 [rows], either may be None)."""
    x, rows, vocab, stride = _logits(logits)
    dx, d_rows, d_vocab, d_stride = _logits(d_logits, "d_logits")
    if (d_rows, d_vocab) != (rows, vocab) or d_logits.dtype != logits.dtype:
        raise ValueError("d_logits must have the shape and dtype of the logits")
    _check((_lib or load()).cpes_logprobs_backward(x, _dtype_code(logits, "logits"), rows, vocab, stride, scale,
                                                   _buffer(targets, "targets", rows, _torch().int64), _floats(stats, "stats", 2 * rows),
                                                   _floats(entropy, "entropy", rows), _floats(d_logp, "d_logp", rows),
                                                   _floats(d_entropy, "d_entropy", rows), dx, d_stride, _stream(stream)))


def cpes_sample_workspace_bytes(rows: int, vocab: int) -> int:
    """Enough for any number of rows up to ``rows``."""
    return int(load().cpes_sample_workspace_bytes(rows, vocab))


def cpes_sample(logits, uniforms, tokens, logp=None, scale: float = 1.0, top_k: int = 0, top_p: float = 1.0,
                min_p: float = 0.0, workspace=None, stream=None) -> None:
    """tokens[r] (int64) drawn from logits [rows, vocabulary] times ``scale`` by uniforms[r] (float32, in [0, 1)), among
    the ``top_k`` most likely (0: all), the fewest of them that hold ``top_p`` of their probability, and those with
    at least ``min_p`` of the largest one; logp float32 [rows], among these."""
    x, rows, vocab, stride = _logits(logits)
    ws, size = _workspace(workspace)
    _check((_lib or load()).cpes_sample(x, _dtype_code(logits, "logits"), rows, vocab, stride, scale, top_k, top_p, min_p,
                                        _floats(uniforms, "uniforms", rows), _buffer(tokens, "tokens", rows, _torch().int64),
                                        _floats(logp, "logp", rows), ws, size, _stream(stream)))


def cpes_debug_philox(seed: int, domain: int, q0: int, nblocks: int, out, stream=None) -> None:
    if out is not None and out.numel() * out.element_size() < 16 * nblocks:
        raise ValueError(f"out holds {out.numel() * out.element_size()} bytes, {16 * nblocks} needed")
    _check((_lib or load()).cpes_debug_philox(seed, domain, q0, nblocks, _dev_ptr(out, "out"), _stream(stream)))


def cpes_debug_normals(seed: int, j0: int, n: int, out, stream=None) -> None:
    _need(out, "out", n, _torch().float32)
    _check((_lib or load()).cpes_debug_normals(seed, j0, n, _dev_ptr(out, "out"), _stream(stream)))


def cpes_debug_bm_grid(m0: int, n: int, rho=None, cos=None, sin=None, stream=None) -> None:
    for t, what in ((rho, "rho"), (cos, "cos"), (sin, "sin")):
        _need(t, what, n, _torch().float64)
    _check((_lib or load()).cpes_debug_bm_grid(m0, n, _dev_ptr(rho, "rho"), _dev_ptr(cos, "cos"), _dev_ptr(sin, "sin"),
                                     _stream(stream)))


def cpes_debug_prp(seed: int, d: int, K: int, i0: int, n: int, perm=None, bucket=None, stream=None) -> None:
    _need(perm, "perm", n, _torch().int64)
    _need(bucket, "bucket", n, _torch().int32)
    _check((_lib or load()).cpes_debug_prp(seed, d, K, i0, n, _dev_ptr(perm, "perm"), _dev_ptr(bucket, "bucket"),
                                 _stream(stream)))


def cpes_rng_probe(seed: int, n: int, sink, stream=None) -> None:
    if sink is not None and sink.numel() * sink.element_size() < 4:
        raise ValueError("sink needs at least 4 bytes")
    _check((_lib or load()).cpes_rng_probe(seed, n, _dev_ptr(sink, "sink"), _stream(stream)))


def cpes_probe_map_copy(w, s: Subspace, buf, direction: int, stream=None) -> None:
    """Plain gather (direction 0: buf[j] = w[p(j)]) or scatter (1: w[p(j)] =
    buf[j]) through the subspace's element map: a measurement reference."""
    _need(buf, "buf", s.length, w.dtype)
    _check((_lib or load()).cpes_probe_map_copy(_dev_ptr(w, "w"), w.numel(), _dtype_code(w), ctypes.byref(s),
                                      _dev_ptr(buf, "buf"), direction, _stream(stream)))


def cpes_probe_copy(src, dst, nbytes: int, nontemporal: bool = False, stream=None) -> None:
    """dst[:nbytes] = src[:nbytes], one 16-byte vector per thread (non-temporal
    accesses if asked): a measurement reference."""
    for t, what in ((src, "src"), (dst, "dst")):
        if t.numel() * t.element_size() < nbytes:
            raise ValueError(f"{what} holds fewer than {nbytes} bytes")
    _check((_lib or load()).cpes_probe_copy(_dev_ptr(src, "src"), _dev_ptr(dst, "dst"), nbytes, int(bool(nontemporal)),
                                  _stream(stream)))


def cpes_abi_version() -> int:
    return int(load().cpes_abi_version())
