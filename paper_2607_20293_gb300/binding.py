"""ctypes binding of the C ABI in include/evo.h (argument marshalling only).

Every computation happens in libevo.so.  torch is used for device memory and
streams: device arguments are torch CUDA tensors (their data pointers are
passed through), host lattices are numpy uint8 arrays.  load() raises if the
library has not been built; there is no other implementation to fall back to.
"""
from __future__ import annotations

import ctypes
import os
import weakref

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libevo.so")
LIB_PATH_DEBUG = os.path.join(HERE, "libevo_debug.so")

OK, ERR_ARG, ERR_SHAPE, ERR_SCHEDULE, ERR_CUDA, ERR_TIMEOUT, ERR_OOM, ERR_UNSUPPORTED, ERR_CORRUPT = range(9)
SAMPLERS = {"ddpm": 0, "ddim": 1}
DTYPES = {"fp32": 0, "bf16": 1}
EMPTY = {"zero": 0, "force": 1}

_FIELDS = ["n_layer", "n_emb", "n_head", "horizon", "action_dim", "n_obs", "obs_dim", "n_steps",
           "train_steps", "sampler", "dtype", "empty_cache", "cluster", "job_samples", "debug_sync", "wide_rows"]


class EvoConfig(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in _FIELDS]


class SearchConfig(ctypes.Structure):
    _fields_ = [("n_units", ctypes.c_int32), ("n_steps", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("block_wise", ctypes.c_int32), ("population", ctypes.c_int32), ("elites", ctypes.c_int32),
                ("generations", ctypes.c_int32), ("tournament", ctypes.c_int32), ("guided", ctypes.c_int32),
                ("gamma", ctypes.c_int32), ("eps", ctypes.c_float), ("pad_", ctypes.c_float),
                ("crossover_rate", ctypes.c_double), ("mutation_rate", ctypes.c_double),
                ("early_stop", ctypes.c_int32), ("pad2_", ctypes.c_int32), ("q_base", ctypes.c_double),
                ("delta_acc", ctypes.c_double), ("seed", ctypes.c_uint64)]


class MemoryView(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int32) for f in ("dtype", "format", "n_head", "n_kv_head", "head_dim", "page_tokens",
                                               "n_pages", "max_pages", "n_seq", "pad_")]
                + [(f, ctypes.c_void_p) for f in ("k_pages", "v_pages", "k_scales", "v_scales", "table", "lens",
                                                  "starts", "status")])


class SearchResult(ctypes.Structure):
    _fields_ = [("best_fitness", ctypes.c_double), ("generations", ctypes.c_int32), ("evaluations", ctypes.c_int32),
                ("formal_evaluations", ctypes.c_int32), ("memo_hits", ctypes.c_int32),
                ("stopped_early", ctypes.c_int32), ("pad_", ctypes.c_int32)]


FITNESS_FN = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p, ctypes.POINTER(ctypes.c_uint8), ctypes.c_int32,
                              ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_double))


class EvoError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        detail = ""
        if code == ERR_CUDA and _lib is not None:
            detail = f", CUDA error {_lib.evo_last_cuda_error()}"
        super().__init__(f"{what}: {status_string(code)} ({code}{detail})")


_lib = None
_lib_debug = None
# handles alive in this process (their guard bands can be checked after a test)
_live: "weakref.WeakSet[Evo]" = weakref.WeakSet()
# guard failures found when a handle was closed
guard_failures: list[str] = []


def load(debug: bool = False) -> ctypes.CDLL:
    """The library (debug=True: the build with device-side index checks)."""
    global _lib, _lib_debug
    if (_lib_debug if debug else _lib) is not None:
        return _lib_debug if debug else _lib
    path = LIB_PATH_DEBUG if debug else LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2607_20293_gb300.build.build("
                           f"{'debug=True' if debug else ''})")
    lib = ctypes.CDLL(path)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    cfgp = ctypes.POINTER(EvoConfig)
    memp = ctypes.POINTER(MemoryView)
    sig = {
        "evo_weight_count": (SZ, [cfgp]),
        "evo_create": (I32, [P, SZ, cfgp, I32, ctypes.POINTER(P)]),
        "evo_destroy": (I32, [P]),
        "evo_denoise": (I32, [P, P, P, P, I32, I32, P, P]),
        "evo_denoise_trace": (I32, [P, P, P, P, I32, I32, P, P, P]),
        "evo_denoise_noalloc": (I32, [P, P, P, P, I32, I32, P, P]),
        "evo_test_wait_timeout": (I32, [P, I32, ctypes.c_int64, P]),
        "evo_check_guards": (I32, [P]),
        "evo_test_gelu": (I32, [P, P, ctypes.c_int64, I32, P]),
        "evo_denoise_population": (I32, [P, P, P, P, I32, I32, I32, P, P, P]),
        "evo_flops": (I32, [P, P, I32, ctypes.POINTER(I64)]),
        "evo_flops_cfg": (I32, [cfgp, P, I32, ctypes.POINTER(I64)]),
        "evo_schedule_from_positions": (I32, [P, I32, I32, I32, P]),
        "evo_schedule_fixed_interval": (I32, [I32, I32, I32, P]),
        "evo_get_status": (I32, [P]),
        "evo_set_profile_events": (I32, [P, P, P]),
        "evo_get_launch_info": (I32, [P, ctypes.POINTER(I32), ctypes.POINTER(I32), ctypes.POINTER(I32),
                                      ctypes.POINTER(I32)]),
        "evo_get_last_call": (I32, [P, ctypes.POINTER(I32), ctypes.POINTER(I64)]),
        "evo_last_cuda_error": (I32, []),
        "evo_search": (I32, [ctypes.POINTER(SearchConfig), P, FITNESS_FN, FITNESS_FN, P, P, ctypes.POINTER(SearchResult)]),
        "evo_redundancy_scratch_bytes": (SZ, [I32, I32, I32, I32, I32]),
        "evo_redundancy_map": (I32, [P, I32, I32, I32, I32, I32, P, P, P]),
        "evo_guided_schedules": (I32, [P, I32, I32, I32, ctypes.c_float, I32, P, I32, P, P]),
        "evo_cache_write": (I32, [P, I32, P, I32, I32, I32, P, P, P, P, P]),
        "evo_cache_add": (I32, [P, P, P, I32, I32, I32, I32, P, P, P]),
        "evo_rotation_table": (I32, [I32, I32, ctypes.c_double, P]),
        "evo_memory_append": (I32, [memp, P, P, P, I64, I64, I64, I32, P, P, ctypes.c_float, P, I32, P, P, I64, P]),
        "evo_memory_scratch_bytes": (SZ, [memp, I32, I32, I32]),
        "evo_memory_attend": (I32, [memp, P, I64, I32, I32, I32, ctypes.c_float, I32, I32, P, I64, P, P]),
        "evo_status_string": (ctypes.c_char_p, [I32]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if debug:
        _lib_debug = lib
    else:
        _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().evo_status_string(code).decode()


def _check(code: int, what: str):
    if code != OK:
        raise EvoError(code, what)


def make_config(cfg: dict, cluster: int = 0, job_samples: int = 0, empty: str = "zero",
                debug_sync: bool = False, wide_rows: int = 0) -> EvoConfig:
    return EvoConfig(cfg["n_layer"], cfg["n_emb"], cfg["n_head"], cfg["horizon"], cfg["action_dim"],
                     cfg["n_obs"], cfg["obs_dim"], cfg["n_steps"], cfg["train_steps"],
                     SAMPLERS[cfg["sampler"]], DTYPES[cfg["dtype"]], EMPTY[empty], cluster, job_samples,
                     int(debug_sync), wide_rows)


def weight_names(cfg: dict) -> list[str]:
    names = ["obs_w", "obs_b", "cond_pos", "cm_w1", "cm_b1", "cm_w2", "cm_b2", "in_w", "in_b", "pos"]
    per = ["ln1_g", "ln1_b", "sa_wqkv", "sa_bqkv", "sa_wo", "sa_bo", "ln2_g", "ln2_b", "ca_wq", "ca_bq",
           "ca_wkv", "ca_bkv", "ca_wo", "ca_bo", "ln3_g", "ln3_b", "ff_w1", "ff_b1", "ff_w2", "ff_b2"]
    for l in range(cfg["n_layer"]):
        names += [f"l{l}.{n}" for n in per]
    return names + ["lnf_g", "lnf_b", "head_w", "head_b"]


def pack_blob(cfg: dict, weights: dict) -> np.ndarray:
    """Concatenate named float32 tensors in the blob order of evo_weight_count."""
    blob = np.concatenate([np.ascontiguousarray(weights[n], dtype=np.float32).ravel() for n in weight_names(cfg)])
    want = load().evo_weight_count(ctypes.byref(make_config(cfg)))
    if blob.size != want:
        raise ValueError(f"weight blob has {blob.size} floats, the library expects {want}")
    return blob


def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, np.ndarray):
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("arrays passed to the C ABI must be C-contiguous")
        return x.ctypes.data
    if not x.is_contiguous():
        raise ValueError("tensors passed to the C ABI must be contiguous")
    return x.data_ptr()


def _lattice(S):
    """numpy lattices are passed as host memory (C-contiguous uint8); torch uint8
    tensors on the GPU as device memory."""
    if isinstance(S, np.ndarray):
        S = np.ascontiguousarray(S, dtype=np.uint8)
    return S


def _stream(stream) -> int | None:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def flops_cfg(cfg: dict, S, empty: str = "zero") -> int:
    S = np.ascontiguousarray(S, dtype=np.uint8)
    out = ctypes.c_int64()
    c = make_config(cfg, empty=empty)
    _check(load().evo_flops_cfg(ctypes.byref(c), S.ctypes.data, S.shape[0], ctypes.byref(out)), "evo_flops")
    return out.value


def schedule_from_positions(positions, n_units: int, T: int) -> np.ndarray:
    bt = np.ascontiguousarray(np.asarray(positions, dtype=np.int16).reshape(-1, 2))
    out = np.zeros((n_units, T), dtype=np.uint8)
    _check(load().evo_schedule_from_positions(bt.ctypes.data if bt.size else None, bt.shape[0], n_units, T,
                                              out.ctypes.data), "evo_schedule_from_positions")
    return out


def schedule_fixed_interval(n_units: int, T: int, M: int) -> np.ndarray:
    """Fixed-interval baseline lattice [n_units][T]: every unit at t = floor(i T / M), i < M."""
    out = np.zeros((n_units, T), dtype=np.uint8)
    _check(load().evo_schedule_fixed_interval(n_units, T, M, out.ctypes.data), "evo_schedule_fixed_interval")
    return out


class Evo:
    """One evo_handle: packed weights, caches and workspace on the current GPU."""

    def __init__(self, cfg: dict, weights: dict, max_batch: int, cluster: int = 0, job_samples: int = 0,
                 empty: str = "zero", debug_sync: bool = False, wide_rows: int = 0, debug_lib: bool = False):
        lib = self._lib = load(debug_lib)
        self.cfg = dict(cfg)
        self._c = make_config(cfg, cluster, job_samples, empty, debug_sync, wide_rows)
        self._blob = pack_blob(cfg, weights)
        h = ctypes.c_void_p()
        _check(lib.evo_create(self._blob.ctypes.data, self._blob.size, ctypes.byref(self._c), max_batch,
                              ctypes.byref(h)), "evo_create")
        self._h = h
        self.max_batch = max_batch
        _live.add(self)

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            rc = self._lib.evo_check_guards(self._h)
            if rc != OK:
                guard_failures.append(f"handle {self.cfg.get('n_emb')}x{self.cfg.get('n_layer')}: "
                                      f"{status_string(rc)}")
            self._lib.evo_destroy(self._h)
            self._h = ctypes.c_void_p()
            _live.discard(self)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def launch_info(self) -> dict:
        v = [ctypes.c_int32() for _ in range(4)]
        _check(self._lib.evo_get_launch_info(self._h, *[ctypes.byref(x) for x in v]), "evo_get_launch_info")
        return dict(cluster=v[0].value, job_samples=v[1].value, max_clusters=v[2].value, smem_bytes=v[3].value)

    def last_call(self) -> dict:
        """path of the last call ("cluster" or "wide") and the kernels it launched"""
        path, k = ctypes.c_int32(), ctypes.c_int64()
        _check(self._lib.evo_get_last_call(self._h, ctypes.byref(path), ctypes.byref(k)), "evo_get_last_call")
        return dict(path="wide" if path.value == 1 else "cluster", kernels=k.value)

    def denoise(self, obs, noise, S, out=None, stream=None, trace=None):
        import torch
        N = obs.shape[0]
        if out is None:
            out = torch.empty((N, self.cfg["horizon"], self.cfg["action_dim"]), dtype=torch.float32,
                              device=obs.device)
        S = _lattice(S)
        if trace is None:
            rc = self._lib.evo_denoise(self._h, _ptr(obs), _ptr(noise), _ptr(S), S.shape[0], N, _ptr(out),
                                    _stream(stream))
        else:
            rc = self._lib.evo_denoise_trace(self._h, _ptr(obs), _ptr(noise), _ptr(S), S.shape[0], N, _ptr(out),
                                          _ptr(trace), _stream(stream))
        _check(rc, "evo_denoise")
        return out

    def denoise_noalloc(self, obs, noise, S, out, stream=None):
        """evo_denoise with its per-call scratch in the library's static device
        array (no device allocation); `out` must be provided."""
        S = _lattice(S)
        rc = self._lib.evo_denoise_noalloc(self._h, _ptr(obs), _ptr(noise), _ptr(S), S.shape[0], obs.shape[0],
                                        _ptr(out), _stream(stream))
        _check(rc, "evo_denoise_noalloc")
        return out

    def population(self, obs, noise, S_pop, out=None, dev=None, stream=None, want_actions=True):
        import torch
        N_obs = obs.shape[0]
        S_pop = _lattice(S_pop)
        P = S_pop.shape[0]
        if out is None and want_actions:
            out = torch.empty((P, N_obs, self.cfg["horizon"], self.cfg["action_dim"]), dtype=torch.float32,
                              device=obs.device)
        if dev is None:
            dev = torch.empty((P,), dtype=torch.float32, device=obs.device)
        rc = self._lib.evo_denoise_population(self._h, _ptr(obs), _ptr(noise), _ptr(S_pop), P, S_pop.shape[1], N_obs,
                                           _ptr(out), _ptr(dev), _stream(stream))
        _check(rc, "evo_denoise_population")
        return out, dev

    def flops(self, S) -> int:
        S = np.ascontiguousarray(S, dtype=np.uint8)
        out = ctypes.c_int64()
        _check(self._lib.evo_flops(self._h, S.ctypes.data, S.shape[0], ctypes.byref(out)), "evo_flops")
        return out.value

    def set_profile_events(self, start=None, stop=None):
        """Bracket every denoising-loop kernel launch with these torch.cuda.Events
        (they must have been recorded once, so that their CUDA events exist)."""
        sp = start.cuda_event if start is not None else None
        ep = stop.cuda_event if stop is not None else None
        _check(self._lib.evo_set_profile_events(self._h, sp, ep), "evo_set_profile_events")

    def status(self) -> int:
        return self._lib.evo_get_status(self._h)

    def check_guards(self) -> int:
        """evo_check_guards: OK, or ERR_CORRUPT if a kernel wrote past an activation buffer."""
        return self._lib.evo_check_guards(self._h)

    def test_wait_timeout(self, helper: int, limit: int, stream=None):
        """Run the bounded-wait helper of the loop kernel (0) or the tensor-core
        kernels (1) on a barrier nothing arrives at, so that it gives up."""
        _check(self._lib.evo_test_wait_timeout(self._h, helper, limit, _stream(stream)), "evo_test_wait_timeout")


METRICS = {"cosine": 0, "mse": 1, "l1": 2, "w1": 3}


def redundancy_map(trace, metric: str = "cosine", stream=None):
    """Eq. 6 map d [U][T] from a device trace [T][U][N][H][E] (evo_denoise_trace
    with the all-refresh lattice)."""
    import torch
    T, U, N = trace.shape[:3]
    n = int(np.prod(trace.shape[3:]))
    m = METRICS[metric]
    lib = load()
    nb = lib.evo_redundancy_scratch_bytes(T, U, N, n, m)
    if nb == 0:
        raise EvoError(ERR_SHAPE, "evo_redundancy_scratch_bytes")
    scratch = torch.empty(nb, dtype=torch.uint8, device=trace.device)
    d = torch.empty((U, T), dtype=torch.float32, device=trace.device)
    _check(lib.evo_redundancy_map(_ptr(trace), T, U, N, n, m, _ptr(d), _ptr(scratch), _stream(stream)),
           "evo_redundancy_map")
    return d


def test_gelu(x, packed: bool = False, stream=None):
    """evo_test_gelu: the feed-forward units' device GELU (scalar form, or the
    packed pair form of the GEMM epilogue) applied to a contiguous fp32 CUDA
    tensor (a new tensor of the same shape)."""
    import torch
    y = torch.empty_like(x)
    _check(load().evo_test_gelu(_ptr(x), _ptr(y), x.numel(), int(packed), _stream(stream)), "evo_test_gelu")
    return y


def guided_schedules(d, K: int, rnd, eps: float = 0.05, gamma: int = 2, stream=None):
    """P lattices [P][U][T] of K cells each by Eq. 7 from the device map d [U][T];
    rnd: device uint64 tensor [P][K] (torch has no uint64: pass int64 with the same bits)."""
    import torch
    U, T = d.shape
    P = rnd.shape[0]
    S = torch.empty((P, U, T), dtype=torch.uint8, device=d.device)
    _check(load().evo_guided_schedules(_ptr(d), U, T, K, float(eps), int(gamma), _ptr(rnd), P, _ptr(S),
                                       _stream(stream)), "evo_guided_schedules")
    return S


CACHE_FORMATS = {"fp32": 0, "bf16": 1, "e4m3": 2}
UNIT_GROUP = 32          # values of a unit's cache that share a scale


# The small calls below take as long as their checks: names of torch and of the library are looked
# up once, and every tensor is looked at once.
_torch = _F32 = _BF16 = _U8 = _I32 = _raw_stream = _current_device = None


def _load_torch():
    global _torch, _F32, _BF16, _U8, _I32, _raw_stream, _current_device
    import torch
    _F32, _BF16, _U8, _I32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _current_device = getattr(torch._C, "_cuda_getDevice", None)
    load()
    _torch = torch
    return torch


def _misfit(t, what: str, dtype, shape, index) -> ValueError:
    return ValueError(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device}, contiguous: {t.is_contiguous()}; expected a "
                      f"contiguous {dtype} {tuple(shape)} on device {index}")


def _need(t, what: str, dtype, shape, index):
    """Address of a contiguous tensor of this type and shape on this device, or ValueError."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise _misfit(t, what, dtype, shape, index)
    return t.data_ptr()


def _launch_stream(index: int, stream):
    """The stream's handle (None: the current one); the tensors' device has to be the current one,
    because the library launches there."""
    if index < 0 or index != _current_device():
        raise ValueError(f"tensors are on device {index}, the call runs on the current CUDA device")
    if stream is None:
        return _raw_stream(index)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _new(shape, dtype, device, stream):
    """A tensor from the pool of the stream that the call runs on: one of another stream's pool may
    still be in use there."""
    if stream is None:
        return _torch.empty(shape, dtype=dtype, device=device)
    with _torch.cuda.stream(_torch.cuda.ExternalStream(stream, device) if isinstance(stream, int) else stream):
        return _torch.empty(shape, dtype=dtype, device=device)


def cache_write(r, codes, scales, x=None, refresh=None, out=None, stream=None):
    """evo_cache_write: the residual r [N][H][E] (fp32 or bf16) to the unit's 8-bit
    cache (codes [N][H][E], scales [N][H][E/32], uint8) for the samples whose
    refresh [N] (uint8) is not zero, or all.  Returns y = x + r for those samples
    and x for the others (in `out`, which may be x), or None without x."""
    _torch or _load_torch()
    index, dtype, shape = r.get_device(), r.dtype, r.shape
    st = _launch_stream(index, stream)
    if dtype is not _F32 and dtype is not _BF16:
        raise _misfit(r, "r", "float32 or bfloat16", shape, index)
    N, H, E = shape
    xp = yp = None
    if x is not None:
        xp = _need(x, "x", _F32, shape, index)
        if out is None:
            out = _torch.empty_like(x) if stream is None else _new(shape, _F32, x.device, stream)
            yp = out.data_ptr()
        else:
            yp = _need(out, "out", _F32, shape, index)
    elif out is not None:
        raise ValueError("out without x")
    rc = _lib.evo_cache_write(_need(r, "r", dtype, shape, index), 0 if dtype is _F32 else 1,
                              None if refresh is None else _need(refresh, "refresh", _U8, (N,), index), N, H, E, xp, yp,
                              _need(codes, "codes", _U8, shape, index),
                              _need(scales, "scales", _U8, (N, H, E // UNIT_GROUP), index), st)
    if rc:
        _check(rc, "evo_cache_write")
    return out


def cache_add(codes, scales, x, reuse=None, out=None, stream=None):
    """evo_cache_add: x [N][H][E] (fp32) plus the cached values of a run of units
    (codes [U][N][H][E], scales [U][N][H][E/32]) where reuse [U][N] is not zero, or
    of all; in `out` (which may be x) or a new tensor."""
    _torch or _load_torch()
    index, shape = x.get_device(), x.shape
    st = _launch_stream(index, stream)
    N, H, E = shape
    U = codes.shape[0]
    xp = _need(x, "x", _F32, shape, index)
    if out is None:
        out = _torch.empty_like(x) if stream is None else _new(shape, _F32, x.device, stream)
        yp = out.data_ptr()
    else:
        yp = _need(out, "out", _F32, shape, index)
    rc = _lib.evo_cache_add(_need(codes, "codes", _U8, (U, N, H, E), index),
                            _need(scales, "scales", _U8, (U, N, H, E // UNIT_GROUP), index),
                            None if reuse is None else _need(reuse, "reuse", _U8, (U, N), index), U, N, H, E, xp, yp, st)
    if rc:
        _check(rc, "evo_cache_add")
    return out


def rotation_table(n_pos: int, head_dim: int, base: float = 10000.0) -> np.ndarray:
    """Cosines and sines [n_pos][head_dim] of positions 0 .. n_pos-1 (evo_rotation_table), float32 on the host."""
    out = np.empty((n_pos, head_dim), dtype=np.float32)
    _check(load().evo_rotation_table(n_pos, head_dim, float(base), out.ctypes.data), "evo_rotation_table")
    return out


class Memory:
    """A paged memory (evo_memory) over caller-owned CUDA tensors.

    k_pages, v_pages  [n_pages][n_kv_head][page_tokens][head_dim]: of `dtype`, or uint8
                      e4m3 codes with k_scales, v_scales [n_pages][n_kv_head][page_tokens]
    table [n_seq][max_pages], lens [n_seq], starts [n_seq + 1] or None (equal chunks),
    status [1] or None: int32.  The tensors are kept; their contents may change between calls.
    Calls report what they cannot read or place, and waits that ran out, in status; None: in
    a word of the memory's own.  status() reads it.
    """

    def __init__(self, k_pages, v_pages, table, lens, n_head: int, k_scales=None, v_scales=None, starts=None,
                 status=None, dtype: str = "bf16"):
        _torch or _load_torch()
        self.device, dev = k_pages.device, k_pages.get_device()
        self.index = dev
        e4m3 = k_pages.dtype.itemsize == 1
        self.dtype = _F32 if dtype == "fp32" else _BF16
        n_pages, n_kv, page, dim = k_pages.shape
        n_seq, cols = table.shape
        kind, shape, u8, i32 = _U8 if e4m3 else self.dtype, k_pages.shape, _U8, _I32
        if e4m3 != (k_scales is not None) or e4m3 != (v_scales is not None):
            raise ValueError("scales belong to pages of 8-bit codes")
        v = MemoryView(DTYPES[dtype], CACHE_FORMATS["e4m3" if e4m3 else dtype], n_head, n_kv, dim, page, n_pages, cols,
                       n_seq, 0)
        v.k_pages = _need(k_pages, "k_pages", kind, shape, dev)
        v.v_pages = _need(v_pages, "v_pages", kind, shape, dev)
        if e4m3:
            v.k_scales = _need(k_scales, "k_scales", u8, shape[:3], dev)
            v.v_scales = _need(v_scales, "v_scales", u8, shape[:3], dev)
        v.table = _need(table, "table", i32, (n_seq, cols), dev)
        v.lens = _need(lens, "lens", i32, (n_seq,), dev)
        v.starts = None if starts is None else _need(starts, "starts", i32, (n_seq + 1,), dev)
        if status is None:
            status = _torch.zeros(1, dtype=i32, device=self.device)
        v.status = _need(status, "status", i32, (1,), dev)
        self.view, self._ref = v, ctypes.byref(v)
        self.n_head, self.n_kv_head, self.head_dim, self.n_seq = n_head, n_kv, dim, n_seq
        self.max_len = cols * page
        self.uniform = starts is None
        self._scratch = {}                          # bytes of scratch by (rows, max_new, max_len)
        self.tensors = (k_pages, v_pages, table, lens, k_scales, v_scales, starts, status)

    def status(self) -> int:
        """What calls have reported since it was last read: OK, ERR_CORRUPT (an entry, length, start or
        position out of its bounds) or ERR_TIMEOUT.  Waits for the device's work, and clears it."""
        if self.device.type == "cuda":
            _torch.cuda.synchronize(self.device)
        code = int(self.tensors[-1])
        if code:
            with _torch.inference_mode():           # the word may have been made under it
                self.tensors[-1].zero_()
        return code

    def _rows(self, t, what: str, rows: int, heads: int):
        """(address, elements between rows) of [rows][heads][head_dim], heads of a row contiguous."""
        dim = self.head_dim
        ld, between, within = t.stride() if t.dim() == 3 else (0, 0, 0)
        if (t.dtype is not self.dtype or t.get_device() != self.index or t.shape != (rows, heads, dim) or within != 1
                or (between != dim and heads > 1)):
            raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}; expected {self.dtype} "
                             f"({rows}, {heads}, {dim}) on {self.device}, the heads of a row contiguous")
        return t.data_ptr(), ld if rows > 1 else heads * dim

    def _like(self, q, ldq: int, rows: int, stream):
        """A contiguous tensor for q's rows, its address and the elements between its rows."""
        row = self.n_head * self.head_dim
        if stream is None and ldq == row:
            out = _torch.empty_like(q)
        else:
            out = _new((rows, self.n_head, self.head_dim), self.dtype, self.device, stream)
        return out, out.data_ptr(), row

    def append(self, q, k, v, q_gain=None, k_gain=None, eps: float = 1e-6, rotation=None, pos0=None, out=None,
               max_new=None, stream=None):
        """evo_memory_append: keys and values [rows][n_kv_head][head_dim] to their pages, and the
        normed and rotated queries [rows][n_head][head_dim] (in `out`, which may be q, or a new
        tensor).  q may be None (returns None), or k and v.  max_new is not needed here."""
        index, dim = self.index, self.head_dim
        st = _launch_stream(index, stream)
        if q is None and k is None:
            raise ValueError("neither queries nor keys")
        if (k is None) != (v is None):
            raise ValueError("keys and values come together")
        rows = (k if q is None else q).shape[0]
        qp = kp = vp = op = gq = gk = rot = at0 = None
        ldq = ldk = ldv = ldo = n_pos = 0
        if q is not None:
            heads = self.n_head
            qp, ldq = self._rows(q, "q", rows, heads)
            if out is None:
                out, op, ldo = self._like(q, ldq, rows, stream)
            else:
                op, ldo = self._rows(out, "out", rows, heads)
        if k is not None:
            kp, ldk = self._rows(k, "k", rows, self.n_kv_head)
            vp, ldv = self._rows(v, "v", rows, self.n_kv_head)
        if q_gain is not None:
            gq = _need(q_gain, "q_gain", _F32, (dim,), index)
        if k_gain is not None:
            gk = _need(k_gain, "k_gain", _F32, (dim,), index)
        if rotation is not None:
            n_pos = rotation.shape[0]
            rot = _need(rotation, "rotation", _F32, (n_pos, dim), index)
        if pos0 is not None:
            at0 = _need(pos0, "pos0", _I32, (self.n_seq,), index)
        rc = _lib.evo_memory_append(self._ref, qp, kp, vp, ldq, ldk, ldv, rows, gq, gk, eps, rot, n_pos, at0, op, ldo, st)
        if rc:
            _check(rc, "evo_memory_append")
        return out if q is not None else None

    def attend(self, q, scale=None, causal: bool = True, window: int = 0, max_new=None, max_len=None, out=None,
               stream=None):
        """evo_memory_attend: attention of q [rows][n_head][head_dim] over the memories, in `out` or
        a new tensor (rows of no sequence are left as they are: unset in a new tensor).  scale
        None: head_dim ** -0.5.  max_new, max_len: bounds on the chunks and memories (None: the
        rows, or their equal share, and what the table can hold)."""
        heads, dim = self.n_head, self.head_dim
        st = _launch_stream(self.index, stream)
        rows = q.shape[0]
        qp, ldq = self._rows(q, "q", rows, heads)
        if out is None:
            out, op, ldo = self._like(q, ldq, rows, stream)
        else:
            op, ldo = self._rows(out, "out", rows, heads)
        if rows == 0:
            return out
        if max_new is None:
            max_new = rows // max(1, self.n_seq) if self.uniform else rows
        if max_len is None:
            max_len = self.max_len
        if (window | max_new | max_len) >> 31:      # the library's numbers have 32 bits: the nearest that it takes or refuses
            window, max_new, max_len = (max(-1, min(int(x), 2 ** 31 - 1)) for x in (window, max_new, max_len))
        nb = self._scratch.get((rows, max_new, max_len))
        if nb is None:
            if len(self._scratch) >= 1024:          # max_len may grow with every token
                self._scratch.clear()
            nb = self._scratch[rows, max_new, max_len] = _lib.evo_memory_scratch_bytes(self._ref, rows, max_new, max_len)
        sp = None
        if nb:
            scratch = _new(nb, _U8, self.device, stream)   # back in that pool once this returns, for later work of the stream
            sp = scratch.data_ptr()
        rc = _lib.evo_memory_attend(self._ref, qp, ldq, rows, max_new, max_len, dim ** -0.5 if scale is None else scale,
                                    causal, window, op, ldo, sp, st)
        if rc:
            _check(rc, "evo_memory_attend")
        return out


def search(n_units: int, n_steps: int, budget: int, quick, formal=None, d_map=None, block_wise: bool = False,
           population: int = 30, elites: int = 10, generations: int = 30, tournament: int = 3, guided: int = 0,
           crossover_rate: float = 0.9, mutation_rate: float = 0.02, eps: float = 0.05, gamma: int = 2,
           early_stop: bool = False, q_base: float = 0.0, delta_acc: float = 0.0, seed: int = 0):
    """evo_search with Python fitness callables: f(S [P][n_units][T] uint8) -> [P] floats.
    Returns (best lattice, best fitness, stats dict)."""
    cfg = SearchConfig(n_units, n_steps, budget, int(block_wise), population, elites, generations, tournament,
                       guided, gamma, eps, 0.0, crossover_rate, mutation_rate, int(early_stop), 0, q_base,
                       delta_acc, seed & ((1 << 64) - 1))
    errors = []

    def wrap(f):
        if f is None:
            return ctypes.cast(None, FITNESS_FN)

        def cb(user, S, P, U, T, out):
            try:
                arr = np.ctypeslib.as_array(S, shape=(P, U, T)).copy()
                vals = f(arr)
                for i in range(P):
                    out[i] = float(vals[i])
                return 0
            except Exception as e:          # reported after the call returns
                errors.append(e)
                return 1
        return FITNESS_FN(cb)

    qf, ff = wrap(quick), wrap(formal)
    dm = None if d_map is None else np.ascontiguousarray(d_map, dtype=np.float32)
    best = np.zeros((n_units, n_steps), dtype=np.uint8)
    res = SearchResult()
    rc = load().evo_search(ctypes.byref(cfg), None if dm is None else dm.ctypes.data, qf, ff, None,
                           best.ctypes.data, ctypes.byref(res))
    if errors:
        raise errors[0]
    _check(rc, "evo_search")
    stats = dict(generations=res.generations, evaluations=res.evaluations,
                 formal_evaluations=res.formal_evaluations, memo_hits=res.memo_hits,
                 stopped_early=res.stopped_early)
    return best, res.best_fitness, stats
