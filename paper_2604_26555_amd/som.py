"""Thin ctypes binding of libsom's C ABI: argument marshalling only, every step runs in the HIP kernels.

The functions keep the C names (som_bmu, som_accumulate, som_neighborhood_update, som_epoch, som_epoch_host)
and take torch tensors that live on the GPU; torch is used for device memory and streams, nothing else.
There is no CPU fallback: if the shared library is missing or no gfx950 device is present, loading or
``Som()`` raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SOM_LIB") or os.path.join(_HERE, "libsom.so")   # SOM_LIB: another build of the library

SOM_OK, SOM_EINVAL, SOM_ENOMEM, SOM_EHIP, SOM_EIO, SOM_ESTATE = 0, -1, -2, -3, -4, -5
SOM_KERNEL_GAUSSIAN = 0
SOM_SAFEGUARD_THRESHOLD = 0
SOM_SAFEGUARD_SHIFT = 1
SOM_SEARCH_AUTO = 0
SOM_SEARCH_FLOAT32 = 1
SOM_TOPOLOGY_MST = 1
SOM_TOPOLOGY_RNG = 2
SOM_ROWS_FLOAT, SOM_ROWS_BFLOAT, SOM_ROWS_HALF = 0, 1, 2
SOM_ACT_NONE, SOM_ACT_RELU, SOM_ACT_SILU, SOM_ACT_GELU, SOM_ACT_GELU_TANH = 0, 1, 2, 3, 4

EXPORTS = [
    "som_create", "som_destroy", "som_strerror", "som_last_error", "som_sync", "som_bmu", "som_accumulate",
    "som_neighborhood_update", "som_epoch", "som_epoch_host", "som_profile", "som_profile_read",
    "som_set_update_rule", "som_topology", "som_set_safeguard", "som_set_reproducible", "som_set_search",
    "som_matrix_pipe_probe", "som_matrix_pipe_probe_parts", "som_neighborhood_update_static", "som_epoch_file", "som_read_probe", "som_mfma_rate_probe",
    "som_group", "som_dispatch", "som_combine", "som_combine_grad", "som_node_product", "som_node_product_grad",
]


class SomStats(C.Structure):
    _fields_ = [
        ("sum_dist", C.c_double), ("sum_dist2", C.c_double), ("m", C.c_int64), ("n_recheck", C.c_int64),
        ("n_empty", C.c_int32), ("n_guarded", C.c_int32), ("ms_bmu_acc", C.c_float), ("ms_update", C.c_float),
        ("ms_h2d", C.c_float),
    ]


class SomError(RuntimeError):
    def __init__(self, code: int, what: str, detail: str):
        super().__init__(f"{what} failed: {detail} (code {code})")
        self.code = code


_lib = None


def load_library(path: str = LIB_PATH) -> C.CDLL:
    """Load libsom.so and declare the prototypes.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with `python -m paper_2604_26555_amd.build`")
    lib = C.CDLL(path)
    vp, i32, i64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_double
    lib.som_create.argtypes = [C.POINTER(vp), C.c_int, vp]
    lib.som_create.restype = C.c_int
    lib.som_destroy.argtypes = [vp]
    lib.som_destroy.restype = None
    lib.som_strerror.argtypes = [C.c_int]
    lib.som_strerror.restype = C.c_char_p
    lib.som_last_error.argtypes = [vp]
    lib.som_last_error.restype = C.c_char_p
    lib.som_sync.argtypes = [vp]
    lib.som_sync.restype = C.c_int
    lib.som_set_update_rule.argtypes = [vp, f64, f64, vp]
    lib.som_set_update_rule.restype = C.c_int
    lib.som_profile.argtypes = [vp, C.c_int]
    lib.som_profile.restype = C.c_int
    lib.som_profile_read.argtypes = [vp, C.POINTER(C.c_float), i32, C.POINTER(i32)]
    lib.som_profile_read.restype = C.c_int
    lib.som_bmu.argtypes = [vp, vp, i64, i32, i64, vp, i64, vp, i32, vp, vp, vp]
    lib.som_bmu.restype = C.c_int
    lib.som_accumulate.argtypes = [vp, vp, i64, i32, i64, vp, i64, vp, i32, vp, vp, C.c_int]
    lib.som_accumulate.restype = C.c_int
    lib.som_neighborhood_update.argtypes = [vp, vp, vp, vp, i32, i32, f64, C.c_int, f64, vp, vp]
    lib.som_neighborhood_update.restype = C.c_int
    lib.som_neighborhood_update_static.argtypes = [vp, vp, vp, vp, i32, i32, f64, C.c_int, f64, vp, vp]
    lib.som_neighborhood_update_static.restype = C.c_int
    lib.som_set_reproducible.argtypes = [vp, C.c_int]
    lib.som_set_reproducible.restype = C.c_int
    lib.som_set_search.argtypes = [vp, C.c_int]
    lib.som_set_search.restype = C.c_int
    lib.som_set_safeguard.argtypes = [vp, C.c_int]
    lib.som_set_safeguard.restype = C.c_int
    lib.som_topology.argtypes = [vp, vp, i32, i32, C.c_int, vp]
    lib.som_topology.restype = C.c_int
    lib.som_matrix_pipe_probe.argtypes = [vp, vp, vp, vp, vp, i64]
    lib.som_matrix_pipe_probe.restype = C.c_int
    lib.som_matrix_pipe_probe_parts.argtypes = [vp, C.c_int, vp, vp, vp, vp, i64]
    lib.som_matrix_pipe_probe_parts.restype = C.c_int
    lib.som_epoch.argtypes = [vp, vp, i64, i32, i64, vp, i64, vp, i32, vp, f64, C.c_int, f64, C.POINTER(SomStats)]
    lib.som_epoch.restype = C.c_int
    lib.som_epoch_host.argtypes = [vp, vp, i64, i32, i64, C.c_int, vp, i32, vp, f64, C.c_int, f64,
                                   C.POINTER(SomStats)]
    lib.som_epoch_host.restype = C.c_int
    lib.som_mfma_rate_probe.argtypes = [vp, C.c_int, C.c_int, C.c_int]
    lib.som_mfma_rate_probe.restype = C.c_int
    lib.som_read_probe.argtypes = [vp, vp, i64]
    lib.som_read_probe.restype = C.c_int
    lib.som_epoch_file.argtypes = [vp, C.c_int, i64, i64, i32, i64, vp, i32, vp, f64, C.c_int, f64, C.POINTER(SomStats)]
    lib.som_epoch_file.restype = C.c_int
    lib.som_group.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp]
    lib.som_group.restype = C.c_int
    lib.som_dispatch.argtypes = [vp, C.c_int, vp, i64, i32, i64, vp, i32, vp, vp, i64, i64]
    lib.som_dispatch.restype = C.c_int
    lib.som_combine.argtypes = [vp, C.c_int, vp, i64, i32, i64, vp, i64, i32, vp, vp, i64]
    lib.som_combine.restype = C.c_int
    lib.som_combine_grad.argtypes = [vp, C.c_int, vp, i64, i32, i64, vp, i64, i64, vp, i32, vp, vp, i64, vp]
    lib.som_combine_grad.restype = C.c_int
    lib.som_node_product.argtypes = [vp, C.c_int, vp, i64, i32, i64, vp, i32, vp, i32, vp, C.c_int, vp, i64, vp, i64, vp, i64]
    lib.som_node_product.restype = C.c_int
    lib.som_node_product_grad.argtypes = [vp, C.c_int, vp, i64, i32, i64, vp, i32, i64, vp, i32, vp, vp, i64, C.c_int, vp, i64, vp, vp]
    lib.som_node_product_grad.restype = C.c_int
    _lib = lib
    return lib


# same-width signed types are accepted for the unsigned arguments (row numbers below 2^31, counts below 2^63)
_ALIASES = {torch.uint32: (torch.uint32, torch.int32), torch.uint64: (torch.uint64, torch.int64)}


def _ptr(t: Optional[torch.Tensor], dtype: torch.dtype, name: str, device=None) -> Optional[int]:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype and t.dtype not in _ALIASES.get(dtype, ()):
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() == 1 and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} lives on {t.device}, the context is on {device}")
    return t.data_ptr()


def _matrix(t: torch.Tensor, name: str):
    # (each attribute of a tensor is read once: a small call's time is the host's, and this was 1.1 us of an epoch's 11)
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or stride[1] != 1 or (shape[0] > 1 and stride[0] < shape[1]):
        raise ValueError(f"{name} must be a row-major 2-D tensor")
    (rows, columns), ld = shape, stride[0]
    return rows, columns, ld if rows > 1 else max(columns, ld)


# address of the current stream: without making a Stream object (2 us) where torch has a way to
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)

_ROWS = {torch.float32: SOM_ROWS_FLOAT, torch.bfloat16: SOM_ROWS_BFLOAT, torch.float16: SOM_ROWS_HALF}
_ACTIVATIONS = {"none": SOM_ACT_NONE, "relu": SOM_ACT_RELU, "silu": SOM_ACT_SILU, "gelu": SOM_ACT_GELU, "gelu_tanh": SOM_ACT_GELU_TANH}


@dataclass
class EpochStats:
    sum_dist: float
    sum_dist2: float
    m: int
    n_recheck: int
    n_empty: int
    n_guarded: int
    ms_bmu_acc: float
    ms_update: float
    ms_h2d: float

    @property
    def qe(self) -> float:
        return self.sum_dist / self.m if self.m else 0.0


def _stats(s: SomStats) -> EpochStats:
    return EpochStats(s.sum_dist, s.sum_dist2, s.m, s.n_recheck, s.n_empty, s.n_guarded, s.ms_bmu_acc, s.ms_update,
                      s.ms_h2d)


class Som:
    """One libsom context bound to a GPU and to the torch stream that is current when it is created."""

    def __init__(self, device: int | str | torch.device = 0, stream: Optional[torch.cuda.Stream] = None):
        self.lib = load_library()
        dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        if dev.type != "cuda":
            raise ValueError("libsom runs on a GPU only")
        self.device = torch.device("cuda", dev.index or 0)
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: libsom has no CPU path")
        with torch.cuda.device(self.device):
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        handle = C.c_void_p()
        rc = self.lib.som_create(C.byref(handle), self.device.index, C.c_void_p(self.stream.cuda_stream))
        if rc != SOM_OK:
            raise SomError(rc, "som_create", self.lib.som_strerror(rc).decode())
        self._h = handle
        self._raw = self.stream.cuda_stream

    def close(self):
        if getattr(self, "_h", None):
            self.lib.som_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _check(self, rc: int, what: str):
        if rc != SOM_OK:
            detail = self.lib.som_last_error(self._h).decode() or self.lib.som_strerror(rc).decode()
            raise SomError(rc, what, detail)

    def som_sync(self):
        self._check(self.lib.som_sync(self._h), "som_sync")

    def som_set_update_rule(self, eta: float = 1.0, mu: float = 0.0, velocity=None):
        """Learning rate and momentum of every later update on this context; velocity is a K x D float32 GPU tensor."""
        if velocity is not None and not velocity.is_contiguous():
            raise ValueError("velocity must be contiguous")
        self._velocity = velocity                       # keep the caller's buffer alive while the library uses it
        self._check(self.lib.som_set_update_rule(self._h, float(eta), float(mu),
                                                 _ptr(velocity, torch.float32, "velocity", self.device)),
                    "som_set_update_rule")

    def som_profile(self, enable: bool):
        self._check(self.lib.som_profile(self._h, 1 if enable else 0), "som_profile")

    def som_profile_read(self, capacity: int = 4096):
        """Durations (ms) of the main BMU kernel launches recorded since the last read."""
        buf = (C.c_float * capacity)()
        count = C.c_int32(0)
        self._check(self.lib.som_profile_read(self._h, buf, capacity, C.byref(count)), "som_profile_read")
        return [buf[i] for i in range(min(capacity, count.value))]

    def som_mfma_rate_probe(self, fold_steps=0, waves_per_simd=2, iters=20000):
        """Enqueue a loop of 8 * iters bf16 MFMAs per wavefront on random operands (time it from outside)."""
        self._check(self.lib.som_mfma_rate_probe(self._h, int(fold_steps), int(waves_per_simd), int(iters)), "som_mfma_rate_probe")

    def som_read_probe(self, t):
        """One plain streaming read of tensor t's bytes on the context's stream (time it from outside)."""
        nbytes = t.numel() * t.element_size() // 16 * 16
        self._check(self.lib.som_read_probe(self._h, C.c_void_p(t.data_ptr()), nbytes), "som_read_probe")

    def som_matrix_pipe_probe(self, A, Bt, Cm, Dout=None):
        """One bf16 MFMA per problem: Dout = Cm + A @ Bt^T.  A, Bt: (n, 32, 16) bf16; Cm: (n, 32, 32) float32."""
        n = A.shape[0]
        if A.shape != (n, 32, 16) or Bt.shape != (n, 32, 16) or Cm.shape != (n, 32, 32) or not (
                A.is_contiguous() and Bt.is_contiguous() and Cm.is_contiguous()):
            raise ValueError("shapes: A, Bt (n, 32, 16) bf16, C (n, 32, 32) float32, all contiguous")
        if Dout is None:
            Dout = torch.empty_like(Cm)
        rc = self.lib.som_matrix_pipe_probe(self._h, _ptr(A, torch.bfloat16, "A", self.device),
                                            _ptr(Bt, torch.bfloat16, "Bt", self.device),
                                            _ptr(Cm, torch.float32, "C", self.device),
                                            _ptr(Dout, torch.float32, "Dout", self.device), n)
        self._check(rc, "som_matrix_pipe_probe")
        return Dout

    def som_matrix_pipe_probe_parts(self, kind, A, Bt, Cm):
        """One half-precision (kind 0: A, Bt (n, 32, 16)) or fp6 (kind 1: (n, 32, 64)) MFMA per problem: Cm + A @ Bt^T."""
        n, k = A.shape[0], 16 if kind == 0 else 64
        if A.shape != (n, 32, k) or Bt.shape != (n, 32, k) or Cm.shape != (n, 32, 32) or not (
                A.is_contiguous() and Bt.is_contiguous() and Cm.is_contiguous()):
            raise ValueError("shapes: A, Bt (n, 32, 16 or 64) float16, C (n, 32, 32) float32, all contiguous")
        Dout = torch.empty_like(Cm)
        rc = self.lib.som_matrix_pipe_probe_parts(self._h, kind, _ptr(A, torch.float16, "A", self.device),
                                                  _ptr(Bt, torch.float16, "Bt", self.device),
                                                  _ptr(Cm, torch.float32, "C", self.device),
                                                  _ptr(Dout, torch.float32, "Dout", self.device), n)
        self._check(rc, "som_matrix_pipe_probe_parts")
        return Dout

    # ------------------------------------------------------------------ stage 1
    def som_bmu(self, X, W, idx=None, bmu=None, d2=None, qe=None):
        """bmu[i] = best-matching unit of presented sample i; returns (bmu, d2, qe) tensors (those requested)."""
        N, D, ldx = _matrix(X, "X")
        K, Dw, _ = _matrix(W, "W")
        if Dw != D or not W.is_contiguous():
            raise ValueError("W must be a contiguous K x D tensor with X's D")
        m = N if idx is None else idx.numel()
        if bmu is None:
            bmu = torch.empty(m, dtype=torch.int32, device=self.device)
        rc = self.lib.som_bmu(self._h, _ptr(X, torch.float32, "X", self.device), N, D, ldx,
                              _ptr(idx, torch.uint32, "idx", self.device) if idx is not None else None, m,
                              _ptr(W, torch.float32, "W", self.device), K,
                              _ptr(bmu, torch.int32, "bmu", self.device), _ptr(d2, torch.float32, "d2", self.device),
                              _ptr(qe, torch.float64, "qe", self.device))
        self._check(rc, "som_bmu")
        return bmu, d2, qe

    # ------------------------------------------------------------------ stage 2
    def som_accumulate(self, X, bmu, K, S, n, idx=None, zero_first=True):
        N, D, ldx = _matrix(X, "X")
        m = N if idx is None else idx.numel()
        if bmu.numel() != m:
            raise ValueError("bmu must have one entry per presented sample")
        if S.shape != (K, D) or not S.is_contiguous() or n.numel() != K:
            raise ValueError("S must be K x D contiguous and n of length K")
        rc = self.lib.som_accumulate(self._h, _ptr(X, torch.float32, "X", self.device), N, D, ldx,
                                     _ptr(idx, torch.uint32, "idx", self.device) if idx is not None else None, m,
                                     _ptr(bmu, torch.int32, "bmu", self.device), K,
                                     _ptr(S, torch.float64, "S", self.device), _ptr(n, torch.uint64, "n", self.device),
                                     1 if zero_first else 0)
        self._check(rc, "som_accumulate")
        return S, n

    # ------------------------------------------------------------------ stage 3
    def som_neighborhood_update(self, S, n, G, sigma, W, eps_h=0.0, n_guarded=None, kernel=SOM_KERNEL_GAUSSIAN):
        K, D, _ = _matrix(W, "W")
        if not W.is_contiguous() or S.shape != (K, D) or not S.is_contiguous() or G.shape != (K, K) \
                or not G.is_contiguous() or n.numel() != K:
            raise ValueError("shapes: W K x D, S K x D, G K x K, n K (all contiguous)")
        rc = self.lib.som_neighborhood_update(self._h, _ptr(S, torch.float64, "S", self.device),
                                              _ptr(n, torch.uint64, "n", self.device),
                                              _ptr(G, torch.float32, "G", self.device), K, D, float(sigma), kernel,
                                              float(eps_h), _ptr(W, torch.float32, "W", self.device),
                                              _ptr(n_guarded, torch.int32, "n_guarded", self.device))
        self._check(rc, "som_neighborhood_update")
        return W

    def som_neighborhood_update_static(self, S, n, G, sigma, W, eps_h=0.0, n_guarded=None, kernel=SOM_KERNEL_GAUSSIAN):
        """som_neighborhood_update without any device allocation (fixed per-GPU workspace; K * (D + 1) <= 65536)."""
        K, D, _ = _matrix(W, "W")
        if not W.is_contiguous() or S.shape != (K, D) or not S.is_contiguous() or G.shape != (K, K) \
                or not G.is_contiguous() or n.numel() != K:
            raise ValueError("shapes: W K x D, S K x D, G K x K, n K (all contiguous)")
        rc = self.lib.som_neighborhood_update_static(self._h, _ptr(S, torch.float64, "S", self.device),
                                                     _ptr(n, torch.uint64, "n", self.device),
                                                     _ptr(G, torch.float32, "G", self.device), K, D, float(sigma), kernel,
                                                     float(eps_h), _ptr(W, torch.float32, "W", self.device),
                                                     _ptr(n_guarded, torch.int32, "n_guarded", self.device))
        self._check(rc, "som_neighborhood_update_static")
        return W

    def som_set_reproducible(self, on=True):
        self._check(self.lib.som_set_reproducible(self._h, 1 if on else 0), "som_set_reproducible")

    def som_set_search(self, mode):
        if isinstance(mode, str):
            mode = {"auto": SOM_SEARCH_AUTO, "float32": SOM_SEARCH_FLOAT32}[mode]
        self._check(self.lib.som_set_search(self._h, int(mode)), "som_set_search")

    def som_set_safeguard(self, mode):
        if isinstance(mode, str):
            mode = {"threshold": SOM_SAFEGUARD_THRESHOLD, "shift": SOM_SAFEGUARD_SHIFT}[mode]
        self._check(self.lib.som_set_safeguard(self._h, int(mode)), "som_set_safeguard")

    # ------------------------------------------------------------------ topology rebuild
    def som_topology(self, W, kind, G=None):
        K, D, _ = _matrix(W, "W")
        if not W.is_contiguous():
            raise ValueError("W must be contiguous")
        if isinstance(kind, str):
            kind = {"mst": SOM_TOPOLOGY_MST, "rng": SOM_TOPOLOGY_RNG}[kind]
        if G is None:
            G = torch.empty((K, K), dtype=torch.float32, device=W.device)
        elif G.shape != (K, K) or not G.is_contiguous():
            raise ValueError("G must be K x K contiguous")
        rc = self.lib.som_topology(self._h, _ptr(W, torch.float32, "W", self.device), K, D, int(kind),
                                   _ptr(G, torch.float32, "G", self.device))
        self._check(rc, "som_topology")
        return G

    # ------------------------------------------------------------------ local models: one matrix per node
    # (The calls read tensors as they are, also those that require a gradient: results carry no graph of torch's.  The way back is the
    # calls whose names end in _grad.)
    def _empty(self, shape, dtype):
        """A new tensor that this context's stream may write at once: its memory comes from that stream's pool."""
        if _raw_stream(self.device.index) == self._raw:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _zeros(self, shape, dtype):
        """The same, cleared: for outputs some of whose rows a call may leave as they were."""
        if _raw_stream(self.device.index) == self._raw:
            return torch.zeros(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.zeros(shape, dtype=dtype, device=self.device)

    def _rows(self, t, name, dtype=None, shape=None):
        """(address, rows, columns, leading dimension) of a matrix of a local model's rows."""
        if dtype is not None and t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if t.dtype not in _ROWS:
            raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
        if t.device != self.device:
            raise ValueError(f"{name} lives on {t.device}, the context is on {self.device}")
        rows, columns, ld = _matrix(t, name)
        if shape is not None and (rows, columns) != shape:
            raise ValueError(f"{name} must be {shape[0]} x {shape[1]}, got {rows} x {columns}")
        return t.data_ptr(), rows, columns, ld if rows > 1 else columns

    def _pairs(self, t, name, dtype):
        """(address, rows, nodes per row) of an array with an entry for each pair of row and node: (T,) or (T, k)."""
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if t.device != self.device:
            raise ValueError(f"{name} lives on {t.device}, the context is on {self.device}")
        if t.dim() not in (1, 2) or not t.is_contiguous() or (t.dim() == 2 and t.shape[1] < 1):
            raise ValueError(f"{name} must be a contiguous (T,) or (T, k) tensor")
        return t.data_ptr(), t.shape[0], t.shape[1] if t.dim() == 2 else 1

    def _weights(self, weight, slot):
        if weight is None:
            return None
        if weight.shape != slot.shape:
            raise ValueError("weight must have slot's shape")
        return self._pairs(weight, "weight", torch.float32)[0]

    def _nodes(self, X, A, offsets):
        """(K, Dout, Din, address of the offsets) of the nodes' matrices A: (K, Dout, Din), or (Dout, Din) without offsets."""
        shape = A.shape if A.dim() == 3 else (1, *A.shape)
        if len(shape) != 3 or not A.is_contiguous():
            raise ValueError("A must be a contiguous (K, Dout, Din) or, for one node, (Dout, Din) tensor")
        if A.dtype != X.dtype:
            raise TypeError(f"A must be {X.dtype}, got {A.dtype}")
        if A.device != self.device:
            raise ValueError(f"A lives on {A.device}, the context is on {self.device}")
        if offsets is None:
            if shape[0] != 1:
                raise ValueError("without offsets there is one node")
        elif offsets.numel() != shape[0] + 1 or offsets.dim() != 1:
            raise ValueError("offsets must have K + 1 entries")
        return (*shape, _ptr(offsets, torch.int32, "offsets", self.device))

    def _bias(self, t, name, A, K, Dout):
        if t.numel() != K * Dout or t.shape[-1] != Dout or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous K x Dout tensor")
        return _ptr(t, A.dtype, name, self.device)

    def som_group(self, node, K, offsets=None, order=None, slot=None):
        """Sorts the pairs of row and node by node, stably; node: int32 (T,) or (T, k), entries outside [0, K) have no place.
        Returns (offsets (K + 1), order (T k), slot (node's shape)): node e has places offsets[e] .. offsets[e + 1] - 1, order
        holds the pair t * k + j at each place, slot the place of each pair; -1 stands for none."""
        at, T, k = self._pairs(node, "node", torch.int32)
        if offsets is None:
            offsets = self._empty(int(K) + 1, torch.int32)
        elif offsets.numel() != int(K) + 1 or offsets.dim() != 1:
            raise ValueError("offsets must have K + 1 entries")
        if order is None:
            order = self._empty(T * k, torch.int32)
        elif order.numel() != T * k or order.dim() != 1:
            raise ValueError("order must have one entry per pair")
        if slot is None:
            slot = self._empty(node.shape, torch.int32)
        elif slot.shape != node.shape:
            raise ValueError("slot must have node's shape")
        rc = self.lib.som_group(self._h, at, T, k, int(K), _ptr(offsets, torch.int32, "offsets", self.device),
                                _ptr(order, torch.int32, "order", self.device), self._pairs(slot, "slot", torch.int32)[0])
        self._check(rc, "som_group")
        return offsets, order, slot

    def som_dispatch(self, X, slot, weight=None, out=None):
        """Rows to their places: out[slot[t, j]] = weight[t, j] * X[t] (without weights: X[t]).  out: T k rows unless given.
        Rows that are no pair's place are left as they were in a given out (which saves the clearing) and are zeros in a new one."""
        x, T, D, ldx = self._rows(X, "X")
        s, Ts, k = self._pairs(slot, "slot", torch.int32)
        if Ts != T:
            raise ValueError("slot must have one row per row of X")
        if out is None:
            out = self._zeros((T * k, D), X.dtype)
        y, M, Dy, ldy = self._rows(out, "out", X.dtype)
        if Dy != D:
            raise ValueError("out must have X's width")
        rc = self.lib.som_dispatch(self._h, _ROWS[X.dtype], x, T, D, ldx, s, k, self._weights(weight, slot), y, M, ldy)
        self._check(rc, "som_dispatch")
        return out

    def som_combine(self, Y, slot, weight=None, out=None):
        """Rows back: out[t] = sum_j weight[t, j] * Y[slot[t, j]]."""
        y, M, D, ldy = self._rows(Y, "Y")
        s, T, k = self._pairs(slot, "slot", torch.int32)
        if out is None:
            out = self._empty((T, D), Y.dtype)
        o, _, _, ldo = self._rows(out, "out", Y.dtype, (T, D))
        rc = self.lib.som_combine(self._h, _ROWS[Y.dtype], y, M, D, ldy, s, T, k, self._weights(weight, slot), o, ldo)
        self._check(rc, "som_combine")
        return out

    def som_combine_grad(self, dout, Y, slot, weight=None, dY=None, dweight=None):
        """Gradient of som_combine: (dY, dweight).  Either is left out, and returned as None, where False is given for it.
        Rows that are no pair's place are left as they were in a given dY and are zeros in a new one."""
        y, M, D, ldy = self._rows(Y, "Y")
        s, T, k = self._pairs(slot, "slot", torch.int32)
        g, _, _, lddo = self._rows(dout, "dout", Y.dtype, (T, D))
        dy = lddy = dw = None
        if dY is None:
            dY = self._zeros((M, D), Y.dtype)
        if dY is not False:
            dy, _, _, lddy = self._rows(dY, "dY", Y.dtype, (M, D))
        if dweight is None:
            dweight = self._empty(slot.shape, torch.float32)
        if dweight is not False:
            if dweight.shape != slot.shape:
                raise ValueError("dweight must have slot's shape")
            dw = self._pairs(dweight, "dweight", torch.float32)[0]
        rc = self.lib.som_combine_grad(self._h, _ROWS[Y.dtype], g, T, D, lddo, y, M, ldy, s, k, self._weights(weight, slot), dy, lddy or D, dw)
        self._check(rc, "som_combine_grad")
        return (dY if dY is not False else None), (dweight if dweight is not False else None)

    def som_node_product(self, X, A, offsets=None, bias=None, activation="none", residual=None, pre=None, out=None):
        """Every row times its node's matrix: out[s] = activation(A[e] X[s] + bias[e]) + residual[s] for the rows
        offsets[e] <= s < offsets[e + 1] of node e; without offsets A is one matrix for all rows.  pre, if given, receives the values
        before the activation.  activation: none, relu, silu, gelu or gelu_tanh.  Rows of no node are left as they were in a given out and
        are zeros in a new one."""
        x, M, Din, ldx = self._rows(X, "X")
        K, Dout, Da, off = self._nodes(X, A, offsets)
        if Da != Din:
            raise ValueError("A must have X's width")
        c = None if bias is None else self._bias(bias, "bias", A, K, Dout)
        r = ldr = z = ldz = None
        if residual is not None:
            r, _, _, ldr = self._rows(residual, "residual", X.dtype, (M, Dout))
        if pre is not None:
            z, _, _, ldz = self._rows(pre, "pre", X.dtype, (M, Dout))
        if out is None:
            out = (self._empty if offsets is None else self._zeros)((M, Dout), X.dtype)
        y, _, _, ldy = self._rows(out, "out", X.dtype, (M, Dout))
        rc = self.lib.som_node_product(self._h, _ROWS[X.dtype], x, M, Din, ldx, off, K, A.data_ptr(), Dout, c, _ACTIVATIONS[activation], r, ldr or Dout,
                                       z, ldz or Dout, y, ldy)
        self._check(rc, "som_node_product")
        return out

    def som_node_product_grad(self, dY, X, A, offsets=None, pre=None, activation="none", dX=None, dA=None, dbias=None):
        """Gradient of som_node_product: (dX, dA, dbias); pre as som_node_product filled it, needed where there is an activation.
        Each is left out, and returned as None, where False is given for it.  The residual's gradient is dY.
        With an activation and 16-bit rows, dX and dA are products of dz = dY activation'(pre) rounded to that type (float16: infinite
        from 65520 on); dbias sums it in float32.  Rows of no node are left as they were in a given dX and are zeros in a new one."""
        x, M, Din, ldx = self._rows(X, "X")
        K, Dout, Da, off = self._nodes(X, A, offsets)
        if Da != Din:
            raise ValueError("A must have X's width")
        g, _, _, lddy = self._rows(dY, "dY", X.dtype, (M, Dout))
        z = ldz = dx = lddx = da = dc = None
        if pre is not None:
            z, _, _, ldz = self._rows(pre, "pre", X.dtype, (M, Dout))
        if dX is None:
            dX = (self._empty if offsets is None else self._zeros)((M, Din), X.dtype)
        if dX is not False:
            dx, _, _, lddx = self._rows(dX, "dX", X.dtype, (M, Din))
        if dA is None:
            dA = self._empty(A.shape, X.dtype)
        if dA is not False:
            if dA.shape != A.shape or not dA.is_contiguous():
                raise ValueError("dA must be contiguous and have A's shape")
            da = _ptr(dA, X.dtype, "dA", self.device)
        if dbias is None:
            dbias = self._empty((*A.shape[:-2], Dout), X.dtype)
        if dbias is not False:
            dc = self._bias(dbias, "dbias", A, K, Dout)
        rc = self.lib.som_node_product_grad(self._h, _ROWS[X.dtype], g, M, Dout, lddy, x, Din, ldx, off, K, A.data_ptr(), z, ldz or Dout,
                                            _ACTIVATIONS[activation], dx, lddx or Din, da, dc)
        self._check(rc, "som_node_product_grad")
        return tuple(None if t is False else t for t in (dX, dA, dbias))

    # ------------------------------------------------------------------ whole epoch
    def som_epoch(self, X, W, G, sigma, idx=None, eps_h=0.0, want_stats=True, kernel=SOM_KERNEL_GAUSSIAN):
        N, D, ldx = _matrix(X, "X")
        K, Dw, _ = _matrix(W, "W")
        if Dw != D or not W.is_contiguous() or G.shape != (K, K) or not G.is_contiguous():
            raise ValueError("shapes: W K x D contiguous with X's D, G K x K contiguous")
        m = N if idx is None else idx.numel()
        st = SomStats() if want_stats else None
        rc = self.lib.som_epoch(self._h, _ptr(X, torch.float32, "X", self.device), N, D, ldx,
                                _ptr(idx, torch.uint32, "idx", self.device) if idx is not None else None, m,
                                _ptr(W, torch.float32, "W", self.device), K, _ptr(G, torch.float32, "G", self.device),
                                float(sigma), kernel, float(eps_h), C.byref(st) if want_stats else None)
        self._check(rc, "som_epoch")
        return _stats(st) if want_stats else None

    def som_epoch_host(self, Xhost, W, G, sigma, chunk_rows, eps_h=0.0, pinned=None, kernel=SOM_KERNEL_GAUSSIAN):
        """Xhost: CPU float32 tensor or numpy array (C order, N x D), e.g. backed by a memory-mapped file."""
        import numpy as np
        if isinstance(Xhost, torch.Tensor):
            if Xhost.device.type != "cpu" or Xhost.dtype != torch.float32 or not Xhost.is_contiguous() or Xhost.dim() != 2:
                raise ValueError("Xhost must be a contiguous CPU float32 matrix")
            N, D = Xhost.shape
            addr = Xhost.data_ptr()
            if pinned is None:
                pinned = Xhost.is_pinned()
        else:
            a = Xhost
            if not isinstance(a, np.ndarray) or a.dtype != np.float32 or a.ndim != 2 or not a.flags["C_CONTIGUOUS"]:
                raise ValueError("Xhost must be a C-contiguous float32 numpy matrix")
            N, D = a.shape
            addr = a.ctypes.data
            pinned = bool(pinned)
        K, Dw, _ = _matrix(W, "W")
        if Dw != D or not W.is_contiguous() or G.shape != (K, K) or not G.is_contiguous():
            raise ValueError("shapes: W K x D contiguous with X's D, G K x K contiguous")
        st = SomStats()
        rc = self.lib.som_epoch_host(self._h, C.c_void_p(addr), N, D, int(chunk_rows), 1 if pinned else 0,
                                     _ptr(W, torch.float32, "W", self.device), K,
                                     _ptr(G, torch.float32, "G", self.device), float(sigma), kernel, float(eps_h),
                                     C.byref(st))
        self._check(rc, "som_epoch_host")
        return _stats(st)

    def som_epoch_file(self, fd, offset, N, D, W, G, sigma, chunk_rows, eps_h=0.0, kernel=SOM_KERNEL_GAUSSIAN):
        """One epoch on the N x D float32 rows stored from byte ``offset`` of the open file descriptor ``fd``."""
        K, Dw, _ = _matrix(W, "W")
        if Dw != D or not W.is_contiguous() or G.shape != (K, K) or not G.is_contiguous():
            raise ValueError("shapes: W K x D contiguous with the file's D, G K x K contiguous")
        st = SomStats()
        rc = self.lib.som_epoch_file(self._h, int(fd), int(offset), int(N), int(D), int(chunk_rows),
                                     _ptr(W, torch.float32, "W", self.device), K,
                                     _ptr(G, torch.float32, "G", self.device), float(sigma), kernel, float(eps_h),
                                     C.byref(st))
        self._check(rc, "som_epoch_file")
        return _stats(st)
