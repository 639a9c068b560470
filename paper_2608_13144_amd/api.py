"""Torch-facing binding of the certified cache library.

PyTorch provides device memory and the current HIP stream; every step of the
path runs in the HIP kernels behind ``liblipcache.so``.  The functions mirror
the C ABI names (``lipcache_spectral_norm`` -> ``spectral_norm`` ...).
"""
from __future__ import annotations

import ctypes
import functools
import inspect
from dataclasses import dataclass

import torch

from . import _lib as L

_STORE = {"f32": L.F32, "bf16": L.BF16}
_PRECISION = {"f32": L.F32, "f16": L.F16}
_RADIUS = {"conservative": L.RADIUS_CONSERVATIVE, "tight": L.RADIUS_TIGHT}
_SELECT = {"radius_dedup": L.SELECT_RADIUS_DEDUP, "priority": L.SELECT_PRIORITY, "kcenter": L.SELECT_KCENTER}
_BOUNDARY = {"scaled": L.BOUNDARY_SCALED, "global": L.BOUNDARY_GLOBAL, "interclass": L.BOUNDARY_INTERCLASS}


def _p(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device: torch.device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _need_cuda(t: torch.Tensor, name: str, dtype: torch.dtype, ndim: int | None = None) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions")


def workspace(nbytes: int, device: torch.device) -> torch.Tensor:
    """Scratch buffer from torch's allocator (block starts are 512-byte aligned)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


@dataclass
class SpectralNorm:
    sigma: float
    iterations: int
    converged: bool


def spectral_norm(W: torch.Tensor, max_iters: int = 20000, rel_tol: float = 1e-13) -> SpectralNorm:
    """lipcache_spectral_norm: sigma_max(W) by float64 power iteration (sync)."""
    _need_cuda(W, "W", torch.float32, 2)
    lib = L.load()
    C, d = W.shape
    ws = workspace(lib.lipcache_spectral_norm_workspace_bytes(C, d), W.device)
    sigma = ctypes.c_double(0.0)
    iters = ctypes.c_int32(0)
    st = lib.lipcache_spectral_norm(_p(W), C, d, int(max_iters), float(rel_tol), ctypes.byref(sigma),
                                    ctypes.byref(iters), _p(ws), ws.numel(), _stream(W.device))
    L.check("lipcache_spectral_norm", st, allow=(L.OK, L.ENOCONV))
    return SpectralNorm(sigma.value, iters.value, st == L.OK)


@dataclass
class Certified:
    label: torch.Tensor          # int32 [N]
    r: torch.Tensor              # float32 [N]
    margin: torch.Tensor | None  # float32 [N]
    norm2: torch.Tensor | None   # float32 [N]


def certify(z: torch.Tensor, W: torch.Tensor, b: torch.Tensor | None, sigma: float, store: str = "f32",
            radius_mode: str = "conservative", want_margin: bool = False,
            want_norm2: bool = False) -> Certified:
    """lipcache_certify: labels, margins and certified radii of the rows of z (async)."""
    _need_cuda(z, "z", torch.float32, 2)
    _need_cuda(W, "W", torch.float32, 2)
    if b is not None:
        _need_cuda(b, "b", torch.float32, 1)
    lib = L.load()
    N, d = z.shape
    C = W.shape[0]
    dev = z.device
    label = torch.empty(N, dtype=torch.int32, device=dev)
    r = torch.empty(N, dtype=torch.float32, device=dev)
    margin = torch.empty(N, dtype=torch.float32, device=dev) if want_margin else None
    norm2 = torch.empty(N, dtype=torch.float32, device=dev) if want_norm2 else None
    mode = _RADIUS[radius_mode]
    ws = workspace(lib.lipcache_certify_workspace_bytes(C, d, mode), dev)
    st = lib.lipcache_certify(_p(z), N, d, _p(W), _p(b), C, float(sigma), mode, _STORE[store], _p(label),
                              _p(r), _p(margin), _p(norm2), _p(ws), ws.numel(), _stream(dev))
    L.check("lipcache_certify", st)
    return Certified(label, r, margin, norm2)


@dataclass
class LookupResult:
    label: torch.Tensor           # int32 [B], MISS on a miss
    index: torch.Tensor | None    # int64 [B], -1 on a miss
    dist2: torch.Tensor | None    # float32 [B], +inf on a miss
    stats: torch.Tensor           # int64 [4]: hits, re-checked pairs, band pairs, band queries
    band: torch.Tensor | None     # uint8 [B]


class LipCache:
    """The feature cache C = {(z_i, y~_i, r_i)} in device memory (caller-owned tensors)."""

    def __init__(self, d: int, capacity: int, store: str = "f32", device: str | torch.device = "cuda",
                 image: bool = True):
        """``image``: also keep the float16 image of the stored features that
        the f16 filter streams (costs 2 bytes per element; without it the f16
        lookup converts the rows on the fly)."""
        self.d = int(d)
        self.capacity = int(capacity)
        self.store = store
        self.device = torch.device(device)
        zdt = torch.float32 if store == "f32" else torch.bfloat16
        self.z = torch.empty((self.capacity, self.d), dtype=zdt, device=self.device)
        self.zimg = (torch.empty((self.capacity, self.d), dtype=torch.float16, device=self.device)
                     if image else None)
        self.r = torch.empty(self.capacity, dtype=torch.float32, device=self.device)
        self.label = torch.empty(self.capacity, dtype=torch.int32, device=self.device)
        self.norm2 = torch.empty(self.capacity, dtype=torch.float32, device=self.device)
        self.n = 0
        self._ws = None

    def cstruct(self) -> L.LipcacheCache:
        return L.LipcacheCache(self.z.data_ptr(), None if self.zimg is None else self.zimg.data_ptr(),
                               self.r.data_ptr(), self.label.data_ptr(), self.norm2.data_ptr(), self.n,
                               self.capacity, self.d, _STORE[self.store])

    def _workspace(self, nbytes: int) -> torch.Tensor:
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = workspace(nbytes, self.device)
        return self._ws

    def insert(self, z_src: torch.Tensor, label_src: torch.Tensor, r_src: torch.Tensor,
               miss_selector: torch.Tensor | None = None) -> int:
        """lipcache_insert: append selected rows (ascending), all-or-nothing (sync)."""
        _need_cuda(z_src, "z_src", torch.float32, 2)
        _need_cuda(label_src, "label_src", torch.int32, 1)
        _need_cuda(r_src, "r_src", torch.float32, 1)
        if miss_selector is not None:
            _need_cuda(miss_selector, "miss_selector", torch.int32, 1)
        lib = L.load()
        k = z_src.shape[0]
        if z_src.shape[1] != self.d or label_src.shape[0] != k or r_src.shape[0] != k:
            raise ValueError("insert: shapes do not match the cache")
        if miss_selector is not None and miss_selector.shape[0] != k:
            raise ValueError("insert: selector length")
        ws = self._workspace(lib.lipcache_insert_workspace_bytes(k))
        cs = self.cstruct()
        got = ctypes.c_int64(0)
        st = lib.lipcache_insert(ctypes.byref(cs), _p(z_src), _p(label_src), _p(r_src), _p(miss_selector), k,
                                 ctypes.byref(got), _p(ws), ws.numel(), _stream(self.device))
        L.check("lipcache_insert", st)
        self.n = int(cs.n)
        return int(got.value)

    def lookup(self, zq: torch.Tensor, precision: str = "f16", want_index: bool = True,
               want_dist2: bool = True, want_band: bool = True, out: LookupResult | None = None,
               prune: bool = False) -> LookupResult:
        """lipcache_lookup: nearest certified hit per query, or MISS (async).
        ``prune``: LIPCACHE_LOOKUP_PRUNE (prefix pruning; same answers; large
        lookups take it by themselves)."""
        _need_cuda(zq, "zq", torch.float32, 2)
        if zq.shape[1] != self.d:
            raise ValueError("lookup: query width differs from the cache's d")
        lib = L.load()
        B = zq.shape[0]
        dev = self.device
        if out is None:
            out = LookupResult(
                torch.empty(B, dtype=torch.int32, device=dev),
                torch.empty(B, dtype=torch.int64, device=dev) if want_index else None,
                torch.empty(B, dtype=torch.float32, device=dev) if want_dist2 else None,
                torch.zeros(4, dtype=torch.int64, device=dev),
                torch.empty(B, dtype=torch.uint8, device=dev) if want_band else None)
        prec = _PRECISION[precision] | (L.LOOKUP_PRUNE if prune else 0)
        # a large lookup takes the prefix scan whenever the workspace holds it
        ws = self._workspace(lib.lipcache_lookup_workspace_bytes(B, self.n, self.d, prec | L.LOOKUP_PRUNE))
        cs = self.cstruct()
        st = lib.lipcache_lookup(ctypes.byref(cs), _p(zq), B, prec, _p(out.label), _p(out.index), _p(out.dist2),
                                 _p(out.stats), _p(out.band), _p(ws), ws.numel(), _stream(dev))
        L.check("lipcache_lookup", st)
        return out

    def lookup_prunes(self, precision: str = "f16") -> bool:
        """lipcache_lookup_prunes: whether ``prune=True`` applies to this cache
        (else it changes nothing)."""
        cs = self.cstruct()
        return bool(L.load().lipcache_lookup_prunes(ctypes.byref(cs), _PRECISION[precision] | L.LOOKUP_PRUNE))

    def lookup_noalloc(self, zq: torch.Tensor, precision: str = "f16",
                       out: LookupResult | None = None, prune: bool = False) -> LookupResult:
        """lipcache_lookup_noalloc: lookup on the library's static per-GPU
        workspace (no device allocation in the library; async)."""
        _need_cuda(zq, "zq", torch.float32, 2)
        if zq.shape[1] != self.d:
            raise ValueError("lookup_noalloc: query width differs from the cache's d")
        lib = L.load()
        B = zq.shape[0]
        dev = self.device
        if out is None:
            out = LookupResult(torch.empty(B, dtype=torch.int32, device=dev),
                               torch.empty(B, dtype=torch.int64, device=dev),
                               torch.empty(B, dtype=torch.float32, device=dev),
                               torch.zeros(4, dtype=torch.int64, device=dev),
                               torch.empty(B, dtype=torch.uint8, device=dev))
        cs = self.cstruct()
        prec = _PRECISION[precision] | (L.LOOKUP_PRUNE if prune else 0)
        st = lib.lipcache_lookup_noalloc(ctypes.byref(cs), _p(zq), B, prec, _p(out.label),
                                         _p(out.index), _p(out.dist2), _p(out.stats), _p(out.band), _stream(dev))
        L.check("lipcache_lookup_noalloc", st)
        return out

    def serve(self, zq: torch.Tensor, W: torch.Tensor, b: torch.Tensor | None, sigma: float,
              precision: str = "f16", out: LookupResult | None = None):
        """One round of certified serving (Alg. 2): look every query up, certify
        every query with the head (the label and radius a miss is cached with;
        for a bfloat16 store the rounded query is certified), and write the
        misses back.  Returns (lookup result, certified queries, rows appended).
        """
        res = self.lookup(zq, precision=precision, out=out)
        cq = certify(zq, W, b, sigma, store=self.store)
        inserted = self.insert(zq, cq.label, cq.r, res.label)
        return res, cq, inserted

    def construct(self, z: torch.Tensor, label: torch.Tensor, r: torch.Tensor, strategy: str = "radius_dedup",
                  budget: int = -1, per_class: int = 0, n_classes: int = 0, priority: torch.Tensor | None = None,
                  guard_label: torch.Tensor | None = None):
        """lipcache_construct: select candidates (Alg. 1) and append them (sync).

        Returns (rows appended, int64 tensor of the selected candidate indices
        in append order)."""
        _need_cuda(z, "z", torch.float32, 2)
        _need_cuda(label, "label", torch.int32, 1)
        _need_cuda(r, "r", torch.float32, 1)
        if priority is not None:
            _need_cuda(priority, "priority", torch.float32, 1)
        if guard_label is not None:
            _need_cuda(guard_label, "guard_label", torch.int32, 1)
        n = z.shape[0]
        if z.shape[1] != self.d or label.shape[0] != n or r.shape[0] != n:
            raise ValueError("construct: shapes do not match the cache")
        lib = L.load()
        strat = _SELECT[strategy]
        cs = self.cstruct()
        bud = self.capacity - self.n if budget < 0 else int(budget)
        sel = torch.full((max(bud, 1),), -1, dtype=torch.int64, device=self.device)
        ws = self._workspace(lib.lipcache_construct_workspace_bytes(ctypes.byref(cs), n, int(n_classes), int(budget)))
        got = ctypes.c_int64(0)
        st = lib.lipcache_construct(ctypes.byref(cs), _p(z), _p(label), _p(r), _p(guard_label), _p(priority), n,
                                    strat, int(budget), int(per_class), int(n_classes), _p(sel), ctypes.byref(got),
                                    _p(ws), ws.numel(), _stream(self.device))
        L.check("lipcache_construct", st)
        self.n = int(cs.n)
        return int(got.value), sel[: got.value]

    def boundary_radius(self, mode: str, factor: float, n_classes: int = 0) -> torch.Tensor:
        """lipcache_boundary_radius: per-entry radii of a reuse boundary (async)."""
        lib = L.load()
        out = torch.empty(max(self.n, 1), dtype=torch.float32, device=self.device)
        ws = workspace(lib.lipcache_boundary_radius_workspace_bytes(self.d, int(n_classes)), self.device)
        cs = self.cstruct()
        st = lib.lipcache_boundary_radius(ctypes.byref(cs), _BOUNDARY[mode], float(factor), int(n_classes),
                                          _p(out), _p(ws), ws.numel(), _stream(self.device))
        L.check("lipcache_boundary_radius", st)
        return out[: self.n]

    def with_radii(self, r: torch.Tensor) -> "LipCache":
        """A lookup-only view of this cache whose radii are ``r`` (features,
        labels and norms shared)."""
        _need_cuda(r, "r", torch.float32, 1)
        if r.shape[0] < self.n:
            raise ValueError("with_radii: one radius per live entry")
        v = LipCache.__new__(LipCache)
        v.__dict__.update(self.__dict__)
        v.r = r
        v._ws = None
        return v

    def build_index(self, K: int, iters: int = 4) -> "ClusterIndex":
        """lipcache_index_build over the current rows (async; the index owns its arrays)."""
        lib = L.load()
        n, d = self.n, self.d
        if n < 1:
            raise ValueError("build_index: the cache is empty")
        ix = ClusterIndex.__new__(ClusterIndex)
        ix.sorted = LipCache(d, n, store=self.store, device=self.device, image=self.zimg is not None)
        ix.perm = torch.empty(n, dtype=torch.int64, device=self.device)
        ix.offsets = torch.empty(int(K) + 1, dtype=torch.int64, device=self.device)
        ix.centers = torch.empty((int(K), d), dtype=torch.float32, device=self.device)
        ix.bound = torch.empty(int(K), dtype=torch.float32, device=self.device)
        ix.K, ix.n_indexed = int(K), 0
        ws = workspace(lib.lipcache_index_build_workspace_bytes(n, d, int(K)), self.device)
        cs = self.cstruct()
        st_ = ix.cstruct()
        st = lib.lipcache_index_build(ctypes.byref(cs), int(K), int(iters), ctypes.byref(st_), _p(ws), ws.numel(),
                                      _stream(self.device))
        L.check("lipcache_index_build", st)
        ix.n_indexed = int(st_.n_indexed)
        ix.sorted.n = int(st_.sorted.n)
        ix._build_ws = ws  # kept alive until the build has run
        return ix

    def lookup_indexed(self, index: "ClusterIndex", zq: torch.Tensor, precision: str = "f16",
                       out: LookupResult | None = None) -> tuple[LookupResult, int]:
        """lipcache_lookup_indexed: the lookup's outputs through a cluster index
        (sync).  Returns (result, query-entry pairs the filter scanned)."""
        _need_cuda(zq, "zq", torch.float32, 2)
        if zq.shape[1] != self.d:
            raise ValueError("lookup_indexed: query width differs from the cache's d")
        lib = L.load()
        B = zq.shape[0]
        dev = self.device
        if out is None:
            out = LookupResult(torch.empty(B, dtype=torch.int32, device=dev),
                               torch.empty(B, dtype=torch.int64, device=dev),
                               torch.empty(B, dtype=torch.float32, device=dev),
                               torch.zeros(4, dtype=torch.int64, device=dev),
                               torch.empty(B, dtype=torch.uint8, device=dev))
        prec = _PRECISION[precision]
        ws = self._workspace(lib.lipcache_lookup_indexed_workspace_bytes(B, self.n, self.d, index.K, index.n_indexed))
        cs = self.cstruct()
        ic = index.cstruct()
        pairs = ctypes.c_int64(0)
        st = lib.lipcache_lookup_indexed(ctypes.byref(cs), ctypes.byref(ic), _p(zq), B, prec, _p(out.label),
                                         _p(out.index), _p(out.dist2), _p(out.stats), _p(out.band),
                                         ctypes.byref(pairs), _p(ws), ws.numel(), _stream(dev))
        L.check("lipcache_lookup_indexed", st)
        return out, int(pairs.value)

    def filter_dump(self, zq: torch.Tensor, precision: str = "f16"):
        """lipcache_lookup_filter_dump: matrix-core dot products and filter decisions (small sizes)."""
        _need_cuda(zq, "zq", torch.float32, 2)
        lib = L.load()
        B = zq.shape[0]
        g_hat = torch.full((B, self.n), float("nan"), dtype=torch.float32, device=self.device)
        cand = torch.zeros((B, self.n), dtype=torch.uint8, device=self.device)
        prec = _PRECISION[precision]
        ws = self._workspace(lib.lipcache_lookup_workspace_bytes(B, self.n, self.d, prec))
        cs = self.cstruct()
        st = lib.lipcache_lookup_filter_dump(ctypes.byref(cs), _p(zq), B, prec, _p(g_hat), _p(cand), _p(ws),
                                             ws.numel(), _stream(self.device))
        L.check("lipcache_lookup_filter_dump", st)
        return g_hat, cand


class ClusterIndex:
    """Exact cluster index of a LipCache (lipcache_index): the indexed rows in
    cluster order, the cluster offsets, centres and bounds R_c."""

    sorted: LipCache
    perm: torch.Tensor      # int64 [n_indexed]: cache row of sorted row j
    offsets: torch.Tensor   # int64 [K + 1]
    centers: torch.Tensor   # float32 [K, d]
    bound: torch.Tensor     # float32 [K]
    K: int
    n_indexed: int

    def cstruct(self) -> L.LipcacheIndex:
        return L.LipcacheIndex(self.sorted.cstruct(), self.perm.data_ptr(), self.offsets.data_ptr(),
                               self.centers.data_ptr(), self.bound.data_ptr(), self.K, self.n_indexed)


def consistency(lookup_label: torch.Tensor, head_label: torch.Tensor) -> tuple[int, int]:
    """lipcache_consistency: (hits, hits returning the head's own label) (sync)."""
    _need_cuda(lookup_label, "lookup_label", torch.int32, 1)
    _need_cuda(head_label, "head_label", torch.int32, 1)
    if lookup_label.shape != head_label.shape:
        raise ValueError("consistency: shapes differ")
    lib = L.load()
    counts = torch.empty(2, dtype=torch.int64, device=lookup_label.device)
    st = lib.lipcache_consistency(_p(lookup_label), _p(head_label), lookup_label.shape[0], _p(counts),
                                  _stream(lookup_label.device))
    L.check("lipcache_consistency", st)
    h, c = counts.cpu().tolist()
    return int(h), int(c)


# ------------------------------------------------------- adapting a shared head
_DTYPE = {torch.float32: L.F32, torch.bfloat16: L.BF16, torch.float16: L.F16}


def _dtype(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(device: torch.device) -> int:
    """The current stream's handle; torch.cuda.current_stream builds an object around it (2 us a call)."""
    if _raw_stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index if device.index is not None else torch.cuda.current_device())


def _need_rows(t: torch.Tensor, name: str, dtype: torch.dtype, device: torch.device, rows: int, width: int) -> int:
    """Checks a [rows, width] matrix whose rows may lie apart; returns their distance in elements."""
    if t.dtype is dtype and t.device == device and t.shape == (rows, width):
        if t.is_contiguous():
            return width
        if (width == 1 or t.stride(1) == 1) and (rows == 1 or t.stride(0) >= width):
            return t.stride(0) if rows > 1 else width
        raise ValueError(f"{name} must have contiguous, non-overlapping rows")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must be [{rows}, {width}], got {list(t.shape)}")


def _need_shape(t: torch.Tensor, name: str, dtype: torch.dtype, device: torch.device, shape: tuple) -> None:
    if t.dtype is dtype and t.device == device and t.shape == shape and t.is_contiguous():
        return
    if t.device != device:
        raise ValueError(f"{name} must be on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _adapters(A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor, offsets: torch.Tensor, adapter: torch.Tensor,
              dtype: torch.dtype, device: torch.device, K: int, N: int) -> L.LipcacheAdapters:
    if A.dim() != 3:
        raise ValueError("A must be [S, r, K]")
    S, r, _ = A.shape
    _need_shape(A, "A", dtype, device, (S, r, K))
    _need_shape(B, "B", dtype, device, (S, N, r))
    _need_shape(scale, "scale", torch.float32, device, (S,))
    if adapter.dim() != 1:
        raise ValueError("adapter must be [R]")
    R = adapter.shape[0]
    _need_shape(adapter, "adapter", torch.int32, device, (R,))
    _need_shape(offsets, "offsets", torch.int32, device, (R + 1,))
    return L.LipcacheAdapters(A.data_ptr(), B.data_ptr(), scale.data_ptr(), offsets.data_ptr(), adapter.data_ptr(),
                              S, r, R)


@dataclass
class AdapterOutput:
    y: torch.Tensor           # [T, N], x's type
    v: torch.Tensor | None    # float32 [T, r]: A_a x of every row (zero without a pair)


def adapter_forward(x: torch.Tensor, W: torch.Tensor, bias: torch.Tensor | None, A: torch.Tensor, B: torch.Tensor,
                    scale: torch.Tensor, offsets: torch.Tensor, adapter: torch.Tensor, keep: bool = False,
                    out: AdapterOutput | None = None) -> AdapterOutput:
    """lipcache_adapter_forward: W x + bias + scale_a B_a (A_a x) for every row of a batch of requests (async).

    x [T, K] and W [N, K] of one type (float32, bfloat16 or float16; rows may
    lie apart), bias float32 [N] or None, A [S, r, K], B [S, N, r], scale
    float32 [S]; request i owns the rows offsets[i]:offsets[i + 1] (int32,
    R + 1 of them) and names the pair adapter[i] (int32, -1: none).  ``keep``
    also returns v, which the backward pass takes; ``out.v``, if it is there, is
    written without it.  ``out`` must not overlap what is read."""
    code = _dtype(x, "x")
    dev, dt = x.device, x.dtype
    if x.dim() != 2 or W.dim() != 2:
        raise ValueError("x must be [T, K] and W [N, K]")
    T, K = x.shape
    N = W.shape[0]
    ldx = _need_rows(x, "x", dt, dev, T, K)
    ldw = _need_rows(W, "W", dt, dev, N, K)
    if bias is not None:
        _need_shape(bias, "bias", torch.float32, dev, (N,))
    ad = _adapters(A, B, scale, offsets, adapter, dt, dev, K, N)
    if out is None:
        out = AdapterOutput(x.new_empty((T, N)),
                            torch.empty((T, ad.r), dtype=torch.float32, device=dev) if keep else None)
        ldy = N
    else:
        ldy = _need_rows(out.y, "out.y", dt, dev, T, N)
        if out.v is None and keep:
            out.v = torch.empty((T, ad.r), dtype=torch.float32, device=dev)
        elif out.v is not None:
            _need_shape(out.v, "out.v", torch.float32, dev, (T, ad.r))
    lib = L.load()
    ws = workspace(lib.lipcache_adapter_forward_workspace_bytes(T, K, N, ad.r, ad.S, code), dev)
    st = lib.lipcache_adapter_forward(x.data_ptr(), ldx, T, W.data_ptr(), ldw, None if bias is None else bias.data_ptr(),
                                      K, N, ctypes.byref(ad), code, out.y.data_ptr(), ldy,
                                      None if out.v is None else out.v.data_ptr(), ws.data_ptr(), ws.numel(),
                                      _stream_of(dev))
    L.check("lipcache_adapter_forward", st)
    return out


@dataclass
class AdapterGradients:
    dx: torch.Tensor | None   # [T, K]
    dA: torch.Tensor | None   # [S, r, K]
    dB: torch.Tensor | None   # [S, N, r]


def adapter_backward(dy: torch.Tensor, x: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                     scale: torch.Tensor, offsets: torch.Tensor, adapter: torch.Tensor, v: torch.Tensor | None = None,
                     want_dx: bool = True, want_pairs: bool = True) -> AdapterGradients:
    """lipcache_adapter_backward: gradients of the rows and of every pair, W and bias frozen (async).

    dy [T, N] is the gradient of y; ``v`` is the forward pass's (computed
    again when None); the others are the forward pass's arguments."""
    code = _dtype(x, "x")
    dev, dt = x.device, x.dtype
    if x.dim() != 2 or W.dim() != 2:
        raise ValueError("x must be [T, K] and W [N, K]")
    T, K = x.shape
    N = W.shape[0]
    ldx = _need_rows(x, "x", dt, dev, T, K)
    lddy = _need_rows(dy, "dy", dt, dev, T, N)
    ldw = _need_rows(W, "W", dt, dev, N, K)
    ad = _adapters(A, B, scale, offsets, adapter, dt, dev, K, N)
    if v is not None:
        _need_shape(v, "v", torch.float32, dev, (T, ad.r))
    g = AdapterGradients(x.new_empty((T, K)) if want_dx else None,
                         torch.empty_like(A) if want_pairs else None, torch.empty_like(B) if want_pairs else None)
    lib = L.load()
    ws = workspace(lib.lipcache_adapter_backward_workspace_bytes(T, K, N, ad.r, ad.S, code), dev)
    st = lib.lipcache_adapter_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, T, W.data_ptr(), ldw, K, N,
                                       ctypes.byref(ad), code, None if v is None else v.data_ptr(),
                                       g.dx.data_ptr() if want_dx else None, K, g.dA.data_ptr() if want_pairs else None,
                                       g.dB.data_ptr() if want_pairs else None, ws.data_ptr(), ws.numel(),
                                       _stream_of(dev))
    L.check("lipcache_adapter_backward", st)
    return g


# Brings singular values to about [0.7, 1.2] in five steps (K. Jordan et al., "Muon: An optimizer for hidden layers in neural
# networks", 2024).
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def _coefficients(steps: int, coefficients):
    """float[steps][3] from one (a, b, c) for all steps or one for each."""
    rows = list(coefficients)
    if rows and not hasattr(rows[0], "__len__"):
        rows = [rows] * int(steps)
    if len(rows) != int(steps) or any(len(row) != 3 for row in rows):
        raise ValueError("coefficients must be one (a, b, c), or one for each step")
    return (ctypes.c_float * max(1, 3 * int(steps)))(*[float(c) for row in rows for c in row])


def _stack(t: torch.Tensor, name: str) -> tuple[int, int, int]:
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be a matrix or a stack of them")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return (1, *t.shape) if t.dim() == 2 else tuple(t.shape)


def orthogonalise(G: torch.Tensor, steps: int = 5, coefficients=NEWTON_SCHULZ, eps: float = 1e-7,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """lipcache_orthogonalise: Newton-Schulz products of a matrix [m, n] or a stack [b, m, n] (async).

    ``coefficients``: one (a, b, c) for all steps or one for each; ``out`` may be G."""
    code = _dtype(G, "G")
    b, m, n = _stack(G, "G")
    if out is None:
        out = torch.empty_like(G)
    else:
        _need_shape(out, "out", G.dtype, G.device, tuple(G.shape))
    coef = _coefficients(steps, coefficients)
    lib = L.load()
    ws = workspace(lib.lipcache_orthogonalise_workspace_bytes(b, m, n, code), G.device)
    st = lib.lipcache_orthogonalise(G.data_ptr(), b, m, n, code, int(steps), coef, float(eps), out.data_ptr(),
                                    ws.data_ptr(), ws.numel(), _stream_of(G.device))
    L.check("lipcache_orthogonalise", st)
    return out


def muon_step(W: torch.Tensor, G: torch.Tensor, M: torch.Tensor, lr: float, momentum: float = 0.95,
              weight_decay: float = 0.0, nesterov: bool = True, scale: float | None = None, steps: int = 5,
              coefficients=NEWTON_SCHULZ, eps: float = 1e-7, short_operands: bool = False) -> None:
    """lipcache_muon_step: one step along the orthogonalised momentum, W and M in place (async).

    W and G [m, n] or [b, m, n] of one type, M float32 of the same shape.
    ``scale``: the update's factor, sqrt(max(1, m / n)) when None.
    ``short_operands`` (16-bit W): products of 11-bit operands in place of
    22-bit ones, 2.5 times as fast on large matrices; the update is then 2e-3 to 4e-3
    of its norm off."""
    code = _dtype(W, "W")
    b, m, n = _stack(W, "W")
    _need_shape(G, "G", W.dtype, W.device, tuple(W.shape))
    _need_shape(M, "M", torch.float32, W.device, tuple(W.shape))
    if scale is None:
        scale = max(1.0, m / max(n, 1)) ** 0.5
    coef = _coefficients(steps, coefficients)
    opt = L.LipcacheMuon(float(lr), float(momentum), float(weight_decay), float(scale), float(eps),
                         int(bool(nesterov)) | (L.MUON_SHORT_OPERANDS if short_operands else 0), int(steps), ctypes.cast(coef, ctypes.POINTER(ctypes.c_float)))
    lib = L.load()
    ws = workspace(lib.lipcache_muon_step_workspace_bytes(b, m, n, code), W.device)
    st = lib.lipcache_muon_step(W.data_ptr(), G.data_ptr(), M.data_ptr(), b, m, n, code, ctypes.byref(opt),
                                ws.data_ptr(), ws.numel(), _stream_of(W.device))
    L.check("lipcache_muon_step", st)


# ------------------------------------------- scoring answers, learning from a teacher
@dataclass
class LogProbs:
    logp: torch.Tensor                # float32 [T]: log probability of the row's label, 0 where it has none
    lse: torch.Tensor                 # float32 [T]: log of the sum of exponentials
    entropy: torch.Tensor             # float32 [T]
    top_index: torch.Tensor | None    # int32 [T, top]: classes by falling logit, -1 where a row has fewer
    top_logp: torch.Tensor | None     # float32 [T, top]: their log probabilities


def _on_device(call):
    """The call with its first tensor's device current: a stream's handle alone does not say which device's it is."""
    name = next(iter(inspect.signature(call).parameters))

    @functools.wraps(call)
    def on_device(*args, **kw):
        first = args[0] if args else kw.get(name)
        if not isinstance(first, torch.Tensor) or not first.is_cuda or first.device.index == torch.cuda.current_device():
            return call(*args, **kw)
        with torch.cuda.device(first.device):
            return call(*args, **kw)
    return on_device


def _rows_of(t: torch.Tensor, name: str) -> tuple[int, int, int]:
    """[T, C] rows: T, C and the distance between rows."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be [T, C]")
    T, C = t.shape
    return T, C, _need_rows(t, name, t.dtype, t.device, T, C)


def _of_rows(t: torch.Tensor | None, name: str, dtype: torch.dtype, device: torch.device, shape: tuple):
    """The address of a [T] or [T, k] tensor, None where it is None."""
    if t is None:
        return None
    _need_shape(t, name, dtype, device, shape)
    return t.data_ptr()


def _few_rows(query: str, T: int, C: int, k: int, code: int, device: torch.device):
    """The workspace of a call: its address and size, and what holds it until the call is made."""
    if T > L.FEW_ROWS:
        return None, 0, None
    need = getattr(L.load(), query)(T, C, k, code)
    if need == 0:
        return None, 0, None
    ws = workspace(need, device)
    return ws.data_ptr(), ws.numel(), ws


def _entries(index: torch.Tensor | None, value: torch.Tensor | None, names: tuple[str, str], device: torch.device, T: int):
    """k and the addresses of [T, k] classes and their values."""
    if (index is None) != (value is None):
        raise ValueError(f"{names[0]} and {names[1]} go together")
    if index is None:
        return 0, None, None
    if index.dim() != 2:
        raise ValueError(f"{names[0]} must be [T, k]")
    k = index.shape[1]
    return (k, _of_rows(index, names[0], torch.int32, device, (T, k)),
            _of_rows(value, names[1], torch.float32, device, (T, k)))


@_on_device
def logprobs(logits: torch.Tensor, labels: torch.Tensor | None = None, top: int = 0, temperature: float = 1.0,
             out: LogProbs | None = None) -> LogProbs:
    """lipcache_logprobs: log probabilities of labels, entropies and the ``top`` most likely classes of rows (async).

    logits [T, C] float32, bfloat16 or float16 (rows may lie apart), labels int32 [T]
    (outside [0, C): none) or None.  ``out`` must not overlap what is read."""
    code = _dtype(logits, "logits")
    T, C, ld = _rows_of(logits, "logits")
    dev, k = logits.device, int(top)
    if not 0 <= k <= L.MOST_TOP:
        raise ValueError(f"top must be 0 to {L.MOST_TOP}")
    label = _of_rows(labels, "labels", torch.int32, dev, (T,))
    f32, i32 = torch.float32, torch.int32
    if out is None:
        each = torch.empty((3, T), dtype=f32, device=dev)
        out = LogProbs(*each.unbind(0), None, None)
        at = each.data_ptr()
        logp, lse, entropy, index, value = at, at + 4 * T, at + 8 * T, None, None
        if k:
            out.top_index = torch.empty((T, k), dtype=i32, device=dev)
            out.top_logp = torch.empty((T, k), dtype=f32, device=dev)
            index, value = out.top_index.data_ptr(), out.top_logp.data_ptr()
    else:
        if k and (out.top_index is None or out.top_logp is None):
            raise ValueError("out lacks top_index or top_logp")
        logp, lse, entropy = (_of_rows(getattr(out, name), "out." + name, f32, dev, (T,)) for name in ("logp", "lse", "entropy"))
        index = _of_rows(out.top_index, "out.top_index", i32, dev, (T, k)) if k else None
        value = _of_rows(out.top_logp, "out.top_logp", f32, dev, (T, k)) if k else None
    ws, size, held = _few_rows("lipcache_logprobs_workspace_bytes", T, C, k, code, dev)
    st = L.load().lipcache_logprobs(logits.data_ptr(), ld, T, C, code, float(temperature), label, k, logp, lse, entropy,
                                    index, value, ws, size, _stream_of(dev))
    L.check("lipcache_logprobs", st)
    return out


@_on_device
def logprobs_backward(logits: torch.Tensor, labels: torch.Tensor | None = None, g_logp: torch.Tensor | None = None,
                      g_lse: torch.Tensor | None = None, g_entropy: torch.Tensor | None = None,
                      top_index: torch.Tensor | None = None, g_top: torch.Tensor | None = None,
                      temperature: float = 1.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """lipcache_logprobs_backward: the gradient of ``logprobs`` with regard to the logits [T, C], their type (async).

    g_logp, g_lse, g_entropy float32 [T] and g_top float32 [T, k] are the gradients of
    what ``logprobs`` gave (None: zero), top_index int32 [T, k] its classes, or any others.  ``out`` may be logits."""
    code = _dtype(logits, "logits")
    T, C, ld = _rows_of(logits, "logits")
    dev, f32 = logits.device, torch.float32
    label = _of_rows(labels, "labels", torch.int32, dev, (T,))
    if g_logp is not None and labels is None:
        raise ValueError("g_logp needs labels")
    k, index, value = _entries(top_index, g_top, ("top_index", "g_top"), dev, T)
    if k > L.MOST_ENTRIES:
        raise ValueError(f"g_top must have at most {L.MOST_ENTRIES} columns")
    if out is None:
        out, ldd = logits.new_empty((T, C)), C
    else:
        ldd = _need_rows(out, "out", logits.dtype, dev, T, C)
    ws, size, held = _few_rows("lipcache_logprobs_backward_workspace_bytes", T, C, k, code, dev)
    st = L.load().lipcache_logprobs_backward(
        logits.data_ptr(), ld, T, C, code, float(temperature), label, _of_rows(g_logp, "g_logp", f32, dev, (T,)),
        _of_rows(g_lse, "g_lse", f32, dev, (T,)), _of_rows(g_entropy, "g_entropy", f32, dev, (T,)), k, index, value,
        out.data_ptr(), ldd, ws, size, _stream_of(dev))
    L.check("lipcache_logprobs_backward", st)
    return out


@dataclass
class Distilled:
    ce: torch.Tensor            # float32 [T]: cross entropy with the label, 0 where there is none
    kl: torch.Tensor            # float32 [T]: divergence from the teacher's entries, 0 where there are none
    grad: torch.Tensor | None   # [T, C], the logits' type: gradient of sum weight (hard ce + soft kl)


@_on_device
def distill(logits: torch.Tensor, teacher: torch.Tensor | None, index: torch.Tensor | None,
            labels: torch.Tensor | None = None, weight: torch.Tensor | None = None, hard: float = 0.0, soft: float = 1.0,
            temperature: float = 1.0, want_grad: bool = True, out: torch.Tensor | None = None) -> Distilled:
    """lipcache_distill: losses against labels and a teacher's top logits, and their gradient, in one call (async).

    logits [T, C] (rows may lie apart), teacher float32 [T, k] at the classes index
    int32 [T, k] (outside [0, C): no entry), labels int32 [T] or None, weight float32 [T] or
    None (1).  ``out``: where the gradient goes; may be logits."""
    code = _dtype(logits, "logits")
    T, C, ld = _rows_of(logits, "logits")
    dev, f32 = logits.device, torch.float32
    k, at, value = _entries(index, teacher, ("index", "teacher"), dev, T)
    if k > L.MOST_ENTRIES:
        raise ValueError(f"teacher must have at most {L.MOST_ENTRIES} columns")
    label = _of_rows(labels, "labels", torch.int32, dev, (T,))
    each = torch.empty((2, T), dtype=f32, device=dev)
    losses, ldd = each.data_ptr(), C
    if out is not None:
        if not want_grad:
            raise ValueError("out is the gradient's: it goes with want_grad")
        ldd = _need_rows(out, "out", logits.dtype, dev, T, C)
    elif want_grad:
        out = logits.new_empty((T, C))
    ws, size, held = _few_rows("lipcache_distill_workspace_bytes", T, C, k, code, dev)
    st = L.load().lipcache_distill(logits.data_ptr(), ld, T, C, code, float(temperature), float(hard), float(soft), k, value,
                                   at, label, _of_rows(weight, "weight", f32, dev, (T,)), losses, losses + 4 * T,
                                   None if out is None else out.data_ptr(), ldd, ws, size, _stream_of(dev))
    L.check("lipcache_distill", st)
    return Distilled(*each.unbind(0), out)


@_on_device
def head_logprobs(x: torch.Tensor, W: torch.Tensor, bias: torch.Tensor | None, labels: torch.Tensor | None = None,
                  temperature: float = 1.0) -> LogProbs:
    """lipcache_head_logprobs: ``logprobs`` of W x + bias without the logits in memory (async).

    x [T, K] and W [C, K] of one type (float32, bfloat16 or float16; rows may lie
    apart), bias float32 [C] or None, labels int32 [T] or None."""
    code = _dtype(x, "x")
    dev, dt = x.device, x.dtype
    if x.dim() != 2 or W.dim() != 2:
        raise ValueError("x must be [T, K] and W [C, K]")
    T, K = x.shape
    C = W.shape[0]
    ldx = _need_rows(x, "x", dt, dev, T, K)
    ldw = _need_rows(W, "W", dt, dev, C, K)
    each = torch.empty((3, T), dtype=torch.float32, device=dev)
    scores = each.data_ptr()
    lib = L.load()
    at_x, at_W = x.data_ptr(), W.data_ptr()
    ws = workspace(lib.lipcache_head_logprobs_workspace_bytes(at_x, ldx, T, at_W, ldw, K, C, code), dev)
    st = lib.lipcache_head_logprobs(at_x, ldx, T, at_W, ldw, _of_rows(bias, "bias", torch.float32, dev, (C,)), K, C, code,
                                    float(temperature), _of_rows(labels, "labels", torch.int32, dev, (T,)), scores,
                                    scores + 4 * T, scores + 8 * T, ws.data_ptr(), ws.numel(), _stream_of(dev))
    L.check("lipcache_head_logprobs", st)
    return LogProbs(*each.unbind(0), None, None)
