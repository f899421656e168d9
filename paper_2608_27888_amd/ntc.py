"""Python binding of libntc (ctypes): argument marshalling only.

Every step of the decode path runs in the HIP kernels of ``libntc.so``; this
module passes device pointers (``tensor.data_ptr()``) and the current HIP
stream.  PyTorch is used for device memory and streams only.  There is no
fallback: if the library is missing the import of the binding fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libntc.so")

NTC_OK = 0
NTC_ERR_ARG = -1
NTC_ERR_UNSUPPORTED = -2
NTC_ERR_CAPACITY = -3
NTC_ERR_HIP = -4
NTC_ERR_INDEX = -5
NTC_PAD = 0xFFFFFFFF
MAX_LEVELS = 4
MAX_LAYERS = 8


class NtcError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {status} ({status_string(status)})")
        self.status = status


class Grids(ctypes.Structure):
    _fields_ = [("n_textures", ctypes.c_int32), ("n_levels", ctypes.c_int32),
                ("res", ctypes.c_int32 * MAX_LEVELS), ("channels", ctypes.c_int32 * MAX_LEVELS),
                ("latents", ctypes.c_void_p)]


class Decoders(ctypes.Structure):
    _fields_ = [("n_decoders", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("dims", ctypes.c_int32 * (MAX_LAYERS + 1)), ("params", ctypes.c_void_p)]


class Queries(ctypes.Structure):
    _fields_ = [("tex_id", ctypes.c_void_p), ("uv", ctypes.c_void_p), ("mip", ctypes.c_void_p),
                ("n", ctypes.c_int64)]


class RouteOptions(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int32), ("renormalize", ctypes.c_int32),
                ("scale", ctypes.c_float), ("n_groups", ctypes.c_int32),
                ("top_groups", ctypes.c_int32), ("group_top", ctypes.c_int32)]


class LinearLayer(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("in_dim", ctypes.c_int32),
                ("out_dim", ctypes.c_int32), ("type", ctypes.c_int32),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


class LinearRows(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64),
                ("slots_per_row", ctypes.c_int32), ("bin_offset", ctypes.c_void_p),
                ("perm", ctypes.c_void_p), ("perm_capacity", ctypes.c_int64)]


class LinearEpilogue(ctypes.Structure):
    _fields_ = [("activation", ctypes.c_int32), ("leaky_slope", ctypes.c_float),
                ("output_format", ctypes.c_int32), ("residual", ctypes.c_void_p),
                ("residual_stride", ctypes.c_int64), ("pre", ctypes.c_void_p),
                ("pre_stride", ctypes.c_int64)]


class LinearGradsArgs(ctypes.Structure):
    _fields_ = [("dy", ctypes.c_void_p), ("dy_stride", ctypes.c_int64),
                ("dy_format", ctypes.c_int32), ("dx", ctypes.c_void_p),
                ("dx_stride", ctypes.c_int64), ("dweight", ctypes.c_void_p),
                ("dbias", ctypes.c_void_p), ("grad_format", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2608_27888_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.ntc_status_string.argtypes = [ctypes.c_int]
        L.ntc_status_string.restype = ctypes.c_char_p
        L.ntc_bins_workspace_bytes.argtypes = [i64, i32]
        L.ntc_bins_workspace_bytes.restype = sz
        L.ntc_bins_capacity.argtypes = [i64, i32, i32]
        L.ntc_bins_capacity.restype = i64
        L.ntc_build_bins.argtypes = [P, i64, P, i32, i32, i32, P, P, P, i64, P, sz, P]
        L.ntc_build_bins_noalloc.argtypes = [P, i64, P, i32, i32, i32, P, P, P, i64, P, P]
        L.ntc_get_device_error.argtypes = [P, P, P]
        L.ntc_decode.argtypes = [ctypes.POINTER(Grids), ctypes.POINTER(Decoders), P,
                                 ctypes.POINTER(Queries), P, P, i64, i32, P, P]
        L.ntc_decode_ex.argtypes = [ctypes.POINTER(Grids), ctypes.POINTER(Decoders), P,
                                    ctypes.POINTER(Queries), P, P, i64, i32, P, P, P]
        L.ntc_gather_features.argtypes = [ctypes.POINTER(Grids), ctypes.POINTER(Queries), P, i32,
                                          P]
        L.ntc_divergence_stats.argtypes = [P, i64, P, i32, i32, P, i64, i32, P, P, P]
        L.ntc_divergence_map.argtypes = [P, i32, i32, i32, P, i32, i32, i32, i32, P, P, i32, P, P]
        L.ntc_kmeans_workspace_bytes.argtypes = [i32, i32]
        L.ntc_kmeans_workspace_bytes.restype = sz
        L.ntc_kmeans.argtypes = [P, i32, i32, i32, P, i32, P, P, P, P, sz, P]
        L.ntc_kmeans_result.argtypes = [P, i32, i32, P, P, P]
        R = ctypes.POINTER
        L.ntc_route.argtypes = [P, i64, i32, i64, i32, i32, P, P, R(RouteOptions), P, P, P]
        L.ntc_route_backward.argtypes = [P, i64, i32, i64, i32, i32, P, P, R(RouteOptions), P, i64,
                                         P]
        L.ntc_linear_workspace_bytes.argtypes = [R(LinearLayer), R(LinearRows)]
        L.ntc_linear_workspace_bytes.restype = sz
        L.ntc_linear.argtypes = [R(LinearLayer), R(LinearRows), R(LinearEpilogue), P, i64, P, sz,
                                 P]
        L.ntc_linear_backward_workspace_bytes.argtypes = [R(LinearLayer), R(LinearRows),
                                                          R(LinearEpilogue), R(LinearGradsArgs)]
        L.ntc_linear_backward_workspace_bytes.restype = sz
        L.ntc_linear_backward.argtypes = [R(LinearLayer), R(LinearRows), R(LinearEpilogue),
                                          R(LinearGradsArgs), P, sz, P]
        L.ntc_combine.argtypes = [P, i64, i32, i64, i32, i32, P, P, i32, P, i64, P, i64, P]
        L.ntc_combine_backward.argtypes = [P, i64, P, i64, i32, i64, i32, i32, P, P, i32, P, i64, P,
                                           P]
        d = ctypes.c_double
        L.ntc_freeze_scale.argtypes = [d, d, d]
        L.ntc_freeze_scale.restype = d
        for f in ("ntc_build_bins", "ntc_build_bins_noalloc", "ntc_get_device_error", "ntc_decode", "ntc_decode_ex",
                  "ntc_gather_features",
                  "ntc_divergence_stats", "ntc_divergence_map", "ntc_kmeans",
                  "ntc_kmeans_result", "ntc_route", "ntc_route_backward", "ntc_linear",
                  "ntc_linear_backward", "ntc_combine", "ntc_combine_backward"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().ntc_status_string(int(status)).decode()


def _check(fn: str, status: int):
    if status != NTC_OK:
        raise NtcError(fn, status)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libntc takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libntc takes contiguous tensors")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream: Optional[torch.cuda.Stream]):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


# ----------------------------------------------------------------------------- binning


def workspace_bytes(n: int, n_decoders: int) -> int:
    return int(lib().ntc_bins_workspace_bytes(n, n_decoders))


def perm_capacity(n: int, n_decoders: int, align: int = 64) -> int:
    return int(lib().ntc_bins_capacity(n, n_decoders, align))


@dataclass
class Bins:
    """Outputs of ntc_build_bins (device tensors, uint32 stored as int32)."""

    bin_count: torch.Tensor
    bin_offset: torch.Tensor
    perm: torch.Tensor
    workspace: torch.Tensor
    align: int

    @property
    def capacity(self) -> int:
        return int(self.perm.numel())


def alloc_bins(n: int, n_decoders: int, align: int = 64, device="cuda") -> Bins:
    cap = perm_capacity(n, n_decoders, align)
    ws = workspace_bytes(n, n_decoders)
    if cap < 0 or ws == 0:
        raise NtcError("alloc_bins", NTC_ERR_ARG)
    return Bins(torch.empty(n_decoders, dtype=torch.int32, device=device),
                torch.empty(n_decoders + 1, dtype=torch.int32, device=device),
                torch.empty(max(cap, 1), dtype=torch.int32, device=device),
                torch.empty(ws, dtype=torch.uint8, device=device), align)


def build_bins(tex_id: torch.Tensor, tex_to_dec: torch.Tensor, n_decoders: int, align: int = 64,
               n_textures: Optional[int] = None, bins: Optional[Bins] = None,
               stream=None) -> Bins:
    n = int(tex_id.numel())
    T = int(tex_to_dec.numel()) if n_textures is None else int(n_textures)
    if bins is None:
        bins = alloc_bins(n, n_decoders, align, tex_id.device)
    _check("ntc_build_bins", lib().ntc_build_bins(
        _ptr(tex_id), n, _ptr(tex_to_dec), T, n_decoders, align, _ptr(bins.bin_count),
        _ptr(bins.bin_offset), _ptr(bins.perm), bins.capacity, _ptr(bins.workspace),
        int(bins.workspace.numel()), _stream(stream)))
    return bins


NOALLOC_SCRATCH_BYTES = 5 << 20  # NTC_NOALLOC_SCRATCH_BYTES


def build_bins_noalloc(tex_id: torch.Tensor, tex_to_dec: torch.Tensor, n_decoders: int,
                       bin_count: torch.Tensor, bin_offset: torch.Tensor, perm: torch.Tensor,
                       align: int = 64, n_textures: Optional[int] = None,
                       n_invalid: Optional[torch.Tensor] = None, stream=None) -> None:
    """ntc_build_bins_noalloc: binning into caller-owned outputs with the library's
    own device scratch (no workspace); n_invalid (one int32 on the device, or
    None) receives the count of queries left out of every bin."""
    n = int(tex_id.numel())
    T = int(tex_to_dec.numel()) if n_textures is None else int(n_textures)
    _check("ntc_build_bins_noalloc", lib().ntc_build_bins_noalloc(
        _ptr(tex_id), n, _ptr(tex_to_dec), T, n_decoders, align, _ptr(bin_count),
        _ptr(bin_offset), _ptr(perm), int(perm.numel()), _ptr(n_invalid), _stream(stream)))


def device_error(bins: Bins, stream=None) -> int:
    """Synchronises; returns the number of queries left out of every bin."""
    v = ctypes.c_uint64(0)
    st = lib().ntc_get_device_error(_ptr(bins.workspace), ctypes.byref(v), _stream(stream))
    if st not in (NTC_OK, NTC_ERR_INDEX):
        raise NtcError("ntc_get_device_error", st)
    return int(v.value)


# ----------------------------------------------------------------------------- decode


@dataclass
class DeviceModel:
    """Latent grids, decoders and the texture -> decoder map, resident on the device."""

    n_textures: int
    res: list
    channels: list
    latents: torch.Tensor      # int16 view of fp16 bits
    n_decoders: int
    dims: list
    params: torch.Tensor       # int16 view of fp16 bits
    tex_to_dec: torch.Tensor   # int32 view of uint32
    pe_octaves: int = 0        # positional-encoding octaves of the decoder input

    def grids(self) -> Grids:
        g = Grids()
        g.n_textures = self.n_textures
        g.n_levels = len(self.res)
        for i, (r, c) in enumerate(zip(self.res, self.channels)):
            g.res[i] = r
            g.channels[i] = c
        g.latents = _ptr(self.latents)
        return g

    def decoders(self) -> Decoders:
        d = Decoders()
        d.n_decoders = self.n_decoders
        d.n_layers = len(self.dims) - 1
        for i, v in enumerate(self.dims):
            d.dims[i] = v
        d.params = _ptr(self.params)
        return d

    @property
    def out_dim(self) -> int:
        return int(self.dims[-1])


@dataclass
class DeviceQueries:
    tex_id: torch.Tensor          # int32 view of uint32 [n]
    uv: torch.Tensor              # float32 [n, 2]
    mip: Optional[torch.Tensor]   # float32 [n] or None

    @property
    def n(self) -> int:
        return int(self.tex_id.numel())

    def struct(self) -> Queries:
        q = Queries()
        q.tex_id = _ptr(self.tex_id)
        q.uv = _ptr(self.uv)
        q.mip = _ptr(self.mip)
        q.n = self.n
        return q


def _dev(a: np.ndarray, dtype, device) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a).view(dtype)).to(device)


def upload(w, device="cuda"):
    """Host workload (paper_2608_27888_amd.workloads.Workload) -> (DeviceModel, DeviceQueries)."""
    model = DeviceModel(w.n_textures, list(w.res), list(w.channels),
                        _dev(w.latents, np.int16, device), w.n_decoders, list(w.dims),
                        _dev(w.params, np.int16, device), _dev(w.tex_to_dec, np.int32, device),
                        int(getattr(w, "pe_octaves", 0)))
    queries = DeviceQueries(_dev(w.tex_id, np.int32, device), _dev(w.uv, np.float32, device),
                            None if w.mip is None else _dev(w.mip, np.float32, device))
    return model, queries


NTC_ACT_RELU, NTC_ACT_LEAKY_RELU = 0, 1
NTC_OUT_F32, NTC_OUT_F16 = 0, 1
NTC_ENGINE_MFMA, NTC_ENGINE_FMA, NTC_ENGINE_FMA_DIRECT = 0, 1, 2
ENGINES = {"mfma": NTC_ENGINE_MFMA, "fma": NTC_ENGINE_FMA, "fma_direct": NTC_ENGINE_FMA_DIRECT}
NTC_GATHER_DIRECT, NTC_GATHER_STAGED = 0, 1
GATHERS = {"direct": NTC_GATHER_DIRECT, "staged": NTC_GATHER_STAGED}


class DecodeOptions(ctypes.Structure):
    _fields_ = [("hidden_activation", ctypes.c_int32), ("leaky_slope", ctypes.c_float),
                ("output_format", ctypes.c_int32), ("pe_octaves", ctypes.c_int32),
                ("engine", ctypes.c_int32), ("gather", ctypes.c_int32)]


def decode(model: DeviceModel, queries: DeviceQueries, bins: Optional[Bins] = None,
           out: Optional[torch.Tensor] = None, stream=None, leaky_slope: Optional[float] = None,
           out_dtype: torch.dtype = torch.float32, engine: str = "mfma",
           gather: str = "direct") -> torch.Tensor:
    """Binned mode when `bins` is given, stream (divergent) mode otherwise.  Hidden
    activation ReLU, or LeakyReLU max(x, slope x) when leaky_slope is given; output
    rows float32 or float16; the model's positional-encoding octaves extend the
    decoder input.  engine "mfma" (tensor path), "fma" (per-lane vector FMA with
    the LDS decoder cache) or "fma_direct" (per-lane vector FMA, weights through
    the caches); the FMA engines take stream mode only.  gather "direct" or "staged" (taps staged in LDS, binned
    MFMA decode only)."""
    if engine not in ENGINES:
        raise ValueError("engine must be 'mfma', 'fma' or 'fma_direct'")
    if gather not in GATHERS:
        raise ValueError("gather must be 'direct' or 'staged'")
    if out_dtype not in (torch.float32, torch.float16):
        raise ValueError("out_dtype must be float32 or float16")
    if out is None:
        out = torch.empty((queries.n, model.out_dim), dtype=out_dtype,
                          device=queries.tex_id.device)
    elif out.dtype != out_dtype:
        raise ValueError("out has the wrong dtype")
    g, d, q = model.grids(), model.decoders(), queries.struct()
    opt = DecodeOptions(NTC_ACT_RELU if leaky_slope is None else NTC_ACT_LEAKY_RELU,
                        0.0 if leaky_slope is None else float(leaky_slope),
                        NTC_OUT_F16 if out_dtype == torch.float16 else NTC_OUT_F32,
                        int(model.pe_octaves), ENGINES[engine], GATHERS[gather])
    if bins is not None:
        st = lib().ntc_decode_ex(ctypes.byref(g), ctypes.byref(d), _ptr(model.tex_to_dec),
                                 ctypes.byref(q), _ptr(bins.bin_offset), _ptr(bins.perm),
                                 bins.capacity, bins.align, ctypes.byref(opt), _ptr(out),
                                 _stream(stream))
    else:
        st = lib().ntc_decode_ex(ctypes.byref(g), ctypes.byref(d), _ptr(model.tex_to_dec),
                                 ctypes.byref(q), None, None, 0, 0, ctypes.byref(opt), _ptr(out),
                                 _stream(stream))
    _check("ntc_decode_ex", st)
    return out


def gather_features(model: DeviceModel, queries: DeviceQueries, out: Optional[torch.Tensor] = None,
                    out_dtype: torch.dtype = torch.float32, stream=None) -> torch.Tensor:
    """ntc_gather_features: the feature vector of every query (the decode's gather
    step without the MLP), rows [n][n_levels * channels] of float32 or float16."""
    if out_dtype not in (torch.float32, torch.float16):
        raise ValueError("out_dtype must be float32 or float16")
    F = sum(model.channels)
    if out is None:
        out = torch.empty((queries.n, F), dtype=out_dtype, device=queries.tex_id.device)
    elif out.dtype != out_dtype:
        raise ValueError("out has the wrong dtype")
    g, q = model.grids(), queries.struct()
    _check("ntc_gather_features", lib().ntc_gather_features(
        ctypes.byref(g), ctypes.byref(q), _ptr(out),
        NTC_OUT_F16 if out_dtype == torch.float16 else NTC_OUT_F32, _stream(stream)))
    return out


# ----------------------------------------------------------------------------- divergence


def divergence_stats(tex_id: torch.Tensor, tex_to_dec: torch.Tensor, n_decoders: int,
                     order: Optional[torch.Tensor] = None, wave: int = 64,
                     n_textures: Optional[int] = None, stream=None):
    """-> (per_wave_distinct int32 tensor, totals int64 tensor [4])."""
    n = int(tex_id.numel())
    T = int(tex_to_dec.numel()) if n_textures is None else int(n_textures)
    ln = n if order is None else int(order.numel())
    per = torch.empty(max(1, (ln + wave - 1) // wave), dtype=torch.int32, device=tex_id.device)
    tot = torch.empty(4, dtype=torch.int64, device=tex_id.device)
    _check("ntc_divergence_stats", lib().ntc_divergence_stats(
        _ptr(tex_id), n, _ptr(tex_to_dec), T, n_decoders, _ptr(order), ln, wave, _ptr(per),
        _ptr(tot), _stream(stream)))
    return per[: (ln + wave - 1) // wave], tot


def divergence_map(tex_id: torch.Tensor, width: int, height: int, tex_to_dec: torch.Tensor,
                   n_decoders: int, spp: int = 1, block_w: int = 8, block_h: int = 8,
                   hist_len: int = 65, n_textures: Optional[int] = None, stream=None):
    """Distinct decoders per screen block -> (map int32 [Hb, Wb], histogram int32
    [hist_len], totals int64 [4])."""
    T = int(tex_to_dec.numel()) if n_textures is None else int(n_textures)
    if int(tex_id.numel()) != width * height * spp:
        raise ValueError("tex_id must hold width * height * spp queries")
    bx, by = (width + block_w - 1) // block_w, (height + block_h - 1) // block_h
    dmap = torch.empty((by, bx), dtype=torch.int32, device=tex_id.device)
    hist = torch.empty(hist_len, dtype=torch.int32, device=tex_id.device)
    tot = torch.empty(4, dtype=torch.int64, device=tex_id.device)
    _check("ntc_divergence_map", lib().ntc_divergence_map(
        _ptr(tex_id), width, height, spp, _ptr(tex_to_dec), T, n_decoders, block_w, block_h,
        _ptr(dmap), _ptr(hist), hist_len, _ptr(tot), _stream(stream)))
    return dmap, hist, tot


# ----------------------------------------------------------------------------- clustering


@dataclass
class Clusters:
    assign: torch.Tensor     # int32 [n]: c(i), the texture -> decoder map
    centroids: torch.Tensor  # float64 [m][dim]
    counts: torch.Tensor     # int32 [m]: k_g
    iterations: int
    converged: bool


def kmeans(features: torch.Tensor, init, max_iter: int = 100, stream=None) -> Clusters:
    """k-means of per-texture feature vectors (float32 [n][dim] on the device) into
    m = len(init) groups seeded by the textures `init` (host integers); the labels
    are a texture -> decoder map.  Synchronises to read the iteration count."""
    if features.dtype != torch.float32 or features.dim() != 2 or not features.is_contiguous():
        raise ValueError("features must be a contiguous float32 [n][dim] tensor")
    n, dim = features.shape
    seeds = np.ascontiguousarray(np.asarray(init, dtype=np.uint32))
    m = int(seeds.size)
    dev = features.device
    assign = torch.empty(n, dtype=torch.int32, device=dev)
    centroids = torch.empty((m, dim), dtype=torch.float64, device=dev)
    counts = torch.empty(m, dtype=torch.int32, device=dev)
    wsb = lib().ntc_kmeans_workspace_bytes(m, int(max_iter))
    ws = torch.empty(max(wsb, 4), dtype=torch.uint8, device=dev)
    st = lib().ntc_kmeans(_ptr(features), n, dim, m, seeds.ctypes.data_as(ctypes.c_void_p),
                          int(max_iter), _ptr(assign), _ptr(centroids), _ptr(counts), _ptr(ws),
                          wsb, _stream(stream))
    _check("ntc_kmeans", st)
    it, conv = ctypes.c_int32(0), ctypes.c_int32(0)
    _check("ntc_kmeans_result", lib().ntc_kmeans_result(_ptr(ws), m, int(max_iter), ctypes.byref(it),
                                                        ctypes.byref(conv), _stream(stream)))
    return Clusters(assign, centroids, counts, int(it.value), bool(conv.value))


def freeze_scale(epoch: float, freeze_start: Optional[float], freeze_duration: float) -> float:
    """Gradual decoder-freezing factor lambda(epoch); freeze_start None = never."""
    start = float("nan") if freeze_start is None else float(freeze_start)
    return float(lib().ntc_freeze_scale(float(epoch), start, float(freeze_duration)))


# ----------------------------------------------------------------------------- experts

# Nothing here is recorded by torch's autograd: results carry no history, whether or not the
# arguments require gradients.  The gradients are calls of their own (*_backward), which a
# torch.autograd.Function can make.

NTC_OUT_BF16 = 2
NTC_ACT_NONE, NTC_ACT_GELU, NTC_ACT_SILU = 2, 3, 4
TYPES = {torch.float32: NTC_OUT_F32, torch.float16: NTC_OUT_F16, torch.bfloat16: NTC_OUT_BF16}
SCORES = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {"none": NTC_ACT_NONE, "relu": NTC_ACT_RELU, "leaky_relu": NTC_ACT_LEAKY_RELU,
               "gelu": NTC_ACT_GELU, "silu": NTC_ACT_SILU}


class _Call:
    """The tensors of one call: checked to be on one device and, when the call runs on
    another stream than the current one, kept from reuse until that stream is done."""

    __slots__ = ("device", "raw", "side")

    def __init__(self, stream, lead: torch.Tensor):
        if not lead.is_cuda:
            raise ValueError("libntc takes device tensors")
        self.device = device = lead.device
        raw = torch._C._cuda_getCurrentRawStream(device.index)
        self.side = None
        if stream is not None:
            if stream.device != device:
                raise ValueError("the stream is on another device than the tensors")
            if stream.cuda_stream != raw:
                self.side = stream
                raw = stream.cuda_stream
        self.raw = raw

    def take(self, t, what, dtype, shape=None):
        """(address, row stride) of a tensor (None: (None, 0)): 2-D with rows of
        consecutive elements and any row stride, or contiguous.  dtype: the one it must
        have, or a container of those it may have."""
        if t is None:
            return None, 0
        if t.device != self.device:
            raise ValueError(f"{what} is on another device")
        if t.dtype is not dtype and (isinstance(dtype, torch.dtype) or t.dtype not in dtype):
            raise ValueError(f"{what} has the wrong dtype")
        size = t.shape
        if shape is not None and size != shape:
            raise ValueError(f"{what} must have the shape {tuple(shape)}")
        if len(size) == 2:
            (rows, cols), (stride, step) = size, t.stride()
            if (cols > 1 and step != 1) or (rows > 1 and stride < cols):
                raise ValueError(f"{what} must have rows of consecutive elements that don't "
                                 "overlap")
            if rows <= 1:
                stride = max(cols, 1)
        else:
            if not t.is_contiguous():
                raise ValueError(f"{what} must be contiguous")
            stride = size[-1] if size else 1
        if self.side is not None:
            t.record_stream(self.side)
        return t.data_ptr() or None, stride

    def empty(self, shape, dtype):
        if self.side is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        # memory that earlier work of the current stream may still use isn't that stream's
        with torch.cuda.stream(self.side):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(torch.cuda.current_stream(self.device))
        return t

    def workspace(self, size):
        """(tensor that keeps it, address)."""
        if size == 0:
            return None, None
        if self.side is None:
            t = torch.empty(size, dtype=torch.uint8, device=self.device)
        else:  # allocated on the stream that uses it: it goes back to that stream's calls
            with torch.cuda.stream(self.side):
                t = torch.empty(size, dtype=torch.uint8, device=self.device)
        return t, t.data_ptr()

    def run(self, fn, *args):
        call = getattr(lib(), fn)
        if torch.cuda.current_device() == self.device.index:
            status = call(*args, self.raw)
        else:
            with torch.cuda.device(self.device):
                status = call(*args, self.raw)
        if status != NTC_OK:
            raise NtcError(fn, status)


def _int32(v, what):
    """v as the library takes it; ctypes would cut off higher bits."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{what} doesn't fit 32 bits")
    return v


def _route_options(score, renormalize, scale, n_groups=1, top_groups=1, group_top=1):
    if score not in SCORES:
        raise ValueError("score must be 'softmax' or 'sigmoid'")
    return RouteOptions(SCORES[score], int(bool(renormalize)), float(scale),
                        _int32(n_groups, "n_groups"), _int32(top_groups, "top_groups"),
                        _int32(group_top, "group_top"))


@dataclass
class Routes:
    ids: torch.Tensor      # int32 view of uint32 [n][k], -1 (NTC_PAD) in empty slots
    weights: torch.Tensor  # float32 [n][k]


def route(logits: torch.Tensor, k: int, score: str = "softmax",
          bias: Optional[torch.Tensor] = None, n_groups: int = 1, top_groups: int = 1,
          group_top: int = 1, renormalize: bool = True, scale: float = 1.0,
          mask: Optional[torch.Tensor] = None, stream=None) -> Routes:
    """ntc_route: the k experts of every item and their weights from logits [n][experts]
    (float32, float16 or bfloat16).  bias (float32 [experts]) only moves the choice; with
    n_groups > 1 the experts come from the top_groups best groups, a group's value the
    sum of its group_top best; items whose mask (bool or uint8 [n]) is 0 get empty slots,
    as do items with fewer than k experts of a logit above -inf."""
    if logits.dim() != 2:
        raise ValueError("logits must be [n][experts]")
    n, E = logits.shape
    call = _Call(stream, logits)
    lp, ls = call.take(logits, "logits", TYPES)
    bp, _ = call.take(bias, "bias", torch.float32, (E,))
    mp, _ = call.take(mask, "mask", (torch.bool, torch.uint8), (n,))
    opt = _route_options(score, renormalize, scale, n_groups, top_groups, group_top)
    k = _int32(k, "k")
    if k < 1:
        raise ValueError("k must be at least 1")
    ids, weights = call.empty((n, k), torch.int32), call.empty((n, k), torch.float32)
    call.run("ntc_route", lp, ls, TYPES[logits.dtype], n, E, k, bp, mp, ctypes.byref(opt),
             ids.data_ptr() or None, weights.data_ptr() or None)
    return Routes(ids, weights)


def route_backward(logits: torch.Tensor, ids: torch.Tensor, dweights: torch.Tensor,
                   score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                   stream=None) -> torch.Tensor:
    """ntc_route_backward: the gradient of the logits (their dtype) from that of the
    weights (float32 [n][k]), the choice held fixed."""
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits must be [n][experts] and ids [n][k]")
    n, E = logits.shape
    k = int(ids.shape[1])
    call = _Call(stream, logits)
    lp, ls = call.take(logits, "logits", TYPES)
    ip = _rows_of(call, ids, "ids", torch.int32, (n, k))
    gp = _rows_of(call, dweights, "dweights", torch.float32, (n, k))
    opt = _route_options(score, renormalize, scale)
    out = call.empty((n, E), logits.dtype)
    op, os_ = call.take(out, "out", logits.dtype)
    call.run("ntc_route_backward", lp, ls, TYPES[logits.dtype], n, E, k, ip, gp,
             ctypes.byref(opt), op, os_)
    return out


def _rows_of(call, t, what, dtype, shape):
    """Pointer of a contiguous tensor."""
    if t is not None and not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return call.take(t, what, dtype, shape)[0]


def _layer(call, x, weight, bias, bins, slots_per_row):
    """(layer, rows, slots) of a linear call."""
    if x.dim() != 2 or weight.dim() != (2 if bins is None else 3):
        raise ValueError("x must be [rows][in] and weight [out][in], or [experts][out][in] "
                         "with bins")
    if x.dtype not in (torch.float16, torch.bfloat16):
        raise ValueError("x must be float16 or bfloat16")
    if _int32(slots_per_row, "slots_per_row") < 1:
        raise ValueError("slots_per_row must be at least 1")
    out_dim, in_dim = weight.shape[-2:]
    if x.shape[1] != in_dim:
        raise ValueError("x and weight differ in in_dim")
    E = 1 if bins is None else int(weight.shape[0])
    xp, xs = call.take(x, "x", x.dtype)
    wp = _rows_of(call, weight, "weight", x.dtype, weight.shape)
    bp = _rows_of(call, bias, "bias", x.dtype, weight.shape[:-1])
    layer = LinearLayer(E, in_dim, out_dim, TYPES[x.dtype], wp, bp)
    n = int(x.shape[0]) * int(slots_per_row)
    rows = LinearRows(n, xp, xs, int(slots_per_row), None, None, 0)
    if bins is not None:
        rows.bin_offset = _rows_of(call, bins.bin_offset, "bin_offset", torch.int32, (E + 1,))
        rows.perm = _rows_of(call, bins.perm, "perm", torch.int32, None)
        rows.perm_capacity = bins.capacity
    return layer, rows, n


def _epilogue(activation, leaky_slope, out_type):
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    if (activation == "leaky_relu") != (leaky_slope is not None):
        raise ValueError("leaky_slope goes with activation 'leaky_relu'")
    return LinearEpilogue(ACTIVATIONS[activation], float(leaky_slope or 0.0), out_type, None, 0,
                          None, 0)


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
           residual: Optional[torch.Tensor] = None, activation: str = "none",
           leaky_slope: Optional[float] = None, bins: Optional[Bins] = None,
           slots_per_row: int = 1, out: Optional[torch.Tensor] = None,
           out_dtype: Optional[torch.dtype] = None, pre: Optional[torch.Tensor] = None,
           stream=None) -> torch.Tensor:
    """ntc_linear: act(x weight^T + bias) + residual in one kernel, rows of x float16 or
    bfloat16 with any row stride, output rows of that dtype or float32.  With `bins`
    (build_bins of the slots' expert ids) weight is [experts][out][in], slot s reads row
    s // slots_per_row of x and writes row s; rows of slots in no bin are left as they
    are.  pre (x's dtype), if given, receives x weight^T + bias for linear_backward."""
    call = _Call(stream, x)
    layer, rows, n = _layer(call, x, weight, bias, bins, slots_per_row)
    if out is not None and out_dtype is None:
        out_dtype = out.dtype
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's dtype or float32")
    shape = (n, layer.out_dim)
    ep = _epilogue(activation, leaky_slope, TYPES[out_dtype])
    ep.residual, ep.residual_stride = call.take(residual, "residual", out_dtype, shape)
    ep.pre, ep.pre_stride = call.take(pre, "pre", x.dtype, shape)
    if out is None:
        out = call.empty(shape, out_dtype)
    yp, ys = call.take(out, "out", out_dtype, shape)
    layer, rows = ctypes.byref(layer), ctypes.byref(rows)
    size = lib().ntc_linear_workspace_bytes(layer, rows)
    ws, wp = call.workspace(size)
    call.run("ntc_linear", layer, rows, ctypes.byref(ep), yp, ys, wp, size)
    return out


@dataclass
class LinearGrads:
    x: Optional[torch.Tensor]       # [rows][in], x's dtype
    weight: Optional[torch.Tensor]  # weight's shape
    bias: Optional[torch.Tensor]    # weight's shape without in


def linear_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor,
                    pre: Optional[torch.Tensor] = None, activation: str = "none",
                    leaky_slope: Optional[float] = None, bins: Optional[Bins] = None,
                    slots_per_row: int = 1, input_grad: bool = True, weight_grad: bool = True,
                    bias_grad: bool = True, grad_dtype: Optional[torch.dtype] = None,
                    stream=None) -> LinearGrads:
    """ntc_linear_backward: gradients of linear's input, weight and bias from dy (x's dtype
    or float32); pre as linear wrote it (not needed for activation 'none').  Weight and
    bias gradients in x's dtype or float32 (grad_dtype).  A residual's gradient is dy."""
    call = _Call(stream, dy)
    layer, rows, n = _layer(call, x, weight, None, bins, slots_per_row)
    ep = _epilogue(activation, leaky_slope, layer.type)
    shape = (n, layer.out_dim)
    if activation != "none":
        if pre is None:
            raise ValueError("activation's gradient needs pre")
        ep.pre, ep.pre_stride = call.take(pre, "pre", x.dtype, shape)
    grad_dtype = x.dtype if grad_dtype is None else grad_dtype
    if grad_dtype not in (x.dtype, torch.float32):
        raise ValueError("grad_dtype must be x's dtype or float32")
    dyp, dys = call.take(dy, "dy", (x.dtype, torch.float32), shape)
    dx = call.empty(tuple(x.shape), x.dtype) if input_grad else None
    dw = call.empty(tuple(weight.shape), grad_dtype) if weight_grad else None
    db = call.empty(tuple(weight.shape[:-1]), grad_dtype) if bias_grad else None
    dxp, dxs = call.take(dx, "dx", x.dtype)
    g = LinearGradsArgs(dyp, dys, TYPES[dy.dtype], dxp, dxs,
                        None if dw is None else dw.data_ptr(),
                        None if db is None else db.data_ptr(), TYPES[grad_dtype])
    args = (ctypes.byref(layer), ctypes.byref(rows), ctypes.byref(ep), ctypes.byref(g))
    size = lib().ntc_linear_backward_workspace_bytes(*args)
    ws, wp = call.workspace(size)
    call.run("ntc_linear_backward", *args, wp, size)
    return LinearGrads(dx, dw, db)


def combine(rows: torch.Tensor, weights: Optional[torch.Tensor] = None,
            ids: Optional[torch.Tensor] = None, n_experts: Optional[int] = None,
            residual: Optional[torch.Tensor] = None, k: Optional[int] = None,
            out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """ntc_combine: out[t] = residual[t] + sum_j weights[t][j] rows[t k + j] over rows
    [n k][dim] of float32, float16 or bfloat16.  Without weights (then `k` is needed) the
    rows are added up; slots whose ids are not below n_experts are skipped."""
    call = _Call(stream, rows)
    if rows.dim() != 2:
        raise ValueError("rows must be [n k][dim]")
    n, k = _slots(rows, weights, ids, n_experts, k)
    dim = int(rows.shape[1])
    rp, rs = call.take(rows, "rows", TYPES)
    wp = _rows_of(call, weights, "weights", torch.float32, (n, k))
    ip = _rows_of(call, ids, "ids", torch.int32, (n, k))
    sp, ss = call.take(residual, "residual", rows.dtype, (n, dim))
    if out is None:
        out = call.empty((n, dim), rows.dtype)
    op, os_ = call.take(out, "out", rows.dtype, (n, dim))
    call.run("ntc_combine", rp, rs, TYPES[rows.dtype], n, k, dim, wp, ip,
             _int32(n_experts or 0, "n_experts"), sp, ss, op, os_)
    return out


def combine_backward(dout: torch.Tensor, rows: torch.Tensor,
                     weights: Optional[torch.Tensor] = None, ids: Optional[torch.Tensor] = None,
                     n_experts: Optional[int] = None, k: Optional[int] = None,
                     rows_grad: bool = True, weights_grad: bool = True, stream=None):
    """ntc_combine_backward: (gradient of the rows, gradient of the weights), None where not
    wanted; skipped slots get 0.  A residual's gradient is dout."""
    call = _Call(stream, rows)
    if rows.dim() != 2:
        raise ValueError("rows must be [n k][dim]")
    n, k = _slots(rows, weights, ids, n_experts, k)
    dim = int(rows.shape[1])
    dp, ds = call.take(dout, "dout", rows.dtype, (n, dim))
    rp, rs = call.take(rows, "rows", TYPES)
    wp = _rows_of(call, weights, "weights", torch.float32, (n, k))
    ip = _rows_of(call, ids, "ids", torch.int32, (n, k))
    drows = call.empty((n * k, dim), rows.dtype) if rows_grad else None
    dweights = call.empty((n, k), torch.float32) if weights_grad else None
    op, os_ = call.take(drows, "drows", rows.dtype)
    gp, _ = call.take(dweights, "dweights", torch.float32)
    call.run("ntc_combine_backward", dp, ds, rp, rs, TYPES[rows.dtype], n, k, dim, wp, ip,
             _int32(n_experts or 0, "n_experts"), op, os_, gp)
    return drows, dweights


def _slots(rows, weights, ids, n_experts, k):
    """(n, k) of rows [n k][dim]."""
    given = weights if weights is not None else ids
    if given is not None:
        if given.dim() != 2 or (k is not None and int(k) != given.shape[1]):
            raise ValueError("weights and ids must be [n][k]")
        n, k = given.shape
    elif k is None or int(k) < 1 or rows.shape[0] % int(k):
        raise ValueError("rows must hold k slots of every item")
    else:
        n = rows.shape[0] // int(k)
    if rows.shape[0] != n * int(k):
        raise ValueError("rows must hold k slots of every item")
    if ids is not None and n_experts is None:
        raise ValueError("ids need n_experts")
    return int(n), _int32(k, "k")
