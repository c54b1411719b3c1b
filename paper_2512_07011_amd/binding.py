"""ctypes binding of libbsfa.so (see include/bsfa.h).  Argument marshalling only: every step of
the attention path runs inside the library's HIP kernels.  PyTorch supplies device memory and
the current stream; there is no fallback — if the library is missing or a call fails, this
module raises."""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbsfa.so")

BSFA_OK = 0
STATUS_NAMES = {0: "BSFA_OK", -1: "BSFA_ERR_NULL", -2: "BSFA_ERR_SHAPE", -3: "BSFA_ERR_DTYPE",
                -4: "BSFA_ERR_UNSUPPORTED", -5: "BSFA_ERR_WORKSPACE", -6: "BSFA_ERR_HIP"}
EXPORTS = ["bsfa_forward", "bsfa_forward_workspace_bytes", "bsfa_calibrate", "bsfa_calibrate_noalloc",
           "bsfa_calibrate_noalloc_max_values", "bsfa_calibrate_topk",
           "bsfa_calibrate_workspace_bytes", "bsfa_query_build", "bsfa_cache_append", "bsfa_paged_attention",
           "bsfa_prefix_attention", "bsfa_paged_workspace_bytes",
           "bsfa_mfma_rate_probe", "bsfa_mfma_rate_probe_sink_bytes", "bsfa_mfma_rate_probe_flops",
           "bsfa_status_string", "bsfa_last_error"]


DTYPES = {torch.bfloat16: 0, torch.float16: 1}       # bsfa_dtype


def _same_16bit(name, *ts):
    if ts[0].dtype not in DTYPES or any(t.dtype != ts[0].dtype for t in ts):
        raise TypeError("%s: tensors must all be bfloat16 or all float16" % name)


class BsfaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, str(status)), message))
        self.status = status


class bsfa_problem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "n_q_heads", "n_kv_heads", "seqlen", "head_dim", "block_m", "block_n")] + \
               [(n, ctypes.c_int64) for n in
                ("q_stride_b", "q_stride_n", "q_stride_h", "k_stride_b", "k_stride_n", "k_stride_h",
                 "v_stride_b", "v_stride_n", "v_stride_h", "o_stride_b", "o_stride_n", "o_stride_h")] + \
               [("dtype", ctypes.c_int32), ("thresholds_per_tile", ctypes.c_int32),
                ("threshold_tiles", ctypes.c_int32), ("seqlens", ctypes.c_void_p),
                ("single_head_groups", ctypes.c_int32), ("gate_mode", ctypes.c_int32), ("qk_fp8", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_int64)]


class bsfa_skip_stats(ctypes.Structure):
    _fields_ = [("counts", ctypes.c_void_p), ("skip_mask", ctypes.c_void_p), ("block_max", ctypes.c_void_p),
                ("lse", ctypes.c_void_p)]


class bsfa_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")] + \
               [(n, ctypes.c_int64) for n in ("k_stride_page", "k_stride_n", "k_stride_h", "v_stride_page", "v_stride_n", "v_stride_h")] + \
               [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]


class bsfa_append(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_q_heads", "seqlen")] + \
               [("%s_stride_%s" % (t, x), ctypes.c_int64) for t in ("q", "k", "v", "qo", "ko") for x in "bnh"] + \
               [("seqlens", ctypes.c_void_p), ("start", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
                ("table_stride_b", ctypes.c_int64), ("table_pages", ctypes.c_int32), ("cos_sin", ctypes.c_void_p),
                ("n_positions", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class bsfa_paged(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "n_q_heads", "seqlen")] + \
               [("%s_stride_%s" % (t, x), ctypes.c_int64) for t in "qo" for x in "bnh"] + \
               [("q_lens", ctypes.c_void_p), ("cache_lens", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
                ("table_stride_b", ctypes.c_int64), ("table_pages", ctypes.c_int32), ("max_cache_len", ctypes.c_int32),
                ("prefix_table", ctypes.c_void_p), ("prefix_len", ctypes.c_int32), ("prefix_pages", ctypes.c_int32),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """Opens libbsfa.so (built in-tree by build.build_lib / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                "%s is missing: build it with `python -m paper_2512_07011_amd.build` "
                "(there is no fallback path)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp = ctypes.c_void_p
        L.bsfa_forward.restype = ctypes.c_int
        L.bsfa_forward.argtypes = [ctypes.POINTER(bsfa_problem), vp, vp, vp, vp, ctypes.c_int, vp,
                                   ctypes.POINTER(bsfa_skip_stats), vp]
        L.bsfa_calibrate.restype = ctypes.c_int
        L.bsfa_calibrate.argtypes = [ctypes.POINTER(bsfa_problem), vp, vp, ctypes.c_int,
                                     ctypes.POINTER(ctypes.c_float), ctypes.c_int,
                                     ctypes.POINTER(ctypes.c_float), vp, ctypes.c_size_t, vp]
        L.bsfa_calibrate_noalloc.restype = ctypes.c_int
        L.bsfa_calibrate_noalloc.argtypes = [ctypes.POINTER(bsfa_problem), vp, vp, ctypes.c_int,
                                             ctypes.POINTER(ctypes.c_float), ctypes.c_int, vp, vp]
        L.bsfa_calibrate_noalloc_max_values.restype = ctypes.c_size_t
        L.bsfa_calibrate_noalloc_max_values.argtypes = []
        L.bsfa_calibrate_topk.restype = ctypes.c_int
        L.bsfa_calibrate_topk.argtypes = [ctypes.POINTER(bsfa_problem), vp, vp, ctypes.c_int,
                                          ctypes.POINTER(ctypes.c_int32), ctypes.c_int, ctypes.c_int,
                                          ctypes.POINTER(ctypes.c_float), vp, ctypes.c_size_t, vp]
        L.bsfa_calibrate_workspace_bytes.restype = ctypes.c_size_t
        L.bsfa_calibrate_workspace_bytes.argtypes = [ctypes.POINTER(bsfa_problem)]
        L.bsfa_forward_workspace_bytes.restype = ctypes.c_size_t
        L.bsfa_forward_workspace_bytes.argtypes = [ctypes.POINTER(bsfa_problem)]
        i32p = ctypes.POINTER(ctypes.c_int32)
        L.bsfa_query_build.restype = ctypes.c_int
        L.bsfa_query_build.argtypes = [i32p, i32p, i32p, ctypes.c_int]
        L.bsfa_mfma_rate_probe.restype = ctypes.c_int
        L.bsfa_mfma_rate_probe.argtypes = [vp, vp, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, vp]
        L.bsfa_mfma_rate_probe_sink_bytes.restype = ctypes.c_size_t
        L.bsfa_mfma_rate_probe_sink_bytes.argtypes = [ctypes.c_int]
        L.bsfa_mfma_rate_probe_flops.restype = ctypes.c_double
        L.bsfa_mfma_rate_probe_flops.argtypes = [ctypes.c_int, ctypes.c_int]
        L.bsfa_cache_append.restype = ctypes.c_int
        L.bsfa_cache_append.argtypes = [vp] * 8
        for f in (L.bsfa_paged_attention, L.bsfa_prefix_attention):
            f.restype = ctypes.c_int
            f.argtypes = [vp, vp, vp, ctypes.c_int, vp, vp, vp]
        L.bsfa_paged_workspace_bytes.restype = ctypes.c_size_t
        L.bsfa_paged_workspace_bytes.argtypes = [vp, vp]
        L.bsfa_status_string.restype = ctypes.c_char_p
        L.bsfa_status_string.argtypes = [ctypes.c_int]
        L.bsfa_last_error.restype = ctypes.c_char_p
        L.bsfa_last_error.argtypes = []
        _lib = L
    return _lib


def _check(status: int):
    if status != BSFA_OK:
        raise BsfaError(status, lib().bsfa_last_error().decode())


def make_problem(q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor], out: Optional[torch.Tensor],
                 block_m: int, block_n: int, thresholds_per_tile: bool = False, threshold_tiles: int = 0,
                 seqlens: Optional[torch.Tensor] = None, single_head_groups: bool = False) -> bsfa_problem:
    """Descriptor for [B, N, H, d] views (any strides with a contiguous last dimension)."""
    B, N, Hq, d = q.shape
    qs, ks = q.stride(), k.stride()
    vs, os_ = v.stride() if v is not None else ks, out.stride() if out is not None else qs
    if qs[3] != 1 or ks[3] != 1 or vs[3] != 1 or os_[3] != 1:
        name = "qkvo"[[t[3] != 1 for t in (qs, ks, vs, os_)].index(True)]
        raise ValueError("%s: head dimension must be contiguous" % name)
    # (members in order; one call: setting them one by one is a quarter of a small forward call's host time)
    p = bsfa_problem(B, Hq, k.shape[2], N, d, block_m, block_n, *qs[:3], *ks[:3], *vs[:3], *os_[:3], DTYPES[q.dtype],
                     int(thresholds_per_tile), int(threshold_tiles), None, int(bool(single_head_groups)))
    if seqlens is not None:
        if seqlens.dtype != torch.int32 or not seqlens.is_contiguous() or tuple(seqlens.shape) != (B,) or not seqlens.is_cuda:
            raise TypeError("bsfa: seqlens must be a contiguous int32 GPU tensor of shape [batch]")
        p.seqlens = seqlens.data_ptr()
    return p


def n_tiles(n: int, block: int) -> int:
    """Query tiles / key blocks of a sequence of n tokens (the last one may be partial)."""
    return -(-n // block)


@dataclass
class SkipStats:
    counts: Optional[torch.Tensor] = None      # [B, Hq, 3] int64: skipped, gateable, reachable
    skip_mask: Optional[torch.Tensor] = None   # [B, Hq, M_Q, ceil(M_KV/32)] int32 bit mask
    block_max: Optional[torch.Tensor] = None   # [B, Hq, M_Q, M_KV] fp32, NaN where not gateable
    lse: Optional[torch.Tensor] = None         # [B, N, Hq] fp32, log-sum-exp over the kept blocks


def alloc_stats(q: torch.Tensor, block_m: int, block_n: int, counts=True, skip_mask=False, block_max=False,
                lse=False) -> SkipStats:
    B, N, Hq, _ = q.shape
    mq, mkv = n_tiles(N, block_m), n_tiles(N, block_n)
    s = SkipStats()
    if counts:
        s.counts = torch.empty(B, Hq, 3, dtype=torch.int64, device=q.device)
    if skip_mask:
        s.skip_mask = torch.empty(B, Hq, mq, (mkv + 31) // 32, dtype=torch.int32, device=q.device)
    if block_max:
        s.block_max = torch.empty(B, Hq, mq, mkv, dtype=torch.float32, device=q.device)
    if lse:
        s.lse = torch.empty(B, N, Hq, dtype=torch.float32, device=q.device)
    return s


def _scratch(nbytes: int, device, stream) -> torch.Tensor:
    """Scratch memory of one call, from torch's allocator on the stream that the call's kernels run on: dropped
    after the launch, it is handed out again only to later work of that stream, so calls on other streams, from other
    threads or in a captured graph (whose allocations stay in the graph's own pool) never write into it."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def forward_workspace_bytes(q: torch.Tensor, k: torch.Tensor, block_m: int = 128, block_n: int = 64,
                            qk_fp8: bool = False) -> int:
    """Bytes of workspace bsfa_forward can use for these shapes (0: no call of that shape uses one)."""
    p = make_problem(q, k, None, None, block_m, block_n)
    p.qk_fp8 = int(bool(qk_fp8))
    return int(lib().bsfa_forward_workspace_bytes(ctypes.byref(p)))


def _dev_check(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("bsfa: tensors must live on the GPU")


def _raw_stream(stream, device) -> int:
    """hipStream_t of ``stream``, or of torch's current stream on ``device`` (asked for without building a
    stream object where this torch can: 0.2 us instead of 1.9)."""
    if stream is not None:
        return stream.cuda_stream
    try:
        return torch._C._cuda_getCurrentRawStream(device.index)
    except AttributeError:                     # (no public name)
        return torch.cuda.current_stream(device).cuda_stream


def bsfa_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, thresholds: torch.Tensor,
                 causal: bool = True, out: Optional[torch.Tensor] = None,
                 skip_stats: Optional[SkipStats] = None, block_m: int = 128, block_n: int = 64,
                 stream: Optional[torch.cuda.Stream] = None,
                 seqlens: Optional[torch.Tensor] = None, single_head_groups: bool = False,
                 workspace=True, gate_mode: int = 0, qk_fp8: bool = False) -> torch.Tensor:
    """out = block-sparse attention of bf16 (or fp16) q [B,N,Hq,d], k, v [B,N,Hkv,d]; thresholds fp32 on the
    GPU, [Hq] or [Hq, T] (T tiles calibrated; later tiles use the last one).  ``seqlens`` (int32
    GPU tensor [B], causal only) gives each batch element its own length.  ``workspace``: a uint8
    GPU tensor of at least forward_workspace_bytes(...) bytes (calls that overlap need one each), True
    (scratch memory of the call's own, from torch's allocator) or False/None (no workspace: V is read
    in place).  ``gate_mode`` 1 selects the running-maximum comparison predicate (thresholds then hold its lambda).  Enqueues on ``stream`` (default:
    torch's current stream)."""
    _dev_check(q, k, v, thresholds, out)
    if out is None:
        _same_16bit("bsfa_forward", q, k, v)
    else:
        _same_16bit("bsfa_forward", q, k, v, out)
    if thresholds.dtype != torch.float32 or not thresholds.is_contiguous():
        raise TypeError("bsfa_forward: thresholds must be contiguous float32")
    _, _, Hq, _ = q.shape
    ts = thresholds.shape
    per_tile = len(ts) == 2
    if len(ts) not in (1, 2) or ts[0] != Hq or (per_tile and ts[1] < 1):
        raise ValueError("bsfa_forward: thresholds shape %s, expected [Hq] or [Hq, tiles]" % (tuple(ts),))
    if out is None:
        out = torch.empty_like(q)
    L = lib()
    p = make_problem(q, k, v, out, block_m, block_n, per_tile, ts[1] if per_tile else 0, seqlens, single_head_groups)
    p.gate_mode = int(gate_mode)
    p.qk_fp8 = int(bool(qk_fp8))
    pref = ctypes.byref(p)
    if workspace is True:
        need = L.bsfa_forward_workspace_bytes(pref)
        workspace = _scratch(need, q.device, stream) if need else None
    if workspace is not None and workspace is not False:
        _dev_check(workspace)
        p.workspace = workspace.data_ptr()
        p.workspace_bytes = workspace.numel() * workspace.element_size()
    st = None
    if skip_stats is not None:
        st = ctypes.byref(bsfa_skip_stats(*[None if t is None else t.data_ptr() for t in (
            skip_stats.counts, skip_stats.skip_mask, skip_stats.block_max, skip_stats.lse)]))
    rc = L.bsfa_forward(pref, q.data_ptr(), k.data_ptr(), v.data_ptr(), thresholds.data_ptr(), 1 if causal else 0,
                        out.data_ptr(), st, _raw_stream(stream, q.device))
    if rc != BSFA_OK:
        _check(rc)
    return out


def bsfa_calibrate(q: torch.Tensor, k: torch.Tensor, target_skip_fractions: Sequence[float],
                   causal: bool = True, block_m: int = 128, block_n: int = 64,
                   workspace: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None,
                   seqlens: Optional[torch.Tensor] = None, qk_fp8: bool = False) -> torch.Tensor:
    """Per-head thresholds for each target skip fraction: CPU float32 tensor [n_levels, Hq]."""
    _dev_check(q, k, workspace)
    _same_16bit("bsfa_calibrate", q, k)
    p = make_problem(q, k, None, None, block_m, block_n, seqlens=seqlens)
    p.qk_fp8 = int(bool(qk_fp8))
    need = lib().bsfa_calibrate_workspace_bytes(ctypes.byref(p))
    if need == 0:
        _check(lib().bsfa_calibrate(ctypes.byref(p), q.data_ptr(), k.data_ptr(), int(bool(causal)), None, 0, None, None, 0, None))
    if workspace is None:
        workspace = _scratch(need, q.device, stream)
    n = len(target_skip_fractions)
    fr = (ctypes.c_float * n)(*[float(f) for f in target_skip_fractions])
    outp = (ctypes.c_float * (n * q.shape[2]))()
    s = stream if stream is not None else torch.cuda.current_stream(q.device)
    _check(lib().bsfa_calibrate(ctypes.byref(p), q.data_ptr(), k.data_ptr(), int(bool(causal)), fr, n, outp,
                                workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                ctypes.c_void_p(s.cuda_stream)))
    return torch.frombuffer(outp, dtype=torch.float32).clone().view(n, q.shape[2])


def bsfa_calibrate_noalloc(q: torch.Tensor, k: torch.Tensor, target_skip_fractions: Sequence[float],
                           thresholds_out: torch.Tensor, causal: bool = True, block_m: int = 128, block_n: int = 64,
                           stream: Optional[torch.cuda.Stream] = None,
                           seqlens: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bsfa_calibrate without allocations: the thresholds go to ``thresholds_out``, a contiguous
    float32 GPU tensor [n_levels, Hq] the caller provides; kernels are only enqueued."""
    _dev_check(q, k, thresholds_out)
    _same_16bit("bsfa_calibrate_noalloc", q, k)
    n = len(target_skip_fractions)
    if thresholds_out.dtype != torch.float32 or not thresholds_out.is_contiguous() or tuple(thresholds_out.shape) != (n, q.shape[2]):
        raise TypeError("bsfa_calibrate_noalloc: thresholds_out must be contiguous float32 [n_levels, Hq]")
    p = make_problem(q, k, None, None, block_m, block_n, seqlens=seqlens)
    fr = (ctypes.c_float * n)(*[float(f) for f in target_skip_fractions])
    s = stream if stream is not None else torch.cuda.current_stream(q.device)
    _check(lib().bsfa_calibrate_noalloc(ctypes.byref(p), q.data_ptr(), k.data_ptr(), int(bool(causal)), fr, n,
                                        thresholds_out.data_ptr(), ctypes.c_void_p(s.cuda_stream)))
    return thresholds_out


def mfma_rate_probe(operands: torch.Tensor, workgroups: int, iters: int, sink: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> float:
    """Enqueues the matrix-instruction rate probe (measurement utility) on ``operands`` (4096 float32 values on
    the GPU) and returns the floating-point operations it performs; the caller times it with events."""
    if not operands.is_cuda or operands.dtype != torch.float32 or not operands.is_contiguous() or operands.numel() < 4096:
        raise TypeError("mfma_rate_probe: operands must be a contiguous float32 GPU tensor of at least 4096 values")
    need = lib().bsfa_mfma_rate_probe_sink_bytes(int(workgroups))
    if sink is None:
        sink = _scratch(max(need, 4), operands.device, stream)
    s = stream if stream is not None else torch.cuda.current_stream(operands.device)
    _check(lib().bsfa_mfma_rate_probe(operands.data_ptr(), sink.data_ptr(), sink.numel() * sink.element_size(),
                                      int(workgroups), int(iters), ctypes.c_void_p(s.cuda_stream)))
    return float(lib().bsfa_mfma_rate_probe_flops(int(workgroups), int(iters)))


def bsfa_calibrate_topk(samples, ks: Sequence[int], causal: bool = True, block_m: int = 128, block_n: int = 64,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Per-query-tile thresholds for each sparsity level k (number of retained gateable blocks),
    averaged over the calibration samples: CPU float32 tensor [n_levels, Hq, ceil(N/block_m)].
    ``samples`` is a list of (q, k) pairs of equal shape; every batch element is one sample."""
    n = len(ks)
    out = None
    ws = None
    done = 0
    kk = (ctypes.c_int32 * n)(*[int(x) for x in ks])
    for q, k in samples:
        _dev_check(q, k)
        _same_16bit("bsfa_calibrate_topk", q, k)
        p = make_problem(q, k, None, None, block_m, block_n)
        need = lib().bsfa_calibrate_workspace_bytes(ctypes.byref(p))
        if ws is None or ws.numel() < need:
            ws = _scratch(max(need, 1), q.device, stream)
        if out is None:
            out = (ctypes.c_float * (n * q.shape[2] * n_tiles(q.shape[1], block_m)))()
        s = stream if stream is not None else torch.cuda.current_stream(q.device)
        _check(lib().bsfa_calibrate_topk(ctypes.byref(p), q.data_ptr(), k.data_ptr(), int(bool(causal)), kk, n, done,
                                         out, ws.data_ptr(), ws.numel(), ctypes.c_void_p(s.cuda_stream)))
        done += q.shape[0]
    q0 = samples[0][0]
    return torch.frombuffer(out, dtype=torch.float32).clone().view(n, q0.shape[2], n_tiles(q0.shape[1], block_m))


# ---- paged K/V cache ---------------------------------------------------------------------------------------
def alloc_cache(n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda"):
    """Keys and values of a paged cache, [n_pages, page_size, n_kv_heads, head_dim] each; a head's tokens lie together in
    a page.  (The entry points take any other order with a contiguous last dimension as well.)"""
    return tuple(torch.empty(n_pages, n_kv_heads, page_size, head_dim, dtype=dtype, device=device).transpose(1, 2) for _ in "kv")


def rotary_table(n_positions: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """[n_positions, rot_dim] fp32: of every position the cosines of its rot_dim / 2 angles
    position * base ** (-2 i / rot_dim), then their sines.  The angles are taken in 64 bits."""
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rotary_table: rot_dim must be positive and even, is %d" % rot_dim)
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


# The descriptors as they lie in memory, filled in one go (a tenth of a ctypes.Structure's time; a small call's is the
# host's): the members of bsfa_cache, bsfa_append and bsfa_paged in order.
_PACK_CACHE = struct.Struct("@5i6q2P").pack
_PACK_APPEND = struct.Struct("@3i15q3PqiP3i").pack
_PACK_PAGED = struct.Struct("@3i6q3Pq2iP2iPq").pack


def _same_device(name, q, *ts):
    d = q.get_device()
    if d < 0:
        raise ValueError("bsfa: tensors must live on the GPU")
    for t in ts:
        if t is not None and t.get_device() != d:
            raise ValueError("%s: tensors must live on one GPU" % name)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device     # (0.1 us less; no public name)


def _on_device(device, stream, call, *args):
    """call(*args, stream) with `device` current: the kernels of a stream are launched from its own device."""
    if stream is not None and stream.device != device:
        raise ValueError("bsfa: the stream must be one of the tensors' GPU")
    if device.index == _current_device():
        rc = call(*args, _raw_stream(stream, device))
    else:
        with torch.cuda.device(device):
            rc = call(*args, _raw_stream(stream, device))
    if rc:
        _check(rc)


def _lens(name, t, n):
    """Address of a contiguous int32 tensor of n elements."""
    if t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous():
        raise TypeError("%s must be contiguous int32 of shape [%d]" % (name, n))
    return t.data_ptr()


def _pages(name, t, n):
    """Address, row stride and row length of an int32 tensor of n rows, contiguous in its last dimension."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not torch.int32 or len(shape) != 2 or shape[0] != n or (stride[1] != 1 and shape[1] > 1):
        raise TypeError("%s must be int32 [%d, pages], contiguous in its last dimension" % (name, n))
    return t.data_ptr(), stride[0], shape[1]


def _strides(name, t, shape):
    """Strides of a [B, N, H, d] tensor (batch, token, head)."""
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, list(t.shape), list(shape)))
    stride = t.stride()
    if stride[3] != 1:
        raise ValueError("%s: head dimension must be contiguous" % name)
    return stride[:3]


def _cache(name, k_cache, v_cache):
    """Descriptor of the cache, its shape and its type."""
    shape, dtype = k_cache.shape, k_cache.dtype
    if len(shape) != 4 or dtype not in DTYPES or v_cache.dtype is not dtype:
        raise TypeError("%s: k_cache and v_cache must be [n_pages, page_size, n_kv_heads, head_dim], both bfloat16 or both float16" % name)
    ks, vs = k_cache.stride(), v_cache.stride()
    if v_cache.shape != shape or ks[3] != 1 or vs[3] != 1:
        _strides("k_cache", k_cache, shape), _strides("v_cache", v_cache, shape)         # (raises)
    return _PACK_CACHE(*shape, DTYPES[dtype], *ks[:3], *vs[:3], k_cache.data_ptr(), v_cache.data_ptr()), shape, dtype


def bsfa_cache_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                      block_table: torch.Tensor, start: torch.Tensor, cos_sin: Optional[torch.Tensor] = None,
                      seqlens: Optional[torch.Tensor] = None, interleaved: bool = False, q_out: Optional[torch.Tensor] = None,
                      k_out=None, stream: Optional[torch.cuda.Stream] = None):
    """Appends the new tokens k, v [B,N,Hkv,d] to the paged cache [n_pages, page_size, Hkv, d]: element b's token i goes to
    position start[b] + i, that is to page block_table[b, position // page_size].  ``cos_sin`` (fp32 [positions, rot_dim],
    see rotary_table; at least as many positions as a row of the table holds) rotates keys and queries by their positions;
    without it q must be None.  ``seqlens`` (int32 GPU tensor [B]) gives each element its own number of new tokens: rows
    behind it are left alone.  ``interleaved``: adjacent elements are a pair, not halves.
    Returns the rotated queries (``q_out``, which may be q; None without q) and, where ``k_out`` is True or a tensor, the
    rotated keys: what bsfa_forward takes for a prompt; else None.  Enqueues on ``stream`` (default: torch's current
    stream)."""
    name = "bsfa_cache_append"
    if k_out is True or k_out is False:
        k_out = _empty_like(k, stream) if k_out else None
    _same_device(name, k, q, v, k_cache, v_cache, block_table, start, cos_sin, seqlens, q_out, k_out)
    c, (_, _, Hkv, d), dtype = _cache(name, k_cache, v_cache)
    shape = k.shape
    if len(shape) != 4 or shape[2] != Hkv or shape[3] != d:
        raise ValueError("%s: k has shape %s, expected [B, N, %d, %d]" % (name, list(shape), Hkv, d))
    if k.dtype is not dtype or v.dtype is not dtype or (k_out is not None and k_out.dtype is not dtype):
        raise TypeError("%s: tensors and cache must be of one type" % name)
    ks, vs = k.stride(), v.stride()
    if v.shape != shape or ks[3] != 1 or vs[3] != 1:
        _strides("k", k, shape), _strides("v", v, shape)                                 # (raises)
    B, N, Hq = shape[0], shape[1], Hkv
    qs = qos = kos = (0, 0, 0)
    q_ptr = qo_ptr = ko_ptr = cs_ptr = positions = rot = 0
    if q is not None:
        if cos_sin is None:
            raise ValueError("%s: q without cos_sin: nothing would be done to it" % name)
        q_shape = q.shape
        if len(q_shape) != 4 or q_shape[0] != B or q_shape[1] != N or q_shape[3] != d:
            raise ValueError("%s: q has shape %s, expected [%d, %d, Hq, %d]" % (name, list(q_shape), B, N, d))
        if q_out is None:
            q_out = _empty_like(q, stream)
        if q.dtype is not dtype or q_out.dtype is not dtype:
            raise TypeError("%s: tensors and cache must be of one type" % name)
        Hq = q_shape[2]
        qs, qos = q.stride(), q_out.stride()
        if q_out.shape != q_shape or qs[3] != 1 or qos[3] != 1:
            _strides("q", q, q_shape), _strides("q_out", q_out, q_shape)                 # (raises)
        q_ptr, qo_ptr = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("%s: q_out without q" % name)
    if k_out is not None:
        kos, ko_ptr = _strides("k_out", k_out, shape), k_out.data_ptr()
    if cos_sin is not None:
        if cos_sin.dtype is not torch.float32 or cos_sin.dim() != 2 or not cos_sin.is_contiguous():
            raise TypeError("%s: cos_sin must be contiguous float32 [positions, rot_dim]" % name)
        (positions, rot), cs_ptr = cos_sin.shape, cos_sin.data_ptr()
    table, table_stride, pages = _pages("block_table", block_table, B)
    p = _PACK_APPEND(B, Hq, N, *qs[:3], *ks[:3], *vs[:3], *qos[:3], *kos,
                     0 if seqlens is None else _lens("seqlens", seqlens, B), _lens("start", start, B), table, table_stride, pages,
                     cs_ptr, positions, rot, 1 if interleaved else 0)
    device = k.device
    _on_device(device, stream, lib().bsfa_cache_append, c, p, q_ptr, k.data_ptr(), v.data_ptr(), qo_ptr, ko_ptr)
    return q_out, k_out


def _empty_like(t, stream):
    if stream is None:
        return torch.empty(t.shape, dtype=t.dtype, device=t.device)
    with torch.cuda.stream(stream):
        return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _attend(call, name, q, k_cache, v_cache, prefix_table, prefix_len, block_table, cache_lens, q_lens, causal, out, lse, max_cache_len, workspace,
            stream):
    """The two entry points' common part; call None: the bytes of workspace they need."""
    _same_device(name, q, k_cache, v_cache, prefix_table, block_table, cache_lens, q_lens, out, lse)
    c, (_, _, _, d), dtype = _cache(name, k_cache, v_cache)
    shape = q.shape
    if len(shape) != 4 or shape[3] != d:
        raise ValueError("%s: q has shape %s, expected [B, N, Hq, %d]" % (name, list(shape), d))
    if out is None:
        out = _empty_like(q, stream)
    if q.dtype is not dtype or out.dtype is not dtype:
        raise TypeError("%s: tensors and cache must be of one type" % name)
    B, N, Hq, _ = shape
    lse_ptr = prefix = pages_p = 0
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.shape != (B, N, Hq) or not lse.is_contiguous():
            raise TypeError("%s: lse must be contiguous float32 [B, N, Hq]" % name)
        lse_ptr = lse.data_ptr()
    if prefix_table is not None:
        pages_p = prefix_table.numel()
        prefix = _lens("prefix_table", prefix_table, pages_p)
    table, table_stride, pages = _pages("block_table", block_table, B)
    qs, os_ = q.stride(), out.stride()
    if out.shape != shape or qs[3] != 1 or os_[3] != 1:
        _strides("q", q, shape), _strides("out", out, shape)                             # (raises)
    if call is None:
        os_ = (N * Hq * d, Hq * d, d)                        # (`out` stands for a result of q's shape: q itself may repeat)
    members = (B, Hq, N, *qs[:3], *os_[:3], 0 if q_lens is None else _lens("q_lens", q_lens, B),
               _lens("cache_lens", cache_lens, B), table, table_stride, pages, max_cache_len, prefix, prefix_len, pages_p)
    ws_ptr = ws_bytes = 0
    if workspace is True or call is None:
        ws_bytes = lib().bsfa_paged_workspace_bytes(c, _PACK_PAGED(*members, 0, 0))
        if call is None:
            return ws_bytes
        if ws_bytes:
            workspace = _scratch(ws_bytes, q.device, stream)
            ws_ptr = workspace.data_ptr()
    elif workspace is not None and workspace is not False:
        _same_device(name, q, workspace)
        if not workspace.is_contiguous():
            raise TypeError("%s: workspace must be contiguous" % name)
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    device = q.device
    _on_device(device, stream, call, c, _PACK_PAGED(*members, ws_ptr, ws_bytes), q.data_ptr(), 1 if causal else 0, out.data_ptr(), lse_ptr)
    return out


def bsfa_paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
                         cache_lens: torch.Tensor, q_lens: Optional[torch.Tensor] = None, causal: bool = True,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, max_cache_len: int = 0,
                         workspace=True, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out = attention of the new tokens q [B,N,Hq,d] over a paged cache [n_pages, page_size, Hkv, d]: element b's
    cache_lens[b] tokens (int32 GPU tensor [B]) lie in the pages of block_table[b] (int32), its new tokens are the last
    q_lens[b] of them (default N; rows behind that are left alone) and see, if ``causal``, the places up to their own, else
    all.  ``lse``: fp32 [B,N,Hq], written if given.  ``max_cache_len``: a bound of the lengths that the host may know.
    ``workspace``: a uint8 GPU tensor of paged_workspace_bytes(...) bytes (calls that overlap need one each), or True
    (scratch memory of the call's own).  Enqueues on ``stream`` (default: torch's current stream)."""
    return _attend(lib().bsfa_paged_attention, "bsfa_paged_attention", q, k_cache, v_cache, None, 0, block_table, cache_lens, q_lens, causal,
                   out, lse, max_cache_len, workspace, stream)


def bsfa_prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_table: torch.Tensor,
                          prefix_len: int, block_table: torch.Tensor, cache_lens: torch.Tensor,
                          q_lens: Optional[torch.Tensor] = None, causal: bool = True, out: Optional[torch.Tensor] = None,
                          lse: Optional[torch.Tensor] = None, max_cache_len: int = 0, workspace=True,
                          stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """bsfa_paged_attention for a batch whose elements share the ``prefix_len`` tokens in the pages of ``prefix_table``
    (int32 GPU tensor): every new token sees them, before its element's own, which alone block_table and cache_lens
    count.  The prefix is read once for the batch."""
    if prefix_table is None:
        raise TypeError("bsfa_prefix_attention: prefix_table is missing")
    return _attend(lib().bsfa_prefix_attention, "bsfa_prefix_attention", q, k_cache, v_cache, prefix_table, prefix_len, block_table, cache_lens,
                   q_lens, causal, out, lse, max_cache_len, workspace, stream)


def paged_workspace_bytes(q: torch.Tensor, k_cache: torch.Tensor, block_table: torch.Tensor, prefix_table: Optional[torch.Tensor] = None,
                          prefix_len: int = 0, max_cache_len: int = 0) -> int:
    """Bytes of workspace bsfa_paged_attention (with prefix_table: bsfa_prefix_attention) needs for these shapes."""
    lens = torch.empty(q.shape[0], dtype=torch.int32, device=q.device)
    return int(_attend(None, "paged_workspace_bytes", q, k_cache, k_cache, prefix_table, prefix_len, block_table, lens, None, True, q, None, max_cache_len,
                       True, None))


def bsfa_query_build():
    """List of (block_m, block_n, head_dim) triples the library was built for."""
    n = lib().bsfa_query_build(None, None, None, 0)
    bm, bn, hd = ((ctypes.c_int32 * n)() for _ in range(3))
    lib().bsfa_query_build(bm, bn, hd, n)
    return [(bm[i], bn[i], hd[i]) for i in range(n)]
