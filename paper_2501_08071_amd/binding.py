"""Thin Python binding of the C-ABI library (include/attn.h): argument marshalling only.

The entry points on torch tensors go through a small module of C++ (csrc/binding_fast.cpp) where the arguments are the usual
ones; the Python below it is for the rest, and says what is wrong with a call.

PyTorch supplies device memory and the stream; every step of the attention path runs inside
the HIP kernel.  There is no CPU or PyTorch fallback: if the shared library is missing the
import fails loudly.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os

# torch first: it carries its own copy of the HIP runtime (same soname as the system one), and the
# process must end up with ONE runtime that owns both torch's streams and this library's kernels
import torch

from . import build as _build

F16 = 0
BF16 = 1


class AttnError(RuntimeError):
    def __init__(self, status: int, msg: str, what: str = "attn_fwd"):
        super().__init__(f"{what} failed with status {status}: {msg}")
        self.status = status


class PagedCache(ctypes.Structure):
    """attn_paged_t of include/attn.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_longlong), ("n_pages", ctypes.c_int),
                ("page_size", ctypes.c_int), ("Hk", ctypes.c_int), ("D", ctypes.c_int), ("dtype", ctypes.c_int),
                ("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int), ("width", ctypes.c_int),
                ("cu_q", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("B", ctypes.c_int), ("T", ctypes.c_int)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(_build.LIB):
        try:
            _build.build_lib()
        except Exception as e:  # no compiler, or the build failed: there is nothing to fall back to
            raise ImportError(f"{_build.LIB} is missing and could not be built: {e}") from e
    lib = ctypes.CDLL(_build.LIB)
    vp = ctypes.c_void_p
    lib.attn_fwd.argtypes = [vp, vp, vp, vp, vp] + [ctypes.c_int] * 5 + [ctypes.c_float, ctypes.c_int, vp]
    lib.attn_fwd.restype = ctypes.c_int
    lib.attn_fwd_o16.argtypes = lib.attn_fwd.argtypes
    lib.attn_fwd_o16.restype = ctypes.c_int
    lib.attn_supported.argtypes = [ctypes.c_int] * 4
    lib.attn_supported.restype = ctypes.c_int
    lib.attn_status_str.argtypes = [ctypes.c_int]
    lib.attn_status_str.restype = ctypes.c_char_p
    lib.attn_kernel_name.argtypes = [ctypes.c_int] * 6
    lib.attn_kernel_name.restype = ctypes.c_char_p
    for f in (lib.attn_tile_rows, lib.attn_tile_keys):
        f.argtypes = [ctypes.c_int] * 3
        f.restype = ctypes.c_int
    for f in (lib.attn_launch_rows, lib.attn_workgroup_rows):
        f.argtypes = [ctypes.c_int] * 6
        f.restype = ctypes.c_int
    cache, ll, ci = ctypes.POINTER(PagedCache), ctypes.c_longlong, ctypes.c_int
    lib.attn_kv_append.argtypes = [cache, vp, vp, vp, ll, ll, ll, vp, vp, vp] + [ci] * 5 + [vp]
    lib.attn_kv_append.restype = ci
    lib.attn_paged_fwd.argtypes = [cache, vp, ll, vp, vp, vp] + [ci] * 4 + [ctypes.c_float, vp, ll, vp]
    lib.attn_paged_fwd.restype = ci
    lib.attn_paged_workspace.argtypes = [ci] * 8
    lib.attn_paged_workspace.restype = ll
    # include/probe.h
    lib.probe_mfma.argtypes = [vp] + [ctypes.c_int] * 4 + [vp]
    lib.probe_mfma.restype = ctypes.c_longlong
    lib.probe_softmax_valu.argtypes = [vp] + [ctypes.c_int] * 3 + [vp]
    lib.probe_softmax_valu.restype = ctypes.c_longlong
    lib.probe_l2_read.argtypes = [vp, vp] + [ctypes.c_int] * 3 + [vp]
    lib.probe_l2_read.restype = ctypes.c_longlong
    lib.probe_empty.argtypes = [ctypes.c_int, ctypes.c_int, vp]
    lib.probe_empty.restype = ctypes.c_int
    lib.probe_issue_share.argtypes = [vp] + [ctypes.c_int] * 4 + [vp]
    lib.probe_issue_share.restype = ctypes.c_int
    # include/rowops.h
    lib.softmax_rows_fwd.argtypes = [vp, vp, ctypes.c_longlong, ctypes.c_int, ctypes.c_int, vp]
    lib.softmax_rows_fwd.restype = ctypes.c_int
    lib.rmsnorm_fwd.argtypes = [vp, vp, vp, ctypes.c_longlong, ctypes.c_int, ctypes.c_float, ctypes.c_int, vp]
    lib.rmsnorm_fwd.restype = ctypes.c_int
    lib.residual_rmsnorm_fwd.argtypes = [vp] * 6 + [ctypes.c_longlong, ctypes.c_int, ctypes.c_float] + [ctypes.c_int] * 3 + [vp]
    lib.residual_rmsnorm_fwd.restype = ctypes.c_int
    lib.rowops_path.argtypes = [ctypes.c_int] * 3
    lib.rowops_path.restype = ctypes.c_int
    lib.rowops_status_str.argtypes = [ctypes.c_int]
    lib.rowops_status_str.restype = ctypes.c_char_p
    # include/gemm.h
    lib.gemm_leakyrelu_fwd.argtypes = [vp, vp, vp] + [ctypes.c_int] * 4 + [ctypes.c_float, ctypes.c_int, vp]
    lib.gemm_leakyrelu_fwd.restype = ctypes.c_int
    lib.gemm_path.argtypes = [ctypes.c_int] * 5
    lib.gemm_path.restype = ctypes.c_int
    lib.gemm_status_str.argtypes = [ctypes.c_int]
    lib.gemm_status_str.restype = ctypes.c_char_p
    return lib


lib = _load()


def _load_fast():
    path = _build.binding_path()
    if not os.path.exists(path):
        try:
            _build.build_binding(path)
        except Exception as e:
            raise ImportError(f"{path} is missing and could not be built: {e}") from e
    spec = importlib.util.spec_from_file_location(__package__ + "._binding_fast", path)
    fast = importlib.util.module_from_spec(spec)
    fast.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                (lib.attn_fwd, lib.attn_fwd_o16, lib.softmax_rows_fwd, lib.rmsnorm_fwd, lib.gemm_leakyrelu_fwd, lib.residual_rmsnorm_fwd,
                 lib.attn_kv_append, lib.attn_paged_fwd, lib.attn_paged_workspace)))
    return fast


_fast = _load_fast()


def _new(shape, dtype, device, stream, returned=True):
    """Memory that a call on `stream` (None: the current one) writes.  For another stream it comes from that stream's own pool: what is free in the current
    one's may still be written by work under way there, for which `stream` does not wait.  A result (`returned`) is then told of the current
    stream, where it is likely to be read: it is not handed out again before that is done."""
    current = torch.cuda.current_stream(device)
    if stream is None or stream == current:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if returned:
        t.record_stream(current)
    return t


def _int32(x, name: str) -> int:
    """x as the C call takes it (ctypes would drop what lies above 32 bits without a word)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must fit 32 bits")
    return x


def attn_status_str(status: int) -> str:
    return lib.attn_status_str(int(status)).decode()


def attn_supported(S: int, D: int, dtype: int, causal: bool) -> bool:
    return bool(lib.attn_supported(int(S), int(D), int(dtype), int(bool(causal))))


def attn_kernel_name(B: int, H: int, S: int, D: int, dtype: int, causal: bool):
    n = lib.attn_kernel_name(int(B), int(H), int(S), int(D), int(dtype), int(bool(causal)))
    return n.decode() if n else None


def attn_tile_rows(D: int, dtype: int, causal: bool) -> int:
    return int(lib.attn_tile_rows(int(D), int(dtype), int(bool(causal))))


def attn_tile_keys(D: int, dtype: int, causal: bool) -> int:
    return int(lib.attn_tile_keys(int(D), int(dtype), int(bool(causal))))


def attn_launch_rows(B: int, H: int, S: int, D: int, dtype: int, causal: bool) -> int:
    return int(lib.attn_launch_rows(int(B), int(H), int(S), int(D), int(dtype), int(bool(causal))))


def attn_workgroup_rows(B: int, H: int, S: int, D: int, dtype: int, causal: bool) -> int:
    return int(lib.attn_workgroup_rows(int(B), int(H), int(S), int(D), int(dtype), int(bool(causal))))


# ---- include/probe.h: measuring aids (no product path calls them) -------------------------------

def _timed_probe(launch, repeats: int) -> float:
    """Best rate (units of the launch's return value per second) of `repeats` launches after one warm-up."""
    st = torch.cuda.current_stream()
    best = 0.0
    for i in range(repeats + 1):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(st)
        n = int(launch(st.cuda_stream))
        e1.record(st)
        torch.cuda.synchronize()
        if n < 0:
            raise RuntimeError("probe: bad argument or refused launch")
        if i:
            best = max(best, n / (e0.elapsed_time(e1) * 1e-3))
    return best


def probe_mfma(iters: int = 2000, dtype: int = BF16, random_operands: bool = True, workgroups: int = 2048,
               repeats: int = 5) -> float:
    """TFLOP/s that nothing but matrix instructions sustain (best of `repeats` launches, HIP events)."""
    out = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
    return _timed_probe(lambda st: lib.probe_mfma(out.data_ptr(), workgroups, iters, int(dtype), int(bool(random_operands)), st),
                        repeats) / 1e12


def probe_softmax_valu(iters: int = 4000, full: bool = True, workgroups: int = 2048, repeats: int = 3) -> float:
    """Scores per second whose softmax vector work (multiply-add, exp2; with `full` also the row-sum addition and the
    conversion to bfloat16) the vector pipes sustain when they do nothing else."""
    out = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
    return _timed_probe(lambda st: lib.probe_softmax_valu(out.data_ptr(), workgroups, iters, int(bool(full)), st), repeats)


def probe_l2_read(region_kib: int = 1024, iters: int = 64, workgroups: int = 2048, repeats: int = 3) -> float:
    """Bytes per second the compute units read from regions that stay in their XCD's L2."""
    buf = torch.zeros(8 * region_kib * 256, dtype=torch.int32, device="cuda")
    out = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
    return _timed_probe(lambda st: lib.probe_l2_read(buf.data_ptr(), out.data_ptr(), region_kib, workgroups, iters, st), repeats)


def probe_launch_floor_us(workgroups: int = 256, threads: int = 256, launches: int = 200) -> float:
    """Microseconds per launch of a kernel that does nothing, back to back on the current stream (mean)."""
    st = torch.cuda.current_stream()
    for _ in range(20):
        lib.probe_empty(workgroups, threads, st.cuda_stream)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record(st)
    for _ in range(launches):
        if lib.probe_empty(workgroups, threads, st.cuda_stream) != 0:
            raise RuntimeError("probe_empty: bad argument or refused launch")
    e1.record(st)
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) * 1e3 / launches


def probe_issue_share(iters: int = 400, workgroups: int = 256) -> dict:
    """What the two wavefronts of a SIMD cost each other, in shader-clock cycles (medians over all wavefronts):
    mfma_cycles_alone                       per 32x32x16 matrix instruction, its wavefront alone on the SIMD
    valu_cycles_per_64_scores_{bf16,f16}    the softmax's vector work of one score in each of the 64 lanes (the
                                            bfloat16 kernel's mix, or the binary16 one with its dot instructions),
                                            the wavefront alone on the SIMD
    ..._next_to_mfma                        the same while the other wavefront streams matrix instructions
    mfma_cycles_next_to_{bf16,f16}          per matrix instruction of that other wavefront meanwhile
    mfma_issue_cycles                       what one matrix instruction adds to the time of a vector wavefront without
                                            dot instructions (the bfloat16 mix)"""
    out = torch.zeros(workgroups * 16, dtype=torch.int64, device="cuda")
    st = torch.cuda.current_stream()

    def run(matrix_on, vmode):
        for _ in range(2):   # the second launch counts
            if lib.probe_issue_share(out.data_ptr(), workgroups, iters, matrix_on, vmode, st.cuda_stream) != 0:
                raise RuntimeError("probe_issue_share: bad argument or refused launch")
        torch.cuda.synchronize()
        r = out.cpu().reshape(workgroups, 8, 2).to(torch.float64)
        return r[:, :4].reshape(-1, 2), r[:, 4:].reshape(-1, 2)     # matrix wavefronts, vector wavefronts: (cycles, iterations)

    def med(t):
        return float(t.median())

    res = {}
    m, _ = run(1, 0)
    res["mfma_cycles_alone"] = med(m[:, 0] / (32.0 * m[:, 1]))
    for vmode, name in ((1, "bf16"), (2, "f16")):
        _, v0 = run(0, vmode)
        alone = med(v0[:, 0] / (32.0 * v0[:, 1]))
        m, v = run(1, vmode)
        together = med(v[:, 0] / (32.0 * v[:, 1]))
        mfma_per_cycle = med(32.0 * m[:, 1] / m[:, 0])
        res[f"valu_cycles_per_64_scores_{name}"] = alone
        res[f"valu_cycles_per_64_scores_{name}_next_to_mfma"] = together
        res[f"mfma_cycles_next_to_{name}"] = 1.0 / mfma_per_cycle
        if vmode == 1:
            res["mfma_issue_cycles"] = (together - alone) / (together * mfma_per_cycle)
    return res


def attn_fwd_raw(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, H, S, D, causal, scale, dtype, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.attn_fwd(q_ptr or None, k_ptr or None, v_ptr or None, o_ptr or None, lse_ptr or None,
                            int(B), int(H), int(S), int(D), int(causal), float(scale), int(dtype),
                            stream or None))


def attn_fwd_o16_raw(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, H, S, D, causal, scale, dtype, stream) -> int:
    """attn_fwd_o16 as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.attn_fwd_o16(q_ptr or None, k_ptr or None, v_ptr or None, o_ptr or None, lse_ptr or None,
                                int(B), int(H), int(S), int(D), int(causal), float(scale), int(dtype),
                                stream or None))


def attn_fwd_o16(q, k, v, causal: bool, scale: float, o=None, lse=None, stream=None, want_lse: bool = True):
    """attn_fwd_o16 on torch device tensors: as attn_fwd, with o in the dtype of q, k, v."""
    return attn_fwd(q, k, v, causal, scale, o=o, lse=lse, stream=stream, want_lse=want_lse, _o16=True)


def attn_fwd(q, k, v, causal: bool, scale: float, o=None, lse=None, stream=None, want_lse: bool = True,
             _o16: bool = False):
    """attn_fwd on torch device tensors.

    q, k, v : [B,H,S,D] contiguous torch.float16 or torch.bfloat16 tensors on the GPU.
    o, lse  : optional preallocated fp32 outputs ([B,H,S,D], [B,H,S]); allocated if None.
    stream  : a torch.cuda.Stream (default: the current stream).
    Returns (o, lse).  Asynchronous, like the C call.
    """
    done = _fast.attn_fwd(q, k, v, causal, scale, o, lse, stream, want_lse, _o16)
    if done is not None:
        return done
    if q.dtype == torch.float16:
        dtype = F16
    elif q.dtype == torch.bfloat16:
        dtype = BF16
    else:
        raise TypeError("q, k, v must be float16 or bfloat16")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share one dtype")
    if q.dim() != 4 or k.shape != q.shape or v.shape != q.shape:
        raise ValueError("q, k, v must be [B,H,S,D] of one shape")
    for t in (q, k, v):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous device tensors")
    B, H, S, D = q.shape
    odt = q.dtype if _o16 else torch.float32
    if o is None:
        o = _new((B, H, S, D), odt, q.device, stream)
    if lse is None and want_lse:
        lse = _new((B, H, S), torch.float32, q.device, stream)
    for t, shp, dt in ((o, (B, H, S, D), odt), (lse, (B, H, S), torch.float32)):
        if t is not None and (t.dtype != dt or tuple(t.shape) != shp or not t.is_contiguous() or not t.is_cuda):
            raise ValueError("o / lse must be contiguous device tensors of shape [B,H,S,D] / [B,H,S] (lse fp32; o fp32, "
                             "or the input dtype for attn_fwd_o16)")
    st = (stream or torch.cuda.current_stream(q.device)).cuda_stream
    rc = (attn_fwd_o16_raw if _o16 else attn_fwd_raw)(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                                      lse.data_ptr() if lse is not None else 0, B, H, S, D, causal, scale,
                                                      dtype, st)
    if rc != 0:
        raise AttnError(rc, attn_status_str(rc))
    return o, lse


# ---- include/attn.h: a paged key/value cache ----------------------------------------------------

def attn_paged_workspace(B: int, T: int, Hq: int, Hk: int, D: int, max_q: int, max_kv: int, prefix_len: int = 0) -> int:
    """Bytes of workspace attn_paged_fwd needs for these sizes (-1: sizes it refuses)."""
    sizes = [int(n) for n in (B, T, Hq, Hk, D, max_q, max_kv, prefix_len)]
    return int(lib.attn_paged_workspace(*sizes)) if all(-2 ** 31 <= n < 2 ** 31 for n in sizes) else -1


def attn_kv_append_raw(cache: PagedCache, q_ptr, k_ptr, v_ptr, q_stride, k_stride, v_stride, q_out_ptr, cos_ptr, sin_ptr, rot, interleaved,
                       n_angles, pos_offset, Hq, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.attn_kv_append(ctypes.byref(cache), q_ptr or None, k_ptr or None, v_ptr or None, int(q_stride), int(k_stride), int(v_stride),
                                  q_out_ptr or None, cos_ptr or None, sin_ptr or None, int(rot), int(interleaved), int(n_angles),
                                  int(pos_offset), int(Hq), stream or None))


def attn_paged_fwd_raw(cache: PagedCache, q_ptr, q_stride, o_ptr, lse_ptr, prefix_table_ptr, prefix_len, Hq, max_q, max_kv, scale,
                       workspace_ptr, workspace_bytes, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.attn_paged_fwd(ctypes.byref(cache), q_ptr or None, int(q_stride), o_ptr or None, lse_ptr or None, prefix_table_ptr or None,
                                  int(prefix_len), int(Hq), int(max_q), int(max_kv), float(scale), workspace_ptr or None,
                                  int(workspace_bytes), stream or None))


def _heads(t, name, T=None, D=None):
    """t [T, heads, D] on the GPU, the heads of a token contiguous; the elements between two tokens."""
    if t.dim() != 3 or not t.is_cuda or (T is not None and t.shape[0] != T) or (D is not None and t.shape[2] != D):
        raise ValueError(f"{name} must be a device tensor [T, heads, D]")
    if t.numel() and (t.stride(2) != 1 and t.shape[2] > 1 or t.stride(1) != t.shape[2] and t.shape[1] > 1):
        raise ValueError(f"the heads of a token of {name} must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _ints(t, name, shape):
    if t.dtype != torch.int32 or not t.is_cuda or t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{name} must be an int32 device tensor of shape {['any' if n is None else n for n in shape]}")
    if t.numel() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    return t


def _paged_cache(k_cache, v_cache, page_table, cu_q, kv_len, T) -> PagedCache:
    dtype = {torch.float16: F16, torch.bfloat16: BF16}.get(k_cache.dtype)
    if dtype is None or v_cache.dtype != k_cache.dtype:
        raise TypeError("k_cache and v_cache must be float16 or bfloat16, both of one dtype")
    if k_cache.dim() != 4 or v_cache.shape != k_cache.shape or not k_cache.is_cuda or not v_cache.is_cuda:
        raise ValueError("k_cache and v_cache must be device tensors [n_pages, Hk, page_size, D] of one shape")
    n_pages, Hk, page, D = k_cache.shape
    for t in (k_cache, v_cache):
        if t.numel() and (not t[0].is_contiguous() or (n_pages > 1 and t.stride(0) != k_cache.stride(0))):
            raise ValueError("a page of k_cache and v_cache must be contiguous, and the pages of both equally far apart")
    B = kv_len.shape[0] if kv_len.dim() == 1 else -1
    _ints(kv_len, "kv_len", (None,)), _ints(cu_q, "cu_q", (B + 1,)), _ints(page_table, "page_table", (B, None))
    return PagedCache(k_cache.data_ptr() or None, v_cache.data_ptr() or None, k_cache.stride(0) if n_pages > 1 else Hk * page * D, n_pages, page, Hk, D,
                      dtype, page_table.data_ptr() or None,
                      _int32(page_table.stride(0), "page_table's stride") if B > 1 else page_table.shape[1], page_table.shape[1],
                      cu_q.data_ptr() or None, kv_len.data_ptr() or None, B, T)


def attn_kv_append(q, k, v, k_cache, v_cache, page_table, cu_q, kv_len, cos=None, sin=None, interleaved: bool = False, pos_offset: int = 0,
                   q_out=None, stream=None):
    """attn_kv_append on torch device tensors: the new tokens' keys and values go to their pages, queries and keys rotated on the way.

    q, k, v          : [T, Hq, D], [T, Hk, D], [T, Hk, D] of one 16-bit dtype, a token's heads contiguous (parts of one projection's rows
                       will do); q may be None (keys and values only).
    k_cache, v_cache : [n_pages, Hk, page_size, D], written.
    page_table       : [B, width] int32;  cu_q [B + 1], kv_len [B] int32: the new tokens, and the keys with them, of every sequence.
    cos, sin         : [positions, rot / 2] fp32, or None: no rotation.
    pos_offset       : added to a token's place in its sequence for its row of cos and sin (the length of a shared prefix).
    q_out            : optional preallocated [T, Hq, D] output.
    Returns q_out (None where q is).  Asynchronous, like the C call.
    """
    done = _fast.attn_kv_append(q, k, v, k_cache, v_cache, page_table, cu_q, kv_len, cos, sin, interleaved, pos_offset, q_out, stream)
    if done is not None:
        return done
    T, D = k.shape[0], k_cache.shape[-1]
    cache = _paged_cache(k_cache, v_cache, page_table, cu_q, kv_len, T)
    if any(t.dtype != k_cache.dtype for t in (q, k, v, q_out) if t is not None):
        raise TypeError("q, k, v, q_out and the cache must share one dtype")
    ks, vs = _heads(k, "k", T, D), _heads(v, "v", T, D)
    if k.shape[1] != cache.Hk or v.shape[1] != cache.Hk:
        raise ValueError("k and v must have the cache's number of heads")
    qs, Hq = (_heads(q, "q", T, D), q.shape[1]) if q is not None else (0, 0)
    if q is None:
        q_out = None
    elif q_out is None:
        q_out = _new(q.shape, q.dtype, q.device, stream)
    elif q_out.shape != q.shape or not q_out.is_cuda or not q_out.is_contiguous():
        raise ValueError("q_out must be a contiguous device tensor of q's shape")
    rot = n_angles = 0
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin go together")
    if cos is not None:
        if cos.dtype != torch.float32 or sin.dtype != torch.float32:
            raise TypeError("cos and sin must be float32")
        if cos.dim() != 2 or sin.shape != cos.shape or not cos.is_cuda or not sin.is_cuda or not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous device tensors [positions, rot / 2] of one shape")
        n_angles, rot = cos.shape[0], 2 * cos.shape[1]
    pos_offset = _int32(pos_offset, "pos_offset")
    st = (stream or torch.cuda.current_stream(k.device)).cuda_stream
    ptr = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
    rc = attn_kv_append_raw(cache, ptr(q), ptr(k), ptr(v), qs, ks, vs, ptr(q_out), ptr(cos), ptr(sin), rot, bool(interleaved), n_angles,
                            pos_offset, Hq, st)
    if rc != 0:
        raise AttnError(rc, attn_status_str(rc), "attn_kv_append")
    return q_out


def attn_paged_fwd(q, k_cache, v_cache, page_table, cu_q, kv_len, scale: float, max_q=None, max_kv=None, prefix_table=None,
                   prefix_len: int = 0, o=None, lse=None, stream=None, want_lse: bool = True, workspace=None):
    """attn_paged_fwd on torch device tensors: the new tokens' attention over a paged cache.

    q                : [T, Hq, D], a token's heads contiguous; Hq a multiple of the cache's Hk.
    k_cache, v_cache, page_table, cu_q, kv_len : as for attn_kv_append.
    max_q            : the most new tokens any sequence has (default T, which is safe, and slow for a decode step: 64 sequences of 1 to 1024 keys take 29 us
                       with it and 14.5 with 1); rows past it, and rows that no sequence owns, are not written.
    max_kv           : the most own keys (a hint of how to share out the work; default what the table holds).
    prefix_table, prefix_len : int32 pages of a prefix in front of every sequence, and its length.
    o, lse           : optional preallocated outputs [T, Hq, D] of q's dtype, [T, Hq] fp32.
    workspace        : optional uint8 tensor of attn_paged_workspace(...) bytes; allocated for the call if None.
    Returns (o, lse).  Asynchronous, like the C call.
    """
    done = _fast.attn_paged_fwd(q, k_cache, v_cache, page_table, cu_q, kv_len, scale, max_q, max_kv, prefix_table, prefix_len, o, lse, stream,
                                want_lse, workspace)
    if done is not None:
        return done
    T, D = q.shape[0], k_cache.shape[-1]
    cache = _paged_cache(k_cache, v_cache, page_table, cu_q, kv_len, T)
    if q.dtype != k_cache.dtype:
        raise TypeError("q and the cache must share one dtype")
    qs, Hq = _heads(q, "q", T, D), q.shape[1]
    if cache.Hk == 0 or Hq == 0 or Hq % cache.Hk:
        raise ValueError("the heads of q must be a multiple of the cache's")
    max_q = T if max_q is None else _int32(max_q, "max_q")
    max_kv = min(cache.width * cache.page_size, 2 ** 31 - 1) if max_kv is None else _int32(max_kv, "max_kv")
    prefix_len = _int32(prefix_len, "prefix_len")
    if prefix_len:
        need = -(-prefix_len // max(1, cache.page_size))
        if prefix_table is None or prefix_table.dim() != 1 or prefix_table.shape[0] < need:
            raise ValueError("prefix_table must hold the pages of prefix_len keys")
        _ints(prefix_table, "prefix_table", (None,))
    if o is None:
        o = _new(q.shape, q.dtype, q.device, stream)
    if lse is None and want_lse:
        lse = _new(q.shape[:2], torch.float32, q.device, stream)
    for t, shp, dt in ((o, q.shape, q.dtype), (lse, q.shape[:2], torch.float32)):
        if t is not None and (t.dtype != dt or t.shape != shp or not t.is_contiguous() or not t.is_cuda):
            raise ValueError("o / lse must be contiguous device tensors [T, Hq, D] of q's dtype / [T, Hq] fp32")
    need = max(0, attn_paged_workspace(cache.B, T, Hq, cache.Hk, D, max_q, max_kv, prefix_len))
    if workspace is None:
        workspace = _new(need, torch.uint8, q.device, stream, returned=False)
    elif workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 device tensor")
    st = (stream or torch.cuda.current_stream(q.device)).cuda_stream
    rc = attn_paged_fwd_raw(cache, q.data_ptr(), qs, o.data_ptr(), lse.data_ptr() if lse is not None else 0,
                            prefix_table.data_ptr() if prefix_len else 0, prefix_len, Hq, max_q, max_kv, scale, workspace.data_ptr(),
                            workspace.numel(), st)
    if rc != 0:
        raise AttnError(rc, attn_status_str(rc), "attn_paged_fwd")
    return o, lse


# ---- include/rowops.h ------------------------------------------------------------------------

class RowopsError(RuntimeError):
    def __init__(self, what: str, status: int, msg: str):
        super().__init__(f"{what} failed with status {status}: {msg}")
        self.status = status


def rowops_status_str(status: int) -> str:
    return lib.rowops_status_str(int(status)).decode()


def rowops_path(op: int, row_len: int, dtype: int) -> int:
    return int(lib.rowops_path(int(op), int(row_len), int(dtype)))


def softmax_rows_fwd_raw(x_ptr, y_ptr, n_rows, n_cols, dtype, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.softmax_rows_fwd(x_ptr or None, y_ptr or None, int(n_rows), int(n_cols), int(dtype), stream or None))


def rmsnorm_fwd_raw(x_ptr, w_ptr, y_ptr, n_rows, d, eps, dtype, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.rmsnorm_fwd(x_ptr or None, w_ptr or None, y_ptr or None, int(n_rows), int(d), float(eps), int(dtype),
                               stream or None))


def _row_args(x, y, stream):
    if x.dtype == torch.float16:
        dtype = F16
    elif x.dtype == torch.bfloat16:
        dtype = BF16
    else:
        raise TypeError("x must be float16 or bfloat16")
    if x.dim() < 1 or not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous device tensor with the rows along the last dimension")
    if y is None:
        y = _new(x.shape, x.dtype, x.device, stream)
    elif y.dtype != x.dtype or y.shape != x.shape or not y.is_cuda or not y.is_contiguous():
        raise ValueError("y must be a contiguous device tensor of the shape and dtype of x")
    n = x.shape[-1]
    return dtype, y, (x.numel() // n if n else 0), n


def softmax_rows_fwd(x, y=None, stream=None):
    """softmax_rows_fwd on a torch device tensor: softmax over the last dimension, result in x's dtype."""
    done = _fast.softmax_rows_fwd(x, y, stream)
    if done is not None:
        return done
    dtype, y, n_rows, n = _row_args(x, y, stream)
    st = (stream or torch.cuda.current_stream(x.device)).cuda_stream
    rc = softmax_rows_fwd_raw(x.data_ptr(), y.data_ptr(), n_rows, n, dtype, st)
    if rc != 0:
        raise RowopsError("softmax_rows_fwd", rc, rowops_status_str(rc))
    return y


def rmsnorm_fwd(x, w, eps: float, y=None, stream=None):
    """rmsnorm_fwd on torch device tensors: x [..., d], w [d] of one dtype; result in x's dtype."""
    done = _fast.rmsnorm_fwd(x, w, eps, y, stream)
    if done is not None:
        return done
    dtype, y, n_rows, n = _row_args(x, y, stream)
    if w.dtype != x.dtype or tuple(w.shape) != (n,) or not w.is_cuda or not w.is_contiguous():
        raise ValueError("w must be a contiguous device tensor [d] of x's dtype")
    st = (stream or torch.cuda.current_stream(x.device)).cuda_stream
    rc = rmsnorm_fwd_raw(x.data_ptr(), w.data_ptr(), y.data_ptr(), n_rows, n, eps, dtype, st)
    if rc != 0:
        raise RowopsError("rmsnorm_fwd", rc, rowops_status_str(rc))
    return y


def residual_rmsnorm_fwd_raw(x_ptr, r_ptr, w_ptr, y_ptr, scale_ptr, r_out_ptr, n_rows, d, eps, dtype, fp8, group, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.residual_rmsnorm_fwd(x_ptr or None, r_ptr or None, w_ptr or None, y_ptr or None, scale_ptr or None, r_out_ptr or None,
                                        int(n_rows), int(d), float(eps), int(dtype), int(fp8), int(group), stream or None))


def _residual_norm(x, r, w, eps, fp8, group, y, scale, r_out, stream):
    group = _int32(group, "group")
    dtype, y16, n_rows, n = _row_args(x, x if fp8 else y, stream)
    if w.dtype != x.dtype or tuple(w.shape) != (n,) or not w.is_cuda or not w.is_contiguous():
        raise ValueError("w must be a contiguous device tensor [d] of x's dtype")
    if r is None:
        r_out = None
    elif r_out is None:
        r_out = _new(x.shape, x.dtype, x.device, stream)
    for t in (r, r_out):
        if t is not None and (t.dtype != x.dtype or t.shape != x.shape or not t.is_cuda or not t.is_contiguous()):
            raise ValueError("r and r_out must be contiguous device tensors of the shape and dtype of x")
    if not fp8:
        y = y16
    elif y is None:
        y = _new(x.shape, torch.float8_e4m3fn, x.device, stream)
    if fp8:
        if y.dtype != torch.float8_e4m3fn or y.shape != x.shape or not y.is_cuda or not y.is_contiguous():
            raise ValueError("y must be a contiguous float8_e4m3fn device tensor of the shape of x")
        shape = (*x.shape[:-1], -(-n // group) if group else 1)
        if scale is None:
            scale = _new(shape, torch.float32, x.device, stream)
        elif scale.dtype != torch.float32 or scale.shape != shape or not scale.is_cuda or not scale.is_contiguous():
            raise ValueError("scale must be a contiguous float32 device tensor [..., 1], or [..., ceil(d / group)]")
    st = (stream or torch.cuda.current_stream(x.device)).cuda_stream
    rc = residual_rmsnorm_fwd_raw(x.data_ptr(), r.data_ptr() if r is not None else 0, w.data_ptr(), y.data_ptr(), scale.data_ptr() if fp8 else 0,
                                  r_out.data_ptr() if r is not None else 0, n_rows, n, eps, dtype, fp8, group, st)
    if rc != 0:
        raise RowopsError("residual_rmsnorm_fwd", rc, rowops_status_str(rc))
    return y, scale, r_out


def residual_rmsnorm_fwd(x, r, w, eps: float, y=None, r_out=None, stream=None):
    """residual_rmsnorm_fwd on torch device tensors: the RMS norm of h = x + r, and h for the next residual.

    x, r  : [..., d] contiguous float16 or bfloat16 tensors of one shape and dtype; r None: h = x.
    w     : [d] of that dtype.
    y, r_out : optional preallocated outputs (r_out may be r or x).
    Returns (y, r_out), both in x's dtype; r_out is None where r is.
    """
    done = _fast.residual_rmsnorm_fwd(x, r, w, eps, y, r_out, stream)
    if done is not None:
        return done
    y, _, r_out = _residual_norm(x, r, w, eps, False, 0, y, None, r_out, stream)
    return y, r_out


def residual_rmsnorm_fwd_fp8(x, r, w, eps: float, group: int = 0, y=None, scale=None, r_out=None, stream=None):
    """The same with y in 8 bits: y (float8_e4m3fn) times scale (fp32 [..., 1], or with group=128 [..., ceil(d / 128)], one for each 128
    columns) is the norm's result.  Returns (y, scale, r_out)."""
    done = _fast.residual_rmsnorm_fwd_fp8(x, r, w, eps, group, y, scale, r_out, stream)
    if done is not None:
        return done
    return _residual_norm(x, r, w, eps, True, group, y, scale, r_out, stream)


# ---- include/gemm.h --------------------------------------------------------------------------

class GemmError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"gemm_leakyrelu_fwd failed with status {status}: {msg}")
        self.status = status


def gemm_status_str(status: int) -> str:
    return lib.gemm_status_str(int(status)).decode()


def gemm_path(batch: int, M: int, N: int, K: int, dtype: int) -> int:
    return int(lib.gemm_path(int(batch), int(M), int(N), int(K), int(dtype)))


def gemm_leakyrelu_fwd_raw(a_ptr, b_ptr, c_ptr, batch, M, N, K, slope, dtype, stream) -> int:
    """The C entry point as is: device addresses as ints (0 = NULL), returns the status."""
    return int(lib.gemm_leakyrelu_fwd(a_ptr or None, b_ptr or None, c_ptr or None, int(batch), int(M), int(N), int(K),
                                      float(slope), int(dtype), stream or None))


def gemm_leakyrelu_fwd(a, b, slope: float = 0.01, c=None, stream=None):
    """gemm_leakyrelu_fwd on torch device tensors: a [batch, M, K] (or [M, K]), b [batch, K, N] (or [K, N])
    of one 16-bit dtype; returns c [batch, M, N] (or [M, N]) in that dtype."""
    done = _fast.gemm_leakyrelu_fwd(a, b, slope, c, stream)
    if done is not None:
        return done
    if a.dtype == torch.float16:
        dtype = F16
    elif a.dtype == torch.bfloat16:
        dtype = BF16
    else:
        raise TypeError("a and b must be float16 or bfloat16")
    if b.dtype != a.dtype or a.dim() != b.dim() or a.dim() not in (2, 3):
        raise TypeError("a and b must share one dtype and be both [M,K],[K,N] or both [batch,M,K],[batch,K,N]")
    a3, b3 = (a, b) if a.dim() == 3 else (a[None], b[None])
    if a3.shape[0] != b3.shape[0] or a3.shape[2] != b3.shape[1]:
        raise ValueError("a must be [batch, M, K] and b [batch, K, N]")
    for t in (a, b):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("a and b must be contiguous device tensors")
    batch, M, K = a3.shape
    N = b3.shape[2]
    shape = (batch, M, N) if a.dim() == 3 else (M, N)
    if c is None:
        c = _new(shape, a.dtype, a.device, stream)
    elif c.dtype != a.dtype or tuple(c.shape) != shape or not c.is_cuda or not c.is_contiguous():
        raise ValueError("c must be a contiguous device tensor [batch, M, N] of the dtype of a")
    st = (stream or torch.cuda.current_stream(a.device)).cuda_stream
    rc = gemm_leakyrelu_fwd_raw(a.data_ptr(), b.data_ptr(), c.data_ptr(), batch, M, N, K, slope, dtype, st)
    if rc != 0:
        raise GemmError(rc, gemm_status_str(rc))
    return c
