"""ctypes binding of librvq.so: the same entry points as include/rvq.h, argument marshalling only.

PyTorch is used for device memory and streams; every step of the method runs inside the
library's HIP kernels.  Importing this module fails loudly when the library has not been built
(``python -m paper_2410_15704_amd.build``): there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
import os

# PyTorch comes first: it carries its own HIP runtime, and librvq.so must bind to that copy.  Loaded
# the other way round, the system's runtime is in the process before PyTorch's and PyTorch then
# finds no GPU.
import torch  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librvq.so")

RVQ_OK, RVQ_EINVAL, RVQ_ENOCODEBOOK, RVQ_EHIP, RVQ_ENOMEM = 0, -1, -2, -3, -4
RVQ_EWORKSPACE, RVQ_EKERNEL = -5, -6
DEFAULT_ROWS = 131072
STATIC_MAX_ROWS = 1048576
F32, BF16, F16 = 0, 1, 2
CONTIGUOUS, STRIDED = 0, 1
PATH_AUTO, PATH_EXACT, PATH_SCREEN = 0, 1, 2
DTYPES = {"fp32": F32, "bf16": BF16, "fp16": F16}

EXPORTS = ("rvq_create", "rvq_destroy", "rvq_set_codebooks", "rvq_get_codebooks", "rvq_encode",
           "rvq_decode", "rvq_ema_update", "rvq_strerror", "rvq_last_hip_error", "rvq_version",
           "rvq_get_counters", "rvq_packed_record_bytes", "rvq_pack_codes", "rvq_unpack_codes",
           "rvq_decode_packed", "rvq_decode_rope", "rvq_reserve", "rvq_reserved_rows",
           "rvq_check_kernels", "rvq_debug_set_wait_polls", "rvq_encode_static",
           "rvq_probe_gather_rates", "rvq_attn_decode", "rvq_attn_workspace_bytes",
           "rvq_rope_tables", "rvq_rope", "rvq_cache8_append", "rvq_cache8_read",
           "rvq_cache8_attn", "rvq_cache8_attn_workspace_bytes")
ROPE_ADJACENT, ROPE_HALVES = 0, 1
PAGE_TOKENS = 64
MOST_TOKENS = 2**31 - 1  # of a sequence


class rvq_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "d", "dhat", "depth", "K", "grouping", "scale", "std_ddof", "in_dtype", "out_dtype",
        "std_dtype", "encode_path", "reserved")]


class rvq_cache8(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("table", ctypes.c_void_p),
                ("table_pages", ctypes.c_int32), ("n_seqs", ctypes.c_int32), ("lengths", ctypes.c_void_p)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2410_15704_amd.build` "
            "(hipcc, gfx950). There is no fallback path.")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    lib.rvq_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(rvq_config)]
    lib.rvq_destroy.argtypes = [vp]
    lib.rvq_set_codebooks.argtypes = [vp, vp, vp]
    lib.rvq_get_codebooks.argtypes = [vp, vp, vp]
    lib.rvq_encode.argtypes = [vp, vp, i64, i64, i32, i32, vp, vp, vp, vp]
    lib.rvq_encode_static.argtypes = [vp, vp, i64, i64, i32, i32, vp, vp, vp, vp]
    lib.rvq_decode.argtypes = [vp, vp, vp, i64, i32, vp, i64, vp]
    lib.rvq_ema_update.argtypes = [vp, i32, vp, vp, i64, i64, f32, f32, vp, vp, vp]
    lib.rvq_get_counters.argtypes = [vp, ctypes.POINTER(ctypes.c_int64)]
    lib.rvq_packed_record_bytes.argtypes = [vp]
    lib.rvq_packed_record_bytes.restype = ctypes.c_int64
    lib.rvq_pack_codes.argtypes = [vp, vp, i64, vp, vp]
    lib.rvq_unpack_codes.argtypes = [vp, vp, i64, vp, vp]
    lib.rvq_decode_packed.argtypes = [vp, vp, vp, i64, i32, vp, i64, vp]
    lib.rvq_decode_rope.argtypes = [vp, vp, vp, i64, i32, vp, vp, i32, vp, i64, vp]
    lib.rvq_reserve.argtypes = [vp, i64]
    lib.rvq_reserved_rows.argtypes = [vp]
    lib.rvq_reserved_rows.restype = ctypes.c_int64
    lib.rvq_check_kernels.argtypes = [vp]
    lib.rvq_debug_set_wait_polls.argtypes = [vp, i64]
    lib.rvq_probe_gather_rates.argtypes = [ctypes.POINTER(ctypes.c_double)]
    lib.rvq_strerror.argtypes = [ctypes.c_int]
    lib.rvq_strerror.restype = ctypes.c_char_p
    lib.rvq_last_hip_error.argtypes = [vp]
    lib.rvq_version.restype = ctypes.c_int
    lib.rvq_attn_workspace_bytes.argtypes = [i64, i32, i32]
    lib.rvq_attn_workspace_bytes.restype = i64
    lib.rvq_attn_decode.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, i32, i64, vp, vp, f32, vp, vp, i64, vp]
    f64, view = ctypes.c_double, ctypes.POINTER(rvq_cache8)
    lib.rvq_rope_tables.argtypes = [vp, i64, i32, f64, f64, f64, f64, f64, f64, vp, vp, vp]
    lib.rvq_rope.argtypes = [vp, i32, i64, i32, i32, i32, i32, i64, i64, vp, vp, vp, i64, i64, vp]
    lib.rvq_cache8_append.argtypes = [view, vp, vp, i32, i64, i64, i64, i64, i64, vp, vp, vp, i32, i32, vp]
    lib.rvq_cache8_read.argtypes = [view, vp, vp, i64, vp, vp, i32, i32, i32, vp, i64, i64, vp, i64, i64, vp]
    lib.rvq_cache8_attn_workspace_bytes.argtypes = [view, i32, i64, i32]
    lib.rvq_cache8_attn_workspace_bytes.restype = i64
    lib.rvq_cache8_attn.argtypes = [view, vp, i32, i64, i32, i64, i64, vp, f32, i32, i32, vp, i64, i64, vp, i64, vp]
    for name in EXPORTS:
        getattr(lib, name)
        if name not in ("rvq_strerror", "rvq_version", "rvq_packed_record_bytes",
                        "rvq_reserved_rows", "rvq_attn_workspace_bytes", "rvq_cache8_attn_workspace_bytes"):
            getattr(lib, name).restype = ctypes.c_int
    return lib


lib = _load()


class RvqError(RuntimeError):
    def __init__(self, code, ctx=None):
        self.code = code
        msg = lib.rvq_strerror(code).decode()
        if code == RVQ_EHIP and ctx:
            msg += f" (hipError {lib.rvq_last_hip_error(ctx)})"
        super().__init__(f"librvq: {msg} [{code}]")


def _ptr(t):
    """Device pointer of a torch tensor (or None / int passthrough)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ---- the entry points, same names as the header -----------------------------------------------
def rvq_version() -> int:
    return lib.rvq_version()


def rvq_strerror(code: int) -> str:
    return lib.rvq_strerror(code).decode()


def rvq_create(*, d, dhat=32, depth=8, K=2048, grouping=CONTIGUOUS, scale=1, std_ddof=0,
               in_dtype=F32, out_dtype=F16, std_dtype=F16, encode_path=PATH_AUTO, check=True):
    cfg = rvq_config(d, dhat, depth, K, grouping, scale, std_ddof, in_dtype, out_dtype, std_dtype,
                     encode_path, 0)
    ctx = ctypes.c_void_p()
    rc = lib.rvq_create(ctypes.byref(ctx), ctypes.byref(cfg))
    if rc != RVQ_OK:
        if check:
            raise RvqError(rc)
        return rc
    return ctx


def rvq_destroy(ctx):
    return lib.rvq_destroy(ctx)


def _chk(rc, ctx):
    if rc != RVQ_OK:
        raise RvqError(rc, ctx)
    return rc


def rvq_reserve(ctx, max_rows):
    return _chk(lib.rvq_reserve(ctx, max_rows), ctx)


def rvq_reserved_rows(ctx) -> int:
    return int(lib.rvq_reserved_rows(ctx))


def rvq_check_kernels(ctx, check=True):
    rc = lib.rvq_check_kernels(ctx)
    return _chk(rc, ctx) if check else rc


def rvq_debug_set_wait_polls(ctx, polls):
    return _chk(lib.rvq_debug_set_wait_polls(ctx, polls), ctx)


def rvq_probe_gather_rates():
    out = (ctypes.c_double * 3)()
    _chk(lib.rvq_probe_gather_rates(out), None)
    return dict(lds_random_GBs=out[0], lds_consecutive_GBs=out[1], l2_rows_random_GBs=out[2])


def rvq_set_codebooks(ctx, dC, stream=None):
    return _chk(lib.rvq_set_codebooks(ctx, _ptr(dC), _stream(stream)), ctx)


def rvq_get_codebooks(ctx, dC, stream=None):
    return _chk(lib.rvq_get_codebooks(ctx, _ptr(dC), _stream(stream)), ctx)


def rvq_encode(ctx, dX, N, ldx, stage_begin, stage_end, dCodes, dStd, dResidual=None, stream=None):
    return _chk(lib.rvq_encode(ctx, _ptr(dX), N, ldx, stage_begin, stage_end, _ptr(dCodes),
                               _ptr(dStd), _ptr(dResidual), _stream(stream)), ctx)


def rvq_encode_static(ctx, dX, N, ldx, stage_begin, stage_end, dCodes, dStd, dResidual=None,
                      stream=None):
    return _chk(lib.rvq_encode_static(ctx, _ptr(dX), N, ldx, stage_begin, stage_end, _ptr(dCodes),
                                      _ptr(dStd), _ptr(dResidual), _stream(stream)), ctx)


def rvq_decode(ctx, dCodes, dStd, N, depth_used, dOut, ldo, stream=None):
    return _chk(lib.rvq_decode(ctx, _ptr(dCodes), _ptr(dStd), N, depth_used, _ptr(dOut), ldo,
                               _stream(stream)), ctx)


def rvq_ema_update(ctx, stage, dR, dCodes, code_stride, M, decay, eps, dClusterSize, dEmbedSum,
                   stream=None):
    return _chk(lib.rvq_ema_update(ctx, stage, _ptr(dR), _ptr(dCodes), code_stride, M, decay, eps,
                                   _ptr(dClusterSize), _ptr(dEmbedSum), _stream(stream)), ctx)


def rvq_packed_record_bytes(ctx) -> int:
    return int(lib.rvq_packed_record_bytes(ctx))


def rvq_pack_codes(ctx, dCodes, N, dPacked, stream=None):
    return _chk(lib.rvq_pack_codes(ctx, _ptr(dCodes), N, _ptr(dPacked), _stream(stream)), ctx)


def rvq_unpack_codes(ctx, dPacked, N, dCodes, stream=None):
    return _chk(lib.rvq_unpack_codes(ctx, _ptr(dPacked), N, _ptr(dCodes), _stream(stream)), ctx)


def rvq_decode_packed(ctx, dPacked, dStd, N, depth_used, dOut, ldo, stream=None):
    return _chk(lib.rvq_decode_packed(ctx, _ptr(dPacked), _ptr(dStd), N, depth_used, _ptr(dOut),
                                      ldo, _stream(stream)), ctx)


def rvq_decode_rope(ctx, dCodes, dStd, N, depth_used, dCos, dSin, head_dim, dOut, ldo, stream=None):
    return _chk(lib.rvq_decode_rope(ctx, _ptr(dCodes), _ptr(dStd), N, depth_used, _ptr(dCos),
                                    _ptr(dSin), head_dim, _ptr(dOut), ldo, _stream(stream)), ctx)


def rvq_attn_workspace_bytes(N, n_q_heads, n_kv_heads):
    return int(lib.rvq_attn_workspace_bytes(N, n_q_heads, n_kv_heads))


def rvq_attn_decode(kctx, vctx, dQ, n_q_heads, n_kv_heads, dKCodes, dKStd, dVCodes, dVStd, N, dCos,
                    dSin, scale, dOut, dWorkspace, workspace_bytes, stream=None, packed=0):
    return _chk(lib.rvq_attn_decode(kctx, vctx, _ptr(dQ), n_q_heads, n_kv_heads, _ptr(dKCodes),
                                    _ptr(dKStd), _ptr(dVCodes), _ptr(dVStd), packed, N, _ptr(dCos),
                                    _ptr(dSin), scale, _ptr(dOut), _ptr(dWorkspace), workspace_bytes,
                                    _stream(stream)), kctx)


def rvq_get_counters(ctx):
    out = (ctypes.c_int64 * 16)()  # debug builds report more
    _chk(lib.rvq_get_counters(ctx, out), ctx)
    return dict(zip(("slow_searches", "exact_rescored", "groups_rescored", "searches",
                     "group_exact_passes"), list(out)))


class Quantizer:
    """Owns one rvq_ctx; thin convenience over the entry points above (allocation of outputs and
    shape bookkeeping only)."""

    def __init__(self, **cfg):
        self.cfg = dict(d=None, dhat=32, depth=8, K=2048, grouping=CONTIGUOUS, scale=1, std_ddof=0,
                        in_dtype=F32, out_dtype=F16, std_dtype=F16, encode_path=PATH_AUTO)
        self.cfg.update(cfg)
        self.ctx = rvq_create(**self.cfg)
        self.G = self.cfg["d"] // self.cfg["dhat"]

    def close(self):
        if self.ctx is not None:
            rvq_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_codebooks(self, C):
        import torch
        assert C.dtype == torch.float32 and C.is_cuda and C.is_contiguous()
        assert tuple(C.shape) == (self.cfg["depth"], self.cfg["K"], self.cfg["dhat"])
        rvq_set_codebooks(self.ctx, C)

    def get_codebooks(self):
        import torch
        C = torch.empty((self.cfg["depth"], self.cfg["K"], self.cfg["dhat"]), dtype=torch.float32,
                        device="cuda")
        rvq_get_codebooks(self.ctx, C)
        return C

    def _std_torch_dtype(self):
        import torch
        return torch.float16 if self.cfg["std_dtype"] == F16 else torch.float32

    def encode(self, X, want_residual=False, stages=None, codes=None):
        import torch
        N = X.shape[0]
        depth = self.cfg["depth"]
        sb, se = stages if stages is not None else (0, depth)
        if codes is None:
            codes = torch.empty((N, self.G, depth), dtype=torch.int16, device=X.device)
        std = (torch.empty((N,), dtype=self._std_torch_dtype(), device=X.device)
               if self.cfg["scale"] else None)
        res = (torch.empty((N, self.G, self.cfg["dhat"]), dtype=torch.float32, device=X.device)
               if want_residual else None)
        if N > rvq_reserved_rows(self.ctx):
            rvq_reserve(self.ctx, N)  # set-up call: grows the context's workspace
        rvq_encode(self.ctx, X, N, X.stride(0) if N else self.cfg["d"], sb, se, codes, std, res)
        return codes, std, res

    def decode(self, codes, std, depth_used=None, out=None):
        import torch
        N = codes.shape[0]
        if out is None:
            dt = torch.float16 if self.cfg["out_dtype"] == F16 else torch.float32
            out = torch.empty((N, self.cfg["d"]), dtype=dt, device=codes.device)
        rvq_decode(self.ctx, codes, std, N, depth_used or self.cfg["depth"], out,
                   out.stride(0) if N else self.cfg["d"])
        return out

    def decode_rope(self, codes, std, cos, sin, head_dim, depth_used=None, out=None):
        import torch
        N = codes.shape[0]
        if out is None:
            dt = torch.float16 if self.cfg["out_dtype"] == F16 else torch.float32
            out = torch.empty((N, self.cfg["d"]), dtype=dt, device=codes.device)
        rvq_decode_rope(self.ctx, codes, std, N, depth_used or self.cfg["depth"], cos, sin, head_dim,
                        out, out.stride(0) if N else self.cfg["d"])
        return out

    def pack(self, codes):
        import torch
        N = codes.shape[0]
        rec = rvq_packed_record_bytes(self.ctx)
        packed = torch.empty((N, self.G, rec), dtype=torch.uint8, device=codes.device)
        rvq_pack_codes(self.ctx, codes, N, packed)
        return packed

    def unpack(self, packed):
        import torch
        N = packed.shape[0]
        codes = torch.empty((N, self.G, self.cfg["depth"]), dtype=torch.int16, device=packed.device)
        rvq_unpack_codes(self.ctx, packed, N, codes)
        return codes

    def decode_packed(self, packed, std, depth_used=None, out=None):
        import torch
        N = packed.shape[0]
        if out is None:
            dt = torch.float16 if self.cfg["out_dtype"] == F16 else torch.float32
            out = torch.empty((N, self.cfg["d"]), dtype=dt, device=packed.device)
        rvq_decode_packed(self.ctx, packed, std, N, depth_used or self.cfg["depth"], out,
                          out.stride(0) if N else self.cfg["d"])
        return out

    def ema_update(self, stage, R, codes, cluster_size, embed_sum, decay=0.99, eps=1e-5,
                   code_stride=1):
        rvq_ema_update(self.ctx, stage, R, codes, code_stride, R.shape[0], decay, eps,
                       cluster_size, embed_sum)


# ---- rotary positions and the paged cache of 8-bit codes: tensors in, tensors out ---------------
# Checks of types, shapes and devices; sizes, strides and alignment are checked by the entry points.  The work goes to the
# current stream of the tensors' device.
_ELEMENTS = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _dtype(t, what):
    code = _ELEMENTS.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: fp32, bf16 or fp16 expected, got {t.dtype}")
    return code


def _whole(t, what, dtype, shape, device):
    """Address of a contiguous tensor of that type and shape on that device."""
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {dtype} {tuple(shape)} on {device} expected, got {t.dtype} "
                         f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr()


def _heads(t, what, heads, hd, device, rows=None):
    """Address, row and head stride of [rows][heads][hd] with neighbouring channels."""
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != hd or t.device != device or (rows is not None and shape[0] != rows):
        ok = False
    else:
        ld, hs, one = t.stride()
        ok = one == 1
    if not ok:
        raise ValueError(f"{what}: [{'rows' if rows is None else rows}][{heads}][{hd}] with neighbouring channels on "
                         f"{device} expected, got {tuple(shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr(), ld, hs


def _at(device, call, *args):
    """call(*args) with the device current in this thread, as the entry points want it.  (The interpreter's part of a small
    call is longer than its kernels: this lookup and the one of the stream are the cheap ones.)"""
    if torch._C._cuda_getDevice() == device.index:
        return call(*args)
    with torch.cuda.device(device.index):
        return call(*args)


def _run(device, call, *args):
    """The call on the device's current stream."""
    rc = _at(device, call, *args, torch._C._cuda_getCurrentRawStream(device.index))
    if rc != RVQ_OK:
        raise RvqError(rc)


def _on_gpu(device):
    if device.type != "cuda":
        raise ValueError(f"tensors on a GPU expected, got {device}")
    return device


def _tables(cos, sin, rows, device):
    """Addresses of the tables and the channels that they rotate."""
    if cos is None or sin is None:
        if cos is not sin:
            raise ValueError("cos and sin belong together")
        return None, None, 0
    shape = (rows, cos.shape[-1])
    return (_whole(cos, "cos", torch.float32, shape, device), _whole(sin, "sin", torch.float32, shape, device), 2 * shape[1])


def rope_tables(positions, rot, base=10000.0, factor=1.0, orig_len=0.0, alpha=1.0, beta=32.0, amplitude=1.0, out=None):
    """cos, sin, fp32 [N][rot / 2], of int64 positions [N] (rvq_rope_tables); out: a pair of such tensors."""
    dev = _on_gpu(positions.device)
    shape = (positions.numel(), max(rot, 0) // 2)
    p = _whole(positions, "positions", torch.int64, shape[:1], dev)
    if out is None:
        cos, sin = torch.empty((2, *shape), dtype=torch.float32, device=dev).unbind()
        pc, ps = cos.data_ptr(), sin.data_ptr()
    else:
        cos, sin = out
        pc, ps = _whole(cos, "out", torch.float32, shape, dev), _whole(sin, "out", torch.float32, shape, dev)
    _run(dev, lib.rvq_rope_tables, p, shape[0], rot, base, factor, orig_len, alpha, beta, amplitude, pc, ps)
    return cos, sin


def rope(x, cos, sin, layout=ROPE_ADJACENT, out=None):
    """Head vectors x [N][heads][head_dim] with the first 2 * cos.shape[1] channels of each rotated (rvq_rope).
    out: a tensor like x, x itself to rotate in place; rows and heads may be strided in both."""
    dtype, dev = _dtype(x, "x"), _on_gpu(x.device)
    if x.dim() != 3:
        raise ValueError(f"x: [rows][heads][head_dim] expected, got {tuple(x.shape)}")
    N, heads, hd = x.shape
    px, ldx, hsx = _heads(x, "x", heads, hd, dev)
    c, s, rot = _tables(cos, sin, N, dev)
    if out is None:
        out = torch.empty((N, heads, hd), dtype=x.dtype, device=dev)
        po, ldo, hso = out.data_ptr(), heads * hd, hd
    elif out.dtype != x.dtype:
        raise ValueError(f"out: {x.dtype} expected, got {out.dtype}")
    else:
        po, ldo, hso = _heads(out, "out", heads, hd, dev, N)
    _run(dev, lib.rvq_rope, px, dtype, N, heads, hd, rot, layout, ldx, hsx, c, s, po, ldo, hso)
    return out


class Cache8:
    """Paged cache of keys and values in 8 bits (rvq_cache8): owns, or is given, the codes `pages`, uint8
    [n_pages][n_kv_heads][2][64 * head_dim], and `scales`, fp32 [n_pages][n_kv_heads][2].

    A step brings rows cu[b] .. cu[b + 1] of sequence b; `lengths` counts every sequence's tokens with them, `table`
    [sequences][entries] names its pages.  All three are int32 tensors on the device, so that a captured step can be
    replayed with other lengths and pages.  Which pages are free is the caller's business."""

    def __init__(self, pages, scales):
        shape = pages.shape
        if len(shape) != 4 or shape[2] != 2 or shape[3] % PAGE_TOKENS:
            raise ValueError(f"pages: [n_pages][n_kv_heads][2][{PAGE_TOKENS} * head_dim] expected, got {tuple(shape)}")
        self.device = pages.device
        self.n_pages, self.n_kv_heads, _, size = shape
        self.head_dim = size // PAGE_TOKENS
        self.pages, self.scales = pages, scales
        self._pool = (_whole(pages, "pages", torch.uint8, shape, self.device),
                      _whole(scales, "scales", torch.float32, shape[:3], self.device), self.n_pages, self.n_kv_heads, self.head_dim)

    @classmethod
    def empty(cls, n_pages, n_kv_heads, head_dim, device="cuda"):
        shape = (n_pages, n_kv_heads, 2, PAGE_TOKENS * head_dim)
        return cls(torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(shape[:3], dtype=torch.float32, device=device))

    def _step(self, cu, table, lengths):
        dev = _on_gpu(self.device)
        shape = table.shape
        if len(shape) != 2:
            raise ValueError(f"table: [sequences][entries] expected, got {tuple(shape)}")
        n = shape[0]
        view = rvq_cache8(*self._pool, _whole(table, "table", torch.int32, shape, dev), shape[1], n,
                          _whole(lengths, "lengths", torch.int32, (n,), dev))
        return view, _whole(cu, "cu", torch.int32, (n + 1,), dev)

    def append(self, k, v, cu, table, lengths, cos=None, sin=None, layout=ROPE_ADJACENT):
        """Stores the step's keys, rotated when tables are given, and values, [rows][n_kv_heads][head_dim] (rvq_cache8_append)."""
        dtype, rows, dev = _dtype(k, "k"), k.shape[0], self.device
        if v.dtype != k.dtype:
            raise ValueError(f"v: {k.dtype} expected, got {v.dtype}")
        view, pcu = self._step(cu, table, lengths)
        pk, ldk, hsk = _heads(k, "k", self.n_kv_heads, self.head_dim, dev)
        pv, ldv, hsv = _heads(v, "v", self.n_kv_heads, self.head_dim, dev, rows)
        c, s, rot = _tables(cos, sin, rows, dev)
        _run(dev, lib.rvq_cache8_append, view, pk, pv, dtype, rows, ldk, hsk, ldv, hsv, pcu, c, s, rot, layout)

    def read(self, rows, cu, first, table, lengths, dtype=torch.float16, cos=None, sin=None, layout=ROPE_ADJACENT, out=None):
        """k, v [rows][n_kv_heads][head_dim]: row cu[b] + i is the token of sequence b at position first[b] + i; with
        tables, keys as they were before the rotation (rvq_cache8_read).  out: a pair of such tensors."""
        dev = self.device
        view, pcu = self._step(cu, table, lengths)
        pf = _whole(first, "first", torch.int32, lengths.shape, dev)
        c, s, rot = _tables(cos, sin, rows, dev)
        if out is None:
            out = torch.empty((2, rows, self.n_kv_heads, self.head_dim), dtype=dtype, device=dev).unbind()
        k, v = out
        code = _dtype(k, "out")
        if v.dtype != k.dtype:
            raise ValueError(f"out: one type expected, got {k.dtype} and {v.dtype}")
        pk, ldk, hsk = _heads(k, "out", self.n_kv_heads, self.head_dim, dev, rows)
        pv, ldv, hsv = _heads(v, "out", self.n_kv_heads, self.head_dim, dev, rows)
        _run(dev, lib.rvq_cache8_read, view, pcu, pf, rows, c, s, rot, layout, code, pk, ldk, hsk, pv, ldv, hsv)
        return k, v

    def workspace_bytes(self, q, n_seqs):
        """Bytes of workspace that attend() needs for queries of that shape and type from so many sequences."""
        view = rvq_cache8(*self._pool, None, 1, n_seqs, None)  # the rest of the step does not matter
        return _at(_on_gpu(self.device), lib.rvq_cache8_attn_workspace_bytes, view, _dtype(q, "q"), q.shape[0], q.shape[1])

    def attend(self, q, cu, table, lengths, scale=None, window=0, sinks=0, out=None, workspace=None):
        """Attention of the step's query tokens q [rows][heads][head_dim], already rotated, over the cache (rvq_cache8_attn).
        scale: 1 / sqrt(head_dim) if not given; workspace: uint8, at least workspace_bytes(), allocated if not given."""
        dtype, dev = _dtype(q, "q"), self.device
        if q.dim() != 3:
            raise ValueError(f"q: [rows][heads][head_dim] expected, got {tuple(q.shape)}")
        if window > MOST_TOKENS or sinks > MOST_TOKENS:  # 32 bits would make another number of it
            raise ValueError(f"window and sinks up to {MOST_TOKENS} expected, got {window} and {sinks}")
        view, pcu = self._step(cu, table, lengths)
        rows, heads, hd = q.shape
        pq, ldq, hsq = _heads(q, "q", heads, self.head_dim, dev)
        if out is None:
            out = torch.empty((rows, heads, hd), dtype=q.dtype, device=dev)
            po, ldo, hso = out.data_ptr(), heads * hd, hd
        elif out.dtype != q.dtype:
            raise ValueError(f"out: {q.dtype} expected, got {out.dtype}")
        else:
            po, ldo, hso = _heads(out, "out", heads, hd, dev, rows)
        if workspace is None:
            size = _at(dev, lib.rvq_cache8_attn_workspace_bytes, view, dtype, rows, heads)
            workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        pw = _whole(workspace, "workspace", torch.uint8, workspace.shape, dev)
        _run(dev, lib.rvq_cache8_attn, view, pq, dtype, rows, heads, ldq, hsq, pcu, scale if scale is not None else hd**-0.5,
             window, sinks, po, ldo, hso, pw, workspace.numel())
        return out
