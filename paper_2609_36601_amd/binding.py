"""ctypes binding of libsaki.so (include/saki.h, saki_kv.h, saki_distill.h).

Argument marshalling only: every step of the path runs in the HIP library.
Tensors are torch device tensors; the library sees their data pointers and the
current torch stream.  If the built library is missing the binding raises; it
has no fallback.
"""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsaki.so")

SAKI_F32, SAKI_BF16 = 0, 1
SAKI_OP_COUPLE, SAKI_OP_ROUTE, SAKI_OP_VERIFY, SAKI_OP_SELECT = 0, 1, 2, 3
SAKI_OP_KV_RESERVE, SAKI_OP_KV_COMPACT, SAKI_OP_KV_ATTENTION = 4, 5, 6
SAKI_OP_TOP_LOGITS, SAKI_OP_DISTILL_TOP = 7, 8
SAKI_TARGET_MODE, SAKI_TARGET_SAMPLE = 0, 1
SAKI_KL_FORWARD, SAKI_KL_REVERSE = 0, 1
SAKI_SELECT_RANDOM, SAKI_SELECT_TV_WEIGHTED = 0, 1
SAKI_MAX_VOCAB = 1 << 21
SAKI_STATIC_MAX_ROWS = 262144
SAKI_CHUNK = 1024
ROW_OK, ROW_NONFINITE, ROW_BAD_DRAFT, ROW_SKIPPED, ROW_BAD_TARGET = 0, 1, 2, 3, 4

STATUS = {0: "SAKI_OK", 1: "SAKI_E_NULLPTR", 2: "SAKI_E_SHAPE", 3: "SAKI_E_VALUE",
          4: "SAKI_E_DTYPE", 5: "SAKI_E_ALIGN", 6: "SAKI_E_WORKSPACE", 7: "SAKI_E_DEVICE",
          8: "SAKI_E_LAUNCH"}

EXPORTED = ["saki_workspace_bytes", "saki_couple", "saki_couple_static", "saki_route_loss", "saki_spec_verify",
            "saki_select_positions", "saki_probe_metrics", "saki_sample", "saki_commit",
            "saki_status_str", "saki_last_error"]
EXPORTED_KV = ["saki_kv_reserve", "saki_kv_commit", "saki_kv_fork", "saki_kv_compact", "saki_kv_append",
               "saki_kv_attention"]  # of include/saki_kv.h
EXPORTED_DISTILL = ["saki_top_logits", "saki_distill_top", "saki_linear_ce",
                    "saki_linear_ce_workspace_bytes"]  # of include/saki_distill.h
SAKI_MAX_TOP_K, SAKI_MAX_HIDDEN = 256, 65536
KV_OK, KV_NO_PAGES, KV_TOO_LONG, KV_BAD = 0, 1, 2, 3
SEQ_RUNNING, SEQ_FINISHED, SEQ_STOPPED = 0, 1, 2
SAKI_MAX_PROBE_K = 64


class SakiRows(ctypes.Structure):
    _fields_ = [("student", ctypes.c_void_p), ("teacher", ctypes.c_void_p),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("n_rows", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("row_stride", ctypes.c_int64), ("row_offset", ctypes.c_int64)]


COUPLE_FLOAT_FIELDS = ["lambda", "kl", "tv", "accept_prob", "margin", "logp_token",
                       "logt_token", "logq_token"]
COUPLE_INT_FIELDS = ["proposal", "token", "teacher_argmax", "target"]
COUPLE_U8_FIELDS = ["corrected", "row_status"]
# struct order of saki_couple_out
COUPLE_FIELDS = COUPLE_FLOAT_FIELDS + ["proposal", "token", "teacher_argmax"] + COUPLE_U8_FIELDS + ["target"]


class SakiCoupleOut(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in COUPLE_FIELDS]


class SakiRouteArgs(ctypes.Structure):
    _fields_ = [("valid_mask", ctypes.c_void_p), ("grad_scale", ctypes.c_float),
                ("grad_dtype", ctypes.c_int32), ("row_loss", ctypes.c_void_p),
                ("loss_sum", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("grad_stride", ctypes.c_int64), ("correction_target", ctypes.c_int32)]


# struct order of saki_traj after (n_seq, max_len)
TRAJ_FIELDS = ["tokens", "corrected", "lambda", "kl", "tv", "logp_token", "logt_token",
               "teacher_argmax", "length", "done"]
TRAJ_DTYPES = dict(tokens=torch.int32, corrected=torch.uint8, teacher_argmax=torch.int32,
                   length=torch.int32, done=torch.uint8)


class SakiTraj(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int64), ("max_len", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in TRAJ_FIELDS]


class SakiKVTable(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("n_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("pages", "length", "held", "refs")]


class SakiKVPool(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_int64) for n in ("n_layers", "layer_stride", "page_stride", "head_stride",
                                              "token_stride")]


class SakiKVTokens(ctypes.Structure):
    _fields_ = [("offsets", ctypes.c_void_p), ("n_tokens", ctypes.c_int64), ("n_new", ctypes.c_int32),
                ("shift", ctypes.c_int32)]


class SakiKVHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class SakiKVRope(ctypes.Structure):
    _fields_ = [("freq", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("amplitude", ctypes.c_float)]


class SakiTopList(ctypes.Structure):
    _fields_ = [("token", ctypes.c_void_p), ("logit", ctypes.c_void_p), ("rest_logit", ctypes.c_void_p),
                ("stride", ctypes.c_int64), ("k", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class SakiHead(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("hidden_stride", ctypes.c_int64),
                ("weight_stride", ctypes.c_int64), ("n_rows", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("hidden_size", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class SakiCEArgs(ctypes.Structure):
    _fields_ = [("token", ctypes.c_void_p), ("row_weight", ctypes.c_void_p), ("valid_mask", ctypes.c_void_p),
                ("grad_scale", ctypes.c_float), ("reserved", ctypes.c_uint32)] + \
               [(n, ctypes.c_void_p) for n in ("row_loss", "logp_token", "loss_sum", "row_status", "grad_hidden",
                                               "grad_weight")] + \
               [("grad_hidden_stride", ctypes.c_int64), ("grad_weight_stride", ctypes.c_int64)]


class SakiError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__(f"{STATUS.get(status, status)}: {detail}")
        self.status = status


_lib = None


def load(path=LIB_PATH):
    """Load libsaki.so once and declare its C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libsaki.so not built at {path}; run __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    lib.saki_workspace_bytes.restype = ctypes.c_size_t
    lib.saki_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_int64, ctypes.c_int64]
    lib.saki_couple.restype = ctypes.c_int
    lib.saki_couple.argtypes = [ctypes.POINTER(SakiRows), ctypes.c_double, ctypes.c_uint64,
                                ctypes.POINTER(SakiCoupleOut), ctypes.POINTER(SakiRouteArgs),
                                ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.saki_couple_static.restype = ctypes.c_int
    lib.saki_couple_static.argtypes = [ctypes.POINTER(SakiRows), ctypes.c_double, ctypes.c_uint64,
                                       ctypes.POINTER(SakiCoupleOut), ctypes.POINTER(SakiRouteArgs),
                                       ctypes.c_void_p]
    lib.saki_route_loss.restype = ctypes.c_int
    lib.saki_route_loss.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64,
                                    ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.POINTER(SakiRouteArgs), ctypes.c_void_p,
                                    ctypes.c_size_t, ctypes.c_void_p]
    lib.saki_spec_verify.restype = ctypes.c_int
    lib.saki_spec_verify.argtypes = [ctypes.POINTER(SakiRows), ctypes.c_int32, ctypes.c_void_p,
                                     ctypes.c_double, ctypes.c_uint64, ctypes.c_int32,
                                     ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.POINTER(SakiCoupleOut), ctypes.c_void_p,
                                     ctypes.c_size_t, ctypes.c_void_p]
    lib.saki_select_positions.restype = ctypes.c_int
    lib.saki_select_positions.argtypes = [ctypes.c_int32, ctypes.c_int64, ctypes.c_int64,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int64,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                          ctypes.c_void_p]
    lib.saki_probe_metrics.restype = ctypes.c_int
    lib.saki_probe_metrics.argtypes = [ctypes.POINTER(SakiRows), ctypes.c_int32, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.saki_sample.restype = ctypes.c_int
    lib.saki_sample.argtypes = [ctypes.POINTER(SakiRows), ctypes.c_int64, ctypes.c_uint64,
                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.saki_commit.restype = ctypes.c_int
    lib.saki_commit.argtypes = [ctypes.POINTER(SakiTraj), ctypes.c_int32, ctypes.c_int32,
                                ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(SakiCoupleOut),
                                ctypes.c_void_p, ctypes.c_void_p]
    P, I32, I64 = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64
    ptr, size = ctypes.c_void_p, ctypes.c_size_t
    for name, args in (
            ("reserve", [P(SakiKVTable), P(SakiKVPool), ptr, I32, ptr, ptr, size, ptr]),
            ("commit", [P(SakiKVTable), ptr, ptr, ptr, ptr]),
            ("fork", [P(SakiKVTable), I64, ptr, ptr, ptr, ptr]),
            ("compact", [P(SakiKVTable), P(SakiKVPool), ptr, ptr, size, ptr]),
            ("append", [P(SakiKVTable), P(SakiKVPool), I64, P(SakiKVTokens), P(SakiKVRope), I32] +
             [P(SakiKVHeads)] * 4 + [ptr]),
            ("attention", [P(SakiKVTable), P(SakiKVPool), I64, P(SakiKVTokens), I32, P(SakiKVHeads), P(SakiKVHeads), ptr,
                           ctypes.c_float, I32, I32, ptr, size, ptr])):
        f = getattr(lib, "saki_kv_" + name)
        f.restype, f.argtypes = ctypes.c_int, args
    F32 = ctypes.c_float
    for name, args in (
            ("top_logits", [ptr, I32, I64, I64, I64, I32, F32, ptr, ptr, I64, ptr, ptr, ptr, size, ptr]),
            ("distill_top", [ptr, I32, I64, I64, I64, P(SakiTopList), F32, I32, ptr, F32, ptr, ptr, ptr, I32, I64, ptr, ptr,
                             size, ptr]),
            ("linear_ce", [P(SakiHead), P(SakiCEArgs), ptr, size, ptr])):
        f = getattr(lib, "saki_" + name)
        f.restype, f.argtypes = ctypes.c_int, args
    lib.saki_linear_ce_workspace_bytes.restype = size
    lib.saki_linear_ce_workspace_bytes.argtypes = [P(SakiHead), I32]
    lib.saki_status_str.restype = ctypes.c_char_p
    lib.saki_status_str.argtypes = [ctypes.c_int]
    lib.saki_last_error.restype = ctypes.c_char_p
    lib.saki_last_error.argtypes = []
    _lib = lib
    return lib


def _check(status):
    if status != 0:
        raise SakiError(status, _lib.saki_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dense(*ts):
    """Per-row arrays are passed as bare pointers: they must be contiguous."""
    for t in ts:
        if t is not None and not t.is_contiguous():
            raise ValueError("per-row arrays must be contiguous tensors")


def _dtype_code(dt):
    if dt == torch.float32:
        return SAKI_F32
    if dt == torch.bfloat16:
        return SAKI_BF16
    raise ValueError(f"unsupported dtype {dt}")


def _stream(stream):
    if stream is None:  # (the handle without a Stream object around it: 1.4 us a call, 0.4 without)
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def _rows(student, teacher, row_offset):
    assert student.dim() == 2 and student.shape == teacher.shape
    assert student.dtype == teacher.dtype and student.stride() == teacher.stride()
    assert student.stride(1) == 1
    return SakiRows(_ptr(student), _ptr(teacher), _dtype_code(student.dtype), 0,
                    student.shape[0], student.shape[1], student.stride(0), row_offset)


def workspace_bytes(op, n_rows, vocab):
    load()
    return int(_lib.saki_workspace_bytes(op, n_rows, vocab))


def alloc_rows(n_rows, vocab, dtype, device):
    """[n_rows, vocab] tensor whose row pitch is a multiple of 16 bytes (the ABI's layout rule)."""
    per = 16 // torch.tensor([], dtype=dtype).element_size()
    pitch = (vocab + per - 1) // per * per
    return torch.empty(n_rows, pitch, dtype=dtype, device=device)[:, :vocab]


def alloc_couple_out(n_rows, device, fields=COUPLE_FIELDS):
    out = {}
    for f in fields:
        if f in COUPLE_FLOAT_FIELDS:
            out[f] = torch.empty(n_rows, dtype=torch.float32, device=device)
        elif f in COUPLE_INT_FIELDS:
            out[f] = torch.empty(n_rows, dtype=torch.int32, device=device)
        else:
            out[f] = torch.empty(n_rows, dtype=torch.uint8, device=device)
    return out


def _couple_struct(out):
    return SakiCoupleOut(*[_ptr(out.get(f)) for f in COUPLE_FIELDS])


def _route_struct(valid_mask, grad_scale, row_loss, loss_sum, grad, correction_target=SAKI_TARGET_MODE):
    gdt = _dtype_code(grad.dtype) if grad is not None else SAKI_F32
    gstride = grad.stride(0) if grad is not None else 0
    return SakiRouteArgs(_ptr(valid_mask), float(grad_scale), gdt, _ptr(row_loss),
                         _ptr(loss_sum), _ptr(grad), gstride, int(correction_target))


def saki_couple(student, teacher, eps, seed, row_offset=0, out=None, route=None,
                workspace=None, stream=None):
    """Call saki_couple on preallocated buffers.

    out:   dict field -> tensor (missing fields are not written)
    route: None, or dict with optional keys valid_mask, grad_scale, row_loss,
           loss_sum (float64 tensor of 1), grad (2-D float32/bfloat16 tensor),
           correction_target (SAKI_TARGET_MODE or SAKI_TARGET_SAMPLE).
    """
    load()
    rows = _rows(student, teacher, row_offset)
    co = _couple_struct(out or {})
    rt = None
    if route is not None:
        rt = _route_struct(route.get("valid_mask"), route.get("grad_scale", 1.0),
                           route.get("row_loss"), route.get("loss_sum"), route.get("grad"),
                           route.get("correction_target", SAKI_TARGET_MODE))
    ws_b = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.saki_couple(ctypes.byref(rows), float(eps), int(seed) & (2**64 - 1),
                          ctypes.byref(co), ctypes.byref(rt) if rt is not None else None,
                          _ptr(workspace), ws_b, _stream(stream))
    _check(st)


def saki_couple_static(student, teacher, eps, seed, row_offset=0, out=None, route=None, stream=None):
    """Call saki_couple_static (no workspace: the library's static scratch) on
    preallocated buffers; out and route as for saki_couple."""
    load()
    rows = _rows(student, teacher, row_offset)
    co = _couple_struct(out or {})
    rt = None
    if route is not None:
        rt = _route_struct(route.get("valid_mask"), route.get("grad_scale", 1.0),
                           route.get("row_loss"), route.get("loss_sum"), route.get("grad"),
                           route.get("correction_target", SAKI_TARGET_MODE))
    st = _lib.saki_couple_static(ctypes.byref(rows), float(eps), int(seed) & (2**64 - 1),
                                 ctypes.byref(co), ctypes.byref(rt) if rt is not None else None,
                                 _stream(stream))
    _check(st)


def saki_route_loss(student, token, corrected, teacher_argmax, advantage, valid_mask=None,
                    grad_scale=1.0, row_loss=None, loss_sum=None, grad=None, workspace=None,
                    stream=None):
    load()
    rt = _route_struct(valid_mask, grad_scale, row_loss, loss_sum, grad)
    ws_b = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.saki_route_loss(_ptr(student), _dtype_code(student.dtype), student.shape[0],
                              student.shape[1], student.stride(0), _ptr(token), _ptr(corrected),
                              _ptr(teacher_argmax), _ptr(advantage), ctypes.byref(rt),
                              _ptr(workspace), ws_b, _stream(stream))
    _check(st)


def saki_spec_verify(student, teacher, k, draft, eps, seed, row_offset=0, eos_id=-1,
                     accepted_len=None, correction=None, per_pos=None, workspace=None,
                     stream=None):
    load()
    rows = _rows(student, teacher, row_offset)
    pp = _couple_struct(per_pos) if per_pos is not None else None
    ws_b = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.saki_spec_verify(ctypes.byref(rows), int(k), _ptr(draft), float(eps),
                               int(seed) & (2**64 - 1), int(eos_id), _ptr(accepted_len),
                               _ptr(correction), ctypes.byref(pp) if pp is not None else None,
                               _ptr(workspace), ws_b, _stream(stream))
    _check(st)


# ---------------------------------------------------------------------------
# Convenience wrappers that allocate their outputs (tests, examples).
# ---------------------------------------------------------------------------
def couple(student, teacher, eps, seed, row_offset=0, route=False, grad_dtype=None,
           valid_mask=None, grad_scale=1.0, correction_target=SAKI_TARGET_MODE, stream=None):
    n, V = student.shape
    dev = student.device
    out = alloc_couple_out(n, dev)
    rargs = None
    if route:
        rargs = dict(valid_mask=valid_mask, grad_scale=grad_scale,
                     row_loss=torch.empty(n, dtype=torch.float32, device=dev),
                     loss_sum=torch.empty(1, dtype=torch.float64, device=dev),
                     correction_target=correction_target)
        if grad_dtype is not None:
            rargs["grad"] = alloc_rows(n, V, grad_dtype, dev)
    ws = torch.empty(max(workspace_bytes(SAKI_OP_COUPLE, n, V), 8), dtype=torch.uint8, device=dev)
    saki_couple(student, teacher, eps, seed, row_offset, out, rargs, ws, stream)
    if rargs is not None:
        out.update({k: v for k, v in rargs.items() if k in ("row_loss", "loss_sum", "grad")})
    return out


def route_loss(student, token, corrected, teacher_argmax, advantage, valid_mask=None,
               grad_scale=1.0, grad_dtype=torch.float32, stream=None):
    n, V = student.shape
    dev = student.device
    row_loss = torch.empty(n, dtype=torch.float32, device=dev)
    loss_sum = torch.empty(1, dtype=torch.float64, device=dev)
    grad = alloc_rows(n, V, grad_dtype, dev) if grad_dtype is not None else None
    ws = torch.empty(max(workspace_bytes(SAKI_OP_ROUTE, n, V), 8), dtype=torch.uint8, device=dev)
    saki_route_loss(student, token, corrected, teacher_argmax, advantage, valid_mask, grad_scale,
                    row_loss, loss_sum, grad, ws, stream)
    return dict(row_loss=row_loss, loss_sum=loss_sum, grad=grad)


def spec_verify(student, teacher, k, draft, eps, seed, row_offset=0, eos_id=-1, per_pos=True,
                stream=None):
    n, V = student.shape
    dev = student.device
    nb = n // k
    acc = torch.empty(nb, dtype=torch.int32, device=dev)
    corr = torch.empty(nb, dtype=torch.int32, device=dev)
    pp = alloc_couple_out(n, dev) if per_pos else None
    ws = torch.empty(max(workspace_bytes(SAKI_OP_VERIFY, n, V), 8), dtype=torch.uint8, device=dev)
    saki_spec_verify(student, teacher, k, draft, eps, seed, row_offset, eos_id, acc, corr, pp,
                     ws, stream)
    out = dict(accepted_len=acc, correction=corr)
    if pp is not None:
        out["per_pos"] = pp
    return out


def saki_select_positions(mode, traj_offsets, tv, corrected, selected, seed, valid_mask=None,
                          row_offset=0, workspace=None, stream=None):
    """Call saki_select_positions on preallocated buffers (traj_offsets: int64 [n_traj + 1])."""
    load()
    n_traj = traj_offsets.numel() - 1
    n_rows = tv.numel()
    ws_b = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.saki_select_positions(int(mode), n_traj, n_rows, _ptr(traj_offsets), _ptr(tv),
                                    _ptr(corrected), _ptr(valid_mask), int(seed) & (2**64 - 1),
                                    int(row_offset), _ptr(selected), _ptr(workspace), ws_b,
                                    _stream(stream))
    _check(st)


def select_positions(mode, traj_offsets, tv, corrected, seed, valid_mask=None, row_offset=0,
                     stream=None):
    """Placement-control selection mask (uint8 [n_rows]); allocates its output and workspace."""
    n = tv.numel()
    sel = torch.empty(n, dtype=torch.uint8, device=tv.device)
    ws = torch.empty(max(workspace_bytes(SAKI_OP_SELECT, n, 0), 8), dtype=torch.uint8,
                     device=tv.device)
    saki_select_positions(mode, traj_offsets, tv, corrected, sel, seed, valid_mask, row_offset, ws,
                          stream)
    return sel


def saki_probe_metrics(student, teacher, k, c1=None, ck=None, kl_ts=None, entropy=None, topk=None,
                       row_status=None, stream=None):
    """Call saki_probe_metrics on preallocated outputs (any may be None)."""
    load()
    rows = _rows(student, teacher, 0)
    st = _lib.saki_probe_metrics(ctypes.byref(rows), int(k), _ptr(c1), _ptr(ck), _ptr(kl_ts),
                                 _ptr(entropy), _ptr(topk), _ptr(row_status), _stream(stream))
    _check(st)


def probe_metrics(student, teacher, k=16, stream=None):
    """Probe metrics per row; allocates its outputs."""
    n = student.shape[0]
    dev = student.device
    out = dict(c1=torch.empty(n, dtype=torch.float32, device=dev),
               ck=torch.empty(n, dtype=torch.float32, device=dev),
               kl_ts=torch.empty(n, dtype=torch.float32, device=dev),
               entropy=torch.empty(n, dtype=torch.float32, device=dev),
               topk=torch.empty(n, k, dtype=torch.int32, device=dev),
               row_status=torch.empty(n, dtype=torch.uint8, device=dev))
    saki_probe_metrics(student, teacher, k, stream=stream, **out)
    return out


def saki_sample(student, token, seed, row_offset=0, row_step=1, row_status=None, stream=None):
    """Call saki_sample: token[r] ~ softmax(student[r]) keyed by row_offset + r * row_step.

    student is a [n_rows, V] tensor whose rows may be strided (stride(1) == 1)."""
    load()
    assert student.dim() == 2 and student.stride(1) == 1
    _dense(token, row_status)
    rows = SakiRows(_ptr(student), None, _dtype_code(student.dtype), 0, student.shape[0],
                    student.shape[1], student.stride(0), int(row_offset))
    st = _lib.saki_sample(ctypes.byref(rows), int(row_step), int(seed) & (2**64 - 1), _ptr(token),
                          _ptr(row_status), _stream(stream))
    _check(st)


def sample(student, seed, row_offset=0, row_step=1, stream=None):
    """Draws one token per row; allocates token (int32) and row_status (uint8)."""
    n = student.shape[0]
    tok = torch.empty(n, dtype=torch.int32, device=student.device)
    status = torch.empty(n, dtype=torch.uint8, device=student.device)
    saki_sample(student, tok, seed, row_offset, row_step, status, stream)
    return tok, status


def alloc_traj(n_seq, max_len, device, fields=TRAJ_FIELDS):
    """Trajectory buffers: tokens -1, float metadata NaN, length 0, done running."""
    out = {}
    for f in fields:
        dt = TRAJ_DTYPES.get(f, torch.float32)
        shape = (n_seq,) if f in ("length", "done") else (n_seq, max_len)
        if f == "tokens" or f == "teacher_argmax":
            out[f] = torch.full(shape, -1, dtype=dt, device=device)
        elif dt == torch.float32:
            out[f] = torch.full(shape, float("nan"), dtype=dt, device=device)
        else:
            out[f] = torch.zeros(shape, dtype=dt, device=device)
    return out


def saki_commit(traj, max_len, k, eos_id, accepted_len, correction, per_pos, n_commit=None,
                stream=None):
    """Call saki_commit on trajectory buffers `traj` (dict of TRAJ_FIELDS tensors)."""
    load()
    _dense(*traj.values(), accepted_len, correction, n_commit, *per_pos.values())
    n_seq = traj["length"].numel()
    tr = SakiTraj(n_seq, int(max_len), *[_ptr(traj.get(f)) for f in TRAJ_FIELDS])
    pp = _couple_struct(per_pos)
    st = _lib.saki_commit(ctypes.byref(tr), int(k), int(eos_id), _ptr(accepted_len),
                          _ptr(correction), ctypes.byref(pp), _ptr(n_commit), _stream(stream))
    _check(st)


# ---------------------------------------------------------------------------
# Paged key-value caches.  Tables and pools are described once (kv_table, kv_pool)
# and used by many calls; cache.PagedKV holds both and allocates outputs and workspaces.
# ---------------------------------------------------------------------------
def _want(name, t, dtype, shape, device):
    """A dense tensor of this type, shape and device."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}: got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")


def kv_table(pages, length, held, refs, page_size):
    """Descriptor of a table (int32 tensors pages [n_seq, max_pages], length and held [n_seq], refs [n_pages])."""
    n_seq, max_pages = pages.shape
    for name, t, shape in (("pages", pages, (n_seq, max_pages)), ("length", length, (n_seq,)), ("held", held, (n_seq,)),
                           ("refs", refs, (refs.numel(),))):
        _want(name, t, torch.int32, shape, pages.device)
    return SakiKVTable(n_seq, max_pages, refs.numel(), page_size, 0, _ptr(pages), _ptr(length), _ptr(held), _ptr(refs))


def kv_pool(k, v):
    """Descriptor of a pool: k and v [n_layers, n_pages, n_kv_heads, page_size, head_dim] of equal strides."""
    if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.stride() != v.stride():
        raise ValueError("k and v must be [n_layers, n_pages, n_kv_heads, page_size, head_dim] tensors alike")
    if k.stride(4) != 1:
        raise ValueError("the elements of a head must be consecutive")
    s = k.stride()
    return SakiKVPool(_ptr(k), _ptr(v), _dtype_code(k.dtype), k.shape[2], k.shape[4], 0, k.shape[0], s[0], s[1], s[2], s[3])


def _heads(t):
    """Reference to the descriptor of a token array, or None."""
    if t is None:
        return None
    stride = t.stride()
    if len(stride) != 3 or stride[2] != 1:
        raise ValueError("token arrays must be [n_tokens, heads, head_dim] with consecutive elements of a head")
    return ctypes.byref(SakiKVHeads(t.data_ptr(), stride[0], stride[1]))


def _ref(s):
    return None if s is None else ctypes.byref(s)


def _addr(t):
    """A tensor's address for a void * argument (declared as such: a number will do), or None."""
    return None if t is None else t.data_ptr()


def _ws_bytes(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


def saki_kv_reserve(table, pool, n_new, status=None, workspace=None, stream=None):
    """Call saki_kv_reserve; n_new: an int32 tensor [n_seq], or one number for every sequence."""
    _lib or load()
    each = isinstance(n_new, torch.Tensor)
    _dense(n_new if each else None, status, workspace)
    if not each and not 0 <= n_new < 2**31:
        raise ValueError("n_new outside [0, 2^31)")
    _check(_lib.saki_kv_reserve(_ref(table), _ref(pool), _addr(n_new) if each else None, 0 if each else int(n_new),
                                _addr(status), _addr(workspace), _ws_bytes(workspace), _stream(stream)))


def saki_kv_commit(table, delta, done=None, status=None, stream=None):
    _lib or load()
    _dense(delta, done, status)
    _check(_lib.saki_kv_commit(_ref(table), _addr(delta), _addr(done), _addr(status), _stream(stream)))


def saki_kv_fork(table, src, dst, status=None, stream=None):
    _lib or load()
    _dense(src, dst, status)
    _check(_lib.saki_kv_fork(_ref(table), src.numel(), _addr(src), _addr(dst), _addr(status), _stream(stream)))


def saki_kv_compact(table, pool, n_live=None, workspace=None, stream=None):
    _lib or load()
    _dense(n_live, workspace)
    _check(_lib.saki_kv_compact(_ref(table), _ref(pool), _addr(n_live), _addr(workspace), _ws_bytes(workspace),
                                _stream(stream)))


def saki_kv_append(table, pool, layer, tokens, k, v, q=None, q_out=None, rope=None, stream=None):
    """Call saki_kv_append; tokens: a SakiKVTokens, rope: a SakiKVRope or None."""
    _lib or load()
    _check(_lib.saki_kv_append(_ref(table), _ref(pool), int(layer), _ref(tokens), _ref(rope),
                               0 if q is None else q.shape[1], _heads(q), _heads(q_out), _heads(k), _heads(v), _stream(stream)))


def saki_kv_attention(table, pool, layer, tokens, q, out, lse=None, scale=1.0, window=0, sinks=0, workspace=None,
                      stream=None):
    _lib or load()
    _dense(lse, workspace)
    for name, x in (("window", window), ("sinks", sinks)):
        if not 0 <= x < 2**31:
            raise ValueError(f"{name} outside [0, 2^31)")
    _check(_lib.saki_kv_attention(_ref(table), _ref(pool), int(layer), _ref(tokens), q.shape[1], _heads(q), _heads(out),
                                  _addr(lse), float(scale), int(window), int(sinks), _addr(workspace),
                                  _ws_bytes(workspace), _stream(stream)))


# ---------------------------------------------------------------------------
# A teacher's top logits, distillation from them, cross entropy from hidden states.
# ---------------------------------------------------------------------------
def _hold(stream, *tensors):
    """What a call on `stream` reads or writes stays allocated until it has run, also if the caller lets go of it."""
    for t in tensors:
        if t is not None and t.is_cuda and t.device == stream.device:
            t.record_stream(stream)


def _on(device, stream, **tensors):
    """The arguments of one call lie on one device, the current one, and take no part in autograd; those of a call on a
    stream that is named are held for it."""
    for name, t in tensors.items():
        if t is None:
            continue
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, the call's first tensor on {device}")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which this call does not record: pass it detached (gradients "
                             "are outputs)")
    if device.type != "cuda":
        raise ValueError(f"the call's tensors are on {device}: the library runs on the GPU")
    if stream is not None and stream.device != device:
        raise ValueError(f"a stream of {stream.device} for tensors on {device}")
    if torch.cuda.current_device() != device.index:
        raise ValueError(f"the call's tensors are on {device}, the current device is {torch.cuda.current_device()}")
    if stream is not None:
        _hold(stream, *tensors.values())


def _typed(n, **tensors):
    """Dense [n] arrays: name=(tensor, dtypes)."""
    for name, (t, dtypes) in tensors.items():
        if t is not None and (t.dtype not in dtypes or tuple(t.shape) != (n,) or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous {' or '.join(map(str, dtypes))} tensor of shape ({n},): got "
                             f"{t.dtype} {tuple(t.shape)}, strides {t.stride()}")


_F32, _I32, _U8, _F64 = (torch.float32,), (torch.int32,), (torch.uint8, torch.bool), (torch.float64,)


def _matrix(name, t, shape, dtypes):
    """A 2-D tensor whose rows are consecutive elements, and may be strided."""
    if t.dtype not in dtypes or tuple(t.shape) != tuple(shape) or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a {' or '.join(map(str, dtypes))} tensor of shape {tuple(shape)} with "
                         f"consecutive elements in a row: got {t.dtype} {tuple(t.shape)}, strides {t.stride()}")


def _pitch(t):
    """Elements between rows (of one row, whose stride means nothing: its length in whole 16 bytes)."""
    if t.shape[0] > 1:
        return t.stride(0)
    per = 16 // t.element_size()
    return (t.shape[1] + per - 1) // per * per


_LOGITS = (torch.float32, torch.bfloat16)


def saki_top_logits(logits, k, top_logit, top_token, rest_logit=None, row_status=None, temperature=1.0, workspace=None,
                    stream=None):
    """Call saki_top_logits on preallocated outputs: top_logit (float32) and top_token (int32) [n, k], whose rows
    may be strided alike; rest_logit (float32), row_status (uint8) [n] or None."""
    _lib or load()
    if logits.dim() != 2:
        raise ValueError("logits must be [n_rows, vocab]")
    n, V = logits.shape
    _on(logits.device, stream, logits=logits, top_logit=top_logit, top_token=top_token, rest_logit=rest_logit,
        row_status=row_status, workspace=workspace)
    _matrix("logits", logits, (n, V), _LOGITS)
    _matrix("top_logit", top_logit, (n, k), _F32)
    _matrix("top_token", top_token, (n, k), _I32)
    _typed(n, rest_logit=(rest_logit, _F32), row_status=(row_status, _U8))
    _dense(workspace)
    if n > 1 and top_logit.stride(0) != top_token.stride(0):
        raise ValueError("top_logit and top_token must have rows equally far apart")
    _check(_lib.saki_top_logits(_addr(logits), _dtype_code(logits.dtype), n, V, _pitch(logits), int(k), float(temperature),
                                _addr(top_logit), _addr(top_token), top_logit.stride(0) if n > 1 else k,
                                _addr(rest_logit), _addr(row_status), _addr(workspace), _ws_bytes(workspace),
                                _stream(stream)))


def top_logits(logits, k, temperature=1.0, stream=None):
    """The k largest logits of each row and the others' log-sum-exp; allocates its outputs and workspace."""
    if stream is not None:  # what is allocated here is that stream's
        _hold(stream, logits)
        with torch.cuda.stream(stream):
            return top_logits(logits, k, temperature)
    n, V = logits.shape
    dev = logits.device
    out = dict(top_logit=torch.empty(n, k, dtype=torch.float32, device=dev),
               top_token=torch.empty(n, k, dtype=torch.int32, device=dev),
               rest_logit=torch.empty(n, dtype=torch.float32, device=dev),
               row_status=torch.empty(n, dtype=torch.uint8, device=dev))
    ws = torch.empty(workspace_bytes(SAKI_OP_TOP_LOGITS, n, V), dtype=torch.uint8, device=dev)
    saki_top_logits(logits, k, temperature=temperature, workspace=ws, stream=stream, **out)
    return out


def saki_distill_top(student, top_token, top_logit, rest_logit=None, temperature=1.0, direction=SAKI_KL_FORWARD,
                     valid_mask=None, grad_scale=1.0, row_loss=None, loss_sum=None, grad=None, row_status=None,
                     workspace=None, stream=None):
    """Call saki_distill_top on preallocated outputs: row_loss (float32), row_status (uint8) [n], loss_sum (float64,
    one entry), grad [n, V] (float32 or bfloat16), each may be None."""
    _lib or load()
    if student.dim() != 2 or top_token.dim() != 2:
        raise ValueError("student must be [n_rows, vocab], top_token [n_rows, k]")
    n, V = student.shape
    k = top_token.shape[1]
    _on(student.device, stream, student=student, top_token=top_token, top_logit=top_logit, rest_logit=rest_logit,
        valid_mask=valid_mask, row_loss=row_loss, loss_sum=loss_sum, grad=grad, row_status=row_status, workspace=workspace)
    _matrix("student", student, (n, V), _LOGITS)
    _matrix("top_token", top_token, (n, k), _I32)
    _matrix("top_logit", top_logit, (n, k), _F32)
    _typed(n, rest_logit=(rest_logit, _F32), valid_mask=(valid_mask, _U8), row_loss=(row_loss, _F32), row_status=(row_status, _U8))
    _typed(1, loss_sum=(loss_sum, _F64))
    if grad is not None:
        _matrix("grad", grad, (n, V), _LOGITS)
    _dense(workspace)
    if n > 1 and top_logit.stride(0) != top_token.stride(0):
        raise ValueError("top_logit and top_token must have rows equally far apart")
    rows = SakiTopList(_addr(top_token), _addr(top_logit), _addr(rest_logit), top_token.stride(0) if n > 1 else k, k, 0)
    _check(_lib.saki_distill_top(_addr(student), _dtype_code(student.dtype), n, V, _pitch(student), _ref(rows),
                                 float(temperature), int(direction), _addr(valid_mask), float(grad_scale), _addr(row_loss),
                                 _addr(loss_sum), _addr(grad), SAKI_F32 if grad is None else _dtype_code(grad.dtype),
                                 0 if grad is None else _pitch(grad), _addr(row_status), _addr(workspace),
                                 _ws_bytes(workspace), _stream(stream)))


def distill_top(student, top_token, top_logit, rest_logit=None, temperature=1.0, direction=SAKI_KL_FORWARD, valid_mask=None,
                grad_scale=1.0, grad_dtype=torch.float32, stream=None):
    """Divergence from a teacher's top logits and its gradient (grad_dtype None: none); allocates its outputs."""
    if stream is not None:  # what is allocated here is that stream's
        _hold(stream, student, top_token, top_logit, rest_logit, valid_mask)
        with torch.cuda.stream(stream):
            return distill_top(student, top_token, top_logit, rest_logit, temperature, direction, valid_mask, grad_scale,
                               grad_dtype)
    n, V = student.shape
    dev = student.device
    out = dict(row_loss=torch.empty(n, dtype=torch.float32, device=dev),
               loss_sum=torch.empty(1, dtype=torch.float64, device=dev),
               grad=alloc_rows(n, V, grad_dtype, dev) if grad_dtype is not None else None,
               row_status=torch.empty(n, dtype=torch.uint8, device=dev))
    ws = torch.empty(max(workspace_bytes(SAKI_OP_DISTILL_TOP, n, V), 8), dtype=torch.uint8, device=dev)
    saki_distill_top(student, top_token, top_logit, rest_logit, temperature, direction, valid_mask, grad_scale,
                     workspace=ws, stream=stream, **out)
    return out


def _head(hidden, weight):
    if hidden.dim() != 2 or weight.dim() != 2 or hidden.dtype != weight.dtype:
        raise ValueError("hidden must be [n_rows, D] and weight [vocab, D], of one dtype")
    _matrix("hidden", hidden, hidden.shape, _LOGITS)
    _matrix("weight", weight, (weight.shape[0], hidden.shape[1]), _LOGITS)
    return SakiHead(_addr(hidden), _addr(weight), _pitch(hidden), _pitch(weight), hidden.shape[0], weight.shape[0],
                    hidden.shape[1], _dtype_code(hidden.dtype), 0)


def linear_ce_workspace_bytes(hidden, weight, train=True, grad_hidden=None, grad_weight=None):
    """Workspace of one saki_linear_ce call; train: with both gradients, unless grad_hidden or grad_weight say otherwise."""
    _lib or load()
    grads = (train if grad_hidden is None else grad_hidden) * 1 + (train if grad_weight is None else grad_weight) * 2
    return int(_lib.saki_linear_ce_workspace_bytes(_ref(_head(hidden, weight)), int(grads)))


def saki_linear_ce(hidden, weight, token, row_weight=None, valid_mask=None, grad_scale=1.0, row_loss=None, logp_token=None,
                   loss_sum=None, row_status=None, grad_hidden=None, grad_weight=None, workspace=None, stream=None):
    """Call saki_linear_ce on preallocated outputs: row_loss, logp_token (float32), row_status (uint8) [n], loss_sum
    (float64, one entry), grad_hidden and grad_weight like hidden and weight; each may be None."""
    _lib or load()
    head = _head(hidden, weight)
    n = hidden.shape[0]
    _on(hidden.device, stream, hidden=hidden, weight=weight, token=token, row_weight=row_weight, valid_mask=valid_mask,
        row_loss=row_loss, logp_token=logp_token, loss_sum=loss_sum, row_status=row_status, grad_hidden=grad_hidden,
        grad_weight=grad_weight, workspace=workspace)
    _typed(n, token=(token, _I32), row_weight=(row_weight, _F32), valid_mask=(valid_mask, _U8), row_loss=(row_loss, _F32),
           logp_token=(logp_token, _F32), row_status=(row_status, _U8))
    _typed(1, loss_sum=(loss_sum, _F64))
    for name, g, x in (("grad_hidden", grad_hidden, hidden), ("grad_weight", grad_weight, weight)):
        if g is not None:
            _matrix(name, g, x.shape, (x.dtype,))
    _dense(workspace)
    args = SakiCEArgs(_addr(token), _addr(row_weight), _addr(valid_mask), float(grad_scale), 0, _addr(row_loss),
                      _addr(logp_token), _addr(loss_sum), _addr(row_status), _addr(grad_hidden), _addr(grad_weight),
                      0 if grad_hidden is None else _pitch(grad_hidden), 0 if grad_weight is None else _pitch(grad_weight))
    _check(_lib.saki_linear_ce(_ref(head), _ref(args), _addr(workspace), _ws_bytes(workspace), _stream(stream)))


def linear_ce(hidden, weight, token, row_weight=None, valid_mask=None, grad_scale=1.0, train=True, stream=None):
    """Cross entropy from hidden states and (train) the gradients of hidden and weight; allocates its outputs."""
    if stream is not None:  # what is allocated here is that stream's
        _hold(stream, hidden, weight, token, row_weight, valid_mask)
        with torch.cuda.stream(stream):
            return linear_ce(hidden, weight, token, row_weight, valid_mask, grad_scale, train)
    n, dev = hidden.shape[0], hidden.device
    out = dict(row_loss=torch.empty(n, dtype=torch.float32, device=dev),
               logp_token=torch.empty(n, dtype=torch.float32, device=dev),
               loss_sum=torch.empty(1, dtype=torch.float64, device=dev),
               row_status=torch.empty(n, dtype=torch.uint8, device=dev),
               grad_hidden=torch.empty(hidden.shape, dtype=hidden.dtype, device=dev) if train else None,
               grad_weight=torch.empty(weight.shape, dtype=weight.dtype, device=dev) if train else None)
    ws = torch.empty(max(linear_ce_workspace_bytes(hidden, weight, train), 8), dtype=torch.uint8, device=dev)
    saki_linear_ce(hidden, weight, token, row_weight, valid_mask, grad_scale, workspace=ws, stream=stream, **out)
    return out
