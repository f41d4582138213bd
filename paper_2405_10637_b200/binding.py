"""ctypes binding of liblckv.so: the same entry points as include/lckv.h, argument marshalling only.

Tensors are torch CUDA tensors (torch supplies device memory and streams); every step of the
computation runs in the library's own kernels.  There is no fallback: if the library is missing
or does not load, the first call raises.
"""
import ctypes as C
import importlib.util
import os

import torch

from . import build as _build

OK, EINVAL, ECAPACITY, ENOMEM, ECUDA, ETIMEOUT, ESTATICLIMIT = range(7)
MODE_CONDENSED, MODE_STANDARD = 0, 1


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_layers", C.c_int32), ("n_warmup", C.c_int32),
                ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("max_batch", C.c_int32), ("max_seq", C.c_int32), ("softmax_scale", C.c_float),
                ("top_variant", C.c_int32), ("out_dtype", C.c_int32), ("host_staging", C.c_int32),
                ("use_graph", C.c_int32), ("stream_sink", C.c_int32), ("page_rows", C.c_int32), ("n_pages", C.c_int32),
                ("kernel_kind", C.c_int32)]


class Info(C.Structure):
    _fields_ = [("n_slots", C.c_int32), ("n_workers", C.c_int32), ("rows_per_tile", C.c_int32),
                ("kernel_kind", C.c_int32), ("launches_per_step", C.c_int32),
                ("sm_count", C.c_int32), ("slot_bytes", C.c_uint64),
                ("workspace_bytes", C.c_uint64)]


class Rope(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32),
                ("positions", C.c_int32), ("cos", C.c_void_p), ("sin", C.c_void_p)]


class RopeScaling(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("kind", C.c_int32), ("base", C.c_double),
                ("factor", C.c_double), ("original", C.c_double), ("low", C.c_double),
                ("high", C.c_double), ("amplitude", C.c_double)]


# name -> (restype, argtypes); also the list of symbols the header declares
_vp, _i32, _i32p, _i64 = C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_int64
_vpp = C.POINTER(C.c_void_p)
SIGNATURES = {
    "lckv_plan": (C.c_int, [_i32, _i32, _i32, _i32p, _i32p, _i32p, _i32p, _i32p, _i32p]),
    "lckv_cache_bytes": (C.c_size_t, [C.POINTER(Config)]),
    "lckv_cache_alloc": (C.c_int, [_vpp, C.POINTER(Config), _vp, C.c_size_t]),
    "lckv_cache_free": (C.c_int, [_vp]),
    "lckv_cache_info": (C.c_int, [_vp, C.POINTER(Info)]),
    "lckv_cache_reset": (C.c_int, [_vp, _i32p, _i32, _vp]),
    "lckv_cache_lengths": (C.c_int, [_vp, _i32p, _i32, _vp]),
    "lckv_cache_status": (C.c_int, [_vp, _i32p, _vp]),
    "lckv_cache_set_wait_limit": (C.c_int, [_vp, C.c_uint32]),
    "lckv_cache_set_worker_limit": (C.c_int, [_vp, _i32]),
    "lckv_cache_slot_ptrs": (C.c_int, [_vp, _i32, _vpp, _vpp]),
    "lckv_cache_page_table": (C.c_int, [_vp, _i32p, _i32p]),
    "lckv_append_kv": (C.c_int, [_vp, _i32, _vp, _vp, _i32, _i32, _vp]),
    "lckv_project_append_kv": (C.c_int, [_vp, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp]),
    "lckv_decode_attention": (C.c_int, [_vp, _i32, _i32, _vp, _vp, _vp, _i32, _vp]),
    "lckv_layer_stack_step": (C.c_int, [_vp, _vpp, _vpp, _vpp, _vpp, _i32, _vp]),
    "lckv_layer_stack_step_host": (C.c_int, [_vp, _vpp, _vpp, _vpp, _vpp, _i32, _vp]),
    "lckv_prefill_write_kv": (C.c_int, [_vp, _i32, _vp, _vp, _i32, _i32, _vp]),
    "lckv_prefill_attention": (C.c_int, [_vp, _i32, _i32, _vp, _vp, _i32, _i32, _vp]),
    "lckv_prefill_iteration": (C.c_int, [_vp, _vpp, _vpp, _vpp, _vpp, _i32, _i32, _vp]),
    "lckv_decode_attention_static": (C.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32,
                                              _i32, C.c_int64, _i32, C.c_float, _i32, _vp]),
    "lckv_read_stream_probe": (C.c_int, [_vp, C.c_size_t, _i32, _i32, C.c_float, _vp, _vp, _vp]),
    "lckv_rope_tables": (C.c_int, [_vp, _vp, _i32, _i32, _vp, _vp]),
    "lckv_rope_apply": (C.c_int, [_vp, _vp, _vp, _i64, _i64, _vp, _i64, _i64, _i32, _i32, _i32, _i32, _i32, _vp]),
    "lckv_rope_append_kv": (C.c_int, [_vp, _i32, _vp, _vp, _i64, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _vp]),
    "lckv_rope_prefill_write_kv": (C.c_int, [_vp, _i32, _vp, _vp, _i64, _vp, _vp, _vp, _i64, _i32, _i32, _vp]),
    "lckv_rms_norm": (C.c_int, [_vp, _i64, _i32, _vp, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _i32, _i32,
                                C.c_float, _vp]),
    "lckv_quant_bytes": (C.c_size_t, [_i32, _i32, _i32, _i32]),
    "lckv_quant_pack": (C.c_int, [_vp, _vp, _vp, _i32, _i32, _i32, _vp, C.c_size_t, _vp]),
    "lckv_quant_linear": (C.c_int, [_vp, _i32, _i32, _i32, _i32, _vp, _i64, _i32, _vp, _i32, _vp, _i64, _i32, _i32,
                                    _vp, _vp]),
    "lckv_quant_set_copy_limits": (C.c_int, [_i32, _i32]),
    "lckv_status_string": (C.c_char_p, [C.c_int]),
    "lckv_last_cuda_error": (C.c_int, []),
}

_LIB = None


def lib():
    """Load (building first if the sources are newer) the CUDA library.  Raises if impossible."""
    global _LIB
    if _LIB is None:
        path = _build.build()
        L = C.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _LIB = L
    return _LIB


class LckvError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        msg = lib().lckv_status_string(status).decode()
        extra = f", cudaError {lib().lckv_last_cuda_error()}" if status == ECUDA else ""
        super().__init__(f"{what}: {msg} (status {status}{extra})")


def _chk(rc, what):
    if rc != OK:
        raise LckvError(rc, what)


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _ptr_array(ts):
    arr = (C.c_void_p * len(ts))()
    for i, t in enumerate(ts):
        arr[i] = None if t is None else t.data_ptr()
    return C.cast(arr, _vpp)


def lckv_plan(n_layers, n_warmup, top_variant=0):
    """Host-only layer plan; returns a dict of lists + n_slots."""
    arrs = [(C.c_int32 * max(n_layers, 1))() for _ in range(5)]
    n = C.c_int32(0)
    rc = lib().lckv_plan(n_layers, n_warmup, top_variant, *arrs, C.byref(n))
    _chk(rc, "lckv_plan")
    keys = ["is_warmup", "read_slot", "mode", "write_slot", "write_before"]
    out = {k: list(a)[:n_layers] for k, a in zip(keys, arrs)}
    out["n_slots"] = n.value
    return out


def make_config(n_layers, n_warmup, n_q_heads, n_kv_heads, head_dim, max_batch, max_seq,
                softmax_scale=0.0, top_variant=0, out_dtype=0, host_staging=0, use_graph=0,
                kernel_kind=0, stream_sink=0, page_rows=0, n_pages=0):
    return Config(C.sizeof(Config), n_layers, n_warmup, n_q_heads, n_kv_heads, head_dim,
                  max_batch, max_seq, softmax_scale, top_variant, out_dtype, host_staging,
                  use_graph, stream_sink, page_rows, n_pages, kernel_kind)


def lckv_cache_bytes(cfg):
    return int(lib().lckv_cache_bytes(C.byref(cfg)))


def lckv_decode_attention_static(k, v, lens, q, out, mode, lse=None, dev_status=None,
                                 softmax_scale=0.0, stream=None):
    """Decode attention for callers that must not allocate: k, v [B, H_kv, T_cap, d_h] bf16,
    lens [B] int32, q [B, H_q, d_h] bf16 and `out` (bf16 or fp32, caller-provided) are CUDA
    tensors; the library's scratch is a fixed array inside its device image, so nothing is
    allocated here or there.  One call at a time per GPU: all calls share that scratch."""
    B, Hkv, T_cap, d = k.shape
    Hq = q.shape[1]
    rc = lib().lckv_decode_attention_static(
        _ptr(k), _ptr(v), _ptr(lens), _ptr(q), _ptr(out), _ptr(lse), _ptr(dev_status), q.shape[0],
        Hq, Hkv, d, T_cap, mode, softmax_scale, 1 if out.dtype == torch.float32 else 0,
        _stream(stream))
    _chk(rc, "lckv_decode_attention_static")
    return out


def lckv_read_stream_probe(src, nbytes, kind, dev_sum, dev_status, repeats=1, l2_keep=0.0, stream=None):
    """Read-only stream over the first nbytes of the CUDA tensor `src`, `repeats` passes in one launch;
    dev_sum (uint32/int32 [1]) and dev_status (int32 [1]) are CUDA tensors."""
    _chk(lib().lckv_read_stream_probe(_ptr(src), nbytes, kind, repeats, l2_keep, _ptr(dev_sum),
                                      _ptr(dev_status), _stream(stream)), "lckv_read_stream_probe")


# -- operators around the attention ------------------------------------------------------------
# A decode step makes these calls several times per layer, so their checks and marshalling are native
# (csrc/lckv_calls.cpp); what a call takes of its tensors is stated there and in include/lckv.h.
_CALLS = None
_BAD_TENSOR = -1


def calls():
    """Load (building first if the sources are newer) the native calls.  Raises if impossible."""
    global _CALLS
    if _CALLS is None:
        lib()
        path = _build.build_calls()
        spec = importlib.util.spec_from_file_location("_lckv_calls", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        _CALLS = module
    return _CALLS


def _fail(rc, name, takes):
    raise LckvError(EINVAL, f"{name}: {takes}") if rc == _BAD_TENSOR else LckvError(rc, name)


def _require(ok, what):
    if not ok:
        raise LckvError(EINVAL, what)


def _address(device, stream):
    """cudaStream_t of a stream that the caller gave; it has to belong to the tensors' device."""
    _require(stream.device.index == device, "the stream belongs to another device than the tensors")
    return stream.cuda_stream


def _made(make, stream, shape, **kw):
    """An output made here: by the stream that will write it, so that neither what its memory held before nor a fill of
    it is still under way on another one."""
    if stream is None:
        return make(shape, **kw)
    with torch.cuda.stream(stream):
        return make(shape, **kw)


def make_rope_scaling(kind=0, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0, amplitude=0.0):
    """Frequencies of rotary tables: kind 0 none, 1 linear, 2 base, 3 by parts (include/lckv.h)."""
    r = RopeScaling(C.sizeof(RopeScaling), kind, base, factor, original, low, high, amplitude)
    r.address = C.addressof(r)
    return r


def lckv_rope_tables(cos, sin, scaling, stream=None):
    """Fills the CUDA tensors cos, sin [positions, rot_dim / 2] fp32; returns them."""
    rc = (_CALLS or calls()).rope_tables(cos, sin, scaling.address,
                                         None if stream is None else _address(cos.get_device(), stream))
    if rc:
        _fail(rc, "lckv_rope_tables", "cos and sin are contiguous fp32 CUDA tensors of one shape")
    return cos, sin


def make_rope(cos, sin, interleaved=False):
    """A rotation described by its tables, cos and sin [positions, rot_dim / 2] fp32 on the device.  The result keeps
    the tables alive."""
    _require(cos.dtype == torch.float32 and sin.dtype == torch.float32 and cos.dim() == 2 and cos.shape == sin.shape
             and cos.is_contiguous() and sin.is_contiguous() and cos.get_device() >= 0 and sin.get_device() == cos.get_device(),
             "make_rope: cos and sin are contiguous fp32 CUDA tensors of one shape")
    r = Rope(C.sizeof(Rope), 2 * cos.shape[1], 1 if interleaved else 0, cos.shape[0], cos.data_ptr(), sin.data_ptr())
    r.tables, r.device, r.address = (cos, sin), cos.get_device(), C.addressof(r)
    return r


def lckv_rope_apply(rope, positions, x, out=None, transpose=False, stream=None):
    """x [tokens, heads, d_h] bf16 or fp32 (any strides, the last 1) rotated by positions [tokens] int32, into `out`
    (made if None; may be x)."""
    if out is None:
        out = _made(torch.empty, stream, x.shape, dtype=x.dtype, device=x.device)
    rc = (_CALLS or calls()).rope_apply(rope.address, rope.device, positions, x, out, 1 if transpose else 0,
                                        None if stream is None else _address(rope.device, stream))
    if rc:
        _fail(rc, "lckv_rope_apply", "x and out are [tokens, heads, d_h] bf16 or fp32, positions [tokens] int32, all on the "
                                     "tables' device")
    return out


def lckv_rms_norm(x, weight, out, residual=None, residual_out=None, out_scale=None, scale_group=0, eps=1e-6,
                  stream=None):
    """out = norm(x + residual) * weight over the last dimension of x [rows, width]; the sum goes to residual_out.
    out is bf16, fp32, or float8_e4m3fn with out_scale fp32 ([rows, 1] or [rows], or [rows, ceil(width / 128)] with
    scale_group=128)."""
    rc = (_CALLS or calls()).rms_norm(x, weight, out, residual, residual_out, out_scale, scale_group, eps,
                                      None if stream is None else _address(x.get_device(), stream))
    if rc:
        _fail(rc, "lckv_rms_norm", "x is [rows, width], weight [width], residual, residual_out (like residual) and out have x's "
                                   "shape and are contiguous, bf16 or fp32 (out also float8_e4m3fn, with out_scale fp32, one "
                                   "per row or per 128 columns), all on one device")
    return out


class QuantWeight:
    """A 4-bit weight [n, k] laid out by lckv_quant_pack, and the buffer behind it."""

    def __init__(self, n, k, group, has_zeros, buf):
        self.n, self.k, self.group, self.has_zeros, self.buf = n, k, group, has_zeros, buf
        self.device = buf.get_device()
        self.call = (buf.data_ptr(), self.device, n, k, group, has_zeros)


def lckv_quant_pack(codes, scales, zeros=None, stream=None):
    """codes [n, k / 2] uint8 (low nibble = even column), scales [n, k / group] bf16, zeros [n, k / group] uint8 or None
    -> QuantWeight.  Synchronises the stream."""
    dev = codes.get_device()
    _require(codes.dim() == 2 and codes.dtype == torch.uint8 and codes.is_contiguous() and scales.dtype == torch.bfloat16
             and scales.is_contiguous() and scales.dim() == 2 and scales.shape[0] == codes.shape[0] and scales.shape[1] > 0
             and 2 * codes.shape[1] % scales.shape[1] == 0 and dev == scales.get_device() and dev >= 0,
             "lckv_quant_pack: codes [n, k / 2] uint8, scales [n, k / group] bf16, on one device")
    _require(zeros is None or (zeros.dtype == torch.uint8 and zeros.is_contiguous() and zeros.shape == scales.shape
                               and zeros.get_device() == dev), "lckv_quant_pack: zeros are uint8 of the scales' shape")
    n, k = codes.shape[0], 2 * codes.shape[1]
    group = k // scales.shape[1]
    nbytes = lib().lckv_quant_bytes(n, k, group, 0 if zeros is None else 1)
    _require(nbytes > 0, "lckv_quant_pack: group is 32, 64 or 128")
    with torch.cuda.device(dev):
        buf = _made(torch.empty, stream, nbytes, dtype=torch.uint8, device=codes.device)
        st = torch.cuda.current_stream(dev).cuda_stream if stream is None else _address(dev, stream)
        _chk(lib().lckv_quant_pack(codes.data_ptr(), scales.data_ptr(), None if zeros is None else zeros.data_ptr(), n, k,
                                   group, buf.data_ptr(), nbytes, st), "lckv_quant_pack")
    return QuantWeight(n, k, group, 0 if zeros is None else 1, buf)


def lckv_quant_linear(w, x, out=None, x_scale=None, dev_status=None, stream=None):
    """out [rows, n] (bf16 or fp32) = x [rows, k] (bf16, or float8_e4m3fn with x_scale) times the 4-bit weight w.
    dev_status: optional CUDA int32 tensor that receives ETIMEOUT if a device-side wait gave up.  The kernel in front of the
    call must not be one that writes w.buf (lckv_quant_pack never is): the first weights are requested before it has ended."""
    if out is None:
        out = _made(torch.empty, stream, (x.shape[0], w.n), dtype=torch.bfloat16, device=x.device)
    rc = (_CALLS or calls()).quant_linear(*w.call, x, out, x_scale, dev_status,
                                          None if stream is None else _address(w.device, stream))
    if rc:
        _fail(rc, "lckv_quant_linear", "x is [rows, k] bf16 or float8_e4m3fn (with x_scale fp32, one per row or per 128 columns), "
                                       "out [rows, n] bf16 or fp32, on the weight's device")
    return out


def lckv_quant_set_copy_limits(weights=-1, x=-1):
    """For tests of the bounded waits: blocks of weights and of x that products of more than 16 rows request (include/lckv.h)."""
    _chk(lib().lckv_quant_set_copy_limits(weights, x), "lckv_quant_set_copy_limits")


class Cache:
    """Owner of one lckv_cache_t and of the torch buffer behind it."""

    def __init__(self, cfg, device="cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        with torch.cuda.device(self.device):
            nbytes = lckv_cache_bytes(cfg)
            if nbytes == 0:
                raise LckvError(EINVAL, "lckv_cache_bytes")
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            h = C.c_void_p()
            _chk(lib().lckv_cache_alloc(C.byref(h), C.byref(cfg), _ptr(self.buf), nbytes),
                 "lckv_cache_alloc")
        self.h = h
        self.call = (h.value, self.buf.get_device())       # what the native calls take
        self.heads = (cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim)
        info = Info()
        _chk(lib().lckv_cache_info(self.h, C.byref(info)), "lckv_cache_info")
        self.info = info
        self.out_torch_dtype = torch.float32 if cfg.out_dtype else torch.bfloat16

    def close(self):
        if getattr(self, "h", None):
            lib().lckv_cache_free(self.h)
            self.h = None
            self.call = (None, -1)
            self.buf = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C entry points, same names ---------------------------------------------------------
    def lckv_cache_reset(self, host_lens=None, batch=None, stream=None):
        if host_lens is not None:
            arr = (C.c_int32 * len(host_lens))(*[int(x) for x in host_lens])
            batch = len(host_lens) if batch is None else batch
            rc = lib().lckv_cache_reset(self.h, arr, batch, _stream(stream))
        else:
            rc = lib().lckv_cache_reset(self.h, None, batch or self.cfg.max_batch, _stream(stream))
        _chk(rc, "lckv_cache_reset")

    def lckv_cache_lengths(self, batch=None, stream=None):
        batch = batch or self.cfg.max_batch
        arr = (C.c_int32 * batch)()
        _chk(lib().lckv_cache_lengths(self.h, arr, batch, _stream(stream)), "lckv_cache_lengths")
        return list(arr)

    def lckv_cache_status(self, stream=None):
        s = C.c_int32(0)
        _chk(lib().lckv_cache_status(self.h, C.byref(s), _stream(stream)), "lckv_cache_status")
        return s.value

    def lckv_cache_set_wait_limit(self, polls):
        _chk(lib().lckv_cache_set_wait_limit(self.h, polls), "lckv_cache_set_wait_limit")

    def lckv_cache_set_worker_limit(self, workers):
        _chk(lib().lckv_cache_set_worker_limit(self.h, workers), "lckv_cache_set_worker_limit")

    def lckv_cache_slot_ptrs(self, slot):
        k, v = C.c_void_p(), C.c_void_p()
        _chk(lib().lckv_cache_slot_ptrs(self.h, slot, C.byref(k), C.byref(v)),
             "lckv_cache_slot_ptrs")
        return k.value, v.value

    def lckv_cache_page_table(self):
        """Paged caches: torch int64 tensor [B_max, entries_per_seq] of page ids (-1 = none)."""
        n = C.c_int32(0)
        _chk(lib().lckv_cache_page_table(self.h, None, C.byref(n)), "lckv_cache_page_table")
        arr = (C.c_int32 * (self.cfg.max_batch * n.value))()
        _chk(lib().lckv_cache_page_table(self.h, arr, C.byref(n)), "lckv_cache_page_table")
        return torch.tensor(list(arr), dtype=torch.int64).view(self.cfg.max_batch, n.value)

    def slot_tensors(self, slot):
        """torch views of a slot's K and V (same memory): [B_max, H_kv, T_cap, d_h] bf16, or
        [n_pages, H_kv, page_rows, d_h] for a paged cache."""
        k, v = self.lckv_cache_slot_ptrs(slot)
        c = self.cfg
        shape = (c.max_batch, c.n_kv_heads, c.max_seq, c.head_dim)
        if c.page_rows:
            shape = (c.n_pages, c.n_kv_heads, c.page_rows, c.head_dim)
        n = 2 * shape[0] * shape[1] * shape[2] * shape[3]
        base = self.buf.data_ptr()
        kt = self.buf[k - base:k - base + n].view(torch.bfloat16).view(shape)
        vt = self.buf[v - base:v - base + n].view(torch.bfloat16).view(shape)
        return kt, vt

    def lckv_append_kv(self, slot, k_new, v_new, batch=None, advance_len=0, stream=None):
        batch = k_new.shape[0] if batch is None else batch
        _chk(lib().lckv_append_kv(self.h, slot, _ptr(k_new), _ptr(v_new), batch, advance_len,
                                  _stream(stream)), "lckv_append_kv")

    def lckv_project_append_kv(self, slot, x, w_k, w_v, rope_cos=None, rope_sin=None, batch=None,
                               advance_len=0, stream=None):
        """x [batch, d_model], w_k / w_v [H_kv*d_h, d_model] bf16 device tensors; optional rotary
        tables [positions, d_h/2] fp32."""
        batch = x.shape[0] if batch is None else batch
        n_pos = 0 if rope_cos is None else rope_cos.shape[0]
        _chk(lib().lckv_project_append_kv(self.h, slot, _ptr(x), x.shape[1], _ptr(w_k), _ptr(w_v),
                                          _ptr(rope_cos), _ptr(rope_sin), n_pos, batch, advance_len,
                                          _stream(stream)), "lckv_project_append_kv")

    def _rope_call(self, name, slot, rope, q, k, v, q_out, advance, stream):
        h, dev = self.call
        rc = (_CALLS or calls()).rope_cache(h, dev, slot, rope.address, rope.device, *self.heads, q, k, v, q_out, advance,
                                            None if stream is None else _address(dev, stream))
        if rc:
            _fail(rc, name, "q, k, v are bf16 [batch, tokens, heads, d_h] (or [batch, heads, d_h]) on the cache's device, heads "
                            "dense, one stride between tokens, k and v alike; q_out is like q, contiguous")
        return q_out

    def lckv_rope_append_kv(self, slot, rope, q, k_new, v_new, q_out=None, advance_len=0, stream=None):
        """Rotated append of one ([batch, heads, d_h]) or several ([batch, n, heads, d_h]) new tokens per sequence;
        q, or k_new and v_new, may be None.  Views of a fused projection are taken as they are.  Returns q_out."""
        if q is not None and q_out is None:
            q_out = _made(torch.empty, stream, q.shape, dtype=q.dtype, device=q.device)
        return self._rope_call("lckv_rope_append_kv", slot, rope, q, k_new, v_new, q_out, 1 if advance_len else 0, stream)

    def lckv_rope_prefill_write_kv(self, slot, rope, q, k, v, q_out=None, stream=None):
        """The same for prompts [batch, n_max, heads, d_h] whose lengths the cache holds already.  Rows of q_out behind a
        prompt are left as they were (zero where q_out is made here)."""
        if q is not None and q_out is None:
            q_out = _made(torch.zeros, stream, q.shape, dtype=q.dtype, device=q.device)
        return self._rope_call("lckv_rope_prefill_write_kv", slot, rope, q, k, v, q_out, -1, stream)

    def lckv_decode_attention(self, slot, mode, q, out=None, lse=None, batch=None, stream=None):
        batch = q.shape[0] if batch is None else batch
        if out is None:
            out = torch.empty(q.shape, dtype=self.out_torch_dtype, device=q.device)
        _chk(lib().lckv_decode_attention(self.h, slot, mode, _ptr(q), _ptr(out), _ptr(lse), batch,
                                         _stream(stream)), "lckv_decode_attention")
        return out

    def lckv_layer_stack_step(self, q_layers, out_layers, k_new_layers, v_new_layers, batch=None,
                              stream=None):
        batch = q_layers[0].shape[0] if batch is None else batch
        _chk(lib().lckv_layer_stack_step(self.h, _ptr_array(q_layers), _ptr_array(out_layers),
                                         _ptr_array(k_new_layers), _ptr_array(v_new_layers),
                                         batch, _stream(stream)), "lckv_layer_stack_step")

    def lckv_layer_stack_step_host(self, q_layers, out_layers, k_new_layers, v_new_layers,
                                   batch=None, stream=None):
        """Same, with HOST (ideally pinned) torch tensors."""
        batch = q_layers[0].shape[0] if batch is None else batch
        _chk(lib().lckv_layer_stack_step_host(self.h, _ptr_array(q_layers),
                                              _ptr_array(out_layers), _ptr_array(k_new_layers),
                                              _ptr_array(v_new_layers), batch, _stream(stream)),
             "lckv_layer_stack_step_host")

    # -- prompt encoding (token-major tensors [B, n_max, H, d_h]) -------------------------------
    def lckv_prefill_write_kv(self, slot, k, v, stream=None):
        _chk(lib().lckv_prefill_write_kv(self.h, slot, _ptr(k), _ptr(v), k.shape[1], k.shape[0],
                                         _stream(stream)), "lckv_prefill_write_kv")

    def lckv_prefill_attention(self, slot, mode, q, out=None, stream=None):
        if out is None:
            out = torch.zeros(q.shape, dtype=self.out_torch_dtype, device=q.device)
        _chk(lib().lckv_prefill_attention(self.h, slot, mode, _ptr(q), _ptr(out), q.shape[1],
                                          q.shape[0], _stream(stream)), "lckv_prefill_attention")
        return out

    def lckv_prefill_iteration(self, q_layers, out_layers, k_layers, v_layers, stream=None):
        q0 = q_layers[0]
        _chk(lib().lckv_prefill_iteration(self.h, _ptr_array(q_layers), _ptr_array(out_layers),
                                          _ptr_array(k_layers), _ptr_array(v_layers), q0.shape[1],
                                          q0.shape[0], _stream(stream)), "lckv_prefill_iteration")
