"""ctypes binding of include/pe.h.  Argument marshalling only.  A call whose stream is left out runs on the stream that is current in
torch on the handle's device; 0 is the default stream."""
import ctypes as C
import os
import sys

PE_F32, PE_BF16, PE_CKPT = 0, 1, 2
PE_RELPOS_PAIR, PE_RELPOS_HEADS = 0, 1
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libpe_mi355x.so")


class PEError(RuntimeError):
    pass


class PEDims(C.Structure):
    _fields_ = [("s", C.c_int), ("r", C.c_int), ("c_m", C.c_int), ("c_z", C.c_int),
                ("h_msa", C.c_int), ("d_msa", C.c_int), ("h_pair", C.c_int), ("d_pair", C.c_int),
                ("c_tri", C.c_int), ("c_opm", C.c_int), ("n_trans", C.c_int), ("col_global", C.c_int),
                ("dtype", C.c_int), ("ln_eps", C.c_float), ("opm_eps", C.c_float), ("variant", C.c_int)]

    @classmethod
    def from_dict(cls, d):
        return cls(**{k: d.get(k, 0) if k == "variant" else d[k] for k, _ in cls._fields_})


class _ParamEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("offset", C.c_longlong), ("ndim", C.c_int),
                ("shape", C.c_int * 2), ("fan_in", C.c_int), ("kind", C.c_int)]


class _CtxEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("offset_bytes", C.c_longlong), ("count", C.c_longlong),
                ("dtype", C.c_int)]


class _TimingEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("kernel", C.c_char * 64), ("launches", C.c_int), ("total_ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


class _Relpos(C.Structure):
    _fields_ = [(k, C.c_int) for k in ("n_q", "n_k", "c", "n_edges", "segments", "layout", "dtype")] + [("ld", C.c_longlong)]


_lib = None
_KINDS = {0: "weight", 1: "ln_gamma", 2: "ln_beta", 3: "bias"}


def lib():
    """Load the HIP library; fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise PEError("HIP library %s is missing: run paper_2211_00235_amd.build.build() "
                      "(there is no CPU fallback)" % _LIB_PATH)
    L = C.CDLL(_LIB_PATH)
    vp, dp, fp = C.c_void_p, C.POINTER(PEDims), C.c_void_p
    L.pe_create.argtypes = [C.POINTER(vp)]
    L.pe_destroy.argtypes = [vp]
    L.pe_set_option.argtypes = [vp, C.c_int, C.c_int]
    L.pe_check_dims.argtypes = [dp]
    L.pe_dims_error.argtypes = [dp]
    L.pe_dims_error.restype = C.c_char_p
    L.pe_param_count.argtypes = [dp]
    L.pe_param_count.restype = C.c_longlong
    L.pe_param_table.argtypes = [dp, C.POINTER(_ParamEntry), C.c_int]
    L.pe_ctx_table.argtypes = [dp, C.POINTER(_CtxEntry), C.c_int]
    L.pe_ctx_bytes.argtypes = [dp]
    L.pe_ctx_bytes.restype = C.c_size_t
    L.pe_workspace_bytes.argtypes = [dp, C.c_int]
    L.pe_workspace_bytes.restype = C.c_size_t
    L.pe_stack_workspace_bytes.argtypes = [C.c_int, dp, C.c_int, dp]
    L.pe_stack_workspace_bytes.restype = C.c_size_t
    L.pe_stack_workspace_bytes_keep.argtypes = [C.c_int, dp, C.c_int, dp]
    L.pe_stack_workspace_bytes_keep.restype = C.c_size_t
    L.pe_stack_workspace_bytes_ckpt.argtypes = [C.c_int, dp, C.c_int, dp]
    L.pe_stack_workspace_bytes_ckpt.restype = C.c_size_t
    L.pe_block_fwd.argtypes = [vp, dp, vp, vp, fp, fp, fp, vp, vp, vp, vp, C.c_size_t, vp, vp]
    L.pe_static_scratch_bytes.argtypes = []
    L.pe_static_scratch_bytes.restype = C.c_size_t
    L.pe_block_fwd_static.argtypes = [vp, dp, vp, vp, fp, fp, fp, vp, vp, vp, vp]
    L.pe_block_bwd.argtypes = [vp, dp, vp, vp, fp, fp, fp, vp, vp, vp, vp, fp, vp, vp, C.c_size_t, vp, vp]
    L.pe_stack_fwd_bwd.argtypes = [vp, C.c_int, dp, C.c_int, dp, vp, vp, vp, fp, fp, fp, fp, vp, vp,
                                   vp, vp, vp, vp, vp, fp, vp, C.c_size_t, vp, vp]
    ll, rp, size = C.c_longlong, C.POINTER(_Relpos), C.c_size_t
    L.pe_handle_device.argtypes = [vp]
    L.pe_layernorm_fwd.argtypes = [vp, ll, C.c_int, C.c_int, vp, ll, vp, ll, fp, fp, C.c_float, vp, ll, fp, vp, vp]
    L.pe_layernorm_workspace_bytes.argtypes = [ll, C.c_int]
    L.pe_layernorm_workspace_bytes.restype = size
    L.pe_layernorm_bwd.argtypes = [vp, ll, C.c_int, C.c_int, C.c_int, vp, ll, fp, fp, vp, ll, vp, ll, vp, ll, fp, fp, C.c_int, vp, size, vp]
    L.pe_ckpt_bytes.argtypes = [ll, C.c_int]
    L.pe_ckpt_bytes.restype = size
    L.pe_ckpt_pack.argtypes = [vp, ll, C.c_int, C.c_int, vp, ll, vp, vp]
    L.pe_ckpt_unpack.argtypes = [vp, ll, C.c_int, C.c_int, vp, vp, ll, vp]
    L.pe_relpos_workspace_bytes.argtypes = [rp]
    L.pe_relpos_workspace_bytes.restype = size
    L.pe_relpos_fwd.argtypes = [vp, rp, vp, vp, vp, vp, vp, fp, vp, vp, vp]
    L.pe_relpos_bwd.argtypes = [vp, rp, vp, vp, vp, vp, vp, vp, fp, C.c_int, vp, size, vp]
    L.pe_timing_collect.argtypes = [vp, C.POINTER(_TimingEntry), C.c_int]
    L.pe_strerror.argtypes = [C.c_int]
    L.pe_strerror.restype = C.c_char_p
    L.pe_last_error.argtypes = [vp]
    L.pe_last_error.restype = C.c_char_p
    _lib = L
    return L


def strerror(code):
    return lib().pe_strerror(code).decode()


def _dims(d):
    return d if isinstance(d, PEDims) else PEDims.from_dict(d)


def check_dims(d):
    return lib().pe_check_dims(C.byref(_dims(d)))


def dims_error(d):
    """Text of the requirement that check_dims found violated ('' if the dims are supported)."""
    return lib().pe_dims_error(C.byref(_dims(d))).decode()


def param_count(d):
    return int(lib().pe_param_count(C.byref(_dims(d))))


def param_table(d):
    dd = _dims(d)
    n = lib().pe_param_table(C.byref(dd), None, 0)
    if n < 0:
        raise PEError(strerror(n))
    arr = (_ParamEntry * n)()
    lib().pe_param_table(C.byref(dd), arr, n)
    return [dict(name=e.name.decode(), offset=int(e.offset),
                 shape=tuple(e.shape[:e.ndim]), fan_in=int(e.fan_in), kind=_KINDS[e.kind]) for e in arr]


def ctx_table(d):
    dd = _dims(d)
    n = lib().pe_ctx_table(C.byref(dd), None, 0)
    if n < 0:
        raise PEError(strerror(n))
    arr = (_CtxEntry * n)()
    lib().pe_ctx_table(C.byref(dd), arr, n)
    return [dict(name=e.name.decode(), offset_bytes=int(e.offset_bytes), count=int(e.count), dtype=int(e.dtype))
            for e in arr]


def ctx_bytes(d):
    return int(lib().pe_ctx_bytes(C.byref(_dims(d))))


def workspace_bytes(d, with_ctx):
    return int(lib().pe_workspace_bytes(C.byref(_dims(d)), int(with_ctx)))


def stack_workspace_bytes(n_extra, extra, n_main, main, keep=False, ckpt=False):
    """keep, ckpt: with the handle's option for kept activations (5) or for block inputs in 8 bits (7)."""
    e = C.byref(_dims(extra)) if extra is not None else None
    m = C.byref(_dims(main)) if main is not None else None
    f = (lib().pe_stack_workspace_bytes_keep if keep else lib().pe_stack_workspace_bytes_ckpt if ckpt
         else lib().pe_stack_workspace_bytes)
    return int(f(n_extra, e, n_main, m))


class Handle:
    def __init__(self):
        self._h = C.c_void_p()
        rc = lib().pe_create(C.byref(self._h))
        if rc:
            raise PEError("pe_create: " + strerror(rc))
        self.device = int(lib().pe_handle_device(self._h))      # index of the device that was current

    def set_option(self, opt, value):
        rc = lib().pe_set_option(self._h, opt, value)
        if rc:
            raise PEError(strerror(rc))

    def timing_collect(self):
        """Per-label kernel timings since the last call (PE_OPT_KERNEL_TIMING = 3 must be on)."""
        n = lib().pe_timing_collect(self._h, None, 0)
        if n < 0:
            raise PEError(strerror(n))
        arr = (_TimingEntry * max(n, 1))()
        n = lib().pe_timing_collect(self._h, arr, n)
        if n < 0:
            raise PEError(strerror(n))
        return [dict(name=e.name.decode(), kernel=e.kernel.decode(), launches=int(e.launches), total_ms=float(e.total_ms),
                     flops=float(e.flops), bytes=float(e.bytes)) for e in arr[:n]]

    def last_error(self):
        return lib().pe_last_error(self._h).decode()

    def close(self):
        if self._h:
            lib().pe_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _p(t):
    """Device pointer of a torch tensor (or None / int passthrough)."""
    if t is None:
        return None
    if isinstance(t, int):
        return C.c_void_p(t)
    return C.c_void_p(t.data_ptr())


_raw_stream = None      # torch's function device -> pointer of the current stream, once torch uses the GPU


def _find_raw_stream():
    global _raw_stream
    torch = sys.modules.get("torch")
    if torch is None or not torch.cuda.is_initialized():
        return None
    # 0.1 us; by the public call 1.1, a sixth of a small operator's call
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream


def _current_stream(device):
    """The stream that is current in torch on a device (0: the default stream, also where torch does not use the GPU)."""
    raw = _raw_stream or _find_raw_stream()
    return raw(device) if raw is not None else 0


def _s(h, stream):
    """hipStream_t of a stream argument: a torch stream, a pointer (0: the default stream), or None: torch's current stream."""
    return _current_stream(h.device) if stream is None else getattr(stream, "cuda_stream", stream)


def _raise(h, rc, what, dims=None):
    if rc:
        why = dims_error(dims) if (rc == -2 and dims is not None) else h.last_error()
        raise PEError("%s: %s %s" % (what, strerror(rc), why))


def block_fwd(h, dims, msa_in, pair_in, msa_mask, pair_mask, params, msa_out, pair_out, ctx, workspace,
              stream_msa=None, stream_pair=None):
    rc = lib().pe_block_fwd(h._h, C.byref(_dims(dims)), _p(msa_in), _p(pair_in), _p(msa_mask), _p(pair_mask),
                            _p(params), _p(msa_out), _p(pair_out), _p(ctx), _p(workspace),
                            workspace.numel() * workspace.element_size(), _s(h, stream_msa), _s(h, stream_pair))
    _raise(h, rc, "pe_block_fwd", dims)


def static_scratch_bytes():
    return int(lib().pe_static_scratch_bytes())


def block_fwd_static(h, dims, msa_in, pair_in, msa_mask, pair_mask, params, msa_out, pair_out,
                     stream_msa=None, stream_pair=None):
    rc = lib().pe_block_fwd_static(h._h, C.byref(_dims(dims)), _p(msa_in), _p(pair_in), _p(msa_mask), _p(pair_mask),
                                   _p(params), _p(msa_out), _p(pair_out), _s(h, stream_msa), _s(h, stream_pair))
    _raise(h, rc, "pe_block_fwd_static", dims)


def block_bwd(h, dims, msa_in, pair_in, msa_mask, pair_mask, params, d_msa_out, d_pair_out, d_msa_in, d_pair_in,
              d_params, ctx, workspace, stream_msa=None, stream_pair=None):
    rc = lib().pe_block_bwd(h._h, C.byref(_dims(dims)), _p(msa_in), _p(pair_in), _p(msa_mask), _p(pair_mask),
                            _p(params), _p(d_msa_out), _p(d_pair_out), _p(d_msa_in), _p(d_pair_in), _p(d_params),
                            _p(ctx), _p(workspace), workspace.numel() * workspace.element_size(),
                            _s(h, stream_msa), _s(h, stream_pair))
    _raise(h, rc, "pe_block_bwd", dims)


def stack_fwd_bwd(h, n_extra, extra, n_main, main, extra_msa_in, msa_in, pair_in, extra_mask, msa_mask, pair_mask,
                  params, d_msa_out, d_pair_out, msa_out, pair_out, d_extra_msa_in, d_msa_in, d_pair_in, d_params,
                  workspace, stream_msa=None, stream_pair=None):
    e = C.byref(_dims(extra)) if extra is not None else None
    m = C.byref(_dims(main)) if main is not None else None
    rc = lib().pe_stack_fwd_bwd(h._h, n_extra, e, n_main, m, _p(extra_msa_in), _p(msa_in), _p(pair_in),
                                _p(extra_mask), _p(msa_mask), _p(pair_mask), _p(params), _p(d_msa_out),
                                _p(d_pair_out), _p(msa_out), _p(pair_out), _p(d_extra_msa_in), _p(d_msa_in),
                                _p(d_pair_in), _p(d_params), _p(workspace),
                                workspace.numel() * workspace.element_size(), _s(h, stream_msa), _s(h, stream_pair))
    _raise(h, rc, "pe_stack_fwd_bwd")


# ---------------------------------------------------------------------------
# Operators around the trunk (include/pe.h says what they compute).  Tensors are torch tensors on the handle's device; a
# tensor [..., c] counts as rows of c channels, with gaps between the rows only where it has two dimensions.
# ---------------------------------------------------------------------------
_DTYPES = {}      # by torch type, filled as types come

# A size is passed as a C int, of which ctypes keeps the low 32 bits, and those may be a size in range: n >> 31 is 0 where n is one.


def _dtype(t):
    d = _DTYPES.get(t.dtype)
    if d is None:
        d = _DTYPES[t.dtype] = {"torch.float32": PE_F32, "torch.bfloat16": PE_BF16, "torch.uint8": PE_CKPT,
                                "torch.int32": "int32"}.get(str(t.dtype), "other")
    return d


def _on(h, t, what):
    if t.get_device() != h.device:      # -1: host memory
        raise PEError("%s: not on the handle's device" % what)


def _rows(h, t, what, like=None):
    """(type, rows, c, row stride) of a tensor of activations; `like`: what another one has to agree with."""
    if t.get_device() != h.device:
        _on(h, t, what)
    d, shape = _DTYPES.get(t.dtype), t.shape
    if d is None:
        d = _dtype(t)
    if (d != PE_F32 and d != PE_BF16) or not shape:
        raise PEError("%s: a float32 or bfloat16 tensor [..., c] is wanted" % what)
    c = shape[-1]
    if c >> 31:
        raise PEError("%s: %d channels are more than an operator takes" % (what, c))
    if t.is_contiguous():
        rows, ld = (t.numel() // c if c else 0), c
    elif len(shape) == 2 and (c == 1 or t.stride(1) == 1):
        rows, ld = shape[0], (t.stride(0) if shape[0] > 1 else c)
    else:
        raise PEError("%s: channels have to be neighbours in memory, rows of a tensor with more than two dimensions too" % what)
    if like is not None and (d, rows, c) != like:
        raise PEError("%s: shape or type differs" % what)
    return d, rows, c, ld


def _vec(h, t, n, what, dtype=PE_F32):
    """Device pointer of a contiguous tensor of n elements (None: NULL)."""
    if t is None:
        return None
    if t.get_device() != h.device:
        _on(h, t, what)
    if _dtype(t) != dtype or t.numel() != n or not t.is_contiguous():
        raise PEError("%s: a contiguous tensor of %d elements is wanted" % (what, n))
    return t.data_ptr()


def _bytes(h, t, n, what):
    if t is None:
        return None
    _on(h, t, what)
    if not t.is_contiguous() or t.nbytes < n:
        raise PEError("%s: %d contiguous bytes are wanted" % (what, n))
    return t.data_ptr()


def _op(h, rc, what):
    if rc:
        raise PEError("%s: %s %s" % (what, strerror(rc), h.last_error()))


def layernorm_fwd(h, x, gain, offset, y, eps=1e-5, add=None, stats=None, ckpt=None, stream=None):
    """y = [add +] LayerNorm(x); stats float32 [rows, 2]; ckpt: uint8 tensor of ckpt_bytes(rows, c) bytes that receives x."""
    d, rows, c, ld = _rows(h, x, "x")
    like = (d, rows, c)
    ldy = _rows(h, y, "y", like)[3]
    lda = _rows(h, add, "add", like)[3] if add is not None else 0
    _op(h, lib().pe_layernorm_fwd(
        h._h, rows, c, d, x.data_ptr(), ld, None if add is None else add.data_ptr(), lda, _vec(h, gain, c, "gain"),
        _vec(h, offset, c, "offset"), eps, y.data_ptr(), ldy, _vec(h, stats, 2 * rows, "stats"),
        None if ckpt is None else _bytes(h, ckpt, ckpt_bytes(rows, c), "ckpt"), _s(h, stream)), "pe_layernorm_fwd")


def layernorm_workspace_bytes(rows, c):
    return 0 if c >> 31 else int(lib().pe_layernorm_workspace_bytes(rows, c))


def layernorm_bwd(h, dy, x, stats, gain, dx, d_gain, d_offset, workspace, add=None, accumulate=False, stream=None):
    """Gradients of layernorm_fwd.  x: its input, or the uint8 checkpoint that it wrote.  dx, d_gain, d_offset: None where
    not wanted."""
    d, rows, c, ldy = _rows(h, dy, "dy")
    like = (d, rows, c)
    kept = _dtype(x) == PE_CKPT
    if kept:
        px, ldx = _bytes(h, x, ckpt_bytes(rows, c), "x"), 0
    else:
        ldx, px = _rows(h, x, "x", like)[3], x.data_ptr()
    lda = _rows(h, add, "add", like)[3] if add is not None else 0
    ldd = _rows(h, dx, "dx", like)[3] if dx is not None else 0
    ws = 0 if workspace is None else workspace.nbytes
    _op(h, lib().pe_layernorm_bwd(
        h._h, rows, c, d, PE_CKPT if kept else d, px, ldx, _vec(h, stats, 2 * rows, "stats"), _vec(h, gain, c, "gain"),
        dy.data_ptr(), ldy, None if add is None else add.data_ptr(), lda, None if dx is None else dx.data_ptr(), ldd,
        _vec(h, d_gain, c, "d_gain"), _vec(h, d_offset, c, "d_offset"), int(accumulate), _bytes(h, workspace, 0, "workspace"),
        ws, _s(h, stream)), "pe_layernorm_bwd")


def ckpt_bytes(rows, c):
    return 0 if c >> 31 else int(lib().pe_ckpt_bytes(rows, c))


def ckpt_pack(h, x, ckpt, stream=None):
    """x [..., c] in 8 bits into the uint8 tensor ckpt (ckpt_bytes(rows, c) bytes)."""
    d, rows, c, ld = _rows(h, x, "x")
    _op(h, lib().pe_ckpt_pack(h._h, rows, c, d, x.data_ptr(), ld, _bytes(h, ckpt, ckpt_bytes(rows, c), "ckpt"), _s(h, stream)),
        "pe_ckpt_pack")


def ckpt_unpack(h, ckpt, y, stream=None):
    d, rows, c, ld = _rows(h, y, "y")
    _op(h, lib().pe_ckpt_unpack(h._h, rows, c, d, _bytes(h, ckpt, ckpt_bytes(rows, c), "ckpt"), y.data_ptr(), ld, _s(h, stream)),
        "pe_ckpt_unpack")


_LAYOUTS = {"pair": PE_RELPOS_PAIR, "heads": PE_RELPOS_HEADS}


def _relpos(h, pos_q, pos_k, edges, t, seg_q, seg_k, layout, what):
    """Description of a call from its tensors: t is out or d_out, [q, k, c] or [c, q, k] with unit stride along its last axis
    ("pair": the last two axes without gaps)."""
    _on(h, t, what)
    if layout not in _LAYOUTS:
        raise PEError("layout: 'pair' or 'heads'")
    if (seg_q is None) != (seg_k is None):
        raise PEError("segments: seg_q and seg_k belong together")
    if edges.is_cuda or _dtype(edges) != "int32" or not edges.is_contiguous():
        raise PEError("edges: a contiguous int32 tensor in host memory is wanted")
    n_q, n_k = pos_q.numel(), pos_k.numel()
    pair, d = layout == "pair", _dtype(t)
    if d not in (PE_F32, PE_BF16) or t.dim() != 3:
        raise PEError("%s: a float32 or bfloat16 tensor of three dimensions is wanted" % what)
    s, st = t.shape, t.stride()
    c = s[2] if pair else s[0]
    if tuple(s) != ((n_q, n_k, c) if pair else (c, n_q, n_k)):
        raise PEError("%s: shape differs from the positions'" % what)
    if (n_q | n_k | c | edges.numel()) >> 31:
        raise PEError("%s: n_q and n_k up to 2^24, c up to 1024 and 254 edges are wanted" % what)
    ld = 0
    if not t.is_contiguous():
        ld = st[0] if pair or n_q == 1 else st[1]            # the stride of an axis of one element says nothing
        ok = (st[2] == 1 or s[2] == 1) and ((st[1] == c or n_k == 1) if pair else (st[0] == n_q * ld or c == 1))
        if not ok or ld < (n_k * c if pair else n_k):
            raise PEError("%s: gaps are allowed between rows q only" % what)
    p = _Relpos(n_q, n_k, c, edges.numel(), 0 if seg_q is None else 1, _LAYOUTS[layout], d, ld)
    ptr = (edges.data_ptr() if edges.numel() else None, _vec(h, pos_q, n_q, "pos_q", "int32"), _vec(h, pos_k, n_k, "pos_k", "int32"),
           _vec(h, seg_q, n_q, "seg_q", "int32"), _vec(h, seg_k, n_k, "seg_k", "int32"))
    return p, ptr, (edges.numel() + (1 if seg_q is None else 2)) * c


def relpos_fwd(h, pos_q, pos_k, edges, table, out, seg_q=None, seg_k=None, add=None, layout="pair", stream=None):
    """out = [add +] table[bucket(pos_q - pos_k)]; edges: int32 tensor in host memory, table float32 [buckets, c]."""
    p, ptr, n = _relpos(h, pos_q, pos_k, edges, out, seg_q, seg_k, layout, "out")
    if add is not None:
        _on(h, add, "add")
        same = add.dtype == out.dtype and add.shape == out.shape
        if same and add.stride() != out.stride() and not (add.is_contiguous() and out.is_contiguous()):
            same = all(a == o or n < 2 for a, o, n in zip(add.stride(), out.stride(), out.shape))      # of an axis of one element: any
        if not same:
            raise PEError("add: laid out as out is wanted")
    _op(h, lib().pe_relpos_fwd(h._h, C.byref(p), *ptr, _vec(h, table, n, "table"), None if add is None else add.data_ptr(),
                               out.data_ptr(), _s(h, stream)), "pe_relpos_fwd")


def relpos_workspace_bytes(n_q, n_k, c, buckets, layout="pair"):
    """Bytes for relpos_bwd; buckets: rows of the table."""
    segments = int(buckets > 1)
    if (n_q | n_k | c | buckets) >> 31:
        return 0
    p = _Relpos(n_q, n_k, c, buckets - 1 - segments, segments, _LAYOUTS[layout], PE_F32, 0)
    return int(lib().pe_relpos_workspace_bytes(C.byref(p)))


def relpos_bwd(h, pos_q, pos_k, edges, d_out, d_table, workspace, seg_q=None, seg_k=None, layout="pair", accumulate=False, stream=None):
    """d_table [buckets, c] = sum of d_out over the pairs of each bucket."""
    p, ptr, n = _relpos(h, pos_q, pos_k, edges, d_out, seg_q, seg_k, layout, "d_out")
    if workspace is None:
        raise PEError("workspace: relpos_workspace_bytes bytes are wanted")
    _op(h, lib().pe_relpos_bwd(h._h, C.byref(p), *ptr, d_out.data_ptr(), _vec(h, d_table, n, "d_table"), int(accumulate),
                               _bytes(h, workspace, 0, "workspace"), workspace.nbytes, _s(h, stream)),
        "pe_relpos_bwd")
