"""Thin Python binding of libhalp.so, the MI355X (gfx950) HALP epoch library.

Argument marshalling only: every step of the epoch runs in the library's HIP
kernels.  PyTorch is used for device memory and the stream handle.  There is
no CPU fallback: if the library has not been built, or a kernel does not cover
a shape, the call raises.
"""
import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhalp.so")

LOSS_SQUARED, LOSS_LOGISTIC, LOSS_SOFTMAX = 0, 1, 2
ALG_HALP, ALG_LPSVRG, ALG_SVRG = 0, 1, 2
OPT_INNER_VARIANT, OPT_TIMING, OPT_FULLGRAD_BLOCKS, OPT_INNER_WAVES, OPT_OPTION_II = 1, 2, 4, 5, 6
OPT_INNER_PARTS, OPT_EXCHANGE_SPIN_LIMIT, OPT_INNER_PACKED, OPT_INNER_HELPERS = 7, 8, 9, 10
OPT_EXCHANGE_POLL_DELAY = 11
OPT_GRADIENT_FP32 = 12
ERR_NULL, ERR_INVALID, ERR_UNSUPPORTED, ERR_NOT_BOUND, ERR_HIP, ERR_ALIGN = -1, -2, -3, -4, -5, -6
ERR_TOO_LARGE = -7
ERR_EXCHANGE_TIMEOUT = -8
TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
ROUND_NEAREST, ROUND_STOCHASTIC = 0, 1
STATIC_SCRATCH_BYTES = 16 << 20

EXPORTS = [
    "halp_create", "halp_destroy", "halp_bind", "halp_set_option", "halp_set_chain_hyper",
    "halp_set_feature_scale",
    "halp_quantize_data",
    "halp_full_gradient", "halp_full_gradient_static", "halp_recenter", "halp_inner_loop", "halp_epoch",
    "halp_inner_loop_trace", "halp_get_stats", "halp_debug_stream_words",
    "halp_debug_zround_bits", "halp_debug_read_bandwidth", "halp_debug_step_latency",
    "halp_mx4_quantize", "halp_mx4_dequantize", "halp_mx4_product", "halp_mx4_product_workspace", "halp_mx4_row_product",
    "halp_adamw_create", "halp_adamw_destroy", "halp_adamw_step", "halp_adamw_grad_norm", "halp_adamw_read_moments",
    "halp_strerror", "halp_last_error_detail", "halp_version",
]


class HalpError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        detail = lib().halp_last_error_detail().decode() if code == ERR_HIP else ""
        super().__init__(f"{what}: {strerror(code)} ({code})" + (f" [{detail}]" if detail else ""))


class Params(C.Structure):
    _fields_ = [
        ("N", C.c_int64), ("d", C.c_int32), ("K", C.c_int32), ("R", C.c_int32), ("loss", C.c_int32),
        ("b", C.c_int32), ("B", C.c_int32), ("share_data", C.c_int32), ("algorithm", C.c_int32),
        ("T", C.c_int64), ("alpha", C.c_double), ("mu", C.c_double), ("lam", C.c_double),
        ("delta_d", C.c_double), ("seed", C.c_uint64), ("delta", C.c_double),
    ]


class Buffers(C.Structure):
    _fields_ = [
        ("X", C.c_void_p), ("ldx", C.c_int64), ("Xq", C.c_void_p), ("ldxq", C.c_int64),
        ("y", C.c_void_p), ("w", C.c_void_p), ("phi", C.c_void_p), ("g", C.c_void_p),
        ("z", C.c_void_p), ("h", C.c_void_p), ("scales", C.c_void_p), ("counters", C.c_void_p),
    ]


class Stats(C.Structure):
    _fields_ = [
        ("delta_m", C.c_double), ("delta_i", C.c_double), ("delta_s", C.c_double),
        ("grad_norm", C.c_double), ("loss", C.c_double), ("status", C.c_int32),
        ("inner_variant", C.c_int32), ("n_clamped_z", C.c_uint64), ("n_clamped_gamma", C.c_uint64),
        ("n_reg_draws", C.c_uint64), ("ms_full_gradient", C.c_float), ("ms_recenter", C.c_float),
        ("ms_inner_loop", C.c_float), ("timed_epochs", C.c_int32),
        ("n_exchange_timeouts", C.c_uint64),
    ]


class Mx4Struct(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("ldc", C.c_int64), ("scales", C.c_void_p), ("lds", C.c_int64),
                ("rows", C.c_int64), ("cols", C.c_int64)]


class AdamWTensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_int64)]


class AdamWArgs(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("step", C.c_int64), ("step_at", C.c_void_p), ("lr_at", C.c_void_p),
                ("grad_scale", C.c_void_p)]


_lib = None


def lib():
    """Loads libhalp.so; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1803_03383_amd.build`")
        # torch first: the process must end up with ONE HIP runtime, the one torch's
        # allocations and streams live in; libhalp.so then binds to that copy
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        vp, i64, i32, u64, u32 = C.c_void_p, C.c_int64, C.c_int32, C.c_uint64, C.c_uint32
        L.halp_create.argtypes = [C.POINTER(vp), C.POINTER(Params)]
        L.halp_destroy.argtypes = [vp]
        L.halp_bind.argtypes = [vp, C.POINTER(Buffers)]
        L.halp_set_option.argtypes = [vp, i32, i64]
        L.halp_set_chain_hyper.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double)]
        L.halp_set_feature_scale.argtypes = [vp, vp]
        L.halp_quantize_data.argtypes = [vp, vp]
        L.halp_full_gradient.argtypes = [vp, vp]
        L.halp_full_gradient_static.argtypes = [C.POINTER(Params), C.POINTER(Buffers), vp]
        L.halp_recenter.argtypes = [vp, i64, vp]
        L.halp_inner_loop.argtypes = [vp, i64, vp]
        L.halp_epoch.argtypes = [vp, i64, vp]
        L.halp_inner_loop_trace.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp]
        L.halp_get_stats.argtypes = [vp, i32, vp, C.POINTER(Stats)]
        L.halp_debug_stream_words.argtypes = [u64, u32, u32, u64, i64, vp, vp]
        L.halp_debug_zround_bits.argtypes = [u64, u32, u64, i32, i32, i32, vp, vp]
        L.halp_debug_read_bandwidth.argtypes = [vp, i64, vp, vp]
        L.halp_debug_step_latency.argtypes = [i32, i64, i32, vp, vp]
        mx = C.POINTER(Mx4Struct)
        L.halp_mx4_quantize.argtypes = [vp, i32, i64, i64, i64, mx, mx, i32, u64, i64, vp]
        L.halp_mx4_dequantize.argtypes = [mx, vp, i32, i64, vp]
        L.halp_mx4_product.argtypes = [mx, mx, vp, i32, i64, i32, vp, i64, vp]
        L.halp_mx4_product_workspace.argtypes = [i64, i64, i64, C.POINTER(i64)]
        L.halp_mx4_row_product.argtypes = [vp, i32, i64, i64, mx, vp, i32, i64, vp]
        L.halp_adamw_create.argtypes = [C.POINTER(vp), C.POINTER(AdamWTensor), i64, i32, i32, i32, u64]
        L.halp_adamw_destroy.argtypes = [vp]
        L.halp_adamw_step.argtypes = [vp, C.POINTER(AdamWArgs), vp]
        L.halp_adamw_grad_norm.argtypes = [vp, C.c_double, vp, vp]
        L.halp_adamw_read_moments.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp]
        for name in EXPORTS:
            getattr(L, name).restype = C.c_int
        L.halp_strerror.restype = C.c_char_p
        L.halp_strerror.argtypes = [C.c_int]
        L.halp_last_error_detail.restype = C.c_char_p
        L.halp_last_error_detail.argtypes = []
        L.halp_version.restype = C.c_char_p
        L.halp_version.argtypes = []
        _lib = L
    return _lib


def strerror(code):
    return lib().halp_strerror(int(code)).decode()


def version():
    return lib().halp_version().decode()


def _check(rc, what):
    if rc != 0:
        raise HalpError(rc, what)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    return C.c_void_p(int(stream))


class Halp:
    """One handle: R chains of an N x d problem.  Tensors are torch CUDA tensors
    owned by the caller; the handle keeps references so they outlive it."""

    def __init__(self, N, d, K=1, R=1, loss=LOSS_SQUARED, b=8, B=1, T=0, alpha=0.01, mu=1.0,
                 lam=0.0, delta_d=1.0, seed=0, share_data=False, algorithm=ALG_HALP, delta=0.0):
        self.params = Params(N=N, d=d, K=K, R=R, loss=loss, b=b, B=B, share_data=int(share_data),
                             algorithm=algorithm, T=T, alpha=alpha, mu=mu, lam=lam,
                             delta_d=delta_d, seed=seed, delta=delta)
        self._h = C.c_void_p()
        _check(lib().halp_create(C.byref(self._h), C.byref(self.params)), "halp_create")
        self._keep = {}

    def close(self):
        if self._h:
            lib().halp_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def bind(self, X=None, Xq=None, y=None, w=None, phi=None, g=None, z=None, h=None, scales=None,
             counters=None, ldx=None, ldxq=None):
        self._keep = dict(X=X, Xq=Xq, y=y, w=w, phi=phi, g=g, z=z, h=h, scales=scales,
                          counters=counters, fscale=self._keep.get("fscale"))
        b = Buffers()
        b.X, b.Xq, b.y, b.w, b.phi, b.g = _ptr(X), _ptr(Xq), _ptr(y), _ptr(w), _ptr(phi), _ptr(g)
        b.z, b.h, b.scales, b.counters = _ptr(z), _ptr(h), _ptr(scales), _ptr(counters)
        b.ldx = int(ldx if ldx is not None else (X.stride(-2) if X is not None else self.params.d))
        b.ldxq = int(ldxq if ldxq is not None else (Xq.stride(-2) if Xq is not None else self.params.d))
        _check(lib().halp_bind(self._h, C.byref(b)), "halp_bind")

    def set_option(self, option, value):
        _check(lib().halp_set_option(self._h, option, value), "halp_set_option")

    def set_chain_hyper(self, alpha=None, mu=None):
        """Per-chain step size and mu (sequences of R floats, or None for the handle's)."""
        def arr(v):
            if v is None:
                return None
            v = [float(x) for x in v]
            if len(v) != self.params.R:
                raise ValueError("one value per chain expected")
            return (C.c_double * len(v))(*v)
        _check(lib().halp_set_chain_hyper(self._h, arr(alpha), arr(mu)), "halp_set_chain_hyper")

    def set_feature_scale(self, s=None):
        """Per-feature data scales: a float32 CUDA tensor of d entries, or None to switch off."""
        self._keep["fscale"] = s
        _check(lib().halp_set_feature_scale(self._h, _ptr(s)), "halp_set_feature_scale")

    def quantize_data(self, stream=None):
        _check(lib().halp_quantize_data(self._h, _stream(stream)), "halp_quantize_data")

    def full_gradient(self, stream=None):
        _check(lib().halp_full_gradient(self._h, _stream(stream)), "halp_full_gradient")

    def recenter(self, epoch, stream=None):
        _check(lib().halp_recenter(self._h, epoch, _stream(stream)), "halp_recenter")

    def inner_loop(self, epoch, stream=None):
        _check(lib().halp_inner_loop(self._h, epoch, _stream(stream)), "halp_inner_loop")

    def epoch(self, epoch, stream=None):
        _check(lib().halp_epoch(self._h, epoch, _stream(stream)), "halp_epoch")

    def inner_loop_trace(self, epoch, M, idx=None, D=None, beta=None, gamma=None, ztraj=None,
                         stream=None):
        _check(lib().halp_inner_loop_trace(self._h, epoch, M, _ptr(idx), _ptr(D), _ptr(beta),
                                           _ptr(gamma), _ptr(ztraj), _stream(stream)),
               "halp_inner_loop_trace")

    def get_stats(self, chain=0, stream=None):
        s = Stats()
        rc = lib().halp_get_stats(self._h, chain, _stream(stream), C.byref(s))
        if rc == ERR_EXCHANGE_TIMEOUT:  # the statistics are complete; the caller sees both
            err = HalpError(rc, "halp_get_stats")
            err.stats = s
            raise err
        _check(rc, "halp_get_stats")
        return s


def full_gradient_static(params, X, y, w, phi, g, scales, ldx=None, stream=None):
    """halp_full_gradient without a handle and without any allocation: the partial sums go
    through the library's fixed device array.  params: a Params; the rest torch CUDA tensors."""
    b = Buffers()
    b.X, b.y, b.w, b.phi, b.g, b.scales = _ptr(X), _ptr(y), _ptr(w), _ptr(phi), _ptr(g), _ptr(scales)
    b.ldx = int(ldx if ldx is not None else X.stride(-2))
    _check(lib().halp_full_gradient_static(C.byref(params), C.byref(b), _stream(stream)),
           "halp_full_gradient_static")


def alloc_state(N, d, K=1, R=1, b=8, device="cuda"):
    """Allocates the library's output / state buffers as torch tensors."""
    import torch

    zt = torch.int8 if b == 8 else torch.int16
    ht = torch.int16 if b == 8 else torch.int32
    return dict(
        w=torch.zeros((R, K, d), dtype=torch.float32, device=device),
        phi=torch.zeros((R, N, K), dtype=torch.float32, device=device),
        g=torch.zeros((R, K, d), dtype=torch.float32, device=device),
        z=torch.zeros((R, K, d), dtype=zt, device=device),
        h=torch.zeros((R, K, d), dtype=ht, device=device),
        scales=torch.zeros((R, 8), dtype=torch.float64, device=device),
        counters=torch.zeros((R, 4), dtype=torch.int64, device=device),
    )


def debug_stream_words(seed, purpose, epoch, n0, count, stream=None):
    import torch

    out = torch.zeros((count,), dtype=torch.int32, device="cuda")
    _check(lib().halp_debug_stream_words(seed, purpose, epoch, n0, count, _ptr(out),
                                         _stream(stream)), "halp_debug_stream_words")
    return out


def debug_zround_bits(seed, epoch, t, d, b, K, stream=None):
    import torch

    out = torch.zeros((K, d), dtype=torch.int32, device="cuda")
    _check(lib().halp_debug_zround_bits(seed, epoch, t, d, b, K, _ptr(out), _stream(stream)),
           "halp_debug_zround_bits")
    return out


def debug_read_bandwidth(t, out=None, stream=None):
    """Reads tensor t (contiguous, a multiple of 16 bytes) once; returns the checksum tensor."""
    import torch
    if out is None:
        out = torch.empty(2048, dtype=torch.int32, device=t.device)
    nbytes = t.numel() * t.element_size()
    _check(lib().halp_debug_read_bandwidth(_ptr(t), nbytes, _ptr(out), _stream(stream)),
           "halp_debug_read_bandwidth")
    return out


def debug_step_latency(waves, steps, blocks, out=None, stream=None):
    """Runs the isolated dependent chain of an 8-bit inner-loop step; returns its output tensor."""
    import torch
    if out is None:
        out = torch.empty(blocks * waves * 64, dtype=torch.int32, device="cuda")
    if out.numel() < blocks * waves * 64:
        raise ValueError("out holds fewer than blocks * waves * 64 words")
    _check(lib().halp_debug_step_latency(waves, steps, blocks, _ptr(out), _stream(stream)),
           "halp_debug_step_latency")
    return out


# ---- operators without a handle: 4-bit microscaled matrices, AdamW ---------------------------

_torch = None
_TYPES = {}


def _load_torch():
    global _torch
    if _torch is None:
        import torch
        _TYPES.update({torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16})
        _torch = torch
    return _torch


def _type(t, what):
    _load_torch()
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what}: float32, bfloat16 or float16 expected, not {t.dtype}")
    return code


def _matrix(t, what, rows=None, cols=None):
    """A 2-D tensor with unit stride along its rows; returns its row stride."""
    if t.dim() != 2:
        raise ValueError(f"{what}: a 2-D tensor expected")
    (m, n), (ld, one) = t.shape, t.stride()
    if n > 1 and one != 1:
        raise ValueError(f"{what}: a unit stride along the rows expected")
    if rows is not None and (m != rows or n != cols):
        raise ValueError(f"{what}: shape ({rows}, {cols}) expected, not ({m}, {n})")
    return ld if m > 1 else max(n, 1)  # the stride of a single row is whatever torch has it be


def _same_device(t, *others):
    """The index of the GPU that all tensors are on."""
    dev = t.get_device()
    for o in others:
        if o is not None and o.get_device() != dev:
            raise ValueError(f"tensors on {t.device} and {o.device}")
    if dev < 0:
        raise ValueError(f"GPU tensors expected, not {t.device}")
    return dev


def _count(n):
    """A number that the library takes in 32 of 64 bits; -1, which it refuses, in place of what ctypes would cut to 64."""
    return n if 0 <= n < 2 ** 32 else -1


def _run(name, dev, stream, *args):
    """Calls the library with device `dev` current, on the stream given or on that device's current one."""
    torch = _load_torch()
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(dev)
    f = getattr(lib(), name)
    if torch._C._cuda_getDevice() == dev:
        rc = f(*args, stream)
    else:
        with torch.cuda.device(dev):
            rc = f(*args, stream)
    if rc != 0:
        raise HalpError(rc, name)


class Mx4:
    """A matrix in 4-bit microscaled form: codes uint8 [rows, >= 64 groups], scales uint8 [rows, >= 4 groups],
    groups = ceil(cols / 128)."""

    def __init__(self, codes, scales, cols):
        torch = _load_torch()
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
            raise ValueError("codes and scales are uint8 tensors")
        groups = (cols + 127) // 128
        ldc, lds = _matrix(codes, "codes"), _matrix(scales, "scales")
        if codes.shape[0] != scales.shape[0] or codes.shape[1] < 64 * groups or scales.shape[1] < 4 * groups:
            raise ValueError(f"codes {tuple(codes.shape)} and scales {tuple(scales.shape)} do not hold rows of {cols} columns")
        if codes.device != scales.device:
            raise ValueError("codes and scales are on two devices")
        self.codes, self.scales, self.rows, self.cols = codes, scales, codes.shape[0], cols
        # a single row has no stride to speak of: whole groups
        self.c = Mx4Struct(codes.data_ptr(), ldc if self.rows > 1 else 64 * groups, scales.data_ptr(),
                           lds if self.rows > 1 else 4 * groups, self.rows, cols)
        self.ref = C.byref(self.c)


def mx4_empty(rows, cols, device="cuda"):
    """Allocates an Mx4 whose contents are not set."""
    torch = _load_torch()
    groups = (cols + 127) // 128
    return Mx4(torch.empty((rows, 64 * groups), dtype=torch.uint8, device=device),
               torch.empty((rows, 4 * groups), dtype=torch.uint8, device=device), cols)


def mx4_quantize(x, q=None, qt=None, rounding=ROUND_NEAREST, seed=0, epoch=0, stream=None):
    """x [rows, cols] into q (Mx4 of its rows) and qt (Mx4 of its transpose), whichever are given."""
    dev = _same_device(x, q and q.codes, qt and qt.codes)
    _run("halp_mx4_quantize", dev, stream, x.data_ptr(), _type(x, "x"), x.shape[0], x.shape[-1], _matrix(x, "x"),
         q and q.ref, qt and qt.ref, rounding, seed & (2 ** 64 - 1), _count(epoch))


def mx4_dequantize(q, out, stream=None):
    """The values of q into out [rows, cols]."""
    ldo = _matrix(out, "out", q.rows, q.cols)
    _run("halp_mx4_dequantize", _same_device(out, q.codes), stream, q.ref, out.data_ptr(), _type(out, "out"), ldo)


def mx4_product_workspace(M, N, K):
    """Bytes of workspace with which mx4_product can cut K, on the current device."""
    n = C.c_int64()
    _check(lib().halp_mx4_product_workspace(M, N, K, C.byref(n)), "halp_mx4_product_workspace")
    return n.value


def mx4_product(a, b, out, accumulate=False, workspace=None, stream=None):
    """out [M, N] = a [M, K] b [N, K]^T, added to out where accumulate is set; workspace: a contiguous tensor or None."""
    ldc = _matrix(out, "out", a.rows, b.rows)
    dev = _same_device(out, a.codes, b.codes, workspace)
    at, room = None, 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace: a contiguous tensor expected")
        at, room = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _run("halp_mx4_product", dev, stream, a.ref, b.ref, out.data_ptr(), _type(out, "out"), ldc, 1 if accumulate else 0, at, room)


def mx4_row_product(x, w, out, stream=None):
    """out [M, N] = x [M, K], quantized to the nearest on the way, times w [N, K]^T; M <= 16."""
    M = x.shape[0]
    ldx, ldy = _matrix(x, "x", M, w.cols), _matrix(out, "out", M, w.rows)
    _run("halp_mx4_row_product", _same_device(x, w.codes, out), stream, x.data_ptr(), _type(x, "x"), M, ldx, w.ref,
         out.data_ptr(), _type(out, "out"), ldy)


class AdamW:
    """The AdamW step of a list of tensors as one launch.  tensors: dicts of contiguous GPU tensors
    p (float32), g (one of three types, the same for all), m, v (float32; with state_bits 8 uint8 codes), with
    state_bits 8 also m_scale, v_scale (uint8, ceil(n / 32)), and optionally copy (the new p in a
    narrower type).  The handle keeps references to them."""

    def __init__(self, tensors, state_bits=32, seed=0):
        torch = _load_torch()
        self._h = C.c_void_p()
        tensors = [dict(t) for t in tensors]
        if not tensors:
            raise ValueError("at least one tensor expected")
        self._keep = tensors
        state, dev = (torch.float32 if state_bits == 32 else torch.uint8), tensors[0]["p"].device
        copies = {_type(t["copy"], "copy") for t in tensors if t.get("copy") is not None}
        grads = {_type(t["g"], "g") for t in tensors}
        if len(grads) > 1 or len(copies) > 1:
            raise ValueError("all g have one type, and all copy")
        want = {"p": torch.float32, "g": None, "copy": None, "m": state, "v": state}
        if state_bits == 8:
            want |= {"m_scale": torch.uint8, "v_scale": torch.uint8}
        arr = (AdamWTensor * len(tensors))()
        for a, t in zip(arr, tensors):
            a.n = t["p"].numel()
            for name, dtype in want.items():
                x = t.get(name)
                if x is None:
                    if name != "copy":
                        raise ValueError(f"{name} is missing")
                    continue
                if (dtype is not None and x.dtype != dtype) or not x.is_contiguous() or x.device != dev:
                    raise ValueError(f"{name}: a contiguous {dtype or 'floating-point'} tensor on {dev} expected")
                if x.numel() != ((a.n + 31) // 32 if name.endswith("_scale") else a.n):
                    raise ValueError(f"{name}: {x.numel()} elements for a tensor of {a.n}")
                setattr(a, name, x.data_ptr())
        self._dev = _same_device(tensors[0]["p"])
        with torch.cuda.device(self._dev):
            _check(lib().halp_adamw_create(C.byref(self._h), arr, len(tensors), state_bits, grads.pop(),
                                           copies.pop() if copies else TYPE_BF16, seed & (2 ** 64 - 1)), "halp_adamw_create")

    def close(self):
        if self._h:
            lib().halp_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=None, step_at=None,
             lr_at=None, stream=None):
        """One step.  step counts from 1; step_at (int64) and lr_at (float32), one-element GPU tensors, take the place of
        step and lr where given; grad_scale (float32, one element) scales the gradients.  Where one of the three is out
        of its range on the GPU (step_at from 1 to 2^32 - 1, lr_at finite and not negative, grad_scale finite), the step is skipped."""
        at = []
        for name, t, dtype in (("step_at", step_at, _torch.int64), ("lr_at", lr_at, _torch.float32),
                               ("grad_scale", grad_scale, _torch.float32)):
            if t is None:
                at.append(None)
                continue
            if t.dtype != dtype or t.numel() != 1:
                raise ValueError(f"{name}: one {dtype} expected")
            if _same_device(t) != self._dev:
                raise ValueError(f"{name}: on {t.device}, the tensors on cuda:{self._dev}")
            at.append(t.data_ptr())
        a = AdamWArgs(lr, beta1, beta2, eps, weight_decay, _count(step), *at)
        _run("halp_adamw_step", self._dev, stream, self._h, C.byref(a))

    def grad_norm(self, max_norm, out, stream=None):
        """out (float32 [2]): the norm of all gradients, and the grad_scale that clips it to max_norm."""
        if out.dtype != _torch.float32 or out.numel() != 2 or not out.is_contiguous():
            raise ValueError("out: two contiguous float32 expected")
        if _same_device(out) != self._dev:
            raise ValueError(f"out: on {out.device}, the tensors on cuda:{self._dev}")
        _run("halp_adamw_grad_norm", self._dev, stream, self._h, max_norm, out.data_ptr())


def adamw_read_moments(m, m_scale, v, v_scale, m_out, v_out, stream=None):
    """The values of 8-bit states (uint8 codes and scales) as float32."""
    torch, n = _load_torch(), m.numel()
    k = (n + 31) // 32
    for name, t, dtype, count in (("m", m, torch.uint8, n), ("m_scale", m_scale, torch.uint8, k), ("v", v, torch.uint8, n),
                                  ("v_scale", v_scale, torch.uint8, k), ("m_out", m_out, torch.float32, n),
                                  ("v_out", v_out, torch.float32, n)):
        if t.dtype != dtype or t.numel() != count or not t.is_contiguous():
            raise ValueError(f"{name}: {count} contiguous {dtype} expected")
    _run("halp_adamw_read_moments", _same_device(m, m_scale, v, v_scale, m_out, v_out), stream, m.data_ptr(), m_scale.data_ptr(),
         v.data_ptr(), v_scale.data_ptr(), n, m_out.data_ptr(), v_out.data_ptr())
