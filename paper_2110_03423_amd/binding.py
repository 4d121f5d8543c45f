"""ctypes binding of the C ABI in include/rsvd.h (argument marshalling only)."""
import ctypes as C
import os

F32, F64 = 0, 1
DEVICE_NONE = -1        # rsvd_create: planning context, no HIP call
ERR_NO_DEVICE = 5
JOB_S, JOB_SV, JOB_SUV = 0, 1, 2

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class RsvdError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"rsvd error {code}: {text}")
        self.code = code


class _Info(C.Structure):
    _fields_ = [("status", C.c_int32), ("jacobi_sweeps", C.c_int32),
                ("refilled_columns", C.c_int32), ("skipped_reorth", C.c_int32), ("raised_pivots", C.c_int32)]


def library_path():
    return os.path.join(_HERE, "librsvd_gfx950.so")


_I64, _INT, _U64, _U32, _VP, _SZ = C.c_int64, C.c_int, C.c_uint64, C.c_uint32, C.c_void_p, C.c_size_t

# name -> argument types; mirrors include/rsvd.h
PROTOTYPES = {
    "rsvd_create": [C.POINTER(_VP), _INT],
    "rsvd_destroy": [_VP],
    "rsvd_status_string": [_INT],
    "rsvd_last_hip_error": [_VP],
    "rsvd_profile_enable": [_VP, _INT],
    "rsvd_profile_read": [_VP, _INT, C.POINTER(C.c_double), C.POINTER(_INT)],
    "rsvd_profile_kind_name": [_INT],
    "rsvd_workspace_bytes": [_VP, _INT, _I64, _I64, _INT, _INT, _INT, _INT, C.POINTER(_SZ)],
    "rsvd_run": [_VP, _VP, _INT, _INT, _I64, _I64, _VP, _I64, _INT, _INT, _INT, _U64,
                 _VP, _VP, _I64, _VP, _I64, _VP, _SZ, C.POINTER(_Info)],
    "rsvd_run_static": [_VP, _VP, _INT, _INT, _I64, _I64, _VP, _I64, _INT, _INT, _INT, _U64,
                        _VP, _VP, _I64, _VP, _I64, C.POINTER(_Info)],
    "rsvd_static_scratch_bytes": [],
    "rsvd_run_centered": [_VP, _VP, _INT, _INT, _I64, _I64, _VP, _I64, _INT, _INT, _INT, _U64,
                          _VP, _VP, _I64, _VP, _I64, _VP, _SZ, C.POINTER(_Info), _VP],
    "rsvd_workspace_bytes_batched": [_VP, _INT, _INT, _I64, _I64, _INT, _INT, _INT, _INT, C.POINTER(_SZ)],
    "rsvd_run_batched": [_VP, _VP, _INT, _INT, _INT, _I64, _I64, _VP, _I64, _I64, _INT, _INT, _INT, _U64,
                         _VP, _I64, _VP, _I64, _I64, _VP, _I64, _I64, _VP, _SZ, C.POINTER(_Info)],
    "rsvd_stage_workspace_bytes": [_VP, _INT, _I64, _I64, C.POINTER(_SZ)],
    "rsvd_stage_sketch": [_VP, _VP, _INT, _U64, _U32, _I64, _I64, _VP, _I64],
    "rsvd_stage_philox_raw": [_VP, _VP, _U64, _U32, _U64, _I64, _VP],
    "rsvd_stage_gemm_an": [_VP, _VP, _INT, _I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _SZ],
    "rsvd_stage_gemm_atn": [_VP, _VP, _INT, _I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _SZ],
    "rsvd_stage_orth": [_VP, _VP, _INT, _I64, _I64, _VP, _I64, _VP, _U64, _U32, _VP, _SZ, C.POINTER(_Info)],
    "rsvd_stage_small_svd": [_VP, _VP, _INT, _I64, _I64, _VP, _I64, _VP, _VP, _VP, _I64, _U64, _VP, _SZ,
                             C.POINTER(_Info)],
    "rsvd_stage_jacobi": [_VP, _VP, _INT, _I64, _VP, _VP, _VP, _VP, _VP, _SZ, C.POINTER(_Info)],
    "rsvd_stage_lift": [_VP, _VP, _INT, _I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _INT, _VP, _SZ],
    "rsvd_q8_rows": [_VP, _VP, _INT, _I64, _I64, _VP, _I64, _VP, _I64, _VP],
    "rsvd_q8_product_bytes": [_VP, _INT, _I64, _I64, _I64, _I64, C.POINTER(_SZ)],
    "rsvd_q8_product_grad_bytes": [_VP, _INT, _I64, _I64, _I64, _I64, C.POINTER(_SZ)],
    "rsvd_keep8_grad_bytes": [_VP, _INT, _I64, _I64, _I64, C.POINTER(_SZ)],
    "rsvd_q8_product": [_VP, _VP, _INT, _I64, _I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _VP, _I64, _VP, _I64, _VP, _VP,
                        _I64, _VP, _SZ],
    "rsvd_q8_product_grad": [_VP, _VP, _INT, _I64, _I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _VP, _I64, _VP, _I64, _VP,
                             _I64, _VP, _SZ],
    "rsvd_keep8_save": [_VP, _VP, _INT, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64],
    "rsvd_keep8_load": [_VP, _VP, _INT, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64],
    "rsvd_keep8_grad": [_VP, _VP, _INT, _I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _INT, _VP, _SZ],
}
X_BF16, X_F16, X_F32 = 0, 1, 2


def load_library():
    """Load librsvd_gfx950.so; raises if it has not been built (no fallback path exists)."""
    global _LIB
    if _LIB is None:
        # torch first: it brings its own HIP runtime, and the library must bind to that one
        # (loading the library first pulls in another copy and torch then sees no GPU)
        import torch  # noqa: F401
        path = library_path()
        if not os.path.exists(path):
            raise RsvdError(-1, f"{path} is missing: build it with `python -m paper_2110_03423_amd.build`")
        lib = C.CDLL(path)
        for name, argtypes in PROTOTYPES.items():
            fn = getattr(lib, name)
            fn.argtypes = argtypes
            if name in ("rsvd_status_string", "rsvd_last_hip_error", "rsvd_profile_kind_name"):
                fn.restype = C.c_char_p
            elif name == "rsvd_static_scratch_bytes":
                fn.restype = C.c_size_t
            else:
                fn.restype = C.c_int
        _LIB = lib
    return _LIB


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.float64:
        return F64
    raise TypeError("fp32 or fp64 tensors only")


_XTYPES = {}


def _xtype_code(dtype):
    if not _XTYPES:
        import torch
        _XTYPES.update({torch.bfloat16: X_BF16, torch.float16: X_F16, torch.float32: X_F32})
    try:
        return _XTYPES[dtype]
    except KeyError:
        raise TypeError("bf16, fp16 or fp32 tokens only") from None


def _empty_codes(rows, n, device):
    """Room for `rows` rows of 8-bit codes, each a multiple of 128 bytes long; the view has n columns."""
    import torch
    codes = torch.empty((rows, -(-n // 128) * 128), dtype=torch.int8, device=device)
    return codes if n % 128 == 0 else codes[:, :n]


def _laid_out(codes):
    """The codes in rows as the C entry points want them (a copy unless they are already)."""
    rows, n = codes.shape
    if codes.stride(1) == 1 and codes.stride(0) % 128 == 0 and codes.stride(0) >= n and codes.data_ptr() % 16 == 0:
        # (rows are read in 16-byte pieces; the last one's may reach behind what the tensor was cut out of)
        if codes.storage_offset() + (rows - 1) * codes.stride(0) + -(-n // 16) * 16 <= codes.untyped_storage().nbytes():
            return codes
    out = _empty_codes(rows, n, codes.device)
    out.copy_(codes)
    return out


def _together(first, **others):
    """The device that all of a layer's (or a kept activation's) tensors are on."""
    for name, t in others.items():
        if t is not None and t.device != first.device:
            raise ValueError(f"{name}: on {t.device}, the codes on {first.device}")
    return first.device


def _ld(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


class Weight8:
    """A linear layer's weight (m x n) as rsvd_q8_product takes it: 8-bit codes with a scale for each row, and beside them
    bf16 factors U (m x r), Vt (r x n) or None; bias: m values or None.

    The layer's tensors are `codes`, `scale`, `U`, `Vt` and `bias`: those that were given where they lie as the kernels want
    them (contiguous; codes in rows of a multiple of 128 bytes; an fp32 bias), copies where they do not.  Their values may change in
    place, and every call takes what they hold then."""

    def __init__(self, codes, scale, U=None, Vt=None, bias=None):
        import torch
        if codes.dtype != torch.int8 or codes.dim() != 2:
            raise TypeError("codes: an int8 matrix")
        m, n = codes.shape
        if scale.dtype != torch.float32 or scale.shape != (m,):
            raise ValueError("scale: one fp32 value for each row of codes")
        if (U is None) != (Vt is None):
            raise ValueError("U and Vt come together")
        self.device = _together(codes, scale=scale, U=U, Vt=Vt, bias=bias)
        self.codes, self.scale = _laid_out(codes), scale.contiguous()
        self.m, self.n, self.r = m, n, 0
        self.U = self.Vt = None
        if U is not None and U.shape[1] > 0:
            if U.dtype != torch.bfloat16 or Vt.dtype != torch.bfloat16:
                raise TypeError("U, Vt: bf16 factors")
            if U.shape[0] != m or Vt.shape != (U.shape[1], n):
                raise ValueError("U, Vt: m x r and r x n")
            self.r = U.shape[1]
            self.U, self.Vt = U.contiguous(), Vt.contiguous()
        if bias is not None and bias.shape != (m,):
            raise ValueError("bias: m values")
        self.bias = None if bias is None else bias.float().contiguous()
        self._index = self.codes.get_device()      # (-1: not on a GPU)
        self._sizes = (n, m, self.r)

    # The factors by rows of the other index, for the backward pass.  Made anew each time: nothing tells reliably whether U and Vt
    # have changed since (an optimizer that writes through `.data` leaves no trace), or on which stream.
    @property
    def Ut(self):
        return None if self.U is None else self.U.t().contiguous()

    @property
    def V(self):
        return None if self.Vt is None else self.Vt.t().contiguous()

    def __setattr__(self, name, value):
        if "_sizes" in self.__dict__:
            raise AttributeError("a Weight8 keeps its tensors (their values may change): make another one")
        object.__setattr__(self, name, value)


class Kept8:
    """Activations (tokens x n) kept in 8 bits: codes, and a byte of power for each 32 of them (rsvd_keep8_save).  `dtype` is
    the type of the activations."""

    def __init__(self, codes, powers, dtype):
        import torch
        if codes.dtype != torch.int8 or codes.dim() != 2 or powers.dtype != torch.uint8:
            raise TypeError("codes: an int8 matrix; powers: uint8")
        if powers.shape != (codes.shape[0], -(-codes.shape[1] // 32)):
            raise ValueError("powers: one byte for each 32 columns of codes")
        _xtype_code(dtype)
        _together(codes, powers=powers)
        if powers.stride(0) < powers.shape[1] or (powers.stride(1) != 1 and powers.shape[1] > 1):
            powers = powers.contiguous()
        self._set(_laid_out(codes), powers, dtype)

    def _set(self, codes, powers, dtype):
        self.codes, self.powers, self.dtype = codes, powers, dtype
        self.tokens, self.n = codes.shape
        self.device, self._index = codes.device, codes.get_device()
        return self


def _at(t):
    return t.data_ptr() if t is not None else None


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


class Rsvd:
    """One context per device.  Methods mirror the C entry points by name."""

    def __init__(self, device=0):
        """device=None gives a planning context (RSVD_DEVICE_NONE): workspace sizes and argument checks only,
        no GPU and no torch needed."""
        self.lib = load_library()
        self._ws = None
        self._needs = {}        # workspace of the layer calls, by their sizes
        self._layer = {}        # and the workspaces themselves, one for each stream
        h = C.c_void_p()
        if device is None:
            self.torch = None
            self.device = self._index = None
            rc = self.lib.rsvd_create(C.byref(h), DEVICE_NONE)
        else:
            import torch
            self.torch = torch
            self.device, self._index = torch.device("cuda", device), device
            rc = self.lib.rsvd_create(C.byref(h), device)
        if rc != 0:
            raise RsvdError(rc, "rsvd_create failed (no such device?)")
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.rsvd_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- helpers
    def _check(self, rc):
        if rc != 0:
            text = self.lib.rsvd_status_string(rc).decode()
            if rc == 3 and getattr(self, "h", None):
                text += " (" + self.lib.rsvd_last_hip_error(self.h).decode() + ")"
            raise RsvdError(rc, text)

    def _stream(self):
        return C.c_void_p(self.torch.cuda.current_stream(self.device).cuda_stream)

    def _raw_stream(self):
        """The current stream's handle, by the short way where torch has it (a tenth of the time, which small layer calls notice)."""
        get = getattr(self.torch._C, "_cuda_getCurrentRawStream", None)
        return get(self.device.index) if get is not None else self.torch.cuda.current_stream(self.device).cuda_stream

    def rsvd_profile_enable(self, on):
        self._check(self.lib.rsvd_profile_enable(self.h, int(on)))

    def rsvd_profile_read(self):
        """{kernel class name: (total ms, launches)} since the last read."""
        n = 12
        ms = (C.c_double * n)()
        cnt = (C.c_int * n)()
        self._check(self.lib.rsvd_profile_read(self.h, n, ms, cnt))
        return {self.lib.rsvd_profile_kind_name(i).decode(): (ms[i], cnt[i]) for i in range(n) if cnt[i] > 0}

    def workspace_bytes(self, dtype, m, n, k, p, q=0, job=JOB_SUV):
        out = C.c_size_t()
        self._check(self.lib.rsvd_workspace_bytes(self.h, dtype, m, n, k, p, q, job, C.byref(out)))
        return out.value

    def workspace(self, dtype, m, n, k, p):
        """A cached uint8 tensor large enough for the problem (grown on demand).  The cache is one buffer per
        context: calls that rely on it must stay on one stream (a call on another stream could still be using
        the buffer that a growing request replaces); pass `workspace=` to own the buffer yourself."""
        return self._grow(self.workspace_bytes(dtype, m, n, k, p))

    def _grow(self, need):
        if self._ws is None or self._ws.numel() < need:
            self._ws = None
            self._ws = self.torch.empty(need, dtype=self.torch.uint8, device=self.device)
        return self._ws

    def stage_workspace(self, dtype, rows, l):
        """Cached workspace for the stage calls on one rows x l panel (orth, small_svd, jacobi)."""
        out = C.c_size_t()
        self._check(self.lib.rsvd_stage_workspace_bytes(self.h, dtype, rows, l, C.byref(out)))
        return self._grow(out.value)

    def _empty(self, shape, like):
        return self.torch.empty(shape, dtype=like.dtype, device=self.device)

    # ---- Algorithm 1
    def rsvd_run_centered(self, A, k, p, q, seed=0, job=JOB_SUV, workspace=None, want_info=True, out=None):
        """PCA front end: decomposition of A minus its column means.  Returns (S, U, Vt, info, mean)."""
        mean = self._empty((A.shape[1],), A)
        S, U, Vt, info = self.rsvd_run(A, k, p, q, seed, job, workspace, want_info, out, _mean=mean)
        return S, U, Vt, info, mean

    def rsvd_run(self, A, k, p, q, seed=0, job=JOB_SUV, workspace=None, want_info=True, out=None, _mean=None):
        """Returns (S, U, Vt, info).  A: row-major (m, n) device tensor, stride(1) == 1."""
        assert A.is_cuda and A.dim() == 2 and A.stride(1) == 1
        m, n = A.shape
        dt = _dtype_code(A)
        ws = workspace if workspace is not None else self.workspace(dt, m, n, k, p)
        if out is None:
            S = self._empty((k,), A)
            U = self._empty((m, k), A) if job == JOB_SUV else None
            Vt = self._empty((k, n), A) if job >= JOB_SV else None
        else:
            S, U, Vt = out
        info = _Info()
        args = (self.h, self._stream(), dt, job, m, n, _ptr(A), A.stride(0), k, p, q, seed,
                _ptr(S), _ptr(U), U.stride(0) if U is not None else 0,
                _ptr(Vt), Vt.stride(0) if Vt is not None else 0,
                _ptr(ws), ws.numel(), C.byref(info) if want_info else None)
        if _mean is None:
            rc = self.lib.rsvd_run(*args)
        else:
            rc = self.lib.rsvd_run_centered(*args, _ptr(_mean))
        self._check(rc)
        return S, U, Vt, (info if want_info else None)

    def rsvd_run_static(self, A, k, p, q, seed=0, job=JOB_SUV, want_info=True, out=None):
        """rsvd_run on the library's own static scratch buffer (no workspace argument).  `out` = (S, U, Vt)
        tensors of the caller; without it they are allocated here, by torch, before the call."""
        assert A.is_cuda and A.dim() == 2 and A.stride(1) == 1
        m, n = A.shape
        dt = _dtype_code(A)
        if out is None:
            S = self._empty((k,), A)
            U = self._empty((m, k), A) if job == JOB_SUV else None
            Vt = self._empty((k, n), A) if job >= JOB_SV else None
        else:
            S, U, Vt = out
        info = _Info()
        self._check(self.lib.rsvd_run_static(
            self.h, self._stream(), dt, job, m, n, _ptr(A), A.stride(0), k, p, q, seed,
            _ptr(S), _ptr(U), U.stride(0) if U is not None else 0,
            _ptr(Vt), Vt.stride(0) if Vt is not None else 0, C.byref(info) if want_info else None))
        return S, U, Vt, (info if want_info else None)

    def rsvd_run_batched(self, A, k, p, q, seed=0, job=JOB_SUV, workspace=None, want_info=True, out=None):
        """A: (batch, m, n) device tensor, each matrix row-major.  Returns (S (batch, k), U (batch, m, k),
        Vt (batch, k, n), info of the whole batch).  Problem b uses seed + b."""
        assert A.is_cuda and A.dim() == 3 and A.stride(2) == 1
        batch, m, n = A.shape
        dt = _dtype_code(A)
        if workspace is None:
            need = C.c_size_t()
            self._check(self.lib.rsvd_workspace_bytes_batched(self.h, dt, batch, m, n, k, p, q, job, C.byref(need)))
            if self._ws is None or self._ws.numel() < need.value:
                self._ws = None
                self._ws = self.torch.empty(need.value, dtype=self.torch.uint8, device=self.device)
            workspace = self._ws
        if out is None:
            S = self._empty((batch, k), A)
            U = self._empty((batch, m, k), A) if job == JOB_SUV else None
            Vt = self._empty((batch, k, n), A) if job >= JOB_SV else None
        else:
            S, U, Vt = out
        info = _Info()
        self._check(self.lib.rsvd_run_batched(
            self.h, self._stream(), dt, job, batch, m, n, _ptr(A), A.stride(1), A.stride(0), k, p, q, seed,
            _ptr(S), S.stride(0), _ptr(U), U.stride(1) if U is not None else 0, U.stride(0) if U is not None else 0,
            _ptr(Vt), Vt.stride(1) if Vt is not None else 0, Vt.stride(0) if Vt is not None else 0,
            _ptr(workspace), workspace.numel(), C.byref(info) if want_info else None))
        return S, U, Vt, (info if want_info else None)

    # ---- stages
    def rsvd_stage_sketch(self, seed, rows, cols, dtype, stream_id=0, out=None):
        t = self.torch
        if out is None:
            out = t.empty((rows, cols), dtype=t.float32 if dtype == F32 else t.float64, device=self.device)
        self._check(self.lib.rsvd_stage_sketch(self.h, self._stream(), dtype, seed, stream_id, rows, cols,
                                               _ptr(out), out.stride(0) if rows > 0 and cols > 0 else cols))
        return out

    def rsvd_stage_philox_raw(self, seed, first_group, n_groups, stream_id=0):
        t = self.torch
        out = t.empty((n_groups, 4), dtype=t.int32, device=self.device)
        self._check(self.lib.rsvd_stage_philox_raw(self.h, self._stream(), seed, stream_id, first_group, n_groups,
                                                   _ptr(out)))
        return out

    def _stage_gemm(self, fn, A, X, out_rows):
        m, n = A.shape
        l = X.shape[1]
        dt = _dtype_code(A)
        ws = self.workspace(dt, m, n, l, 0)
        Y = self._empty((out_rows, l), A)
        self._check(fn(self.h, self._stream(), dt, m, n, l, _ptr(A), A.stride(0), _ptr(X), X.stride(0),
                       _ptr(Y), Y.stride(0), _ptr(ws), ws.numel()))
        return Y

    def rsvd_stage_gemm_an(self, A, X):
        return self._stage_gemm(self.lib.rsvd_stage_gemm_an, A, X, A.shape[0])

    def rsvd_stage_gemm_atn(self, A, X):
        return self._stage_gemm(self.lib.rsvd_stage_gemm_atn, A, X, A.shape[1])

    def rsvd_stage_orth(self, Y, seed=0, refill_stream=16, want_r=False):
        """In place on Y.  Returns (Y, R or None, info)."""
        rows, l = Y.shape
        dt = _dtype_code(Y)
        ws = self.stage_workspace(dt, rows, l)
        R = self.torch.empty((l, l), dtype=self.torch.float64, device=self.device) if want_r else None
        info = _Info()
        self._check(self.lib.rsvd_stage_orth(self.h, self._stream(), dt, rows, l, _ptr(Y), Y.stride(0), _ptr(R),
                                             seed, refill_stream, _ptr(ws), ws.numel(), C.byref(info)))
        return Y, R, info

    def rsvd_stage_small_svd(self, Bt, seed=0):
        """Bt (n, l) is overwritten.  Returns (sigma, Ub, V, info)."""
        n, l = Bt.shape
        dt = _dtype_code(Bt)
        ws = self.stage_workspace(dt, n, l)
        sigma = self._empty((l,), Bt)
        Ub = self._empty((l, l), Bt)
        V = self._empty((n, l), Bt)
        info = _Info()
        self._check(self.lib.rsvd_stage_small_svd(self.h, self._stream(), dt, n, l, _ptr(Bt), Bt.stride(0),
                                                  _ptr(sigma), _ptr(Ub), _ptr(V), V.stride(0), seed,
                                                  _ptr(ws), ws.numel(), C.byref(info)))
        return sigma, Ub, V, info

    def rsvd_stage_jacobi(self, M):
        """M (l, l) is overwritten.  Returns (sigma, X, W, info)."""
        l = M.shape[0]
        dt = _dtype_code(M)
        ws = self.stage_workspace(dt, l, l)
        sigma = self._empty((l,), M)
        X = self._empty((l, l), M)
        W = self._empty((l, l), M)
        info = _Info()
        self._check(self.lib.rsvd_stage_jacobi(self.h, self._stream(), dt, l, _ptr(M), _ptr(sigma), _ptr(X),
                                               _ptr(W), _ptr(ws), ws.numel(), C.byref(info)))
        return sigma, X, W, info

    def rsvd_stage_lift(self, Q, W, k, transpose_out=False):
        m, l = Q.shape
        dt = _dtype_code(Q)
        U = self._empty((k, m) if transpose_out else (m, k), Q)
        self._check(self.lib.rsvd_stage_lift(self.h, self._stream(), dt, m, l, k, _ptr(Q), Q.stride(0),
                                             _ptr(W), W.stride(0), _ptr(U), U.stride(0), int(transpose_out),
                                             None, 0))
        return U

    # ---- a linear layer held in 8 bits
    def _rows(self, t, cols, what, rows=None, dtype=None):
        """A matrix with `cols` columns (and `rows` rows of `dtype`) whose rows are contiguous, on the context's GPU."""
        if t.get_device() != self._index:
            self._elsewhere(t, what)
        if t.dim() != 2 or t.shape[1] != cols or (cols > 1 and t.stride(1) != 1) or t.stride(0) < 0:
            raise ValueError(f"{what}: a row-major GPU matrix with {cols} columns is needed")
        if (rows is not None and t.shape[0] != rows) or (dtype is not None and t.dtype != dtype):
            raise ValueError(f"{what}: {rows} rows of {dtype} are needed")
        return t.shape[0]

    def _elsewhere(self, t, what):
        raise ValueError(f"{what}: on {t.device}, not on the context's device ({self.device or 'none: it is for planning'})")

    def _given(self, workspace):
        if workspace.get_device() != self._index:
            self._elsewhere(workspace, "workspace")
        if not workspace.is_contiguous():
            raise ValueError("workspace: a contiguous tensor is needed")
        return workspace.data_ptr(), workspace.numel() * workspace.element_size()

    def rsvd_q8_rows(self, X):
        """Rows of X (bf16, fp16, fp32) to 8 bits.  Returns (codes int8, scale fp32), the codes laid out for Weight8."""
        self._rows(X, X.shape[1], "X")
        rows, n = X.shape
        codes = _empty_codes(rows, n, X.device)
        scale = self.torch.empty(rows, dtype=self.torch.float32, device=X.device)
        self._check(self.lib.rsvd_q8_rows(self.h, self._raw_stream(), _xtype_code(X.dtype), rows, n, _at(X), _ld(X), _at(codes),
                                          _ld(codes), _at(scale)))
        return codes, scale

    def _layer_ws(self, stream, name, sizes):
        """Address and bytes of the workspace that is kept for calls on `stream`; what a call of these sizes needs is asked for once.
        A call that is captured has a workspace of its graph's own: the kept one may be replaced, and used, while the graph lives."""
        need = self._needs.get((name, sizes))
        if need is None:
            out = C.c_size_t()
            self._check(getattr(self.lib, name)(self.h, *sizes, C.byref(out)))
            if len(self._needs) >= 1024:
                self._needs.clear()
            need = self._needs[(name, sizes)] = out.value
        if self.torch.cuda.is_current_stream_capturing():
            return self._room(need)
        kept = self._layer.get(stream)
        if kept is None or kept[1] < need:
            self._layer.pop(stream, None)
            kept = self._layer[stream] = self._room(need)
        return kept

    def _room(self, need):
        ws = self.torch.empty(need, dtype=self.torch.uint8, device=self.device)
        return ws.data_ptr(), need, ws

    def rsvd_q8_product(self, X, weight, workspace=None, out=None):
        """X (tokens x n) through the layer `weight` (Weight8): tokens x m, in the type of X."""
        w = weight
        n, m, r = sizes = w._sizes
        tokens, xt = self._rows(X, n, "X"), _xtype_code(X.dtype)
        if w._index != self._index:
            self._elsewhere(w, "weight")
        stream = self._raw_stream()
        ws = self._given(workspace) if workspace is not None else self._layer_ws(stream, "rsvd_q8_product_bytes", (xt, tokens, *sizes))
        Y = X.new_empty((tokens, m)) if out is None else out
        if out is not None:
            self._rows(out, m, "out", tokens, X.dtype)
        self._check(self.lib.rsvd_q8_product(self.h, stream, xt, tokens, n, m, r, X.data_ptr(), _ld(X),
                                             w.codes.data_ptr(), _ld(w.codes), w.scale.data_ptr(),
                                             _at(w.U), r, _at(w.Vt), n, _at(w.bias), Y.data_ptr(), _ld(Y), ws[0], ws[1]))
        return Y

    def rsvd_q8_product_grad(self, dY, weight, workspace=None, out=None):
        """Gradient of rsvd_q8_product with respect to X: dY (tokens x m) to tokens x n, in the type of dY."""
        w = weight
        n, m, r = sizes = w._sizes
        tokens, xt = self._rows(dY, m, "dY"), _xtype_code(dY.dtype)
        if w._index != self._index:
            self._elsewhere(w, "weight")
        stream = self._raw_stream()
        ws = self._given(workspace) if workspace is not None else self._layer_ws(stream, "rsvd_q8_product_grad_bytes", (xt, tokens, *sizes))
        Ut, V = w.Ut, w.V
        dX = dY.new_empty((tokens, n)) if out is None else out
        if out is not None:
            self._rows(out, n, "out", tokens, dY.dtype)
        self._check(self.lib.rsvd_q8_product_grad(self.h, stream, xt, tokens, n, m, r, dY.data_ptr(), _ld(dY),
                                                  w.codes.data_ptr(), _ld(w.codes), w.scale.data_ptr(),
                                                  _at(Ut), m, _at(V), r, dX.data_ptr(), _ld(dX), ws[0], ws[1]))
        return dX

    def rsvd_keep8_save(self, X):
        """X (tokens x n) kept in 8 bits for the backward pass (Kept8)."""
        tokens, n = self._rows(X, X.shape[-1], "X"), X.shape[1]
        codes = _empty_codes(tokens, n, X.device)
        powers = X.new_empty((tokens, -(-n // 32)), dtype=self.torch.uint8)
        self._check(self.lib.rsvd_keep8_save(self.h, self._raw_stream(), _xtype_code(X.dtype), tokens, n, X.data_ptr(), _ld(X),
                                             codes.data_ptr(), codes.stride(0), powers.data_ptr(), -(-n // 32)))
        return Kept8.__new__(Kept8)._set(codes, powers, X.dtype)

    def rsvd_keep8_load(self, kept, out=None):
        """The kept activations, in their type."""
        if kept._index != self._index:
            self._elsewhere(kept, "kept")
        tokens, n, codes, powers = kept.tokens, kept.n, kept.codes, kept.powers
        X = codes.new_empty((tokens, n), dtype=kept.dtype) if out is None else out
        if out is not None:
            self._rows(out, n, "out", tokens, kept.dtype)
        self._check(self.lib.rsvd_keep8_load(self.h, self._raw_stream(), _xtype_code(kept.dtype), tokens, n,
                                             codes.data_ptr(), _ld(codes), powers.data_ptr(), _ld(powers), X.data_ptr(), _ld(X)))
        return X

    def rsvd_keep8_grad(self, dY, kept, out=None, accumulate=False, workspace=None):
        """Gradients of a weight and a bias from dY (tokens x m) and the kept activations: (dW (m x n), db (m)), fp32.
        `out` = (dW, db) of the caller, db may be None; accumulate: they are added to."""
        if dY.shape[0] != kept.tokens:
            raise ValueError("dY: one row for each kept token")
        self._rows(dY, dY.shape[1], "dY")
        if kept._index != self._index:
            self._elsewhere(kept, "kept")
        if accumulate and out is None:
            raise ValueError("accumulate: into which gradients?")
        xt, m = _xtype_code(dY.dtype), dY.shape[1]
        t = self.torch
        if out is None:
            dW = t.empty((m, kept.n), dtype=t.float32, device=dY.device)
            db = t.empty(m, dtype=t.float32, device=dY.device)
        else:
            dW, db = out
            self._rows(dW, kept.n, "dW")
            if dW.dtype != t.float32 or dW.shape[0] != m or (db is not None and (db.dtype != t.float32 or db.shape != (m,) or not db.is_contiguous())):
                raise ValueError("out: fp32 gradients, m x n and m")
            if db is not None and db.get_device() != self._index:
                self._elsewhere(db, "db")
        stream = self._raw_stream()
        ws = self._given(workspace) if workspace is not None else self._layer_ws(stream, "rsvd_keep8_grad_bytes", (xt, kept.tokens, kept.n, m))
        self._check(self.lib.rsvd_keep8_grad(
            self.h, stream, xt, kept.tokens, kept.n, m, _at(dY), _ld(dY), _at(kept.codes), _ld(kept.codes),
            _at(kept.powers), _ld(kept.powers), _at(dW), _ld(dW), _at(db), int(accumulate), ws[0], ws[1]))
        return dW, db
