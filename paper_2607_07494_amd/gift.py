"""Thin ctypes binding of ``libgift.so`` (the C ABI in ``include/gift.h``).

Argument marshalling only: every computation runs in the library's HIP
kernels.  Tensors are torch tensors on the GPU (device memory and streams are
all torch is used for); the wrappers check every tensor's shape against the
sizes the call is given (the library sizes its loops and buffer ranges from
those sizes, so a short tensor would be read or written out of bounds), then
dtype, device and contiguity, pass ``data_ptr()`` and raise
:class:`GiftError` with the library's message when a call fails.  A shape
mismatch raises ``ValueError`` before anything is enqueued.  There is no
fallback: if ``libgift.so`` is missing, importing this module raises.
"""

from __future__ import annotations

import array
import ctypes
import operator
import os
import weakref

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libgift.so")

OK, EINVAL, ESHAPE, ENOMEM, EHIP, EUNSUPPORTED = 0, -1, -2, -3, -4, -5
F32, BF16 = 0, 1
SIDE_INPUT, SIDE_OUTPUT, SIDE_BOTH = 1, 2, 3
SCALE_LOCAL, SCALE_SHARED = 0, 1
KERNELS = {
    "amax": 0, "quant": 1, "project": 2, "update_amax": 3, "update_quant": 4,
    "update_store": 5, "reduce": 6, "syrk": 7, "factor": 8, "small": 9,
    "chol": 10, "eig": 11, "decode_project": 12, "chol_transform": 13, "mxfp4": 14,
    "embed": 15, "embed_grad": 16, "norm": 17, "optimizer": 18,
}
I32, I64 = 0, 1
_DTYPE, _SHAPE, _NBYTES = (operator.attrgetter(name) for name in ("dtype", "shape", "nbytes"))
MOMENTS = {"f32": 0, "e4m3": 1}

_STATUS = {OK: "GIFT_OK", EINVAL: "GIFT_EINVAL", ESHAPE: "GIFT_ESHAPE", ENOMEM: "GIFT_ENOMEM",
           EHIP: "GIFT_EHIP", EUNSUPPORTED: "GIFT_EUNSUPPORTED"}


class GiftError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


class _AdamWTensor(ctypes.Structure):
    """``gift_adamw_tensor``."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("copy", ctypes.c_void_p), ("numel", ctypes.c_int64), ("weight_decay", ctypes.c_double)]


class _AdamWOptions(ctypes.Structure):
    """``gift_adamw_options``."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("grad_dtype", ctypes.c_int32), ("moments", ctypes.c_int32), ("lr_dev", ctypes.c_void_p),
                ("step_dev", ctypes.c_void_p), ("grad_scale", ctypes.c_void_p)]


def _load():
    # torch first: its bundled HIP runtime then satisfies libgift.so's
    # libamdhip64 dependency by soname.  Loaded the other way round, the
    # process holds two HIP runtimes and the second one sees no device.
    import torch  # noqa: F401

    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2607_07494_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, U64, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
    PP = ctypes.POINTER(ctypes.c_void_p)
    sigs = {
        "gift_abi_version": ([], I32),
        "gift_last_error": ([], ctypes.c_char_p),
        "gift_ctx_create": ([P, PP], I32),
        "gift_ctx_set_stream": ([P, P], I32),
        "gift_ctx_destroy": ([P], None),
        "gift_ctx_set_statistics_event": ([P, P], I32),
        "gift_ctx_profile_enable": ([P, I32], I32),
        "gift_ctx_profile_select": ([P, ctypes.c_uint32], I32),
        "gift_ctx_profile_read": ([P, I32, ctypes.POINTER(I64), ctypes.POINTER(ctypes.c_double)], I32),
        "gift_ctx_profile_reset": ([P], I32),
        "gift_factor_create": ([P, I64, I64, I32, I32, F, U64, PP], I32),
        "gift_factor_destroy": ([P], None),
        "gift_factor_update": ([P, P, P, P, I64, I32, I32], I32),
        "gift_statistics": ([P, P, I64, I64, I32, P], I32),
        "gift_factor_update_batch": ([P, I32, P, P, P, I64, I32, I32], I32),
        "gift_factor_export": ([P, P, I32, P, P, P, P], I32),
        "gift_factor_import": ([P, P, I32, P, P, P, P], I32),
        "gift_factor_create_chol": ([P, I64, I64, I32, I32, F, PP], I32),
        "gift_factor_export_chol": ([P, P, I32, P, P], I32),
        "gift_factor_import_chol": ([P, P, I32, P, P], I32),
        "gift_encode": ([P, P, P, I32, I64, I64, I32, I32, I32, P, P, P, P], I32),
        "gift_encode_hits": ([P, P, P, I32, I64, I64, I32, I32, I32, P, P, P, P, P], I32),
        "gift_encode_noalloc": ([P, P, P, I32, I64, I64, I32, I32, I32, P, P, P, P], I32),
        "gift_reduce_local": ([P, P, P, I32, I64, I64, I32, I32, P], I32),
        "gift_encode_mxfp4": ([P, P, P, I32, I64, I64, P, P, P, P], I32),
        "gift_reduce_local_mxfp4": ([P, P, P, I32, I64, I64, P], I32),
        "gift_decode": ([P, P, P, I64, I64, P], I32),
        "gift_decode_batch": ([P, I32, P, P, P, I64, I64], I32),
        "gift_embedding": ([P, P, I32, I64, I64, P, I32, I64, F, P, I32], I32),
        "gift_embedding_grad_scratch": ([I32, I64, I64, I64], U64),
        "gift_embedding_grad": ([P, P, I32, P, I32, I32, I64, I64, I64, F, I32, P, P, U64], I32),
        "gift_grad_norm": ([P, I32, P, P, I32, ctypes.c_double, P, P, U64], I32),
        "gift_adamw_step": ([P, I32, ctypes.POINTER(_AdamWTensor), ctypes.POINTER(_AdamWOptions)], I32),
    }
    for name, (args, res) in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


LIB = _load()


def _check(status: int):
    if status != OK:
        raise GiftError(status, LIB.gift_last_error().decode(errors="replace"))


def exported_symbols():
    """Names declared by include/gift.h that this binding calls."""
    return sorted(n for n in dir(LIB) if n.startswith("gift_"))


def _ptr(t, dtype=None, name="tensor"):
    if t is None:
        return None
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, not {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _expect(t, shape, name):
    """Raise ValueError unless tensor ``t`` (may be None) has exactly ``shape``."""
    if t is None:
        return
    got = tuple(getattr(t, "shape", ()))
    if got != tuple(int(d) for d in shape):
        raise ValueError(f"{name} must have shape {tuple(int(d) for d in shape)}, not {got}")


def _dims(t, k, name):
    """The shape of ``t``, which must be a ``k``-dimensional tensor."""
    shape = tuple(getattr(t, "shape", ()))
    if len(shape) != k:
        raise ValueError(f"{name} must be {k}-dimensional, not of shape {shape}")
    return shape


def scale_grid(m: int, n: int, block_rows: int = 0, block_cols: int = 0):
    """``(nbr, nbc)``: scale-grid shape for allocating the scales output."""
    br = m if block_rows <= 0 else min(block_rows, m)
    bc = n if block_cols <= 0 else min(block_cols, n)
    return -(-m // br), -(-n // bc)


class Context:
    """A library context bound to one HIP stream (default: torch's current)."""

    def __init__(self, stream=None):
        if stream is None:
            import torch
            stream = torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
        self._h = ctypes.c_void_p()
        self._factors = weakref.WeakSet()
        self._stream = int(stream)
        _check(LIB.gift_ctx_create(ctypes.c_void_p(int(stream)), ctypes.byref(self._h)))

    @property
    def handle(self):
        return self._h

    def set_stream(self, stream):
        _check(LIB.gift_ctx_set_stream(self._h, ctypes.c_void_p(int(stream))))
        self._stream = int(stream)

    def set_statistics_event(self, event):
        """Record ``event`` (a torch.cuda.Event, or None) after the statistics
        kernels of every later factor refresh on this context.  The context
        keeps a reference to the event so that it outlives the registration."""
        h = None
        self._stats_event = event
        if event is not None:
            import torch  # noqa: F401
            event.record()          # creates the underlying HIP event
            h = ctypes.c_void_p(event.cuda_event)
        _check(LIB.gift_ctx_set_statistics_event(self._h, h))

    def profile(self, enable: bool = True):
        _check(LIB.gift_ctx_profile_enable(self._h, 1 if enable else 0))

    def profile_select(self, families=None):
        """Time only these kernel families (names or ids; None = all)."""
        if families is None:
            mask = 0xFFFFFFFF
        else:
            mask = 0
            for k in families:
                mask |= 1 << (KERNELS[k] if isinstance(k, str) else int(k))
        _check(LIB.gift_ctx_profile_select(self._h, mask))

    def profile_read(self, kernel):
        k = KERNELS[kernel] if isinstance(kernel, str) else int(kernel)
        n = ctypes.c_int64()
        ms = ctypes.c_double()
        _check(LIB.gift_ctx_profile_read(self._h, k, ctypes.byref(n), ctypes.byref(ms)))
        return n.value, ms.value

    def profile_reset(self):
        _check(LIB.gift_ctx_profile_reset(self._h))

    def close(self):
        """Destroy the context; factors created on it are destroyed first."""
        if self._h:
            for f in list(self._factors):
                f.close()
            LIB.gift_ctx_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Factor:
    """Transform state of one m x n weight matrix (``gift_factor``)."""

    def __init__(self, ctx: Context, m: int, n: int, rank: int, sides: int = SIDE_INPUT,
                 damping: float = 1e-6, seed: int = 0):
        self.ctx, self.m, self.n, self.rank, self.sides = ctx, m, n, rank, sides
        self._h = ctypes.c_void_p()
        if not ctx.handle:
            raise GiftError(EINVAL, "the context is closed")
        _check(LIB.gift_factor_create(ctx.handle, m, n, rank, sides, damping, seed,
                                      ctypes.byref(self._h)))
        ctx._factors.add(self)

    @property
    def handle(self):
        return self._h

    def update(self, acts=None, out_grads=None, iters: int = 4):
        import torch
        x = acts if acts is not None else out_grads
        if x is None:
            raise ValueError("update needs acts and/or out_grads")
        if x.dtype == torch.float32:
            dt = F32
        elif x.dtype == torch.bfloat16:
            dt = BF16
        else:
            raise TypeError("statistics inputs must be float32 or bfloat16")
        T = x.shape[0]
        for t, nm in ((acts, "acts"), (out_grads, "out_grads")):
            if t is not None and (t.dim() != 2 or t.shape[0] != T or t.dtype != x.dtype):
                raise ValueError(f"{nm} must be [T, dim] with the common T and dtype")
        _check_stats_inputs(self, acts, out_grads, T)
        _check(LIB.gift_factor_update(self.ctx.handle, self._h, _ptr(acts, None, "acts"),
                                      _ptr(out_grads, None, "out_grads"), T, dt, iters))

    def export(self, side: int):
        import torch
        dim = self.n if side == SIDE_INPUT else self.m
        dev = torch.device("cuda", torch.cuda.current_device())
        U = torch.empty((dim, self.rank), dtype=torch.float32, device=dev)
        cf = torch.empty(self.rank, dtype=torch.float32, device=dev)
        ci = torch.empty(self.rank, dtype=torch.float32, device=dev)
        s2 = torch.empty(1, dtype=torch.float32, device=dev)
        _check(LIB.gift_factor_export(self.ctx.handle, self._h, side, _ptr(U), _ptr(cf), _ptr(ci),
                                      _ptr(s2)))
        return U, cf, ci, s2

    def import_(self, side: int, U, c_fwd, c_inv, sigma2):
        import torch
        f = torch.float32
        if side not in (SIDE_INPUT, SIDE_OUTPUT):
            raise ValueError("side must be SIDE_INPUT or SIDE_OUTPUT")
        dim = self.n if side == SIDE_INPUT else self.m
        _expect(U, (dim, self.rank), "U")
        _expect(c_fwd, (self.rank,), "c_fwd")
        _expect(c_inv, (self.rank,), "c_inv")
        _expect(sigma2, (1,), "sigma2")
        _check(LIB.gift_factor_import(self.ctx.handle, self._h, side, _ptr(U, f, "U"),
                                      _ptr(c_fwd, f, "c_fwd"), _ptr(c_inv, f, "c_inv"),
                                      _ptr(sigma2, f, "sigma2")))

    def close(self):
        if self._h:
            LIB.gift_factor_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class CholFactor(Factor):
    """Cholesky-form factor (``gift_factor_create_chol``): block 0 = full
    factor, 1 = diagonal, b = b x b diagonal blocks of A + delta I."""

    def __init__(self, ctx: Context, m: int, n: int, block: int = 0, sides: int = SIDE_INPUT,
                 damping: float = 1e-6):
        self.ctx, self.m, self.n, self.block, self.sides = ctx, m, n, block, sides
        self.rank = 0
        self._h = ctypes.c_void_p()
        if not ctx.handle:
            raise GiftError(EINVAL, "the context is closed")
        _check(LIB.gift_factor_create_chol(ctx.handle, m, n, block, sides, damping,
                                           ctypes.byref(self._h)))
        ctx._factors.add(self)

    def block_shape(self, side: int):
        """``(nblk, b_eff)`` of one side's stored blocks."""
        dim = self.n if side == SIDE_INPUT else self.m
        b = dim if self.block <= 0 or self.block >= dim else self.block
        return -(-dim // b), b

    def export(self, side: int):
        import torch
        nblk, b = self.block_shape(side)
        dev = torch.device("cuda", torch.cuda.current_device())
        R = torch.empty((nblk, b, b), dtype=torch.float32, device=dev)
        Ri = torch.empty((nblk, b, b), dtype=torch.float32, device=dev)
        _check(LIB.gift_factor_export_chol(self.ctx.handle, self._h, side, _ptr(R), _ptr(Ri)))
        return R, Ri

    def import_(self, side: int, R, Rinv):
        import torch
        nblk, b = self.block_shape(side)
        for t, nm in ((R, "R"), (Rinv, "Rinv")):
            if tuple(t.shape) != (nblk, b, b):
                raise ValueError(f"{nm} must have shape {(nblk, b, b)}")
        _check(LIB.gift_factor_import_chol(self.ctx.handle, self._h, side,
                                           _ptr(R, torch.float32, "R"),
                                           _ptr(Rinv, torch.float32, "Rinv")))


def _stats_dtype(x):
    import torch
    if x.dtype == torch.float32:
        return F32
    if x.dtype == torch.bfloat16:
        return BF16
    raise TypeError("statistics inputs must be float32 or bfloat16")


def _check_stats_inputs(factor, acts, out_grads, T):
    """acts [T, n] for a factor with the input side, out_grads [T, m] for one
    with the output side (the refresh reads T x dim values of each)."""
    sides = getattr(factor, "sides", 0)
    if sides & SIDE_INPUT:
        if acts is None:
            raise ValueError("acts is required for a factor with the input side")
        _expect(acts, (T, factor.n), "acts")
    if sides & SIDE_OUTPUT:
        if out_grads is None:
            raise ValueError("out_grads is required for a factor with the output side")
        _expect(out_grads, (T, factor.m), "out_grads")


def factor_update_batch(ctx: Context, factors, acts=None, out_grads=None, iters: int = 4):
    """``gift_factor_update_batch``: refresh many factors in one launch sequence.

    ``acts`` / ``out_grads`` are lists (one entry per factor, ``None`` where a
    factor lacks that side) of [T, dim] tensors with a common T and dtype.
    """
    count = len(factors)
    if count == 0:
        return
    acts = list(acts) if acts is not None else [None] * count
    out_grads = list(out_grads) if out_grads is not None else [None] * count
    if len(acts) != count or len(out_grads) != count:
        raise ValueError("acts / out_grads must have one entry per factor")
    tensors = [x for x in acts + out_grads if x is not None]
    if not tensors:
        raise ValueError("factor_update_batch needs statistics inputs")
    T, dt = tensors[0].shape[0], _stats_dtype(tensors[0])
    for x in tensors:
        if x.dim() != 2 or x.shape[0] != T or _stats_dtype(x) != dt:
            raise ValueError("statistics inputs must be [T, dim] with a common T and dtype")
    for f, a, g in zip(factors, acts, out_grads):
        _check_stats_inputs(f, a, g, T)
    arr = ctypes.c_void_p * count
    fa = arr(*[f.handle.value for f in factors])
    aa = arr(*[(_ptr(x).value if x is not None else None) for x in acts])
    ga = arr(*[(_ptr(x).value if x is not None else None) for x in out_grads])
    _check(LIB.gift_factor_update_batch(ctx.handle, count, fa, aa, ga, T, dt, iters))


def statistics(ctx: Context, x, A):
    """``gift_statistics``: x [T, dim] (float32 or bfloat16) -> A [dim, dim] = x^T x / T."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must be [T, dim]")
    T, dim = x.shape
    if tuple(A.shape) != (dim, dim):
        raise ValueError("A must be [dim, dim]")
    _check(LIB.gift_statistics(ctx.handle, _ptr(x, None, "x"), T, dim, _stats_dtype(x),
                               _ptr(A, torch.float32, "A")))


def encode(ctx: Context, factor, grads, codes, scales, block_rows: int = 0, block_cols: int = 0,
           mode: int = SCALE_LOCAL, ef=None, transformed=None, hits=None):
    """``gift_encode``: grads [N, m, n] f32 -> codes [N, m, n] u8, scales [N, nbr, nbc] f32.

    With ``hits`` (an int32 [N, 2] tensor, bit pattern of the uint32 counters)
    this is ``gift_encode_hits``: the per-rank upper / lower boundary hits are
    added to it.
    """
    import torch
    N, m, n = _dims(grads, 3, "grads")
    if factor is not None and (factor.m, factor.n) != (m, n):
        raise ValueError(f"the factor was created for {factor.m} x {factor.n}, not {m} x {n}")
    _expect(codes, (N, m, n), "codes")
    _expect(scales, (N,) + scale_grid(m, n, block_rows, block_cols), "scales")
    _expect(ef, (N, m, n), "ef")
    _expect(transformed, (N, m, n), "transformed")
    _expect(hits, (N, 2), "hits")
    args = [ctx.handle, factor.handle if factor is not None else None,
            _ptr(grads, torch.float32, "grads"), N, m, n, block_rows, block_cols,
            mode, _ptr(ef, torch.float32, "ef"), _ptr(codes, torch.uint8, "codes"),
            _ptr(scales, torch.float32, "scales"), _ptr(transformed, torch.float32, "transformed")]
    if hits is None:
        _check(LIB.gift_encode(*args))
        return
    _check(LIB.gift_encode_hits(*args, _ptr(hits, torch.int32, "hits")))


NOALLOC_SCRATCH_BYTES = 64 * 1024 * 1024


def encode_noalloc(ctx: Context, factor, grads, codes, scales, block_rows: int = 0, block_cols: int = 0,
                   mode: int = SCALE_LOCAL, ef=None, transformed=None):
    """``gift_encode_noalloc``: :func:`encode` with its scratch in the library's
    fixed per-device array (no device allocation; calls on one device must
    not overlap)."""
    import torch
    N, m, n = _dims(grads, 3, "grads")
    if factor is not None and (factor.m, factor.n) != (m, n):
        raise ValueError(f"the factor was created for {factor.m} x {factor.n}, not {m} x {n}")
    _expect(codes, (N, m, n), "codes")
    _expect(scales, (N,) + scale_grid(m, n, block_rows, block_cols), "scales")
    _expect(ef, (N, m, n), "ef")
    _expect(transformed, (N, m, n), "transformed")
    _check(LIB.gift_encode_noalloc(ctx.handle, factor.handle if factor is not None else None,
                                   _ptr(grads, torch.float32, "grads"), N, m, n, block_rows, block_cols,
                                   mode, _ptr(ef, torch.float32, "ef"), _ptr(codes, torch.uint8, "codes"),
                                   _ptr(scales, torch.float32, "scales"),
                                   _ptr(transformed, torch.float32, "transformed")))


def reduce_local(ctx: Context, codes, scales, mean, block_rows: int = 0, block_cols: int = 0):
    """``gift_reduce_local``: codes [N, m, n], scales -> mean [m, n] f32."""
    import torch
    N, m, n = _dims(codes, 3, "codes")
    _expect(scales, (N,) + scale_grid(m, n, block_rows, block_cols), "scales")
    _expect(mean, (m, n), "mean")
    _check(LIB.gift_reduce_local(ctx.handle, _ptr(codes, torch.uint8, "codes"),
                                 _ptr(scales, torch.float32, "scales"), N, m, n, block_rows,
                                 block_cols, _ptr(mean, torch.float32, "mean")))


def encode_mxfp4(ctx: Context, factor, grads, codes, scales, ef=None, transformed=None):
    """``gift_encode_mxfp4``: grads [N, m, n] f32 -> codes [N, m, n/2] u8 (packed
    E2M1), scales [N, m, n/32] u8 (E8M0)."""
    import torch
    N, m, n = _dims(grads, 3, "grads")
    if factor is not None and (factor.m, factor.n) != (m, n):
        raise ValueError(f"the factor was created for {factor.m} x {factor.n}, not {m} x {n}")
    if n % 32:
        raise ValueError("MXFP4 needs n to be a multiple of 32")
    _expect(codes, (N, m, n // 2), "codes")
    _expect(scales, (N, m, n // 32), "scales")
    _expect(ef, (N, m, n), "ef")
    _expect(transformed, (N, m, n), "transformed")
    _check(LIB.gift_encode_mxfp4(ctx.handle, factor.handle if factor is not None else None,
                                 _ptr(grads, torch.float32, "grads"), N, m, n, _ptr(ef, torch.float32, "ef"),
                                 _ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.uint8, "scales"),
                                 _ptr(transformed, torch.float32, "transformed")))


def reduce_local_mxfp4(ctx: Context, codes, scales, mean):
    """``gift_reduce_local_mxfp4``: codes [N, m, n/2], scales [N, m, n/32] -> mean [m, n] f32."""
    import torch
    N, m, half = _dims(codes, 3, "codes")
    if (2 * half) % 32:
        raise ValueError("MXFP4 needs n = 2 * codes.shape[2] to be a multiple of 32")
    _expect(scales, (N, m, 2 * half // 32), "scales")
    _expect(mean, (m, 2 * half), "mean")
    _check(LIB.gift_reduce_local_mxfp4(ctx.handle, _ptr(codes, torch.uint8, "codes"),
                                       _ptr(scales, torch.uint8, "scales"), N, m, 2 * half,
                                       _ptr(mean, torch.float32, "mean")))


def decode(ctx: Context, factor, mean, out):
    """``gift_decode``: inverse transform of the rank mean [m, n] f32 into out."""
    import torch
    m, n = _dims(mean, 2, "mean")
    if factor is not None and (factor.m, factor.n) != (m, n):
        raise ValueError(f"the factor was created for {factor.m} x {factor.n}, not {m} x {n}")
    _expect(out, (m, n), "out")
    _check(LIB.gift_decode(ctx.handle, factor.handle if factor is not None else None,
                           _ptr(mean, torch.float32, "mean"), m, n, _ptr(out, torch.float32, "out")))


def decode_batch(ctx: Context, factors, means, outs):
    """``gift_decode_batch``: ``outs[i] = decode(factors[i], means[i])`` for
    matrices of one shape, one launch per pass when the factors allow."""
    import torch
    count = len(means)
    if len(factors) != count or len(outs) != count:
        raise ValueError("factors, means and outs must have one entry per matrix")
    if count == 0:
        return
    m, n = _dims(means[0], 2, "means[0]")
    for i in range(count):
        _expect(means[i], (m, n), f"means[{i}]")
        _expect(outs[i], (m, n), f"outs[{i}]")
        f = factors[i]
        if f is not None and (f.m, f.n) != (m, n):
            raise ValueError(f"factor {i} was created for {f.m} x {f.n}, not {m} x {n}")
    arr = ctypes.c_void_p * count
    fa = arr(*[(f.handle.value if f is not None else None) for f in factors])
    ma = arr(*[_ptr(t, torch.float32, "means").value for t in means])
    oa = arr(*[_ptr(t, torch.float32, "outs").value for t in outs])
    _check(LIB.gift_decode_batch(ctx.handle, count, fa, ma, oa, m, n))


# ---------------------------------------------------------------------------
# The training step around the codec
# ---------------------------------------------------------------------------
# (small calls take less time on the GPU than in Python: torch is a module
# global here, it was imported before the library)
import torch  # noqa: E402

_VALUES = {torch.float32: F32, torch.bfloat16: BF16}
_INDICES = {torch.int32: I32, torch.int64: I64}


def _value_dtype(t, name):
    dt = _VALUES.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return dt


def _index_type(t, name):
    it = _INDICES.get(t.dtype)
    if it is None:
        raise TypeError(f"{name} must be int32 or int64, not {t.dtype}")
    return it


def _on_current_device(**tensors):
    """Raise ValueError unless every tensor is contiguous and on the current device."""
    dev = None
    for name, t in tensors.items():
        at = t.get_device()
        if at < 0:
            raise ValueError(f"{name} must be a GPU tensor")
        if dev is None:
            dev = torch.cuda.current_device()
        if at != dev:
            raise ValueError(f"{name} is on {t.device}, not on the current device")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _scratch(t):
    """``(pointer, bytes)`` of a scratch tensor, or of none."""
    if t is None:
        return None, 0
    _on_current_device(scratch=t)
    return t.data_ptr(), t.numel() * t.element_size()


def embedding(ctx: Context, table, tokens, out, scale: float = 1.0):
    """``gift_embedding``: ``out[...] = scale * table[tokens[...]]``; table [V, d] and out
    [*tokens.shape, d] float32 or bfloat16, tokens int32 or int64 (ids outside [0, V): zeros)."""
    V, d = _dims(table, 2, "table")
    if out.shape != tokens.shape + (d,):
        _expect(out, tuple(tokens.shape) + (d,), "out")
    td, it, od = _value_dtype(table, "table"), _index_type(tokens, "tokens"), _value_dtype(out, "out")
    _on_current_device(table=table, tokens=tokens, out=out)
    _check(LIB.gift_embedding(ctx._h, table.data_ptr(), td, V, d, tokens.data_ptr(), it, tokens.numel(), scale,
                              out.data_ptr(), od))


def _int32(n):
    """n, or the largest int32 in place of a larger number (ctypes takes it modulo 2^32); the library refuses it."""
    return min(n, 2 ** 31 - 1)


def embedding_grad_scratch(N: int, T: int, V: int, d: int) -> int:
    """Scratch bytes of :func:`embedding_grad` (``gift_embedding_grad_scratch``)."""
    return LIB.gift_embedding_grad_scratch(_int32(N), T, V, d)


def embedding_grad(ctx: Context, tokens, dout, grads, scale: float = 1.0, accumulate: bool = False, scratch=None):
    """``gift_embedding_grad``: tokens [N, T], dout [N, T, d] (float32 or bfloat16) ->
    grads [N, V, d] float32, each rank's gradient of the lookup; with ``accumulate``
    added to what grads holds.  ``scratch``: a tensor of at least
    :func:`embedding_grad_scratch` bytes (needed under graph capture), else the
    context's workspace."""
    N, V, d = _dims(grads, 3, "grads")
    T = _dims(tokens, 2, "tokens")[1]
    _expect(tokens, (N, T), "tokens")
    _expect(dout, (N, T, d), "dout")
    it, dt = _index_type(tokens, "tokens"), _value_dtype(dout, "dout")
    if grads.dtype != torch.float32:
        raise TypeError(f"grads must have dtype torch.float32, not {grads.dtype}")
    _on_current_device(tokens=tokens, dout=dout, grads=grads)
    ws, ws_bytes = _scratch(scratch)
    _check(LIB.gift_embedding_grad(ctx._h, tokens.data_ptr(), it, dout.data_ptr(), dt, _int32(N), T, V, d, scale,
                                   1 if accumulate else 0, grads.data_ptr(), ws, ws_bytes))


GRAD_NORM_SCRATCH_BYTES = 16384


def _all_on_current_device(tensors, name):
    """Raise ValueError unless every tensor of a list is contiguous and on the current device.

    Loops of C functions: a model has hundreds of tensors, and a step's kernels
    take less time than hundreds of passes through Python."""
    devices = set(map(torch.Tensor.get_device, tensors))
    if devices and min(devices) < 0:
        raise ValueError(f"{name} must be GPU tensors")
    if devices and devices != {torch.cuda.current_device()}:
        raise ValueError(f"{name} must be on the current device, not on {devices}")
    if not all(map(torch.Tensor.is_contiguous, tensors)):
        raise ValueError(f"{name} must be contiguous")


def _gradient_list(grads):
    """``(dtype, data pointers)`` of a list of gradients on the current device, of one dtype."""
    dt = _value_dtype(grads[0], "gradients")
    if len(set(map(_DTYPE, grads))) > 1:
        raise TypeError(f"gradients must have one dtype: {set(map(_DTYPE, grads))}")
    _all_on_current_device(grads, "gradients")
    return dt, array.array("Q", map(torch.Tensor.data_ptr, grads))


def grad_norm(ctx: Context, grads, out, max_norm: float = float("inf"), scratch=None):
    """``gift_grad_norm``: out [2] float32 = the norm over all tensors of the list ``grads``
    (all float32 or all bfloat16) and the coefficient that clips it to ``max_norm``
    (NaN when the norm is not finite).  ``scratch``: a tensor of at least
    ``GRAD_NORM_SCRATCH_BYTES`` bytes (needed under graph capture), else the
    context's workspace."""
    grads = list(grads)
    _expect(out, (2,), "out")
    if out.dtype != torch.float32:
        raise TypeError(f"out must have dtype torch.float32, not {out.dtype}")
    _on_current_device(out=out)
    count = len(grads)
    dt, ptrs = _gradient_list(grads) if count else (F32, array.array("Q"))
    sizes = array.array("q", map(torch.Tensor.numel, grads))
    ws, ws_bytes = _scratch(scratch)
    _check(LIB.gift_grad_norm(ctx._h, count, ptrs.buffer_info()[0], sizes.buffer_info()[0], dt, max_norm,
                              out.data_ptr(), ws, ws_bytes))


def _scalar(x, dtype, name):
    """Address of a tensor of one element on the current device, else None."""
    if not isinstance(x, torch.Tensor):
        return None
    if x.dtype != dtype or x.numel() != 1:
        raise TypeError(f"{name} must be one {dtype} element")
    _on_current_device(**{name: x})
    return x.data_ptr()


class AdamW:
    """AdamW over a list of float32 tensors (``gift_adamw_step``).

    ``moments``: ``"f32"``, or ``"e4m3"`` for FP8 E4M3 codes with a float32 scale
    per 256 consecutive elements.  ``weight_decay``: one value, or one for each
    tensor.  ``copies``: bfloat16 tensors of the parameters' shapes that every
    step rewrites (entries may be ``None``).  ``state``: the moments, flat
    tensors used in place (:meth:`state_sizes`); made as zeros when not given.
    Tensor i's elements lie in ``m`` and ``v`` from ``starts[i]`` on (a multiple of
    512), its scales in ``m_scales`` and ``v_scales`` from ``starts[i] // 256``.

    ``params``, ``copies`` and ``state`` may change between steps: a step works on the
    tensors that they hold, where those lie, at the time of the call (after
    ``param.data = other`` or ``state["m"] = loaded`` on the other memory).  Shapes
    and dtypes must stay.  ``betas``, ``eps`` and ``seed`` may be set between steps too.
    A captured step keeps what it was captured with.
    """

    ALIGN, BLOCK = 512, 256

    def __init__(self, ctx: Context, params, betas=(0.9, 0.95), eps: float = 1e-8, weight_decay=0.0,
                 moments: str = "f32", seed: int = 0, state=None, copies=None):
        if moments not in MOMENTS:
            raise ValueError(f"moments must be one of {sorted(MOMENTS)}, not {moments!r}")
        self._options = _AdamWOptions(moments=MOMENTS[moments])
        self._moments, self.betas, self.eps, self.seed = moments, betas, eps, seed
        self.ctx, self.params, self.steps = ctx, list(params), 0
        self._own = []          # moments made here
        count = len(self.params)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * count
        self.copies = list(copies) if copies is not None else [None] * count
        if len(decay) != count or len(self.copies) != count:
            raise ValueError("weight_decay and copies must have one entry per parameter")
        self._shapes = list(map(_SHAPE, self.params))
        self.starts, total = self._starts(self.params)
        self._sizes = self._state_of(total, moments)
        self._tensors = (_AdamWTensor * count)()
        # the tensors' fields, as 64-bit words
        self._words = memoryview(self._tensors).cast("B").cast("Q") if count else memoryview(array.array("Q"))
        self._check_tensors(state)
        if state is None:
            dev = torch.device("cuda", torch.cuda.current_device()) if count else torch.device("cpu")
            state = {name: torch.zeros(n, dtype=dtype, device=dev) for name, (n, dtype) in self._sizes.items()}
            if count:
                # the zeros are written on torch's stream, the steps run on the context's
                torch.cuda.current_stream().synchronize()
                self._own = list(state.values())
        self.state = dict(state)
        self._fill("numel", map(torch.Tensor.numel, self.params))
        self._fill("weight_decay", decay, "d")
        self._bind()
        self._grad_words = self._field("grad")

    @property
    def moments(self):
        return self._moments

    @property
    def betas(self):
        return self._options.beta1, self._options.beta2

    @betas.setter
    def betas(self, betas):
        self._options.beta1, self._options.beta2 = betas

    @property
    def eps(self):
        return self._options.eps

    @eps.setter
    def eps(self, eps):
        self._options.eps = eps

    @property
    def seed(self):
        return self._options.seed

    @seed.setter
    def seed(self, seed):
        self._options.seed = seed & (2 ** 64 - 1)

    def _field(self, name):
        return self._words[getattr(_AdamWTensor, name).offset // 8::ctypes.sizeof(_AdamWTensor) // 8]

    def _fill(self, name, values, typecode="Q"):
        self._field(name)[:] = memoryview(array.array(typecode, values)).cast("B").cast("Q")

    def _check_tensors(self, state):
        """Raise unless params, copies and state (None: still to be made) can be used."""
        given = [c for c in self.copies if c is not None]
        for name, tensors, dtype in (("parameters", self.params, torch.float32), ("copies", given, torch.bfloat16)):
            if any(d != dtype for d in map(_DTYPE, tensors)):
                raise TypeError(f"{name} must be {str(dtype)[6:]}, not {set(map(_DTYPE, tensors)) - {dtype}}")
        if len(self.params) != len(self._shapes) or len(self.copies) != len(self._shapes):
            raise ValueError("params and copies must keep their lengths")
        places = [shape for shape, c in zip(self._shapes, self.copies) if c is not None]
        for name, tensors, shapes in (("a parameter", self.params, self._shapes), ("a copy", given, places)):
            if list(map(_SHAPE, tensors)) != shapes:
                for t, shape in zip(tensors, shapes):
                    _expect(t, shape, name)
        if state is not None:
            if set(state) != set(self._sizes):
                raise ValueError(f"state must hold {sorted(self._sizes)}, not {sorted(state)}")
            for name, (n, dtype) in self._sizes.items():
                _expect(state[name], (n,), f"state[{name!r}]")
                if state[name].dtype != dtype:
                    raise TypeError(f"state[{name!r}] must have dtype {dtype}, not {state[name].dtype}")
        _all_on_current_device(self.params, "parameters")
        _all_on_current_device(given, "copies")
        if state is not None and self.params:
            _on_current_device(**state)

    def _where(self):
        """What tells that a tensor is another one or has other memory than at the last step
        (the copies' places in the list, as some may be None)."""
        copies = [c for c in self.copies if c is not None]
        return list(map(torch.Tensor.data_ptr, self.params + copies + list(self.state.values()))), list(
            map(_NBYTES, self.params)), list(map(id, self.copies))

    def _bind(self):
        """Write the addresses that a step passes on; raise if tensors overlap."""
        where = self._where()
        begins, count = where[0], len(self.params)
        given = [c for c in self.copies if c is not None]
        sizes = where[1] + list(map(_NBYTES, given)) + list(map(_NBYTES, self.state.values()))
        spans = sorted((at, at + size) for at, size in zip(begins, sizes) if size)
        if any(x[1] > y[0] for x, y in zip(spans, spans[1:])):
            raise ValueError("parameters, copies and moments must not overlap")
        self._fill("param", begins[:count])
        places = iter(begins[count:])
        self._fill("copy", [0 if c is None else next(places) for c in self.copies])
        for name, t in self.state.items():
            per = self.BLOCK if name.endswith("_scales") else 1
            base, size = t.data_ptr(), t.element_size()
            self._fill(name, [base + at // per * size for at in self.starts])
        # moments made here that others have taken the place of: steps that use them may still run
        for t in self._own:
            if self.ctx._h and not any(t is x for x in self.state.values()):
                t.record_stream(self._stream())
        self._own = [t for t in self._own if any(t is x for x in self.state.values())]
        self._bound, self._last_copies = where, list(self.copies)   # (which keeps the ids from being used anew)

    def _follow(self):
        """Bind anew if a tensor is another one or has other memory than at the last step."""
        if self._where() != self._bound or not all(map(torch.Tensor.is_contiguous, self.params)):
            self._check_tensors(self.state)
            self._bind()

    def _stream(self):
        # (ExternalStream of 0 is not the null stream but one of torch's pool)
        handle = self.ctx._stream
        return torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()

    @classmethod
    def _starts(cls, params):
        starts, at = [], 0
        for p in params:
            starts.append(at)
            at += -(-p.numel() // cls.ALIGN) * cls.ALIGN
        return starts, at

    @classmethod
    def state_sizes(cls, params, moments: str = "f32"):
        """``{name: (elements, dtype)}`` of the flat state tensors."""
        return cls._state_of(cls._starts(params)[1], moments)

    @classmethod
    def _state_of(cls, total, moments):
        if moments == "f32":
            return {"m": (total, torch.float32), "v": (total, torch.float32)}
        return {"m": (total, torch.uint8), "v": (total, torch.uint8),
                "m_scales": (total // cls.BLOCK, torch.float32), "v_scales": (total // cls.BLOCK, torch.float32)}

    def step(self, grads, lr, step=None, grad_scale=None):
        """One step with ``grads`` (one per parameter, all float32 or all bfloat16).

        ``lr``: a number, or a float32 tensor of one element.  ``step``: the step's
        number from 1 (default: one more than the last one's), or an int64
        tensor of one element, which the caller advances (below 1 it skips the
        step).  A captured step needs
        both as tensors where they change from replay to replay.
        ``grad_scale``: a float32 tensor of one element; NaN skips the step (which
        counts all the same: the host does not know).
        """
        grads = list(grads)
        if self._tensors is None:
            raise GiftError(EINVAL, "the optimizer is closed")
        if len(grads) != len(self.params):
            raise ValueError("grads must have one entry per parameter")
        shapes = list(map(_SHAPE, grads))
        if shapes != self._shapes:
            if len(shapes) != len(self._shapes):
                raise ValueError("params and copies must keep their lengths")
            got, want = next((g, p) for g, p in zip(shapes, self._shapes) if g != p)
            raise ValueError(f"a gradient must have shape {tuple(want)}, not {tuple(got)}")
        if grad_scale is not None and not isinstance(grad_scale, torch.Tensor):
            raise TypeError("grad_scale must be a tensor")
        o = self._options
        o.lr_dev, o.step_dev = _scalar(lr, torch.float32, "lr"), _scalar(step, torch.int64, "step")
        o.grad_scale = _scalar(grad_scale, torch.float32, "grad_scale")
        on_device = o.step_dev is not None
        number = 0 if on_device else self.steps + 1 if step is None else int(step)
        o.lr, o.step = 0.0 if o.lr_dev is not None else lr, number
        self._follow()
        if grads:
            o.grad_dtype, ptrs = _gradient_list(grads)
            self._grad_words[:] = memoryview(ptrs)
        _check(LIB.gift_adamw_step(self.ctx._h, len(grads), self._tensors, ctypes.byref(o)))
        if not on_device:
            self.steps = number

    def close(self):
        """Wait for the context's stream, if the moments are this object's own, and let go of them."""
        if self._own and self.ctx._h:
            self._stream().synchronize()
        self._own, self._last_copies, self.state, self._tensors, self.params = [], [], {}, None, []
        self._shapes = self._grad_words = self._words = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
