"""Thin ctypes binding of libagzo.so: argument marshalling only.

Function names and argument order are those of include/agzo.h.  Tensors are
torch tensors on the GPU (torch is used for device memory and streams only);
nothing is computed here, and there is no fallback: if the HIP library is not
built, importing the entry points raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libagzo.so")

F32, BF16 = 0, 1
LOSS_NONE, LOSS_MSE, LOSS_CE = 0, 1, 2
SKETCH_NONE, SKETCH_RANGE, SKETCH_POWER, SKETCH_RANGE_FUSED = 0, 1, 2, 3
TAG_G, TAG_OMEGA, TAG_Q0, TAG_DENSE = 0, 1, 2, 3
ONE_SIDED, NAIVE_INPLACE, INIT_FEATURE, SHARED_FORWARD = 1, 2, 4, 8
OK, EINVAL, ENOMEM, ENUMERIC, EHIP = 0, -1, -2, -3, -4

TILING_AUTO, TILING_LARGE = 0, 1
PROF_GEMM, PROF_UPDATE, PROF_XQ, PROF_XTT, PROF_QR, PROF_FILL = range(6)
PROF_ALL = 63

EXPORTS = ["agzo_create", "agzo_destroy", "agzo_last_error", "agzo_check", "agzo_profile_enable",
           "agzo_profile_read", "agzo_profile_clock", "agzo_probe_mfma", "agzo_philox_words", "agzo_fill_normal",
           "agzo_layer_forward_sketch", "agzo_qr", "agzo_basis", "agzo_perturbed_forward", "agzo_two_point", "agzo_dense_perturb", "agzo_update", "agzo_update_noalloc",
           "agzo_update_many", "agzo_step", "agzo_step_no_update", "agzo_basis_many", "agzo_step_many",
           "agzo_glue_rmsnorm", "agzo_glue_swiglu", "agzo_glue_add", "agzo_glue_attention",
           "agzo_glue_qk_norm_rope", "agzo_glue_qk_norm_rope_backward", "agzo_glue_attention_packed", "agzo_glue_attention_packed_backward",
           "agzo_ce_forward", "agzo_ce_backward"]


class AgzoLayer(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int64), ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
                ("r", ctypes.c_int32), ("dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32),
                ("tiling", ctypes.c_int32), ("ldw", ctypes.c_int64), ("ldx", ctypes.c_int64),
                ("ldy", ctypes.c_int64)]


class AgzoLossSpec(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("target_dtype", ctypes.c_int32), ("target", ctypes.c_void_p),
                ("ldt", ctypes.c_int64)]


class AgzoUpdateItem(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("B", ctypes.c_void_p), ("g_dev", ctypes.c_void_p),
                ("d_out", ctypes.c_int64), ("d_in", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("r", ctypes.c_int32), ("dtype", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("lr", ctypes.c_float), ("reserved", ctypes.c_int32)]


class AgzoBasisItem(ctypes.Structure):
    _fields_ = [("layer", AgzoLayer), ("X", ctypes.c_void_p), ("seed", ctypes.c_uint64), ("S0", ctypes.c_void_p),
                ("B", ctypes.c_void_p)]


class AgzoStepItem(ctypes.Structure):
    _fields_ = [("layer", AgzoLayer), ("W", ctypes.c_void_p), ("X", ctypes.c_void_p), ("loss", AgzoLossSpec),
                ("seed", ctypes.c_uint64), ("out_dev", ctypes.c_void_p), ("B_out", ctypes.c_void_p)]


class AgzoPackedAttention(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("ldq", ctypes.c_int64), ("ldk", ctypes.c_int64), ("ldv", ctypes.c_int64),
                ("cu_q", ctypes.c_void_p), ("cu_k", ctypes.c_void_p), ("k_len", ctypes.c_void_p), ("n_q", ctypes.c_int64), ("n_k", ctypes.c_int64),
                ("n_seq", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("scale", ctypes.c_float)]


class AgzoError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("agzo error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load():
    """Load the built library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libagzo.so is not built: run `python -m paper_2601_17261_amd.build` "
                          "(there is no CPU fallback for the HIP path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                                   ctypes.c_uint64, ctypes.c_float)
    lp, sp = ctypes.POINTER(AgzoLayer), ctypes.POINTER(AgzoLossSpec)
    lib.agzo_create.argtypes = [ctypes.POINTER(vp), vp]
    lib.agzo_destroy.argtypes = [vp]
    lib.agzo_destroy.restype = None
    lib.agzo_last_error.argtypes = [vp]
    lib.agzo_last_error.restype = ctypes.c_char_p
    lib.agzo_check.argtypes = [vp]
    lib.agzo_profile_enable.argtypes = [vp, i32]
    lib.agzo_profile_read.argtypes = [vp, i32, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double)]
    lib.agzo_profile_clock.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double)]
    lib.agzo_probe_mfma.argtypes = [vp, vp, i32, i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.agzo_philox_words.argtypes = [vp, vp, i64, i32, u64, u32]
    lib.agzo_fill_normal.argtypes = [vp, vp, i64, i32, u64, u32]
    lib.agzo_layer_forward_sketch.argtypes = [vp, lp, vp, vp, vp, i32, vp, u64, vp, sp, vp]
    lib.agzo_qr.argtypes = [vp, vp, i64, i32, vp]
    lib.agzo_basis.argtypes = [vp, lp, vp, i32, u64, vp, i32, vp]
    lib.agzo_perturbed_forward.argtypes = [vp, lp, vp, vp, vp, u64, f32, vp, sp, vp]
    lib.agzo_two_point.argtypes = [vp, vp, f32, i32]
    lib.agzo_dense_perturb.argtypes = [vp, vp, i32, i64, i64, i64, u64, f32, vp]
    lib.agzo_update.argtypes = [vp, lp, vp, vp, u64, f32, vp]
    lib.agzo_update_noalloc.argtypes = [vp, lp, vp, vp, u64, f32, vp]
    lib.agzo_update_many.argtypes = [vp, ctypes.POINTER(AgzoUpdateItem), i32]
    lib.agzo_basis_many.argtypes = [vp, ctypes.POINTER(AgzoBasisItem), i32, i32, i32]
    lib.agzo_step_many.argtypes = [vp, ctypes.POINTER(AgzoStepItem), i32, i32, f32, f32, i32]
    lib.agzo_glue_rmsnorm.argtypes = [vp, vp, i64, vp, i64, vp, i64, i64, f32]
    lib.agzo_glue_swiglu.argtypes = [vp, vp, i64, vp, i64, vp, i64, i64, i64]
    lib.agzo_glue_add.argtypes = [vp, vp, i64, vp, i64, i64, i64]
    lib.agzo_glue_attention.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, f32]
    pp = ctypes.POINTER(AgzoPackedAttention)
    lib.agzo_glue_qk_norm_rope.argtypes = [vp, vp, i64, vp, i64, vp, vp, i64, vp, i64, i64, i32, i32, i32, vp, vp, f32, f32]
    lib.agzo_glue_qk_norm_rope_backward.argtypes = [vp, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, f32, f32]
    lib.agzo_glue_attention_packed.argtypes = [vp, pp, vp, i64, vp]
    lib.agzo_glue_attention_packed_backward.argtypes = [vp, pp, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, i64]
    lib.agzo_ce_forward.argtypes = [vp, lp, vp, vp, sp, vp, vp]
    lib.agzo_ce_backward.argtypes = [vp, lp, vp, vp, sp, vp, vp, vp, i64, vp, i64]
    lib.agzo_step.argtypes = [vp, lp, vp, vp, sp, i32, f32, f32, u64, i32, vp]
    lib.agzo_step_no_update.argtypes = [vp, lp, vp, vp, sp, i32, f32, u64, i32, vp, vp]
    for name in EXPORTS:
        if name not in ("agzo_destroy", "agzo_last_error"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dt(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("unsupported dtype %s" % t.dtype)


# (the calls on packed batches take some microseconds, so what is asked of each tensor on the way to them is asked once.  device: an index; None: any)
def _elsewhere(t, device):
    raise ValueError("a tensor on %s, and the context is of cuda:%d" % (t.device, device))


def _matrix(t, name, device=None, dtype=torch.bfloat16):
    """(pointer, leading dimension, rows, values of a row) of a matrix, bf16 unless another type is asked for."""
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if device is not None and t.get_device() != device:
        _elsewhere(t, device)
    shape, strides = t.shape, t.stride()
    if len(strides) != 2 or (strides[1] != 1 and shape[1] > 1 and shape[0]):
        raise ValueError("%s must be a matrix with unit stride along its last axis" % name)
    n, d = shape
    # (the stride of a single row says nothing)
    return t.data_ptr(), strides[0] if n > 1 else d, n, d


def _rows(t, name, n=None, d=None, device=None, dtype=torch.bfloat16):
    """(pointer, leading dimension) of a matrix, of n x d if these are given; of None, nothing."""
    if t is None:
        return None, 0
    p, ld, n_, d_ = _matrix(t, name, device, dtype)
    if n is not None and (n_ != n or d_ != d):
        raise ValueError("%s must have the shape %s" % (name, (n, d)))
    return p, ld


def _flat(t, name, dtype, numel, device=None):
    """Pointer of a contiguous tensor of so many values; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if device is not None and t.get_device() != device:
        _elsewhere(t, device)
    if t.numel() != numel or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous values" % (name, numel))
    return t.data_ptr()


def _same_shape(name, t, like):
    if t is not None and (like is None or t.shape != like.shape):
        raise ValueError("%s must have the shape %s" % (name, None if like is None else tuple(like.shape)))


def make_layer(W=None, X=None, r=1, Y=None, d_out=None):
    """Descriptor for row-major 2-D tensors W [d_out][d_in], X [n][d_in], optional Y [n][d_out]."""
    L = AgzoLayer()
    L.n_tokens, L.d_in = X.shape
    L.d_out = W.shape[0] if W is not None else (d_out or 0)
    L.r = r
    L.dtype = _dt(X)
    L.y_dtype = _dt(Y) if Y is not None else F32
    L.ldx = X.stride(0)
    L.ldw = W.stride(0) if W is not None else L.d_in
    L.ldy = Y.stride(0) if Y is not None else L.d_out
    return L


def make_loss(target=None, kind=LOSS_MSE):
    s = AgzoLossSpec()
    if target is None:
        s.kind = LOSS_NONE
        return s
    s.kind = kind
    s.target = target.data_ptr()
    s._target = target      # (as long as the address is in use; what ce_forward and ce_backward look at)
    if kind == LOSS_CE and target.dtype != torch.int32:
        raise TypeError("cross-entropy targets must be int32 ids")
    if kind == LOSS_MSE:
        s.target_dtype = _dt(target)
        s.ldt = target.stride(0)
    return s


class Context:
    """Owns an agzo_ctx bound to a torch stream (default: the current one)."""

    def __init__(self, stream=None):
        self.lib = load()
        if not torch.cuda.is_available():
            raise RuntimeError("the AGZO HIP path needs a GPU")
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        h = ctypes.c_void_p()
        rc = self.lib.agzo_create(ctypes.byref(h), ctypes.c_void_p(self.stream.cuda_stream))
        if rc != 0:
            raise AgzoError(rc, "agzo_create failed")
        self.h = h
        self.device = self.stream.device.index

    def close(self):
        if getattr(self, "h", None):
            self.lib.agzo_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rc(self, rc):
        if rc != 0:
            raise AgzoError(rc, self.lib.agzo_last_error(self.h).decode())

    # --- one method per C entry point, same name without the prefix -------------------------
    def check(self):
        self._rc(self.lib.agzo_check(self.h))

    def profile_enable(self, on):
        """on: False / True (all kernel classes) or a mask of (1 << PROF_x) bits."""
        mask = (PROF_ALL if on else 0) if isinstance(on, bool) else int(on)
        self._rc(self.lib.agzo_profile_enable(self.h, mask))

    def profile_read(self, kind):
        n, ms = ctypes.c_int64(0), ctypes.c_double(0.0)
        self._rc(self.lib.agzo_profile_read(self.h, kind, ctypes.byref(n), ctypes.byref(ms)))
        return n.value, ms.value

    def profile_clock(self):
        n, ghz = ctypes.c_int64(0), ctypes.c_double(0.0)
        self._rc(self.lib.agzo_profile_clock(self.h, ctypes.byref(n), ctypes.byref(ghz)))
        return n.value, ghz.value

    def probe_mfma(self, operands, duty, iters):
        """operands: 32 KiB device tensor of bf16 bit patterns; duty 1..8 of 8 groups of 32x32x16 instructions, or 9 for
        the flop count of all 8 from 16x16x32 instructions.  Returns (TFLOP/s, shader clock in GHz)."""
        if operands.numel() * operands.element_size() < 32768 or not operands.is_contiguous():
            raise ValueError("operands must be a contiguous device tensor of at least 32 KiB")
        tf, ghz = ctypes.c_double(0.0), ctypes.c_double(0.0)
        self._rc(self.lib.agzo_probe_mfma(self.h, _ptr(operands), duty, iters, ctypes.byref(tf), ctypes.byref(ghz)))
        return tf.value, ghz.value

    def philox_words(self, dst, seed, tag):
        rows, cols = dst.shape
        self._rc(self.lib.agzo_philox_words(self.h, _ptr(dst), rows, cols, seed, tag))

    def fill_normal(self, dst, seed, tag):
        rows, cols = dst.shape
        self._rc(self.lib.agzo_fill_normal(self.h, _ptr(dst), rows, cols, seed, tag))

    def layer_forward_sketch(self, L, W, X, Y, mode, Q, seed, S, loss, loss_dev):
        self._rc(self.lib.agzo_layer_forward_sketch(self.h, ctypes.byref(L), _ptr(W), _ptr(X), _ptr(Y), mode,
                                                    _ptr(Q), seed, _ptr(S),
                                                    ctypes.byref(loss) if loss is not None else None,
                                                    _ptr(loss_dev)))

    def qr(self, S, Q):
        d, r = S.shape
        self._rc(self.lib.agzo_qr(self.h, _ptr(S), d, r, _ptr(Q)))

    def basis(self, L, X, K, seed, S0, flags, B):
        self._rc(self.lib.agzo_basis(self.h, ctypes.byref(L), _ptr(X), K, seed, _ptr(S0), flags, _ptr(B)))

    def perturbed_forward(self, L, W, X, B, seed, eps_signed, Y, loss, loss_dev):
        self._rc(self.lib.agzo_perturbed_forward(self.h, ctypes.byref(L), _ptr(W), _ptr(X), _ptr(B), seed,
                                                 eps_signed, _ptr(Y),
                                                 ctypes.byref(loss) if loss is not None else None, _ptr(loss_dev)))

    def two_point(self, out4_dev, eps, flags=0):
        if out4_dev.dtype != torch.float64 or out4_dev.numel() < 4 or not out4_dev.is_contiguous():
            raise TypeError("out4_dev must be 4 contiguous float64 values on the device")
        self._rc(self.lib.agzo_two_point(self.h, _ptr(out4_dev), eps, flags))

    def dense_perturb(self, theta, seed, scale, g_dev=None):
        """theta: 1-D (taken as one row) or 2-D device tensor, fp32 or bf16, unit stride along the last axis."""
        if theta.dim() == 1:
            rows, cols, ld = 1, theta.shape[0], theta.shape[0]
        else:
            rows, cols = theta.shape
            ld = theta.stride(0)
        if theta.numel() and theta.stride(-1) != 1:
            raise ValueError("theta must have unit stride along its last axis")
        self._rc(self.lib.agzo_dense_perturb(self.h, _ptr(theta), _dt(theta), rows, cols, ld, seed, scale, _ptr(g_dev)))

    def update(self, L, W, B, seed, lr, g_dev):
        self._rc(self.lib.agzo_update(self.h, ctypes.byref(L), _ptr(W), _ptr(B), seed, lr, _ptr(g_dev)))

    def update_noalloc(self, L, W, B, seed, lr, g_dev):
        self._rc(self.lib.agzo_update_noalloc(self.h, ctypes.byref(L), _ptr(W), _ptr(B), seed, lr, _ptr(g_dev)))

    def update_many(self, items):
        """items: sequence of (W, B, seed, lr, g_dev) with W a 2-D device tensor (unit stride along d_in), B [d_in][r]."""
        arr = (AgzoUpdateItem * max(len(items), 1))()
        for it, (W, B, seed, lr, g_dev) in zip(arr, items):
            it.W, it.B, it.g_dev = W.data_ptr(), B.data_ptr(), (0 if g_dev is None else g_dev.data_ptr())
            it.d_out, it.d_in, it.ldw = W.shape[0], W.shape[1], W.stride(0)
            it.r, it.dtype, it.seed, it.lr, it.reserved = B.shape[1], _dt(W), seed, lr, 0
        self.update_many_raw(arr, len(items))

    def update_many_raw(self, arr, n):
        self._rc(self.lib.agzo_update_many(self.h, arr, n))

    def basis_many(self, items, K, flags=0):
        """items: sequence of (L, X, seed, S0 or None, B)."""
        arr = (AgzoBasisItem * max(len(items), 1))()
        for it, (L, X, seed, S0, B) in zip(arr, items):
            it.layer, it.X, it.seed = L, X.data_ptr(), seed
            it.S0, it.B = (0 if S0 is None else S0.data_ptr()), B.data_ptr()
        self._rc(self.lib.agzo_basis_many(self.h, arr, len(items), K, flags))

    def make_step_items(self, items):
        """items: sequence of (L, W, X, loss, seed, out_dev, B_out or None) -> ctypes array for step_many_raw (the seeds
        can be rewritten in place between steps)."""
        arr = (AgzoStepItem * max(len(items), 1))()
        for it, (L, W, X, loss, seed, out_dev, B_out) in zip(arr, items):
            it.layer, it.W, it.X, it.loss, it.seed = L, W.data_ptr(), X.data_ptr(), loss, seed
            it.out_dev, it.B_out = out_dev.data_ptr(), (0 if B_out is None else B_out.data_ptr())
        return arr

    def step_many_raw(self, arr, n, K, eps, lr, flags=0):
        self._rc(self.lib.agzo_step_many(self.h, arr, n, K, eps, lr, flags))

    def step_many(self, items, K, eps, lr, flags=0):
        self.step_many_raw(self.make_step_items(items), len(items), K, eps, lr, flags)

    def glue_rmsnorm(self, x, y, gain=None, eps=1e-6):
        n, d = x.shape
        self._rc(self.lib.agzo_glue_rmsnorm(self.h, _ptr(x), x.stride(0), _ptr(y), y.stride(0), _ptr(gain), n, d, eps))

    def glue_swiglu(self, a, u, m):
        n, d = a.shape
        self._rc(self.lib.agzo_glue_swiglu(self.h, _ptr(a), a.stride(0), _ptr(u), u.stride(0), _ptr(m), m.stride(0), n, d))

    def glue_add(self, h, delta):
        n, d = h.shape
        self._rc(self.lib.agzo_glue_add(self.h, _ptr(h), h.stride(0), _ptr(delta), delta.stride(0), n, d))

    def glue_attention(self, q, k, v, out, n_seq, seq_len, rope_theta=1.0e6):
        n_heads, n_kv = q.shape[1] // 128, k.shape[1] // 128
        self._rc(self.lib.agzo_glue_attention(self.h, _ptr(q), q.stride(0), _ptr(k), k.stride(0), _ptr(v), v.stride(0),
                                              _ptr(out), out.stride(0), n_seq, seq_len, n_heads, n_kv, rope_theta))

    def _same_device(self, *tensors):
        device = self.device
        for t in tensors:
            if t is not None and t.get_device() != device:
                raise ValueError("a tensor on %s, and the context is of %s" % (t.device, self.stream.device))

    def _ce_operands(self, L, W, X, loss):
        """Pointers of W and X, which have to be those that L describes, and the ids as many as its tokens."""
        dtype, at = torch.bfloat16 if L.dtype == BF16 else torch.float32, self.device
        pointers = []
        for t, name, n, ld in ((W, "W", L.d_out, L.ldw), (X, "X", L.n_tokens, L.ldx)):
            p, ld_, n_, d_ = (None, ld, n, L.d_in) if t is None else _matrix(t, name, at, dtype)
            if n_ != n or d_ != L.d_in or (n > 1 and ld_ != ld):
                raise ValueError("%s is %d x %d with rows %d apart, the layer's %d x %d, %d apart" % (name, n_, d_, ld_, n, L.d_in, ld))
            pointers.append(p)
        if loss.kind == LOSS_CE:
            ids = getattr(loss, "_target", None)
            if ids is None or (_flat(ids, "ids", torch.int32, L.n_tokens, at) or None) != loss.target:
                raise ValueError("the loss must be make_loss(ids, LOSS_CE)")
        return pointers

    def ce_forward(self, L, W, X, loss, loss_dev, lse=None):
        """L: make_layer(W, X); loss: make_loss(ids, LOSS_CE), ids int32 [n_tokens]; loss_dev: one float64 on the device; lse: float32 [n_tokens] or None."""
        w, x = self._ce_operands(L, W, X, loss)
        self._same_device(loss_dev, lse)
        self._rc(self.lib.agzo_ce_forward(self.h, ctypes.byref(L), w, x, ctypes.byref(loss), _flat(loss_dev, "loss_dev", torch.float64, 1),
                                          _flat(lse, "lse", torch.float32, L.n_tokens)))

    def ce_backward(self, L, W, X, loss, lse, dX, dW, g_dev=None):
        """L, loss: as for ce_forward, and lse of it; dX like X, dW like W (either may be None); g_dev: one float64 on the device or None (1)."""
        w, x = self._ce_operands(L, W, X, loss)
        self._same_device(lse, dX, dW, g_dev)
        _same_shape("dX", dX, X)
        _same_shape("dW", dW, W)
        self._rc(self.lib.agzo_ce_backward(self.h, ctypes.byref(L), w, x, ctypes.byref(loss), _flat(lse, "lse", torch.float32, L.n_tokens),
                                           _flat(g_dev, "g_dev", torch.float64, 1), *_rows(dX, "dX", dtype=X.dtype), *_rows(dW, "dW", dtype=X.dtype)))

    def glue_qk_norm_rope(self, q, k, positions, q_out, k_out, head_dim=128, q_gain=None, k_gain=None, eps=1e-6, rope_theta=1.0e6):
        """q [n][heads * head_dim], k [n][key heads * head_dim] -> q_out, k_out; either side may be None with its result."""
        (pq, lq, _, wq), (pk, lk, n, wk) = self._heads(q, k, head_dim)
        f32, at = torch.float32, self.device
        oq, loq = _rows(q_out, "q_out", n, wq, at)
        ok, lok = _rows(k_out, "k_out", n, wk, at)
        self._rc(self.lib.agzo_glue_qk_norm_rope(
            self.h, pq, lq, pk, lk, _flat(positions, "positions", torch.int32, n, at), oq, loq, ok, lok, n, wq // head_dim, wk // head_dim, head_dim,
            _flat(q_gain, "q_gain", f32, head_dim, at), _flat(k_gain, "k_gain", f32, head_dim, at), eps, rope_theta))

    def glue_qk_norm_rope_backward(self, q, k, positions, dq_out, dk_out, dq, dk, head_dim=128, q_gain=None, k_gain=None, dq_gain=None, dk_gain=None,
                                   eps=1e-6, rope_theta=1.0e6):
        """q, k: the inputs of glue_qk_norm_rope; dq_out, dk_out: the gradients with respect to its results -> dq, dk and, where given, dq_gain and
        dk_gain (float32 [head_dim])."""
        (pq, lq, _, wq), (pk, lk, n, wk) = self._heads(q, k, head_dim)
        f32, at = torch.float32, self.device
        self._rc(self.lib.agzo_glue_qk_norm_rope_backward(
            self.h, pq, lq, pk, lk, _flat(positions, "positions", torch.int32, n, at), *_rows(dq_out, "dq_out", n, wq, at), *_rows(dk_out, "dk_out", n, wk, at),
            *_rows(dq, "dq", n, wq, at), *_rows(dk, "dk", n, wk, at), n, wq // head_dim, wk // head_dim, head_dim, _flat(q_gain, "q_gain", f32, head_dim, at),
            _flat(k_gain, "k_gain", f32, head_dim, at), _flat(dq_gain, "dq_gain", f32, head_dim, at), _flat(dk_gain, "dk_gain", f32, head_dim, at), eps, rope_theta))

    def _heads(self, q, k, head_dim):
        if q is None and k is None:
            raise ValueError("neither q nor k is given")
        a = None if q is None else _matrix(q, "q", self.device)
        b = (None, 0, a[2], 0) if k is None else _matrix(k, "k", self.device)
        a = a or (None, 0, b[2], 0)
        if a[2] != b[2] or a[3] % head_dim or b[3] % head_dim:
            raise ValueError("%d rows of %d values, %d of %d: need as many rows, of multiples of %d" % (*a[2:], *b[2:], head_dim))
        return a, b

    def _packed(self, q, k, v, cu_q, cu_k, k_len, head_dim, scale, causal):
        at = self.device
        pq, lq, nq, wq = _matrix(q, "q", at)
        pk, lk, nk, wk = _matrix(k, "k", at)
        if wq % head_dim or wk % head_dim:
            raise ValueError("rows of %d and %d values: need multiples of %d" % (wq, wk, head_dim))
        pv, lv = _rows(v, "v", nk, wk, at)
        n_seq, i32 = cu_q.numel() - 1, torch.int32
        return AgzoPackedAttention(pq, pk, pv, lq, lk, lv, _flat(cu_q, "cu_q", i32, n_seq + 1, at), _flat(cu_k, "cu_k", i32, n_seq + 1, at), _flat(k_len, "k_len", i32, n_seq, at),
                                   nq, nk, n_seq, wq // head_dim, wk // head_dim, head_dim, causal, head_dim ** -0.5 if scale is None else scale), nq, wq, nk, wk

    def glue_attention_packed(self, q, k, v, out, cu_q, cu_k, head_dim=128, scale=None, causal=True, lse=None, k_len=None):
        """q [n_q][heads * head_dim], k, v [n_k][key heads * head_dim] -> out like q; cu_q, cu_k: int32 offsets of the sequences
        (n_seq + 1 each); scale None: head_dim ** -0.5; lse: float32 [n_q][heads] or None; k_len: int32 [n_seq], how many keys each has
        of its room (a cache), or None: all."""
        a, nq, wq, _, _ = self._packed(q, k, v, cu_q, cu_k, k_len, head_dim, scale, causal)
        o, ldo = _rows(out, "out", nq, wq, self.device)
        self._rc(self.lib.agzo_glue_attention_packed(self.h, ctypes.byref(a), o, ldo, _flat(lse, "lse", torch.float32, nq * (wq // head_dim), self.device)))

    def glue_attention_packed_backward(self, q, k, v, out, lse, dout, dq, dk, dv, cu_q, cu_k, head_dim=128, scale=None, causal=True):
        """out, lse: of glue_attention_packed with the same arguments; dout: the gradient with respect to out -> dq, dk, dv."""
        a, nq, wq, nk, wk = self._packed(q, k, v, cu_q, cu_k, None, head_dim, scale, causal)
        at = self.device
        self._rc(self.lib.agzo_glue_attention_packed_backward(
            self.h, ctypes.byref(a), *_rows(out, "out", nq, wq, at), _flat(lse, "lse", torch.float32, nq * (wq // head_dim), at), *_rows(dout, "dout", nq, wq, at),
            *_rows(dq, "dq", nq, wq, at), *_rows(dk, "dk", nk, wk, at), *_rows(dv, "dv", nk, wk, at)))

    def step_no_update(self, L, W, X, loss, K, eps, seed, flags, out_dev, B_out):
        self._rc(self.lib.agzo_step_no_update(self.h, ctypes.byref(L), _ptr(W), _ptr(X), ctypes.byref(loss), K, eps,
                                              seed, flags, _ptr(out_dev), _ptr(B_out)))

    def step(self, L, W, X, loss, K, eps, lr, seed, flags, out_dev):
        self._rc(self.lib.agzo_step(self.h, ctypes.byref(L), _ptr(W), _ptr(X), ctypes.byref(loss), K, eps, lr,
                                    seed, flags, _ptr(out_dev)))
