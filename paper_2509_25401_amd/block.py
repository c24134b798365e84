"""ctypes binding of include/sparse_block.h: the operators around attention in a block -- argument marshalling only.

As in binding.py, results go to tensors that the caller brings, work is enqueued on `stream` (default: torch's current
stream), wrong arguments raise ValueError, errors of the library raise SparseAttnError.
"""
import ctypes

from . import binding
from .binding import _check, _dev_ptr, _raise, _stream_ptr

BF16, F32, E4M3, I32 = 0, 1, 2, 3
_NORMS = {"rms": 0, "layer": 1}
_PAIRS = {"adjacent": 0, "halves": 1}

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float


class _NormArgs(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("x", "y", "x_out", "h", "h_scales", "weight", "scale", "shift", "gate", "post_weight")]
                + [(n, _i64) for n in ("rows", "rows_per_vector", "scale_stride", "shift_stride", "gate_stride")]
                + [(n, _i32) for n in ("channels", "norm", "x_dtype", "vector_dtype", "h_dtype")]
                + [(n, _f32) for n in ("alpha", "eps", "post_eps")])


class _NormBackwardArgs(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("dh", "dx_out", "x_out", "y", "dx", "dy", "weight", "scale", "gate", "post_weight",
                                    "dweight", "dscale", "dshift", "dgate", "dpost_weight")]
                + [(n, _i64) for n in ("rows", "rows_per_vector", "scale_stride", "gate_stride")]
                + [(n, _i32) for n in ("channels", "norm", "x_dtype", "vector_dtype")]
                + [(n, _f32) for n in ("alpha", "eps", "post_eps")])


class _RotaryArgs(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("qkv", "positions", "Q", "K", "V", "q_weight", "k_weight", "axis_channels", "inv_freq")]
                + [(n, _i64) for n in ("qkv_stride_b", "qkv_stride_l", "q_stride_b", "q_stride_h", "q_stride_l", "k_stride_b",
                                       "k_stride_h", "k_stride_l", "v_stride_b", "v_stride_h", "v_stride_l")]
                + [(n, _i32) for n in ("B", "L", "heads_q", "heads_kv", "D", "axes", "halves", "positions_per_batch",
                                       "position_dtype")]
                + [("eps", _f32), ("theta", ctypes.c_double)])


_lib = None
_torch = None


def _library():
    global _lib, _torch
    if _lib is None:
        import torch
        lib = binding.load_library()
        lib.sparse_block_norm.argtypes = [ctypes.POINTER(_NormArgs), _vp]
        lib.sparse_block_norm_backward.argtypes = [ctypes.POINTER(_NormBackwardArgs), _vp]
        lib.sparse_rotary_heads.argtypes = [ctypes.POINTER(_RotaryArgs), _vp]
        lib.sparse_rotary_heads_backward.argtypes = [ctypes.POINTER(_RotaryArgs), _vp, _i64, _i64, _vp, _vp, _vp]
        lib.sparse_rotary_frequencies.argtypes = [_i32, _vp, ctypes.c_double, _vp]
        lib.sparse_rotary_frequencies.restype = None
        lib.sparse_fp8_quantize.argtypes = [_vp] * 5 + [_i64] * 3 + [_i32, _vp]
        lib.sparse_fp8_gemm.argtypes = [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _i32, _i64, _i64, _i64, _vp]
        lib.sparse_fp8_linear.argtypes = [_vp] * 5 + [_i32, _i64, _i64, _i64, _vp]
        lib.sparse_fp8_linear_backward.argtypes = [_vp] * 6 + [_i32, _vp, _i64, _i64, _i64, _vp]
        for name in ("sparse_block_norm", "sparse_block_norm_backward", "sparse_rotary_heads", "sparse_rotary_heads_backward",
                     "sparse_fp8_quantize", "sparse_fp8_gemm", "sparse_fp8_linear", "sparse_fp8_linear_backward"):
            getattr(lib, name).restype = _i32
        _torch, _lib = torch, lib
    return _lib


def _float_dtype(t, name):
    if t.dtype is _torch.bfloat16:
        return BF16
    if t.dtype is _torch.float32:
        return F32
    raise ValueError(f"{name} must have dtype torch.bfloat16 or torch.float32, got {t.dtype}")


def _rows(t, name):
    """(batches, tokens, channels) of [B, L, C] or [rows, C]."""
    s = t.shape
    if len(s) == 3:
        return s[0], s[1], s[2]
    if len(s) == 2:
        return 1, s[0], s[1]
    raise ValueError(f"{name} must be [B, L, C] or [rows, C]")


class _Vectors:
    """The modulation vectors of a call: one type, one number of tokens for each vector."""

    def __init__(self, B, L, C, device):
        self.B, self.L, self.C, self.device = B, L, C, device
        self.rows_per = None
        self.dtype = None

    def _group(self, shape, name):
        """Tokens that share a vector of a tensor of this shape; None where all of them do."""
        B, L, C = self.B, self.L, self.C
        if len(shape) == 1 and shape[0] == C:
            return None
        if len(shape) == 2 and shape[0] == B and shape[1] == C:
            per = L
        elif len(shape) == 3 and shape[0] == B and shape[2] == C and shape[1] > 0 and L % shape[1] == 0:
            per = L // shape[1]
        else:
            raise ValueError(f"{name} must be [C], [B, C] or [B, F, C] with F frames of L / F tokens, got {tuple(shape)}")
        if self.rows_per is not None and self.rows_per != per:
            raise ValueError(f"{name} has another number of vectors than the others")
        self.rows_per = per
        return per

    def _typed(self, t, name):
        if t.get_device() != self.device:
            raise ValueError(f"{name} must live in device memory, on the device of the others")
        d = _float_dtype(t, name)
        if self.dtype is not None and d != self.dtype:
            raise ValueError(f"{name} must have the dtype of the other vectors")
        self.dtype = d

    def add(self, t, name):
        """(address, elements between vectors) of scale, shift or gate."""
        if t is None:
            return None, 0
        self._typed(t, name)
        shape, stride = t.shape, t.stride()
        per = self._group(shape, name)
        if shape[-1] > 1 and stride[-1] != 1:
            raise ValueError(f"{name} must have contiguous channels")
        if per is None:
            return t.data_ptr(), 0
        if len(shape) == 2:
            return t.data_ptr(), stride[0] if shape[0] > 1 else 0
        B, F = shape[0], shape[1]
        if B > 1 and F > 1 and stride[0] != F * stride[1]:
            raise ValueError(f"{name} must have one step between all its vectors")
        return t.data_ptr(), stride[1] if F > 1 else stride[0] if B > 1 else 0

    def weight(self, t, name):
        if t is None:
            return None
        self._typed(t, name)
        if len(t.shape) != 1 or t.shape[0] != self.C or not t.is_contiguous():
            raise ValueError(f"{name} must be [C] and contiguous")
        return t.data_ptr()

    def sums(self, t, name):
        """Address of a gradient of the vectors."""
        if t is None:
            return None
        if self._group(t.shape, name) is None and self.rows_per is None:
            self.rows_per = self.B * self.L
        if t.dtype is not _torch.float32 or t.get_device() != self.device or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 tensor on the device of the others")
        return t.data_ptr()

    def check_sums(self, t, name, rows):
        if t is not None and t.numel() != -(-rows // self.rows_per) * self.C:
            raise ValueError(f"{name} has another number of vectors than the others")


def _norm_kind(norm):
    if norm not in _NORMS:
        raise ValueError(f"norm must be one of {sorted(_NORMS)}, got {norm!r}")
    return _NORMS[norm]


def _tensor(t, name, dtype, shape, device, allow_none=False):
    """Address of a contiguous tensor of this dtype and shape on GPU number `device`."""
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} must not be None")
    if t.dtype is dtype and t.shape == shape and t.get_device() == device >= 0 and t.is_contiguous():
        return t.data_ptr()
    _check(t, name, dtype, shape)
    _dev_ptr(t, name)
    raise ValueError(f"all tensors must live on one device, {name} is on {t.device}")


def sparse_block_norm(x, y, h, x_out=None, norm="layer", eps=1e-6, weight=None, scale=None, shift=None, gate=None,
                      post_weight=None, post_eps=None, alpha=1.0, h_scales=None, stream=None):
    """x' = alpha x + gate * t with t = y, or RMSNorm(y) * post_weight;  h = norm(x') * weight * (1 + scale) + shift.

    x [B,L,C] or [rows,C], bf16 or float32; y bf16 like x, or None (nothing is added); x_out like x, written (may be x);
    h bf16 like x, or float8_e4m3fn with h_scales uint8 [..., ceil(C/128)], or None.  scale, shift, gate: [C], [B,C] or
    [B,F,C] (F frames of L/F tokens), any step between the vectors; weight, post_weight [C]; all of one dtype, bf16 or
    float32.  norm: "layer" or "rms".  Returns (x_out, h)."""
    lib = _lib or _library()
    if x is None:
        raise ValueError("x must not be None")
    B, L, C = _rows(x, "x")
    shape, device = x.shape, x.get_device()
    bf16 = _torch.bfloat16
    xt = _float_dtype(x, "x")
    px = _tensor(x, "x", x.dtype, shape, device)
    py = _tensor(y, "y", bf16, shape, device, True)
    po = _tensor(x_out, "x_out", x.dtype, shape, device, y is None)
    ht, ps = BF16, None
    if h is not None and h.dtype is _torch.float8_e4m3fn:
        ht = E4M3
        ph = _tensor(h, "h", h.dtype, shape, device)
        ps = _tensor(h_scales, "h_scales", _torch.uint8, (*shape[:-1], -(-C // 128)), device)
    else:
        ph = _tensor(h, "h", bf16, shape, device, True)
        if h_scales is not None:
            raise ValueError("h_scales goes with a float8_e4m3fn h")
    v = _Vectors(B, L, C, device)
    ps_, ss = v.add(scale, "scale")
    pb_, bs = v.add(shift, "shift")
    pg_, gs = v.add(gate, "gate")
    pw, pp = v.weight(weight, "weight"), v.weight(post_weight, "post_weight")
    args = _NormArgs(px, py, po, ph, ps, pw, ps_, pb_, pg_, pp, B * L, v.rows_per or B * L, ss, bs, gs, C, _norm_kind(norm), xt,
                     v.dtype or 0, ht, alpha, eps, eps if post_eps is None else post_eps)
    rc = lib.sparse_block_norm(ctypes.byref(args), _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return x_out, h


def sparse_block_norm_backward(dh, dx_out, x_out, y, dx, dy=None, norm="layer", eps=1e-6, weight=None, scale=None, gate=None,
                               post_weight=None, post_eps=None, alpha=1.0, dweight=None, dscale=None, dshift=None, dgate=None,
                               dpost_weight=None, stream=None):
    """Gradients of sparse_block_norm for dh (of h, bf16) and dx_out (of x_out, or None); x_out is the stored x', y as in the
    forward call.  Written: dx like x_out (may be dx_out), dy bf16; float32 sums dscale, dshift, dgate [C], [B,C] or [B,F,C]
    and dweight, dpost_weight [C], each where given.  Returns (dx, dy)."""
    lib = _lib or _library()
    if x_out is None:
        raise ValueError("x_out must not be None")
    B, L, C = _rows(x_out, "x_out")
    shape, device = x_out.shape, x_out.get_device()
    bf16, f32 = _torch.bfloat16, _torch.float32
    xt = _float_dtype(x_out, "x_out")
    pdh = _tensor(dh, "dh", bf16, shape, device)
    pdo = _tensor(dx_out, "dx_out", x_out.dtype, shape, device, True)
    px = _tensor(x_out, "x_out", x_out.dtype, shape, device)
    py = _tensor(y, "y", bf16, shape, device, True)
    pdx = _tensor(dx, "dx", x_out.dtype, shape, device)
    pdy = _tensor(dy, "dy", bf16, shape, device, True)
    v = _Vectors(B, L, C, device)
    ps, ss = v.add(scale, "scale")
    pg, gs = v.add(gate, "gate")
    pw, pp = v.weight(weight, "weight"), v.weight(post_weight, "post_weight")
    pds, pdb, pdg = v.sums(dscale, "dscale"), v.sums(dshift, "dshift"), v.sums(dgate, "dgate")
    if v.rows_per is None:
        v.rows_per = B * L
    v.check_sums(dscale, "dscale", B * L)
    v.check_sums(dshift, "dshift", B * L)
    v.check_sums(dgate, "dgate", B * L)
    pdw = _tensor(dweight, "dweight", f32, (C,), device, True)
    pdp = _tensor(dpost_weight, "dpost_weight", f32, (C,), device, True)
    args = _NormBackwardArgs(pdh, pdo, px, py, pdx, pdy, pw, ps, pg, pp, pdw, pds, pdb, pdg, pdp, B * L, v.rows_per, ss, gs, C,
                             _norm_kind(norm), xt, v.dtype or 0, alpha, eps, eps if post_eps is None else post_eps)
    rc = lib.sparse_block_norm_backward(ctypes.byref(args), _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return dx, dy


def sparse_rotary_frequencies(axes, theta=10000.0):
    """[theta^(-2i/d) for each axis of d channels and its d/2 pairs i] as the library computes them."""
    if any(d < 0 for d in axes):
        raise ValueError(f"axes must not be negative, got {tuple(axes)}")
    n = sum(int(d) // 2 for d in axes)
    buf = (ctypes.c_double * max(n, 1))()
    (_lib or _library()).sparse_rotary_frequencies(len(axes), (_i32 * len(axes))(*axes), float(theta), buf)
    return list(buf[:n])


def _head_view(t, name, B, H, L, D, device, allow_none):
    """(address, strides of batches, heads and tokens) of a [B,H,L,D] view with contiguous channels."""
    if t is None:
        if allow_none:
            return None, 0, 0, 0
        raise ValueError(f"{name} must not be None")
    if t.dtype is not _torch.bfloat16 or t.shape != (B, H, L, D):
        _check(t, name, _torch.bfloat16, (B, H, L, D))
    if t.get_device() != device:
        raise ValueError(f"{name} must live in device memory, on the device of the others")
    s = t.stride()
    if s[3] != 1:
        raise ValueError(f"{name} must have contiguous channels")
    # the step of a dimension of one entry is never taken
    return t.data_ptr(), s[0] if B > 1 else 0, s[1] if H > 1 else 0, s[2] if L > 1 else 0


def _row_view(t, name, B, L, width, device):
    """(address, strides of batches and tokens) of a [B,L,width] view with contiguous channels."""
    if t.dtype is not _torch.bfloat16 or t.shape != (B, L, width):
        _check(t, name, _torch.bfloat16, (B, L, width))
    if t.get_device() != device:
        raise ValueError(f"{name} must live in device memory, on the device of the others")
    s = t.stride()
    if s[2] != 1:
        raise ValueError(f"{name} must have contiguous channels")
    return t.data_ptr(), s[0] if B > 1 else 0, s[1] if L > 1 else 0


def _rotary_args(qkv, positions, Q, K, V, B, L, Hq, Hkv, D, axes, theta, inv_freq, pairs, q_weight, k_weight, eps, device,
                 allow_none):
    n_axes = len(axes)
    if positions.dtype is _torch.int32:
        pt = I32
    elif positions.dtype is _torch.float32:
        pt = F32
    else:
        raise ValueError(f"positions must have dtype torch.int32 or torch.float32, got {positions.dtype}")
    if positions.shape == (L, n_axes):
        per_batch = 0
    elif positions.shape == (B, L, n_axes):
        per_batch = 1
    else:
        raise ValueError(f"positions must be [L, axes] or [B, L, axes], got {tuple(positions.shape)}")
    pp = _tensor(positions, "positions", positions.dtype, positions.shape, device)
    if pairs not in _PAIRS:
        raise ValueError(f"pairs must be one of {sorted(_PAIRS)}, got {pairs!r}")
    ax = (_i32 * n_axes)(*axes)
    freq = None
    if inv_freq is not None:
        n = sum(d // 2 for d in axes)
        if len(inv_freq) != n:
            raise ValueError(f"inv_freq must hold {n} values, one for each pair, got {len(inv_freq)}")
        freq = (ctypes.c_double * max(n, 1))(*inv_freq)
    q = _head_view(Q, "Q", B, Hq, L, D, device, allow_none)
    k = _head_view(K, "K", B, Hkv, L, D, device, allow_none)
    v = _head_view(V, "V", B, Hkv, L, D, device, allow_none)
    wq = _tensor(q_weight, "q_weight", _torch.bfloat16, (D,), device, True)
    wk = _tensor(k_weight, "k_weight", _torch.bfloat16, (D,), device, True)
    px, sb, sl = (None, 0, 0) if qkv is None else _row_view(qkv, "qkv", B, L, (Hq + 2 * Hkv) * D, device)
    return _RotaryArgs(px, pp, q[0], k[0], v[0], wq, wk, ctypes.addressof(ax), None if freq is None else ctypes.addressof(freq), sb,
                       sl, q[1], q[2], q[3], k[1], k[2], k[3], v[1], v[2], v[3], B, L, Hq, Hkv, D, n_axes, _PAIRS[pairs], per_batch,
                       pt, eps, theta), (ax, freq)


def sparse_rotary_heads(qkv, positions, Q, K, V, axes, theta=10000.0, inv_freq=None, pairs="adjacent", q_weight=None,
                        k_weight=None, eps=1e-6, heads=None, stream=None):
    """Splits the rows of a fused projection into heads, norms queries and keys (q_weight, k_weight [D], None: no norm) and
    turns them by the tokens' positions.

    qkv bf16 [B,L,(Hq+2Hkv)D]; positions int32 or float32 [L,A] or [B,L,A]; axes: the channels that each of the A axes turns
    (the first sum(axes) of a head); theta, or inv_freq: sum(axes)/2 floats; pairs: "adjacent" or "halves".  Q [B,Hq,L,D], K
    and V [B,Hkv,L,D] are written: bf16 views of any strides (a token range of a joint sequence, the slot of a cache).  One of
    them may be None and is left out; heads = (Hq, Hkv, D) then says what the tensors' shapes do not.  Returns (Q, K, V)."""
    _lib or _library()
    if qkv is None or positions is None:
        raise ValueError("qkv and positions must not be None")
    if qkv.dim() != 3:
        raise ValueError("qkv must be [B, L, (Hq + 2 Hkv) D]")
    B, L, _ = qkv.shape
    if heads is None:
        if Q is None or (K is None and V is None):
            raise ValueError("heads=(Hq, Hkv, D) must be given where Q, or both K and V, are None")
        kv = V if K is None else K
        heads = (Q.shape[1], kv.shape[1], Q.shape[3])
    Hq, Hkv, D = heads
    args, keep = _rotary_args(qkv, positions, Q, K, V, B, L, Hq, Hkv, D, axes, theta, inv_freq, pairs, q_weight, k_weight, eps,
                              qkv.get_device(), True)
    rc = _lib.sparse_rotary_heads(ctypes.byref(args), _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return Q, K, V


def sparse_rotary_heads_backward(dQ, dK, dV, qkv, positions, dqkv, axes, theta=10000.0, inv_freq=None, pairs="adjacent",
                                 q_weight=None, k_weight=None, eps=1e-6, dq_weight=None, dk_weight=None, stream=None):
    """Gradients of sparse_rotary_heads: dqkv bf16 [B,L,(Hq+2Hkv)D] (written), dq_weight and dk_weight float32 [D] (written
    where given).  qkv is the forward call's input; it may be None without norm weights.  Returns dqkv."""
    _lib or _library()
    if dQ is None or dK is None or dV is None or positions is None or dqkv is None:
        raise ValueError("dQ, dK, dV, positions and dqkv must not be None")
    if dQ.dim() != 4 or dK.dim() != 4:
        raise ValueError("dQ, dK and dV must be [B, H, L, D]")
    B, Hq, L, D = dQ.shape
    Hkv, device = dK.shape[1], dQ.get_device()
    args, keep = _rotary_args(qkv, positions, dQ, dK, dV, B, L, Hq, Hkv, D, axes, theta, inv_freq, pairs, q_weight, k_weight,
                              eps, device, False)
    pd, sb, sl = _row_view(dqkv, "dqkv", B, L, (Hq + 2 * Hkv) * D, device)
    pq = _tensor(dq_weight, "dq_weight", _torch.float32, (D,), device, True)
    pk = _tensor(dk_weight, "dk_weight", _torch.float32, (D,), device, True)
    rc = _lib.sparse_rotary_heads_backward(ctypes.byref(args), pd, sb, sl, pq, pk, _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return dqkv


def sparse_fp8_quantize(x, q=None, q_scales=None, qt=None, qt_scales=None, block=False, stream=None):
    """8-bit form of x (bf16 [R,C]): e4m3 values and exponent bytes, q * 2^(scale - 127), for groups of 128.

    q float8_e4m3fn [R,C] with q_scales uint8 [R,ceil(C/128)] (groups along a row), and / or the transposed form qt [C,R] with
    qt_scales [C,ceil(R/128)] (groups along the rows of x; the rows of qt start at multiples of 16 bytes, further apart than R if
    need be, and are written up to the next such multiple behind R, zeros from R on: torch.empty(C, -(-R//16)*16)[:, :R]).
    block=True: groups of 128 x 128, scales [ceil(R/128),ceil(C/128)] and transposed.  Returns (q, q_scales, qt, qt_scales)."""
    lib = _lib or _library()
    if x is None or x.dim() != 2:
        raise ValueError("x must be [R, C]")
    R, C = x.shape
    device = x.get_device()
    e4m3, u8 = _torch.float8_e4m3fn, _torch.uint8
    gr, gc = -(-R // 128), -(-C // 128)
    px = _tensor(x, "x", _torch.bfloat16, x.shape, device)
    pq = _tensor(q, "q", e4m3, (R, C), device, True)
    ps = _tensor(q_scales, "q_scales", u8, (gr if block else R, gc), device, q is None)
    pt, pitch = None, 0
    if qt is not None:
        _check(qt, "qt", e4m3, (C, R))
        if qt.get_device() != device or (R > 1 and qt.stride(1) != 1):
            raise ValueError("qt must live on the device of x, with contiguous rows")
        whole = -(-R // 16) * 16                  # what is written of a row
        pt, pitch = qt.data_ptr(), qt.stride(0) if C > 1 else whole
        if qt.untyped_storage().nbytes() - qt.storage_offset() < (C - 1) * pitch + whole:
            raise ValueError(f"the memory of qt must hold {whole} bytes behind the start of each row, its last one too")
    pts = _tensor(qt_scales, "qt_scales", u8, (gc if block else C, gr), device, qt is None)
    rc = lib.sparse_fp8_quantize(px, pq, ps, pt, pts, pitch, R, C, int(bool(block)), _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return q, q_scales, qt, qt_scales


def _scales(t, name, rows, K, device):
    """(address, whether 128 rows share a scale)"""
    groups = -(-K // 128)
    if t is None:
        raise ValueError(f"{name} must not be None")
    block = t.shape == (-(-rows // 128), groups) and rows > 1
    if not block and t.shape != (rows, groups):
        raise ValueError(f"{name} must have shape {(rows, groups)} or {(-(-rows // 128), groups)}, got {tuple(t.shape)}")
    return _tensor(t, name, _torch.uint8, t.shape, device), int(block)


def _result(t, name, shape, device):
    if t is None:
        raise ValueError(f"{name} must not be None")
    return _tensor(t, name, t.dtype, shape, device), _float_dtype(t, name)


def sparse_fp8_gemm(a, a_scales, b, b_scales, bias, out, stream=None):
    """out[m,n] = sum_k a[m,k] b[n,k] (+ bias[n]) for operands in 8-bit form: a float8_e4m3fn [M,K], b [N,K], K a multiple of 16;
    scales uint8 with a row for each row, or for each 128 rows, and a column for each 128 channels; bias bf16 [N] or None;
    out bf16 or float32 [M,N], written."""
    lib = _lib or _library()
    if a is None or b is None or a.dim() != 2 or b.dim() != 2:
        raise ValueError("a must be [M, K] and b [N, K]")
    (M, K), N, device = a.shape, b.shape[0], a.get_device()
    e4m3 = _torch.float8_e4m3fn
    pa, pb = _tensor(a, "a", e4m3, (M, K), device), _tensor(b, "b", e4m3, (N, K), device)
    sa, ba = _scales(a_scales, "a_scales", M, K, device)
    sb, bb = _scales(b_scales, "b_scales", N, K, device)
    pbias = _tensor(bias, "bias", _torch.bfloat16, (N,), device, True)
    po, ot = _result(out, "out", (M, N), device)
    rc = lib.sparse_fp8_gemm(pa, sa, ba, pb, sb, bb, pbias, po, ot, M, N, K, _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return out


def sparse_fp8_linear(x, w, w_scales, bias, out, stream=None):
    """out = x w^T (+ bias): x bf16 [M,K] is brought to 8-bit form inside the call; w float8_e4m3fn [N,K], w_scales uint8
    [ceil(N/128),ceil(K/128)] (sparse_fp8_quantize with block=True), bias bf16 [N] or None, out bf16 or float32 [M,N], written."""
    lib = _lib or _library()
    if x is None or w is None or x.dim() != 2 or w.dim() != 2:
        raise ValueError("x must be [M, K] and w [N, K]")
    (M, K), N, device = x.shape, w.shape[0], x.get_device()
    px, pw = _tensor(x, "x", _torch.bfloat16, (M, K), device), _tensor(w, "w", _torch.float8_e4m3fn, (N, K), device)
    ps = _tensor(w_scales, "w_scales", _torch.uint8, (-(-N // 128), -(-K // 128)), device)
    pbias = _tensor(bias, "bias", _torch.bfloat16, (N,), device, True)
    po, ot = _result(out, "out", (M, N), device)
    rc = lib.sparse_fp8_linear(px, pw, ps, pbias, po, ot, M, N, K, _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return out


def sparse_fp8_linear_backward(dy, x, wt, wt_scales, dx=None, dw=None, dbias=None, stream=None):
    """Gradients of sparse_fp8_linear for dy (bf16 [M,N]): dx bf16 [M,K] from the transposed weight wt float8_e4m3fn [K,N] with
    wt_scales uint8 [ceil(K/128),ceil(N/128)]; dw bf16 or float32 [N,K] from x (bf16 [M,K]); dbias float32 [N].  Each is written
    where given; N and K are multiples of 16.  Returns (dx, dw, dbias)."""
    lib = _lib or _library()
    if dy is None or dy.dim() != 2:
        raise ValueError("dy must be [M, N]")
    (M, N), device = dy.shape, dy.get_device()
    shapes = {t.shape[d] for t, d in ((x, 1), (wt, 0), (dx, 1), (dw, 1)) if t is not None and t.dim() == 2}
    if len(shapes) > 1:
        raise ValueError("shapes of x [M,K], wt [K,N], dx [M,K] and dw [N,K] do not fit together")
    K = shapes.pop() if shapes else 16            # dbias alone: nothing has K channels
    bf16 = _torch.bfloat16
    pdy = _tensor(dy, "dy", bf16, (M, N), device)
    px = _tensor(x, "x", bf16, (M, K), device, dw is None)
    pw = _tensor(wt, "wt", _torch.float8_e4m3fn, (K, N), device, dx is None)
    ps = _tensor(wt_scales, "wt_scales", _torch.uint8, (-(-K // 128), -(-N // 128)), device, dx is None)
    pdx = _tensor(dx, "dx", bf16, (M, K), device, True)
    pdw, wt_type = (None, BF16) if dw is None else _result(dw, "dw", (N, K), device)
    pdb = _tensor(dbias, "dbias", _torch.float32, (N,), device, True)
    rc = lib.sparse_fp8_linear_backward(pdy, px, pw, ps, pdx, pdw, wt_type, pdb, M, N, K, _stream_ptr(stream))
    if rc != 0:
        _raise(rc)
    return dx, dw, dbias
