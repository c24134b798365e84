"""The library's calls beside a stand-in for the HIP runtime (fake_hip.cpp): what they launch, allocate and refuse, without a GPU.

`run(scenario, ...)` builds the stand-in and runs one of the scenarios below in a process of its own, in which the library finds
the stand-in instead of the runtime.  Addresses are numbers that nothing is stored at."""
import ctypes
import json
import os
import subprocess
import sys
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def run(scenario, *args, _built=[]):
    if not _built:
        import tempfile
        _built.append(tempfile.TemporaryDirectory())
        at = _built[0].name
        versions = os.path.join(at, "versions")
        with open(versions, "w") as f:
            f.write("hip_4.2 { global: *; };\n")
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-soname,libamdhip64.so.7", "-Wl,--version-script=" + versions,
                               "-o", os.path.join(at, "libamdhip64.so.7"), os.path.join(HERE, "fake_hip.cpp")])
    env = dict(os.environ, LD_LIBRARY_PATH=_built[0].name, PYTHONPATH=ROOT)
    out = subprocess.run([sys.executable, os.path.abspath(__file__), scenario], input=json.dumps(args).encode(), env=env, stdout=subprocess.PIPE, timeout=120, check=True)
    return json.loads(out.stdout)


# ---------------------------------------------------------------------------------------
# In the child
# ---------------------------------------------------------------------------------------
_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float


def at(n):
    return (n + 1) << 47


class Library:
    def __init__(self):
        from paper_2509_25401_amd import binding, block
        self.lib, self.block = binding.load_library(), block
        self.hip = ctypes.CDLL("libamdhip64.so.7")
        lib = self.lib
        lib.sparse_block_norm.argtypes = lib.sparse_block_norm_backward.argtypes = lib.sparse_rotary_heads.argtypes = [_vp, _vp]
        lib.sparse_rotary_heads_backward.argtypes = [_vp, _vp, _i64, _i64, _vp, _vp, _vp]
        lib.sparse_fp8_quantize.argtypes = [_vp] * 5 + [_i64] * 3 + [_i32, _vp]
        lib.sparse_fp8_gemm.argtypes = [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _i32, _i64, _i64, _i64, _vp]
        lib.sparse_fp8_linear.argtypes = [_vp] * 5 + [_i32, _i64, _i64, _i64, _vp]
        lib.sparse_fp8_linear_backward.argtypes = [_vp] * 6 + [_i32, _vp, _i64, _i64, _i64, _vp]

    def take(self):
        """The record since the last call: [thread, what, ...] each."""
        room = 1 << 16
        while True:
            buf = ctypes.create_string_buffer(room)
            need = self.hip.fake_take(buf, ctypes.c_size_t(room))
            if need <= room:
                return [[int(w) if w.isdigit() else w for w in line.split()] for line in buf.value.decode().splitlines()]
            room = need

    def error(self):
        return self.lib.sparse_attn_last_error().decode()

    # one call of each kind that keeps something in the stream's scratch memory
    def gemm(self, M, N, K, out=at(4), f32=0, a_block=0, b_block=1):
        return self.lib.sparse_fp8_gemm(at(0), at(1), a_block, at(2), at(3), b_block, None, out, f32, M, N, K, None)

    def linear(self, M, N, K):
        return self.lib.sparse_fp8_linear(at(0), at(1), at(2), None, at(3), 0, M, N, K, None)

    def linear_backward(self, M, N, K, dx=True, dw=True, db=True):
        return self.lib.sparse_fp8_linear_backward(at(0), at(1), at(2), at(3), at(4) if dx else None, at(5) if dw else None, 0, at(6) if db else None,
                                                   M, N, K, None)

    def norm_backward(self, rows, per, C, sums=("dweight", "dscale", "dshift", "dgate", "dpost_weight"), **kw):
        names = ("dh", "dx_out", "x_out", "y", "dx", "dy", "weight", "scale", "gate", "post_weight") + tuple(sums)
        args = {n: at(i) for i, n in enumerate(names)}
        args.update(rows=rows, rows_per_vector=per, scale_stride=C, gate_stride=C, channels=C, norm=1, x_dtype=0, vector_dtype=0, alpha=1.0, eps=1e-6, post_eps=1e-6)
        args.update(kw)
        return self.lib.sparse_block_norm_backward(ctypes.byref(self.block._NormBackwardArgs(**args)), None)

    def norm(self, rows, per, C, **kw):
        args = {n: at(i) for i, n in enumerate(("x", "y", "x_out", "h", "scale", "shift", "gate"))}
        args.update(rows=rows, rows_per_vector=per, scale_stride=C, shift_stride=C, gate_stride=C, channels=C, norm=1, alpha=1.0, eps=1e-6, post_eps=1e-6)
        args.update(kw)
        return self.lib.sparse_block_norm(ctypes.byref(self.block._NormArgs(**args)), None)

    def rotary_args(self, B, L, Hq, Hkv, D, weights=True, **kw):
        width = (Hq + 2 * Hkv) * D
        self.axes = (ctypes.c_int * 1)(D)
        args = {n: at(i) for i, n in enumerate(("qkv", "positions", "Q", "K", "V"))}
        args.update(axis_channels=ctypes.addressof(self.axes), B=B, L=L, heads_q=Hq, heads_kv=Hkv, D=D, axes=1, position_dtype=3, eps=1e-6, theta=100.0,
                    qkv_stride_b=L * width, qkv_stride_l=width)
        for t, H in zip("qkv", (Hq, Hkv, Hkv)):
            args.update({f"{t}_stride_b": H * L * D, f"{t}_stride_h": L * D, f"{t}_stride_l": D})
        if weights:
            args.update(q_weight=at(5), k_weight=at(6))
        args.update(kw)
        return self.block._RotaryArgs(**args)

    def rotary(self, *a, **kw):
        return self.lib.sparse_rotary_heads(ctypes.byref(self.rotary_args(*a, **kw)), None)

    def rotary_backward(self, B, L, Hq, Hkv, D):
        width = (Hq + 2 * Hkv) * D
        return self.lib.sparse_rotary_heads_backward(ctypes.byref(self.rotary_args(B, L, Hq, Hkv, D)), at(7), L * width, width, at(8), at(9), None)

    def release(self):
        return self.lib.sparse_attn_release_scratch(None)

    def attention(self, B, H, L, D):
        return self.lib.sparse_attn_fwd(at(0), at(1), at(2), at(3), at(4), None, at(5), B, H, L, D, 128, 128)

    def symbols(self, B, H, L, D):
        return self.lib.sparse_symbols_update(at(0), at(1), at(2), at(3), B, H, L, D, 128, 128, 0.5, 0.5, 0.5)


def threads(kind, sizes):
    """The record of one call of each size alone, and that of two threads with calls of one size each on the same stream."""
    lib = Library()
    call = getattr(lib, kind)
    alone = []
    for s in sizes:
        for _ in range(2):                # the second time the memory is there
            assert call(*s) == 0, lib.error()
            record = lib.take()
        alone.append(record)
    lib.lib.sparse_attn_release_scratch(None)
    lib.take()
    lib.hip.fake_delay(200)
    start = threading.Barrier(len(sizes))

    def many(s):
        start.wait()
        for _ in range(6):
            assert call(*s) == 0

    team = [threading.Thread(target=many, args=(s,)) for s in sizes]
    [t.start() for t in team]
    [t.join() for t in team]
    return alone, lib.take()


def rotary_views(cases):
    """For each case (sizes, and for Q, K, V the first element and the strides of batches, heads and tokens inside one tensor): 0 where
    the forward call takes it, else the message."""
    lib, out = Library(), []
    for sizes, views in cases:
        kw = {}
        for t, (first, b, h, l) in zip("qkv", views):
            kw.update({t.upper(): at(2) + 2 * first, f"{t}_stride_b": b, f"{t}_stride_h": h, f"{t}_stride_l": l})
        rc = lib.rotary(*sizes, **kw)
        out.append(lib.error() if rc else int(any(e[1] == "launch" for e in lib.take())) - 1)
    return out


def calls(cases):
    """[method, arguments, keywords] each: [return value, message, record]"""
    lib, out = Library(), []
    for kind, args, kw in cases:
        rc = getattr(lib, kind)(*args, **kw)
        out.append([rc, lib.error() if rc else "", [e[1:] for e in lib.take()]])
    return out


if __name__ == "__main__":
    print(json.dumps(globals()[sys.argv[1]](*json.load(sys.stdin))))
