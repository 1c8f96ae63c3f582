"""The packed cache's and the rotation's host code at the limits of what its calls take.  No GPU."""
import ctypes as C
import decimal
import functools
import os
import subprocess
import tempfile

import pytest

from paper_2607_20125_b200 import packed
from test_packed_host import INVALID, PTR, Cache, launches

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")


@pytest.mark.parametrize("scale", [1e-60, -1e-60, 2.0 ** -151, 5e-324])
def test_a_scale_that_a_c_float_cannot_hold_is_not_taken_for_the_default(scale):
    with pytest.raises(ValueError, match="softmax_scale"):
        packed.PackedCache(4, 64, 100, softmax_scale=scale)


@pytest.mark.parametrize("scale", [1e-20, 2.0 ** -41, 2.0 ** 41, -1.0, 1e60, float("nan"), float("inf")])
def test_scales_out_of_range_are_refused(scale):
    with pytest.raises(packed.HeadCastError, match="softmax_scale"):
        packed.PackedCache(4, 64, 100, softmax_scale=scale)


# ---------------------------------------------------------------------------------------------- arguments that overlap


def test_arguments_that_overlap_each_other_or_a_cache():
    c, other = Cache(), Cache()
    assert c.append(PTR, PTR, 50, 0, None) == 0
    lib, size = c.lib, c.lib.headcast_packed_bytes(C.byref(c.cfg))
    end = c.at + size
    arena = C.create_string_buffer(c.workspace_bytes(8) + (1 << 20))
    q = (C.addressof(arena) + 255) & ~255
    q_bytes, lse_bytes, ws = 8 * 4 * 64 * 2, 8 * 4 * 4, c.workspace_bytes(8)
    out, lse, at = q + 65536, q + 131072, q + 262144
    keep = (C.c_int32 * 2)(5, 5)
    packed_row = 2 * 64 * 2  # one token's keys, or values
    launches()
    for call in (lambda: c.append(c.at, PTR, 1, 0, None), lambda: c.append(PTR, end - 16, 1, 0, None), lambda: c.append(PTR, (c.at - packed_row + 16), 1, 0, None),
                 lambda: c.append(c.at - 2 * (3 * 256 + 128) + 16, PTR, 4, 256, None),
                 lambda: c.export(0, 5, c.at, None, None), lambda: c.export(0, 5, None, end - 16, None), lambda: c.export(0, 5, q, q + 5 * packed_row - 16, None),
                 lambda: c.export(0, 5, q, q, None),
                 lambda: c.attend(q, end - 16, None, 8, at, ws, None), lambda: c.attend(q, out, C.c_void_p(c.at + 256), 8, at, ws, None),
                 lambda: c.attend(q, out, None, 8, c.at, ws, None), lambda: c.attend(q, out, None, 8, q, ws, None), lambda: c.attend(q, out, None, 8, out, ws, None),
                 lambda: c.attend(at + ws - 16, out, None, 8, at, ws, None), lambda: c.attend(q, at + ws - 16, None, 8, at, ws, None),
                 lambda: c.attend(q, out, C.c_void_p(at + ws - 4), 8, at, ws, None), lambda: c.attend(q, out, C.c_void_p(at - lse_bytes + 4), 8, at, ws, None),
                 lambda: c.observe(c.at + 256, lse, 8, 1.0, at, ws, None), lambda: c.observe(q, end - 4, 8, 1.0, at, ws, None), lambda: c.observe(q, lse, 8, 1.0, c.at, ws, None),
                 lambda: c.observe(at + ws - 16, lse, 8, 1.0, at, ws, None), lambda: c.observe(q, at + ws - 4, 8, 1.0, at, ws, None),
                 lambda: c.evict(other.ptr, keep, 0, 0, c.at, 5, None, 0, None), lambda: c.evict(other.ptr, keep, 0, 0, other.at + size - 4, 5, None, 0, None),
                 lambda: c.evict(other.ptr, keep, 0, 0, other.at - 36, 5, None, 0, None), lambda: c.evict(other.ptr, keep, 0, 0, None, 0, other.at, 1 << 20, None),
                 lambda: c.evict(other.ptr, keep, 0, 0, None, 0, c.at, 1 << 20, None)):
        assert call() == INVALID and "overlaps" in c.error(), c.error()
    assert launches() == [] and c.lens() == [50, 50] and other.lens() == [0, 0]
    # side by side
    for call in (lambda: c.append(PTR, end, 1, 0, None), lambda: c.append(c.at - packed_row, PTR, 1, 0, None), lambda: c.export(0, 5, q, q + 5 * 2 * packed_row // 2, None),
                 lambda: c.attend(at - q_bytes, at + ws, C.c_void_p(at + ws + q_bytes), 8, at, ws + 4096, None),  # a larger workspace is touched as far as it is needed
                 lambda: c.attend(q, q, None, 8, at, ws, None), lambda: c.attend(c.at + 256, out, None, 8, at, ws, None),  # reads its cache, writes elsewhere
                 lambda: c.observe(at + ws, at - lse_bytes, 8, 1.0, at, ws, None), lambda: c.evict(other.ptr, keep, 0, 0, other.at - 40, 5, None, 0, None),
                 lambda: c.evict(other.ptr, keep, 0, 0, other.at + size, 5, None, 0, None)):
        assert call() == 0, c.error()
    none = (C.c_int32 * 2)(0, 0)
    assert c.evict(other.ptr, none, 0, 0, other.at, 0, None, 0, None) == 0  # writes no index


# ---------------------------------------------------------------------------------------------- a rotation's frequencies


@functools.lru_cache(maxsize=None)
def rotation(*flags):
    """packed_api.cu on the CUDA runtime made for tests, and what its rotation hands to the kernel."""
    path = os.path.join(tempfile.mkdtemp(), "rope_fake.so")
    cmd = [os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-cudart", "none", "-shared", "-Xcompiler", ",".join(("-fPIC", "-fno-gnu-unique") + flags), "-Xlinker", "-Bsymbolic",
           "-gencode", "arch=compute_100a,code=sm_100a", "-Xptxas", "-O0", "-std=c++17", "-o", path,
           os.path.join(NATIVE, "rope_on_fake_cuda.cu"), os.path.join(NATIVE, "fake_cuda.cpp")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    lib = C.CDLL(path)
    real = packed.load_library()
    for name in ("headcast_rope_default_config", "headcast_rope", "headcast_rope_last_error"):
        getattr(lib, name).argtypes, getattr(lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    lib.fake_frequencies.argtypes, lib.fake_frequencies.restype = [C.POINTER(C.c_uint64)], C.c_int
    return lib


def frequencies(lib, dims, theta, scales, inverse=0, n=4):
    cfg = packed.RopeConfig()
    lib.headcast_rope_default_config(C.byref(cfg))
    cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.grid_h, cfg.grid_w, cfg.theta = 2, 2, 128, 2, 2, theta
    cfg.dim_t, cfg.dim_h, cfg.dim_w = dims
    cfg.scale_t, cfg.scale_h, cfg.scale_w = scales
    buffer = C.create_string_buffer(4096 + 512 * n)
    rc = lib.headcast_rope(C.byref(cfg), C.addressof(buffer) & ~15, (C.addressof(buffer) + 2048 + 256 * n) & ~15, 0, None, None, 0, n, 0, None, inverse, None)
    assert rc == 0, lib.headcast_rope_last_error()
    out = (C.c_uint64 * 64)()
    assert lib.fake_frequencies(out) == sum(dims) // 2
    return out[: sum(dims) // 2]


CONFIGURATIONS = [((44, 42, 42), 1e4, (1.0, 1.0, 1.0)), ((44, 42, 42), 500.0, (0.25, 1.0, 3.7)), ((128, 0, 0), 1e6, (1.0, 1.0, 1.0)), ((2, 4, 6), 256.0, (1.0, -1.0, -0.3)),
                  ((64, 32, 32), 1.0, (1.0, 6.2831853, 100.0)), ((42, 42, 44), 0.1, (1.0, 0.0, -7.0)), ((2, 62, 64), 1.0000001, (1e-3, 1e-9, 12.5)),
                  ((44, 42, 42), 1e300, (1.0, 1e-300, 1e18)), ((4, 8, 16), 1e-12, (1e-3, 1.0, 1.0)), ((10, 20, 30), 3.0000000000000004, (1.0, 1.0, 1.0)), ((8, 0, 8), 65536.0, (0.5, 1.0, 2.0 ** -40))]


@pytest.mark.parametrize("flags", [(), ("-mlong-double-64",)], ids=["", "64-bit long double"])
@pytest.mark.parametrize("dims,theta,scales", CONFIGURATIONS)
def test_frequencies_are_those_of_exact_arithmetic(flags, dims, theta, scales):
    """On a host whatever its long double is.  In units of u = 2^-64, relative: the constant and the first product are rounded (1 u each); theta r^n is
    off by n u (a power's error doubles with a square, which adds u), the root by an n-th of that, and by 2 u where its correction is cut to whole units;
    every product adds u.  The j-th frequency is off by (2 + 4 j) u of itself, and by less than 2^-64 turns where it is cut."""
    lib = rotation(*flags)
    got = frequencies(lib, dims, theta, scales)
    with decimal.localcontext() as ctx:
        ctx.prec = 80
        pi, i = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798"), 0
        for width, scale in zip(dims, scales):
            for j in range(width // 2):
                turns = decimal.Decimal(scale) / (2 * pi) * decimal.Decimal(theta) ** (decimal.Decimal(-2 * j) / width)
                off = (got[i] - turns * 2 ** 64) % (1 << 64)
                bound = (2 + 4 * j) * abs(turns) * decimal.Decimal("1.001") + 1
                assert min(off, (1 << 64) - off) <= bound, (width, scale, j, turns, off)
                i += 1
    back = frequencies(lib, dims, theta, scales, inverse=1)
    assert all((a + b) % (1 << 64) == 0 for a, b in zip(got, back))


# ---------------------------------------------------------------------------------------------- nothing to do


def test_calls_without_tokens_need_no_addresses():
    """The address of an empty tensor is null."""
    lib = packed.load_library()
    cfg = packed.RopeConfig()
    lib.headcast_rope_default_config(C.byref(cfg))
    cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.dim_t = 2, 2, 64, 64  # no grid: positions are given
    assert lib.headcast_rope(C.byref(cfg), None, None, 0, None, None, 0, 0, 0, None, 0, None) == 0
    assert lib.headcast_rope(C.byref(cfg), PTR, PTR, 0, None, None, 0, 1, 0, None, 0, None) == INVALID and b"grid" in lib.headcast_rope_last_error()
    c, other = Cache(), Cache()
    assert other.append(PTR, PTR, 7, 0, None) == 0
    none = (C.c_int32 * 2)(0, 0)
    launches()
    for keep in (none, (C.c_int32 * 2)(9, 9)):  # the cache is empty
        assert c.evict(other.ptr, keep, 0, 0, None, 0, None, 0, None) == 0 and other.lens() == [0, 0], c.error()
        assert other.append(PTR, PTR, 7, 0, None) == 0
    assert other.evict(c.ptr, none, 0, 0, None, 0, None, 0, None) == 0 and c.lens() == [0, 0] and other.lens() == [7, 7]
    assert other.evict(c.ptr, (C.c_int32 * 2)(0, 1), 0, 0, None, 0, None, 0, None) == INVALID and "workspace" in other.error()
    assert "evict_select_kernel" not in launches()
