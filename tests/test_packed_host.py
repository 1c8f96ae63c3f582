"""The packed cache's and the rotation's host code: refusals, lengths, and the arithmetic by which kernels find their work.  No GPU."""
import ctypes as C
import functools
import os
import random
import re
import subprocess
import tempfile

import pytest

from paper_2607_20125_b200 import packed

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "headcast.h")
INVALID, STATE, CUDA, UNSUPPORTED = -1, -2, -3, -5


@functools.lru_cache(maxsize=None)
def fake():
    """packed_api.cu on the CUDA runtime made for tests."""
    folder = tempfile.mkdtemp()
    path = os.path.join(folder, "packed_fake.so")
    cmd = [os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-cudart", "none", "-shared", "-Xcompiler", "-fPIC,-fno-gnu-unique", "-Xlinker", "-Bsymbolic",
           "-gencode", "arch=compute_100a,code=sm_100a", "-Xptxas", "-O0", "-std=c++17", "-o", path,
           os.path.join(NATIVE, "packed_on_fake_cuda.cu"), os.path.join(NATIVE, "fake_cuda.cpp")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    lib = C.CDLL(path)
    real = packed.load_library()
    for name in re.findall(r"\b(headcast_(?:packed|rope)[a-z_]*)\s*\(", re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)):
        getattr(lib, name).argtypes, getattr(lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    lib.fake_launches.restype = C.c_char_p
    for name, n in (("fake_walk_attention", 4), ("fake_walk_observe", 5)):
        getattr(lib, name).argtypes = [C.POINTER(C.c_int32)] + [C.c_int] * (n - 1) + [C.POINTER(C.c_int32), C.c_int64]
    return lib


BUFFER = C.create_string_buffer(1 << 20)
PTR = (C.addressof(BUFFER) + 255) & ~255


class Cache:
    def __init__(self, heads=4, kv=2, d=64, capacity=1000, scale=0.0):
        self.lib, self.cfg, self.ptr = fake(), packed.PackedConfig(heads, kv, d, capacity, scale), C.c_void_p()
        size = self.lib.headcast_packed_bytes(C.byref(self.cfg))
        self.storage = C.create_string_buffer(size + 256)
        self.at = (C.addressof(self.storage) + 255) & ~255
        assert self.lib.headcast_packed_create(C.byref(self.cfg), self.at, size, None, C.byref(self.ptr)) == 0

    def __getattr__(self, name):
        return lambda *a: getattr(self.lib, "headcast_packed_" + name)(self.ptr, *a)

    def lens(self):
        arr = (C.c_int32 * self.cfg.n_kv_heads)()
        assert self.lengths(arr) == 0
        return list(arr)

    def error(self):
        return self.lib.headcast_packed_last_error(self.ptr).decode()


def launches():
    names = fake().fake_launches().decode()
    fake().fake_clear_launches()
    return re.findall(r"\d+([a-z_]+_kernel)", names)


@pytest.mark.parametrize("cfg", [(0, 1, 64, 10), (65, 1, 64, 10), (4, 0, 64, 10), (4, 3, 64, 10), (4, 8, 64, 10), (4, 4, 96, 10), (4, 4, 64, 0),
                                 (4, 4, 64, (1 << 23) + 1), (4, 4, 64, 10, -1.0), (4, 4, 64, 10, float("nan")), (4, 4, 64, 10, 1e-20), (4, 4, 64, 10, float("inf"))])
def test_configurations_out_of_range(cfg):
    lib = packed.load_library()
    c = packed.PackedConfig(*cfg)
    assert lib.headcast_packed_bytes(C.byref(c)) == INVALID
    out = C.c_void_p(1)
    assert lib.headcast_packed_create(C.byref(c), PTR, 1 << 19, None, C.byref(out)) == INVALID and not out.value


def test_storage_size_and_alignment():
    lib = fake()
    c = packed.PackedConfig(4, 2, 128, 129, 0.0)
    rows = 2 * 256
    size = lib.headcast_packed_bytes(C.byref(c))
    assert size == 256 + rows * (64 + 64 + 8 + 8 + 4)
    out = C.c_void_p()
    for storage, n in ((None, size), (PTR + 16, size), (PTR, size - 1)):
        assert lib.headcast_packed_create(C.byref(c), storage, n, None, C.byref(out)) == INVALID and not out.value
    assert lib.headcast_packed_create(C.byref(c), PTR, size, None, None) == INVALID
    assert lib.headcast_packed_bytes(None) == INVALID and lib.headcast_packed_destroy(None) == 0
    assert lib.headcast_packed_last_error(None) == b"null cache"


def test_lengths_follow_appends_drops_and_evictions():
    c, other = Cache(), Cache(heads=2, capacity=400)
    launches()
    assert c.append(PTR, PTR, 600, 0, None) == 0 and c.lens() == [600, 600] and launches() == ["pack_rows_kernel"]
    assert c.append(PTR, PTR, 0, 0, None) == 0 and c.append(None, None, 0, 0, None) == 0 and launches() == []
    assert c.append(PTR, PTR, 401, 0, None) == STATE and c.lens() == [600, 600] and "no room" in c.error()
    assert c.drop_last(601) == STATE and c.drop_last(-1) == INVALID and c.drop_last(100) == 0 and c.lens() == [500, 500]
    keep = (C.c_int32 * 2)(300, 900)
    assert c.evict(other.ptr, keep, 0, 0, PTR, 500, None, 0, None) == STATE and other.lens() == [0, 0] and launches() == []
    keep[1] = 20
    assert c.evict(other.ptr, keep, 0, 0, PTR, 300, None, 0, None) == 0 and other.lens() == [300, 20] and c.lens() == [500, 500]
    assert launches() == ["evict_select_kernel", "evict_move_kernel"]
    assert other.append(PTR, PTR, 101, 0, None) == STATE and other.append(PTR, PTR, 100, 0, None) == 0 and other.lens() == [400, 120]
    assert other.drop_last(121) == STATE and other.lens() == [400, 120]
    keep[0] = keep[1] = 0
    assert c.evict(other.ptr, keep, 0, 0, PTR, 0, None, 0, None) == 0 and other.lens() == [0, 0]
    assert c.clear() == 0 and c.lens() == [0, 0]


def test_refusals():
    c, other = Cache(), Cache()
    assert c.append(PTR, PTR, 50, 0, None) == 0
    ws = c.workspace_bytes(8)
    keep = (C.c_int32 * 2)(5, 5)
    launches()
    bad = [
        (lambda: c.append(PTR + 2, PTR, 1, 0, None), "aligned"), (lambda: c.append(PTR, None, 1, 0, None), "aligned"),
        (lambda: c.append(PTR, PTR, -1, 0, None), "negative"), (lambda: c.append(PTR, PTR, 1, 127, None), "stride"), (lambda: c.append(PTR, PTR, 1, 132, None), "stride"),
        (lambda: c.append(PTR, PTR, 1, 1 << 31, None), "stride"),
        (lambda: c.export(0, -1, PTR, PTR, None), "range"), (lambda: c.export(-1, 5, PTR, PTR, None), "range"), (lambda: c.export(999, 2, PTR, PTR, None), "range"),
        (lambda: c.export(0, 5, PTR + 8, PTR, None), "aligned"),
        (lambda: c.attend(PTR, PTR, None, -1, PTR, ws, None), "range"), (lambda: c.attend(PTR, PTR, None, 1 << 30, PTR, ws, None), "range"),
        (lambda: c.attend(None, PTR, None, 8, PTR, ws, None), "aligned"), (lambda: c.attend(PTR, PTR + 8, None, 8, PTR, ws, None), "aligned"),
        (lambda: c.attend(PTR, PTR + 512, None, 8, PTR, ws, None), "overlaps"),
        (lambda: c.attend(PTR, PTR, C.c_void_p(PTR + 2), 8, PTR, ws, None), "aligned"),
        (lambda: c.attend(PTR, PTR, None, 8, PTR, ws - 1, None), "workspace"), (lambda: c.attend(PTR, PTR, None, 9, PTR, ws, None), "workspace"),
        (lambda: c.attend(PTR, PTR, None, 8, PTR + 16, ws, None), "workspace"), (lambda: c.attend(PTR, PTR, None, 8, None, ws, None), "workspace"),
        (lambda: c.observe(None, PTR, 8, 1.0, PTR, ws, None), "aligned"), (lambda: c.observe(PTR, None, 8, 1.0, PTR, ws, None), "aligned"),
        (lambda: c.observe(PTR, PTR, 8, -0.5, PTR, ws, None), "decay"), (lambda: c.observe(PTR, PTR, 8, float("nan"), PTR, ws, None), "decay"),
        (lambda: c.observe(PTR, PTR, 8, float("inf"), PTR, ws, None), "decay"), (lambda: c.observe(PTR, PTR, 8, 1.0, PTR, 16, None), "workspace"),
        (lambda: c.evict(c.ptr, keep, 0, 0, PTR, 5, None, 0, None), "another cache"), (lambda: c.evict(None, keep, 0, 0, PTR, 5, None, 0, None), "another cache"),
        (lambda: c.evict(other.ptr, None, 0, 0, PTR, 5, None, 0, None), "another cache"), (lambda: c.evict(other.ptr, keep, -1, 0, PTR, 5, None, 0, None), "negative"),
        (lambda: c.evict(other.ptr, keep, 0, -1, PTR, 5, None, 0, None), "negative"), (lambda: c.evict(other.ptr, (C.c_int32 * 2)(1, -1), 0, 0, PTR, 5, None, 0, None), "negative"),
        (lambda: c.evict(other.ptr, keep, 0, 0, PTR + 2, 5, None, 0, None), "index"), (lambda: c.evict(other.ptr, keep, 0, 0, PTR, 4, None, 0, None), "index"),
        (lambda: c.evict(other.ptr, keep, 0, 0, None, 0, PTR, 100, None), "workspace"),
        (lambda: c.evict(Cache(kv=1).ptr, keep, 0, 0, PTR, 5, None, 0, None), "other key/value heads"),
        (lambda: c.evict(Cache(d=128).ptr, keep, 0, 0, PTR, 5, None, 0, None), "head_dim"),
    ]
    for call, why in bad:
        assert call() == INVALID, why
        assert why in c.error(), (why, c.error())
    assert launches() == [] and c.lens() == [50, 50] and other.lens() == [0, 0]
    assert c.attend(None, None, None, 0, None, 0, None) == 0 and launches() == []  # no queries


def test_another_device_is_refused_everywhere():
    c, other = Cache(), Cache()
    c.append(PTR, PTR, 5, 0, None)
    launches()
    fake().cudaSetDevice(1)
    try:
        calls = (c.append(PTR, PTR, 5, 0, None), c.export(0, 5, PTR, PTR, None), c.attend(PTR, PTR, None, 1, PTR, 1 << 18, None), c.observe(PTR, PTR, 1, 1.0, PTR, 1 << 19, None),
                 c.evict(other.ptr, (C.c_int32 * 2)(1, 1), 0, 0, PTR, 5, None, 0, None), c.check(None))
        there = Cache()
    finally:
        fake().cudaSetDevice(0)
    assert calls == (INVALID,) * 6 and "device" in c.error() and launches() == []
    assert c.evict(there.ptr, (C.c_int32 * 2)(1, 1), 0, 0, PTR, 5, None, 0, None) == INVALID


def test_caches_in_the_same_storage_cannot_evict_into_each_other():
    c = Cache()
    c.append(PTR, PTR, 5, 0, None)
    twin = C.c_void_p()
    assert c.lib.headcast_packed_create(C.byref(c.cfg), c.at, c.lib.headcast_packed_bytes(C.byref(c.cfg)), None, C.byref(twin)) == 0
    assert c.evict(twin, (C.c_int32 * 2)(1, 1), 0, 0, PTR, 5, None, 0, None) == INVALID and "storage" in c.error()


def test_which_kernels_a_call_launches():
    c = Cache(heads=8, kv=2, capacity=5000)
    ws = C.create_string_buffer(64 << 20)
    at = (C.addressof(ws) + 255) & ~255
    launches()
    assert c.attend(PTR, PTR, None, 4, at, 60 << 20, None) == 0 and launches() == ["packed_merge_rows_kernel"]   # no tokens: zeros
    assert c.attend(PTR, PTR, None, 5, at, 60 << 20, None) == 0 and launches() == ["packed_empty_kernel"]
    assert c.observe(PTR, PTR, 5, 1.0, at, 60 << 20, None) == 0 and launches() == []
    c.append(PTR, PTR, 5000, 0, None)
    launches()
    assert c.attend(PTR, PTR, None, 4, at, 60 << 20, None) == 0 and launches() == ["packed_rows_kernel", "packed_merge_rows_kernel"]
    assert c.attend(PTR, PTR, None, 5, at, 60 << 20, None) == 0 and launches() == ["packed_attn_kernel", "packed_merge_kernel"]
    assert c.observe(PTR, PTR, 5, 1.0, at, 60 << 20, None) == 0 and launches() == ["packed_observe_kernel", "packed_observe_merge_kernel"]
    assert c.observe(PTR, PTR, 4, 1.0, at, 60 << 20, None) == 0 and launches() == ["packed_observe_rows_kernel"]
    assert c.observe(PTR, PTR, 0, 0.5, None, 0, None) == 0 and launches() == ["packed_decay_kernel"]
    assert c.observe(PTR, PTR, 0, 1.0, None, 0, None) == 0 and launches() == []


# ---------------------------------------------------------------------------------------------- how the work is dealt


def dealt(seed):
    rng = random.Random(seed)
    kv = rng.choice([1, 1, 2, 3, 5, 12, 64])
    most = rng.choice([1, 128, 129, 1000, 9000])
    return [rng.choice([0, 1, 127, 128, 129, rng.randint(0, most)]) for _ in range(kv)], rng


@pytest.mark.parametrize("seed", range(60))
def test_every_step_of_the_line_is_done_once_and_every_part_is_found(seed):
    lens, rng = dealt(seed)
    arr = (C.c_int32 * len(lens))(*lens)
    n_rows, n_sm = rng.choice([1, 17, 256, 257, 1000, 5000]), rng.choice([148, 148, 3, 1])
    total = sum(-(-n // 128) for n in lens) * -(-n_rows // 256)
    covered = (C.c_int32 * max(total, 1))()
    assert fake().fake_walk_attention(arr, len(lens), n_rows, n_sm, covered, total) == min(n_sm, total) and all(n == 1 for n in covered[:total])
    group, q_tiles = rng.choice([1, 2, 4]), rng.choice([1, 2, 7, 40])
    total = sum(-(-n // 256) for n in lens) * group * q_tiles
    covered = (C.c_int32 * max(total, 1))()
    assert fake().fake_walk_observe(arr, len(lens), group, q_tiles, n_sm, covered, total) == min(n_sm, total) and all(n == 1 for n in covered[:total])
    total = sum(-(-n // 128) for n in lens)
    assert fake().fake_walk_rows(arr, len(lens), n_sm) == min(n_sm, total)


# ---------------------------------------------------------------------------------------------- rotation


def rope(n=4, q=PTR, q_out=PTR + 65536, qs=0, k=None, k_out=None, ks=0, first=0, pos=None, **kw):
    lib = packed.load_library()
    cfg = packed.RopeConfig()
    lib.headcast_rope_default_config(C.byref(cfg))
    for name, value in {**dict(n_heads=2, n_kv_heads=1, head_dim=64, grid_h=2, grid_w=2, dim_t=24, dim_h=20, dim_w=20), **kw}.items():
        setattr(cfg, name, value)
    rc = lib.headcast_rope(C.byref(cfg), q, q_out, qs, k, k_out, ks, n, first, pos, 0, None)
    return rc, lib.headcast_rope_last_error().decode()


def test_rotation_refusals():
    inf = float("inf")
    for kw, why in [(dict(head_dim=96), "head_dim"), (dict(n_heads=0), "heads"), (dict(n_heads=65), "heads"), (dict(dim_t=23), "even"), (dict(dim_w=-2), "even"),
                    (dict(dim_t=26), "together"), (dict(dim_t=0, dim_h=0, dim_w=0), "together"), (dict(theta=0.0), "theta"), (dict(theta=float("nan")), "theta"),
                    (dict(scale_h=inf), "finite"), (dict(grid_w=0), "grid"), (dict(grid_h=1 << 16, grid_w=1 << 16), "grid"), (dict(n=-1), "negative"), (dict(first=(1 << 31) + 1), "first_frame"),
                    (dict(k=PTR + 4096), "belong"), (dict(k=PTR + 4096, k_out=PTR + 8192, n_kv_heads=0), "belong"), (dict(q=PTR + 8), "aligned"), (dict(q_out=None), "aligned"),
                    (dict(pos=PTR + 2), "aligned"), (dict(qs=127), "stride"), (dict(qs=132), "stride"), (dict(q_out=PTR + 256), "overlaps"), (dict(q_out=PTR, qs=256), "overlaps"),
                    (dict(k=PTR + 4096, k_out=PTR + 65536 + 512), "outputs overlap"), (dict(k=PTR + 4096, k_out=PTR + 512), "overlaps"),
                    (dict(theta=1e-300, dim_t=44, dim_h=0, scale_t=1e300), "finite")]:
        rc, error = rope(**kw)
        assert rc == INVALID and why in error, (kw, rc, error)
    rc, error = rope(halves=1, dim_t=20)
    assert rc == UNSUPPORTED and "16" in error
    assert rope(n=0, q=None, q_out=None)[0] == 0


def test_outputs_that_overlap_smaller_inputs_and_outputs():
    c = Cache()
    assert c.append(PTR, PTR, 50, 0, None) == 0
    launches()
    ws, q_bytes = c.workspace_bytes(8), 8 * 4 * 64 * 2
    for lse in (PTR, PTR + q_bytes - 4, PTR + 65536 - 4, PTR + 65536 + q_bytes - 4):
        assert c.attend(PTR, PTR + 65536, C.c_void_p(lse), 8, PTR + 131072, ws, None) == INVALID and "lse overlaps" in c.error()
    assert launches() == []
    assert c.attend(PTR, PTR + 65536, C.c_void_p(PTR + q_bytes), 8, PTR + 131072, ws, None) == 0
    rc, error = rope(pos=PTR + 65536 + 4)
    assert rc == INVALID and "positions" in error
