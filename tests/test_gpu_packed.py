"""GPU: the key/value cache held in 4 bits - packing, attention, accumulated weights, eviction - against the definitions in 64 bits."""
import pytest

import packed_reference as ref

pytestmark = pytest.mark.gpu


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, scale=1.0):
    import torch
    return (scale * torch.randn(*shape, device="cuda", generator=g)).bfloat16()


def make(heads, kv, d, capacity, k=None, v=None, **kw):
    from paper_2607_20125_b200.packed import PackedCache
    cache = PackedCache(heads, d, capacity, n_kv_heads=kv, **kw)
    if k is not None:
        cache.append(k, v)
    return cache


def per_head(x):
    return [h for h in ref.held(x.transpose(0, 1))]


# ---------------------------------------------------------------------------------------------- packing


def awkward(g, n, kv, d):
    """Rows in which scales of every size and all their mantissas meet elements on, and next to, the borders between codes."""
    import torch
    x = torch.randn(n, kv, d, device="cuda", generator=g) * torch.exp2(torch.randint(-30, 24, (n, kv, d // 16, 1), device="cuda", generator=g).float()).expand(
        n, kv, d // 16, 16).reshape(n, kv, d)
    x = x.bfloat16()
    groups = x.view(n, kv, d // 16, 16)
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 0.0, -0.0], device="cuda")
    for m in range(8):
        for e in (-21, -19, -3, 0, 7, 12, 13):
            i = (8 * (e + 21) + m) % (n * kv)
            s = (1 + m / 8) * 2.0 ** e
            row = torch.cat((6 * s * torch.ones(1, device="cuda"), s * borders * (1 if m % 2 else -1))).bfloat16()
            groups[i % n, i // n % kv, (m + e) % (d // 16)] = row
    special = [float("nan"), float("inf"), float("-inf"), 0.0, 3e38, -1e-40, 2.0 ** -133]
    for j, value in enumerate(special):
        groups[(5 * j + 1) % n, j % kv, j % (d // 16), j % 16] = value
    groups[n // 2, 0, 0] = 0.0
    groups[n // 3, 0, 0] = float("nan")
    return x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,kv", [(1, 1), (1, 3), (31, 2), (33, 3), (130, 1), (700, 2)])
def test_held_values_are_those_of_exact_arithmetic(d, n, kv):
    import torch
    g = gen(n + d)
    k, v = awkward(g, n, kv, d), awkward(g, n, kv, d)
    cache = make(kv, kv, d, n, k, v)
    got_k, got_v = cache.export()
    assert torch.equal(got_k.double(), ref.held(k.transpose(0, 1))) and torch.equal(got_v.double(), ref.held(v.transpose(0, 1)))
    assert (cache.weights == 0).all() and cache.lengths() == [n] * kv


def test_appends_of_any_size_and_stride_and_dropped_tokens():
    import torch
    g = gen(1)
    fused = randn(g, 300, 9, 64)
    k, v = fused[:, 3:6], fused[:, 6:]
    whole = make(3, 3, 64, 300, k.contiguous(), v.contiguous())
    cache = make(3, 3, 64, 300)
    at = 0
    for n in (1, 2, 126, 1, 64, 7, 99):
        cache.append(k[at:at + n], v[at:at + n])
        cache.append(v[at:at + n][: 300 - at - n], k[at:at + n][: 300 - at - n])  # taken back
        cache.drop_last(min(n, 300 - at - n))
        at += n
        assert cache.lengths() == [at] * 3
    for a, b in zip(whole.export(), cache.export()):
        assert torch.equal(a, b)
    for a, b in zip(whole.export(first=100, n_tokens=33), cache.export()):
        assert torch.equal(a, b[:, 100:133])


def test_export_leaves_rows_behind_the_last_token():
    import ctypes as C
    import torch
    g = gen(2)
    cache = make(2, 2, 64, 200, randn(g, 50, 2, 64), randn(g, 50, 2, 64))
    out = torch.full((2, 70, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    assert cache.lib.headcast_packed_export(cache._ptr, 0, 70, out.data_ptr(), None, torch.cuda.current_stream().cuda_stream) == 0
    assert (out[:, 50:] == 7.0).all() and not (out[:, :50] == 7.0).all()


# ---------------------------------------------------------------------------------------------- attention


def attend(cache, q, with_lse=True):
    import torch
    out = torch.full_like(q, 99.0)
    lse = torch.full((q.shape[1], q.shape[0]), 99.0, device="cuda") if with_lse else None
    cache.attend(q, out, lse)
    cache.check()
    return out, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(3, 3), (4, 1), (6, 2)])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 127, 128, 129, 257, 700])
def test_ragged_queries_and_tokens(d, heads, kv, n):
    g = gen(n * d + heads)
    k, v = randn(g, n, kv, d, scale=1.5), randn(g, n, kv, d)
    cache = make(heads, kv, d, n + 3, k, v)
    hk, hv = per_head(k), per_head(v)
    for n_q in (1, 2, 4, 5, 16, 17, 64, 65, 128, 129, 257):
        q = randn(g, n_q, heads, d, scale=1.5)
        out, lse = attend(cache, q, with_lse=n_q != 2 and n_q != 129)
        ref.check_attend(out, lse, q, hk, hv)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv,n_q,n", [
    (1, 1, 1, 40000), (1, 1, 16, 20000),         # one head over all SMs: 148 parts of its rows
    (2, 1, 10, 33333), (1, 1, 200, 25000),       # one pair of query tiles in 148 parts
    (5, 5, 130, 9000), (3, 1, 700, 5000),        # pairs in about thirty and ten parts
    (12, 12, 600, 1500), (16, 4, 77, 10007), (64, 64, 3, 513), (40, 40, 300, 129),
])
def test_cut_ranges(d, heads, kv, n_q, n):
    g = gen(n)
    k, v = randn(g, n, kv, d), randn(g, n, kv, d)
    # every tile holds a token that draws some row far above the average: a lost part changes that row
    q = randn(g, n_q, heads, d)
    rows = q[:, :: heads // kv].double()
    for tile in range(0, n, 128):
        row = rows[tile // 128 % n_q]
        k[tile + 37 % min(128, n - tile)] += (10.0 * d ** 0.5 * row / row.square().sum(-1, keepdim=True)).bfloat16()
    cache = make(heads, kv, d, n, k, v)
    out, lse = attend(cache, q)
    ref.check_attend(out, lse, q, per_head(k), per_head(v))


@pytest.mark.parametrize("n_q", [1, 40, 300])
def test_heads_of_different_lengths_and_none(n_q):
    """Lengths as evictions leave them, zero among them."""
    import torch
    g = gen(n_q)
    heads, kv, d, n = 10, 5, 128, 900
    k, v = randn(g, n, kv, d), randn(g, n, kv, d)
    cache = make(heads, kv, d, n, k, v)
    other = make(heads, kv, d, n)
    for keep in ([0, 900, 1, 0, 129], [128, 0, 0, 500, 0], [0, 0, 0, 0, 1], [0] * 5):
        cache.evict_into(other, keep, n_first=n)  # the first ones
        assert other.lengths() == keep
        q = randn(g, n_q, heads, d)
        out, lse = attend(other, q)
        hk, hv = per_head(k), per_head(v)
        ref.check_attend(out, lse, q, [x[:m] for x, m in zip(hk, keep)], [x[:m] for x, m in zip(hv, keep)])
        none = torch.tensor(keep, device="cuda").repeat_interleave(2) == 0
        assert (out[:, none] == 0).all() and (lse[none] == -torch.inf).all()


@pytest.mark.parametrize("n_q", [3, 150])
def test_rows_of_any_size_and_rows_that_are_not_finite(n_q):
    import torch
    g = gen(6)
    heads, d, n = 2, 64, 300
    k, v = randn(g, n, heads, d), randn(g, n, heads, d)
    cache = make(heads, heads, d, n, k, v)
    hk, hv = per_head(k), per_head(v)
    for scale in (0.0, 1e-38, 1e-20, 1e-6, 30.0, 3000.0):
        q = randn(g, n_q, heads, d, scale=scale)
        q[:, :, 5] *= 1e-3  # elements far below their row's largest
        out, lse = attend(cache, q)
        ref.check_attend(out, lse, q, hk, hv)
    q = randn(g, n_q, heads, d)
    bad = q.clone()
    bad[0, 0, 3], bad[1, 1, 60], bad[2, 0, 0] = float("nan"), float("inf"), float("-inf")
    good, good_lse = attend(cache, q)
    out, lse = attend(cache, bad)
    rows = torch.zeros(n_q, heads, dtype=torch.bool, device="cuda")
    rows[0, 0] = rows[1, 1] = rows[2, 0] = True
    assert torch.isnan(out[rows].float()).all() and torch.isnan(lse.T[rows]).all()
    assert torch.equal(out[~rows], good[~rows]) and torch.equal(lse.T[~rows], good_lse.T[~rows])


@pytest.mark.parametrize("n_q", [2, 150])
def test_logits_of_any_size(n_q):
    """Up to the limit rows are as exact as their logits; a row beyond it is NaN, whichever way its logits point, and no other."""
    import torch
    g = gen(14)
    n, d = 700, 64
    k, v, q = randn(g, n, 2, d), randn(g, n, 2, d), randn(g, n_q, 2, d)
    hk, hv = per_head(k), per_head(v)
    for scale in (2.0 ** -30, 1.0, 2.0 ** 10):
        cache = make(2, 2, d, n, k, v, softmax_scale=scale)
        out, lse = attend(cache, q)
        ref.check_attend(out, lse, q, hk, hv, scale)
    cache = make(2, 2, d, n, k, v, softmax_scale=1.0)
    far = q.clone()
    far[0, 0] *= 1e9
    near, near_lse = attend(cache, q)
    out, lse = attend(cache, far)
    assert torch.isnan(out[0, 0].float()).all() and torch.isnan(lse[0, 0])
    assert torch.equal(out[1:], near[1:]) and torch.equal(out[:, 1], near[:, 1]) and torch.equal(lse[1], near_lse[1])
    down = make(2, 2, d, n, k.abs(), v, softmax_scale=1.0)
    far[0, 0] = -far[0, 0].abs()
    out, lse = attend(down, far)
    assert torch.isnan(out[0, 0].float()).all() and torch.isfinite(out[1:].float()).all()


@pytest.mark.parametrize("n_q", [3, 150, 700])
def test_output_in_place_of_the_queries(n_q):
    import torch
    from paper_2607_20125_b200.binding import HeadCastError
    g = gen(15)
    k, v, q = randn(g, 3000, 2, 128), randn(g, 3000, 2, 128), randn(g, n_q + 1, 4, 128)
    cache = make(4, 2, 128, 3000, k, v)
    out, lse = attend(cache, q[:n_q])
    both = q.clone()
    again = torch.empty_like(lse)
    cache.attend(both[:n_q], both[:n_q], again)
    assert torch.equal(both[:n_q], out) and torch.equal(again, lse) and torch.equal(both[n_q:], q[n_q:])
    with pytest.raises(HeadCastError) as e:
        cache.attend(both[:n_q], both[1:], again)
    assert e.value.code == -1


@pytest.mark.parametrize("n_q", [3, 700])
def test_a_kernel_that_gave_up_is_reported_once(n_q):
    """As if a bounded wait of an earlier call had expired: its status word stands in the storage."""
    import torch
    from paper_2607_20125_b200.binding import HeadCastError
    g = gen(16)
    k, v, q = randn(g, 3000, 2, 128), randn(g, 3000, 2, 128), randn(g, n_q, 2, 128)
    cache = make(2, 2, 128, 3000, k, v)
    out, lse = attend(cache, q)
    cache.storage[:4].view(torch.int32).fill_(77)
    cache.attend(q, torch.empty_like(q), torch.empty_like(lse))
    with pytest.raises(HeadCastError) as e:
        cache.check()
    assert e.value.code == -6 and "77" in str(e.value)
    cache.check()
    again, again_lse = attend(cache, q)
    assert torch.equal(again, out) and torch.equal(again_lse, lse)


def test_first_calls_of_a_process_inside_a_capture():
    import subprocess
    import sys
    code = """
import torch
from paper_2607_20125_b200.packed import PackedCache, Rope
caches = [PackedCache(2, 64, 600) for _ in range(2)]
k, v, q, one = (torch.randn(n, 2, 64, device="cuda").bfloat16() for n in (500, 500, 300, 1))
outs = [torch.empty_like(q), torch.empty(2, 300, device="cuda"), torch.empty_like(one), torch.empty(2, 1, device="cuda")]
def calls():
    Rope(2, 64, 10, 10, dims=(24, 20, 20)).apply(q, outs[0])
    caches[0].clear()
    caches[0].append(k, v)
    caches[0].attend(q, outs[0], outs[1])
    caches[0].attend(one, outs[2], outs[3])
    caches[0].observe(q, outs[1], decay=0.0)
    caches[0].evict_into(caches[1], 200)
    return [o.clone() for o in outs] + [caches[0].weights.clone()] + list(caches[1].export())
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    captured = calls()
graph.replay()
torch.cuda.synchronize()
captured = [c.clone() for c in captured]
assert all(torch.equal(a, b) for a, b in zip(captured, calls()))
print("same")
"""
    import os
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=200, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert res.returncode == 0 and "same" in res.stdout, res.stdout + res.stderr


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [5, 200])
def test_row_maximum_grows_and_falls(d, n_q):
    import torch
    g = gen(7)
    n = 128 * 6 + 5
    u = torch.nn.functional.normalize(torch.randn(1, 2, d, device="cuda", generator=g), dim=-1)
    q, k, v = (torch.randn(m, 2, d, device="cuda", generator=g) for m in (n_q, n, n))
    steps = torch.tensor([0.0, 1.0, 0.3, 2.0, 2.9, 2.9, 2.5], device="cuda")[torch.arange(n, device="cuda") // 128]
    sign = torch.tensor([1.0, -1.0, 0.0], device="cuda")[torch.arange(n_q, device="cuda") % 3]
    q = (q + 12.0 * d ** 0.25 * sign[:, None, None] * u).bfloat16()
    k = (k + 1.1 * d ** 0.25 * steps[:, None, None] * u).bfloat16()
    v = v.bfloat16()
    out, lse = attend(make(2, 2, d, n, k, v), q)
    ref.check_attend(out, lse, q, per_head(k), per_head(v))


@pytest.mark.parametrize("n_q", [2, 90])
@pytest.mark.parametrize("scale", [2.0 ** -40, 0.01, 2.0])
def test_other_softmax_scales(n_q, scale):
    g = gen(8)
    k, v, q = randn(g, 333, 2, 128), randn(g, 333, 2, 128), randn(g, n_q, 2, 128)
    out, lse = attend(make(2, 2, 128, 333, k, v, softmax_scale=scale), q)
    ref.check_attend(out, lse, q, per_head(k), per_head(v), scale)


@pytest.mark.parametrize("n_q", [1, 200])
def test_offsets_beyond_32_bits(n_q):
    """Ten heads of 2^23 tokens of room: the last one's keys begin 4.8 GB into their plane."""
    g = gen(9)
    k, v, q = randn(g, 131, 10, 128), randn(g, 131, 10, 128), randn(g, n_q, 10, 128)
    cache = make(10, 10, 128, 1 << 23, k, v)
    out, lse = attend(cache, q)
    ref.check_attend(out, lse, q, per_head(k), per_head(v))
    cache.observe(q, lse, decay=0.0)
    for (w, err), got in zip(ref.observe(q, lse, per_head(k)), cache.weights.double()):
        assert ((got - w).abs() <= err + 2.0 ** -22 * w).all()


def test_results_do_not_vary_between_calls_streams_and_replays():
    import torch
    g = gen(10)
    cases = []
    for heads, kv, n_q, n in ((12, 12, 1, 5000), (4, 1, 3, 9000), (3, 3, 500, 3000), (2, 1, 140, 700)):
        k, v, q = randn(g, n, kv, 128), randn(g, n, kv, 128), randn(g, n_q, heads, 128)
        cache = make(heads, kv, 128, n, k, v)
        out, lse = attend(cache, q)
        cache.observe(q, lse, decay=0.0)
        cases.append((cache, q, out, lse, cache.weights.clone()))
    torch.cuda.synchronize()
    # two streams at once, each with workspaces of its own
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for i, stream in enumerate(streams):
        with torch.cuda.stream(stream):
            for _ in range(4):
                for cache, q, out, lse, _ in (cases if i else reversed(cases)):
                    o, l = torch.empty_like(out), torch.empty_like(lse)
                    cache.attend(q, o, l)
                    results.append((o, l, out, lse))
    torch.cuda.synchronize()
    assert all(torch.equal(o, out) and torch.equal(l, lse) for o, l, out, lse in results)
    # two captured graphs, replayed with calls between
    graphs = []
    for cache, q, out, lse, weights in cases:
        o, l, graph = torch.empty_like(out), torch.empty_like(lse), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(q, o, l)
            cache.observe(q, l, decay=0.0)
        graphs.append((graph, o, l))
    for (graph, o, l), (cache, q, out, lse, weights) in list(zip(graphs, cases)) * 2:
        o.fill_(0)
        cache.weights.fill_(5.0)
        graph.replay()
        other = cases[0]
        other[0].attend(other[1], torch.empty_like(other[2]))
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(cache.weights, weights)


@pytest.mark.parametrize("heads,kv,n_q,n,d", [(12, 12, 300, 4000, 64), (16, 4, 77, 10007, 64), (12, 12, 300, 4000, 128), (12, 12, 512, 4000, 128), (12, 12, 1, 9000, 128),
                                              (4, 1, 4, 9000, 64)])
def test_the_same_call_again_and_again(heads, kv, n_q, n, d):
    """Rings of shared memory whose slots are filled again while others are read: every one of many calls gives the same bits."""
    import torch
    g = gen(n)
    k, v, q = randn(g, n, kv, d), randn(g, n, kv, d), randn(g, n_q, heads, d)
    cache = make(heads, kv, d, n, k, v)
    out, lse = attend(cache, q)
    ref.check_attend(out, lse, q, per_head(k), per_head(v))
    cache.observe(q, lse, decay=0.0)
    weights = cache.weights.clone()
    for wait in (False, True):
        results = []
        for _ in range(100):
            o, l = torch.empty_like(out), torch.empty_like(lse)
            cache.attend(q, o, l)
            cache.observe(q, l, decay=0.0)
            results.append((o, l, cache.weights.clone()))
            if wait:
                torch.cuda.synchronize()
        assert all(torch.equal(o, out) and torch.equal(l, lse) and torch.equal(w, weights) for o, l, w in results)


# ---------------------------------------------------------------------------------------------- accumulated weights


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv,n_q,n", [(2, 2, 1, 1), (3, 3, 1, 300), (4, 1, 2, 1000), (4, 2, 5, 129), (2, 2, 16, 2000), (12, 3, 4, 40000), (2, 2, 17, 131), (4, 2, 127, 128), (4, 1, 128, 129), (2, 2, 129, 256), (6, 2, 300, 257), (1, 1, 2000, 700),
                                            (12, 12, 500, 1600), (1, 1, 33, 60000)])
def test_weights(d, heads, kv, n_q, n):
    import torch
    g = gen(n * 3 + d)
    k, v, q = randn(g, n, kv, d, scale=1.5), randn(g, n, kv, d), randn(g, n_q, heads, d, scale=1.5)
    cache = make(heads, kv, d, n + 5, k, v)
    _, lse = attend(cache, q)
    want = ref.observe(q, lse, per_head(k))
    total = torch.zeros(kv, n, dtype=torch.float64, device="cuda")
    for decay in (1.0, 1.0, 0.5, 0.0):
        if decay == 0.0:
            cache.weights.fill_(float("nan"))
        cache.observe(q, lse, decay=decay)
        cache.check()
        total = (total * decay if decay else 0) + torch.stack([w for w, _ in want])
        tol = torch.stack([e for _, e in want]) * 3 + 2.0 ** -21 * total
        assert ((cache.weights.double() - total).abs() <= tol).all()
    # all rows together have given away one each
    assert torch.allclose(cache.weights.double().sum(1), torch.full((kv,), float(n_q * heads // kv), dtype=torch.float64, device="cuda"), rtol=2e-4)


def test_weights_of_heads_of_different_lengths_and_without_queries():
    import torch
    g = gen(12)
    k, v, q = randn(g, 400, 3, 64), randn(g, 400, 3, 64), randn(g, 70, 3, 64)
    source, cache = make(3, 3, 64, 400, k, v), make(3, 3, 64, 400)
    source.weights.fill_(2.0)
    source.evict_into(cache, [300, 0, 129], n_first=400)
    _, lse = attend(cache, q)
    cache.observe(q[:0], lse[:, :0].contiguous(), decay=0.25)
    assert (cache.weights[0, :300] == 0.5).all() and (cache.weights[2, :129] == 0.5).all()
    cache.observe(q, lse)
    for h, m in ((0, 300), (2, 129)):
        w, err = ref.observe(q[:, h:h + 1], lse[h:h + 1], [per_head(k)[h][:m]])[0]
        assert ((cache.weights[h, :m].double() - w - 0.5).abs() <= err + 2.0 ** -21 * (w + 0.5)).all()
    cache.clear()
    cache.observe(q, lse)  # nothing to do


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [5, 16, 140])
def test_weights_of_rows_that_are_not_finite(d, n_q):
    """One row of NaN makes every weight of its head NaN, wherever it stands; a row of -inf log-sum-exp makes them infinite."""
    import torch
    g = gen(13)
    k, v, q = randn(g, 200, 2, d), randn(g, 200, 2, d), randn(g, n_q, 2, d)
    cache = make(2, 2, d, 200, k, v)
    _, lse = attend(cache, q)
    for row in [r for r in (0, 3, 4, 14, 15, 30, 127, 139) if r < n_q]:
        bad = q.clone()
        bad[row, 1, 7] = float("nan")
        cache.observe(bad, lse, decay=0.0)
        assert torch.isnan(cache.weights[1]).all() and torch.isfinite(cache.weights[0]).all()
        sunk = lse.clone()
        sunk[0, row] = -torch.inf
        cache.observe(q, sunk, decay=0.0)
        assert (cache.weights[0] == torch.inf).all() and torch.isfinite(cache.weights[1]).all()


# ---------------------------------------------------------------------------------------------- eviction


def check_evict(cache, keep, n_first, n_recent, capacity=None):
    import torch
    kv, lengths, weights = cache.n_kv_heads, cache.lengths(), cache.weights.cpu()
    k, v = cache.export()
    want = [ref.keep(weights[h, :lengths[h]].tolist(), min(keep[h], lengths[h]), n_first, n_recent) for h in range(kv)]
    other = make(cache.n_heads, kv, cache.head_dim, capacity or max(1, max(len(w) for w in want)))
    index = torch.full((kv, max(len(w) for w in want) + 3), -7, dtype=torch.int32, device="cuda")
    cache.evict_into(other, keep, n_first, n_recent, index=index)
    assert other.lengths() == [len(w) for w in want] and cache.lengths() == lengths
    ok, ov = other.export()
    for h, places in enumerate(want):
        assert index[h].tolist() == places + [-7] * (index.shape[1] - len(places))
        at = torch.tensor(places, dtype=torch.long, device="cuda")
        assert torch.equal(ok[h, :len(places)], k[h, at]) and torch.equal(ov[h, :len(places)], v[h, at])
        if places:
            got, want_w = other.weights[h, :len(places)], weights[h].cuda()[at]
            assert torch.equal(got.view(torch.int32), want_w.view(torch.int32))
    return other


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 33, 1000, 4096, 4097, 9001, 40000])
def test_eviction(d, n):
    import torch
    g = gen(n)
    kv = 3
    cache = make(kv, kv, d, n + 1, randn(g, n, kv, d), randn(g, n, kv, d))
    cache.weights.copy_(torch.randn(kv, n, device="cuda", generator=g).exp())
    for keep in ([n // 2, n // 3, 1], [n, 0, n + 5], [1, n - 1, n // 2]):
        for first, recent in ((0, 0), (n // 7, n // 5), (n, 0), (3, n)):
            check_evict(cache, keep, first, recent)


def test_eviction_ties_and_weights_that_are_not_numbers():
    import torch
    g = gen(21)
    n, kv = 5000, 4
    cache = make(kv, kv, 64, n, randn(g, n, kv, 64), randn(g, n, kv, 64))
    w = cache.weights
    w[0] = 0.0
    w[1] = torch.randint(0, 3, (n,), device="cuda", generator=g).float()
    pool = torch.tensor([0.0, -0.0, float("nan"), float("inf"), float("-inf"), 1e-42, -1e-42, 3.0], device="cuda")
    w[2] = pool[torch.randint(0, 8, (n,), device="cuda", generator=g)]
    w[3] = float("nan")
    for keep in (1, 700, 2500, 4400, 4999):
        for first, recent in ((0, 0), (100, 300)):
            check_evict(cache, [keep] * kv, first, recent)


def test_eviction_of_long_heads():
    """More tokens than a cluster keeps in shared memory."""
    import torch
    g = gen(22)
    n = 8 * 24576 + 1000
    cache = make(1, 1, 64, n)
    for at in range(0, n, 50000):
        m = min(50000, n - at)
        cache.append(randn(g, m, 1, 64), randn(g, m, 1, 64))
    cache.weights.copy_(torch.randint(0, 100000, (1, n), device="cuda", generator=g).float())
    check_evict(cache, [n // 3], 10, 1000)


@pytest.mark.parametrize("n", [512, 3000, 4096, 9000, 50000])
def test_eviction_where_the_first_digits_settle_it(n):
    """Numbers to keep that end with a digit's bin, one before and one behind: eight powers of two (first digit), 1 + i 2^-13 (second),
    1 + i 2^-23 (third)."""
    import torch
    g = gen(n)
    cache = make(3, 3, 64, n, randn(g, n, 3, 64), randn(g, n, 3, 64))
    order = torch.randperm(n, device="cuda", generator=g)
    w = cache.weights
    w[0] = torch.exp2((order % 8).float())
    w[1] = 1.0 + (order % 2048).float() * 2.0 ** -13
    w[2] = 1.0 + (order % 2048).float() * 2.0 ** -23
    rows = [torch.sort(w[h], descending=True)[0] for h in range(3)]
    for at in (1, n // 3, n // 2, n - 1):
        ends = [int((rows[h] >= rows[h][at]).sum()) for h in range(3)]  # of the bin of the at-th largest
        for off in (-1, 0, 1):
            check_evict(cache, [min(n, max(0, e + off)) for e in ends], 0, 0)
            check_evict(cache, [min(n, max(0, e + off)) for e in ends], 5, 20)


def test_eviction_without_index_equals_that_with_one_and_is_captured():
    import torch
    g = gen(23)
    n = 6000
    cache = make(2, 2, 128, n, randn(g, n, 2, 128), randn(g, n, 2, 128))
    cache.weights.copy_(torch.rand(2, n, device="cuda", generator=g))
    a, b, c = (make(2, 2, 128, n) for _ in range(3))
    cache.evict_into(a, 2000, index=torch.empty(2, 2000, dtype=torch.int32, device="cuda"))
    cache.evict_into(b, 2000)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.evict_into(c, [2000, 2000])
    graph.replay()
    for other in (b, c):
        for x, y in zip(a.export() + (a.weights,), other.export() + (other.weights,)):
            assert torch.equal(x, y)


# ---------------------------------------------------------------------------------------------- together


def test_blocks_of_a_video_with_positions_refresh_and_eviction():
    """Rotate, pack, attend, refresh the newest block, weigh, evict, go on: as a generation loop does it."""
    import torch
    from paper_2607_20125_b200.packed import Rope
    g = gen(30)
    heads, kv, d, gh, gw = 4, 2, 64, 6, 7
    block, budget = 3 * gh * gw, 300
    rope = Rope(heads, d, gh, gw, n_kv_heads=kv, dims=(24, 20, 20))
    cache, spare = make(heads, kv, d, 600), make(heads, kv, d, 600)
    keys, values = [torch.empty(0, d, dtype=torch.float64, device="cuda") for _ in range(kv)], [torch.empty(0, d, dtype=torch.float64, device="cuda") for _ in range(kv)]
    for b in range(6):
        for step in range(2):
            q, k, v = randn(g, block, heads, d), randn(g, block, kv, d), randn(g, block, kv, d)
            rope.apply(q, q, k, k, first_frame=3 * b)
            if step:
                cache.drop_last(block)
            cache.append(k, v)
            now_k = [torch.cat((x, y)) for x, y in zip(keys, per_head(k))]
            now_v = [torch.cat((x, y)) for x, y in zip(values, per_head(v))]
            out, lse = attend(cache, q)
            ref.check_attend(out, lse, q, now_k, now_v)
        keys, values = now_k, now_v
        cache.observe(q, lse, decay=0.9)
        one, one_lse = attend(cache, q[-1:].contiguous())
        ref.check_attend(one, one_lse, q[-1:], keys, values)
        if max(cache.lengths()) > budget:
            weights = cache.weights.cpu()
            places = [ref.keep(weights[h, :m].tolist(), budget - 50 * h, 42, block) for h, m in enumerate(cache.lengths())]
            index = torch.empty(kv, budget, dtype=torch.int32, device="cuda")
            cache.evict_into(spare, [budget, budget - 50], n_first=42, n_recent=block, index=index)
            for h, want in enumerate(places):
                assert index[h, :len(want)].tolist() == want
                at = torch.tensor(want, device="cuda")
                keys[h], values[h] = keys[h][at], values[h][at]
            cache, spare = spare, cache


def test_refusals_leave_the_cache_as_it_was():
    import torch
    from paper_2607_20125_b200.binding import HeadCastError
    g = gen(31)
    cache = make(4, 2, 64, 100, randn(g, 90, 2, 64), randn(g, 90, 2, 64))
    before = [x.clone() for x in cache.export()]
    q = randn(g, 5, 4, 64)
    with pytest.raises(HeadCastError) as e:
        cache.append(randn(g, 11, 2, 64), randn(g, 11, 2, 64))
    assert e.value.code == -2
    for bad in (lambda: cache.append(randn(g, 3, 4, 64), randn(g, 3, 4, 64)), lambda: cache.append(randn(g, 3, 2, 64).float(), randn(g, 3, 2, 64)),
                lambda: cache.append(randn(g, 3, 2, 128)[..., ::2], randn(g, 3, 2, 128)[..., ::2]), lambda: cache.attend(q, torch.empty_like(q)[:4]),
                lambda: cache.attend(q.transpose(0, 1), torch.empty_like(q)), lambda: cache.attend(q, torch.empty_like(q), torch.empty(5, 4, device="cuda")),
                lambda: cache.attend(q.cpu(), torch.empty_like(q)), lambda: cache.observe(q, torch.empty(4, 6, device="cuda")),
                lambda: cache.evict_into(cache, [1]), lambda: cache.evict_into(None, 1)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cache.drop_last(1 << 32), lambda: cache.export(first=1 << 33), lambda: cache.evict_into(make(4, 2, 64, 90), (1 << 32) + 5),
                lambda: make(4, 2, 64, (1 << 32) + 100)):  # numbers that ctypes would cut down to valid ones
        with pytest.raises(ValueError):
            bad()
    for bad, code in ((lambda: cache.evict_into(cache, 10), -1), (lambda: cache.evict_into(make(4, 2, 64, 9), 10), -2), (lambda: cache.evict_into(make(2, 2, 128, 90), 10), -1),
                      (lambda: cache.evict_into(make(4, 2, 64, 90), -1), -1), (lambda: cache.drop_last(91), -2),
                      (lambda: cache.evict_into(make(4, 2, 64, 90), 10, index=torch.empty(2, 9, dtype=torch.int32, device="cuda")), -1),
                      (lambda: cache.observe(q, torch.empty(4, 5, device="cuda"), decay=float("nan")), -1)):
        with pytest.raises(HeadCastError) as e:
            bad()
        assert e.value.code == code, e.value
    assert cache.lengths() == [90, 90]
    for a, b in zip(before, cache.export()):
        assert torch.equal(a, b)
    cache.check()
