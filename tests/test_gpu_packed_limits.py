"""GPU: the packed cache at the limits of what its calls take, against the definitions in 64 bits."""
import pytest

import packed_reference as ref
from test_gpu_packed import attend, check_evict, gen, make, per_head, randn

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- logits far below the others


def far_and_near(n_q, n, near, seed):
    """Two heads of 64.  Every third row looks along element 0, where the tokens outside ``near`` lie at -6144 and those of it at zero: their
    logits there are -3.1e6 and -6.3e6 (from 2.9e6 on a largest logit is too large in magnitude), those of ``near`` ordinary."""
    import torch
    g = gen(seed)
    k, v, q = randn(g, n, 2, 64), randn(g, n, 2, 64), randn(g, n_q, 2, 64)
    far = torch.ones(n, dtype=torch.bool, device="cuda")
    far[near] = False
    k[:, :, 0] = torch.where(far, -6144.0, 0.0).bfloat16()[:, None]
    looks = torch.arange(n_q, device="cuda") % 3 == 0
    q[:, :, 0] = 0.0
    q[looks, :, 0] = torch.where(torch.arange(n_q, device="cuda")[looks] % 2 == 0, 4096.0, 8192.0).bfloat16()[:, None]
    return q, k, v, looks


@pytest.mark.parametrize("n_q", [2, 8, 16, 150, 700])
@pytest.mark.parametrize("n,near", [(700, slice(699, 700)), (700, slice(0, 1)), (700, slice(300, 340)), (20000, slice(19872, 20000)), (20000, slice(9000, 9100)),
                                    (20000, slice(0, 20000, 1009)), (128, slice(17, 18)), (129, slice(128, 129))])
def test_a_row_is_as_large_as_its_largest_logit(n_q, n, near):
    """Tokens far below weigh nothing, wherever they stand and however the work is dealt; the row is that of the others."""
    q, k, v, looks = far_and_near(n_q, n, near, n)
    out, lse = attend(make(2, 2, 64, n, k, v), q)
    hk, hv = per_head(k), per_head(v)
    ref.check_attend(out[looks], lse[:, looks], q[looks], [x[near] for x in hk], [x[near] for x in hv])
    ref.check_attend(out[~looks], lse[:, ~looks], q[~looks], hk, hv)


@pytest.mark.parametrize("n_q", [2, 16, 150, 700])
@pytest.mark.parametrize("n", [100, 20000])
def test_a_row_whose_logits_all_are_far_below_is_nan(n_q, n):
    """Whether its logits are numbers or beyond them, and no other row; so is one with a single logit far above."""
    import torch
    for first in (4096.0, 8192.0, 2.0 ** 60, 2.0 ** 126):
        q, k, v, looks = far_and_near(n_q, n, slice(0, 0), n)
        q[0, 0], q[0, 0, 0] = 0.0, first
        out, lse = attend(make(2, 2, 64, n, k, v), q)
        assert torch.isnan(out[looks].float()).all() and torch.isnan(lse[:, looks]).all()
        ref.check_attend(out[~looks], lse[:, ~looks], q[~looks], per_head(k), per_head(v))
    q, k, v, looks = far_and_near(n_q, n, slice(0, n), n)
    k[n - 1, :, 0] = 6144.0
    out, lse = attend(make(2, 2, 64, n, k, v), q)
    assert torch.isnan(out[looks].float()).all() and torch.isnan(lse[:, looks]).all()
    ref.check_attend(out[~looks], lse[:, ~looks], q[~looks], per_head(k), per_head(v))


@pytest.mark.parametrize("n_q", [2, 16, 150])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_of_zero_whatever_the_row_and_the_scale(n_q, d):
    """A row of 2^112 that meets only zeros, at the largest scale: its logits are zero, though row times scale is more than fp32 holds."""
    import torch
    g = gen(n_q + d)
    n, scale = 700, 2.0 ** 40
    k, v, q = randn(g, n, 2, d), randn(g, n, 2, d), randn(g, n_q, 2, d, scale=1 / scale)
    k[:, :, 0] = q[:, :, 0] = 0.0
    q[::2] = 0.0
    q[::2, :, 0] = 2.0 ** 112
    cache = make(2, 2, d, n, k, v, softmax_scale=scale)
    hk, hv = per_head(k), per_head(v)
    out, lse = attend(cache, q)
    ref.check_attend(out, lse, q, hk, hv, scale)
    cache.observe(q, lse, decay=0.0)
    for (w, err), got in zip(ref.observe(q, lse, hk, scale), cache.weights.double()):
        assert ((got - w).abs() <= err + 2.0 ** -21 * w).all()


# ---------------------------------------------------------------------------------------------- lengths around what eviction keeps in registers


@pytest.mark.parametrize("n", [98303, 98304, 98305])
def test_eviction_at_the_border_of_what_registers_hold(n):
    """Twelve keys for each of 1024 threads of eight blocks."""
    import torch
    g = gen(n)
    cache = make(1, 1, 64, n, randn(g, n, 1, 64), randn(g, n, 1, 64))
    cache.weights.copy_(torch.randint(0, 5000, (1, n), device="cuda", generator=g).float())
    check_evict(cache, [n // 3], 10, 1000)
    check_evict(cache, [n - 1], 0, 0)


def test_eviction_of_heads_on_both_sides_of_that_border():
    import torch
    g = gen(40)
    n, kv = 98400, 4
    source = make(kv, kv, 64, n, randn(g, n, kv, 64), randn(g, n, kv, 64))
    cache = make(kv, kv, 64, n)
    source.evict_into(cache, [98304, 98305, 500, 0], n_first=n)
    cache.weights.copy_(torch.randint(0, 5000, (kv, 98305), device="cuda", generator=g).float())
    check_evict(cache, [30000, 30001, 77, 5], 3, 100)
    check_evict(cache, [98304, 98304, 499, 0], 0, 0)


# ---------------------------------------------------------------------------------------------- nothing to do


def test_calls_with_empty_tensors():
    import torch
    from paper_2607_20125_b200.packed import Rope
    g = gen(50)
    cache, other = make(4, 2, 64, 50, randn(g, 30, 2, 64), randn(g, 30, 2, 64)), make(4, 2, 64, 50, randn(g, 7, 2, 64), randn(g, 7, 2, 64))
    q = randn(g, 5, 4, 64)
    rope = Rope(4, 64, dims=(24, 20, 20))  # no grid: positions are given
    rope.apply(q[:0], q[:0], positions=torch.zeros(0, 3, dtype=torch.int32, device="cuda"))
    cache.append(randn(g, 0, 2, 64), randn(g, 0, 2, 64))
    cache.attend(q[:0], q[:0], torch.empty(4, 0, device="cuda"))
    cache.observe(q[:0], torch.empty(4, 0, device="cuda"))
    assert cache.export(first=3, n_tokens=0)[0].shape == (2, 0, 64) and cache.lengths() == [30, 30]
    cache.evict_into(other, 0, index=torch.empty(2, 0, dtype=torch.int32, device="cuda"))
    assert other.lengths() == [0, 0] and other.export()[0].shape == (2, 0, 64) and other.weights.shape == (2, 0)
    other.evict_into(cache, 9, index=torch.empty(2, 0, dtype=torch.int32, device="cuda"))
    assert cache.lengths() == [0, 0]
