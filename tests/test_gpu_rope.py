"""GPU: rotary positions over time, height and width against the rotation in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


def reference(x, pos, dims, theta, scales, halves, inverse):
    import torch
    angles = []
    for a, (width, s) in enumerate(zip(dims, scales)):
        f = theta ** (-torch.arange(0, width, 2, device=x.device, dtype=torch.float64) / max(width, 1))
        angles.append(pos[:, a].double()[:, None] * (s * f))
    phi = torch.cat(angles, 1)[:, None, :] * (-1 if inverse else 1)
    pairs = phi.shape[-1]
    y = x.double().clone()
    a, b = (slice(0, pairs), slice(pairs, 2 * pairs)) if halves else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    x0, x1 = x.double()[..., a], x.double()[..., b]
    y[..., a] = x0 * torch.cos(phi) - x1 * torch.sin(phi)
    y[..., b] = x0 * torch.sin(phi) + x1 * torch.cos(phi)
    length = torch.zeros_like(y)
    length[..., a] = length[..., b] = torch.hypot(x0, x1)
    return y, length


def check(got, x, pos, dims, theta, scales, halves, inverse):
    """Half a step of bf16, and of the pair's length: two rounded products and a sum in fp32, sines and cosines of an angle that is off by
    2^-24 half turns at most and by 2^-62 turns per position (3.2 * 2^-24 + 4 * 2^-24, doubled for the products)."""
    import torch
    want, length = reference(x, pos, dims, theta, scales, halves, inverse)
    far = pos.abs().max().double() * 2.0 ** -53 * 8
    assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -20 + far) * length).all()
    width = sum(dims)
    assert torch.equal(got[..., width:].view(torch.int16), x[..., width:].contiguous().view(torch.int16))


CASES = [
    # d, heads, kv, grid, frames, first, dims, halves, inverse
    (128, 12, 12, (3, 5), 2, 0, (44, 42, 42), False, False),
    (128, 3, 1, (7, 9), 3, 70000, (44, 42, 42), True, False),
    (64, 1, 2, (1, 1), 1, -5, (24, 20, 20), False, True),
    (64, 5, 5, (13, 22), 3, 1 << 31, (24, 20, 20), True, True),
    (128, 2, 2, (30, 52), 1, 2001, (16, 0, 32), False, False),   # narrower than the row, an axis without width
    (128, 2, 4, (4, 4), 1, 9, (2, 6, 8), True, False),
    (64, 64, 64, (2, 3), 2, 3, (2, 0, 0), False, False),
    (64, 4, 0, (8, 8), 40, 11, (0, 32, 32), True, False),        # queries alone, many tokens
]


@pytest.mark.parametrize("d,heads,kv,grid,frames,first,dims,halves,inverse", CASES)
def test_positions_of_the_grid(d, heads, kv, grid, frames, first, dims, halves, inverse):
    import torch
    from paper_2607_20125_b200.packed import Rope
    gh, gw = grid
    n = frames * gh * gw
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    rope = Rope(heads, d, gh, gw, n_kv_heads=kv, dims=dims, halves=halves, scales=(1.0, 0.5, 1.25))
    i = torch.arange(n, device="cuda")
    pos = torch.stack((first + i // (gh * gw), i // gw % gh, i % gw), 1)
    q = torch.randn(n, heads, d, device="cuda", generator=gen).bfloat16()
    k = torch.randn(n, kv, d, device="cuda", generator=gen).bfloat16() if kv else None
    q_out, k_out = torch.full_like(q, float("nan")), torch.full_like(k, float("nan")) if kv else None
    rope.apply(q, q_out, k, k_out, first_frame=first, inverse=inverse)
    check(q_out, q, pos, dims, 1e4, (1.0, 0.5, 1.25), halves, inverse)
    if kv:
        check(k_out, k, pos, dims, 1e4, (1.0, 0.5, 1.25), halves, inverse)


@pytest.mark.parametrize("halves", [False, True])
def test_given_positions_of_any_size_and_sign(halves):
    import torch
    from paper_2607_20125_b200.packed import Rope
    gen = torch.Generator(device="cuda").manual_seed(2)
    n = 1009
    pos = torch.randint(-2 ** 31, 2 ** 31, (n, 3), device="cuda", generator=gen).int()
    pos[:4] = torch.tensor([[0, 0, 0], [2 ** 31 - 1] * 3, [-2 ** 31] * 3, [1, -1, 7]], device="cuda")
    q = torch.randn(n, 2, 128, device="cuda", generator=gen).bfloat16()
    out = torch.empty_like(q)
    rope = Rope(2, 128, dims=(44, 42, 42), theta=500.0, halves=halves)
    rope.apply(q, out, positions=pos)
    check(out, q, pos.long(), (44, 42, 42), 500.0, (1.0, 1.0, 1.0), halves, False)


@pytest.mark.parametrize("halves", [False, True])
def test_slices_of_a_fused_projection_and_in_place(halves):
    import torch
    from paper_2607_20125_b200.packed import Rope
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, h, d = 77, 3, 64
    fused = torch.randn(n, 3 * h, d, device="cuda", generator=gen).bfloat16()
    q, k = fused[:, :h], fused[:, h:2 * h]
    rope = Rope(h, d, 7, 11, halves=halves, dims=(16, 16, 32))
    want_q, want_k = torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda"), torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda")
    rope.apply(q.contiguous(), want_q, k.contiguous(), want_k, first_frame=4)
    before = fused.clone()
    q_out, k_out = torch.empty_like(want_q), torch.empty_like(want_k)
    rope.apply(q, q_out, k, k_out, first_frame=4)
    assert torch.equal(q_out, want_q) and torch.equal(k_out, want_k) and torch.equal(fused, before)
    x, y = q.contiguous(), k.contiguous()
    rope.apply(x, x, y, y, first_frame=4)
    assert torch.equal(x, want_q) and torch.equal(y, want_k)


def test_inverse_is_the_gradient_and_undoes_the_rotation():
    import torch
    from paper_2607_20125_b200.packed import Rope
    gen = torch.Generator(device="cuda").manual_seed(4)
    rope = Rope(2, 64, 3, 4, dims=(24, 20, 20))
    x, g = (torch.randn(24, 2, 64, device="cuda", generator=gen).bfloat16() for _ in range(2))
    y, back, grad = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    rope.apply(x, y, first_frame=6)
    rope.apply(y, back, first_frame=6, inverse=True)
    i = torch.arange(24, device="cuda")
    pos = torch.stack((6 + i // 12, i // 4 % 3, i % 4), 1)
    pair = x.double().reshape(24, 2, 32, 2).norm(dim=-1).repeat_interleave(2, -1)
    # two roundings to bf16 of values no larger than the pair
    assert ((back.double() - x.double()).abs() <= (2 * 2.0 ** -8 + 2.0 ** -7 * 2.0 ** -8 + 2.0 ** -19) * 1.4143 * pair).all()
    rope.apply(g, grad, first_frame=6, inverse=True)
    leaf = x.double().requires_grad_()
    phi_y = reference(leaf, pos, (24, 20, 20), 1e4, (1, 1, 1), False, False)[0]
    phi_y.backward(g.double())
    pair_g = g.double().reshape(24, 2, 32, 2).norm(dim=-1).repeat_interleave(2, -1)
    assert ((grad.double() - leaf.grad).abs() <= 2.0 ** -8 * leaf.grad.abs() + 2.0 ** -20 * pair_g).all()


def test_infinities_and_nans_stay_in_their_pairs():
    import torch
    from paper_2607_20125_b200.packed import Rope
    q = torch.ones(5, 1, 64, dtype=torch.bfloat16, device="cuda")
    q[1, 0, 60:] = torch.tensor([float("inf"), float("nan"), float("-inf"), float("nan")], device="cuda").bfloat16()  # behind the rotated width
    q[2, 0, 3] = float("nan")
    out = torch.empty_like(q)
    Rope(1, 64, 1, 5, dims=(0, 0, 60)).apply(q, out)
    assert torch.equal(out[..., 60:].view(torch.int16), q[..., 60:].view(torch.int16))
    bad = torch.isnan(out[:, 0, :60].float())
    want = torch.zeros_like(bad)
    want[2, 2:4] = True
    assert torch.equal(bad, want)


def test_captured_and_replayed():
    import torch
    from paper_2607_20125_b200.packed import Rope
    rope = Rope(2, 128, 5, 7)
    q = torch.randn(35, 2, 128, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rope.apply(q, out, q, out2 := torch.zeros_like(q), first_frame=3)
    for _ in range(2):
        q.copy_(torch.randn(35, 2, 128, device="cuda").bfloat16())
        graph.replay()
        want = torch.empty_like(q)
        rope.apply(q, want, first_frame=3)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want)
