"""The packed cache and its operators from their definitions, in 64 bits."""
import torch

CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def held(x):
    """float64, the values that a packed cache holds for x [..., d]: by distance to every candidate."""
    x = x.double()
    x = torch.where(x.isnan(), torch.zeros_like(x), x)
    shape = x.shape
    x = x.reshape(-1, 16)
    wanted = (x.abs().amax(1) / 6).clamp(min=2.0 ** -19, max=2.0 ** 40)
    step = torch.exp2(torch.floor(torch.log2(wanted)) - 3)
    scale = (torch.round(wanted / step) * step).clamp(2.0 ** -19, 1.875 * 2.0 ** 12)[:, None]
    even_first = torch.tensor([CODES[i] for i in (0, 2, 4, 6, 1, 3, 5, 7)], dtype=torch.float64, device=x.device)
    size = x.abs().clamp(max=2.0 ** 60)
    nearest = (size[..., None] - even_first * scale[..., None]).abs().argmin(-1)
    return (torch.sign(x) * even_first[nearest] * scale).reshape(shape)


def attend(q, k, v, scale=None):
    """q [n, H, d]; k, v lists of [n_h, d] float64, one per key/value head.  (out [n, H, d], lse [H, n], sum p |v| [n, H, d], largest
    scale * sum |q k| [H, n])"""
    n, heads, d = q.shape
    group = heads // len(k)
    scale = d ** -0.5 if scale is None else scale
    out, mag = (torch.zeros(n, heads, d, dtype=torch.float64, device=q.device) for _ in range(2))
    lse, size = torch.full((heads, n), -torch.inf, dtype=torch.float64, device=q.device), torch.zeros(heads, n, dtype=torch.float64, device=q.device)
    for h in range(heads):
        kh, vh = k[h // group], v[h // group]
        if len(kh) == 0:
            continue
        s = q[:, h].double() @ kh.T * scale
        lse[h] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[h][:, None])
        out[:, h], mag[:, h] = p @ vh, p @ vh.abs()
        size[h] = (q[:, h].double().abs() @ kh.abs().T * scale).amax(1)
    return out, lse, mag, size


def check_attend(out, lse, q, k, v, scale=None):
    """Against the 64-bit result, element by element.

    out: the final rounding is off by half a step of bf16, 2^-8 of the value; every probability enters the second product rounded to
    fp16, 2^-11 of itself, and below the smallest normal number by 2^-25 absolute, where the row's largest is 2^6 or more (n * 2^-31
    of the largest value held); logits, exponentials and sums are fp32.  A logit is the sum of d products in fp32, off by
    at most (d + 2) 2^-23 of sum |q k| * scale, which changes a probability by that fraction; the exponential's own error and the
    sums' add at most 2^-18.
    lse: the logits' error, the sums' 2^-18, and the rounding of the result."""
    want, want_lse, mag, size = attend(q, k, v, scale)
    n = max(len(x) for x in k)
    top = max([float(x.abs().max()) for x in v if len(x)] + [0.0])
    logit = (q.shape[-1] + 2) * 2.0 ** -23 * size
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -17 + 2 * logit.T[..., None]) * mag + n * 2.0 ** -31 * top
    off = (out.double() - want).abs()
    assert (off <= tol).all(), (off / tol.clamp(min=1e-30)).max()
    if lse is not None:
        none = torch.isinf(want_lse)
        assert torch.equal(none, torch.isinf(lse)) and (lse[none] < 0).all()
        off = (lse.double() - want_lse).abs()[~none]
        assert (off <= logit[~none] + 2.0 ** -17 + 2.0 ** -22 * want_lse.abs()[~none]).all(), off.max()


def observe(q, lse, k, scale=None):
    """(weights, their bound on the logits' error) per key/value head, float64."""
    heads, d = q.shape[1], q.shape[2]
    group = heads // len(k)
    scale = d ** -0.5 if scale is None else scale
    out = []
    for i, kh in enumerate(k):
        w, err = torch.zeros(len(kh), dtype=torch.float64, device=q.device), torch.zeros(len(kh), dtype=torch.float64, device=q.device)
        for h in range(group * i, group * (i + 1)):
            if len(kh) == 0:
                continue
            p = torch.exp(q[:, h].double() @ kh.T * scale - lse[h].double()[:, None])
            size = q[:, h].double().abs() @ kh.abs().T * scale
            w += p.sum(0)
            # as in check_attend, and lse * log2(e) rounded to fp32
            err += (p * ((d + 4) * 2.0 ** -23 * size + 2.0 ** -22 * lse[h].double().abs()[:, None] + 2.0 ** -18)).sum(0)
        out.append((w, err))
    return out


def keep(weights, n_keep, n_first, n_recent):
    """Places that stay of one head's weights (a list of floats), from the definition."""
    n = len(weights)
    always = [i < n_first or i >= n - n_recent for i in range(n)]
    # a NaN is below everything, -0 equals 0
    rank = [(0, 0.0) if a else (1, -w) if w == w else (2, 0.0) for a, w in zip(always, weights)]
    order = sorted(range(n), key=lambda i: (rank[i], i))
    return sorted(order[:n_keep])
