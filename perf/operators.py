"""Timed work of the operators around a key/value cache held in 4 bits, as a program that generates long videos calls them.

A layer that keeps a long history packs each new block's keys and values into four bits, rotates queries and keys by their
position in time, height and width, attends to the packed cache, adds up how much attention every cached token receives, and
drops the tokens that receive the least once the cache is full.  The kinds of case:

    rope     rotary positions of one block's queries and keys
    append   one block's keys and values packed behind the cache, and read back as the values that are held
    attend   attention of some queries over the whole packed cache (outputs and log-sum-exp per row)
    observe  the attention weight that every cached token receives from the queries, summed over them
    evict    the tokens of the largest accumulated weight per head, moved into another cache, and read back

The packed form.  16 neighbouring values of a row share one scale s: the largest magnitude over 6, rounded to four significant
bits (ties to even) and held within 2^-19 .. 1.875 * 2^12.  A value x is held as sign * s * c, where c is the one of
0, 0.5, 1, 1.5, 2, 3, 4, 6 that is nearest to |x| / s (ties go to the even place in this list, larger values to 6).
"""
import math

import torch

own = False

CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 16
SCALE_MIN, SCALE_MAX = 2.0 ** -19, 1.875 * 2.0 ** 12
AXES = {128: (44, 42, 42), 64: (24, 20, 20)}  # rotated width of time, height, width
THETA = 10000.0
CHUNK = 1 << 27  # logits that the plain forms hold at a time


def listed():
    return [
        # one frame of the 30 x 52 grid late in a long video, twelve heads of 128
        dict(name="rope-frame", kind="rope", gh=30, gw=52, frames=1, first=2001, heads=12, kv=12, d=128, halves=False, inverse=False),
        # a block of three frames of the 68 x 120 grid; keys rotated back, as before cached keys get new positions
        dict(name="rope-block-1080p", kind="rope", gh=68, gw=120, frames=3, first=18, heads=12, kv=12, d=128, halves=True, inverse=True),
        # one frame of the 30 x 52 grid joins the cache
        dict(name="append-frame", kind="append", n=1560, kv=12, d=128),
        # a block of the 45 x 80 grid joins the cache
        dict(name="append-block-720p", kind="append", n=10800, kv=12, d=128),
        # a single token over a full window of the 30 x 52 grid: latency and memory
        dict(name="attend-token", kind="attend", q=1, n=32760, heads=12, kv=12, d=128),
        # a few queries with shared key heads of 64 and odd lengths
        dict(name="attend-shared-odd", kind="attend", q=77, n=10007, heads=16, kv=4, d=64),
        # one denoise step of a block over seven cached blocks, 30 x 52 and 45 x 80 grids
        dict(name="attend-block-480p", kind="attend", q=4680, n=32760, heads=12, kv=12, d=128),
        dict(name="attend-block-720p", kind="attend", q=10800, n=75600, heads=12, kv=12, d=128),
        # the newest frame's queries weigh three cached blocks; a block's queries weigh the full window
        dict(name="observe-frame", kind="observe", q=1560, n=14040, heads=12, kv=12, d=128),
        dict(name="observe-block-480p", kind="observe", q=4680, n=32760, heads=12, kv=12, d=128),
        # a preview's window loses a third; a full window of the 45 x 80 grid loses half
        dict(name="evict-small", kind="evict", n=3003, keep=2001, first=286, recent=858, kv=6, d=128),
        dict(name="evict-720p", kind="evict", n=75600, keep=37800, first=3600, recent=10800, kv=12, d=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    kind = rng.choice(["rope", "append", "attend", "attend", "attend", "observe", "evict"])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 6, 8, 12])
    heads = kv * (rng.choice([1, 2, 4]) if kv <= 6 else 1)
    if kind == "rope":
        gh = _log_int(rng, 8, 68)
        gw = max(8, int(round(gh * rng.uniform(1.0, 1.75))))
        return dict(kind=kind, gh=gh, gw=gw, frames=rng.randint(1, 3), first=rng.choice([0, rng.randint(1, 50), _log_int(rng, 50, 100000)]),
                    heads=heads, kv=kv, d=d, halves=rng.random() < 0.5, inverse=rng.random() < 0.3)
    if kind == "append":
        return dict(kind=kind, n=_log_int(rng, 1, 10800), kv=kv, d=d)
    if kind == "evict":
        n = _log_int(rng, 100, 75600)
        keep = rng.randint(n // 4, n)
        return dict(kind=kind, n=n, keep=keep, first=rng.randint(0, keep // 3), recent=rng.randint(0, keep // 3), kv=kv, d=d)
    top = {"attend": 10800 * 75600 * 12, "observe": 4680 * 32760 * 12}[kind]
    while True:
        q, n = rng.choice([1, _log_int(rng, 2, 200), _log_int(rng, 200, 10800)]), _log_int(rng, 1, 75600)
        if q * n * heads <= top:
            return dict(kind=kind, q=q, n=n, heads=heads, kv=kv, d=d)


# ---------------------------------------------------------------------------------------------- inputs


def _kv(gen, n, kv, d):
    """Keys with a few channels that carry an offset, as rotated and normalised keys have; values without."""
    offset = torch.zeros(kv, d, device="cuda")
    offset[:, :: max(1, d // 8)] = 3.0 * torch.randn(kv, len(range(0, d, max(1, d // 8))), device="cuda", generator=gen)
    k = torch.randn(n, kv, d, device="cuda", generator=gen) + offset
    v = torch.randn(n, kv, d, device="cuda", generator=gen)
    return k.bfloat16(), v.bfloat16()


def _queries(gen, n, heads, d):
    """From heads that look everywhere alike to heads that look at a few tokens."""
    sharp = torch.linspace(0.4, 2.5, heads, device="cuda")[None, :, None]
    return (sharp * torch.randn(n, heads, d, device="cuda", generator=gen)).bfloat16()


def _pack(x):
    """(codes uint8 [kv, n, d/2], two to a byte, the even element in the low half; scales float32 [kv, n, d/16])."""
    n, kv, d = x.shape
    g = torch.nan_to_num(x.float(), nan=0.0, posinf=float("inf"), neginf=float("-inf")).permute(1, 0, 2).reshape(kv, n, d // GROUP, GROUP)
    m, e = torch.frexp(g.abs().amax(-1) / 6.0)
    s = torch.ldexp(torch.round(m * 16.0) / 16.0, e).clamp(SCALE_MIN, SCALE_MAX)
    a = g.abs() / s[..., None]
    code = torch.zeros_like(a, dtype=torch.uint8)
    # the border below place i: a tie goes to the even place
    for i in range(1, 8):
        border = (CODES[i - 1] + CODES[i]) / 2
        code += (a >= border) if i % 2 == 0 else (a > border)
    code |= (g < 0).to(torch.uint8) << 3
    code = code.reshape(kv, n, d)
    return code[..., 0::2] | (code[..., 1::2] << 4), s


def _unpack(codes, scales):
    """float32 [kv, n, d]"""
    kv, n, half = codes.shape
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(kv, n, 2 * half)
    table = torch.tensor(CODES + tuple(-v for v in CODES), device=codes.device)
    return table[c.long()] * scales.repeat_interleave(GROUP, -1)


def _cache(case, k, v, heads, capacity=None):
    from paper_2607_20125_b200.packed import PackedCache
    cache = PackedCache(n_heads=heads, n_kv_heads=case["kv"], head_dim=case["d"], capacity=capacity or case["n"])
    if k is not None:
        cache.append(k, v)
    return cache


def _raw(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, d = case["kind"], case["d"]
    if kind == "rope":
        n = case["frames"] * case["gh"] * case["gw"]
        return (torch.randn(n, case["heads"], d, device="cuda", generator=gen).bfloat16(),
                torch.randn(n, case["kv"], d, device="cuda", generator=gen).bfloat16())
    k, v = _kv(gen, case["n"], case["kv"], d)
    if kind == "append":
        return k, v
    if kind == "evict":
        # heavy-tailed weights; the newest tokens have received none yet
        w = torch.exp(2.0 * torch.randn(case["kv"], case["n"], device="cuda", generator=gen))
        w[:, case["n"] - case["n"] // 16:] = 0.0
        return k, v, w
    return k, v, _queries(gen, case["q"], case["heads"], d)


def _log_sum_exp(case, q, k):
    """float32 [heads, rows] of the scaled logits over the keys [kv, n, d]: what the attention before has returned."""
    heads, group = case["heads"], case["heads"] // case["kv"]
    lse = torch.empty(heads, q.shape[0], device="cuda")
    for h in range(heads):
        for r0, r1 in _chunks(q.shape[0], case["n"]):
            s = (q[r0:r1, h].float() @ k[h // group].T) / math.sqrt(case["d"])
            top = s.amax(-1)
            lse[h, r0:r1] = torch.log(torch.exp(s - top[:, None]).sum(-1)) + top
    return lse


def prepare(case, seed):
    kind, raw = case["kind"], _raw(case, seed)
    state = dict(case=case)
    if kind == "rope":
        state.update(q=raw[0], k=raw[1])
        if own:
            from paper_2607_20125_b200.packed import Rope
            state.update(rope=Rope(n_heads=case["heads"], n_kv_heads=case["kv"], head_dim=case["d"], grid_h=case["gh"], grid_w=case["gw"],
                                   dims=AXES[case["d"]], theta=THETA, halves=case["halves"]),
                         q_out=torch.empty_like(raw[0]), k_out=torch.empty_like(raw[1]))
        return state
    if kind == "append":
        state.update(k=raw[0], v=raw[1])
        if own:
            state.update(cache=_cache(case, None, None, case["kv"]))
        return state
    if kind == "evict":
        state.update(weights=raw[2])
        if own:
            cache = _cache(case, raw[0], raw[1], case["kv"])
            cache.weights.copy_(raw[2])
            state.update(cache=cache, kept=_cache(case, None, None, case["kv"], capacity=case["keep"]),
                         index=torch.empty(case["kv"], case["keep"], dtype=torch.int32, device="cuda"))
        else:
            state.update(k=_pack(raw[0]), v=_pack(raw[1]))
        return state
    state.update(q=raw[2])
    if kind == "observe":
        state.update(lse=_log_sum_exp(case, raw[2], _unpack(*_pack(raw[0]))))
    if own:
        state.update(cache=_cache(case, raw[0], raw[1], case["heads"]))
        if kind == "attend":
            state.update(out=torch.empty_like(raw[2]), lse=torch.empty(case["heads"], case["q"], device="cuda"))
    else:
        state.update(k=_pack(raw[0]), v=_pack(raw[1]))
    return state


# ---------------------------------------------------------------------------------------------- one pass


def run(state):
    case = state["case"]
    return (_RUN_OWN if own else _RUN_PLAIN)[case["kind"]](case, state)


def _own_rope(case, st):
    st["rope"].apply(st["q"], st["q_out"], st["k"], st["k_out"], first_frame=case["first"], inverse=case["inverse"])
    return st["q_out"], st["k_out"]


def _own_append(case, st):
    st["cache"].clear()
    st["cache"].append(st["k"], st["v"])
    return st["cache"].export()


def _own_attend(case, st):
    st["cache"].attend(st["q"], st["out"], st["lse"])
    return st["out"], st["lse"]


def _own_observe(case, st):
    st["cache"].observe(st["q"], st["lse"], decay=0.0)
    return st["cache"].weights


def _own_evict(case, st):
    st["cache"].evict_into(st["kept"], case["keep"], n_first=case["first"], n_recent=case["recent"], index=st["index"])
    k, v = st["kept"].export()
    return st["index"], st["kept"].weights, k, v


def _chunks(rows, n):
    step = max(1, CHUNK // n)
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def _angles(case):
    """float64 [tokens, pairs]: position times frequency, axis after axis."""
    gh, gw = case["gh"], case["gw"]
    t = torch.arange(case["frames"] * gh * gw, device="cuda")
    position = (case["first"] + t // (gh * gw), t // gw % gh, t % gw)
    parts = []
    for p, width in zip(position, AXES[case["d"]]):
        frequency = THETA ** (-torch.arange(0, width, 2, device="cuda", dtype=torch.float64) / width)
        parts.append(p.double()[:, None] * frequency)
    return torch.cat(parts, -1)


def _plain_rope(case, st):
    angle = _angles(case)
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if case["inverse"]:
        sin = -sin
    out = []
    for x in (st["q"].float(), st["k"].float()):
        y, pairs = x.clone(), cos.shape[-1]
        first, second = (slice(0, pairs), slice(pairs, 2 * pairs)) if case["halves"] else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., first] * sin + x[..., second] * cos
        out.append(y.bfloat16())
    return tuple(out)


def _plain_append(case, st):
    return _unpack(*_pack(st["k"])).bfloat16(), _unpack(*_pack(st["v"])).bfloat16()


def _plain_attend(case, st):
    k, v, q = _unpack(*st["k"]), _unpack(*st["v"]), st["q"]
    group = case["heads"] // case["kv"]
    out, lse = torch.empty_like(q), torch.empty(case["heads"], case["q"], device="cuda")
    for h in range(case["heads"]):
        for r0, r1 in _chunks(case["q"], case["n"]):
            s = (q[r0:r1, h].float() @ k[h // group].T) * (1.0 / math.sqrt(case["d"]))
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            out[r0:r1, h] = ((p @ v[h // group]) / total).bfloat16()
            lse[h, r0:r1] = (top + torch.log(total))[:, 0]
    return out, lse


def _plain_observe(case, st):
    k, q = _unpack(*st["k"]), st["q"]
    group = case["heads"] // case["kv"]
    weights = torch.zeros(case["kv"], case["n"], device="cuda")
    for h in range(case["heads"]):
        for r0, r1 in _chunks(case["q"], case["n"]):
            s = (q[r0:r1, h].float() @ k[h // group].T) * (1.0 / math.sqrt(case["d"]))
            weights[h // group] += torch.exp(s - st["lse"][h, r0:r1, None]).sum(0)
    return weights


def _keep_order(weights, case):
    """Which tokens stay, in order: the first and the newest ones always, then the largest weights, ties to the lower index."""
    rank = weights.clone()
    rank[:, : case["first"]] = float("inf")
    rank[:, case["n"] - case["recent"]:] = float("inf")
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1]
    return torch.sort(order[:, : case["keep"]], dim=-1)[0]


def _plain_evict(case, st):
    index = _keep_order(st["weights"], case)
    rows = index[..., None]
    moved = [_unpack(torch.gather(c, 1, rows.expand(-1, -1, c.shape[-1])), torch.gather(s, 1, rows.expand(-1, -1, s.shape[-1]))).bfloat16()
             for c, s in (st["k"], st["v"])]
    return index.int(), torch.gather(st["weights"], 1, index), moved[0], moved[1]


_RUN_OWN = dict(rope=_own_rope, append=_own_append, attend=_own_attend, observe=_own_observe, evict=_own_evict)
_RUN_PLAIN = dict(rope=_plain_rope, append=_plain_append, attend=_plain_attend, observe=_plain_observe, evict=_plain_evict)


def work(case):
    d, kv = case["d"], case["kv"]
    row = d // 2 + d // GROUP  # bytes of one packed key or value
    if case["kind"] == "rope":
        values = case["frames"] * case["gh"] * case["gw"] * (case["heads"] + kv) * d
        return {"bytes": 4 * values, "flops": 3 * values}
    if case["kind"] == "append":
        values = 2 * case["n"] * kv * d
        return {"bytes": 2 * values + 4 * case["n"] * kv * row + 2 * values, "flops": 4 * values}
    if case["kind"] == "evict":
        moved = case["keep"] * kv
        return {"bytes": 4 * case["n"] * kv + 8 * moved + 6 * moved * row + 4 * moved * d, "flops": 2 * case["n"] * kv}
    pairs = case["q"] * case["n"] * case["heads"]
    rows = case["q"] * case["heads"]
    if case["kind"] == "attend":
        return {"bytes": 2 * case["n"] * kv * row + 4 * rows * d + 4 * rows, "flops": 4 * pairs * d}
    return {"bytes": case["n"] * kv * (row + 4) + 2 * rows * d + 4 * rows, "flops": 2 * pairs * d}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    return _EXACT[case["kind"]](case, _raw(case, seed))


def _held(x):
    """[kv, n, d] float64: the values that the packed form stands for, by distance to every candidate."""
    x = x.transpose(0, 1).double()
    x = torch.where(x.isnan(), torch.zeros_like(x), x)
    kv, n, d = x.shape
    x = x.reshape(kv * n * (d // GROUP), GROUP)
    wanted = x.abs().max(1).values / 6
    tiny = wanted < SCALE_MIN
    power = torch.floor(torch.log2(torch.where(tiny, torch.full_like(wanted, SCALE_MIN), wanted).clamp(max=2.0 ** 40)))
    step = torch.exp2(power - 3)
    scale = (torch.round(wanted.clamp(max=2.0 ** 40) / step) * step).clamp(SCALE_MIN, SCALE_MAX)
    places = torch.tensor([CODES[i] for i in (0, 2, 4, 6, 1, 3, 5, 7)], dtype=torch.float64, device=x.device)  # the even ones win ties
    held = torch.empty_like(x)
    for i in range(0, x.shape[0], 1 << 20):
        part, s = x[i:i + (1 << 20)], scale[i:i + (1 << 20), None]
        nearest = (part.abs()[..., None] - places * s[..., None]).abs().argmin(-1)
        held[i:i + (1 << 20)] = torch.sign(part) * places[nearest] * s
    return held.reshape(kv, n, d)


def _exact_rope(case, raw):
    inner = torch.exp(1j * _turned(case)).conj() if case["inverse"] else torch.exp(1j * _turned(case))
    width = 2 * inner.shape[1]
    outputs = []
    for x in raw:
        x = x.double()
        body = x[..., :width]
        z = torch.complex(body[..., : width // 2], body[..., width // 2:]) if case["halves"] else torch.view_as_complex(body.reshape(*body.shape[:2], -1, 2).contiguous())
        z = z * inner[:, None]
        body = torch.cat((z.real, z.imag), -1) if case["halves"] else torch.view_as_real(z).flatten(-2)
        outputs.append(torch.cat((body, x[..., width:]), -1))
    return tuple(outputs)


def _turned(case):
    """The angle of every token and pair, from the token's three coordinates."""
    t, y, x = torch.meshgrid(torch.arange(case["first"], case["first"] + case["frames"]), torch.arange(case["gh"]), torch.arange(case["gw"]), indexing="ij")
    columns = []
    for place, width in zip((t, y, x), AXES[case["d"]]):
        for i in range(width // 2):
            columns.append(place.reshape(-1).double() / THETA ** (2 * i / width))
    return torch.stack(columns, 1).cuda()


def _exact_append(case, raw):
    return _held(raw[0]), _held(raw[1])


def _logits(q, key, r0, r1, h, d):
    return torch.einsum("rd,nd->rn", q[r0:r1, h].double(), key) / d ** 0.5


def _exact_attend(case, raw):
    key, value, q = _held(raw[0]), _held(raw[1]), raw[2]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(case["heads"], case["q"], dtype=torch.float64, device="cuda")
    shared = case["heads"] // case["kv"]
    for h in range(case["heads"]):
        for r0, r1 in _chunks(case["q"], case["n"]):
            s = _logits(q, key[h // shared], r0, r1, h, case["d"])
            lse[h, r0:r1] = torch.logsumexp(s, 1)
            out[r0:r1, h] = torch.exp(s - lse[h, r0:r1, None]) @ value[h // shared]
    return out, lse


def _exact_observe(case, raw):
    # the log-sum-exps are inputs of this operator: the same ones that prepare hands over
    lse = _log_sum_exp(case, raw[2], _unpack(*_pack(raw[0]))).double()
    key, shared = _held(raw[0]), case["heads"] // case["kv"]
    weights = torch.zeros(case["kv"], case["n"], dtype=torch.float64, device="cuda")
    for h in range(case["heads"]):
        for r0, r1 in _chunks(case["q"], case["n"]):
            weights[h // shared] += torch.exp(_logits(raw[2], key[h // shared], r0, r1, h, case["d"]) - lse[h, r0:r1, None]).sum(0)
    return weights


def _exact_evict(case, raw):
    k, v, w = raw
    n, keep = case["n"], case["keep"]
    index = []
    for row in w.cpu().tolist():
        always = set(range(case["first"])) | set(range(n - case["recent"], n))
        others = sorted((i for i in range(n) if i not in always), key=lambda i: (-row[i], i))
        index.append(sorted(sorted(always)[:keep] + others[: max(0, keep - len(always))]))
    index = torch.tensor(index, device="cuda")
    heads = torch.arange(case["kv"], device="cuda")[:, None]
    return index.int(), w.double()[heads, index], _held(k)[heads, index], _held(v)[heads, index]


_EXACT = dict(rope=_exact_rope, append=_exact_append, attend=_exact_attend, observe=_exact_observe, evict=_exact_evict)
