"""Decode cache with its type table in 8 bits on the GPU: the codes bit for bit, the steps against 64 bits, against the steps on the
cache that it was packed from, and against the dense mask."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import smat_oracle as so
from paper_2609_36062_b200 import binding as b, synth
from tests.helpers import device_inputs, to_numpy64

pytestmark = pytest.mark.gpu

# d, T, dk, dv, chunk, type, q: tables in fp32 and in bf16, one state and many
CASES = [(1, 512, 64, 64, 64, "f32", 0), (2, 512, 64, 128, 64, "f32", 0), (3, 1024, 128, 64, 32, "f32", 0), (1, 1024, 128, 128, 128, "bf16", 0),
         (2, 1024, 128, 128, 128, "bf16", 0), (3, 2048, 128, 128, 128, "bf16", 0), (4, 2048, 128, 128, 128, "bf16", 5),
         (3, 640, 128, 128, 32, "bf16", 0), (2, 512, 64, 64, 32, "bf16", 0)]


class Cache:
    """Views of a decode cache or of a packed one by the documented layout."""

    def __init__(self, plan, buffer, packed):
        B, H, _, r, p = plan.shape
        g, bh = plan.geometry(), B * H
        at = 0

        def part(dtype, *shape):
            nonlocal at
            n = math.prod(shape) * torch.empty(0, dtype=dtype).element_size()
            v = buffer[at:at + n].view(dtype).view(*shape)
            at += (n + 255) // 256 * 256
            return v

        gated = bool(plan.flags & b.FLAG_GATED)
        if packed:
            self.codes, self.unit = part(torch.int8, bh, g.B, r, p), part(torch.float32, bh, g.B, r)
        else:
            wide = buffer.numel() >= bh * g.B * r * p * 4 + bh * r * p * 4
            self.table = part(torch.float32 if wide else torch.bfloat16, bh, g.B, r, p)
        self.S = part(torch.float32, bh, r, p)
        self.log_g = part(torch.float32, bh) if gated else None
        assert at == buffer.numel()


def codes_of(table):
    """The documented rule: m = 127 / max in fp32 (a quotient next to a number of eight bits may be rounded to it), cut to eight
    significant bits; the rest in 64 bits."""
    top = table.double().abs().amax(-1)
    m = (127.0 / top.float()).clamp(max=2.0 ** 126).double()
    unit = torch.exp2(torch.floor(torch.log2(m)) - 7)
    m = torch.where(top > 0, torch.floor(m / unit) * unit, torch.zeros_like(top))
    return torch.round(table.double() * m[..., None]), torch.where(m > 0, 1 / m, torch.zeros_like(m))


def begin(plan, dev, la=None):
    cache = plan.decode_cache()
    if la is None:
        plan.decode_begin(dev["k"], dev["v"], cache)
    else:
        plan.decode_begin_gated(dev["k"], dev["v"], la, cache)
    return cache


def make(case, gated, batch=1, heads=2, seed=13):
    d, T, dk, dv, c, dtype, q = case
    w = synth.Workload("packed", d, batch, heads, T, dk, dv, c, dtype, "scaled" if dtype == "f32" else "normalised", seed)
    host, dev = device_inputs(w)
    plan = b.SmatPlan(batch, heads, T, dk, dv, d, c, dtype, q_override=q, flags=b.FLAG_GATED if gated else 0)
    la = torch.log(torch.rand(w.bh, T, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * 0.05 + 0.95) if gated else None
    return w, host, dev, plan, la


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_codes_and_values(case, gated):
    w, _, dev, plan, la = make(case, gated)
    cache = begin(plan, dev, la)
    plain = Cache(plan, cache, False)
    plain.S.copy_(torch.randn(plain.S.shape, device="cuda"))          # packed at any token: the running state goes along
    if gated:
        plain.log_g.fill_(-0.25)
    packed = plan.decode_pack(cache)
    v = Cache(plan, packed, True)
    codes, unit = codes_of(plain.table)
    assert torch.equal(v.codes.double(), codes)
    assert float(((v.unit.double() - unit).abs() / unit.clamp(min=1e-300)).max()) <= 2.0 ** -24
    assert torch.equal(v.S, plain.S) and (not gated or torch.equal(v.log_g, plain.log_g))
    back = plan.decode_unpack(packed)
    u = Cache(plan, back, False)
    assert torch.equal(u.table, (v.codes.float() * v.unit[..., None]).to(u.table.dtype))
    assert torch.equal(u.S, plain.S) and (not gated or torch.equal(u.log_g, plain.log_g))
    # a code is off by half a unit at most, (127/128 and 1/127 of the largest entry); the value is then rounded to the table's type
    off = (u.table.double() - plain.table.double()).abs()
    half = 2.0 ** -8 if u.table.dtype == torch.bfloat16 else 2.0 ** -23
    assert bool((off <= plain.table.double().abs().amax(-1, keepdim=True) / 254 * (1 + 2.0 ** -7) + half * (plain.table.double().abs() + off)).all())
    # straight into the packed cache
    direct = torch.full_like(packed, 255)
    plan.decode_begin_packed(dev["k"], dev["v"], direct, log_a=la)
    plan.check_status()
    z = Cache(plan, direct, True)
    assert torch.equal(z.codes, v.codes) and torch.equal(z.unit, v.unit) and bool((z.S == 0).all()) and (not gated or bool((z.log_g == 0).all()))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_steps(case, gated):
    """Every step against 64 bits on the values that the packed table stands for."""
    w, host, dev, plan, la = make(case, gated)
    geo, bh = plan.geometry(), w.bh
    packed = plan.decode_cache_packed()
    plan.decode_begin_packed(dev["k"], dev["v"], packed, log_a=la)
    v = Cache(plan, packed, True)
    table = v.codes.double() * v.unit[..., None].double()
    S = torch.zeros(bh, w.d_k, w.d_v, dtype=torch.float64, device="cuda")
    most, log_g = S.clone(), torch.zeros(bh, dtype=torch.float64, device="cuda")
    other = plan.decode_unpack(packed)
    half = 2.0 ** -8 if case[5] == "bf16" else 2.0 ** -24
    steps = min(geo.m, 96)
    for i in range(steps):
        t = geo.n + i
        q, k, x = (dev[n][:, :, t].contiguous() for n in "qkv")
        lt = la[:, t].contiguous() if gated else None
        o = plan.decode_step_packed(q, k, x, t, packed, log_a_t=lt)
        q64, k64, x64 = (y.double().view(bh, -1) for y in (q, k, x))
        a = lt.double().exp() if gated else torch.ones_like(log_g)
        log_g = log_g + (lt.double() if gated else 0.0)
        outer = k64[:, :, None] * x64[:, None, :]
        S, most = a[:, None, None] * S + outer, a[:, None, None] * most + outer.abs()
        U = table[:, (i + 1) % geo.B] * log_g.exp()[:, None, None]
        want = torch.einsum("hi,hij->hj", q64, U + S)
        # sums of the state (a rounding a token, two more with gates) and of d_k products, exponentials of the gates
        bound = torch.einsum("hi,hij->hj", q64.abs(), U.abs() + most) * (3 * i + 64) * 2.0 ** -23
        off = (o.double().view(bh, -1) - want).abs() - (half * want.abs() + bound)
        assert float(off.max()) <= 0, (t, float(off.max()))
    assert bool(((v.S.double() - S).abs() <= most * (3 * steps + 4) * 2.0 ** -23 + 1e-30).all())
    if gated:
        assert float((v.log_g.double() - log_g).abs().max()) <= steps * 2.0 ** -23 * float(log_g.abs().max())
    if plan.type_table_element_bytes() == 4 and not gated:      # fp32 tables unpack to the same values: the same steps
        for i in range(8):
            t = geo.n + i
            row = [dev[n][:, :, t].contiguous() for n in "qkv"]
            plan.decode_step(*row, t, other)


def test_decoding_near_the_dense_mask():
    """A packed cache's outputs differ from the dense oracle by what 8 bits leave: each entry of U by half a unit at most."""
    case = (3, 1024, 64, 64, 32, "f32", 0)
    w, host, dev, plan, _ = make(case, False)
    geo = so.geometry(w.T, w.chunk, w.d)
    cache = begin(plan, dev)
    table = Cache(plan, cache, False).table.double()
    packed = plan.decode_pack(cache)
    M = so.dense_mask(w.T, w.chunk, w.d)
    ref = [so.forward_dense(*(synth.as_float64(w, host[x][h]) for x in ("q", "k", "v")), M) for h in range(w.bh)]
    for i in range(200):
        t = geo.n + i
        q, k, v = (dev[n][:, :, t].contiguous() for n in "qkv")
        o = to_numpy64(plan.decode_step_packed(q, k, v, t, packed)).reshape(w.bh, -1)
        top = table[:, (i + 1) % geo.B].abs().amax(-1)
        slack = ((q.double().abs().view(w.bh, -1) * top).sum(-1) / 254 * (1 + 2.0 ** -7)).cpu().numpy()
        for h in range(w.bh):
            assert np.abs(o[h] - ref[h][t]).max() <= slack[h] + 1e-4 * np.abs(ref[h]).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_the_edges(dtype):
    """Rows of zeros, of one entry, of the type's smallest and largest values, of values between two codes, and not finite."""
    plan = b.SmatPlan(1, 1, 1024, 128, 128, 2, 128, dtype)
    cache = torch.zeros_like(plan.decode_cache())
    t = Cache(plan, cache, False).table
    big = torch.finfo(t.dtype).max
    t[0, 0, 1, 7] = -3.0
    t[0, 0, 2] = big
    t[0, 0, 3] = 2.0 ** -133                     # below the smallest normal number of either type
    t[0, 0, 4, :4] = torch.tensor([1e-38, -1e-38, 3e-39, 0.0], device="cuda")
    t[0, 0, 5] = torch.arange(128, device="cuda") - 63.5          # the largest is 64.5: codes between two whole numbers
    t[0, 0, 6, :3] = torch.tensor([127.0, 0.5, -2.5], device="cuda")   # m = 1: halves go to the even code
    t[0, 0, 7, 3], t[0, 0, 8, 4], t[0, 0, 9, 5] = math.inf, -math.inf, math.nan
    t[0, 0, 7, 9] = 1.0
    packed = plan.decode_pack(cache)
    v = Cache(plan, packed, True)
    codes, unit = codes_of(t[0, 0, :7])
    assert torch.equal(v.codes[0, 0, :7].double(), codes)
    assert float(((v.unit[0, 0, :7].double() - unit).abs() / unit.clamp(min=1e-300)).max()) <= 2.0 ** -24
    assert v.codes[0, 0, 6, :3].tolist() == [127, 0, -2] and int(v.codes[0, 0, 1, 7]) in (-127, -126)
    assert bool((v.codes[0, 0, 7:10] == 0).all()) and bool(torch.isnan(v.unit[0, 0, 7:10]).all()) and bool((v.unit[0, 0, 10:] == 0).all())
    back = Cache(plan, plan.decode_unpack(packed), False).table
    assert bool(torch.isnan(back[0, 0, 7:10]).all()) and bool(torch.isfinite(back[0, 0, :7]).all()) and bool((back[0, 0, 10:] == 0).all())


def test_long_tables():
    """More than 2^31 entries: offsets of codes, units and values in 64 bits."""
    plan = b.SmatPlan(1, 28, 65536, 128, 128, 4, 128, "bf16")
    cache = plan.decode_cache()
    t = Cache(plan, cache, False).table
    assert t.numel() > 1 << 31
    cache.zero_()
    g = torch.Generator(device="cuda").manual_seed(1)
    spots = [(0, 0), (13, 5000), (27, t.shape[1] - 1)]
    for h, n in spots:
        t[h, n] = torch.randn(128, 128, generator=g, device="cuda").bfloat16()
    packed = torch.full_like(plan.decode_cache_packed(), 85)
    plan.decode_pack(cache, packed)
    v = Cache(plan, packed, True)
    for h, n in spots:
        codes, unit = codes_of(t[h, n])
        assert torch.equal(v.codes[h, n].double(), codes)
    assert int((v.unit != 0).sum()) == 3 * 128 and int(v.codes.view(-1, 1 << 16).any(-1).sum()) <= 6
    cache.fill_(85)
    plan.decode_unpack(packed, cache)
    for h, n in spots:
        assert torch.equal(t[h, n], (v.codes[h, n].float() * v.unit[h, n][:, None]).bfloat16())
    assert int((t.view(-1, 1 << 16) != 0).any(-1).sum()) <= 6
    q = torch.randn(1, 28, 128, generator=g, device="cuda").bfloat16()
    zero = torch.zeros_like(q)
    last = plan.geometry().n + t.shape[1] - 2                   # the step of the last type
    o = plan.decode_step_packed(q, zero, zero, last, packed)
    want = q[0, 27].double() @ (v.codes[27, -1].double() * v.unit[27, -1][:, None].double())
    assert float((o[0, 27].double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-4
    assert bool((o[0, 1:13] == 0).all())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("place", ["q", "k", "v"])
def test_the_output_may_take_the_place_of_an_input_row(place, gated):
    B, H, T = 16, 16, 512
    w = synth.Workload("inplace", 2, 1, 1, T, 128, 128, 128, "bf16", "scaled", 7)
    _, dev = device_inputs(w)
    k, v = (dev[n].expand(B, H, T, 128).contiguous() for n in "kv")
    g = torch.Generator(device="cuda").manual_seed(2)
    la = torch.log(torch.rand(B * H, T, generator=g, device="cuda") * 0.1 + 0.9) if gated else None
    plan = b.SmatPlan(B, H, T, 128, 128, 2, 128, "bf16", flags=b.FLAG_GATED if gated else 0)
    caches = [plan.decode_cache_packed() for _ in range(2)]
    for c in caches:
        plan.decode_begin_packed(k, v, c, log_a=la)
    for t in range(256, 272):
        rows = {n: torch.randn(B, H, 128, generator=g, device="cuda").bfloat16() for n in "qkv"}
        mine = {n: x.clone() for n, x in rows.items()}
        lt = la[:, t].contiguous() if gated else None
        one = plan.decode_step_packed(rows["q"], rows["k"], rows["v"], t, caches[0], log_a_t=lt)
        two = plan.decode_step_packed(mine["q"], mine["k"], mine["v"], t, caches[1], log_a_t=lt, o=mine[place])
        assert two.data_ptr() == mine[place].data_ptr() and torch.equal(one, two), t
    assert torch.equal(caches[0], caches[1])


def test_captured_steps_and_refusals():
    w, _, dev, plan, _ = make((2, 1024, 128, 128, 128, "bf16", 0), False)
    one, two = plan.decode_cache_packed(), plan.decode_cache_packed()
    for c in (one, two):
        plan.decode_begin_packed(dev["k"], dev["v"], c)
    n = plan.geometry().n
    row = [dev[x][:, :, n].contiguous() for x in "qkv"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = plan.decode_step_packed(*row, n, one)
        spare = plan.decode_pack(plan.decode_unpack(one))
    graph.replay()
    graph.replay()
    want = plan.decode_step_packed(*row, n, two)
    want = plan.decode_step_packed(*row, n, two)
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(one, two) and torch.equal(Cache(plan, spare, True).S, Cache(plan, one, True).S)
    for bad in (one[:1024], one.cpu(), one.repeat(2)[::2]):
        with pytest.raises((b.SmatError, ValueError)):
            plan.decode_unpack(bad)
        with pytest.raises((b.SmatError, ValueError)):
            plan.decode_step_packed(*row, n, bad)
        with pytest.raises((b.SmatError, ValueError)):
            plan.decode_begin_packed(dev["k"], dev["v"], bad)
    with pytest.raises(b.SmatError):
        plan.decode_step_packed(*row, n, one[:1024])
    with pytest.raises(b.SmatError):
        plan.decode_step_packed(*row, n - 1, one)
    with pytest.raises(b.SmatError):
        plan.decode_step_packed(*row, n, one, log_a_t=torch.zeros(2, device="cuda"))
    with pytest.raises(b.SmatError):
        plan.decode_pack(one)                              # a packed cache is shorter than a cache


def largest_multiplier(top):
    """The largest number of eight significant bits, at most 2^126, whose product with `top` is at most 127: in whole numbers."""
    t, most = Fraction(top), Fraction(2) ** 126
    if t * most <= 127:
        return float(most) if t else 0.0
    q = Fraction(127) / t
    e = -200
    while Fraction(2) ** (e + 8) <= q:
        e += 1
    return float((q / Fraction(2) ** e).__floor__() * Fraction(2) ** e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_whose_multiplier_is_next_to_a_border(dtype):
    """127 / max within a rounding of fp32 of a number of eight bits: whichever way a quotient in fp32 falls there, the multiplier is the
    largest one that keeps the codes within 127."""
    plan = b.SmatPlan(1, 1, 1024, 128, 128, 2, 128, dtype)
    cache = torch.zeros_like(plan.decode_cache())
    t = Cache(plan, cache, False).table
    rows = t.view(-1, 128)
    tops = []
    for eighth in range(128, 256):
        near = np.float32(127.0 / eighth)
        for top in (np.nextafter(near, np.float32(0)), near, np.nextafter(near, np.float32(9))):
            tops += [float(top), float(top) * 2.0 ** -31, float(top) * 2.0 ** 90]
    tops += [127.0 * 2.0 ** k for k in (-133, -40, 0, 100)] + [2.0 ** k for k in (-149, -130, -126, -3, 127)]
    assert len(tops) <= rows.shape[0]
    g = torch.Generator(device="cuda").manual_seed(3)
    top = torch.tensor(tops, dtype=torch.float64, device="cuda")
    entries = (top[:, None] * (2 * torch.rand(len(tops), 128, generator=g, device="cuda", dtype=torch.float64) - 1)).to(t.dtype)
    entries[:, 5] = top.to(t.dtype)
    rows[:len(tops)] = entries
    m = torch.tensor([largest_multiplier(x) for x in entries.double().abs().amax(-1).tolist()], dtype=torch.float64, device="cuda")
    v = Cache(plan, plan.decode_pack(cache), True)
    codes, unit = v.codes.view(-1, 128)[:len(tops)], v.unit.view(-1)[:len(tops)]
    assert torch.equal(codes.double(), torch.round(entries.double() * m[:, None]))
    assert torch.equal(unit, torch.where(m > 0, 1 / m, torch.zeros_like(m)).float())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_steps_on_the_unpacked_cache(case, gated):
    """A step on a packed cache and on the cache that it unpacks to: the same running state bit for bit, and outputs that differ by the
    values' rounding to the table's type (a packed one is code * unit, not rounded), and by that of the sums."""
    w, _, dev, plan, la = make(case, gated)
    packed = plan.decode_pack(begin(plan, dev, la))
    cache = plan.decode_unpack(packed)
    v, u = Cache(plan, packed, True), Cache(plan, cache, False)
    geo, bh = plan.geometry(), w.bh
    value = 2.0 ** -8 if u.table.dtype == torch.bfloat16 else 2.0 ** -24
    half = 2.0 ** -8 if case[5] == "bf16" else 2.0 ** -24
    for i in range(min(geo.m, 16)):
        t = geo.n + i
        row = [dev[n][:, :, t].contiguous() for n in "qkv"]
        lt = la[:, t].contiguous() if gated else None
        one = plan.decode_step_packed(*row, t, packed, log_a_t=lt)
        two = plan.decode_step_gated(*row, lt, t, cache) if gated else plan.decode_step(*row, t, cache)
        assert torch.equal(v.S, u.S) and (not gated or torch.equal(v.log_g, u.log_g))
        q = row[0].double().abs().view(bh, -1)
        U = u.table[:, (i + 1) % geo.B].double().abs()
        # of the packed side: the unit's product with the gate's factor; of both: a fused sum an entry, and d_k products in turn
        bound = torch.einsum("hi,hij->hj", q, U * (value + 2.0 ** -23) + (U + v.S.double().abs()) * 2 * (w.d_k + 2) * 2.0 ** -24)
        off = (one.double() - two.double()).abs().view(bh, -1) - (half * (one.double().abs() + two.double().abs()).view(bh, -1) + bound)
        assert float(off.max()) <= 0.0, (t, float(off.max()))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", [(2, 512, 64, 64, 64, "f32", 0), (2, 1024, 128, 128, 128, "bf16", 0), (2, 512, 64, 64, 32, "bf16", 0)])
def test_steps_on_rows_at_the_end_of_the_range(case, gated):
    """Half a unit above a row's largest entry there is no number of the type: a step reads the largest one, as unpacking does."""
    w, _, dev, plan, la = make(case, gated)
    cache = begin(plan, dev, la)
    cache.zero_()
    c = Cache(plan, cache, False)
    most = torch.finfo(c.table.dtype).max
    c.table[:, 1, 3], c.table[:, 1, 5, ::2], c.table[:, 1, 7], c.table[:, 1, 9, 1] = most, -most, most / 2, -most
    packed = plan.decode_pack(cache)
    back = Cache(plan, plan.decode_unpack(packed), False).table
    assert bool((back[:, 1, 3] == most).all()) and bool((back[:, 1, 5, ::2] == -most).all()) and bool((back[:, 1, 9, 1] == -most).all())
    n, (B, H, _, r, p) = plan.geometry().n, plan.shape
    zero = torch.zeros(B, H, p, device="cuda", dtype=dev["v"].dtype)
    for i, factor in ((3, 0.25), (5, 2.0 ** -20), (7, 1.0), (9, 0.5)):
        q = torch.zeros(B, H, r, device="cuda", dtype=dev["q"].dtype)
        q[..., i] = factor
        spare = packed.clone()
        lt = torch.full((B * H,), -math.log(2.0), device="cuda") if gated else None
        o = plan.decode_step_packed(q, torch.zeros_like(q), zero, n, spare, log_a_t=lt)
        want = back[:, 1, i].double().view(B, H, p) * factor * (0.5 if gated else 1.0)
        half = torch.finfo(o.dtype).eps / 2
        # of the table's type the value is rounded again (unpacked), of fp32 the gate's exponential and the products
        assert bool(((o.double() - want).abs() <= want.abs() * (half + (2.0 ** -8 if c.table.dtype == torch.bfloat16 else 0.0) + 2.0 ** -21)).all()), i
