"""The gated recurrence of every channel on the GPU against the definition in 64 bits, token by token."""
import math

import pytest
import torch

from paper_2609_36062_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# Error that a token adds in fp32, relative to the absolute sum that the state is part of: exp within 2 units (2^-22), the product
# and the sum (2^-23); and as much again where a piece's map is formed and joined apart from the state.
TOKEN = 2.0 ** -20
# fp32 ends at 2^-149: a gate below that is a closed one, and a product below 2^-126 is off by up to 2^-150 and not by a part of itself.
# Times states of at most 2^4, added up over at most 2^13 tokens, times a state again in dlog_a: 2^-149 + 4 + 13 + 4.
FLOOR = 2.0 ** -128


def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def walk(a, x, state):
    """y_t = a_t y_{t-1} + x_t in order along dimension 1; y before and behind every token."""
    before, behind = [], []
    for t in range(x.shape[1]):
        before.append(state)
        state = torch.where(a[:, t] == 0, x[:, t], a[:, t] * state + x[:, t])
        behind.append(state)
    return torch.stack(before, 1), torch.stack(behind, 1)


def near(got, want, slack, name):
    off = (got.double() - want).abs() - (HALF[got.dtype] * want.abs() + slack + FLOOR)
    assert got.shape == want.shape and float(off.max()) <= 0.0, (name, float(off.max()))


def check_forward(x, log_a, h0=None, **out):
    H, hT = b.recurrence_forward(x, log_a, h0=h0 if h0 is None else h0.clone(), **out)
    a, start = log_a.double().exp(), torch.zeros_like(x[:, 0], dtype=torch.float64) if h0 is None else h0.double()
    _, h = walk(a, x.double(), start)
    _, most = walk(a, x.double().abs(), start.abs())
    _, slack = walk(a, TOKEN * most, torch.zeros_like(start))
    near(H, h, slack, "h")
    near(hT, h[:, -1], slack[:, -1], "hT")
    return H, hT


def check_backward(log_a, H, dH, h0=None, dhT=None, **out):
    dX, dA, d0 = b.recurrence_backward(log_a, H, dH, h0=h0, dhT=dhT, **out)
    a, g = log_a.double().exp(), dH.double()
    zero = torch.zeros_like(g[:, 0])
    end = zero if dhT is None else dhT.double()

    def back(x, end):      # c_t = a_t (x_t + c_{t+1}): before it, and behind it
        before, behind = walk(a.flip(1), torch.where(a == 0, torch.zeros_like(a), a * x).flip(1), end)
        return before.flip(1), behind.flip(1)
    later, c = back(g, end)
    most_later, most = back(g.abs(), end.abs())
    slack_later, slack = back(TOKEN * (g.abs() + most_later), zero)
    previous = torch.cat((zero[:, None] if h0 is None else h0.double()[:, None], H.double()[:, :-1]), 1)
    near(dX, g + later, slack_later + 2.0 ** -23 * (g.abs() + most_later), "dx")
    want = torch.where(a == 0, torch.zeros_like(c), c * previous)
    near(dA, want, torch.where(a == 0, torch.zeros_like(c), (slack + 2.0 ** -23 * most) * previous.abs()), "dlog_a")
    near(d0, c[:, 0], slack[:, 0], "dh0")
    return dX, dA, d0


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)]


def inputs(B, T, C, types, seed, reach=30.0):
    g = generator(seed)
    x = torch.randn(B, T, C, generator=g, device=DEV).to(types[0])
    log_a = (-torch.rand(B, T, C, generator=g, device=DEV) * 2 / reach).to(types[1])
    h0, dhT = (torch.randn(B, C, generator=g, device=DEV) for _ in range(2))
    return x, log_a, h0, dhT, g


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", [1, 7, 8, 60, 64, 72, 200, 2048])
@pytest.mark.parametrize("T", [1, 2, 3, 8, 9, 63, 64, 65, 127, 128, 129, 300])
def test_lengths_and_channels(T, C, types):
    x, log_a, h0, dhT, g = inputs(2, T, C, types, 7 * T + C)
    H, _ = check_forward(x, log_a, h0)
    check_forward(x, log_a)
    dH = torch.randn(2, T, C, generator=g, device=DEV).to(types[0])
    check_backward(log_a, H, dH, h0, dhT)
    check_backward(log_a, H, dH)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("B,T,C,reach", [(1, 5056, 64, 1000.0), (3, 4097, 136, 300.0), (2, 2000, 33, 100.0), (40, 700, 512, 50.0)])
def test_long_sequences(B, T, C, reach, types):
    """Tiles in turn over the CTAs of a cluster, and one CTA a column."""
    x, log_a, h0, dhT, g = inputs(B, T, C, types, T, reach)
    H, _ = check_forward(x, log_a, h0)
    check_backward(log_a, H, torch.randn(B, T, C, generator=g, device=DEV).to(types[0]), h0, dhT)


@pytest.mark.parametrize("types", TYPES)
def test_closed_gates_keep_packed_sequences_apart(types):
    B, T, C = 2, 777, 96
    x, log_a, h0, dhT, g = inputs(B, T, C, types, 3)
    starts = [0, 1, 5, 64, 300, 301, 776]
    log_a[:, starts] = -math.inf
    H, hT = check_forward(x, log_a, h0)
    dH = torch.randn(B, T, C, generator=g, device=DEV).to(types[0])
    check_backward(log_a, H, dH, h0, dhT)
    # what comes before a closed gate does not matter, whatever it is
    bad = x.clone()
    bad[:, 100:300] = math.nan
    bad[:, 64:100:3] = math.inf
    other, last = b.recurrence_forward(bad, log_a, h0=torch.full_like(h0, math.nan))
    assert torch.equal(other[:, 300:], H[:, 300:]) and torch.equal(other[:, :64], H[:, :64]) and torch.equal(last, hT)
    assert bool(torch.isnan(other[:, 100:300]).all())
    dbad, hbad = dH.clone(), H.clone()
    dbad[:, 301:776] = math.nan
    hbad[:, 301:775] = math.inf
    dX, dA, d0 = b.recurrence_backward(log_a, hbad, dbad, h0=h0, dhT=dhT)
    want = b.recurrence_backward(log_a, H, dH, h0=h0, dhT=dhT)
    for got, ref in zip((dX, dA), want):
        assert torch.equal(got[:, :301], ref[:, :301]) and torch.equal(got[:, 776:], ref[:, 776:])
    assert torch.equal(d0, want[2]) and bool((dA[:, starts] == 0).all())


def test_strong_decay_and_open_gates():
    x, log_a, h0, dhT, g = inputs(1, 500, 64, TYPES[2], 5)
    for value in (-1e30, -200.0, -104.0, -60.0, 0.0):
        check_forward(x, torch.full_like(log_a, value), h0)
        check_backward(torch.full_like(log_a, value), x, x, h0, dhT)


def test_single_tokens_continue_a_sequence():
    B, T, C = 5, 40, 136
    x, log_a, h0, _, _ = inputs(B, T, C, TYPES[0], 6)
    H, hT = check_forward(x, log_a, h0)
    state = h0.clone()
    for t in range(T):
        h, same = b.recurrence_forward(x[:, t], log_a[:, t], h0=state, hT=state)
        assert same.data_ptr() == state.data_ptr() and h.shape == (B, C)
        assert float((h.double() - H[:, t].double()).abs().max()) <= 2.0 ** -7 * float(H[:, t].abs().max())
    assert float((state - hT).abs().max()) <= 40 * TOKEN * float(hT.abs().max() + 3)
    check_forward(x[:, :1], log_a[:, :1], h0)
    # pieces of a prompt, the state handed on
    one, mid = b.recurrence_forward(x[:, :17], log_a[:, :17], h0=h0)
    two, last = b.recurrence_forward(x[:, 17:], log_a[:, 17:], h0=mid)
    assert float((last - hT).abs().max()) <= 40 * TOKEN * float(hT.abs().max() + 3)


def test_strides_and_outputs_in_place():
    g = generator(8)
    B, T, C = 2, 200, 64
    both = torch.randn(B, T, 3 * C, generator=g, device=DEV).bfloat16()
    both[..., C:2 * C] = -both[..., C:2 * C].abs() * 0.1
    keep = both.clone()
    x, log_a, rest = both.chunk(3, -1)
    H, hT = check_forward(x, log_a)
    assert torch.equal(both, keep)
    dH = torch.randn(B, T, C, generator=g, device=DEV).bfloat16()
    want = check_backward(log_a, H, dH)
    again, _ = b.recurrence_forward(x, log_a, H=x)                       # h in the place of x
    assert again.data_ptr() == x.data_ptr() and torch.equal(x, H) and torch.equal(rest, keep[..., 2 * C:])
    first = torch.zeros(B, C, device=DEV)
    got = b.recurrence_backward(log_a, H, dH, dhT=first, dX=dH, dlog_a=log_a, dh0=first)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and torch.equal(rest, keep[..., 2 * C:])
    # [T, batch, channels] rows, an odd first column, one gate for all sequences
    x = torch.randn(T, B, C, generator=g, device=DEV).transpose(0, 1)
    la = -torch.rand(1, T, C + 1, generator=g, device=DEV)[..., 1:].expand(B, T, C)
    check_forward(x, la)
    out = torch.full((B, T, C + 8), 5.0, device=DEV)
    check_forward(x, la, H=out[..., :C])
    assert bool((out[..., C:] == 5).all())


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("B,T,C", [(1, 2047, 512), (1, 2048, 512), (1, 2049, 520), (1, 4101, 1000), (1, 3000, 1032), (2, 3001, 264), (16, 2500, 24),
                                   (1, 9000, 8), (8, 2300, 72), (130, 600, 64), (40, 2100, 72),
                                   (1, 1500, 2304), (1, 1100, 2760), (1, 1300, 3201), (3, 700, 1608), (1, 2500, 1728)])
def test_few_channels(B, T, C, types):
    """Tiles of 64, 32 and 16 channels, the last ones in part beyond the row; clusters of every size."""
    x, log_a, h0, dhT, g = inputs(B, T, C, types, B + T + C, 100.0)
    room = torch.full((B, T, C + 8), 5.0, dtype=types[0], device=DEV)
    H, _ = check_forward(x, log_a, h0, H=room[..., :C])
    assert bool((room[..., C:] == 5).all())
    check_forward(x, log_a)
    dH = torch.randn(B, T, C, generator=g, device=DEV).to(types[0])
    check_backward(log_a, H, dH, h0, dhT)
    check_backward(log_a, H, dH)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", [96, 520, 2048])
def test_closed_gates_of_long_sequences(C, types):
    B, T = 1, 2600
    x, log_a, h0, dhT, g = inputs(B, T, C, types, 13, 100.0)
    log_a[:, [0, 1, 300, 301, 1500, 2599]] = -math.inf
    H, hT = check_forward(x, log_a, h0)
    dH = torch.randn(B, T, C, generator=g, device=DEV).to(types[0])
    check_backward(log_a, H, dH, h0, dhT)
    bad, hbad = x.clone(), H.clone()
    bad[:, 310:1500:7] = math.nan
    hbad[:, 301:1499] = math.inf
    dbad = dH.clone()
    dbad[:, 301:1400] = math.nan
    other, last = b.recurrence_forward(bad, log_a, h0=h0)
    assert torch.equal(other[:, :310], H[:, :310]) and torch.equal(other[:, 1500:], H[:, 1500:]) and torch.equal(last, hT)
    want = b.recurrence_backward(log_a, H, dH, h0=h0, dhT=dhT)
    got = b.recurrence_backward(log_a, hbad, dbad, h0=h0, dhT=dhT)
    for p, q in zip(got[:2], want):
        assert torch.equal(p[:, :301], q[:, :301]) and torch.equal(p[:, 1501:], q[:, 1501:])
    assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("B,T,C", [(1, 15, 136), (1, 17, 2048), (300, 32, 132), (300, 33, 132), (300, 63, 131), (300, 65, 132), (2000, 20, 65),
                                   (1200, 104, 132), (1200, 105, 132), (1200, 207, 132), (1200, 209, 132)])
def test_many_sequences(B, T, C, types):
    """A thread a sequence, and lengths at which tiles take over, of either direction."""
    x, log_a, h0, dhT, g = inputs(B, T, C, types, B + T)
    H, _ = check_forward(x, log_a, h0)
    check_forward(x, log_a)
    check_backward(log_a, H, torch.randn(B, T, C, generator=g, device=DEV).to(types[0]), h0, dhT)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", [64, 63])
def test_closed_gates_of_many_sequences(C, types):
    B, T = 700, 21
    x, log_a, h0, dhT, g = inputs(B, T, C, types, 12)
    log_a[::2, 9] = log_a[::3, 0] = log_a[::5, 20] = -math.inf
    H, hT = check_forward(x, log_a, h0)
    dH = torch.randn(B, T, C, generator=g, device=DEV).to(types[0])
    check_backward(log_a, H, dH, h0, dhT)
    bad, hbad = x.clone(), H.clone()
    bad[::2, 3:9] = math.nan
    hbad[::2, 8] = math.inf
    other, last = b.recurrence_forward(bad, log_a, h0=h0)
    assert torch.equal(other[:, 9:], H[:, 9:]) and torch.equal(last, hT) and bool(torch.isnan(other[::2, 3:9]).all())
    got, want = (b.recurrence_backward(log_a, h, dH, h0=h0, dhT=dhT) for h in (hbad, H))
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # outputs in the place of inputs, rows of [T, batch, channels]
    x, log_a = (v.transpose(0, 1).contiguous().transpose(0, 1) for v in (x, log_a))
    state = h0.clone()
    again, _ = b.recurrence_forward(x, log_a, h0=state, H=x, hT=state)
    assert torch.equal(again, H) and torch.equal(state, hT)
    end = dhT.clone()
    got = b.recurrence_backward(log_a, again, dH, h0=h0, dhT=end, dX=dH, dlog_a=log_a, dh0=end)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("types", TYPES)
def test_broadcast_and_overlapping_rows(types):
    """Inputs that repeat (stride 0 over sequences, over tokens) or overlap: no tensor map, an address each."""
    x, log_a, h0, dhT, g = inputs(3, 150, 64, types, 21)
    one, gate = x[:1].expand(3, 150, 64), log_a[:, :1].expand(3, 150, 64)
    H, _ = check_forward(one, gate, h0)
    check_backward(gate, one, H, h0, dhT)
    wide = torch.randn(3, 150 * 32 + 64, generator=g, device=DEV).to(types[0])
    slid = wide.as_strided((3, 150, 64), (wide.shape[1], 32, 1))
    H, _ = check_forward(slid, log_a, h0)
    check_backward(log_a, slid, slid, h0, dhT)


def test_gradients_against_differences():
    x, log_a, h0, dhT, g = inputs(1, 70, 5, TYPES[2], 9)
    dH = torch.randn(1, 70, 5, generator=g, device=DEV)
    H, _ = b.recurrence_forward(x, log_a, h0=h0)
    grads = b.recurrence_backward(log_a, H, dH, h0=h0, dhT=dhT)
    base = dict(x=x.double(), log_a=log_a.double(), h0=h0.double())

    def loss(**kw):
        v = {**base, **kw}
        h = walk(v["log_a"].exp(), v["x"], v["h0"])[1]
        return float((h * dH.double()).sum() + (h[:, -1] * dhT.double()).sum())

    for name, got in zip(("x", "log_a", "h0"), grads):
        e = torch.randn(got.shape, generator=g, device=DEV).double()
        s = 1e-4
        slope = (loss(**{name: base[name] + s * e}) - loss(**{name: base[name] - s * e})) / (2 * s)
        assert abs(slope - float((got.double() * e).sum())) <= 1e-5 * float((got.double() * e).abs().sum()), name


def test_same_from_run_to_run_and_rows_far_apart():
    x, log_a, h0, _, _ = inputs(1, 6000, 192, TYPES[0], 10)
    one, two = (b.recurrence_forward(x, log_a, h0=h0) for _ in range(2))
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    far = (1 << 31) + 64
    store = torch.empty(far + 16384, dtype=torch.bfloat16, device=DEV)
    wide = store.as_strided((2, 100, 64), (far, 64, 1))
    wide.copy_(torch.randn(2, 100, 64, generator=generator(11), device=DEV))
    H, _ = check_forward(wide, log_a[:, :100, :64].expand(2, 100, 64))
    check_backward(log_a[:, :100, :64].expand(2, 100, 64), wide, H)
    b.recurrence_forward(wide, log_a[:, :100, :64].expand(2, 100, 64), H=wide)
    assert torch.equal(wide, H)


def test_refusals():
    x = torch.zeros(2, 4, 64, device=DEV)
    s = torch.zeros(2, 64, device=DEV)
    bad = [dict(X=x.half()), dict(X=x[..., ::2]), dict(X=x[None]), dict(X=x[:, :0]), dict(log_a=x[:1]), dict(log_a=x.double()), dict(h0=s[:1]),
           dict(h0=s.bfloat16()), dict(h0=torch.zeros(64, 2, device=DEV).T), dict(hT=s[:, :32]), dict(H=x[:, :2]), dict(log_a=x.cpu())]
    for kw in bad:
        with pytest.raises(ValueError):
            b.recurrence_forward(**{**dict(X=x, log_a=x), **kw})
    for kw in (dict(log_a=x.bfloat16()), dict(H=x[:1, :1].expand(2, 4, 64))):      # gates narrower than the rows; overlapping rows
        with pytest.raises(b.SmatError):
            b.recurrence_forward(**{**dict(X=x, log_a=x), **kw})
    for kw in (dict(H=x[:1]), dict(dH=x[:1]), dict(dhT=s[:1]), dict(dX=x[:1]), dict(dlog_a=x.bfloat16()), dict(dh0=s[:1])):
        with pytest.raises(ValueError):
            b.recurrence_backward(**{**dict(log_a=x, H=x, dH=x), **kw})


def test_streams_and_graphs():
    x, log_a, h0, dhT, _ = inputs(2, 3000, 256, TYPES[0], 12)
    want = b.recurrence_forward(x, log_a, h0=h0)
    grads = b.recurrence_backward(log_a, want[0], x, h0=h0, dhT=dhT)
    got = []
    for s in [torch.cuda.Stream() for _ in range(2)]:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(4):
                got.append(b.recurrence_forward(x, log_a, h0=h0) + b.recurrence_backward(log_a, want[0], x, h0=h0, dhT=dhT))
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for r in got for p, q in zip(want + grads, r))
    graph, xs, state = torch.cuda.CUDAGraph(), x.clone(), h0.clone()
    with torch.cuda.graph(graph):
        h, _ = b.recurrence_forward(xs, log_a, h0=state, hT=state)
        back = b.recurrence_backward(log_a, h, xs, h0=h0, dhT=dhT)
    state.copy_(h0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    second = b.recurrence_forward(x, log_a, h0=want[1])
    assert torch.equal(h, second[0]) and torch.equal(state, second[1])
    assert all(torch.equal(p, q) for p, q in zip(back, b.recurrence_backward(log_a, h, x, h0=h0, dhT=dhT)))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("B,T,C", [(1, 12, 64), (300, 40, 132), (1, 300, 63), (2, 500, 64), (1, 1500, 2304), (1, 4101, 72), (1, 9000, 8), (1, 3000, 520),
                                   (130, 600, 64), (3, 700, 1608)])
@pytest.mark.parametrize("decay", [-2.0, -12.0, -60.0, -100.0])
def test_open_gates_forget_nothing_that_is_not_finite(decay, B, T, C, types):
    """Products of open gates are zero in fp32 behind a few tokens; only a closed gate ends what is not finite, wherever the pieces of a
    sequence meet, and a gate that is NaN is as if it were open."""
    x, log_a, h0, dhT, g = inputs(B, T, C, types, 31)
    log_a.fill_(decay)
    closed, bad = T // 3, 3 * T // 4
    log_a[:, closed] = -math.inf
    H, _ = b.recurrence_forward(x, log_a, h0=h0)
    assert bool(torch.isfinite(H).all())
    wrong, start = x.clone(), h0.clone()
    wrong[:, bad, ::2] = math.nan
    wrong[:, bad, 1::2] = math.inf
    start[:, ::2] = -math.inf
    start[:, 1::2] = math.nan
    K, hT = b.recurrence_forward(wrong, log_a, h0=start)
    assert not bool(torch.isfinite(K[:, :closed]).any()) and not bool(torch.isfinite(K[:, bad:]).any()) and not bool(torch.isfinite(hT).any())
    assert torch.equal(K[:, closed:bad], H[:, closed:bad])
    assert bool((K[:, bad:, 1::2] == math.inf).all()) and bool((K[:, :closed, ::2] == -math.inf).all())
    # a NaN among the gates, and the closed one behind it
    odd = log_a.clone()
    odd[:, closed // 2] = math.nan
    K, _ = b.recurrence_forward(x, odd, h0=h0)
    assert bool(torch.isnan(K[:, closed // 2:closed]).all()) and torch.equal(K[:, :closed // 2], H[:, :closed // 2]) and torch.equal(K[:, closed:], H[:, closed:])
    # gradients: from the last token to the first
    dH = torch.randn(B, T, C, generator=g, device=DEV).to(types[0])
    one = torch.ones_like(H)
    dX, dA, d0 = b.recurrence_backward(log_a, one, dH, h0=h0, dhT=dhT)
    assert bool(torch.isfinite(dX).all())
    wrong, end = dH.clone(), dhT.clone()
    wrong[:, closed // 2, ::2] = math.nan
    wrong[:, closed // 2, 1::2] = math.inf
    end[:, ::2] = math.inf
    end[:, 1::2] = math.nan
    eX, eA, e0 = b.recurrence_backward(log_a, one, wrong, h0=h0, dhT=end)
    for k in (eX, eA):
        assert not bool(torch.isfinite(k[:, :closed // 2 + 1]).any()) and not bool(torch.isfinite(k[:, closed + 1:]).any())
    assert not bool(torch.isfinite(e0).any()) and not bool(torch.isfinite(eX[:, closed]).any()) and bool((eA[:, closed] == 0).all())
    assert torch.equal(eX[:, closed // 2 + 1:closed], dX[:, closed // 2 + 1:closed]) and torch.equal(eA[:, closed // 2 + 1:closed], dA[:, closed // 2 + 1:closed])


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("B,T,C", [(6, 1023, 13), (1, 20, 100), (1, 3000, 12), (2, 300, 66), (1, 2500, 516), (3, 700, 1601), (1, 5000, 1)])
def test_what_lies_behind_a_row_stays(B, T, C, types):
    """Rows a multiple of 16 bytes apart, whose last element is not the last of 16 bytes: nothing behind it is written."""
    x, log_a, h0, dhT, g = inputs(B, T, C, types, B + T + C, 100.0)
    wide = (C // 8 + 1) * 8

    def apart(v):
        room = torch.full((B, T, wide), 5.0, dtype=v.dtype, device=DEV)
        room[..., :C] = v
        return room, room[..., :C]

    (_, x), (_, log_a) = apart(x), apart(log_a)
    room, H = apart(torch.zeros_like(x))
    check_forward(x, log_a, h0, H=H)
    assert bool((room[..., C:] == 5).all())
    _, dH = apart(torch.randn(B, T, C, generator=g, device=DEV).to(types[0]))
    (dx_room, dX), (da_room, dA) = apart(torch.zeros_like(x)), apart(torch.zeros_like(log_a))
    check_backward(log_a, H, dH, h0, dhT, dX=dX, dlog_a=dA)
    assert bool((dx_room[..., C:] == 5).all()) and bool((da_room[..., C:] == 5).all())
    keep = x.clone()
    room, y = apart(x)
    again, _ = b.recurrence_forward(y, log_a, h0=h0, H=y)                       # in the place of x
    assert torch.equal(again, H) and bool((room[..., C:] == 5).all()) and torch.equal(x, keep)
