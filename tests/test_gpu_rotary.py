"""Rotary positions on the GPU against the definition in 64 bits."""
import pytest
import torch

from paper_2609_36062_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def turned(x, at, f, interleaved, scale, adjoint):
    """Rows x [batch, heads, T, d] in 64 bits; at [batch or 1, T]; and the bound on what is left: of fp32, the products and their sum
    (three roundings of 2^-24), the fraction of a turn (pi 2^-24) and sincospi (two units); of fp64, three roundings of the
    angle by the operator and one here."""
    n = 2 * f.numel()
    x = x.double()
    angle = at[:, None, :, None].double() * f * (-1.0 if adjoint else 1.0)
    c, s = torch.cos(angle) * scale, torch.sin(angle) * scale
    one, two = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    y, slack = x.clone(), torch.zeros_like(x)
    u, v = x[..., one], x[..., two]
    y[..., one], y[..., two] = u * c - v * s, v * c + u * s
    slack[..., one] = slack[..., two] = (u.abs() + v.abs()) * abs(scale) * (2.0 ** -20 + 4 * 2.0 ** -53 * angle.abs())
    return y, slack


def check(got, x, at, f, interleaved=False, scale=1.0, adjoint=False):
    want, slack = turned(x, at, f, interleaved, scale, adjoint)
    off = (got.double() - want).abs() - (HALF[x.dtype] * want.abs() + slack)
    assert float(off.max()) <= 0.0, float(off.max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotated", [(128, 128), (128, 64), (64, 64), (64, 16), (128, 2), (128, 90), (96, 40), (7, 6), (1 + 2, 2), (512, 512), (511, 2)])
def test_layouts_and_widths(d, rotated, interleaved, dtype):
    g = generator(d + rotated)
    f, scale = b.rotary_frequencies(rotated, scaling="yarn", factor=8.0)
    q, k = (torch.randn(2, h, 37, d, generator=g, device=DEV).to(dtype) for h in (3, 2))
    at = torch.arange(11, 48, device=DEV)[None]
    for adjoint in (False, True):
        out = b.rotary(q, k, f, first=11, interleaved=interleaved, scale=scale, adjoint=adjoint)
        for got, x in zip(out, (q, k)):
            assert got.is_contiguous() and got.dtype == dtype
            check(got, x, at, f, interleaved, scale, adjoint)


@pytest.mark.parametrize("T,batch,heads", [(1, 1, 1), (1, 33, 16), (2, 3, 5), (255, 1, 8), (257, 2, 1), (5056, 1, 2)])
def test_lengths(T, batch, heads):
    g = generator(T)
    f, _ = b.rotary_frequencies(64)
    q = torch.randn(batch, heads, T, 64, generator=g, device=DEV).bfloat16()
    at = torch.randint(0, 1 << 20, (batch, T), generator=g, device=DEV)
    check(b.rotary(q, None, f, positions=at), q, at, f)
    check(b.rotary(q, None, f, positions=at[0].contiguous()), q, at[:1], f)
    check(b.rotary(q, None, f, positions=at[:1].expand(batch, T)), q, at[:1], f)
    check(b.rotary(q, None, f), q, torch.arange(T, device=DEV)[None], f)


@pytest.mark.parametrize("far", [0, 4095, 1 << 20, (1 << 31) - 64, 1 << 40, -70000])
def test_far_positions(far):
    """The angle keeps its place in the turn at any position (a product in fp32 would be off by far * 2^-24 radians)."""
    g = generator(3)
    f, _ = b.rotary_frequencies(128)
    q = torch.randn(1, 2, 40, 128, generator=g, device=DEV)
    at = torch.arange(far, far + 40, device=DEV)[None]
    check(b.rotary(q, None, f, first=far), q, at, f)
    check(b.rotary(q, None, f, positions=at), q, at, f)


def test_strides_of_projections_and_outputs():
    g = generator(4)
    f, _ = b.rotary_frequencies(128)
    B, T, H = 2, 130, 4
    at = torch.arange(T, device=DEV)[None]
    packed = torch.randn(B, T, 3 * H, 128, generator=g, device=DEV).bfloat16()
    q, k, v = packed.transpose(1, 2).chunk(3, 1)
    before = packed.clone()
    got = b.rotary(q, k, f)
    check(got[0], q, at, f)
    check(got[1], k, at, f)
    assert torch.equal(packed, before)
    # into the rows of another layout, beside what is not to be touched
    out = torch.full((B, T, 3 * H, 128), 7.0, device=DEV).bfloat16()
    qo, ko, rest = out.transpose(1, 2).chunk(3, 1)
    r = b.rotary(q, k, f, Q_out=qo, K_out=ko)
    assert r[0].data_ptr() == qo.data_ptr() and torch.equal(qo, got[0]) and torch.equal(ko, got[1]) and bool((rest == 7).all())
    # in place, of the packed rows
    b.rotary(q, k, f, Q_out=q, K_out=k)
    assert torch.equal(q, got[0]) and torch.equal(k, got[1]) and torch.equal(v, before.transpose(1, 2)[:, 2 * H:])
    # broadcast heads, odd offsets: an element at a time
    one = torch.randn(B, 1, T, 128, generator=g, device=DEV)
    check(b.rotary(one.expand(B, H, T, 128), None, f), one.expand(B, H, T, 128), at, f)
    odd = torch.randn(B * H * T * 128 + 3, generator=g, device=DEV).bfloat16()[3:].view(B, H, T, 128)
    check(b.rotary(odd, None, f), odd, at, f)


def test_in_place_leaves_the_other_columns():
    f, _ = b.rotary_frequencies(30)
    x = torch.randn(2, 3, 9, 64, generator=generator(5), device=DEV)
    keep = x.clone()
    b.rotary(x, None, f, first=3, Q_out=x)
    assert torch.equal(x[..., 30:], keep[..., 30:])
    check(x, keep, torch.arange(3, 12, device=DEV)[None], f)


def test_values_that_are_not_finite_stay_in_their_pair():
    f, _ = b.rotary_frequencies(64)
    x = torch.randn(1, 1, 4, 128, generator=generator(6), device=DEV)
    x[0, 0, 1, 5], x[0, 0, 2, 100] = float("inf"), float("nan")
    y = b.rotary(x, None, f, first=1)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[0, 0, 1, 5] = want[0, 0, 1, 37] = want[0, 0, 2, 100] = True
    assert torch.equal(bad, want)


def test_single_tokens():
    g = generator(7)
    f, _ = b.rotary_frequencies(128)
    q, k = (torch.randn(5, h, 128, generator=g, device=DEV).bfloat16() for h in (16, 4))
    at = torch.tensor([0, 9, 4000, 65535, 3], device=DEV)
    out = b.rotary(q, k, f, positions=at)
    for got, x in zip(out, (q, k)):
        assert got.shape == x.shape
        check(got[:, :, None], x[:, :, None], at[:, None], f)
    again = b.rotary(q[:, :, None], k[:, :, None], f, positions=at[:, None])
    assert torch.equal(again[0][:, :, 0], out[0]) and torch.equal(again[1][:, :, 0], out[1])
    check(b.rotary(q, None, f, first=12)[:, :, None], q[:, :, None], torch.full((1, 1), 12, device=DEV), f)


def test_adjoint_is_the_gradient():
    g = generator(8)
    f, scale = b.rotary_frequencies(32, scaling="yarn", factor=4.0)
    x, dy = (torch.randn(1, 2, 9, 48, generator=g, device=DEV) for _ in range(2))
    dx = b.rotary(dy, None, f, first=5, scale=scale, adjoint=True).double()
    # <dy, R x> = <dx, x> for the linear map, and differences of it along a direction
    step = torch.randn(1, 2, 9, 48, generator=g, device=DEV).double() * 0.125
    at = torch.arange(5, 14, device=DEV)[None]
    up, down = (turned(x.double() + s * step, at, f, False, scale, False)[0] for s in (1, -1))
    assert abs(float((dy.double() * (up - down)).sum() / 2 - (dx * step).sum())) <= 2.0 ** -20 * float((dx * step).abs().sum())


def test_rows_far_apart():
    """The second sequence begins behind element 2^31."""
    far = (1 << 31) + 64
    f, _ = b.rotary_frequencies(64)
    store = torch.empty(far + 4096, dtype=torch.bfloat16, device=DEV)
    x = store.as_strided((2, 2, 16, 64), (far, 1024, 64, 1))
    x.copy_(torch.randn(2, 2, 16, 64, generator=generator(9), device=DEV))
    keep = x.clone()
    y = b.rotary(x, None, f)
    check(y, keep, torch.arange(16, device=DEV)[None], f)
    b.rotary(x, None, f, Q_out=x)
    assert torch.equal(x, y)


def test_refusals():
    f, _ = b.rotary_frequencies(64)
    q = torch.zeros(2, 3, 8, 64, device=DEV)
    bad = [dict(Q=q.half()), dict(Q=q[..., ::2]), dict(Q=q[:, :, :0]), dict(Q=q[0, 0]), dict(K=q[:, :, :4].contiguous()), dict(K=q.bfloat16()),
           dict(K=q[:1]), dict(frequencies=f.float()), dict(frequencies=f.cpu()), dict(frequencies=f[::2]), dict(Q_out=q[:, :, :4]),
           dict(positions=torch.arange(7, device=DEV)), dict(positions=torch.arange(8)), dict(positions=torch.arange(8, device=DEV).int()),
           dict(positions=torch.arange(16, device=DEV)[::2])]
    for kw in bad:
        with pytest.raises(ValueError):
            b.rotary(**{**dict(Q=q, K=None, frequencies=f), **kw})
    for kw in (dict(frequencies=torch.ones(33, dtype=torch.float64, device=DEV)), dict(Q_out=torch.zeros(1, 1, 8, 64, device=DEV).expand(2, 3, 8, 64))):
        with pytest.raises(b.SmatError):
            b.rotary(**{**dict(Q=q, K=None, frequencies=f), **kw})


def test_streams_and_graphs():
    g = generator(10)
    f, _ = b.rotary_frequencies(128)
    q, k = (torch.randn(4, 8, 128, generator=g, device=DEV).bfloat16() for _ in range(2))
    at = torch.tensor([1, 2, 3, 4], device=DEV)
    want = b.rotary(q, k, f, positions=at + 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        inside = b.rotary(q, k, f, positions=at + 1)
    given = b.rotary(q, k, f, positions=at + 1, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(want, inside, given))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.rotary(q, k, f, positions=at)
        at.add_(1)
    at.copy_(torch.tensor([1, 2, 3, 4], device=DEV) + 1)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, out))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], b.rotary(q, None, f, positions=torch.tensor([3, 4, 5, 6], device=DEV)))
