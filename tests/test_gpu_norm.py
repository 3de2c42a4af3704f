"""Norms around a block on the GPU against the formulas in 64 bits, gradients against differences too."""
import pytest
import torch

from paper_2609_36062_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
EPS = 1e-6
# Relative error of a row's sums and factors in fp32: at most 64 products in a lane, 10 more sums across lanes and warps
# (74 * 2^-24, halved by the root), rsqrt within 2 units, exp and division of the gate within 2^-20 at the gates drawn here.
ROW = 2.0 ** -17
# ... and of sums over rows: a CTA's rows in turn, its slots, the partial rows of all CTAs, at most 110 sums here (2^-17).
SUMS = 2.0 ** -16


def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def act(kind, z):
    s = torch.sigmoid(z)
    return (s, s * (1 - s)) if kind == "sigmoid" else (z * s, s * (1 + z * (1 - s)))


def forward64(x, w, residual=None, scale=None, gate=None, kind="silu", eps=EPS):
    h = x.double() * (1.0 if scale is None else scale.double())
    h = h if residual is None else h + residual.double()
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + eps) * w.double()
    return (y if gate is None else y * act(kind, gate.double())[0]), h


def near(got, want, slack, name):
    off = (got.double() - want).abs() - (HALF.get(got.dtype, 0.0) * want.abs() + slack)
    assert got.shape == want.shape and float(off.max()) <= 0.0, (name, float(off.max()))


def check_forward(x, w, residual=None, scale=None, gate=None, kind="silu", **out):
    got = b.norm_forward(x, w, EPS, residual=residual, scale=scale, gate=gate, activation=kind, **out)
    want, h = forward64(x, w, residual, scale, gate, kind)
    y, kept = got if isinstance(got, tuple) else (got, None)
    # h = residual + scale x: two roundings of its terms, seen through the row's factor
    terms = x.double().abs() * (1.0 if scale is None else scale.double().abs()) + (0.0 if residual is None else residual.double().abs())
    through = w.double().abs() / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS) * (1.0 if gate is None else act(kind, gate.double())[0].abs())
    near(y, want, ROW * want.abs() + 2.0 ** -23 * terms * through, "y")
    if kept is not None:
        near(kept, h, 2.0 ** -23 * terms, "h")
    return got


def check_backward(dy, h, w, gate=None, kind="silu", dh_in=None, x=None, scale=None, **out):
    dH, dX, dW, dS, dG = b.norm_backward(dy, h, w, EPS, gate=gate, activation=kind, dH=dh_in, X=x, scale=scale, **out)
    y64, h64, w64 = dy.double(), h.double(), w.double()
    r = 1 / torch.sqrt(h64.square().mean(-1, keepdim=True) + EPS)
    n = h64 * r
    f, slope = (1.0, 0.0) if gate is None else act(kind, gate.double())
    u = y64 * f
    dn = u * w64
    m = (dn * n).mean(-1, keepdim=True)
    terms = r * (dn.abs() + n.abs() * (dn * n).abs().mean(-1, keepdim=True))
    want = r * (dn - n * m)
    if dh_in is not None:
        want, terms = want + dh_in.double(), terms + dh_in.double().abs()
    near(dH, want, ROW * terms, "dh")
    along = tuple(range(h.dim() - w.dim()))
    if w.dim() == 2 and h.dim() == 3:
        along = (0,)
    near(dW, (u * n).sum(along), SUMS * (u * n).abs().sum(along), "dw")
    if gate is not None:
        near(dG, y64 * n * w64 * slope, ROW * (y64 * n * w64).abs() * (1 + gate.double().abs()), "dgate")
    else:
        assert dG is None
    if scale is None:
        assert dX is dH or dX.data_ptr() == dH.data_ptr()
        assert dS is None
    else:
        near(dX, want * scale.double(), ROW * terms * scale.double().abs(), "dx")
        along = tuple(range(h.dim() - 1))
        near(dS, (want * x.double()).sum(along), SUMS * (terms * x.double().abs()).sum(along), "dscale")
    return dH, dX, dW, dS, dG


WIDTHS = [1, 2, 7, 8, 64, 100, 128, 136, 250, 255, 256, 264, 512, 1000, 1024, 1028, 2048, 4096, 4099, 4104, 8192, 8193, 12000, 16384]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", WIDTHS)
def test_residual_and_scale(width, dtype):
    g = generator(width)
    B, T = (2, 37) if width < 5000 else (1, 5)
    rows = lambda: torch.randn(B, T, width, generator=g, device=DEV).to(dtype)
    x, residual, dy, dh_in = rows(), rows(), rows(), rows()
    w, scale = (torch.randn(width, generator=g, device=DEV) for _ in range(2))
    check_forward(x, w)
    check_forward(x, w, scale=scale)
    check_forward(x, w, residual=residual)
    _, h = check_forward(x, w, residual=residual, scale=scale)
    check_backward(dy, h, w, dh_in=dh_in, x=x, scale=scale)
    check_backward(dy, h, w, dh_in=dh_in)
    check_backward(dy, x, w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["silu", "sigmoid"])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("B,T,G,width", [(1, 1, 1, 128), (2, 70, 16, 128), (3, 33, 8, 64), (1, 300, 5, 72), (2, 9, 3, 33), (1, 4, 70, 2048)])
def test_gate_of_heads(B, T, G, width, grouped, kind, dtype):
    g = generator(T + width)
    # rows as the attention pass leaves them, [batch, heads, T, width]
    x = torch.randn(B, G, T, width, generator=g, device=DEV).to(dtype).transpose(1, 2)
    gate, dy = ((torch.randn(B, T, G, width, generator=g, device=DEV) * 3).to(dtype) for _ in range(2))
    w = torch.randn(*((G, width) if grouped else (width,)), generator=g, device=DEV)
    y = check_forward(x, w, gate=gate, kind=kind)
    assert y.is_contiguous()
    check_backward(dy, x, w, gate=gate, kind=kind)


def test_many_rows_and_partial_sums():
    """More rows than the backward pass has CTAs, several times over: sums of dweight and dscale over all of them, twice the same."""
    g = generator(1)
    B, T, width = 3, 3001, 256
    x, h, dy, dh_in = (torch.randn(B, T, width, generator=g, device=DEV).bfloat16() for _ in range(4))
    w, scale = (torch.randn(width, generator=g, device=DEV) for _ in range(2))
    one = check_backward(dy, h, w, dh_in=dh_in, x=x, scale=scale)
    two = b.norm_backward(dy, h, w, EPS, dH=dh_in, X=x, scale=scale)
    assert all(torch.equal(p, q) for p, q in zip(one[:4], two[:4]))
    ws = torch.empty(b.norm_workspace_bytes(width, scale=True), dtype=torch.uint8, device=DEV)
    three = b.norm_backward(dy, h, w, EPS, dH=dh_in, X=x, scale=scale, workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(one[:4], three[:4]))
    with pytest.raises(b.SmatError) as err:
        b.norm_backward(dy, h, w, EPS, workspace=ws[:1024])
    assert err.value.code == 5


@pytest.mark.parametrize("shape", [(5, 192), (3, 7, 192), (2, 3, 4, 192)])
def test_shapes(shape):
    g = generator(2)
    x, dy = (torch.randn(*shape, generator=g, device=DEV) for _ in range(2))
    w = torch.randn(192, generator=g, device=DEV)
    check_forward(x, w)
    check_backward(dy, x, w)


def test_single_tokens_of_heads():
    g = generator(3)
    x, gate, dy = (torch.randn(6, 16, 128, generator=g, device=DEV).bfloat16() for _ in range(3))
    w = torch.randn(16, 128, generator=g, device=DEV)
    check_forward(x, w, gate=gate)
    check_backward(dy, x, w, gate=gate)


def test_outputs_in_the_place_of_inputs():
    g = generator(4)
    new = lambda: torch.randn(2, 50, 3, 128, generator=g, device=DEV).bfloat16()
    x, residual, gate, dy, dh_in = new(), new(), new(), new(), new()
    w, scale = (torch.randn(128, generator=g, device=DEV) for _ in range(2))
    y, h = b.norm_forward(x, w, residual=residual, scale=scale, gate=gate)
    r, z = residual.clone(), gate.clone()
    y2, h2 = b.norm_forward(x, w, residual=r, scale=scale, gate=z, Y=z, H=r)
    assert y2.data_ptr() == z.data_ptr() and h2.data_ptr() == r.data_ptr() and torch.equal(y, y2) and torch.equal(h, h2)
    want = b.norm_backward(dy, h, w, gate=gate, dH=dh_in, X=x, scale=scale)
    a, c, e = dy.clone(), dh_in.clone(), gate.clone()
    got = b.norm_backward(a, h, w, gate=e, dH=c, X=x, scale=scale, dH_out=c, dX=a, dgate=e)
    assert got[0].data_ptr() == c.data_ptr() and all(torch.equal(p, q) for p, q in zip(want, got))


def test_strided_and_broadcast_rows():
    g = generator(5)
    wide = torch.randn(2, 40, 4 * 128 + 8, generator=g, device=DEV).bfloat16()
    x = wide[..., 128:256]                                     # part of a projection's columns
    w = torch.randn(128, generator=g, device=DEV)
    check_forward(x, w)
    check_forward(wide[..., 3:131], w)                         # ... from an odd column: an element at a time
    one = torch.randn(1, 1, 128, generator=g, device=DEV).bfloat16()
    check_forward(x, w, residual=one.expand(2, 40, 128))
    out = torch.full((2, 40, 256), 9.0, device=DEV).bfloat16()
    check_forward(x, w, Y=out[..., :128])
    assert bool((out[..., 128:] == 9).all())
    check_backward(wide[..., :128], x, w, dh_in=one.expand(2, 40, 128))


def test_rows_of_zeros_and_rows_that_are_not_finite():
    x = torch.randn(1, 4, 128, generator=generator(6), device=DEV)
    x[0, 1] = 0.0
    x[0, 2, 5] = float("nan")
    w = torch.ones(128, device=DEV)
    y = b.norm_forward(x, w)
    assert bool((y[0, 1] == 0).all()) and bool(torch.isnan(y[0, 2]).all()) and bool(torch.isfinite(y[0, [0, 3]]).all())
    dh = b.norm_backward(torch.ones_like(x), x, w)[0]
    assert bool(torch.isfinite(dh[0, [0, 1, 3]]).all())
    near(dh[:, 1], torch.full_like(dh[:, 1], EPS ** -0.5).double(), ROW * EPS ** -0.5, "dh of zeros")


@pytest.mark.parametrize("width", [64, 128, 130, 1000, 2048])
def test_without_epsilon(width):
    """eps = 0 with fewer rows than a CTA has places for: the empty ones leave the sums over rows alone."""
    g = generator(11)
    x, dy, dh_in = (torch.randn(1, 3, width, generator=g, device=DEV) for _ in range(3))
    w, scale = (torch.randn(width, generator=g, device=DEV) for _ in range(2))
    near(b.norm_forward(x, w, eps=0.0), forward64(x, w, eps=0.0)[0], ROW * forward64(x, w, eps=0.0)[0].abs(), "y")
    dH, dX, dW, dS, _ = b.norm_backward(dy, x, w, eps=0.0, dH=dh_in, X=x, scale=scale)
    n = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True))
    near(dW, (dy.double() * n).sum((0, 1)), SUMS * (dy.double() * n).abs().sum((0, 1)), "dw")
    assert bool(torch.isfinite(dH).all()) and bool(torch.isfinite(dX).all()) and bool(torch.isfinite(dS).all())


def test_gradients_against_differences():
    """d/ds of <dy, y(h + s e)> and the like by central differences of the 64-bit formula (error s^2: 1e-6)."""
    g = generator(7)
    x, residual, gate, dy, dh_in = (torch.randn(1, 3, 2, 48, generator=g, device=DEV) for _ in range(5))
    w = torch.randn(2, 48, generator=g, device=DEV)
    scale = torch.randn(48, generator=g, device=DEV)
    h = forward64(x, w, residual, scale)[1].float()
    grads = b.norm_backward(dy, h, w, EPS, gate=gate, dH=dh_in, X=x, scale=scale)
    base = dict(x=x.double(), w=w.double(), residual=(h.double() - x.double() * scale.double()), scale=scale.double(), gate=gate.double())

    def loss(**kw):
        y, hh = forward64(kind="silu", **{**base, **kw})
        return float((y * dy.double()).sum() + (hh * dh_in.double()).sum())

    for name, got in zip(("residual", "x", "w", "scale", "gate"), grads):
        e = torch.randn(got.shape, generator=g, device=DEV).double()
        s = 1e-4
        slope = (loss(**{name: base[name] + s * e}) - loss(**{name: base[name] - s * e})) / (2 * s)
        assert abs(slope - float((got.double() * e).sum())) <= 1e-5 * float((got.double() * e).abs().sum()), name


def test_rows_far_apart():
    far = (1 << 31) + 64
    store = torch.empty(far + 4096, dtype=torch.bfloat16, device=DEV)
    x = store.as_strided((2, 4, 128), (far, 128, 1))
    x.copy_(torch.randn(2, 4, 128, generator=generator(8), device=DEV))
    w = torch.ones(128, device=DEV)
    y = check_forward(x, w)
    dh = check_backward(y, x, w)[0]
    b.norm_forward(x, w, Y=x)
    assert torch.equal(x, y) and bool(torch.isfinite(dh).all())


def test_refusals():
    x, w = torch.zeros(2, 4, 64, device=DEV), torch.ones(64, device=DEV)
    f = lambda **kw: b.norm_forward(**{**dict(X=x, weight=w), **kw})
    k = lambda **kw: b.norm_backward(**{**dict(dY=x, H=x, weight=w), **kw})
    bad = [lambda: f(X=x.half()), lambda: f(X=x[..., ::2]), lambda: f(X=x[0, 0]), lambda: f(X=x[:, :0]), lambda: f(weight=w.bfloat16()),
           lambda: f(weight=w[:32]), lambda: f(weight=w.cpu()), lambda: f(weight=torch.ones(3, 64, device=DEV)), lambda: f(residual=x[:1]),
           lambda: f(gate=x.bfloat16()), lambda: f(scale=w[:1]), lambda: f(Y=x[:1]), lambda: f(activation="tanh"),
           lambda: f(X=x[0], weight=torch.ones(4, 64, device=DEV)), lambda: k(dY=x[:1]), lambda: k(scale=w), lambda: k(dH=x.bfloat16()),
           lambda: k(gate=x, dgate=x[:1]), lambda: k(workspace=torch.zeros(1 << 20, dtype=torch.uint8)),
           lambda: k(workspace=torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)[::2])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
    for call in (lambda: f(eps=-1.0), lambda: f(Y=x[:1, :1].expand(2, 4, 64)), lambda: f(X=torch.zeros(1, 16385, device=DEV), weight=torch.ones(16385, device=DEV))):
        with pytest.raises(b.SmatError):
            call()


def test_streams_and_graphs():
    g = generator(9)
    x, dy = (torch.randn(4, 600, 512, generator=g, device=DEV).bfloat16() for _ in range(2))
    w = torch.randn(512, generator=g, device=DEV)
    want = b.norm_backward(dy, x, w)
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in sides:                                       # two at once, each with a workspace of its own
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(5):
                got.append(b.norm_backward(dy, x, w))
    torch.cuda.synchronize()
    assert all(torch.equal(want[i], r[i]) for r in got for i in (0, 2))
    graph = torch.cuda.CUDAGraph()
    kept = x.clone()
    with torch.cuda.graph(graph):
        y = b.norm_forward(kept, w)
        out = b.norm_backward(dy, kept, w)
    kept.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    again = b.norm_backward(dy, x.flip(0), w)
    assert torch.equal(y, b.norm_forward(x.flip(0), w)) and torch.equal(out[0], again[0]) and torch.equal(out[2], again[2])
