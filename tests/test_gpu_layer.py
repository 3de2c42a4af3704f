"""The operators in a row, as a model runs them: norm, projections, rotary positions, attention pass, gated norm, projection, residual,
a recurrent layer between; forward and gradients against 64 bits, and the same tokens one at a time on a packed cache."""
import math

import pytest
import torch

from oracle import smat_oracle as so
from paper_2609_36062_b200 import binding as b

pytestmark = pytest.mark.gpu
B, T, HEADS, HEAD, WIDTH, D, CHUNK = 2, 512, 2, 64, 96, 2, 64


def weights(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda") / math.sqrt(s[0])
    W = {"qkvz": new(WIDTH, 4 * HEADS * HEAD), "out": new(HEADS * HEAD, WIDTH), "mix": new(WIDTH, 2 * WIDTH)}
    P = {"norm": 1 + 0.1 * new(WIDTH) * math.sqrt(WIDTH), "head": 1 + 0.1 * torch.randn(HEADS, HEAD, generator=g, device="cuda"),
         "scale": 0.5 + 0.1 * torch.randn(WIDTH, generator=g, device="cuda"), "last": torch.ones(WIDTH, device="cuda")}
    x = torch.randn(B, T, WIDTH, generator=g, device="cuda")
    dy = torch.randn(B, T, WIDTH, generator=g, device="cuda")
    return {k: w.to(dtype) for k, w in W.items()}, P, x.to(dtype), dy.to(dtype)


def gates(z):
    """Log-gates of the recurrent layer from its projection."""
    return -torch.nn.functional.softplus(z) * 0.1


def model64(W, P, x, f):
    """The same layer in 64 bits with the dense mask."""
    rms = lambda h, w: h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * w
    M = torch.from_numpy(so.dense_mask(T, CHUNK, D)).double().cuda()
    angle = torch.arange(T, device="cuda", dtype=torch.float64)[:, None] * f
    c, s = torch.cos(angle), torch.sin(angle)
    n = f.numel()
    turn = lambda u: torch.cat((u[..., :n] * c - u[..., n:2 * n] * s, u[..., n:2 * n] * c + u[..., :n] * s, u[..., 2 * n:]), -1)
    y = rms(x, P["norm"])
    q, k, v, z = (y @ W["qkvz"]).view(B, T, 4 * HEADS, HEAD).transpose(1, 2).chunk(4, 1)
    o = (M * (turn(q) / HEAD @ turn(k).transpose(-1, -2))) @ v
    a = (rms(o.transpose(1, 2), P["head"]) * torch.nn.functional.silu(z.transpose(1, 2))).reshape(B, T, -1) @ W["out"]
    h = x + P["scale"] * a
    m = rms(h, P["last"]) @ W["mix"]
    u, la = m.chunk(2, -1)[0], gates(m.chunk(2, -1)[1])
    state, rows = torch.zeros_like(u[:, 0]), []
    for t in range(T):
        state = la[:, t].exp() * state + u[:, t]
        rows.append(state)
    return h + torch.stack(rows, 1)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 6e-2)])
def test_a_layer_forward_and_backward(dtype, tol):
    """Norms of the differences over norms: fp32, products of up to 512 terms in a chain of a dozen operators (each about 1e-6);
    bf16, some fifteen roundings of 2^-8 in a row, the norm behind the attention dividing by rows that differ in size."""
    W, P, x, dy = weights(dtype)
    f, _ = b.rotary_frequencies(32)
    plan = b.SmatPlan(B, HEADS, T, HEAD, HEAD, D, CHUNK, "f32" if dtype == torch.float32 else "bf16")
    torch.backends.cuda.matmul.allow_tf32 = False
    # forward
    y = b.norm_forward(x, P["norm"])
    q, k, v, z = (y.view(-1, WIDTH) @ W["qkvz"]).view(B, T, 4 * HEADS, HEAD).transpose(1, 2).chunk(4, 1)
    qr, kr = b.rotary(q / HEAD, k, f)
    vc = v.contiguous()
    o = plan.forward(qr, kr, vc)
    a = b.norm_forward(o.transpose(1, 2), P["head"], gate=z.transpose(1, 2))
    branch = (a.view(B, T, -1) @ W["out"]).contiguous()
    n, h = b.norm_forward(branch, P["last"], residual=x, scale=P["scale"])
    m = n @ W["mix"]
    u, pre = m.chunk(2, -1)
    la = gates(pre.float()).contiguous()
    r, _ = b.recurrence_forward(u, la)
    out = h + r
    # backward
    du, dla, _ = b.recurrence_backward(la, r, dy)
    dpre = dla * (-0.1 * torch.sigmoid(pre.float()))
    dm = torch.cat((du, dpre.to(dtype)), -1)
    dn = (dm @ W["mix"].T).contiguous()
    dh, dbranch, dlast, dscale, _ = b.norm_backward(dn, h, P["last"], dH=dy, X=branch, scale=P["scale"])
    da = (dbranch @ W["out"].T).view(B, T, HEADS, HEAD)
    do, _, dhead, _, dz = b.norm_backward(da, o.transpose(1, 2), P["head"], gate=z.transpose(1, 2), dH_out=torch.empty_like(o).transpose(1, 2))
    dq, dk, dv = plan.backward(qr, kr, vc, do.transpose(1, 2).contiguous())
    dq, dk = b.rotary(dq, dk, f, adjoint=True)
    dall = torch.cat((dq / HEAD, dk, dv, dz.transpose(1, 2)), 1).transpose(1, 2).reshape(B * T, -1)
    dyn = (dall @ W["qkvz"].T).view(B, T, WIDTH)
    dx, _, dnorm, _, _ = b.norm_backward(dyn, x, P["norm"], dH=dh)
    plan.check_status()
    # the same in 64 bits
    leaves = {**{k2: w.double().requires_grad_() for k2, w in W.items()}}
    params = {k2: p.double().requires_grad_() for k2, p in P.items()}
    x64 = x.double().requires_grad_()
    ref = model64(leaves, params, x64, f)
    grads = torch.autograd.grad(ref, [x64, params["norm"], params["head"], params["scale"], params["last"], leaves["mix"]], dy.double())
    got = [dx, dnorm, dhead, dscale, dlast, n.reshape(-1, WIDTH).T @ dm.reshape(B * T, -1)]
    rel = lambda p, w: float((p.double() - w).norm() / w.norm())
    assert rel(out, ref.detach()) <= tol
    for name, p, w in zip(("x", "norm", "head", "scale", "last", "mix"), got, grads):
        assert rel(p, w) <= tol, (name, rel(p, w))


def test_the_same_tokens_one_at_a_time():
    """fp32, on a packed cache: the type table's part of o in 8 bits (relative to a row's largest entry 1 / 254: about 0.6 % of the norm),
    all else as in the prefill."""
    W, P, x, _ = weights(torch.float32)
    f, _ = b.rotary_frequencies(32)
    plan = b.SmatPlan(B, HEADS, T, HEAD, HEAD, D, CHUNK, "f32")
    torch.backends.cuda.matmul.allow_tf32 = False
    y = b.norm_forward(x, P["norm"])
    q, k, v, z = (y.view(-1, WIDTH) @ W["qkvz"]).view(B, T, 4 * HEADS, HEAD).transpose(1, 2).chunk(4, 1)
    qr, kr = b.rotary(q / HEAD, k, f)
    o = plan.forward(qr, kr, v.contiguous())
    a = b.norm_forward(o.transpose(1, 2), P["head"], gate=z.transpose(1, 2))
    n, h = b.norm_forward((a.view(B, T, -1) @ W["out"]).contiguous(), P["last"], residual=x, scale=P["scale"])
    m = n @ W["mix"]
    r, _ = b.recurrence_forward(m[..., :WIDTH], gates(m[..., WIDTH:]))
    half = plan.geometry().n
    packed = plan.decode_cache_packed()
    plan.decode_begin_packed(kr, v.contiguous(), packed)
    _, state = b.recurrence_forward(m[:, :half, :WIDTH], gates(m[:, :half, WIDTH:]))
    worst = 0.0
    for t in range(half, half + 64):
        yt = b.norm_forward(x[:, t], P["norm"])
        qt, kt, vt, zt = (yt @ W["qkvz"]).view(B, 4 * HEADS, HEAD).chunk(4, 1)
        at = torch.full((B,), t, device="cuda")
        qt, kt = b.rotary(qt / HEAD, kt, f, positions=at)
        assert float((qt - qr[:, :, t]).abs().max()) <= 1e-5 and float((kt - kr[:, :, t]).abs().max()) <= 1e-4
        ot = plan.decode_step_packed(qt, kt, vt.contiguous(), t, packed)
        worst = max(worst, float((ot - o[:, :, t]).norm() / o[:, :, t].norm()))
        an = b.norm_forward(ot, P["head"], gate=zt)
        nt, ht = b.norm_forward(an.view(B, -1) @ W["out"], P["last"], residual=x[:, t], scale=P["scale"])
        mt = nt @ W["mix"]
        rt, _ = b.recurrence_forward(mt[:, :WIDTH].contiguous(), gates(mt[:, WIDTH:]), h0=state, hT=state)
        assert float((ht + rt - h[:, t] - r[:, t]).norm() / (h[:, t] + r[:, t]).norm()) <= 0.05
    assert 0.0 < worst <= 0.02
