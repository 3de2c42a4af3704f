"""Operators around the attention pass: cases, plain forms and exact values.

A case names one operator and its sizes:
  op "rotary"      Q and K of the plan rotated by position (or the gradients rotated back), from rows of any stride
  op "norm"        root-mean-square norm of rows: before a block (residual stream and residual scale) or behind it (gate)
  op "recurrence"  h_t = exp(log_a_t) h_{t-1} + x_t over long sequences, its gradients, and one token at a time
  op "packed"      the decode cache with its type table in 8 bits: written and read back, or one decoding step on it

Shapes are those of the repository's own workloads (paper_2609_36062_b200/synth.py, bench.py) where it has one: 8 or 16
heads of 64 or 128, lengths up to 65536, model widths of heads * d_v.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
MOST_ELEMENTS = 134_217_728       # of one tensor of a case


def listed():
    return [
        # serving, one token of 32 sequences: 16 query and key heads rotated at the positions that each sequence has reached
        {"name": "rotary_decode_32", "op": "rotary", "batch": 32, "heads": 16, "T": 1, "d": 128, "rotated": 128, "interleaved": False,
         "scaling": "yarn", "far": 65536, "per_batch": True, "adjoint": False, "dtype": BF16},
        # a prompt of 16 K: rows as the projections leave them, [batch, T, heads, d], into the plan's layout
        {"name": "rotary_16k", "op": "rotary", "batch": 2, "heads": 16, "T": 16384, "d": 128, "rotated": 128, "interleaved": False,
         "scaling": "yarn", "far": 0, "per_batch": False, "adjoint": False, "dtype": BF16},
        # training in fp32 at an odd length: the gradients rotated back, half of every head, neighbouring pairs
        {"name": "rotary_adjoint_5056_f32", "op": "rotary", "batch": 4, "heads": 8, "T": 5056, "d": 128, "rotated": 64,
         "interleaved": True, "scaling": "none", "far": 0, "per_batch": False, "adjoint": True, "dtype": F32},
        # serving, one token: the residual stream takes in the branch, and is normed for the next block
        {"name": "norm_residual_decode_32", "op": "norm", "batch": 32, "T": 1, "groups": 1, "width": 2048, "residual": True, "scaled": True,
         "gate": "", "grouped_weight": False, "backward": False, "dtype": BF16},
        # behind the attention pass of a training step: every head's rows normed and gated, [b, h, T, d] to [b, T, h d]
        {"name": "norm_gate_8k", "op": "norm", "batch": 8, "T": 8192, "groups": 16, "width": 128, "residual": False, "scaled": False,
         "gate": "silu", "grouped_weight": True, "backward": False, "dtype": BF16},
        # its gradients
        {"name": "norm_gate_8k_backward", "op": "norm", "batch": 8, "T": 8192, "groups": 16, "width": 128, "residual": False,
         "scaled": False, "gate": "silu", "grouped_weight": True, "backward": True, "dtype": BF16},
        # the norm before a block, gradients: the residual stream's own gradient comes in, that of the branch's scale goes out
        {"name": "norm_residual_8k_backward", "op": "norm", "batch": 4, "T": 8192, "groups": 1, "width": 2048, "residual": True,
         "scaled": True, "gate": "", "grouped_weight": False, "backward": True, "dtype": BF16},
        # one long document through a recurrent layer
        {"name": "recurrence_64k", "op": "recurrence", "batch": 1, "T": 65536, "channels": 2048, "mode": "forward", "pieces": 1,
         "dtype": BF16, "gates": BF16},
        # training, sequences packed into rows of 8 K (each begins with a closed gate), gates in fp32
        {"name": "recurrence_8k_backward", "op": "recurrence", "batch": 4, "T": 8192, "channels": 2048, "mode": "backward", "pieces": 5,
         "dtype": BF16, "gates": F32},
        # serving, one token of 32 sequences
        {"name": "recurrence_step_32", "op": "recurrence", "batch": 32, "T": 1, "channels": 2048, "mode": "step", "pieces": 1,
         "dtype": BF16, "gates": BF16},
        # the cache of a 16 K prompt at the richest mask, packed behind the prefill and unpacked again
        {"name": "packed_16k_d4", "op": "packed", "batch": 1, "heads": 16, "T": 16384, "d": 4, "chunk": 128, "width": 128, "mode": "write",
         "gated": False, "dtype": BF16},
        # one decoding step on the packed cache
        {"name": "packed_step_32", "op": "packed", "batch": 32, "heads": 16, "T": 2048, "d": 3, "chunk": 64, "width": 128, "mode": "step",
         "gated": False, "dtype": BF16},
    ]


def _log_int(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    while True:
        op = rng.choice(("rotary", "norm", "norm", "recurrence", "recurrence", "packed"))
        dtype = rng.choice((BF16, BF16, F32))
        if op == "rotary":
            d, T = rng.choice((64, 128)), rng.choice((1, _log_int(rng, 2, 65536)))
            c = {"op": op, "batch": _log_int(rng, 1, 32), "heads": rng.choice((8, 16)), "T": T, "d": d,
                 "rotated": rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2))), "interleaved": rng.random() < 0.5,
                 "scaling": rng.choice(("none", "linear", "ntk", "yarn")), "far": rng.choice((0, _log_int(rng, 1000, 1000000))),
                 "per_batch": rng.random() < 0.5, "adjoint": rng.random() < 0.4, "dtype": dtype}
            elements = c["batch"] * c["heads"] * T * d
        elif op == "norm":
            heads = rng.random() < 0.5       # rows of a head behind the attention, or of the model before a block
            T = rng.choice((1, _log_int(rng, 2, 65536)))
            c = {"op": op, "batch": _log_int(rng, 1, 32), "T": T, "groups": rng.choice((8, 16)) if heads else 1,
                 "width": rng.choice((64, 128)) if heads else rng.choice((512, 1024, 2048, 4096, 8192, _log_int(rng, 100, 8192))),
                 "residual": not heads and rng.random() < 0.8, "scaled": not heads and rng.random() < 0.5,
                 "gate": rng.choice(("silu", "sigmoid")) if heads and rng.random() < 0.8 else "",
                 "grouped_weight": heads and rng.random() < 0.5, "backward": T > 1 and rng.random() < 0.5, "dtype": dtype}
            elements = c["batch"] * T * c["groups"] * c["width"]
        elif op == "recurrence":
            mode = rng.choice(("forward", "backward", "step"))
            c = {"op": op, "batch": _log_int(rng, 1, 64), "T": 1 if mode == "step" else _log_int(rng, 2, 65536),
                 "channels": rng.choice((256, 1024, 2048, 8 * _log_int(rng, 4, 512), _log_int(rng, 20, 4096))), "mode": mode,
                 "pieces": rng.choice((1, 1, rng.randint(2, 9))), "dtype": dtype, "gates": rng.choice((dtype, F32))}
            elements = c["batch"] * c["T"] * c["channels"]
        else:
            mode, width, chunk = rng.choice(("write", "step")), rng.choice((64, 128)), rng.choice((64, 128))
            c = {"op": op, "batch": _log_int(rng, 1, 32), "heads": rng.choice((8, 16)), "T": chunk * _log_int(rng, 8, 128),
                 "d": rng.choice((1, 2, 3, 4)), "chunk": chunk, "width": width, "mode": mode, "gated": rng.random() < 0.4, "dtype": dtype}
            elements = c["batch"] * c["heads"] * _types(c["d"], c["T"], chunk) * width * width // 3     # as much as packed_16k_d4 has
        if elements <= (MOST_ELEMENTS if dtype == BF16 else MOST_ELEMENTS // 2) and (op != "recurrence" or c["pieces"] <= c["T"]):
            return c


# ---- what the cases share ------------------------------------------------------------------------------------------------

def _types(d, T, chunk):
    """Type states of a head: q (q^(d-1) - 1) / (q - 1) for the smallest prime q with q^d >= n."""
    if d == 1:
        return 1
    n, q = chunk * (T // (2 * chunk)), 2
    while q ** d < n or any(q % f == 0 for f in range(2, math.isqrt(q) + 1)):
        q += 1
    return q * (q ** (d - 1) - 1) // (q - 1)


def _dtype(name):
    return torch.bfloat16 if name == BF16 else torch.float32


def _frequencies(case):
    """Radians a token of every pair, in 64 bits, and the factor on the rotated rows: base 10000, contexts of 4096 stretched
    sixteenfold by one of the usual rules."""
    n, base, factor, length = case["rotated"], 10000.0, 16.0, 4096
    if case["scaling"] == "ntk":
        base *= factor ** (n / (n - 2)) if n > 2 else 1.0
    i = torch.arange(0, n, 2, dtype=torch.float64)
    f = base ** (-i / n)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] != "yarn":
        return f, 1.0
    # pairs that turn more than 32 times in the trained length stay, those that turn less than once are stretched
    place = lambda turns: n * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = max(math.floor(place(32.0)), 0), min(math.ceil(place(1.0)), n - 1)
    ramp = ((torch.arange(n // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
    return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0


def _doubled(a, x):
    """Running values of y_t = a_t y_{t-1} + x_t (y_{-1} = 0) along dimension 1, in log2(T) steps."""
    a, y, s = a.clone(), x.clone(), 1
    while s < y.shape[1]:
        y[:, s:] = y[:, s:] + a[:, s:] * y[:, :-s]
        a[:, s:] = a[:, s:] * a[:, :-s]
        s *= 2
    return y


def _codes(U):
    """Rows in 8 bits: codes x m rounded to even with m the largest number of eight significant bits for which m max|x| <= 127, so
    that a product with an entry is exact and m and the codes are the same in any arithmetic; and what a code counts, 1 / m in fp32.
    The quotient is taken in 64 bits, where a largest entry of 24 bits leaves it on its side of every number of eight bits;
    an fp32 quotient, or the reciprocal times 127, is rounded onto some of them."""
    top = U.abs().amax(-1, keepdim=True).double()
    m = torch.where(top > 0, torch.div(torch.full_like(top, 127.0), top).clamp(max=2.0 ** 126), torch.zeros_like(top))
    m = (m.contiguous().view(torch.int64) & -(1 << 45)).view(torch.float64).float()
    wide = U.float() if U.dtype == torch.bfloat16 else U.double()
    return torch.round(wide * m).to(torch.int8), torch.where(m > 0, 1.0 / m, torch.zeros_like(m)).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = _dtype(case["dtype"])

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)

    st = {"case": case}
    if own:
        from paper_2609_36062_b200 import binding
        st["b"] = binding
    B, T = case["batch"], case["T"]
    if case["op"] == "rotary":
        H, d = case["heads"], case["d"]
        f, factor = _frequencies(case)
        # rows as a projection leaves them, query and key heads side by side; gradients come in the plan's layout
        if case["adjoint"]:
            q, k = normal(B, H, T, d).to(dtype), normal(B, H, T, d).to(dtype)
        else:
            q, k = normal(B, T, 2 * H, d).to(dtype).transpose(1, 2).chunk(2, 1)
        first = torch.randint(case["far"] + 1, (B, 1) if case["per_batch"] else (1,), generator=g, device="cuda")
        st.update(q=q, k=k, f=f.cuda(), factor=factor, at=first + torch.arange(T, device="cuda"))
    elif case["op"] == "norm":
        G, W = case["groups"], case["width"]
        rows = lambda: normal(B, T, G, W).to(dtype)
        st["w"] = 1 + 0.1 * normal(*((G, W) if case["grouped_weight"] else (W,)))
        # heads come as the attention pass leaves them, [batch, heads, T, width]
        st["x"] = normal(B, G, T, W).to(dtype).transpose(1, 2) if G > 1 else rows()
        st["residual"] = rows() if case["residual"] else None
        st["scale"] = 0.1 + 0.05 * normal(W) if case["scaled"] else None
        st["gate"] = rows() if case["gate"] else None
        if case["backward"]:
            st["dy"] = rows()
            st["h"] = rows() if case["residual"] or case["scaled"] else st["x"]      # as the forward left it
            st["dh"] = rows() if case["residual"] else None
    elif case["op"] == "recurrence":
        C = case["channels"]
        # memories of ten to a thousand tokens by channel, each token opening its gate more or less
        reach = torch.exp(uniform(C) * math.log(100.0)) * 10.0
        log_a = (-(0.25 + 1.5 * uniform(B, T, C)) / reach).to(_dtype(case["gates"]))
        for i in range(1, case["pieces"]):
            log_a[:, i * T // case["pieces"]] = -math.inf      # the next sequence of the row begins
        st.update(log_a=log_a, h0=normal(B, C))
        if case["mode"] == "backward":
            st.update(h=(normal(B, T, C) * 3).to(dtype), dh=normal(B, T, C).to(dtype), dhT=normal(B, C))
        else:
            st["x"] = normal(B, T, C).to(dtype)
        if case["mode"] == "step":
            st["state"] = st.pop("h0")
    else:
        _prepare_packed(case, st, normal, uniform, dtype)
    return st


def _prepare_packed(case, st, normal, uniform, dtype):
    B, H, r = case["batch"], case["heads"], case["width"]
    types, bh = _types(case["d"], case["T"], case["chunk"]), B * H
    table = torch.bfloat16 if _table_is_bf16(case) else torch.float32
    plan = None
    if own:
        b = st["b"]
        plan = b.SmatPlan(B, H, case["T"], r, r, case["d"], case["chunk"], case["dtype"], flags=b.FLAG_GATED if case["gated"] else 0)
    U = torch.empty(bh, types, r, r, dtype=table, device="cuda")
    for h in range(bh):      # sums over a type's keys: rows of different size
        U[h] = normal(types, r, r) * torch.exp(normal(types, r, 1))
    S, log_g = normal(B, H, r, r), -uniform(bh) if case["gated"] else None
    st.update(plan=plan, first=case["chunk"] * (case["T"] // (2 * case["chunk"])), types=types, step=0)
    st["count"] = case["T"] - st["first"]
    if case["mode"] == "step":
        unit = lambda: torch.nn.functional.normalize(normal(B, H, r), dim=-1).to(dtype)
        tokens = 16      # rows of the tokens that are decoded one after the other
        st.update(q=[unit() for _ in range(tokens)], k=[unit() for _ in range(tokens)], v=[normal(B, H, r).to(dtype) for _ in range(tokens)])
        st["a"] = [torch.log(uniform(bh) * 0.002 + 0.998) for _ in range(tokens)] if case["gated"] else [None] * tokens
    if not own:
        st.update(U=U, S=S, log_g=log_g)
        if case["mode"] == "step":
            st["codes"], st["unit"] = _codes(U)
        return
    cache = plan.decode_cache()
    pad = lambda n: (n + 255) // 256 * 256
    views = {}
    for name, t in (("U", U), ("S", S), ("log_g", log_g)):      # the cache's layout as the library documents it
        if t is not None:
            at = sum(pad(v.numel() * v.element_size()) for v in views.values())
            views[name] = cache[at:at + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
            views[name].copy_(t)
    st["packed"] = plan.decode_cache_packed()
    if case["mode"] == "step":
        plan.decode_pack(cache, st["packed"])
        tail = sum(pad(v.numel() * v.element_size()) for n, v in views.items() if n != "U")
        at = st["packed"].numel() - tail
        st["S"] = st["packed"][at:at + S.numel() * 4].view(torch.float32).view(S.shape)
        st["log_g"] = st["packed"][at + pad(S.numel() * 4):][:bh * 4].view(torch.float32) if case["gated"] else None
        return
    st.update(cache=cache, again=torch.empty_like(cache))
    st["again_U"] = st["again"][:U.numel() * U.element_size()].view(table).view(U.shape)
    at = pad(U.numel() * U.element_size())
    st["again_S"] = st["again"][at:at + S.numel() * 4].view(torch.float32).view(S.shape)


def _table_is_bf16(case):
    """The element type that a plan keeps its type table in: bf16 where it is made on the tensor cores (heads of 128, blocks of
    whole 128-token tiles), else fp32."""
    n = case["chunk"] * (case["T"] // (2 * case["chunk"]))
    return case["dtype"] == BF16 and case["width"] == 128 and n % 128 == 0 and (case["T"] - n) % 128 == 0 and case["d"] > 1


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    case, b = st["case"], st["b"]
    if case["op"] == "rotary":
        q, k = b.rotary(st["q"], st["k"], st["f"], positions=st["at"], interleaved=case["interleaved"], scale=st["factor"],
                        adjoint=case["adjoint"])
        return {"q": q, "k": k}
    if case["op"] == "norm":
        kind = {"gate": st["gate"], "activation": case["gate"] or "silu"}
        if not case["backward"]:
            out = b.norm_forward(st["x"], st["w"], residual=st["residual"], scale=st["scale"], **kind)
            return {"y": out[0], "h": out[1]} if case["residual"] or case["scaled"] else {"y": out}
        extra = {"X": st["x"], "scale": st["scale"]} if case["scaled"] else {}
        dh, dx, dw, ds, dg = b.norm_backward(st["dy"], st["h"], st["w"], dH=st["dh"], **extra, **kind)
        return _named(dh=dh, dx=dx if case["scaled"] else None, dw=dw, ds=ds, dg=dg)
    if case["op"] == "recurrence":
        if case["mode"] == "backward":
            dx, dla, dh0 = b.recurrence_backward(st["log_a"], st["h"], st["dh"], h0=st["h0"], dhT=st["dhT"])
            return {"dx": dx, "dlog_a": dla, "dh0": dh0}
        if case["mode"] == "step":
            h, state = b.recurrence_forward(st["x"], st["log_a"], h0=st["state"], hT=st["state"])
            return {"h": h, "state": state}
        h, last = b.recurrence_forward(st["x"], st["log_a"], h0=st["h0"])
        return {"h": h, "last": last}
    plan = st["plan"]
    if case["mode"] == "write":
        plan.decode_pack(st["cache"], st["packed"])
        plan.decode_unpack(st["packed"], st["again"])
        return {"U": st["again_U"], "S": st["again_S"]}
    i, st["step"] = st["step"], st["step"] + 1
    j = i % len(st["q"])
    o = plan.decode_step_packed(st["q"][j], st["k"][j], st["v"][j], st["first"] + i % st["count"], st["packed"], log_a_t=st["a"][j])
    return _named(o=o, S=st["S"], log_g=st["log_g"])


def _named(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _act(kind, z):
    """The gate's factor and its derivative."""
    s = 1 / (1 + torch.exp(-z))
    return (s, s * (1 - s)) if kind == "sigmoid" else (z * s, s * (1 + z * (1 - s)))


def _run_plain(st):
    case = st["case"]
    dtype = _dtype(case["dtype"])
    if case["op"] == "rotary":
        n = case["rotated"]
        angle = st["at"][..., None].double() * st["f"]
        cos, sin = (torch.cos(angle) * st["factor"]).float(), (torch.sin(angle) * st["factor"]).float()
        if case["per_batch"]:
            cos, sin = cos[:, None], sin[:, None]
        if case["adjoint"]:
            sin = -sin
        out = []
        for x in (st["q"], st["k"]):
            x = x.float()
            a, b = (x[..., 0:n:2], x[..., 1:n:2]) if case["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])
            a, b = a * cos - b * sin, b * cos + a * sin
            turned = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
            out.append(torch.cat((turned, x[..., n:]), -1).to(dtype))
        return {"q": out[0], "k": out[1]}
    if case["op"] == "norm":
        w = st["w"]
        if not case["backward"]:
            h = st["x"].float()
            if case["scaled"]:
                h = h * st["scale"]
            if case["residual"]:
                h = h + st["residual"].float()
            y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * w
            if case["gate"]:
                y = y * _act(case["gate"], st["gate"].float())[0]
            return {"y": y.to(dtype), "h": h.to(dtype)} if case["residual"] or case["scaled"] else {"y": y.to(dtype)}
        h, dy = st["h"].float(), st["dy"].float()
        r = torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6)
        n = h * r
        dg, up = None, dy
        if case["gate"]:
            f, slope = _act(case["gate"], st["gate"].float())
            up, dg = dy * f, (dy * n * w * slope).to(dtype)
        along = (0, 1) if case["grouped_weight"] else (0, 1, 2)
        dw, dn = (up * n).sum(along), up * w
        dh = r * (dn - n * (dn * n).mean(-1, keepdim=True))
        if case["residual"]:
            dh = dh + st["dh"].float()
        dx = ds = None
        if case["scaled"]:
            dx, ds = (dh * st["scale"]).to(dtype), (dh * st["x"].float()).sum((0, 1, 2))
        return _named(dh=dh.to(dtype), dx=dx, dw=dw, ds=ds, dg=dg)
    if case["op"] == "recurrence":
        a = torch.exp(st["log_a"].float())
        if case["mode"] == "step":
            st["state"].mul_(a[:, 0]).add_(st["x"][:, 0].float())
            return {"h": st["state"][:, None].to(dtype), "state": st["state"]}
        if case["mode"] == "forward":
            x = st["x"].to(torch.float32, copy=True)      # (a tensor of fp32 is its own .float())
            x[:, 0] += a[:, 0] * st["h0"]
            h = _doubled(a, x)
            return {"h": h.to(dtype), "last": h[:, -1].clone()}
        # c_t = a_t (dh_t + c_{t+1}), c_T = dhT; dx_t = dh_t + c_{t+1}, dlog_a_t = c_t h_{t-1}, dh0 = c_0
        dh = st["dh"].to(torch.float32, copy=True)
        dh[:, -1] += st["dhT"]
        c = _doubled(a.flip(1), (a * dh).flip(1)).flip(1)
        before = torch.cat((st["h0"][:, None], st["h"][:, :-1].float()), 1)
        dh[:, :-1] += c[:, 1:]
        return {"dx": dh.to(dtype), "dlog_a": (c * before).to(st["log_a"].dtype), "dh0": c[:, 0].clone()}
    if case["mode"] == "write":
        codes, unit = _codes(st["U"])
        return {"U": (codes.float() * unit).to(st["U"].dtype), "S": st["S"].clone()}
    i, st["step"] = st["step"], st["step"] + 1
    j = i % len(st["q"])
    q, k, v = (st[x][j].float() for x in "qkv")
    t = (st["first"] + i % st["count"] - st["first"] + 1) % st["types"]
    U = (st["codes"][:, t].float() * st["unit"][:, t]).view(st["S"].shape)
    if case["gated"]:
        st["log_g"].add_(st["a"][j])
        st["S"].mul_(torch.exp(st["a"][j]).view(*q.shape[:2], 1, 1))
        U = U * torch.exp(st["log_g"]).view(*q.shape[:2], 1, 1)
    st["S"].add_(k[..., None] * v[..., None, :])
    o = (q[..., None] * (U + st["S"])).sum(-2).to(dtype)
    return _named(o=o, S=st["S"], log_g=st["log_g"])


# ---- what one pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == BF16 else 4
    B, T = case["batch"], case["T"]
    if case["op"] == "rotary":
        rows = 2 * B * case["heads"] * T      # of Q and K: read and written, the pairs' two products and sums
        return {"bytes": rows * 2 * case["d"] * e + (B if case["per_batch"] else 1) * T * 8 + case["rotated"] * 4,
                "flops": rows * 3 * case["rotated"]}
    if case["op"] == "norm":
        n = B * T * case["groups"] * case["width"]
        if not case["backward"]:
            tensors = 2 + (2 if case["residual"] else 1 if case["scaled"] else 0) + (1 if case["gate"] else 0)
            return {"bytes": n * e * tensors, "flops": n * (6 + (4 if case["gate"] else 0))}
        tensors = 3 + (1 if case["residual"] else 0) + (2 if case["scaled"] else 0) + (2 if case["gate"] else 0)
        return {"bytes": n * e * tensors, "flops": n * (12 + (8 if case["gate"] else 0) + (3 if case["scaled"] else 0))}
    if case["op"] == "recurrence":
        n, s, a = B * T * case["channels"], B * case["channels"] * 4, 2 if case["gates"] == BF16 else 4
        if case["mode"] == "backward":
            return {"bytes": n * (3 * e + 2 * a) + 3 * s, "flops": 5 * n}
        return {"bytes": n * (2 * e + a) + 2 * s, "flops": 3 * n}
    r, bh = case["width"], B * case["heads"]
    state = 2 if _table_is_bf16(case) else 4
    if case["mode"] == "write":      # the table read, its codes and units written and read, the table written; S with it
        rows = bh * _types(case["d"], T, case["chunk"]) * r
        return {"bytes": rows * (2 * r * state + 2 * r + 8) + bh * r * r * 16, "flops": rows * r * 3}
    return {"bytes": bh * (r * r * 9 + r * 4 + 4 * r * e), "flops": bh * 6 * r * r}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    mine, own = own, False
    try:
        st = prepare(case, seed)      # inputs only
    finally:
        own = mine
    return {"rotary": _exact_rotary, "norm": _exact_norm, "recurrence": _exact_recurrence, "packed": _exact_packed}[case["op"]](case, st)


def _exact_rotary(case, st):
    """A pair as one complex number, multiplied by factor * exp(i position frequency), or by its conjugate."""
    n = case["rotated"]
    turn = torch.polar(torch.full_like(st["f"], st["factor"]), st["at"].double()[..., None] * st["f"])
    turn = turn.conj() if case["adjoint"] else turn
    turn = turn.unsqueeze(1) if case["per_batch"] else turn
    out = {}
    for name in ("q", "k"):
        x = st[name].double().clone()
        one = slice(0, n, 2) if case["interleaved"] else slice(0, n // 2)
        two = slice(1, n, 2) if case["interleaved"] else slice(n // 2, n)
        z = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * turn
        x[..., one], x[..., two] = z.real, z.imag
        out[name] = x
    return out


def _exact_norm(case, st):
    """The formula in 64 bits; gradients by torch's differentiation of it, a slice of the batch at a time."""
    cut = max(1, (1 << 26) // (case["T"] * case["groups"] * case["width"]))
    wide = lambda t, s: None if t is None else t[s].double()
    w = st["w"].double().requires_grad_()
    scale = None if st["scale"] is None else st["scale"].double().requires_grad_()

    def gated(h, z):
        y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * w
        if z is None:
            return y
        return y * (torch.sigmoid(z) if case["gate"] == "sigmoid" else z * torch.sigmoid(z))

    parts, total = [], {}
    for b in range(0, case["batch"], cut):
        s = slice(b, b + cut)
        x, res, z = wide(st["x"], s), wide(st["residual"], s), wide(st["gate"], s)
        if not case["backward"]:
            with torch.no_grad():
                h = x if scale is None else x * scale
                h = h if res is None else h + res
                parts.append({"y": gated(h, z), "h": h} if case["residual"] or case["scaled"] else {"y": gated(h, z)})
            continue
        # h as it was kept is the input; what the branch's rows and scale get follows from h = residual + scale x
        h = wide(st["h"], s).requires_grad_()
        if z is not None:
            z.requires_grad_()
        leaves = [h, w] + ([z] if z is not None else [])
        got = torch.autograd.grad(gated(h, z), leaves, wide(st["dy"], s))
        dh = got[0] if st["dh"] is None else got[0] + wide(st["dh"], s)
        part = {"dh": dh}
        total["dw"] = total.get("dw", 0) + got[1]
        if scale is not None:
            part["dx"] = dh * scale.detach()
            total["ds"] = total.get("ds", 0) + (dh * x).sum((0, 1, 2))
        if z is not None:
            part["dg"] = got[2]
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]).detach() for k in parts[0]}
    out.update(total)
    return {k: out[k] for k in ("y", "h", "dh", "dx", "dw", "ds", "dg") if k in out}


def _in_order(a, x, y):
    """y_t = a_t y_{t-1} + x_t token by token; blocks of about sqrt(T) tokens side by side, then joined in order."""
    B, T, C = x.shape
    L = max(1, math.isqrt(T))
    pad = -T % L
    if pad:
        a = torch.cat((a, a.new_ones(B, pad, C)), 1)
        x = torch.cat((x, x.new_zeros(B, pad, C)), 1)
    a, x = a.reshape(B, -1, L, C).clone(), x.reshape(B, -1, L, C).clone()
    for i in range(1, L):
        x[:, :, i] += a[:, :, i] * x[:, :, i - 1]
        a[:, :, i] *= a[:, :, i - 1]
    for j in range(x.shape[1]):
        x[:, j] += a[:, j] * y[:, None]
        y = x[:, j, -1]
    return x.reshape(B, -1, C)[:, :T]


def _exact_recurrence(case, st):
    a = st["log_a"].double().exp()
    if case["mode"] == "step":
        h = a[:, 0] * st["state"].double() + st["x"][:, 0].double()
        return {"h": h[:, None], "state": h}
    if case["mode"] == "forward":
        h = _in_order(a, st["x"].double(), st["h0"].double())
        return {"h": h, "last": h[:, -1]}
    # the loss sum(dh h) + sum(dhT h_last): its gradient by h_t, in order from the last token
    later = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1).flip(1)
    g = st["dh"].double()
    g[:, -1] += st["dhT"].double()
    g = _in_order(later, g.flip(1), torch.zeros_like(g[:, 0])).flip(1)
    before = torch.cat((st["h0"].double()[:, None], st["h"].double()[:, :-1]), 1)
    return {"dx": g, "dlog_a": g * a * before, "dh0": g[:, 0] * a[:, 0]}


def _exact_codes(U):
    """Codes and multipliers of the rows of U: floor to eight significant bits of the quotient, rounding to even, in 64 bits."""
    quotient = 127 / U.abs().amax(-1, keepdim=True).double()
    bits = 2.0 ** (7 - torch.floor(torch.log2(quotient)))
    m = torch.floor(quotient * bits) / bits
    return torch.round(U.double() * m), m


def _exact_packed(case, st):
    if case["mode"] == "write":
        if st["U"].numel() > 1 << 29:
            return None
        codes, m = _exact_codes(st["U"])
        return {"U": codes / m, "S": st["S"].double()}
    j = 0
    q, k, v = (st[x][j].double() for x in "qkv")
    codes, m = _exact_codes(st["U"][:, 1 % st["types"]])
    U = (codes / m).view(st["S"].shape)
    S, log_g = st["S"].double(), None
    if case["gated"]:
        log_g = st["log_g"].double() + st["a"][j].double()
        S = S * st["a"][j].double().exp().view(*q.shape[:2], 1, 1)
        U = U * log_g.exp().view(*q.shape[:2], 1, 1)
    S = S + torch.einsum("bhi,bhj->bhij", k, v)
    return _named(o=torch.einsum("bhi,bhij->bhj", q, U + S), S=S, log_g=log_g)
