"""The operators around the pass on the CPU: refusals before any launch, sizes, and the formulas of the rotary frequencies."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_36062_b200 import binding as b

OK, NULL, SHAPE, DTYPE, WORKSPACE, ALIGN, ARCH, UNSUPPORTED = 0, 1, 2, 3, 5, 6, 7, 10
BIG = 1 << 40


def rows(data=4096, batch=8192, head=1024, token=128):
    return ctypes.byref(b.Rows(data, batch, head, token))


def launched():
    """What a call that passes its checks answers: no device here, a launch on a GPU machine is not tried by these tests."""
    return ARCH


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only where nothing can be launched")


def rotary_code(q=None, k=None, qo=None, ko=None, **kw):
    p = dict(batch=1, q_heads=2, k_heads=2, T=8, d=128, rotated=128, interleaved=0, adjoint=0, scale=1.0, dtype=b.SMAT_BF16,
             frequencies=4096, positions=None, positions_batch=0, first=0)
    p.update(kw)
    return b.load_library().smat_rotary(ctypes.byref(b.RotaryProblem(**p)), q or rows(), k or rows(), qo or rows(), ko or rows(), None)


@no_gpu
def test_rotary_refusals():
    lib = b.load_library()
    assert rotary_code() == launched()
    assert lib.smat_rotary(None, rows(), None, rows(), None, None) == NULL
    assert rotary_code(frequencies=None) == NULL
    assert rotary_code(q=rows(data=None)) == NULL
    p = ctypes.byref(b.RotaryProblem(batch=1, q_heads=2, T=8, d=128, rotated=128, dtype=1, frequencies=4096))
    assert lib.smat_rotary(p, rows(), rows(), rows(), None, None) == NULL          # k without its output
    assert lib.smat_rotary(p, rows(), None, rows(), None, None) == launched()      # q alone
    assert rotary_code(dtype=2) == DTYPE
    for bad in (dict(batch=0), dict(q_heads=0), dict(k_heads=0), dict(T=0), dict(d=0), dict(d=513), dict(rotated=0), dict(rotated=3),
                dict(rotated=130), dict(T=1 << 31), dict(batch=1 << 16, T=1 << 15), dict(positions=8, positions_batch=-1),
                dict(q_heads=1 << 15)):
        assert rotary_code(**bad) == SHAPE, bad
    assert rotary_code(q=rows(token=-128)) == SHAPE
    assert rotary_code(q=rows(token=0)) == launched()                               # a broadcast input
    for bad in (rows(token=0), rows(token=64), rows(head=0), rows(head=512), rows(token=1 << 61)):
        assert rotary_code(qo=bad) == SHAPE                                         # rows of an output that overlap
    assert rotary_code(qo=rows(batch=0)) == launched()                              # one sequence: its stride does not matter
    assert rotary_code(q=rows(data=4097)) == ALIGN and rotary_code(frequencies=4100) == ALIGN
    assert rotary_code(positions=4100) == ALIGN
    assert rotary_code(q=rows(data=4098)) == launched()                             # an element's alignment is enough


def norm_problem(**kw):
    p = dict(batch=2, T=8, groups=2, width=128, dtype=b.SMAT_BF16, activation=0, eps=1e-6, weight=4096, weight_group=0, scale=None)
    p.update(kw)
    return ctypes.byref(b.NormProblem(**p))


@no_gpu
def test_norm_refusals():
    lib = b.load_library()
    fwd = lambda p, x=None, r=None, g=None, y=None, h=None: lib.smat_norm_forward(p, x or rows(), r, g, y or rows(), h, None)
    assert fwd(norm_problem()) == launched()
    assert fwd(None) == NULL and fwd(norm_problem(weight=None)) == NULL and fwd(norm_problem(), r=rows(data=None)) == NULL
    assert lib.smat_norm_forward(norm_problem(), None, None, None, rows(), None, None) == NULL
    assert fwd(norm_problem(dtype=3)) == DTYPE and fwd(norm_problem(activation=2)) == UNSUPPORTED
    for bad in (dict(batch=0), dict(T=0), dict(groups=0), dict(groups=65536), dict(width=0), dict(width=16385), dict(T=1 << 31),
                dict(batch=1 << 16, T=1 << 15), dict(weight_group=64), dict(eps=-1.0), dict(eps=math.nan)):
        assert fwd(norm_problem(**bad)) == SHAPE, bad
    assert fwd(norm_problem(), y=rows(token=64)) == SHAPE and fwd(norm_problem(), h=rows(head=0)) == SHAPE
    assert fwd(norm_problem(), x=rows(data=4097)) == ALIGN and fwd(norm_problem(weight=4098)) == ALIGN

    def bwd(p, g=None, x=None, dh_in=None, dx=None, dg=None, dw=4096, ds=None, ws=4096, size=BIG):
        return lib.smat_norm_backward(p, rows(), rows(), g, x, dh_in, rows(), dx, dg, dw, ds, ws, size, None)
    assert bwd(norm_problem()) == launched()
    assert bwd(norm_problem(), g=rows()) == NULL and bwd(norm_problem(), dg=rows()) == NULL     # a gate comes with its gradient
    assert bwd(norm_problem(scale=4096), ds=4096) == NULL                                      # dscale needs x
    assert bwd(norm_problem(), ds=4096, x=rows()) == NULL and bwd(norm_problem(), dx=rows()) == NULL   # ... and the scale
    assert bwd(norm_problem(scale=4096), ds=4096, x=rows(), dx=rows()) == launched()
    assert bwd(norm_problem(), ws=None) == NULL and bwd(norm_problem(), ws=4100) == ALIGN
    assert bwd(norm_problem(), ws=None, dw=None) == launched()                                  # no sums, no workspace
    need = lib.smat_norm_workspace_bytes(norm_problem())
    assert bwd(norm_problem(), size=need - 1) == WORKSPACE and bwd(norm_problem(), size=need) == launched()
    assert bwd(norm_problem(), dw=4097) == ALIGN


def test_norm_workspace():
    lib = b.load_library()
    need = lib.smat_norm_workspace_bytes(norm_problem())
    assert lib.smat_norm_workspace_bytes(norm_problem(scale=4096)) == 2 * need
    assert lib.smat_norm_workspace_bytes(norm_problem(width=0)) == 0 and lib.smat_norm_workspace_bytes(None) == 0
    assert b.norm_workspace_bytes(128, groups=2) == need and b.norm_workspace_bytes(128, groups=2, scale=True) == 2 * need
    assert lib.smat_norm_workspace_bytes(norm_problem(groups=60000)) >= 60000 * 128 * 4


def recurrence_problem(**kw):
    p = dict(batch=2, T=8, channels=128, dtype=b.SMAT_BF16, gate_dtype=b.SMAT_BF16)
    p.update(kw)
    return ctypes.byref(b.RecurrenceProblem(**p))


@no_gpu
def test_recurrence_refusals():
    lib = b.load_library()
    fwd = lambda p, x=None, a=None, h=None, h0=None, hT=None: lib.smat_recurrence_forward(p, x or rows(), a or rows(), h0, h or rows(), hT, None)
    assert fwd(recurrence_problem()) == launched() and fwd(None) == NULL and fwd(recurrence_problem(), x=rows(data=None)) == NULL
    assert lib.smat_recurrence_forward(recurrence_problem(), rows(), None, None, rows(), None, None) == NULL
    for bad in (dict(dtype=2), dict(gate_dtype=2), dict(dtype=b.SMAT_F32, gate_dtype=b.SMAT_BF16)):
        assert fwd(recurrence_problem(**bad)) == DTYPE, bad
    assert fwd(recurrence_problem(gate_dtype=b.SMAT_F32)) == launched()
    for bad in (dict(batch=0), dict(batch=65536), dict(T=0), dict(T=1 << 41), dict(channels=0), dict(channels=(1 << 20) + 1)):
        assert fwd(recurrence_problem(**bad)) == SHAPE, bad
    assert fwd(recurrence_problem(), h=rows(token=64)) == SHAPE and fwd(recurrence_problem(), x=rows(token=0)) == launched()
    assert fwd(recurrence_problem(), x=rows(data=4097)) == ALIGN and fwd(recurrence_problem(), h0=4098) == ALIGN
    bwd = lambda p, **kw: lib.smat_recurrence_backward(p, kw.get("a", rows()), rows(), rows(), kw.get("h0"), kw.get("dhT"), kw.get("dx", rows()),
                                                       kw.get("da", rows()), kw.get("dh0"), None)
    assert bwd(recurrence_problem()) == launched() and bwd(recurrence_problem(), da=None) == NULL
    assert bwd(recurrence_problem(), dx=rows(batch=0)) == SHAPE and bwd(recurrence_problem(), da=rows(batch=512)) == SHAPE
    assert bwd(recurrence_problem(), dh0=4097) == ALIGN


@no_gpu
def test_packed_cache_refusals():
    lib = b.load_library()
    plan = b.SmatPlan(1, 2, 512, 64, 64, 2, 64, "f32")
    gated = b.SmatPlan(1, 2, 512, 64, 64, 2, 64, "f32", flags=b.FLAG_GATED)
    h = plan.handle
    cache, packed = lib.smat_decode_cache_bytes(h), lib.smat_decode_packed_bytes(h)
    g = plan.geometry()
    pad = lambda n: (n + 255) // 256 * 256
    assert packed == pad(2 * g.B * 64 * 64) + pad(2 * g.B * 64 * 4) + pad(2 * 64 * 64 * 4)
    assert lib.smat_decode_packed_bytes(gated.handle) == packed + 256 and lib.smat_decode_packed_bytes(None) == 0
    at = 1 << 30
    assert lib.smat_decode_pack(h, 4096, cache, at, packed, None) == launched()
    assert lib.smat_decode_pack(None, 4096, cache, at, packed, None) == NULL
    assert lib.smat_decode_pack(h, None, cache, at, packed, None) == NULL and lib.smat_decode_unpack(h, at, packed, None, cache, None) == NULL
    assert lib.smat_decode_pack(h, 4096, cache - 1, at, packed, None) == WORKSPACE
    assert lib.smat_decode_unpack(h, at, packed - 1, 4096, cache, None) == WORKSPACE
    assert lib.smat_decode_pack(h, 4096, cache, 8192, packed, None) == SHAPE          # one in the other
    assert lib.smat_decode_pack(h, 4112, cache, at, packed, None) == ALIGN and lib.smat_decode_unpack(h, at + 16, packed, 4096, cache, None) == ALIGN
    begin = lambda hh, la=None, K=4096, size=packed, dst=at, ws=4096: lib.smat_decode_begin_packed(hh, K, 4096, la, dst, size, ws, BIG, None)
    assert begin(h) == launched() and begin(h, K=None) == NULL and begin(None) == NULL and begin(h, ws=None) == NULL
    assert begin(h, la=4096) == UNSUPPORTED and begin(gated.handle) == NULL           # gates and gated plans come together
    assert begin(h, size=packed - 1) == WORKSPACE and begin(h, dst=at + 16) == ALIGN
    step = lambda hh, la=None, t=300, size=BIG, dst=at, q=4096: lib.smat_decode_step_packed(hh, q, 4096, 4096, la, t, 4096, dst, size, None)
    assert step(h) == launched() and step(h, q=None) == NULL and step(None) == NULL
    assert step(h, la=4096) == UNSUPPORTED and step(gated.handle) == NULL and step(gated.handle, la=4096) == launched()
    assert step(h, t=255) == SHAPE and step(h, t=512) == SHAPE and step(h, size=packed - 1) == WORKSPACE and step(h, dst=at + 16) == ALIGN


def test_tensors_of_the_host_are_refused():
    x, w = torch.zeros(1, 2, 8, 64), torch.ones(64)
    with pytest.raises(ValueError):
        b.rotary(x, None, torch.ones(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        b.norm_forward(x, w)
    with pytest.raises(ValueError):
        b.norm_forward(x, w, activation="relu")
    with pytest.raises(ValueError):
        b.recurrence_forward(x[0], x[0])
    with pytest.raises(ValueError):
        b.SmatPlan(1, 1, 512, 64, 64, 2, 64, "f32").decode_pack(torch.zeros(8, dtype=torch.uint8), torch.zeros(8, dtype=torch.uint8))


def test_rotary_frequencies():
    f, s = b.rotary_frequencies(64, device="cpu")
    assert s == 1.0 and f.dtype == torch.float64 and f.shape == (32,)
    assert f[0] == 1.0 and math.isclose(float(f[16]), 10000.0 ** -0.5, rel_tol=1e-14)
    g, s = b.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu")
    assert s == 1.0 and torch.equal(g, f / 4.0)
    g, s = b.rotary_frequencies(64, scaling="ntk", factor=4.0, device="cpu")
    assert s == 1.0 and g[0] == 1.0 and math.isclose(float(g[-1]), float(f[-1]) / 4.0, rel_tol=1e-12)     # the slowest: all of it
    g, s = b.rotary_frequencies(64, scaling="yarn", factor=16.0, trained_length=4096, device="cpu")
    assert math.isclose(s, 0.1 * math.log(16.0) + 1.0)
    turns = f * 4096 / (2 * math.pi)
    assert torch.equal(g[turns > 64], f[turns > 64]) and torch.allclose(g[turns < 0.5], f[turns < 0.5] / 16.0, rtol=1e-14)
    assert bool((g <= f).all()) and bool((g >= f / 16.0).all())
    same, s = b.rotary_frequencies(64, scaling="yarn", factor=1.0, device="cpu")
    assert s == 1.0 and torch.allclose(same, f, rtol=1e-14)
    for bad in (dict(rotated=7), dict(rotated=0), dict(rotated=8, scaling="other"), dict(rotated=8, factor=0.5), dict(rotated=8, base=1.0),
                dict(rotated=8, scaling="yarn", fast_turns=1.0, slow_turns=2.0), dict(rotated=8, scaling="yarn", trained_length=0)):
        with pytest.raises(ValueError):
            b.rotary_frequencies(device="cpu", **bad)


ROOM = r"""
#include "smat_room.h"
#include <cstdio>
int main() {
  static SmatRoom<8> room;
  int asked = 0;
  const auto says = [&](int n) { return [&asked, n] { ++asked; return n; }; };
  // an answer that could not be had is passed on and asked for again; one that was, none among it, is kept
  if (room(0, 8, says(-1)) != -1 || room(0, 8, says(-1)) != -1 || asked != 2) return 1;
  if (room(0, 8, says(33)) != 33 || room(0, 8, says(-1)) != 33 || asked != 3) return 2;
  if (room(0, 4, says(0)) != 0 || room(0, 4, says(7)) != 0 || asked != 4) return 3;
  if (room(1, 8, says(16)) != 16 || room(0, 8, says(5)) != 33 || asked != 5) return 4;      // by device
  if (room(64, 8, says(3)) != 3 || room(64, 8, says(4)) != 4 || room(-1, 8, says(5)) != 5 || asked != 8) return 5;      // not kept
  std::puts("ok");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")
def test_answers_of_the_device_are_kept_only_where_there_is_one(tmp_path):
    (tmp_path / "room.cpp").write_text(ROOM)
    csrc = os.path.join(os.path.dirname(b.__file__), "csrc")
    subprocess.run(["g++", "-std=c++17", f"-I{csrc}", "-o", str(tmp_path / "room"), str(tmp_path / "room.cpp")], check=True)
    assert subprocess.run([str(tmp_path / "room")], check=True, capture_output=True, text=True).stdout == "ok\n"
