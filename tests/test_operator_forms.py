"""Plain forms of the operators' cases on the CPU: repeated passes on the same inputs, and the rule of the packed rows in whole numbers."""
import importlib.util
import os
from fractions import Fraction

import numpy as np
import pytest
import torch

spec = importlib.util.spec_from_file_location("operator_cases", os.path.join(os.path.dirname(__file__), "..", "perf", "operators.py"))
cases = importlib.util.module_from_spec(spec)
spec.loader.exec_module(cases)


@pytest.mark.parametrize("mode", ["forward", "backward"])
@pytest.mark.parametrize("dtype,gates", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_recurrence_leaves_its_inputs_as_they_are(mode, dtype, gates):
    g = torch.Generator().manual_seed(1)
    B, T, C = 2, 40, 3
    rows = lambda: torch.randn(B, T, C, generator=g).to(cases._dtype(dtype))
    st = {"case": {"op": "recurrence", "mode": mode, "dtype": dtype, "gates": gates, "batch": B, "T": T, "channels": C},
          "x": rows(), "h": rows(), "dh": rows(), "log_a": (-torch.rand(B, T, C, generator=g) * 0.1).to(cases._dtype(gates)),
          "h0": torch.randn(B, C, generator=g), "dhT": torch.randn(B, C, generator=g)}
    before = {k: v.clone() for k, v in st.items() if torch.is_tensor(v)}
    one = {k: v.clone() for k, v in cases.run(st).items()}
    two = cases.run(st)
    assert all(torch.equal(before[k], st[k]) for k in before)
    assert all(torch.equal(one[k], two[k]) for k in one)
    want = cases._exact_recurrence(st["case"], st)
    for k in one:      # outputs rounded to their type (2^-8, 2^-24); sums of at most 41 terms, twice each (2^-24 * 82 < 2^-17)
        half = 2.0 ** -8 if one[k].dtype == torch.bfloat16 else 2.0 ** -24
        assert float((one[k].double() - want[k]).norm()) <= (half + 2.0 ** -17) * float(want[k].norm())


def largest_multiplier(top):
    """The largest number of eight significant bits whose product with `top` is at most 127, in whole numbers."""
    q = Fraction(127) / Fraction(top)
    e = -200
    while Fraction(2) ** (e + 8) <= q:
        e += 1
    return float((q / Fraction(2) ** e).__floor__() * Fraction(2) ** e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed_rows_next_to_a_border(dtype):
    """Largest entries for which 127 / max is a number of eight bits or within a rounding of fp32 of one."""
    tops = [127.0 * 2.0 ** k for k in range(-20, 21)] + [2.0 ** k for k in range(-20, 21)]
    for eighth in range(128, 256):
        near = np.float32(127.0 / eighth)
        tops += [float(x) * 2.0 ** k for x in (np.nextafter(near, np.float32(0)), near, np.nextafter(near, np.float32(9))) for k in (-20, 0, 30)]
    g = torch.Generator().manual_seed(2)
    top = torch.tensor(tops, dtype=torch.float64)
    U = (top[:, None] * (2 * torch.rand(len(tops), 16, generator=g, dtype=torch.float64) - 1)).to(dtype)
    U[:, 3] = -top.to(dtype)
    m = torch.tensor([largest_multiplier(x) for x in U.double().abs().amax(-1).tolist()], dtype=torch.float64)[:, None]
    codes, unit = cases._codes(U)
    assert torch.equal(codes.double(), torch.round(U.double() * m)) and torch.equal(unit, (1 / m).float())
    exact, multiplier = cases._exact_codes(U)
    assert torch.equal(exact, torch.round(U.double() * m)) and torch.equal(multiplier, m)
