"""The rotary plan's frequencies against 60-digit decimals (no GPU needed).

A frequency is kept as turns a position in units of 2^-64, rounded to nearest: half
a unit.  Before that it is a 64-bit-mantissa float below 0.16 turns, e = 2^-64 a
step's half: two for the power, one each for 2 pi, the division by it and by `factor`, and
the exponent's own rounding, which counts x ln b e^-x ln b < 0.4 times; NTK's base, off
by three and its exponent's, counts 2i / part of that.  0.16 (5 + 1) < 1.  YaRN's
ramp is off by r / (fast - slow) < 32 / 31 times five, and three of its own: 0.16 * 14 < 2.3."""

import os
from decimal import Decimal, getcontext

import pytest

P = pytest.importorskip("paper_2608_15211_amd")
pytest.importorskip("torch")

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libterra_swin.so not built")

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def turns(part, base, scaling="none", factor=1.0, orig_len=0):
    getcontext().prec = 60
    b, s = Decimal(base), Decimal(factor)
    if scaling == "ntk":
        b = b * s ** (Decimal(part) / (part - 2))
    out = []
    for i in range(part // 2):
        f = b ** (Decimal(-2 * i) / part) / (2 * PI)
        if scaling == "linear":
            f /= s
        if scaling == "yarn":
            keep = min(Decimal(1), max(Decimal(0), (Decimal(orig_len) * f - 1) / 31))
            f *= keep + (1 - keep) / s
        out.append(f * 2 ** 64)
    return out


@pytest.mark.parametrize("head_dim", [2, 6, 32, 64, 128, 250, 256])
@pytest.mark.parametrize("base", [1.0, 100.0, 10000.0, 1e6, 1e30])
@pytest.mark.parametrize("kw,most", [
    ({}, 1.5), ({"scaling": "linear", "factor": 3.7}, 1.5), ({"scaling": "ntk", "factor": 8.0}, 1.5), ({"scaling": "ntk", "factor": 1e9}, 1.5),
    ({"scaling": "yarn", "factor": 8.0, "orig_len": 64}, 2.8), ({"scaling": "yarn", "factor": 32.0, "orig_len": 8192}, 2.8)])
def test_frequencies(head_dim, base, kw, most):
    if kw.get("scaling") == "ntk" and head_dim == 2:
        pytest.skip("NTK needs two pairs")
    plan = P.terra_plan_rope(head_dim, base=base, **kw)
    off = max(abs(Decimal(plan.turns[i]) - f) for i, f in enumerate(turns(head_dim, base, **kw)))
    assert off <= Decimal(most), "%.2f units of 2^-64" % off
