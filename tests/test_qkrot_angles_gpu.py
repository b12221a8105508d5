"""Angles of large frequencies and far positions, against exact whole numbers.

A frequency is kept to the nearest 2^-64 of a turn, so that the angle at position p
is off by at most p 2^-65 turns, here counted as p 2^-64 2 pi radians on top of
test_qkrot_gpu's 21 units.
"""
import math

import pytest

from test_qkrot_gpu import U, make, plan_for, reference, within

pytestmark = pytest.mark.gpu

FREQUENCIES = [1e6, -1e6, 999999.9375, 123456.789, 1e3, -1e3, 37.5, 10.0, math.pi, -0.3, 1e-3, 1e-9, 5e-324, 2 * math.pi, 0.0, -1e-7]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("first", [0, 1000003, (1 << 31) - 7, (1 << 40) + 12345, -9, -(1 << 33)])
def test_large_frequencies(first, inter):
    import torch
    d = 2 * len(FREQUENCIES)
    s = make(2, 40, 2, 1, d, "f32", first=first)
    plan = plan_for(2, 1, d, "f32", d, inter, frequencies=FREQUENCIES)
    q, k = plan.forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])
    more = (abs(first) + 1000) * 2.0 ** -64 * 2 * math.pi / U
    for x, w, z in ((s["q"], s["qw"], q), (s["k"], s["kw"], k)):
        ref = reference(x, w, s["positions"], torch.zeros_like(x), d, inter, frequencies=FREQUENCIES)
        within(z, ref[0], ref[1], 21 + more)
    dq, dk, _, _ = plan.backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])
    for x, w, dz, dx in ((s["q"], s["qw"], s["dq"], dq), (s["k"], s["kw"], s["dk"], dk)):
        ref = reference(x, w, s["positions"], dz, d, inter, frequencies=FREQUENCIES)
        within(dx, ref[2], ref[3], 75 + 3 * more)
