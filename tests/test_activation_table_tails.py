"""qnn_activation_table where a function is next to zero or to a bound: output
scales fine enough to show its tail, against formulas that don't cancel there."""
import math

import numpy as np
import pytest

from paper_2006_10226_amd import qnn as Q

FORMULA = {
    "gelu": lambda x: 0.5 * x * math.erfc(-x / math.sqrt(2.0)),
    "gelu_tanh": lambda x: x / (1.0 + math.exp(-2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3))),
    "silu": lambda x: x / (1.0 + math.exp(-x)),
    "sigmoid": lambda x: 1.0 / (1.0 + math.exp(-x)),
}


@pytest.mark.parametrize("kind", sorted(FORMULA))
@pytest.mark.parametrize("at", [-4.0, -6.0, -8.0])
def test_tails(kind, at):
    """Inputs about `at`, code -100, whose value is 100 steps of the output."""
    f = FORMULA[kind]
    s_x = float(np.float32(-at / 100))
    s_y = float(np.float32(abs(f(at)) / 100))
    t = Q.activation_table(kind, "i8", s_x, 0, "i8", s_y, 0)
    for q in range(-128, -60):
        v = f(s_x * q) / s_y
        want = math.copysign(math.floor(abs(v) + 0.5), v)
        got = (int(t[q & 255]) ^ 128) - 128
        tie = abs(abs(v) - math.floor(abs(v)) - 0.5) < 1e-6
        assert got == min(max(want, -128), 127) or (tie and abs(got - want) <= 1), (kind, q, v, got)
