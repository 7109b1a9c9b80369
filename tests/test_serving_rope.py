"""The frequencies that qe_rope_init holds, against eighty digits (no GPU)."""
import decimal

import pytest

from paper_2309_01885_gb300 import build, qe

PI = "3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798"
BASE = [500000.0 ** (-2.0 * i / 128) for i in range(64)]
MIXED = [1.0, -1.0, 1000.0, -1000.0, 0.5, -0.3, 0.3, 6.283185307179586, -6.283185307179586, 3.141592653589793, 1e-9, -1e-9, 1e-15, 1e-19, -1e-19, 5e-324, 0.0,
         -0.0, 100.0, 123456.789, -123456.789, 4.0e8, 7.0]


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_lib()
    return qe.load()


@pytest.mark.parametrize("freq", [BASE, [10000.0 ** (-2.0 * i / 80) for i in range(40)], MIXED, [-f for f in BASE]], ids=["base", "odd", "mixed", "negative"])
def test_frequencies_are_held_to_64_bits(freq):
    """inv_freq / 2 pi in two doubles, each rounded to a whole number of 2^-64 turns: half a unit twice, and the quotient's error,
    2^-104 of it (4e8 / 2 pi: 2^-14 of a unit)."""
    decimal.getcontext().prec = 80
    two_pi, turn = 2 * decimal.Decimal(PI), 1 << 64
    held = qe.Rope(2 * len(freq), inv_freq=freq)._c.turns
    for f, t in zip(freq, held):
        off = (decimal.Decimal(t) - decimal.Decimal(f) / two_pi * turn) % turn
        off = min(abs(off), abs(off - turn), abs(off + turn))
        assert off <= decimal.Decimal("1.01"), f"{f}: {off:.1f} units of 2^-64 of a turn off"
