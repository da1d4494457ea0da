"""The rotary plan's turns against rational arithmetic: a frequency over 2 pi, modulo 1, to the last of 64 bits."""
import random
from fractions import Fraction

import __graft_entry__

__graft_entry__._build_module().build()
import paper_2609_35593_gb300 as ress  # noqa: E402

# 2 pi to 140 digits
TWO_PI = Fraction("6.283185307179586476925286766559005768394338798750211641949889184615632812572417997256069650684"
                  "23413596429617302656461329418768921910116446345")


def off(turns, f):
    """Distance of turns 2^-64 from f / 2 pi modulo 1, in units of 2^-64."""
    d = (Fraction(turns, 2 ** 64) - Fraction(f) / TWO_PI) % 1
    return float(min(d, 1 - d) * 2 ** 64)


def test_turns_are_good_to_the_last_bit():
    rng = random.Random(3)
    freq = [100.0, 1000.0, -1e-4, -1.0, 1.0, 0.7, 3.1e-5, 1e-9, -1e-18, 1e-30, -5e-324, 0.0, -0.0, 12345.678, -3e5, 2.0 ** 40,
            6.283185307179586, -6.283185307179586, 3.141592653589793]
    freq += [rng.choice([-1, 1]) * 2.0 ** rng.uniform(-60, 40) for _ in range(100 - len(freq))]
    plan = ress.rope_plan((200,), head_dim=200, layout="halves", freq=freq)
    for k, f in enumerate(freq):
        # the rounding to 64 bits, and that of 1 / 2 pi to two words (2^-106 of the turns)
        assert off(plan.turns[k], f) <= 0.5 + abs(f) / 6.28 * 2.0 ** (64 - 104), f


def test_turns_of_frequencies_beyond_a_turn_of_2_to_the_64():
    """Of frequencies that large the two words of 1 / 2 pi keep 2^-104, and nothing is lost beside that."""
    freq = [2.0 ** 60, -1e20, 3.3e25]
    plan = ress.rope_plan((6,), head_dim=6, layout="halves", freq=freq)
    for k, f in enumerate(freq):
        assert off(plan.turns[k], f) <= 1 + abs(f) / 6.28 * 2.0 ** (64 - 104), f
    ress.rope_plan((2,), head_dim=2, layout="halves", freq=[1.7e308])  # finite: a plan, of some angle


def test_a_negative_frequency_turns_back_what_its_positive_one_turns():
    freq = [0.3, 1e-4, 77.0, 1e-17]
    a = ress.rope_plan((8,), head_dim=8, layout="halves", freq=freq)
    b = ress.rope_plan((8,), head_dim=8, layout="halves", freq=[-f for f in freq])
    for k in range(4):
        assert (a.turns[k] + b.turns[k]) % 2 ** 64 == 0
