"""The time that the library counts for pairs of CTAs is that of a way that the call can go (the library's own model, no GPU)."""
import ctypes

import pytest

from test_fp8_abi import roi  # noqa: F401  (the fixture)


class Plan(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int), ("outputs", ctypes.c_bool)]


@pytest.fixture(scope="module")
def cycles(roi):  # noqa: F811
    # roi::fp8_pair_cycles(long, long, long, bool, int, Fp8PairPlan&)
    f = roi.lib()._ZN3roi15fp8_pair_cyclesElllbiRNS_11Fp8PairPlanE
    f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_bool, ctypes.c_int, ctypes.POINTER(Plan)]
    f.restype = ctypes.c_int64

    def call(T, outs, width, tokens):
        plan = Plan()
        return f(T, outs, width, tokens, 76, ctypes.byref(plan)), plan
    return call


def rounds(m, n, width, at):
    """Cycles by the model of tiles of 256 x `at` on 76 pairs."""
    tiles = -(-m // 256) * -(-n // at)
    return -(-tiles // 76) * ((256 + at) * -(-width // 128) + 2000) + 4000


@pytest.mark.parametrize("T,outs,width", [(4697, 896, 896), (4352, 896, 1001), (500, 6656, 364), (8192, 18944, 3584), (2000, 4880, 1000),
                                          (300, 3328, 6769), (1, 1, 1)])
def test_only_ways_that_are_open_count(cycles, T, outs, width):
    best = lambda m, n: min(rounds(m, n, width, at) for at in range(64, 225, 32))  # noqa: E731
    by_tokens, by_outputs = best(T, outs), best(outs, T)
    got, plan = cycles(T, outs, width, False)
    assert got == by_outputs and plan.outputs and rounds(outs, T, width, plan.n) == got
    got, plan = cycles(T, outs, width, True)
    assert got == min(by_tokens, by_outputs) and plan.outputs == (by_outputs < by_tokens)
    assert rounds(*((outs, T) if plan.outputs else (T, outs)), width, plan.n) == got


def test_a_closed_way_was_counted(cycles):
    """An input gradient of 4697 tokens, 896 x 896: 13376 cycles by outputs, the only way open to it, against 9616 of single CTAs."""
    assert cycles(4697, 896, 896, False)[0] == 13376 > 9616 > cycles(4697, 896, 896, True)[0]
