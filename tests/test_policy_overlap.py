"""The policy loss refuses results in the place of its arguments or of each other: a row's threads read
the arguments while one of them writes the results (no GPU: every call is refused before a launch)."""
import ctypes

import pytest

from paper_2606_10820_amd import binding as Bd

P = ctypes.c_void_p
ARGS = ("x", "tok", "adv", "old", "ref", "w")
RESULTS = ("rl", "lp", "ra", "kl", "h", "loss")


def _call(**kw):
    a = {n: P(0x10000 * (i + 1)) for i, n in enumerate(ARGS + RESULTS + ("d",))}
    a.update(kw)
    return Bd.lib().kf_policy_loss(None, 1, 3, 100, a["x"], 100, a["tok"], a["adv"], a["old"], a["ref"], a["w"], 0.8, 1.2, 0.1, 0.1, a["rl"], a["lp"], a["ra"], a["kl"],
                                   a["h"], a["loss"], a["d"], 100)


@pytest.mark.parametrize("result", RESULTS)
def test_results_over_arguments(result):
    at = P(0x700000)
    for other in ARGS + tuple(n for n in RESULTS if n != result) + ("d",):
        assert _call(**{result: at, other: at}) == Bd.KF_EINVAL, other


@pytest.mark.parametrize("arg", ARGS[1:])
def test_gradient_over_arguments(arg):
    at = P(0x700000)
    assert _call(**{arg: at, "d": at}) == Bd.KF_EINVAL
