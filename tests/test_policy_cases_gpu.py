"""The measured cases of the policy loss: their loss is a number that 32 bits hold, so that kernel, plain form and definition can be compared."""
import random

import pytest

pytestmark = pytest.mark.gpu

# A row's term is off by some units of 2^-24 of it times the size of its log-probability (13 at most here): 10^-6 of the sum of the terms' magnitudes.
# Beside a loss of a twentieth of that sum this is 2e-5.
RELATIVE = 2e-5


def _cases():
    from perf import operators as ops
    few = next(c for c in ops.listed() if c["name"] == "policy_forward_few")
    rng, drawn = random.Random(7), []
    while len(drawn) < 12:
        c = ops.draw(rng)
        if c["op"] == "policy" and c["N"] * c["K"] <= 1 << 22:
            drawn.append(c)
    return [(few, seed) for seed in range(150)] + [(c, seed) for c in drawn for seed in range(8)]


def test_the_loss_of_a_case_does_not_cancel(monkeypatch):
    from perf import operators as ops
    off = []
    for case, seed in _cases():
        exact = float(ops.exact(case, seed)["loss"])
        loss = []
        for own in (False, True):
            monkeypatch.setattr(ops, "own", own)
            loss.append(float(ops.run(ops.prepare(case, seed))["loss"]))
        far = max(abs(loss[0] - exact), abs(loss[1] - exact), abs(loss[0] - loss[1]))
        if not far <= RELATIVE * abs(exact):
            off.append((case.get("name", (case["N"], case["K"])), seed, exact, loss))
    assert not off, off
