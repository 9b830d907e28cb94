"""Cases drawn as the operators' benchmark draws them: the library's calls are taken and give what the plain form gives."""
import os
import random
import sys

import pytest
import torch

from conftest import ROOT

sys.path.insert(0, os.path.join(ROOT, "perf"))
import more_operators as cases  # noqa: E402

pytestmark = pytest.mark.gpu


def drawn(seed):
    c = cases.draw(random.Random(seed))
    work = cases.work(c)
    return c if work["bytes"] <= 1 << 29 and work["flops"] <= 2e11 else None


# the step's gradients without a norm of r, and others of every kind
SEEDS = [s for s in range(60) if drawn(s)]


@pytest.mark.parametrize("seed", SEEDS)
def test_a_drawn_case(seed, monkeypatch):
    c, out = drawn(seed), []
    for own in (False, True):
        monkeypatch.setattr(cases, "own", own)
        out.append({k: t.double().clone() for k, t in cases.run(cases.prepare(c, seed)).items()})
    assert set(out[0]) == set(out[1])
    for k, want in out[0].items():
        # both round once to 8 bits at least: 2^-8 of each value, that of a sum in another order far less; sums of many terms may cancel
        assert float((out[1][k] - want).norm()) <= 2.0 ** -8 * float(want.norm()) + 1e-30, (c, k)


def test_every_kind_is_drawn():
    kinds = {(c["op"], c.get("norm_r")) for c in map(drawn, SEEDS)}
    assert {("step_bwd", "none"), ("step_bwd", "layer"), ("step_fwd", "none"), ("quantize", None), ("product", None), ("clip", None)} <= kinds
