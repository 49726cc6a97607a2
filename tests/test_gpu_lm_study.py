"""Language models trained through the losses on logits and the rounds: every stage gets better at what it minimises, twice the same way."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_every_stage_learns_and_repeats():
    from paper_2102_06280_amd import binding as B
    from paper_2102_06280_amd import lm_study
    a = lm_study.run(workers=4, rounds=30)
    assert a["status"] == B.OK
    first, last = lambda v: np.mean(v[:5]), lambda v: np.mean(v[-5:])
    assert last(a["distill_loss"]) < 0.9 * first(a["distill_loss"])
    assert abs(a["preference_loss"][0] - np.log(2)) < 1e-6 and abs(a["margin"][0]) < 1e-4      # the model is its own reference
    assert last(a["preference_loss"]) < 0.9 * np.log(2) and last(a["margin"]) > 0
    assert last(a["reward"]) > first(a["reward"])
    assert abs(a["kl"][0]) < 0.5 and min(a["kl"]) >= 0
    b = lm_study.run(workers=4, rounds=30)
    assert np.array_equal(a["params"], b["params"])
