"""A language model that has diverged is not sampled from in silence."""
import sys

import pytest
import torch


@pytest.mark.gpu
def test_tokens_of_a_diverged_model_are_counted():
    from paper_2102_06280_amd import lm_study as L
    study = L.Study(3)
    try:
        logits = torch.randn(3, L.ROWS, L.VOCAB, device="cuda")
        study.sample(logits)
        assert study.diverged.item() == 0
        logits[1] = float("nan")
        logits[2, 5, 7] = float("inf")
        tokens = study.sample(logits)
        assert study.diverged.item() == L.ROWS + 1 and tokens.min() >= 0 and tokens.max() < L.VOCAB
        study.sample(logits)
        assert study.diverged.item() == 2 * (L.ROWS + 1)
    finally:
        study.close()


@pytest.mark.gpu
@pytest.mark.parametrize("experts", [0, 4])
def test_a_study_that_does_not_diverge_says_so(experts):
    from paper_2102_06280_amd import lm_study
    assert lm_study.run(workers=3, rounds=2, experts=experts)["diverged"] == 0


@pytest.mark.parametrize("diverged", [0, 7])
def test_the_command_fails_if_models_diverged(monkeypatch, capsys, diverged):
    from paper_2102_06280_amd import lm_study
    monkeypatch.setattr(lm_study, "run", lambda *a: {"distill_loss": [1.0], "status": 0, "diverged": diverged, "params": None})
    monkeypatch.setattr(sys, "argv", ["lm_study"])
    if diverged:
        with pytest.raises(SystemExit, match="7 tokens"):
            lm_study.main()
    else:
        lm_study.main()
    assert '"diverged": %d' % diverged in capsys.readouterr().out
