"""The coefficients of an orthogonalised update, checked before anything else is."""
import pytest
import torch

from paper_2607_24953_b200 import binding as b


@pytest.mark.parametrize("bad", [((1.5, -0.5), (0.0, 1.5, -0.5, 0.0)), ((1.5, -0.5, 0.0), (1.5, -0.5)), ((1.5, -0.5, 0.0, 0.0),), ((),), (), ((1.5, -0.5),) * 3])
def test_steps_that_are_no_triples_are_refused(bad):
    with pytest.raises(ValueError, match="triples"):
        b.fp4q_newton_schulz(torch.zeros(8, 16), coefficients=bad)


def test_triples_of_any_sequence_reach_the_next_check():
    for good in (((1.5, -0.5, 0.0),), [[1.5, -0.5, 0.0]] * 2, torch.tensor([[1.5, -0.5, 0.0]]), iter([(1.5, -0.5, 0.0)])):
        with pytest.raises(ValueError, match="CUDA"):
            b.fp4q_newton_schulz(torch.zeros(8, 16), coefficients=good)
