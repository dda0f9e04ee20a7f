"""The shapes of test_gpu_four_bits_scores.py reach every form of the attentions over keys in 4 bits."""
import test_gpu_four_bits_scores as scores
from test_four_bits_choice import FORMS, choose  # noqa: F401


def test_the_shapes_reach_every_form(choose):  # noqa: F811
    for d in (64, 128):
        assert {x[:2] for x in choose([(d, b * h, n, before + n) for b, h, before, n in scores.STEPS[d]], 1)} == FORMS
        got = choose([(d, b * h, n, keys) for b, h, n, keys in scores.CALLS[d]], 48)
        assert {x[:2] for x in got} == FORMS and any(x[2] > 1 for x in got)
