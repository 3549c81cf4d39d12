"""The example that answers from retrieved passages, against the same model without cache, pages or beams."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_from_passages.py")


@pytest.mark.parametrize("kw", [dict(), dict(queries=5, micro=2, beams=7, new=6, passage_tokens=257, question_tokens=1, seed=3)])
def test_scores_are_those_of_the_answers(kw):
    spec = importlib.util.spec_from_file_location("answer_from_passages", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model, answers = example.answer(**kw)
    for prompt, found in answers:
        scores = [s for s, _ in found]
        assert scores == sorted(scores, reverse=True)
        assert len({tuple(text) for _, text in found}) == len(found)
        for score, text in found:
            # queries, keys, values and attention's results are rounded to 11 bits in each of two layers: a logit of about 6 moves by
            # 8 * 2^-11 of that, and so does the logarithm of the sum
            assert abs(score - example.plain_score(model, prompt, text)) < len(text) * 2 * 6 * 8 * 2.0 ** -11
