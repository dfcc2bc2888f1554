"""Planted mistakes in the oracle's log probabilities, their gradient and the loss from top log
probabilities: each is caught by at least one of its pins."""
import numpy as np
import pytest

import test_oracle_logprobs as TL
from oracle import logprobs as OL

PINS = [
    (TL.test_log_probabilities_are_log_softmax, (0.6,)),
    (TL.test_alternatives_break_ties_by_the_lowest_id, ()),
    (TL.test_rows_without_a_distribution, ()),
    (TL.test_gradient_is_autograd, (True, True, 2.0)),
    (TL.test_full_lists_give_the_full_vocabulary_loss, (False,)),
    (TL.test_topk_gradient_is_autograd, (True, 1.7)),
    (TL.test_topk_gradient_is_autograd, (False, 0.8)),
    (TL.test_teacher_rows_without_entries_and_equal_distributions, ()),
]
forward, backward, topk = OL.token_logprobs, OL.token_logprobs_grad, OL.topk_ce


def _edit(**changes):
    def f(logits, tokens=None, T=1.0, n_top=0):
        out = forward(logits, tokens, T, n_top)
        for k, change in changes.items():
            out[k] = change(out, np.asarray(logits, np.float64), T)
        return out
    return {"token_logprobs": f}


def _highest_id(logits, tokens=None, T=1.0, n_top=0):
    out = forward(np.asarray(logits)[:, ::-1], None, T, n_top)
    ids = np.where(out["top_ids"] >= 0, np.shape(logits)[1] - 1 - out["top_ids"], -1)
    return dict(forward(logits, tokens, T, n_top), top_ids=ids)


MISTAKES = {
    "no temperature": {"token_logprobs": lambda x, tok=None, T=1.0, n_top=0: forward(x, tok, 1.0, n_top)},
    "entropy in bits": _edit(entropy=lambda o, x, T: o["entropy"] / np.log(2.0)),
    "maximum divided by the temperature": _edit(stats=lambda o, x, T: o["stats"] / [[T, 1.0]]),
    "ties by the highest id": {"token_logprobs": _highest_id},
    "masked logits among the alternatives":
        _edit(top_ids=lambda o, x, T: np.argsort(-x, kind="stable")[:, :o["top_ids"].shape[1]]),
    "no inner derivative": {"token_logprobs_grad": lambda x, t, g, h, T=1.0: T * backward(x, t, g, h, T)},
    "entropy's gradient of the other sign":
        {"token_logprobs_grad": lambda x, t, g, h, T=1.0: backward(x, t, g, None if h is None else -np.asarray(h), T)},
    "no tail": {"topk_ce": lambda i, l, x, t, s, T=1.0, tail=True: topk(i, l, x, t, s, T, False)},
    "not renormalised": {"topk_ce": lambda i, l, x, t, s, T=1.0, tail=True: topk(i, l, x, t, s, T, True)},
    "sum over pairs instead of the mean":
        {"topk_ce": lambda i, l, x, t, s, T=1.0, tail=True:
         (lambda r: (r[0] * max(1, len(t)), r[1], r[2] * max(1, len(t))))(topk(i, l, x, t, s, T, tail))},
}


@pytest.mark.parametrize("name", sorted(MISTAKES))
def test_pins_catch(name):
    failed = 0
    with pytest.MonkeyPatch.context() as mp:
        for attr, fn in MISTAKES[name].items():
            mp.setattr(TL, attr, fn)
        for pin, args in PINS:
            try:
                pin(*args)
            except AssertionError:
                failed += 1
    assert failed, name


def test_the_pins_pass_without_a_mistake():
    for pin, args in PINS:
        pin(*args)
