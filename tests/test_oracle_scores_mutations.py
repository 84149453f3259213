"""Mistakes planted in the oracle's label scores and 8-bit checkpoints: the
pins of test_oracle_scores.py catch each of them."""
import numpy as np

from oracle import sscn_oracle as O
from tests import test_oracle_scores as T


def _holds(*checks):
    try:
        for c in checks:
            c()
    except AssertionError:
        return False
    return True


def _scores():
    T.test_label_scores_are_torch_log_softmax(40, 33, True)
    T.test_label_scores_are_torch_log_softmax(40, 7, False)
    T.test_label_scores_special_rows()


def _format():
    T.test_q8_format(60, 32)
    T.test_q8_format(50, 70)


def test_the_pins_hold_unchanged():
    assert _holds(_scores, lambda: T.test_label_scores_gradient(True), _format, T.test_q8_not_finite,
                  T.test_q8_backward_is_autograd_of_the_restored_unit)


def test_unlabelled_rows_scored_caught(monkeypatch):
    orig = O.label_scores
    monkeypatch.setattr(O, "label_scores", lambda z, lab, k=0: orig(z, None if lab is None else np.abs(lab), k))
    assert not _holds(_scores)


def test_ties_to_the_highest_class_caught(monkeypatch):
    orig = O.label_scores

    def bad(z, lab, k=0):
        z = np.asarray(z, np.float64)
        out = list(orig(z[:, ::-1], None if lab is None else z.shape[1] - 1 - np.asarray(lab), k))
        return (*orig(z, lab, k)[:3], z.shape[1] - 1 - out[3], out[4])
    monkeypatch.setattr(O, "label_scores", bad)
    assert not _holds(_scores)


def test_entropy_gradient_without_its_mean_caught(monkeypatch):
    orig = O.label_scores_backward

    def bad(z, lab, g=None, h=None, top=None, t=None):
        d = orig(z, lab, g, h, top, t)
        if h is None:
            return d
        _, H, st, _, _ = O.label_scores(z, None)
        some = ~np.isneginf(st[:, 0])
        p = np.where(some[:, None], np.exp(np.asarray(z) - np.where(some, st.sum(1), 0.0)[:, None]), 0.0)
        return d + h[:, None] * p * H[:, None]
    monkeypatch.setattr(O, "label_scores_backward", bad)
    assert not _holds(lambda: T.test_label_scores_gradient(False))


def test_codes_that_only_round_caught(monkeypatch):
    orig = O.q8_encode

    def bad(x, mean, invstd, scale, gamma, beta):
        return orig(x, mean, invstd, 0 * np.asarray(scale), 0 * np.asarray(gamma), beta)
    monkeypatch.setattr(O, "q8_encode", bad)
    assert not _holds(_format)


def test_a_step_too_large_caught(monkeypatch):
    orig = O.q8_encode

    def bad(*a):
        codes, exps = orig(*a)
        return (codes.astype(int) // 2).astype(np.int8), (exps + (exps < 255)).astype(np.uint8)
    monkeypatch.setattr(O, "q8_encode", bad)
    assert not _holds(_format)


def test_block_with_a_nan_kept_finite_caught(monkeypatch):
    orig = O.q8_values
    monkeypatch.setattr(O, "q8_values", lambda c, e: np.nan_to_num(orig(c, e)))
    assert not _holds(T.test_q8_not_finite)


def test_restored_backward_without_its_mask_caught(monkeypatch):
    orig = O.batch_norm_relu_backward_q8

    def bad(dA, codes, exps, gamma, beta, invstd):
        a, _, dg, db = orig(dA, codes, exps, gamma, beta, invstd)
        return (a, *orig(dA, codes, exps, gamma, np.asarray(beta) + 1e6, invstd)[1:])
    monkeypatch.setattr(O, "batch_norm_relu_backward_q8", bad)
    assert not _holds(T.test_q8_backward_is_autograd_of_the_restored_unit)
