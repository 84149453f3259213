"""Ends of the ranges that the operators on a training step's two ends allow.
Against the fp64 oracle."""
import types
import weakref

import numpy as np
import pytest
import torch

from oracle import sscn_oracle as O
from paper_1711_10275_amd import sscn, train, unet
from paper_1711_10275_amd import synthetic as S
from tests.gpu_common import dev, host
from tests.test_gpu_checkpoint import TD, U, half_step, strided

pytestmark = pytest.mark.gpu


def test_values_of_every_exponent_byte():
    """Row b has the byte b: q * 2^(b - 127), exact, infinite where fp32 is;
    NaN for 255 whatever the codes."""
    rng = np.random.default_rng(1)
    codes = rng.integers(-128, 128, (256, 45)).astype(np.int8)
    codes[:, :6] = [0, 1, -1, 127, -127, -128]
    exps = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 2, axis=1)
    with np.errstate(over="ignore"):
        want = O.q8_values(codes, exps).astype(np.float32)
    q8 = sscn.Q8(dev(codes), dev(exps))
    for kind in TD.values():
        np.testing.assert_array_equal(host(sscn.q8_values(q8, kind)), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bytes_", [(240, 251), (0, 3)])
def test_backward_from_large_and_small_steps(bytes_, dtype):
    """Values up to 2^128 and down to 2^-127.  Tolerances as in
    test_gpu_checkpoint.py: sums are fp64 and rounded once; dx carries up to
    nine half steps of its terms' sizes, which stay far from the ends of the
    type here (dA and dgamma are made small where the values are large)."""
    rng = np.random.default_rng(sum(bytes_))
    n, c = 300, 70
    codes = rng.integers(-31, 32, (n, c)).astype(np.int8)
    exps = rng.integers(*bytes_, (n, 3)).astype(np.uint8)
    v = O.q8_values(codes, exps)
    gamma = rng.uniform(0.5, 1, c).astype(np.float32) * np.where(rng.random(c) < 0.5, 1, -1).astype(np.float32)
    beta = rng.normal(0, 1, c).astype(np.float32)
    big = bytes_[0] > 0
    if not big:
        beta[::2] = 0.0         # the mask goes by the small values themselves
    invstd = rng.uniform(0.5, 2, c).astype(np.float32)
    dA = host(dev((rng.standard_normal((n, c)) * (1e-30 if big else 1)).astype(np.float32), TD[dtype]))
    tA, tg, tb, q8 = dev(dA, TD[dtype]), dev(gamma), dev(beta), sscn.Q8(dev(codes), dev(exps))
    pre = gamma.astype(np.float64) * v + beta
    dz = np.where(pre > 0, dA.astype(np.float64), 0.0)
    got_g, got_b, got_a = sscn.batchnorm_relu_backward_params_q8(tA, q8, tg, tb, restore=True)
    size = np.abs(dA).astype(np.float64)
    least = 2.0 ** -149         # a whole number of these: half of one is a rounding there
    assert (np.abs(host(got_b) - dz.sum(0)) <= U * np.abs(dz.sum(0)) + 2.0 ** -50 * n * size.sum(0) + least).all()
    dg = (dz * v).sum(0)
    assert (np.abs(host(got_g) - dg) <= U * np.abs(dg) + 2.0 ** -50 * n * (size * np.abs(v)).sum(0) + least).all()
    a = np.where(pre <= 0, 0.0, pre)
    assert (np.abs(host(got_a) - a) <= (U + half_step(dtype)) * a * (1 + 1e-6) + 2.0 ** -133).all()
    # the input's gradient: dgamma as the caller gives it
    dA2 = host(dev(rng.standard_normal((n, c)).astype(np.float32), TD[dtype]))
    g2 = (rng.standard_normal(c) * n * (1e-36 if big else 1)).astype(np.float32)
    b2 = (rng.standard_normal(c) * n).astype(np.float32)
    gi = gamma.astype(np.float64) * invstd
    dz = np.where(pre > 0, dA2.astype(np.float64), 0.0)
    dx = gi * (dz - b2.astype(np.float64) / n - v * g2.astype(np.float64) / n)
    terms = np.abs(gi) * (np.abs(dA2) + np.abs(b2) / n + np.abs(v * g2) / n)
    for lo, hi in [(0, 70), (32, 70), (1, 70), (33, 64)]:
        out = sscn.batchnorm_relu_backward_input_q8(dev(dA2, TD[dtype]), q8, tg, tb, dev(invstd), dev(g2), dev(b2),
                                                    torch.empty((n, hi - lo), dtype=TD[dtype], device="cuda:0"), cols=(lo, hi))
        # (dgamma / n may be subnormal: off by half of 2^-149 more, times v)
        b = 9 * U * terms[:, lo:hi] + U * np.abs(dx[:, lo:hi]) + np.abs(gi * v)[:, lo:hi] * 2.0 ** -149
        b = b + half_step(dtype) * (np.abs(dx[:, lo:hi]) + b)
        assert (np.abs(host(out) - dx[:, lo:hi]) <= b).all(), (lo, hi)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_kept_values_near_the_types_end(dtype):
    """Statistics that leave xhat at 10^38: the codes are the oracle's, and the
    backward pass masks what the forward masked."""
    rng = np.random.default_rng(3)
    n, c = 200, 70
    x = host(dev((rng.uniform(-3e38, 3e38, (n, c))).astype(np.float32), TD[dtype]))
    x[::3] *= np.float32(2.0 ** -8)
    gamma = np.where(rng.random(c) < 0.5, 1, -1).astype(np.float32) * rng.uniform(0.25, 0.5, c).astype(np.float32)
    beta = (rng.standard_normal(c) * 3e37).astype(np.float32)
    zero, one = np.zeros(c, np.float32), np.ones(c, np.float32)
    st = types.SimpleNamespace(mean=dev(zero), invstd=dev(one), scale=dev(gamma))
    t = dev(x, TD[dtype])
    a, q8 = sscn.batchnorm_relu_apply_q8(t, st, dev(gamma), dev(beta))
    codes, exps = O.q8_encode(x, zero, one, gamma, gamma, beta)
    np.testing.assert_array_equal(host(q8.exponents), exps)
    np.testing.assert_array_equal(host(q8.codes), codes)
    assert (exps >= 248).mean() > 0.5 and exps.max() < 255
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(host(sscn.q8_values(q8)), O.q8_values(codes, exps).astype(np.float32))
    _, _, back = sscn.batchnorm_relu_backward_params_q8(torch.zeros_like(t), q8, dev(gamma), dev(beta), restore=True)
    assert torch.equal(a > 0, back > 0) and 0.2 < (a > 0).float().mean() < 0.8


@pytest.mark.parametrize("k", [12, 100, 700, 3001])
def test_a_label_that_is_none_in_a_row_that_allows_nothing(k):
    """The label wins: the log probability and the gradient are NaN both."""
    z = np.random.default_rng(k).standard_normal((8, k)).astype(np.float32)
    z[::2] = -np.inf
    lab = np.array([k, k, 0, 0, -1, -1, k + 5, 1], np.int32)
    zt = dev(z)
    got = sscn.label_scores(zt, dev(lab), 2)
    g, t = np.ones(8, np.float32), np.ones((8, 2), np.float32)
    for dtop in (None, t):
        d = host(sscn.label_scores_backward(zt, got, dev(lab), dlogprob=dev(g), dtop=dev(dtop) if dtop is not None else None))
        want = O.label_scores_backward(z, lab, g, None, host(got.top_index), dtop)
        bad = lab >= k
        np.testing.assert_array_equal(np.isnan(host(got.logprob)), bad)
        assert np.isnan(d[bad]).all() and np.isnan(want[bad]).all()
        assert (d[[2, 4]] == 0).all() and (want[[2, 4]] == 0).all()
        assert np.abs(d[~bad] - want[~bad]).max() < 1e-5
    # without a gradient at the log probabilities the label is not looked at
    assert (host(sscn.label_scores_backward(zt, got, dev(lab), dentropy=dev(g)))[::2] == 0).all()


def test_a_training_step_lets_go_of_what_it_restored(monkeypatch):
    """On kept codes a unit's restored activations go before its input's
    gradient is written, and its dA before the next unit's: nothing of one
    unit's backward pass is held through the next one's."""
    restored, grads = [], []
    params, inputs = sscn.batchnorm_relu_backward_params_q8, sscn.batchnorm_relu_backward_input_q8

    def params_(dA, *a, **k):
        assert not [1 for r in grads if r() is not None]
        out = params(dA, *a, **k)
        grads.append(weakref.ref(dA))
        restored.append(weakref.ref(out[2]))
        return out

    def inputs_(*a, **k):
        assert not [1 for r in restored if r() is not None]
        return inputs(*a, **k)
    monkeypatch.setattr(sscn, "batchnorm_relu_backward_params_q8", params_)
    monkeypatch.setattr(sscn, "batchnorm_relu_backward_input_q8", inputs_)
    n_classes, ch = 5, (8, 16)
    coords = S.scenes_small(batch=1, L=32, target_per_sample=1000)
    geom = train.Geometry(dev(coords), (32, 32, 32), levels=2)
    P = train.Params(ch, n_classes, S.train_params)
    x, lab = dev(S.features(coords.shape[0], ch[0], 1)), dev(S.labels(coords.shape[0], n_classes, 2))
    train.train_step(x, lab, geom, P, update=False, keep="q8")
    assert len(restored) == len(unet.units(ch)) + 1
    # traced, the activations stay for the caller
    monkeypatch.undo()
    trace = {}
    train.train_step(x, lab, geom, P, update=False, keep="q8", trace=trace)
    assert all(e["a"].shape == e["da"].shape for e in trace.values())


def test_a_row_of_as_many_classes_as_an_int_counts():
    """The last chunk of a row of 2^31 - 1 logits: best classes from its list,
    from the row itself (more equal logits than a list holds, a NaN), and the
    gradient."""
    k = 2 ** 31 - 1
    z = torch.full((1, k), -float("inf"), dtype=torch.bfloat16, device="cuda:0")
    at = [k - 1, 2 ** 30, 5]
    for j, v in zip(at, (3.0, 2.0, 1.0)):
        z[0, j] = v
    lab = torch.tensor([k - 1], dtype=torch.int32, device="cuda:0")
    got = sscn.label_scores(z, lab, 3)
    want = O.label_scores(np.array([[3.0, 2.0, 1.0]]), [0], 3)
    assert host(got.top_index).tolist() == [at]
    for a, b in zip((got.logprob, got.entropy, got.stats, got.top_logprob), (want[0], want[1], want[2], want[4])):
        assert np.abs(host(a) - b).max() < 1e-6
    d = sscn.label_scores_backward(z, got, lab, dlogprob=torch.ones(1, device="cuda:0"))
    grad = O.label_scores_backward(np.array([[3.0, 2.0, 1.0]]), [0], [1.0])
    assert np.abs(host(d[0, torch.tensor(at, device="cuda:0")]) - grad).max() < 2 ** -8
    assert int(torch.count_nonzero(d)) == 3
    del d
    z[0, k - 3000:] = 3.0
    assert host(sscn.label_scores(z, lab, 2).top_index).tolist() == [[k - 3000, k - 2999]]
    z[0, k - 2] = float("nan")
    got = sscn.label_scores(z, lab, 2)
    assert host(got.top_index).tolist() == [[k - 2, k - 3000]] and torch.isnan(got.entropy).all()
