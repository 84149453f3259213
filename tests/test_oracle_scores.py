"""Pins of the oracle's label scores and 8-bit checkpoints (fp64, CPU): the
scores against torch's log_softmax and their gradient against autograd and
differences; the 8-bit format against its definition value by value, and its
backward pass against autograd of the restored unit."""
import numpy as np
import pytest
import torch

from oracle import sscn_oracle as O

RNG = np.random.default_rng


def _logits(rng, n, k, masked=False):
    z = rng.standard_normal((n, k)) * 3
    if masked:
        z[rng.random((n, k)) < 0.4] = -np.inf
        z[::5] = -np.inf
    return z


@pytest.mark.parametrize("n,k,masked", [(1, 1, False), (9, 2, False), (40, 7, False), (40, 33, True)])
def test_label_scores_are_torch_log_softmax(n, k, masked):
    rng = RNG(n + k)
    z = _logits(rng, n, k, masked)
    lab = rng.integers(-1, k, n)
    lp, H, stats, top, tlp = O.label_scores(z, lab, min(3, k))
    some = ~np.isneginf(z).all(axis=1)
    ref = torch.log_softmax(torch.from_numpy(z[some]), 1).numpy()
    want = np.where(lab[some] < 0, 0.0, ref[np.arange(some.sum()), np.maximum(lab[some], 0)])
    np.testing.assert_allclose(lp[some], want, rtol=1e-12, atol=1e-14)
    p = np.exp(ref)
    np.testing.assert_allclose(H[some], -(p * np.where(p > 0, ref, 0)).sum(axis=1), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(stats[some].sum(axis=1), torch.logsumexp(torch.from_numpy(z[some]), 1).numpy(), rtol=1e-13)
    st = torch.sort(torch.from_numpy(z), stable=True, dim=1, descending=True)
    np.testing.assert_array_equal(top, st.indices.numpy()[:, :top.shape[1]])
    np.testing.assert_allclose(tlp[some], np.take_along_axis(ref, top[some], 1), rtol=1e-12, atol=1e-14)
    assert (H[~some] == 0).all() and (stats[~some] == [-np.inf, 0]).all()
    assert np.isneginf(lp[~some & (lab >= 0)]).all() and (lp[lab < 0] == 0).all()


def test_label_scores_special_rows():
    nan, inf = np.nan, np.inf
    z = np.array([[1.0, nan, 2.0], [inf, 0.0, inf], [nan, inf, nan], [0.0, -0.0, 0.0]])
    lp, H, stats, top, tlp = O.label_scores(z, [0, 1, 2, 3], 3)
    assert np.isnan(lp).all() and np.isnan(H[:3]).all() and np.isnan(stats[:3, 1]).all() and np.isnan(tlp[:3]).all()
    np.testing.assert_array_equal(top, [[1, 2, 0], [0, 2, 1], [0, 2, 1], [0, 1, 2]])


@pytest.mark.parametrize("masked", [False, True])
def test_label_scores_gradient(masked):
    rng = RNG(3)
    n, k = 30, 11
    z = _logits(rng, n, k, masked)
    lab = rng.integers(-1, k, n)
    _, _, _, top, _ = O.label_scores(z, lab, 4)
    g, h, t = rng.standard_normal(n), rng.standard_normal(n), rng.standard_normal((n, 4))
    some = ~np.isneginf(z).all(axis=1)
    t[np.isneginf(np.take_along_axis(z, top, 1))] = 0.0     # a listed class that is excluded: its log p is constant
    g[np.isneginf(z[np.arange(n), np.maximum(lab, 0)])] = 0.0
    got = O.label_scores_backward(z, lab, g, h, top, t)
    assert (got[~some] == 0).all()
    tz = torch.from_numpy(z[some]).requires_grad_(True)
    logp = torch.log_softmax(tz, 1)
    safe = torch.where(torch.isinf(logp), torch.zeros((), dtype=logp.dtype), logp)
    H = -(torch.exp(logp) * safe).sum(1)
    tl = torch.from_numpy(lab[some])
    lp = torch.where(tl >= 0, safe.gather(1, tl.clamp(min=0)[:, None])[:, 0], torch.zeros((), dtype=logp.dtype))
    loss = (torch.from_numpy(g[some]) * lp).sum() + (torch.from_numpy(h[some]) * H).sum()
    loss = loss + (torch.from_numpy(t[some]) * safe.gather(1, torch.from_numpy(top[some]))).sum()
    loss.backward()
    np.testing.assert_allclose(got[some], np.nan_to_num(tz.grad.numpy()), rtol=1e-10, atol=1e-13)
    # and differences of the scores along a direction
    v = np.where(np.isneginf(z), 0.0, rng.standard_normal(z.shape))

    def value(zz):
        lp, H, _, _, _ = O.label_scores(zz, lab)
        logp = zz - np.logaddexp.reduce(np.where(some[:, None], zz, 0.0), axis=1, keepdims=True)
        picked = np.take_along_axis(logp, top, 1)
        return (np.where(g != 0, g * np.where(np.isinf(lp), 0, lp), 0) + np.where(some, h * H, 0)
                + np.where(some[:, None] & (t != 0), t * np.where(np.isinf(picked), 0, picked), 0).sum(1)).sum()
    eps = 1e-5
    diff = (value(z + eps * v) - value(z - eps * v)) / (2 * eps)
    assert abs(diff - (got * v).sum()) < 1e-6 * max(1.0, abs(diff))


@pytest.mark.parametrize("n,c", [(1, 1), (40, 31), (60, 32), (50, 70)])
def test_q8_format(n, c):
    rng = RNG(n + c)
    x = (rng.standard_normal((n, c)) * np.exp(rng.standard_normal((n, 1)) * 4)).astype(np.float32)
    x[n // 2] = 0.0
    x[0, 0] = 126.0                                          # 126 * 2^0 fits the step 2^0 ...
    if n > 1:
        x[1, 0] = np.nextafter(np.float32(126), np.float32(200))   # ... and the next number does not
    gamma = rng.normal(0, 1, c).astype(np.float32)
    gamma[c // 2] = 0.0
    beta = rng.normal(0, 1, c).astype(np.float32)
    one, zero = np.ones(c, np.float32), np.zeros(c, np.float32)
    codes, exps = O.q8_encode(x, zero, one, gamma, gamma, beta)   # xhat = x
    v = O.q8_values(codes, exps)
    step = O._q8_per_channel(np.ldexp(1.0, exps.astype(int) - 127), c)
    for i in range(exps.shape[1]):
        at = slice(32 * i, 32 * i + 32)
        most = np.abs(x[:, at].astype(np.float64)).max(axis=1)
        s = np.ldexp(1.0, exps[:, i].astype(int) - 127)
        assert (most <= 126 * s).all() and ((most > 63 * s) | (exps[:, i] == 1)).all()
    on = gamma.astype(np.float64) * x + beta > 0
    np.testing.assert_array_equal(gamma.astype(np.float64) * v + beta > 0, on)
    off = np.abs(v - x) / step
    moved = off > 0.5
    assert (off <= 1.5).all() and moved.mean() < 0.1
    # a code is moved only where rounding alone changes the mask
    plain = np.rint(x / step) * step
    assert ((gamma.astype(np.float64) * plain + beta > 0) != on)[moved].all()
    if n > 1 and c == 32:
        assert exps[0, 0] == 127 or np.abs(x[0]).max() > 126
        assert exps[n // 2, 0] == 1 and (v[n // 2] == 0).all() or (codes[n // 2] != 0).any()


def test_q8_not_finite():
    x = np.ones((3, 40), np.float32)
    x[0, 3], x[1, 35] = np.nan, -np.inf
    one, zero = np.ones(40, np.float32), np.zeros(40, np.float32)
    codes, exps = O.q8_encode(x, zero, one, one, one, zero)
    np.testing.assert_array_equal(exps == 255, [[True, False], [False, True], [False, False]])
    v = O.q8_values(codes, exps)
    assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:]).all() and np.isfinite(v[2]).all()


def test_q8_backward_is_autograd_of_the_restored_unit():
    """dgamma, dbeta and a from autograd through relu(gamma v + beta); dx is
    the batch normalisation's gradient with v in the normalised input's place:
    the projection of gamma invstd dz that removes its mean and its part along v."""
    rng = RNG(5)
    n, c = 64, 40
    x = rng.standard_normal((n, c)).astype(np.float32)
    mean, var = x.mean(0), x.var(0)
    invstd = (1 / np.sqrt(var + 1e-5)).astype(np.float32)
    gamma, beta = rng.uniform(0.5, 1.5, c).astype(np.float32), rng.normal(0, 0.5, c).astype(np.float32)
    codes, exps = O.q8_encode(x, mean, invstd, gamma * invstd, gamma, beta)
    dA = rng.standard_normal((n, c))
    a, dX, dg, db = O.batch_norm_relu_backward_q8(dA, codes, exps, gamma, beta, invstd)
    v = torch.from_numpy(O.q8_values(codes, exps))
    tg, tb = (torch.from_numpy(t.astype(np.float64)).requires_grad_(True) for t in (gamma, beta))
    y = torch.relu(tg * v + tb)
    (y * torch.from_numpy(dA)).sum().backward()
    np.testing.assert_allclose(a, y.detach().numpy(), rtol=1e-14)
    np.testing.assert_allclose(dg, tg.grad.numpy(), rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(db, tb.grad.numpy(), rtol=1e-11, atol=1e-12)
    # near the full-precision gradient: the codes are off by at most 2^-7 of a block's largest value
    full, fg, fb = O.batch_norm_relu_backward(dA, x, gamma, beta, x.mean(0, np.float64), x.astype(np.float64).var(0))
    assert np.linalg.norm(dX - full) < 2 ** -6 * np.linalg.norm(full)
    np.testing.assert_allclose(db, fb, rtol=1e-9, atol=1e-9)   # the same mask: dbeta does not see the codes
