"""Label scores and their gradient on the GPU against the fp64 oracle.

Tolerances, u = 2^-24 (half a step of fp32), t = sum of exp(x - max) but one
largest, w_k = exp(x_k - max):
 - w_k = 2^(d_k log2 e) is off by (2 + 2.25 |d_k|) u of itself: the difference
   d_k rounded is |d_k| u in the exponent (in units of e), its product with
   log2 e rounded another |d_k| u, the constant itself, 1.44269502162933 for
   1.44269504088896, another 1.34e-8 |d_k| = 0.23 |d_k| u; the power of two is
   good to 1 ulp; a sum over N terms of at most A additions in a row adds A u.
   Additions in a row: at most 64 where one thread adds a row, else a lane's
   share (classes / 64 at most) and the joins; A = min(classes, 64) + classes / 64 + 24.
 - L = log1p(t): t / (1 + t) times t's error, plus 2 ulp of the function.
 - H = L - sum w d / (1 + t): the same for sum w d, whose terms are off by
   (4 + 2.25 |d|) u of themselves.
 - log p_k = (x_k - max) - L: two roundings and L's error.
 - the gradient: log p is off by the above, p by that times p; each product and
   sum of the formula adds a rounding of its terms; one rounding to the
   logits' type at the end.
"""
import numpy as np
import pytest
import torch

from oracle import sscn_oracle as O
from paper_1711_10275_amd import sscn
from paper_1711_10275_amd import synthetic as S
from tests.gpu_common import dev, host

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def draw(n, k, dtype, seed, kind="plain"):
    """Logits (values of the type) and labels, -1 among them."""
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((n, k)).astype(np.float32) * 3
    z[np.arange(n), rng.integers(0, k, n)] += rng.uniform(0, 20, n).astype(np.float32)
    if kind == "masked":
        z[rng.random((n, k)) < 0.5] = -np.inf
        z[::7] = -np.inf
    elif kind == "lowest":      # masks of the type's lowest value, alone in some rows
        low = np.finfo(np.float32).min if dtype == "f32" else -3.3895313892515355e38
        z[rng.random((n, k)) < 0.5] = low
        z[::7] = low
    elif kind == "ties":
        z = np.rint(z / 3).astype(np.float32)
        z[::5] = 0.0
        z[1::5] *= -0.0
    elif kind == "sure":        # one class far above the rest
        z[np.arange(n), rng.integers(0, k, n)] += 60
    lab = rng.integers(-1, k, n).astype(np.int32)
    return (S.bf16_round(z) if dtype == "bf16" else z), lab


def on_gpu(z, dtype, pad=0):
    t = dev(z, TD[dtype])
    if not pad:
        return t
    wide = torch.full((z.shape[0], z.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :z.shape[1]] = t
    return wide[:, :z.shape[1]]


def near(got, want, bound, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)], err_msg=what)
    err = np.abs(got - want)[fine]
    b = np.broadcast_to(bound, want.shape)[fine]
    assert (err <= b).all(), f"{what}: worst {np.max(err / np.maximum(b, 1e-300)):.3g} of its bound"


def sums(z):
    """Per row: d, w, t, and the additions in a row A."""
    z = z.astype(np.float64)
    m = z.max(axis=1, keepdims=True)
    d = np.where(np.isneginf(z), -1e4, z - np.where(np.isneginf(m), 0.0, m))
    w = np.exp(d)
    k = z.shape[1]
    rest = w.copy()
    rest[np.arange(len(z)), w.argmax(axis=1)] = 0.0      # t is a sum without the 1: it may be far below it
    return d, w, rest.sum(axis=1), min(k, 64) + k / 64 + 24


def bounds(z):
    d, w, t, A = sums(z)
    wd, wdd = (w * np.abs(d)).sum(1), (w * d * d).sum(1)
    L = np.log1p(t)
    bL = U * (((A + 2) * t + 2.25 * wd) / (1 + t) + 4 * L)
    bH = (bL + U * ((A + 6) * wd + 2.25 * wdd + wd * ((A + 2) * t + 2.25 * wd) / (1 + t)) / (1 + t)
          + 2 * U * (L + wd / (1 + t)))
    return bL, bH


def check_scores(z, lab, top_k, dtype, pad=0, labels=True):
    zt = on_gpu(z, dtype, pad)
    got = sscn.label_scores(zt, dev(lab) if labels else None, top_k)
    lp, H, st, top, tlp = O.label_scores(z, lab if labels else None, top_k)
    bL, bH = bounds(np.where(np.isfinite(z), z, -np.inf))
    near(host(got.stats)[:, 0], st[:, 0], 0.0, "maximum") if not np.isnan(z).any() else None
    near(host(got.stats)[:, 1], st[:, 1], bL, "log sum")
    near(host(got.entropy), H, bH, "entropy")
    if labels:
        x = np.abs(np.nan_to_num(z[np.arange(len(lab)), np.clip(lab, 0, z.shape[1] - 1)].astype(np.float64) - st[:, 0], posinf=0, neginf=0))
        near(host(got.logprob), lp, bL + 2 * U * (x + np.abs(np.nan_to_num(lp, posinf=0, neginf=0))), "log probability")
    else:
        assert got.logprob is None
    if top_k:
        np.testing.assert_array_equal(host(got.top_index), top)
        x = np.nan_to_num(np.abs(np.take_along_axis(z.astype(np.float64), top, 1) - st[:, :1]), posinf=0)
        near(host(got.top_logprob), tlp, bL[:, None] + 2 * U * (x + np.nan_to_num(np.abs(tlp), posinf=0)), "top")
    else:
        assert got.top_index is None and got.top_logprob is None
    return zt, got


def check_grad(z, lab, top_k, dtype, zt, got, seed, parts="ght", pad=0):
    rng = np.random.default_rng(seed)
    n, k = z.shape
    g = rng.standard_normal(n).astype(np.float32) if "g" in parts else None
    h = rng.standard_normal(n).astype(np.float32) if "h" in parts else None
    t = rng.standard_normal((n, top_k)).astype(np.float32) if "t" in parts and top_k else None
    top = host(got.top_index) if t is not None else None
    want = O.label_scores_backward(z, lab, g, h, top, t)
    dv = lambda a: dev(a) if a is not None else None
    out = on_gpu(np.zeros((n, k), np.float32), dtype, pad)
    d = sscn.label_scores_backward(zt, got, dev(lab), dlogprob=dv(g), dentropy=dv(h), dtop=dv(t), out=out)
    bL, bH = bounds(z)
    _, H, st, _, _ = O.label_scores(z, None)
    lp = np.where(np.isneginf(z), -1e4, z.astype(np.float64) - np.where(np.isneginf(st[:, :1]), 0, st[:, :1])) - st[:, 1:]
    p = np.exp(lp)
    A = np.zeros((n, k))
    if g is not None:
        A[np.arange(n), np.clip(lab, 0, k - 1)] += np.where(lab >= 0, np.abs(g), 0)
    if t is not None:
        np.add.at(A, (np.arange(n)[:, None], top), np.abs(t))
    G = A.sum(1, keepdims=True)
    hh = np.abs(h)[:, None] if h is not None else 0.0
    dl = bL[:, None] + 2 * U * np.abs(np.maximum(lp, -1e3))     # log p's error
    s = np.abs(np.maximum(lp, -1e3)) + np.abs(H)[:, None]
    b = A * (p * dl + 4 * U * -np.expm1(lp)) + p * ((G + hh * s) * (dl + (8 + top_k) * U) + hh * (dl + bH[:, None]))
    b = b + (torch.finfo(TD[dtype]).eps / 2 if dtype == "bf16" else 2 * U) * (np.abs(want) + b) + 1e-37
    near(host(d), want, b, "gradient")
    if pad:
        assert torch.isnan(d._base[:, k:]).all()                # what lies between the rows is left


SIZES = [(1, 1, 1), (1, 2, 2), (5, 3, 0), (255, 20, 3), (257, 64, 16), (100, 65, 5), (33, 200, 8), (300, 129, 1),
         (7, 1000, 16), (5, 2049, 16), (9, 4096, 8), (3, 5001, 4), (2, 40001, 8), (1, 131071, 16), (1, 131072, 0), (1030, 257, 2), (70, 8193, 3),
         (300, 8200, 8), (2, 140001, 16), (1, 300001, 9), ((1 << 18) + 3, 66, 16)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,top_k", SIZES)
def test_scores_and_gradient(n, k, top_k, dtype):
    z, lab = draw(n, k, dtype, n * k)
    zt, got = check_scores(z, lab, top_k, dtype)
    check_grad(z, lab, top_k, dtype, zt, got, n + k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["masked", "lowest", "ties", "sure"])
@pytest.mark.parametrize("n,k,top_k", [(300, 20, 16), (70, 50, 5), (40, 300, 16), (21, 1500, 16), (12, 3001, 16), (9, 9001, 16),
                                       (260, 8193, 5), (3, 70003, 7), (1, 200000, 16)])
def test_masks_ties_and_sure_rows(n, k, top_k, kind, dtype):
    z, lab = draw(n, k, dtype, n + k + len(kind), kind)
    zt, got = check_scores(z, lab, top_k, dtype)
    if kind != "lowest":         # differences of the lowest value are as large as the type allows
        check_grad(z, lab, top_k, dtype, zt, got, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 3, 12, 16])
@pytest.mark.parametrize("n,k,top_k", [(1, 20, 3), (300, 20, 3), (200, 48, 1), (37, 77, 4), (11, 700, 2), (4, 10007, 3)])
def test_strided_rows(n, k, top_k, pad, dtype):
    z, lab = draw(n, k, dtype, n + k + pad)
    zt, got = check_scores(z, lab, top_k, dtype, pad)
    check_grad(z, lab, top_k, dtype, zt, got, n, pad=pad)


@pytest.mark.parametrize("k", [5, 300, 20000])
@pytest.mark.parametrize("parts", ["g", "h", "t", "gh", ""])
def test_gradient_of_each_number(k, parts):
    z, lab = draw(40, k, "f32", k)
    zt, got = check_scores(z, lab, 3, "f32")
    check_grad(z, lab, 3, "f32", zt, got, 1, parts=parts)


@pytest.mark.parametrize("k", [4, 100, 9000])
def test_rows_with_nan_and_infinity(k):
    """They are NaN themselves (the best classes still listed, NaN first) and
    leave the rows beside them alone."""
    z, lab = draw(9, k, "f32", 11)
    lab = np.maximum(lab, 0).astype(np.int32)
    z[1, k // 2] = np.nan
    z[3, [0, k - 1]] = np.inf
    z[5, :] = np.nan
    z[7, 0], z[7, 1], z[7, 2] = np.nan, np.inf, -np.inf
    clean = z.copy()
    clean[1::2] = 0
    top_k = min(k, 5)
    zt, got = check_scores(z, lab, top_k, "f32")
    alone = sscn.label_scores(dev(clean), dev(lab), top_k)
    for a, b in zip(got, alone):
        assert torch.equal(a[0::2], b[0::2])
    d = sscn.label_scores_backward(zt, got, dev(lab), dlogprob=torch.ones(9, device="cuda:0"))
    assert torch.isnan(d[1::2]).all() and torch.isfinite(d[0::2]).all()


def test_labels_outside_and_absent():
    z, lab = draw(50, 12, "f32", 2)
    lab[::4] = -100
    lab[1::4] = 12
    zt, got = check_scores(z, lab, 2, "f32")
    assert torch.isnan(got.logprob[1::4]).all() and (got.logprob[::4] == 0).all()
    d = sscn.label_scores_backward(zt, got, dev(lab), dlogprob=torch.ones(50, device="cuda:0"))
    assert torch.isnan(d[1::4]).all() and (d[::4] == 0).all() and torch.isfinite(d[2::4]).all()
    check_scores(z, lab, 2, "f32", labels=False)


def test_a_class_listed_twice_receives_both():
    z, lab = draw(20, 30, "f32", 3)
    zt = dev(z)
    got = sscn.label_scores(zt, dev(lab), 2)
    twice = got._replace(top_index=got.top_index[:, :1].repeat(1, 2).contiguous())
    t = torch.randn(20, 2, device="cuda:0")
    a = sscn.label_scores_backward(zt, twice, dtop=t)
    b = O.label_scores_backward(z, None, top=host(twice.top_index), dtop=host(t))
    assert np.abs(host(a) - b).max() < 1e-5


def test_no_rows():
    z = torch.empty((0, 7), device="cuda:0")
    got = sscn.label_scores(z, torch.empty(0, dtype=torch.int32, device="cuda:0"), 2)
    assert got.stats.shape == (0, 2) and got.top_index.shape == (0, 2)
    assert sscn.label_scores_backward(z, got, dentropy=got.entropy).shape == (0, 7)


@pytest.mark.parametrize("k", [20, 1000, 9000])
def test_rows_further_apart_than_32_bits_count(k):
    """Three rows, the last of them beyond 2^32 bytes and 2^31 elements."""
    z, lab = draw(3, k, "bf16", 5)
    stride = (1 << 30) + 24
    flat = torch.empty(2 * stride + k, dtype=torch.bfloat16, device="cuda:0")
    rows = flat.as_strided((3, k), (stride, 1))
    rows.copy_(dev(z, torch.bfloat16))
    near_, far = sscn.label_scores(dev(z, torch.bfloat16), dev(lab), 3), sscn.label_scores(rows, dev(lab), 3)
    for a, b in zip(near_, far):
        assert torch.equal(a, b)
    one = torch.ones(3, device="cuda:0")
    want = sscn.label_scores_backward(dev(z, torch.bfloat16), near_, dev(lab), dlogprob=one)
    out = torch.empty(2 * stride + k, dtype=torch.bfloat16, device="cuda:0").as_strided((3, k), (stride, 1))
    got = sscn.label_scores_backward(rows, far, dev(lab), dlogprob=one, out=out)
    assert torch.equal(got, want)


@pytest.mark.parametrize("n,k", [(3000, 20), (50, 500), (2, 100000)])
def test_the_same_bits_every_time(n, k):
    z, lab = draw(n, k, "f32", 7)
    zt, lt = dev(z), dev(lab)
    first = sscn.label_scores(zt, lt, 4)
    for _ in range(3):
        for a, b in zip(first, sscn.label_scores(zt, lt, 4)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n,k", [(500, 20), (3, 30000)])
def test_graphs_and_streams(n, k):
    """Two captured graphs replayed in turn, with the program's own calls and
    new inputs between the replays, and a call on another stream."""
    z, lab = draw(n, k, "f32", 9)
    zt, lt = dev(z), dev(lab)
    one = torch.ones(n, device="cuda:0")

    def calls():
        s = sscn.label_scores(zt, lt, 3)
        return (*s, sscn.label_scores_backward(zt, s, lt, dlogprob=one, dentropy=one))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = calls()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = calls()
        graphs.append((g, out))
    for a, b in zip(on_side, calls()):
        assert torch.equal(a, b)
    for turn in range(3):
        zt.copy_(dev(draw(n, k, "f32", 20 + turn)[0]))
        for g, out in graphs:
            g.replay()
        want = calls()
        torch.cuda.synchronize()
        for g, out in graphs:
            for a, b in zip(out, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("n,k", [(20000, 20), (40, 30000)])
def test_two_streams_at_once(n, k):
    """Calls in flight together, each with its own inputs and workspace."""
    data = [(dev(z), dev(lab)) for z, lab in (draw(n, k, "f32", s) for s in (1, 2))]
    one = torch.ones(n, device="cuda:0")

    def calls(z, lab):
        s = sscn.label_scores(z, lab, 3)
        return (*s, sscn.label_scores_backward(z, s, lab, dlogprob=one))
    want = [calls(*d) for d in data]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(5):
        for st, d in zip(streams, data):
            with torch.cuda.stream(st):
                got.append(calls(*d))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        for a, b in zip(out, want[i % 2]):
            assert torch.equal(a, b)
