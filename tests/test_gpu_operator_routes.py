"""Ways through the kernels that need a shape of their own: a last piece that
slides back in a range that starts inside the row, in bf16 rows at an odd
stride, outputs whose rows lie apart through the C entries, and more rows than
a launch has workgroups for."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import sscn_oracle as O
from paper_1711_10275_amd import sscn
from tests.gpu_common import dev, host
from tests.test_gpu_checkpoint import TD, check_back, check_keep, draw

pytestmark = pytest.mark.gpu


# a piece is 4 values of fp32, 8 of bf16; it slides where its block of 32 holds
# a whole one, the range starts on a piece and its width is no multiple of it
@pytest.mark.parametrize("c,ranges,dtype", [
    (70, [(0, 32), (32, 70)], "f32"), (70, [(0, 28), (28, 39), (39, 70)], "f32"), (103, [(4, 103), (64, 103)], "f32"),
    (93, [(0, 32), (32, 93)], "bf16"), (47, [(8, 47), (32, 47)], "bf16"), (125, [(64, 125), (96, 125)], "bf16")])
@pytest.mark.parametrize("pad", [0, 3])
def test_a_range_whose_last_piece_slides(c, ranges, dtype, pad):
    x, gamma, beta = draw(300, c, dtype, c)
    check_back(x, gamma, beta, dtype, *check_keep(x, gamma, beta, dtype, pad), pad=pad, split=ranges)


@pytest.mark.parametrize("pad", [1, 5, 16])
@pytest.mark.parametrize("n,c", [(1, 31), (333, 31), (200, 45), (77, 93), (64, 541)])
def test_bf16_rows_that_slide(n, c, pad):
    x, gamma, beta = draw(n, c, "bf16", n + c + pad)
    check_back(x, gamma, beta, "bf16", *check_keep(x, gamma, beta, "bf16", pad), pad=pad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,ld", [(300, 32, 33), (120, 70, 77), (50, 31, 40), (40, 5, 8)])
def test_rows_apart_in_the_restored_outputs(n, c, ld, dtype):
    """Values and restored activations at a row stride above c: as contiguous,
    and what lies between the rows is left."""
    x, gamma, beta = draw(n, c, dtype, n + c)
    q8, codes, exps, _ = check_keep(x, gamma, beta, dtype)
    L, code, stream = sscn.lib(), {"f32": 0, "bf16": 1}[dtype], torch.cuda.current_stream().cuda_stream
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    wide = torch.full((n, ld), 7.0, dtype=TD[dtype], device="cuda:0")
    assert L.sscn_q8_values(ptr(q8.codes), ptr(q8.exponents), n, c, code, ptr(wide), ld, stream) == 0
    np.testing.assert_array_equal(host(wide[:, :c]), O.q8_values(codes, exps))
    assert (wide[:, c:] == 7).all()
    dA = torch.randn(n, c, device="cuda:0").to(TD[dtype])
    tg, tb = dev(gamma), dev(beta)
    dg, db, a = sscn.batchnorm_relu_backward_params_q8(dA, q8, tg, tb, restore=True)
    need = ctypes.c_int64()
    assert L.sscn_batchnorm_relu_backward_params_q8_workspace(n, c, ctypes.byref(need)) == 0
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda:0")
    g2, b2 = torch.empty_like(dg), torch.empty_like(db)
    wide.fill_(7.0)
    assert L.sscn_batchnorm_relu_backward_params_q8(ptr(dA), c, ptr(q8.codes), ptr(q8.exponents), n, c, code, ptr(tg),
                                                    ptr(tb), ptr(g2), ptr(b2), ptr(wide), ld, ptr(work), need.value,
                                                    stream) == 0
    assert torch.equal(wide[:, :c], a) and torch.equal(g2, dg) and torch.equal(b2, db)
    assert (wide[:, c:] == 7).all()


# 4 rows to a workgroup, one row, a chunk of one row with and without a join,
# each launched for fewer rows than these
@pytest.mark.parametrize("n,k,dtype", [(131077, 129, "f32"), (131077, 129, "bf16"), (33001, 600, "f32"),
                                       (16391, 4100, "bf16"), (16391, 8200, "bf16")])
def test_more_rows_than_workgroups(n, k, dtype):
    """Every row is what it is among fewer rows, bit for bit; among them rows
    of equal logits, with a NaN and with none allowed."""
    g = torch.Generator(device="cuda:0").manual_seed(k)
    z = torch.randn(n, k, generator=g, device="cuda:0").to(TD[dtype])
    z[5::97] = 1.5
    z[6::89, k // 3] = float("nan")
    z[7::83] = -float("inf")
    z[8::79, ::2] = -float("inf")
    lab = torch.randint(-1, k, (n,), generator=g, device="cuda:0", dtype=torch.int32)
    w, t = torch.randn(n, generator=g, device="cuda:0"), torch.randn(n, 5, generator=g, device="cuda:0")

    def calls(at):
        s = sscn.label_scores(z[at], lab[at], 5)
        return (*s, sscn.label_scores_backward(z[at], s, lab[at], dlogprob=w[at], dentropy=w[at], dtop=t[at]))
    bits = lambda x: x.contiguous().view({1: torch.int8, 2: torch.int16, 4: torch.int32}[x.element_size()])
    whole = calls(slice(0, n))
    for lo in range(0, n, 4096):
        at = slice(lo, min(n, lo + 4096)) if n - lo > 300 else slice(n - 300, n)
        for a, b in zip(whole, calls(at)):
            assert torch.equal(bits(a[at]), bits(b)), lo
