"""Outputs that share memory with an input they may not replace: refused where
the rows have one stride, column ranges of one buffer beside each other taken."""
import ctypes

import pytest
import torch

from paper_1711_10275_amd import sscn

from tests.test_operator_refusals import INVALID, _apply, _input, _params, _scores_back


def at(i):
    """Address of fp32 element i; never read, every call below is refused."""
    return ctypes.c_void_p(4096 + 4 * i)


@pytest.mark.parametrize("call,bad", [
    # the gradient in columns of dA, one row on, and a row's end in the next row's columns
    (_input, dict(d=at(0), ldd=80, c=80, col0=40, add=None, dx=at(40), ldo=80)),
    (_input, dict(d=at(0), ldd=40, dx=at(40), ldo=40, add=None)),
    (_input, dict(d=at(0), ldd=80, dx=at(79), ldo=80, add=None)),
    (_input, dict(d=at(200), ldd=80, dx=at(1), ldo=80, add=None)),
    (_input, dict(d=at(9999), add=at(0), lda=40, dx=at(1), ldo=40)),
    (_input, dict(n=1, d=at(0), ldd=40, dx=at(39), ldo=99, add=None)),
    (_apply, dict(x=at(0), ldx=64, y=at(8), ldy=64)),
    (_apply, dict(x=at(64), ldx=64, y=at(0), ldy=64)),
    (_params, dict(d=at(0), ldd=64, a=at(39), lda=64)),
    (_scores_back, dict(z=at(0), ldz=16, d=at(7), ldd=16)),
    (_scores_back, dict(z=at(32), ldz=16, d=at(0), ldd=16))])
def test_outputs_on_inputs_are_refused(call, bad):
    assert call(**bad) == INVALID and sscn.lib().sscn_last_error()


@pytest.mark.gpu
def test_column_ranges_of_one_buffer_are_taken():
    """Inputs and outputs side by side in the columns of one buffer."""
    n, c = 300, 24
    wide = torch.randn(n, 4 * c, device="cuda:0")
    part = [wide[:, i * c:(i + 1) * c] for i in range(4)]
    g, b = torch.rand(c, device="cuda:0") + 0.5, torch.randn(c, device="cuda:0")
    x = part[1].clone()
    st = sscn.batchnorm_forward(x, g, b)
    a, q8 = sscn.batchnorm_relu_apply_q8(x, st, g, b)
    for out in (part[0], part[2]):
        assert torch.equal(sscn.batchnorm_relu_apply_q8(part[1], st, g, b, out=out)[0], a)
    assert torch.equal(part[1], x)
    dA, add = x, torch.randn(n, c, device="cuda:0")
    dg, db, _ = sscn.batchnorm_relu_backward_params_q8(part[1], q8, g, b)
    args = (q8, g, b, st.invstd, dg, db)
    want = sscn.batchnorm_relu_backward_input_q8(dA, *args, torch.empty_like(x), add=add)
    part[3].copy_(add)
    assert torch.equal(sscn.batchnorm_relu_backward_input_q8(part[1], *args, part[0], add=part[3]), want)
    assert torch.equal(sscn.batchnorm_relu_backward_input_q8(part[1], *args, part[3], add=part[3]), want)
    lab = torch.randint(0, c, (n,), dtype=torch.int32, device="cuda:0")
    s, one = sscn.label_scores(part[1], lab), torch.ones(n, device="cuda:0")
    want = sscn.label_scores_backward(x, s, lab, dlogprob=one)
    for out in (part[0], part[2]):
        assert torch.equal(sscn.label_scores_backward(part[1], s, lab, dlogprob=one, out=out), want)
    assert torch.equal(part[1], x)
    for bad in (wide[:, c + 4:2 * c + 4], wide[:, c - 1:2 * c - 1]):
        for call in (lambda: sscn.batchnorm_relu_backward_input_q8(part[1], *args, bad),
                     lambda: sscn.batchnorm_relu_apply_q8(part[1], st, g, b, out=bad),
                     lambda: sscn.label_scores_backward(part[1], s, lab, dlogprob=one, out=bad)):
            with pytest.raises(sscn.SSCNError):
                call()
