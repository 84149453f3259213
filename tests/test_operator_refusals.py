"""What the label scores and the 8-bit checkpoints refuse, before any device
work: the binding's checks, and the C entries' (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1711_10275_amd import sscn

INVALID = sscn.STATUS_CODES["invalid_arg"]
P, Q = ctypes.c_void_p(4096), ctypes.c_void_p(8192)      # never read: every call below is refused or has no rows


def _scores(z=P, ldz=8, n=4, k=8, dtype=0, labels=P, top_k=2, logprob=P, entropy=P, stats=P, index=P, top=P, work=P,
            work_bytes=1 << 40):
    return sscn.lib().sscn_label_scores(z, ldz, n, k, dtype, labels, top_k, logprob, entropy, stats, index, top, work,
                                        work_bytes, None)


def _scores_back(z=P, ldz=8, n=4, k=8, dtype=0, labels=P, stats=P, entropy=P, top_k=2, index=P, g=P, h=P, t=P, d=Q,
                 ldd=8):
    return sscn.lib().sscn_label_scores_backward(z, ldz, n, k, dtype, labels, stats, entropy, top_k, index, g, h, t, d,
                                                 ldd, None)


@pytest.mark.parametrize("bad", [dict(z=None), dict(ldz=7), dict(n=-1), dict(k=0, ldz=0), dict(dtype=2), dict(top_k=-1),
                                 dict(top_k=9), dict(k=40, ldz=40, top_k=17), dict(labels=None), dict(logprob=None),
                                 dict(entropy=None), dict(stats=None), dict(index=None), dict(top=None),
                                 dict(z=ctypes.c_void_p(4098))])
def test_label_scores_refuses(bad):
    assert _scores(**bad) == INVALID and sscn.lib().sscn_last_error()


@pytest.mark.parametrize("bad", [dict(z=None), dict(ldz=7), dict(ldd=7), dict(n=-1), dict(dtype=-1), dict(top_k=9),
                                 dict(labels=None), dict(stats=None), dict(entropy=None), dict(index=None),
                                 dict(top_k=0), dict(d=None), dict(d=ctypes.c_void_p(4097)), dict(d=P)])
def test_label_scores_backward_refuses(bad):
    assert _scores_back(**bad) == INVALID and sscn.lib().sscn_last_error()


def test_workspaces():
    L, b = sscn.lib(), ctypes.c_int64(-1)
    assert L.sscn_label_scores_workspace(10, 20, 3, ctypes.byref(b)) == 0 and b.value >= 0
    assert L.sscn_label_scores_workspace(-1, 20, 3, ctypes.byref(b)) == INVALID
    assert L.sscn_label_scores_workspace(10, 20, 17, ctypes.byref(b)) == INVALID
    assert L.sscn_label_scores_workspace(10, 20, 3, None) == INVALID
    q = L.sscn_batchnorm_relu_backward_params_q8_workspace
    assert q(1000, 40, ctypes.byref(b)) == 0 and b.value > 0
    assert q(1000, 0, ctypes.byref(b)) == INVALID and q(1000, 40, None) == INVALID
    need = ctypes.c_int64()
    assert L.sscn_label_scores_workspace(1, 1 << 20, 8, ctypes.byref(need)) == 0
    if need.value:
        assert _scores(n=1, k=1 << 20, ldz=1 << 20, top_k=8, work_bytes=need.value - 1) == INVALID
        assert _scores(n=1, k=1 << 20, ldz=1 << 20, top_k=8, work=None) == INVALID


def _apply(x=P, ldx=40, n=4, c=40, dtype=0, mean=P, gamma=P, y=Q, ldy=40, codes=P, exps=P):
    return sscn.lib().sscn_batchnorm_relu_apply_q8(x, ldx, n, c, dtype, mean, P, P, gamma, P, y, ldy, codes, exps, None)


def _params(d=P, ldd=40, n=4, c=40, dtype=0, codes=P, exps=P, gamma=P, dg=P, a=Q, lda=40, work=P, work_bytes=1 << 40):
    return sscn.lib().sscn_batchnorm_relu_backward_params_q8(d, ldd, codes, exps, n, c, dtype, gamma, P, dg, P, a, lda,
                                                             work, work_bytes, None)


def _input(d=P, ldd=40, n=4, c=40, col0=0, cols=40, dtype=0, codes=P, gamma=P, dg=P, add=P, lda=40, dx=Q, ldo=40):
    return sscn.lib().sscn_batchnorm_relu_backward_input_q8(d, ldd, codes, P, n, c, col0, cols, dtype, gamma, P, P, dg,
                                                            P, add, lda, dx, ldo, None)


@pytest.mark.parametrize("call,bad", [
    (_apply, dict(x=None)), (_apply, dict(ldx=39)), (_apply, dict(ldy=39)), (_apply, dict(n=-1)), (_apply, dict(c=0)),
    (_apply, dict(dtype=2)), (_apply, dict(mean=None)), (_apply, dict(gamma=None)), (_apply, dict(codes=None)),
    (_apply, dict(exps=None)), (_apply, dict(x=ctypes.c_void_p(4098))), (_apply, dict(y=P, ldy=41)),
    (_params, dict(a=P)), (_input, dict(dx=P)), (_input, dict(add=Q, lda=41)),
    (_params, dict(d=None)), (_params, dict(ldd=39)), (_params, dict(codes=None)), (_params, dict(gamma=None)),
    (_params, dict(dg=None)), (_params, dict(lda=39)), (_params, dict(work=None)), (_params, dict(work_bytes=8)),
    (_params, dict(work=ctypes.c_void_p(4100))), (_params, dict(dtype=7)),
    (_input, dict(d=None)), (_input, dict(dx=None)), (_input, dict(col0=-1)), (_input, dict(cols=0)),
    (_input, dict(col0=1)), (_input, dict(col0=2 ** 31 - 1, cols=2)), (_input, dict(lda=39)), (_input, dict(ldo=39)),
    (_input, dict(codes=None)), (_input, dict(gamma=None)), (_input, dict(dg=None)), (_input, dict(dtype=2))])
def test_checkpoints_refuse(call, bad):
    assert call(**bad) == INVALID and sscn.lib().sscn_last_error()


def test_no_rows_is_no_work():
    assert _scores(n=0, z=None, labels=None, entropy=None, stats=None, index=None, top=None) == 0
    assert _scores_back(n=0, z=None, d=None) == 0
    assert _apply(n=0, x=None, y=None, codes=None, exps=None) == 0
    assert _input(n=0, d=None, dx=None, codes=None) == 0
    assert sscn.lib().sscn_q8_values(None, None, 0, 40, 0, None, 40, None) == 0


def test_binding_refuses_cpu_tensors():
    z = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="GPU"):
        sscn.label_scores(z, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        sscn.label_scores_backward(z, sscn.LabelScores(None, z[:, 0], z[:, :2], None, None))
    q8 = sscn.Q8(torch.zeros((4, 8), dtype=torch.int8), torch.zeros((4, 1), dtype=torch.uint8))
    v = torch.ones(8)
    with pytest.raises(ValueError, match="GPU"):
        sscn.q8_values(q8)
    with pytest.raises(ValueError, match="GPU"):
        sscn.batchnorm_relu_backward_params_q8(z, q8, v, v)
    with pytest.raises(ValueError, match="GPU"):
        sscn.batchnorm_relu_backward_input_q8(z, q8, v, v, v, v, v, z)


@pytest.mark.gpu
def test_binding_refuses_on_the_gpu():
    z = torch.zeros((4, 8), device="cuda:0")
    lab = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    s = sscn.label_scores(z, lab, 2)
    refused = [
        lambda: sscn.label_scores(z.half(), lab), lambda: sscn.label_scores(z.t(), lab),
        lambda: sscn.label_scores(z[:1].expand(4, 8), lab), lambda: sscn.label_scores(z, lab.long()),
        lambda: sscn.label_scores(z, lab[:3]), lambda: sscn.label_scores(z, lab.cpu()),
        lambda: sscn.label_scores(z, lab.unsqueeze(1)),
        lambda: sscn.label_scores_backward(z, s, None, dlogprob=s.entropy),
        lambda: sscn.label_scores_backward(z, s._replace(top_index=None), lab, dtop=s.top_logprob),
        lambda: sscn.label_scores_backward(z, s, lab, dtop=s.top_logprob[:, :1]),
        lambda: sscn.label_scores_backward(z, s, lab, dentropy=s.entropy.double()),
        lambda: sscn.label_scores_backward(z, s, lab, dentropy=s.entropy, out=z[:3]),
    ]
    for call in refused:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sscn.SSCNError, match="top_k"):
        sscn.label_scores(z, lab, 9)
    v = torch.ones(8, device="cuda:0")
    st = sscn.batchnorm_forward(z, v, v)
    a, q8 = sscn.batchnorm_relu_apply_q8(z, st, v, v)
    refused = [
        lambda: sscn.batchnorm_relu_apply_q8(z, st, v[:4], v), lambda: sscn.batchnorm_relu_apply_q8(z, st, v.cpu(), v),
        lambda: sscn.batchnorm_relu_apply_q8(z, st, v, v, out=a[:2]), lambda: sscn.q8_values(q8, torch.float16),
        lambda: sscn.q8_values(q8._replace(exponents=q8.exponents[:2])),
        lambda: sscn.q8_values(q8._replace(codes=q8.codes.t())),
        lambda: sscn.batchnorm_relu_backward_params_q8(a[:3], q8, v, v),
        lambda: sscn.batchnorm_relu_backward_input_q8(a, q8, v, v, v, v, v, a[:, :4]),
        lambda: sscn.batchnorm_relu_backward_input_q8(a, q8, v, v, v, v, v, a[:, :4].clone(), add=a, cols=(0, 4)),
    ]
    for call in refused:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sscn.SSCNError, match="column range"):
        sscn.batchnorm_relu_backward_input_q8(a, q8, v, v, v, v, v, torch.empty(4, 4, device="cuda:0"), cols=(6, 10))
