"""Scores of per-site classifiers and 8-bit activation checkpoints, as cases to measure.

Two pairs of operators, each with its plain form (elementary torch
operations) and the library's calls:

  scores       per row of logits: log probability of the row's label, entropy, the best classes
  scores_grad  gradient of those numbers at the logits
  keep         batch normalisation + ReLU that also keeps its normalised input in 8 bits, and the values kept
  keep_grad    the backward pass of that from the 8-bit codes: parameter gradients, the activations
               restored (for the weight gradient that follows), the input gradient

Fields of a case:

  kind            one of the four
  n               rows (active sites)
  dtype           "f32" or "bf16"
  classes, top_k  scores: logits per row, best classes asked for
  pad             elements between rows beyond the row itself
  masked          rows have part of their classes at minus infinity, some rows all of them
  dtop            scores_grad: the best classes' log probabilities have a gradient too
  c               keep: channels
  split           keep_grad: the input is a concatenation whose halves' gradients go to two tensors,
                  the first with a gradient of another consumer added

The 8-bit format: xhat = (x - mean) * invstd in 32 bits; 32 consecutive channels of a row share a scale 2^e, e the least
integer from -126 up with max |xhat| <= 126 * 2^e, stored as the byte e + 127; a code is xhat / 2^e rounded to the nearest
whole number (ties to even), moved by one where the ReLU would otherwise pass the restored value but not the original, or
the original but not the restored one.
"""
import math
import types

import torch

own = False

DEV = "cuda:0"
BLOCK = 32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one small object's predictions while a user waits: latency
        dict(name="scores_1k8_20_f32", kind="scores", n=1799, classes=20, top_k=3, pad=0, masked=False, dtype="f32"),
        # a batch of scenes scored in evaluation, a fifth of the sites without a label
        dict(name="scores_2m_20_bf16", kind="scores", n=1964906, classes=20, top_k=3, pad=0, masked=False, dtype="bf16"),
        # part segmentation: 50 parts, of which a shape has a few; logits in the columns of a wider buffer
        dict(name="scores_100k_50_f32", kind="scores", n=99515, classes=50, top_k=5, pad=14, masked=True, dtype="f32"),
        # an open vocabulary, odd width: rows far longer than a workgroup holds
        dict(name="scores_4k_40001_bf16", kind="scores", n=4096, classes=40001, top_k=8, pad=0, masked=False, dtype="bf16"),
        # one site against a long list
        dict(name="scores_1_131071_f32", kind="scores", n=1, classes=131071, top_k=16, pad=0, masked=False, dtype="f32"),
        # the loss's gradient in training on a batch of scenes: weighted log probabilities and entropy
        dict(name="scores_grad_2m_20_bf16", kind="scores_grad", n=1964906, classes=20, top_k=0, pad=0, masked=False,
             dtop=False, dtype="bf16"),
        # distillation on the best classes of an open vocabulary
        dict(name="scores_grad_1k_40001_f32", kind="scores_grad", n=1024, classes=40001, top_k=4, pad=0, masked=True,
             dtop=True, dtype="f32"),
        # the smallest layer
        dict(name="keep_1k8_c16_f32", kind="keep", n=1799, c=16, pad=0, dtype="f32"),
        # the finest level of a batch of scenes
        dict(name="keep_2m_c32_bf16", kind="keep", n=1964906, c=32, pad=0, dtype="bf16"),
        # odd width in the columns of a wider buffer: no row starts on 16 bytes
        dict(name="keep_200k_c70_f32", kind="keep", n=200003, c=70, pad=3, dtype="f32"),
        # the backward pass at the finest level
        dict(name="keep_grad_2m_c32_bf16", kind="keep_grad", n=1964906, c=32, pad=0, split=False, dtype="bf16"),
        # a decoder's concatenation of skip and upsampled features
        dict(name="keep_grad_100k_c128_f32", kind="keep_grad", n=99515, c=128, pad=0, split=True, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))


def draw(rng):
    kind = rng.choice(["scores", "scores", "scores_grad", "keep", "keep_grad"])
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 3, 16])
    if kind in ("scores", "scores_grad"):
        if rng.random() < 0.6:  # a segmentation network's
            classes = _log(rng, 2, 200)
            n = _log(rng, 1, min(1_960_000, 45_000_000 / classes))
        else:
            classes = _log(rng, 200, 131072)
            n = _log(rng, 1, (160_000_000 if dtype == "bf16" and kind == "scores" else 40_000_000) / classes)
        c = dict(kind=kind, n=n, classes=classes, top_k=min(rng.choice([0, 1, 3, 5, 8, 16]), classes), pad=pad,
                 masked=rng.random() < 0.3, dtype=dtype)
        if kind == "scores_grad":
            c["dtop"] = c["top_k"] > 0 and rng.random() < 0.7
        return c
    w = rng.choice([16, 32, 64, 96, 128, 160, 256]) if rng.random() < 0.6 else _log(rng, 1, 512)
    c = dict(kind=kind, n=_log(rng, 1, min(1_960_000, (60_000_000 if dtype == "bf16" else 12_000_000) / w)), c=w, pad=pad, dtype=dtype)
    if kind == "keep_grad":
        c["split"] = w % 2 == 0 and rng.random() < 0.4
    return c


# ----------------------------------------------------------------- prepare
def _matrix(g, n, width, pad, dtype, scale=1.0):
    """n x width normal values, rows width + pad apart."""
    return (torch.randn((n, width + pad), generator=g, device=DEV) * scale).to(TYPES[dtype])[:, :width]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 29)
    n, dtype = case["n"], case["dtype"]
    uniform = lambda *shape: torch.rand(shape, generator=g, device=DEV)  # noqa: E731
    if case["kind"] in ("scores", "scores_grad"):
        k = case["classes"]
        z = _matrix(g, n, k, case["pad"], dtype, 2.0)
        truth = torch.randint(0, k, (n, 1), generator=g, device=DEV)
        # a trained network: most sites clear, some not
        z.scatter_add_(1, truth, (uniform(n, 1) * 3 * math.log(k + 1)).to(z.dtype))
        if case["masked"]:  # a run of classes around the label is allowed; one row in 64 allows none
            at = torch.arange(k, device=DEV, dtype=torch.int32)
            reach = (uniform(n, 1) * k / 4).to(torch.int32)
            off = (at - truth.to(torch.int32)).abs() > reach
            off |= uniform(n, 1) < 1 / 64
            z.masked_fill_(off, -math.inf)
            del off
        other = torch.randint(0, k, (n,), generator=g, device=DEV)
        labels = torch.where(uniform(n) < 0.8, truth[:, 0], other)
        labels = torch.where(uniform(n) < 0.2, -1, labels).to(torch.int32)
        st = dict(case=case, logits=z, labels=labels)
        if case["kind"] == "scores_grad":
            weight = -(uniform(n) + 0.5) / n  # of each site's class
            st.update(scores=_scores(z, labels, case["top_k"]), dlogprob=weight,
                      dentropy=torch.randn(n, generator=g, device=DEV) * (0.1 / n),
                      dtop=torch.randn((n, case["top_k"]), generator=g, device=DEV) / n if case["dtop"] else None)
        return st
    c = case["c"]
    x = _matrix(g, n, c, case["pad"], dtype, 1.5)
    x += torch.randn(c, generator=g, device=DEV).to(x.dtype)
    gamma, beta = uniform(c) + 0.5, torch.randn(c, generator=g, device=DEV) * 0.3
    var, mean = torch.var_mean(x.double(), 0, correction=0)
    invstd = torch.rsqrt(var + 1e-5).float()
    st = dict(case=case, gamma=gamma, beta=beta, st=types.SimpleNamespace(mean=mean.float(), invstd=invstd, scale=gamma * invstd))
    if case["kind"] == "keep":
        return dict(st, x=x)
    codes, exponents = _encode(x, st["st"], gamma, beta)
    return dict(st, codes=codes, exponents=exponents, dA=_matrix(g, n, c, case["pad"], dtype),
                add=_matrix(g, n, c // 2, 0, dtype) if case["split"] else None)


# ------------------------------------------------------------- plain forms
def _scores(z, labels, top_k):
    x = z.float()
    m = x.amax(1, keepdim=True)
    empty = m == -math.inf
    d = x - torch.where(empty, 0.0, m)
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    # 1 for the largest, and the others: log1p keeps a sure row's small numbers
    log_sum = torch.where(empty, 0.0, torch.where(s < 1.5, torch.log1p(_without_largest(e)), torch.log(s)))
    entropy = torch.where(empty, 0.0, log_sum - (e * torch.where(e > 0, d, 0.0)).sum(1, keepdim=True) / torch.where(empty, 1.0, s))[:, 0]
    picked = (torch.gather(d, 1, labels.clamp(min=0).long()[:, None]) - log_sum)[:, 0]
    out = dict(logprob=torch.where(labels < 0, 0.0, picked), entropy=entropy, stats=torch.cat([m, log_sum], 1),
               top_index=None, top_logprob=None)
    del e
    if top_k:
        # ties go to the lowest index: (value, -index) as one whole number
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
        order = (order << 31) - torch.arange(x.shape[1], device=x.device)
        at = torch.topk(order, top_k, 1).indices
        out.update(top_index=at.to(torch.int32), top_logprob=torch.gather(d, 1, at) - log_sum)
    return out


def _without_largest(e):
    """Row sums of e less one largest element (a 1), added without it."""
    at = e.argmax(1, keepdim=True)
    return e.scatter(1, at, 0.0).sum(1, keepdim=True)


def _scores_grad(z, labels, scores, dlogprob, dentropy, dtop):
    m, log_sum = scores["stats"][:, :1], scores["stats"][:, 1:]
    empty = m == -math.inf
    logp = z.float() - torch.where(empty, 0.0, m) - log_sum
    p = torch.exp(logp)
    has = labels >= 0
    direct = torch.zeros_like(p)
    direct.scatter_(1, labels.clamp(min=0).long()[:, None], torch.where(has, dlogprob, 0.0)[:, None])
    if dtop is not None:
        direct.scatter_add_(1, scores["top_index"].long(), dtop)
    total = torch.where(has, dlogprob, 0.0) + (dtop.sum(1) if dtop is not None else 0.0)
    inner = (total[:, None] - direct) + dentropy[:, None] * torch.where(p > 0, logp + scores["entropy"][:, None], 0.0)
    grad = -direct * torch.expm1(logp) - p * inner
    return torch.where(empty, 0.0, grad).to(z.dtype)


def _blocks(per_block, c):
    """A value per 32 channels, for each of the c channels."""
    return per_block.repeat_interleave(BLOCK, 1)[:, :c]


def _power(exponents):
    return (exponents.to(torch.int32) << 23).view(torch.float32)


def _passes(v, scale, shift):
    """v * scale + shift > 0, decided without rounding."""
    return v.double() * scale.double() + shift.double() > 0


def _encode(x, st, gamma, beta):
    n, c = x.shape
    d = x.float() - st.mean
    v = d * st.invstd
    most = torch.nn.functional.pad(v.abs(), (0, -c % BLOCK)).reshape(n, -1, BLOCK).amax(2)
    mant, ex = torch.frexp(most)  # most = mant 2^ex, 1/2 <= mant < 1; 126 = 0.984375 * 2^7
    e = torch.where(most > 0, ex - 7 + (mant > 0.984375).int(), -126).clamp(min=-126)
    exponents = (e + 127).to(torch.uint8)
    down = _blocks(_power(254 - exponents), c)  # 2^-e
    code = torch.round(v * down)
    restored = code / down
    want, have = _passes(d, st.scale, beta), _passes(restored, gamma, beta)
    code = code + (want.float() - have.float()) * torch.sign(gamma)
    return code.clamp(-127, 127).to(torch.int8), exponents


def _values(codes, exponents):
    return codes.float() * _blocks(_power(exponents), codes.shape[1])


def _keep(x, st, gamma, beta):
    a = torch.relu((x.float() - st.mean) * st.scale + beta).to(x.dtype)
    return dict(a=a, values=_values(*_encode(x, st, gamma, beta)).to(x.dtype))


def _keep_grad(codes, exponents, st, gamma, beta, dA, add):
    n, c = codes.shape
    v = _values(codes, exponents)
    dz = torch.where(_passes(v, gamma, beta), dA.float(), 0.0)
    dbeta, dgamma = dz.double().sum(0).float(), (dz.double() * v).sum(0).float()
    dx = gamma * st.invstd * (dz - dbeta / n - v * (dgamma / n))
    out = dict(dgamma=dgamma, dbeta=dbeta, a=torch.relu(v * gamma + beta).to(dA.dtype))
    if add is None:
        return dict(out, dx=dx.to(dA.dtype))
    h = c // 2
    return dict(out, dskip=(dx[:, :h] + add.float()).to(dA.dtype), dup=dx[:, h:].to(dA.dtype))


# --------------------------------------------------------------------- run
def run(st):
    case = st["case"]
    if own:
        return _run_own(st)
    if case["kind"] == "scores":
        return _scores(st["logits"], st["labels"], case["top_k"])
    if case["kind"] == "scores_grad":
        return _scores_grad(st["logits"], st["labels"], st["scores"], st["dlogprob"], st["dentropy"], st["dtop"])
    if case["kind"] == "keep":
        return _keep(st["x"], st["st"], st["gamma"], st["beta"])
    return _keep_grad(st["codes"], st["exponents"], st["st"], st["gamma"], st["beta"], st["dA"], st["add"])


def _run_own(st):
    from paper_1711_10275_amd import sscn
    case = st["case"]
    if case["kind"] == "scores":
        return sscn.label_scores(st["logits"], st["labels"], top_k=case["top_k"])._asdict()
    if case["kind"] == "scores_grad":
        return sscn.label_scores_backward(st["logits"], sscn.LabelScores(**st["scores"]), st["labels"], dlogprob=st["dlogprob"],
                                          dentropy=st["dentropy"], dtop=st["dtop"])
    gamma, beta = st["gamma"], st["beta"]
    if case["kind"] == "keep":
        a, q8 = sscn.batchnorm_relu_apply_q8(st["x"], st["st"], gamma, beta)
        return dict(a=a, values=sscn.q8_values(q8, a.dtype))
    q8 = sscn.Q8(st["codes"], st["exponents"])
    dA, add, invstd = st["dA"], st["add"], st["st"].invstd
    n, c = q8.codes.shape
    dgamma, dbeta, a = sscn.batchnorm_relu_backward_params_q8(dA, q8, gamma, beta, restore=True)
    out = dict(dgamma=dgamma, dbeta=dbeta, a=a)
    back = lambda lo, hi, add: sscn.batchnorm_relu_backward_input_q8(  # noqa: E731
        dA, q8, gamma, beta, invstd, dgamma, dbeta, torch.empty((n, hi - lo), dtype=dA.dtype, device=dA.device), add=add, cols=(lo, hi))
    if add is None:
        return dict(out, dx=back(0, c, None))
    return dict(out, dskip=back(0, c // 2, add), dup=back(c // 2, c, None))


def work(case):
    n, e = case["n"], {"f32": 4, "bf16": 2}[case["dtype"]]
    if case["kind"] == "scores":
        # logits and labels in; log probability, entropy, statistics and the best classes out
        return {"bytes": n * (case["classes"] * e + 4 + 16 + 8 * case["top_k"]), "flops": 6 * n * case["classes"]}
    if case["kind"] == "scores_grad":
        row = 4 + 8 + 4 + 4 + 4 + (8 * case["top_k"] if case["dtop"] else 0)
        return {"bytes": n * (2 * case["classes"] * e + row), "flops": 8 * n * case["classes"]}
    c, blocks = case["c"], -(-case["c"] // BLOCK)
    if case["kind"] == "keep":
        return {"bytes": n * (3 * c * e + c + blocks) + 20 * c, "flops": 12 * n * c}
    return {"bytes": n * (3 * c * e + c + blocks + (c // 2 * e if case["split"] else 0)) + 20 * c, "flops": 16 * n * c}


# ------------------------------------------------------------------- exact
def exact(case, seed):
    """run()'s outputs from the definitions, in 64 bits."""
    st = prepare(case, seed)
    if case["kind"] == "scores":
        z, labels, k = st["logits"].double(), st["labels"], case["top_k"]
        lse = torch.logsumexp(z, 1)
        none = torch.isneginf(lse)
        lse[none] = 0.0
        logp = z - lse[:, None]
        logprob = logp[torch.arange(case["n"], device=DEV), labels.clamp(min=0).long()]
        logprob[labels < 0] = 0.0
        m = z.max(1).values
        # the sum that the statistics hold, without the row's maximum: lse - m, and what log1p gives where that is small
        rest = torch.sort(z, stable=True, dim=1, descending=True)
        tail = torch.exp(rest.values[:, 1:] - torch.where(none, 0.0, m)[:, None]).sum(1)
        log_sum = torch.where(none, 0.0, torch.log1p(tail))
        top = rest.indices[:, :k].to(torch.int32) if k else None
        surprise = torch.exp(logp)
        surprise = -(surprise * logp).nan_to_num_(nan=0.0).sum(1)
        return dict(logprob=logprob, entropy=torch.where(none, 0.0, surprise), stats=torch.stack([m, log_sum], 1), top_index=top,
                    top_logprob=rest.values[:, :k] - lse[:, None] if k else None)
    if case["kind"] == "scores_grad":
        z, labels, s = st["logits"].double(), st["labels"].long(), st["scores"]
        none = torch.isneginf(z).all(1)
        logp = torch.log_softmax(torch.where(none[:, None], 0.0, z), 1)
        p = logp.exp()
        pl = torch.where(p > 0, p * logp, 0.0)
        # entropy: dH/dx = -p (log p + H)
        grad = st["dentropy"].double()[:, None] * (p * pl.sum(1, keepdim=True) - pl)
        g = torch.where(labels < 0, 0.0, st["dlogprob"].double())
        rows = torch.arange(case["n"], device=DEV)
        grad -= p * g[:, None]
        grad[rows, labels.clamp(min=0)] += g
        if st["dtop"] is not None:
            t = st["dtop"].double()
            grad -= p * t.sum(1, keepdim=True)
            grad.index_put_((rows[:, None].expand_as(t), s["top_index"].long()), t, accumulate=True)
        grad[none] = 0.0
        return grad
    gamma, beta, norm = st["gamma"].double(), st["beta"].double(), st["st"]
    n, c = case["n"], case["c"]
    if case["kind"] == "keep":
        d = st["x"].float() - norm.mean
        xhat = (d * norm.invstd).double()  # what is kept is the 32-bit value
        pre = d.double() * norm.scale.double() + beta
        values = torch.empty_like(xhat)
        for lo in range(0, c, BLOCK):
            v = xhat[:, lo:lo + BLOCK]
            step = torch.exp2(torch.ceil(torch.log2(v.abs().amax(1, keepdim=True).clamp(min=2.0 ** -140) / 126)).clamp(min=-126))
            # log2 may land a whole number off at the border itself
            step = torch.where(v.abs().amax(1, keepdim=True) > 126 * step, 2 * step, step)
            step = torch.where((v.abs().amax(1, keepdim=True) <= 63 * step) & (step > 2.0 ** -126), step / 2, step)
            q = torch.round(v / step)
            on, was = gamma[lo:lo + BLOCK] * q * step + beta[lo:lo + BLOCK] > 0, pre[:, lo:lo + BLOCK] > 0
            up = (gamma[lo:lo + BLOCK] > 0) == was
            q = torch.where(on == was, q, torch.where(up, q + 1, q - 1))
            values[:, lo:lo + BLOCK] = q * step
        return dict(a=pre.clamp(min=0), values=values)
    per = torch.exp2(st["exponents"].double() - 127)
    v = st["codes"].double() * _blocks(per, c)
    pre = gamma * v + beta
    dz = st["dA"].double() * (pre > 0)
    dbeta, dgamma = dz.sum(0), (dz * v).sum(0)
    dx = gamma * norm.invstd.double() * (dz - dz.mean(0) - v * (dz * v).mean(0))
    out = dict(dgamma=dgamma, dbeta=dbeta, a=pre.clamp(min=0))
    if st["add"] is None:
        return dict(out, dx=dx)
    return dict(out, dskip=dx[:, :c // 2] + st["add"].double(), dup=dx[:, c // 2:])
