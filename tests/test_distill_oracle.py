"""The float64 oracle of distillation and of the norm: gradients against central differences
of its own losses, closed forms, and orders."""
import numpy as np
import pytest

from oracle import distill as D


def _differences(f, x, h=1e-6):
    d = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, dn = x.copy(), x.copy()
        up[i] += h
        dn[i] -= h
        d[i] = (f(up) - f(dn)) / (2 * h)
    return d


def _batch(seed, n=9, V=11, k=4):
    g = np.random.Generator(np.random.PCG64(seed))
    x = 2.0 * g.normal(size=(n, V))
    ids = np.stack([g.permutation(V)[:k] for _ in range(n)])
    z = 2.0 * g.normal(size=(n, V))
    lp = z - np.log(np.exp(z).sum(1, keepdims=True))
    sent = np.take_along_axis(lp, ids, 1)
    ids[1, 2] = -1        # absent entries, by id and by probability
    sent[2, 0] = -np.inf
    ids[3] = -1           # a row without entries
    return g, x, ids, sent, g.integers(0, V, n)


# a central difference of step h of a function with third derivative of about 1 is off by
# h^2 / 6 and by 2^-53 |f| / h from rounding: about 1e-10 for f of order 1
@pytest.mark.parametrize("loss", [D.FORWARD, D.REVERSE])
@pytest.mark.parametrize("rest", [D.CLASS, D.NONE])
@pytest.mark.parametrize("ce", [0.0, 0.4])
def test_gradient_is_the_losss(loss, rest, ce):
    g, x, ids, sent, ch = _batch(5)
    kw = dict(chosen=ch, mask=(g.random(9) < 0.8).astype(np.uint8), offsets=[0, 2, 2, 8],
              kl_coef=0.7, ce_coef=ce, temperature=1.4, loss=loss, rest=rest, requests=ce > 0,
              grad_scale=1.0)
    grad = D.distill(x, ids, sent, **kw)[2]
    want = _differences(lambda v: D.distill(v, ids, sent, **kw)[0][0], x)
    assert np.abs(grad - want).max() < 1e-8
    assert np.abs(grad).max() > 1e-3 and not grad[8].any()


def test_divergence_of_a_whole_list_is_the_textbooks():
    g, x, _, _, _ = _batch(7)
    n, V = x.shape
    ids = np.tile(np.arange(V), (n, 1))
    z = g.normal(size=(n, V))
    lp = z - np.log(np.exp(z).sum(1, keepdims=True))
    lq = x - np.log(np.exp(x).sum(1, keepdims=True))
    for rest in (D.CLASS, D.NONE):
        kl = D.distill(x, ids, lp, rest=rest)[1]
        assert np.abs(kl - (np.exp(lp) * (lp - lq)).sum(1)).max() < 1e-12
        kl = D.distill(x, ids, lp, rest=rest, loss=D.REVERSE)[1]
        assert np.abs(kl - (np.exp(lq) * (lq - lp)).sum(1)).max() < 1e-12


def test_orders_and_masked_tokens():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0], [-np.inf] * 5, [0, np.nan, 0, 0, 0],
                  [5.0, -3e38, -np.inf, 4.0, -np.inf]])
    ids, logp = D.top_logits(x, 4)
    assert ids.tolist() == [[1, 2, 4, 0], [-1] * 4, [-1] * 4, [0, 3, -1, -1]]
    assert np.isnan(logp[1:3]).all() and (logp[3, 2:] == -np.inf).all()
    assert abs(np.exp(logp[3, :2]).sum() - 1) < 1e-12


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradient_is_the_norms(rms):
    g = np.random.Generator(np.random.PCG64(2))
    h, w, b, dy = g.normal(size=(3, 7)), g.normal(size=7), g.normal(size=7), g.normal(size=(3, 7))

    def f(h_, w_, b_):
        return (D.norm(h_, w_, b_, rms=rms)[0] * dy).sum()

    _, mean, rstd = D.norm(h, w, b, rms=rms)
    dx, dw, db = D.norm_backward(dy, h, w, mean, rstd, rms=rms)
    assert np.abs(dx - _differences(lambda v: f(v, w, b), h)).max() < 1e-8
    assert np.abs(dw - _differences(lambda v: f(h, v, b), w)).max() < 1e-8
    assert np.abs(db - _differences(lambda v: f(h, w, v), b)).max() < 1e-8
