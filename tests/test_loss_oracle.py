"""The float64 oracle of the training losses: its gradients against central
differences of its losses, and closed forms."""
import numpy as np
import pytest

from oracle import loss as L


def _batch(seed, n=14, V=9):
    g = np.random.Generator(np.random.PCG64(seed))
    x = 2.0 * g.normal(size=(n, V))
    ch = g.integers(0, V, n)
    mask = (g.random(n) < 0.8).astype(np.uint8)
    off = [0, 3, 6, 6, 11, 13]  # an empty request; the last row belongs to none
    return g, x, ch, mask, off


def _differences(f, x, h=1e-6):
    d = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, dn = x.copy(), x.copy()
        up[i] += h
        dn[i] -= h
        d[i] = (f(up) - f(dn)) / (2 * h)
    return d


# a central difference of step h of a function with third derivative of about 1 is off by
# h^2 / 6 and by 2^-53 |f| / h from rounding: about 1e-10 for f of order 1 (1e-8 for the
# squared loss' f of order 100)
@pytest.mark.parametrize("requests,per_request,kl,temperature", [
    (False, False, 0.0, 1.0), (True, True, 0.1, 0.7), (False, True, 0.05, 1.3)])
def test_policy_gradient_is_the_losss(requests, per_request, kl, temperature):
    g, x, ch, mask, off = _batch(3)
    adv = g.normal(size=5 if per_request else 14)
    l, _ = L.rows(x, ch, temperature)
    old, ref = l + 0.3 * g.normal(size=14), l + 0.3 * g.normal(size=14)
    kw = dict(old_logp=old, ref_logp=ref, mask=mask, offsets=off, kl_coef=kl,
              temperature=temperature, requests=requests, per_request=per_request, grad_scale=2.0)
    stats, logp, grad = L.policy(x, ch, adv, **kw)
    d = _differences(lambda y: 2.0 * L.policy(y, ch, adv, **kw)[0][0], x)
    assert np.abs(d - grad).max() < 2e-8
    assert 0 < stats[4] < 1 and (grad[13] == 0).all() and (logp[mask == 0] == 0).all()


@pytest.mark.parametrize("loss", [L.SIGMOID, L.SQUARED, L.HINGE])
@pytest.mark.parametrize("length_norm", [False, True])
def test_preference_gradient_is_the_losss(loss, length_norm):
    g, x, ch, mask, _ = _batch(4)
    off = [0, 3, 5, 9, 13, 13, 14]  # the last pair's first answer is empty
    mask[[0, 4, 6, 10]] = 1
    kw = dict(ref_logp=L.rows(x, ch)[0] + 0.3 * g.normal(size=14), mask=mask, beta=0.4, loss=loss,
              label_smoothing=0.1 if loss == L.SIGMOID else 0.0, length_norm=length_norm)
    stats, s, logp, grad = L.preference(x, ch, off, **kw)
    d = _differences(lambda y: L.preference(y, ch, off, **kw)[0][0], x)
    assert np.abs(d - grad).max() < 2e-7
    assert np.abs(grad[:13]).max() > 0 and (grad[13] == 0).all()


def test_closed_forms():
    # uniform rows: l = -ln V, whatever the level; ratio 1: surrogate = mean advantage
    for level in (0.0, 1e4, -3.4e38):
        stats, logp, grad = L.policy(np.full((2, 5), level), [0, 4], [1.0, 3.0])
        assert np.allclose(logp, -np.log(5)) and np.allclose(stats[:2], [-2.0, 2.0])
        assert np.allclose(grad[0], [-0.4, 0.1, 0.1, 0.1, 0.1])
    # equal answers: h = 0, loss ln 2
    x = np.zeros((2, 3))
    stats, s, _, _ = L.preference(x, [0, 0], [0, 1, 2])
    assert np.isclose(stats[0], np.log(2)) and stats[1] == 0
    # nothing counts
    stats, logp, grad = L.policy(x, [0, 0], [1.0, 1.0], mask=[0, 0])
    assert (stats == 0).all() and (logp == 0).all() and (grad == 0).all()


def test_a_kl_term_of_no_weight_is_no_part_of_the_loss():
    g, x, ch, mask, off = _batch(5)
    l, _ = L.rows(x, ch)
    old, ref = l + 0.1 * g.normal(size=14), l + 0.1
    ref[1], ref[8] = np.inf, np.nan
    mask[[1, 8]] = 1
    adv = g.normal(size=14)
    a = L.policy(x, ch, adv, old, None, mask, off)
    b = L.policy(x, ch, adv, old, ref, mask, off)
    assert np.isfinite(a[0]).all() and not np.isfinite(b[0][2])
    assert (np.delete(a[0], 2) == np.delete(b[0], 2)).all()
    assert (a[1] == b[1]).all() and (a[2] == b[2]).all()


def test_an_answer_without_a_partner_has_no_gradient():
    x = np.random.Generator(np.random.PCG64(6)).normal(size=(8, 5))
    x[1, 2], x[2] = np.nan, np.inf
    _, _, logp, grad = L.preference(x, [0] * 8, [0, 0, 4, 6, 8])
    assert np.isnan(logp[1:3]).all() and not grad[:4].any() and (grad[4:] != 0).all()


def test_rows_belong_to_one_request():
    """In order: the request whose bounds hold the row.  Where offsets decrease each row is
    counted at most once."""
    g = np.random.Generator(np.random.PCG64(7))
    for _ in range(50):
        off = np.sort(g.integers(-1, 14, 6))
        req, count = L.counted(12, None, off)
        for t in range(12):
            own = [r for r in range(5) if 0 <= off[r] <= t < off[r + 1] <= 12]
            assert req[t] == (own[0] if own else -1)
        assert (count == [(req == r).sum() for r in range(5)]).all()
    req, count = L.counted(10, None, [0, 6, 3, 10])
    assert req.tolist() == [0] * 6 + [2] * 4 and count.tolist() == [6, 0, 4]


def test_a_term_of_no_weight_is_no_part_of_the_pair_loss():
    x = np.random.Generator(np.random.PCG64(8)).normal(size=(4, 5))
    x[3, 0] = -np.inf  # the other answer has a masked token: h is infinite
    assert L.preference(x, [0] * 4, [0, 2, 4])[0][0] == 0.0
    assert L.preference(x, [0] * 4, [0, 2, 4], label_smoothing=0.1)[0][0] == np.inf
    assert L.preference(x[::-1], [0] * 4, [0, 2, 4], label_smoothing=1.0)[0][0] == 0.0
    assert np.isinf(L.preference(x[::-1], [0] * 4, [0, 2, 4])[0][0])
