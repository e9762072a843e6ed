"""GPU parity of the training losses (pr_policy_loss, pr_preference_loss) with
the float64 oracle, at the sizes, masks and values where they can go wrong.

Tolerances, from the kernels' arithmetic (2^-24 = 6e-8 per fp32 rounding):
  logp   a row's sum of exponentials is a sum of positive fp32 terms, each off by
         2^-22 and by |z - max| 2^-23 (weighted by the term itself: below 1e-6), in
         chains of up to 500 terms (3e-5 at worst, the roundings' mean far less):
         2e-5; the two roundings of z_y - max and of the difference: 4e-7 |l|
  grad   dL/dl carries logp's error through an exponential and a few products: 1e-4
         relative; p the exponent's error of |z - max| 2^-23 and logp's: 6e-5 relative.
         Together 2e-4 |g|, and 1e-6 of the row's largest entry for those that cancel;
         bf16 (eight significant bits) adds half a unit in the last place, 2^-8
  stats  weighted means of the terms, whose size `scale` gives: 1e-4 of it
"""
import numpy as np
import pytest
import torch

from oracle import loss as L

pytestmark = pytest.mark.gpu
CLIP = dict(clip_low=0.2, clip_high=0.3)


@pytest.fixture(scope="module")
def B():
    from paper_2608_28726_gb300 import build as prbuild
    prbuild.build()
    from paper_2608_28726_gb300 import binding
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.pr_ctx_create(0, 1, 1)
    yield c
    B.pr_ctx_destroy(c)


def to(a, dtype=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def draw(seed, n, V, dtype, scale=3.0, temperature=1.0):
    """(logits as the GPU holds them, their float64 values, chosen, old, ref):
    ratios kept off the clip bounds, where the slope jumps."""
    g = np.random.Generator(np.random.PCG64(seed))
    x = torch.from_numpy((scale * g.normal(size=(n, V))).astype(np.float32))
    x[torch.arange(n), torch.from_numpy(g.integers(0, V, n))] += 6.0
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x64 = x.double().numpy()
    ch = np.where(g.random(n) < 0.5, x64.argmax(1), g.integers(0, V, n)).astype(np.int32)
    l, _ = L.rows(x64, ch, temperature)
    d = 0.3 * g.normal(size=n)
    for edge in (np.log(0.8), np.log(1.3)):
        d = np.where(np.abs(d - edge) < 2e-3, edge + 4e-3, d)
    old = (l - d).astype(np.float32)
    ref = (l + 0.3 * g.normal(size=n)).astype(np.float32)
    return g, x.cuda(), x64, ch, old, ref


def check_rows(got, logp, want, grad, dtype, what=""):
    l = got.double().cpu().numpy()
    bad = ~((np.abs(l - logp) <= 2e-5 + 4e-7 * np.abs(logp)) | (np.isnan(l) & np.isnan(logp))
            | (l == logp))
    assert not bad.any(), "%s logp %s: %s for %s" % (what, np.flatnonzero(bad)[:5], l[bad][:5],
                                                    logp[bad][:5])
    if want is None:
        return
    w = want.double().cpu().numpy()
    rel = 2e-4 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    with np.errstate(invalid="ignore"):
        big = np.abs(grad).max(axis=1, keepdims=True)
        ok = (np.abs(w - grad) <= rel * np.abs(grad) + 1e-6 * big) | (np.isnan(w) & np.isnan(grad))
    assert ok.all(), "%s grad: %d of %d, at %s: %s for %s" % (
        what, (~ok).sum(), ok.size, np.argwhere(~ok)[:4].tolist(), w[~ok][:4], grad[~ok][:4])


def check_stats(got, want, scale):
    s = got.double().cpu().numpy()
    ok = (np.abs(s - want) <= 1e-4 * np.maximum(scale, np.abs(want))) | (np.isnan(s) & np.isnan(want))
    assert ok.all(), (s, want)


def offsets_of(g, n, n_req):
    cut = np.sort(g.integers(0, n + 1, n_req - 1)) if n_req > 1 else np.zeros(0, np.int64)
    return np.r_[0, cut, n].astype(np.int64)


SIZES = [(1, 1), (3, 2), (5, 7), (5, 8), (4, 9), (7, 31), (9, 33), (6, 255), (3, 1000), (37, 1001),
         (200, 515), (2, 4096), (3, 8191), (3, 16384), (5, 32000), (2, 32003), (170, 2050),
         (2, 70001), (3, 151936), (2, 262144), (1, 300007)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_policy_sizes(B, ctx, n, V, dtype):
    T = 1.0 if V % 2 else 0.8
    g, x, x64, ch, old, ref = draw(V * 7 + n, n, V, dtype, temperature=T)
    n_req = min(n, 5)
    off = offsets_of(g, n, n_req)
    mask = (g.random(n) < 0.8).astype(np.uint8)
    per = bool(V % 3)
    adv = g.normal(size=n_req if per else n).astype(np.float32)
    norm = n % 2
    kw = dict(kl_coef=0.05, temperature=T, per_request=per, grad_scale=1.5, **CLIP)
    stats, logp, grad = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), ref_logp=to(ref),
                                         mask=to(mask), offsets=to(off), norm=norm, **kw)
    s, l, gr = L.policy(x64, ch, adv, old, ref, mask, off, requests=bool(norm), **kw)
    check_rows(logp, l, grad, gr, dtype)
    check_stats(stats, s, 2.0 * (mask.any() or 0))
    # the loss alone gives the same bits
    st2, lp2, none = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), ref_logp=to(ref),
                                      mask=to(mask), offsets=to(off), norm=norm, want_grad=False, **kw)
    assert none is None and torch.equal(lp2, logp) and torch.equal(st2, stats)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_preference_sizes(B, ctx, n, V, dtype):
    T = 0.9 if V % 2 else 1.0
    g, x, x64, ch, _, ref = draw(V * 5 + n, n, V, dtype, temperature=T)
    n_req = 2 * min(max(n // 2, 1), 6)
    off = offsets_of(g, n, n_req)
    mask = (g.random(n) < 0.85).astype(np.uint8)
    kind = n % 3
    kw = dict(loss=kind, beta=0.2, label_smoothing=0.1 if kind == 0 else 0.0,
              margin=0.25 if kind != 1 else 0.0, length_norm=bool(V % 2), temperature=T)
    stats, ratio, logp, grad = B.pr_preference_loss(ctx, x, to(ch), to(off), ref_logp=to(ref),
                                                    mask=to(mask), **kw)
    s, r, l, gr = L.preference(x64, ch, off, ref, mask, **kw)
    check_rows(logp, l, grad, gr, dtype)
    # a sum of a request's rows, each off by logp's error
    lim = 2e-5 * np.maximum(np.diff(off), 1) + 1e-6 * np.abs(r) * (1 if kw["length_norm"] else 1)
    assert (np.abs(ratio.double().cpu().numpy() - r) <= lim + 1e-6).all()
    check_stats(stats, s, 0.2 * np.abs(r).max() + 1.0 + (3.0 * np.abs(r).max() + 25.0) * (kind == 1))
    st2, r2, lp2, _ = B.pr_preference_loss(ctx, x, to(ch), to(off), ref_logp=to(ref),
                                           mask=to(mask), want_grad=False, **kw)
    assert torch.equal(lp2, logp) and torch.equal(st2, stats) and torch.equal(r2, ratio)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 1003, 40000])
def test_values_that_a_softmax_can_trip_over(B, ctx, V, dtype):
    """Masked tokens, the type's lowest value, large logits, NaN and infinities, in
    counted and in masked rows."""
    n = 16
    g, x, x64, ch, old, ref = draw(V, n, V, dtype)
    low = torch.finfo(x.dtype).min
    mask = np.ones(n, np.uint8)
    x[0, : V // 2] = -torch.inf
    x[1] = -torch.inf                 # nothing left
    x[2] = low                        # a uniform row of the lowest value
    x[3, 1:] = low                    # one token left
    x[4, 3] = torch.nan
    x[5, V - 1] = torch.inf
    x[6] = 3e4 + x[6]                 # large logits
    x[7] = torch.where(torch.arange(V, device="cuda") % 3 == 0, 3e38, -3e38).to(x.dtype)
    x[8], x[9], x[10] = torch.nan, torch.inf, -torch.inf  # masked rows
    mask[8:11] = 0
    x[11, : V - 1] = -torch.inf       # the last element alone
    x[12, 1:] = -torch.inf            # the first alone
    x[13, ::2] = -torch.inf
    ch[0], ch[3], ch[7], ch[11], ch[12], ch[13] = V - 1, 0, 3, V - 1, 0, 1
    ch[8] = -7                        # masked: not looked at
    ch[14], ch[15] = V, -1            # outside the vocabulary
    x64 = x.double().cpu().numpy()
    l, _ = L.rows(x64, ch)
    old = np.where(np.isfinite(l), l - 0.1, 0.0).astype(np.float32)
    ref = np.where(np.isfinite(l), l + 0.2, 0.0).astype(np.float32)
    adv = g.normal(size=n).astype(np.float32)
    B.pr_ctx_flags(ctx, clear=True)
    stats, logp, grad = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), ref_logp=to(ref),
                                         mask=to(mask), kl_coef=0.1, **CLIP)
    assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_NONFINITE | B.PR_FLAG_BAD_CHOSEN
    s, lo, gr = L.policy(x64, ch, adv, old, ref, mask, kl_coef=0.1, **CLIP)
    assert np.isnan(lo[[1, 4, 5, 14, 15]]).all() and np.isfinite(lo[[0, 2, 3, 6, 7, 11, 12, 13]]).all()
    check_rows(logp, lo, grad, gr, dtype)
    check_stats(stats, s, 1.0)
    assert not grad[8:11].any()
    # without the rows that are NaN by right, everything is finite
    mask[[1, 4, 5, 14, 15]] = 0
    for off in ([0, 16], [0, 4, 9, 16]):
        stats, logp, grad = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old),
                                             ref_logp=to(ref), mask=to(mask), kl_coef=0.1,
                                             offsets=to(off, np.int64), **CLIP)
        s, lo, gr = L.policy(x64, ch, adv, old, ref, mask, off, kl_coef=0.1, **CLIP)
        assert np.isfinite(s).all() and torch.isfinite(grad).all()
        check_rows(logp, lo, grad, gr, dtype)
        check_stats(stats, s, 1.0)
    off = [0, 4, 9, 12, 16]
    st, r, logp, grad = B.pr_preference_loss(ctx, x, to(ch), to(off, np.int64), ref_logp=to(ref),
                                             mask=to(mask))
    s, ro, lo, gr = L.preference(x64, ch, off, ref, mask)
    check_rows(logp, lo, grad, gr, dtype)
    check_stats(st, s, 1.0)
    assert B.pr_ctx_flags(ctx, clear=True) == 0


def test_a_nan_pair_leaves_the_others_gradients(B, ctx):
    g, x, _, ch, _, ref = draw(5, 12, 700, "f32")
    x[1, 17] = torch.nan
    off = np.array([0, 3, 6, 9, 12], np.int64)
    st, r, logp, grad = B.pr_preference_loss(ctx, x, to(ch), to(off), ref_logp=to(ref))
    s, ro, lo, gr = L.preference(x.double().cpu().numpy(), ch, off, ref)
    assert torch.isnan(st[[0, 2, 3]]).all() and torch.isnan(grad[:6]).all()
    check_rows(logp, lo, grad, gr, "f32")
    B.pr_ctx_flags(ctx, clear=True)


def test_batches_without_a_counted_row(B, ctx):
    g, x, x64, ch, old, ref = draw(1, 6, 300, "bf16")
    mask = to(np.zeros(6, np.uint8))
    for norm in (0, 1):
        st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(old), mask=mask, norm=norm,
                                      offsets=to([0, 2, 2, 6], np.int64))
        assert not st.any() and not lp.any() and not gr.any()
    st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to([0, 3, 6], np.int64), mask=mask)
    assert not st.any() and not r.any() and not lp.any() and not gr.any()
    # an answer without rows: its pair says nothing, the other one all
    off = np.array([0, 0, 2, 4, 6], np.int64)
    st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to(off), ref_logp=to(ref))
    s, ro, lo, go = L.preference(x64, ch, off, ref)
    check_rows(lp, lo, gr, go, "bf16")
    check_stats(st, s, 1.0)
    assert not gr[:2].any() and gr[2:].any()
    assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_EMPTY_REQ
    # no rows at all
    empty = x[:0]
    st, lp, gr = B.pr_policy_loss(ctx, empty, to(ch), to(old))
    assert not st.any() and gr.shape == (0, 300)
    st, r, lp, gr = B.pr_preference_loss(ctx, empty, to(ch), to([0, 0, 0], np.int64))
    assert not st.any() and not r.any()
    B.pr_ctx_flags(ctx, clear=True)


def test_offsets_that_leave_the_batch(B, ctx):
    """Bad requests count nothing and are reported; rows outside all requests are
    left out."""
    g, x, x64, ch, old, ref = draw(2, 10, 500, "f32")
    adv = g.normal(size=10).astype(np.float32)
    for off, flag in (([2, 4, 9], 0), ([0, 4, 12], B.PR_FLAG_BAD_OFFSETS),
                      ([-3, 4, 10], B.PR_FLAG_BAD_OFFSETS)):
        st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old),
                                      offsets=to(off, np.int64), norm=1)
        s, lo, go = L.policy(x64, ch, adv, old, None, None, off, requests=True)
        check_rows(lp, lo, gr, go, "f32")
        check_stats(st, s, 1.0)
        assert B.pr_ctx_flags(ctx, clear=True) == flag


def test_on_policy_and_no_reference(B, ctx):
    """old_logp NULL: the ratio is 1 and the slope the advantage; without a reference
    kl_coef has nothing to weigh."""
    g, x, x64, ch, _, _ = draw(3, 8, 4000, "bf16")
    adv = g.normal(size=8).astype(np.float32)
    st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), kl_coef=0.3)
    s, lo, go = L.policy(x64, ch, adv, kl_coef=0.3)
    check_rows(lp, lo, gr, go, "bf16")
    check_stats(st, s, 1.0)
    assert st[3].item() == 1.0 and st[2].item() == 0.0 and st[5].item() == 0.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,stride,start,gstride,gstart", [
    (999, 999, 0, 999, 0), (1000, 1008, 3, 1003, 0), (1000, 1000, 0, 1001, 1), (2051, 2053, 5, 2053, 5),
    (33, 40, 1, 35, 2), (20011, 20011, 7, 20016, 0), (160001, 160001, 1, 160001, 1)])
def test_strides_and_alignments(B, ctx, V, stride, start, gstride, gstart, dtype):
    """Rows off the 16-byte grid, gradients on another grid than their logits; bytes
    between and around the gradient's rows stay as they are."""
    n = 5
    g, x, x64, ch, old, ref = draw(V + stride, n, V, dtype)
    buf = torch.full((start + n * stride + 9,), torch.nan, dtype=x.dtype, device="cuda")
    xs = buf[start:start + n * stride].view(n, stride)[:, :V]
    xs.copy_(x)
    gbuf = torch.full((gstart + n * gstride + 9,), 7.0, dtype=x.dtype, device="cuda")
    gv = gbuf[gstart:gstart + n * gstride].view(n, gstride)
    adv = g.normal(size=n).astype(np.float32)
    st, lp, gr = B.pr_policy_loss(ctx, xs, to(ch), to(adv), old_logp=to(old), ref_logp=to(ref),
                                  kl_coef=0.1, grad=gv[:, :V])
    s, lo, go = L.policy(x64, ch, adv, old, ref, kl_coef=0.1)
    check_rows(lp, lo, gr, go, dtype)
    check_stats(st, s, 1.0)
    out = gbuf.clone()
    out[gstart:gstart + n * gstride].view(n, gstride)[:, :V] = 7.0
    assert (out == 7.0).all()
    off = np.array([0, 2, 5], np.int64)
    gbuf.fill_(7.0)
    st, r, lp, gr = B.pr_preference_loss(ctx, xs, to(ch), to(off), ref_logp=to(ref), grad=gv[:, :V])
    s, ro, lo, go = L.preference(x64, ch, off, ref)
    check_rows(lp, lo, gr, go, dtype)
    out = gbuf.clone()
    out[gstart:gstart + n * gstride].view(n, gstride)[:, :V] = 7.0
    assert (out == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(40, 1001), (330, 5000), (6, 151936), (3, 600003)])
def test_gradient_in_place_of_the_logits(B, ctx, n, V, dtype):
    g, x, _, ch, old, ref = draw(n, n, V, dtype)
    off = offsets_of(g, n, 2)
    adv = g.normal(size=n).astype(np.float32)
    args = dict(ref_logp=to(ref), offsets=to(off))
    a = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), kl_coef=0.1, **args)
    y = x.clone()
    b = B.pr_policy_loss(ctx, y, to(ch), to(adv), old_logp=to(old), kl_coef=0.1, grad=y, **args)
    assert all(torch.equal(u, v) for u, v in zip(a, b)) and b[2].data_ptr() == y.data_ptr()
    a = B.pr_preference_loss(ctx, x, to(ch), **args)
    y = x.clone()
    b = B.pr_preference_loss(ctx, y, to(ch), grad=y, **args)
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_gradient_is_the_difference_of_the_loss(B, ctx):
    """Central differences of the library's own loss in fp32: step 1/16 on the logits of
    the emitted token and of others.  The truncation is h^2 / 6 times a third
    derivative of at most the slope, rounding 2e-6 / h of the loss: 1.5e-3 of the row's
    slope, and 1e-4."""
    n, V = 6, 50
    g, x, x64, ch, old, ref = draw(9, n, V, "f32", scale=1.0)
    off = to([0, 1, 3, 6], np.int64)
    adv = to(np.array([0.8, -1.2, 0.5], np.float32))
    kw = dict(old_logp=to(old), ref_logp=to(ref), offsets=off, per_request=True, kl_coef=0.2,
              norm=B.PR_NORM_REQUESTS, clip_low=1.0, clip_high=9.0)
    pair = dict(ref_logp=to(ref), beta=0.5)

    def policy(y):
        return B.pr_policy_loss(ctx, y, to(ch), adv, want_grad=False, **kw)[0][0].item()

    def preference(y):
        return B.pr_preference_loss(ctx, y, to(ch), to([0, 3, 6], np.int64), want_grad=False,
                                    **pair)[0][0].item()

    for f, grad in ((policy, B.pr_policy_loss(ctx, x, to(ch), adv, **kw)[2]),
                    (preference, B.pr_preference_loss(ctx, x, to(ch), to([0, 3, 6], np.int64),
                                                      **pair)[3])):
        h = 1.0 / 16
        for t in range(n):
            for v in {int(ch[t]), 0, V - 1}:
                up, dn = x.clone(), x.clone()
                up[t, v] += h
                dn[t, v] -= h
                d = (f(up) - f(dn)) / (2 * h)
                assert abs(d - grad[t, v].item()) <= 1.5e-3 * grad[t].abs().max().item() + 1e-4


def test_many_short_rows_and_one_long_request(B, ctx):
    for n, V, n_req in ((5000, 130, 1), (3000, 64, 1500), (20011, 9, 40)):
        g, x, x64, ch, old, ref = draw(n, n, V, "f32")
        off = offsets_of(g, n, n_req)
        mask = (g.random(n) < 0.7).astype(np.uint8)
        adv = g.normal(size=n_req).astype(np.float32)
        st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), mask=to(mask),
                                      offsets=to(off), per_request=True, norm=1)
        # the oracle's loops are slow: its formulas on whole arrays
        req, count = np.full(n, -1), np.zeros(n_req, np.int64)
        own = np.searchsorted(off, np.arange(n), side="right") - 1
        req[mask == 1] = own[mask == 1]
        np.add.at(count, own, mask)
        z = x64 - x64.max(1, keepdims=True)
        p = np.exp(z)
        p /= p.sum(1, keepdims=True)
        l = np.log(p[np.arange(n), ch])
        r = np.exp(l - old)
        A = adv[own]
        free, cut = r * A, np.clip(r, 0.8, 1.2) * A
        keep = (np.abs(r - 0.8) > 1e-3) & (np.abs(r - 1.2) > 1e-3)  # away from the jumps
        w = mask / ((count > 0).sum() * np.maximum(count[own], 1))
        k = w * np.where(cut < free, 0.0, -free)
        go = -k[:, None] * p
        go[np.arange(n), ch] += k
        check_rows(lp, l * mask, None, None, "f32")
        check_rows(lp[torch.from_numpy(keep)], (l * mask)[keep], gr[torch.from_numpy(keep)],
                   go[keep], "f32")
        assert abs(st[0].item() + (w * np.minimum(free, cut)).sum()) < 1e-4


def test_results_repeat_and_survive_other_streams_and_graphs(B, ctx):
    n, V = 400, 9001
    g, x, _, ch, old, ref = draw(21, n, V, "bf16")
    off = to(offsets_of(g, n, 10))
    adv = to(g.normal(size=n).astype(np.float32))
    chd, oldd, refd = to(ch), to(old), to(ref)
    grad = torch.empty_like(x)
    stats, logp = torch.empty(6, device="cuda"), torch.empty(n, device="cuda")
    pstats, ratio, plogp = (torch.empty(5, device="cuda"), torch.empty(10, device="cuda"),
                            torch.empty(n, device="cuda"))
    pgrad = torch.empty_like(x)
    y = x.clone()

    def run():
        B.pr_policy_loss(ctx, y, chd, adv, old_logp=oldd, ref_logp=refd, offsets=off, kl_coef=0.1,
                         stats=stats, logp=logp, grad=grad)
        B.pr_preference_loss(ctx, y, chd, off, ref_logp=refd, stats=pstats, ratio=ratio, logp=plogp,
                             grad=pgrad)

    out = (stats, logp, grad, pstats, ratio, plogp, pgrad)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    side = torch.cuda.Stream()
    for _ in range(4):
        for t in out:
            t.zero_()
        y.zero_()
        y.copy_(x)  # written by the kernel just before the call
        run()
        for t, w in zip(out, want):
            assert torch.equal(t, w)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y.copy_(x)
        run()
    for t in out:
        t.zero_()
    y.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for t, w in zip(out, want):
        assert torch.equal(t, w)


def test_refusals(B, ctx):
    g, x, _, ch, old, ref = draw(2, 4, 64, "f32")
    c, a, off = to(ch), to(old), to([0, 2, 4], np.int64)
    bad = [dict(temperature=0.0), dict(temperature=float("nan")), dict(clip_low=-0.1),
           dict(clip_low=1.5), dict(clip_high=-1.0), dict(kl_coef=-1.0), dict(norm=7),
           dict(grad_scale=float("inf")), dict(per_request=True), dict(grad=x[:, :32]),
           dict(grad=x[:2]), dict(grad=x.bfloat16()), dict(grad=torch.empty(64, 4, device="cuda").t()),
           dict(mask=torch.ones(3, dtype=torch.uint8, device="cuda")), dict(mask=a),
           dict(old_logp=a.double()), dict(ref_logp=a[:3]), dict(stats=a[:2]),
           dict(logp=torch.empty(4)), dict(offsets=off.int())]
    n0 = B.launch_count()
    for k in bad:
        with pytest.raises(B.PRError) as e:
            B.pr_policy_loss(ctx, x, c, a, **k)
        assert e.value.status == B.PR_ERR_INVALID_ARG, k
    with pytest.raises(B.PRError):
        B.pr_policy_loss(ctx, x, c[:3], a)
    # the logits' buffer as the gradient, with another stride
    wide = torch.zeros(8, 64, device="cuda")
    with pytest.raises(B.PRError):
        B.pr_policy_loss(ctx, wide[::2], to(ch), a, grad=wide[:4])
    bad = [dict(beta=0.0), dict(beta=float("inf")), dict(loss=3), dict(label_smoothing=1.5),
           dict(loss=2, label_smoothing=0.1), dict(loss=1, margin=0.5), dict(margin=float("nan")),
           dict(ratio=a[:1]), dict(temperature=-1.0), dict(ref_logp=a[:2])]
    for k in bad:
        with pytest.raises(B.PRError) as e:
            B.pr_preference_loss(ctx, x, c, off, **k)
        assert e.value.status == B.PR_ERR_INVALID_ARG, k
    with pytest.raises(B.PRError):  # three answers are no pairs
        B.pr_preference_loss(ctx, x, c, to([0, 1, 2, 4], np.int64))
    assert B.launch_count() == n0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_overlap_or_end_early_are_refused(B, ctx, dtype):
    g, x, _, ch, old, ref = draw(3, 4, 64, dtype)
    c, a, off = to(ch), to(old), to([0, 2, 4], np.int64)
    one = x[:1].expand(4, 64)
    steps = torch.zeros(200, dtype=x.dtype, device="cuda").as_strided((4, 64), (32, 1))
    n0 = B.launch_count()
    for call in (lambda **k: B.pr_policy_loss(ctx, k.pop("x", x), c, a, **k),
                 lambda **k: B.pr_preference_loss(ctx, k.pop("x", x), c, off, **k)):
        for k in (dict(x=one), dict(x=steps), dict(grad=one), dict(grad=steps), dict(vocab=65),
                  dict(vocab=0), dict(vocab=-1), dict(x=x[0]), dict(x=x.view(2, 2, 64)),
                  dict(x=x[:, :0])):
            with pytest.raises(B.PRError) as e:
                call(**k)
            assert e.value.status == B.PR_ERR_INVALID_ARG, k
    assert B.launch_count() == n0


def test_one_row_has_any_stride(B, ctx):
    """A single row's stride is never used, so whatever a view says of it will do."""
    g, x, x64, ch, old, ref = draw(5, 1, 96, "f32")
    one = torch.zeros(1, 96, device="cuda").as_strided((1, 96), (0, 1)).copy_(x)
    want = B.pr_policy_loss(ctx, x, to(ch), to(old))
    got = B.pr_policy_loss(ctx, one, to(ch), to(old), grad=torch.empty(96, device="cuda").as_strided(
        (1, 96), (3, 1)))
    for w, t in zip(want, got):
        assert torch.equal(w, t)


@pytest.mark.parametrize("n,n_req", [(31, 31), (33, 2), (511, 3), (512, 512), (512, 1), (513, 512),
                                     (300, 513), (513, 4), (1500, 1024), (1500, 1025), (4096, 7),
                                     (4097, 7)])
@pytest.mark.parametrize("keep", [0.02, 0.5, 1.0])
def test_how_rows_are_listed(B, ctx, n, n_req, keep):
    """Rows and requests around the sizes at which the counted rows are listed another
    way: by each CTA, by one CTA, by two kernels."""
    V = 24
    g, x, x64, ch, old, ref = draw(n * 3 + n_req, n, V, "f32")
    off = offsets_of(g, n, n_req)
    mask = (g.random(n) < keep).astype(np.uint8)
    adv = g.normal(size=n_req).astype(np.float32)

    # the same rows in a batch whose further rows and requests are empty: listed by two kernels
    more, more_req = 4200 - n, 1100 - n_req

    def pad(t, k=None):
        k = more if k is None else k
        return None if t is None else np.concatenate([t, np.full((k, *t.shape[1:]), 0, t.dtype)])

    wide = torch.full((n + more, V), torch.nan, device="cuda")
    wide[:n] = x
    for norm in (0, 1):
        kw = dict(norm=norm, per_request=True, kl_coef=0.1)
        stats, logp, grad = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old),
                                             ref_logp=to(ref), mask=to(mask), offsets=to(off), **kw)
        s, l, _ = L.policy(x64, ch, adv, old, ref, mask, off, requests=bool(norm),
                           per_request=True, kl_coef=0.1, clip_low=0.2, clip_high=0.2)
        check_rows(logp, l, None, None, "f32")
        check_stats(stats, s, 2.0 * (mask.any() or 0))
        s2, l2, g2 = B.pr_policy_loss(ctx, wide, to(pad(ch)), to(pad(adv, more_req)),
                                      old_logp=to(pad(old)), ref_logp=to(pad(ref)),
                                      mask=to(pad(mask)),
                                      offsets=to(np.r_[off, np.full(more_req, n)]), **kw)
        assert torch.equal(l2[:n], logp) and torch.equal(g2[:n], grad)
        assert not l2[n:].any() and not g2[n:].any()
        check_stats(s2, s, 2.0 * (mask.any() or 0))
    off = offsets_of(g, n, n_req + n_req % 2)
    kw = dict(beta=0.2, loss=0, label_smoothing=0.1, margin=0.25, length_norm=bool(n % 2))
    stats, ratio, logp, grad = B.pr_preference_loss(ctx, x, to(ch), to(off), ref_logp=to(ref),
                                                    mask=to(mask), **kw)
    s, r, l, _ = L.preference(x64, ch, off, ref, mask, temperature=1.0, **kw)
    check_rows(logp, l, None, None, "f32")
    lim = 2e-5 * np.maximum(np.diff(off), 1) + 1e-6 * np.abs(r)
    assert (np.abs(ratio.double().cpu().numpy() - r) <= lim + 1e-6).all()
    check_stats(stats, s, 0.2 * np.abs(r).max() + 1.0)
    k = 1100 - (len(off) - 1)
    s2, r2, l2, g2 = B.pr_preference_loss(ctx, wide, to(pad(ch)), to(np.r_[off, np.full(k, n)]),
                                          ref_logp=to(pad(ref)), mask=to(pad(mask)), **kw)
    assert torch.equal(l2[:n], logp) and torch.equal(g2[:n], grad) and torch.equal(s2, stats)
    assert torch.equal(r2[:len(r)], ratio) and not r2[len(r):].any()
    assert not l2[n:].any() and not g2[n:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,stride,start", [(1, 1, 0), (7, 9, 3), (515, 515, 0), (3001, 3003, 1),
                                            (3536, 3536, 0), (5504, 5504, 0), (5653, 5660, 5),
                                            (9000, 9008, 8), (11400, 11400, 0), (12474, 12474, 2)])
def test_many_short_rows(B, ctx, V, stride, start, dtype):
    """More rows than the CTAs have places, of lengths that give a warp, a CTA or several
    CTAs to a row, at any alignment, some of them odd; the gradient in place too.

    Gradients: check_rows' bounds, and what an error of 3e-7 (1 + |l|) in l does to the two
    terms of the slope, which may cancel or be small by themselves."""
    n = 1300 if V < 6000 else 700
    g, x, x64, ch, old, ref = draw(V, n, V, dtype)
    off = offsets_of(g, n, 8)
    mask = (g.random(n) < 0.9).astype(np.uint8)
    odd = {3: np.nan, 5: np.inf, 8: -np.inf, 11: float(torch.finfo(x.dtype).min)}
    for t, v in odd.items():
        x[t] = v
        x64[t] = v
        mask[t] = t == 11  # (a row of the lowest value counts, the others must not be seen)
    if V > 7:
        x[14, : V // 2] = -torch.inf
        x64[14, : V // 2] = -np.inf
        ch[14] = V - 1
    l64, p64 = L.rows(x64, ch, 1.0)
    for t in (11, 14):
        old[t], ref[t] = l64[t] - 0.1, l64[t] + 0.1
    ch[3:9:5] = -1  # (ids of masked rows are not looked at)
    adv = g.normal(size=n).astype(np.float32)
    kw = dict(kl_coef=0.1, grad_scale=2.0)

    buf = torch.zeros(start + n * stride + 16, dtype=x.dtype, device="cuda")
    xs = buf[start:start + n * stride].view(n, stride)[:, :V]
    xs.copy_(x)
    B.pr_ctx_flags(ctx, clear=True)
    args = dict(old_logp=to(old), ref_logp=to(ref), mask=to(mask), offsets=to(off))
    stats, logp, grad = B.pr_policy_loss(ctx, xs, to(ch), to(adv), norm=1, **args, **kw)
    s, l, gr = L.policy(x64, ch, adv, old, ref, mask, off, requests=True, clip_low=0.2,
                        clip_high=0.2, **kw)
    assert B.pr_ctx_flags(ctx, clear=True) & ~B.PR_FLAG_EMPTY_REQ == 0
    check_rows(logp, l, None, None, dtype)
    check_stats(stats, s, 2.0)
    req = np.searchsorted(off, np.arange(n), side="right") - 1
    count = np.array([mask[a:b].sum() for a, b in zip(off[:-1], off[1:])])
    on = mask != 0
    with np.errstate(invalid="ignore", over="ignore"):
        share = 2.0 / (count > 0).sum() / np.maximum(count[req], 1)
        terms = share * (0.1 * np.exp(ref - l64) + np.exp(l64 - old) * np.abs(adv))
        one = np.zeros_like(p64)
        one[np.arange(n)[on], ch[on]] = 1.0
        slack = (terms * 3e-7 * (1.0 + np.abs(l64)))[:, None] * np.abs(one - p64)
        rel = 2e-4 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        big = np.abs(gr).max(axis=1, keepdims=True)
        ok = np.abs(f64(grad) - gr) <= rel * np.abs(gr) + 1e-6 * big + np.where(on[:, None], slack, 0.0)
    assert ok.all(), ((~ok).sum(), np.argwhere(~ok)[:4])
    assert not grad[torch.from_numpy(~on).cuda()].any()
    st2, lp2, _ = B.pr_policy_loss(ctx, xs, to(ch), to(adv), norm=1, want_grad=False, **args, **kw)
    assert torch.equal(st2, stats) and torch.equal(lp2, logp)

    pk = dict(beta=0.3, loss=2, length_norm=True)
    stats, ratio, logp2, pgrad = B.pr_preference_loss(ctx, xs, to(ch), to(off), ref_logp=to(ref),
                                                      mask=to(mask), **pk)
    s, r, l, pr = L.preference(x64, ch, off, ref, mask, **pk)
    check_rows(logp2, l, pgrad, pr, dtype)
    assert (np.abs(f64(ratio) - r) <= 2e-5 * np.maximum(np.diff(off), 1) + 1e-6 * np.abs(r)).all()
    check_stats(stats, s, np.abs(r).max() + 1.0)

    after = buf.clone()
    inplace = after[start:start + n * stride].view(n, stride)[:, :V]
    B.pr_policy_loss(ctx, inplace, to(ch), to(adv), norm=1, grad=inplace, **args, **kw)
    assert torch.equal(inplace, grad)
    inplace.copy_(xs)
    assert torch.equal(after.nan_to_num(nan=7.0), buf.nan_to_num(nan=7.0))  # nothing between the rows


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("n", [40, 700, 5000])
def test_bad_offsets_and_empty_batches_of_every_size(B, ctx, n):
    """Bounds outside the batch and batches of masked rows, however the rows are listed."""
    V = 40
    g, x, x64, ch, old, ref = draw(n, n, V, "f32")
    adv = g.normal(size=n).astype(np.float32)
    B.pr_ctx_flags(ctx, clear=True)
    for off, flag in (([n // 4, n // 2, n - 3], 0), ([0, n // 2, n + 2], B.PR_FLAG_BAD_OFFSETS),
                      ([-3, n // 3, n], B.PR_FLAG_BAD_OFFSETS),
                      ([0, n // 5, n // 5, n], B.PR_FLAG_EMPTY_REQ)):
        for mask in (None, (g.random(n) < 0.7).astype(np.uint8)):
            st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), mask=to(mask),
                                          offsets=to(off, np.int64), norm=1)
            s, lo, go = L.policy(x64, ch, adv, old, None, mask, off, requests=True)
            check_rows(lp, lo, gr, go, "f32")
            check_stats(st, s, 1.0)
            assert B.pr_ctx_flags(ctx, clear=True) == flag
    off = [0, n // 4, n // 2, n // 2, n]
    mask = np.zeros(n, np.uint8)
    for k in range(2):
        st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), mask=to(mask), norm=k,
                                      offsets=to(off, np.int64))
        assert not st.any() and not lp.any() and not gr.any()
    st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to(off, np.int64), mask=to(mask))
    assert not st.any() and not r.any() and not lp.any() and not gr.any()
    # the second pair has one answer: its rows have l, and no gradient
    st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to(off, np.int64), ref_logp=to(ref))
    s, ro, lo, go = L.preference(x64, ch, off, ref)
    check_rows(lp, lo, gr, go, "f32")
    check_stats(st, s, 1.0 + np.abs(ro).max())
    assert not gr[n // 2:].any() and gr[:n // 2].any()
    B.pr_ctx_flags(ctx, clear=True)


@pytest.mark.parametrize("n,stride", [(20, 2 ** 27 + 8), (700, 2 ** 22 + 24)])
def test_rows_past_32_bits(B, ctx, n, stride):
    """Rows that lie more than 2^31 elements apart give the bits of rows side by side."""
    V = 1000
    assert (n - 1) * stride > 2 ** 31
    g, x, _, ch, old, ref = draw(17, n, V, "bf16")
    off = offsets_of(g, n, 6)
    buf = torch.empty((n - 1) * stride + V, dtype=x.dtype, device="cuda")
    out = torch.empty_like(buf)
    far, grad = buf.as_strided((n, V), (stride, 1)), out.as_strided((n, V), (stride, 1))
    far.copy_(x)
    want = B.pr_policy_loss(ctx, x, to(ch), to(old), ref_logp=to(ref), kl_coef=0.1)
    got = B.pr_policy_loss(ctx, far, to(ch), to(old), ref_logp=to(ref), kl_coef=0.1, grad=grad)
    for w, t in zip(want, got):
        assert torch.equal(w, t)
    want = B.pr_preference_loss(ctx, x, to(ch), to(off), ref_logp=to(ref))
    got = B.pr_preference_loss(ctx, far, to(ch), to(off), ref_logp=to(ref), grad=grad)
    for w, t in zip(want, got):
        assert torch.equal(w, t)


def both_losses(B, c, n, V, seed):
    """(a call of both losses into buffers of its own, those buffers) of n rows."""
    g, x, _, ch, old, ref = draw(seed, n, V, "bf16")
    n_req = 2 * (1 + n // 50)
    args = [to(t) for t in (ch, g.normal(size=n).astype(np.float32), old, ref, offsets_of(g, n, n_req))]
    f = dict(device="cuda")
    out = [torch.zeros(6, **f), torch.zeros(n, **f), torch.zeros_like(x), torch.zeros(5, **f),
           torch.zeros(n_req, **f), torch.zeros(n, **f), torch.zeros_like(x)]

    def run():
        chd, adv, oldd, refd, off = args
        B.pr_policy_loss(c, x, chd, adv, old_logp=oldd, ref_logp=refd, offsets=off, kl_coef=0.1,
                         norm=1, stats=out[0], logp=out[1], grad=out[2])
        B.pr_preference_loss(c, x, chd, off, ref_logp=refd, stats=out[3], ratio=out[4],
                             logp=out[5], grad=out[6])

    return run, out


def test_graphs_outlive_larger_calls(B):
    """Batches of growing size, each captured, then run; every graph replayed after all
    of them, while other memory has been taken and filled."""
    c = B.pr_ctx_create(0, 1, 1)
    graphs = []
    for i, n in enumerate((30, 600, 5000, 21000)):
        run, out = both_losses(B, c, n, 200, 30 + i)
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append((graph, out, want, run))  # (the call keeps its inputs)
    other = [torch.full((1 << 22,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]
    for _ in range(2):
        for graph, out, want, _ in graphs:
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(t, w) for t, w in zip(out, want))
    assert all((t == -1).all() for t in other)
    # and calls still give what they gave
    run, out = both_losses(B, c, 600, 200, 31)
    run()
    assert all(torch.equal(t, w) for t, w in zip(out, graphs[1][2]))
    B.pr_ctx_destroy(c)


@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
@pytest.mark.parametrize("n", [30, 900, 6000])
def test_the_first_call_of_a_context_captured(B, ctx, n, mode):
    """A context that has no workspace yet takes it during the capture; so does one whose
    workspace is too small."""
    run, want = both_losses(B, ctx, n, 150, n)
    run()
    torch.cuda.synchronize()
    for first in (0, 10):
        c = B.pr_ctx_create(0, 1, 1)
        if first:
            both_losses(B, c, first, 150, 1)[0]()
        run, out = both_losses(B, c, n, 150, n)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, capture_error_mode=mode):
            run()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(out, want))
        B.pr_ctx_destroy(c)


# one CTA and several to a row, a warp to a row, rows of more than eight SMs
KERNELS = [(6, 300), (5, 151936), (700, 40), (3, 1000003)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", KERNELS)
def test_a_kl_term_of_no_weight_is_no_part_of_the_loss(B, ctx, n, V, dtype):
    """kl_coef 0 with a reference 200 above a row's l, and a masked emitted token."""
    g, x, x64, ch, old, ref = draw(n + V, n, V, dtype)
    ref[1] += 200.0
    x[2, ch[2]] = -torch.inf
    x64 = x.double().cpu().numpy()
    adv = g.normal(size=n).astype(np.float32)
    B.pr_ctx_flags(ctx, clear=True)
    for want_grad in (True, False):
        args = dict(old_logp=to(old), want_grad=want_grad, **CLIP)
        a = B.pr_policy_loss(ctx, x, to(ch), to(adv), **args)
        b = B.pr_policy_loss(ctx, x, to(ch), to(adv), ref_logp=to(ref), **args)
        s, l, gr = L.policy(x64, ch, adv, old, ref, **CLIP)
        assert np.isfinite(s[0]) and not torch.isfinite(b[0][B.PR_POL_KL])
        check_stats(b[0][:2], s[:2], 2.0)
        assert torch.equal(a[0][:2], b[0][:2]) and torch.equal(a[0][3:5], b[0][3:5])
        assert torch.equal(a[1], b[1])
        check_rows(b[1], l, b[2], gr, dtype)
        assert not want_grad or torch.equal(a[2], b[2])
    assert B.pr_ctx_flags(ctx, clear=True) == 0


@pytest.mark.parametrize("n,V", KERNELS)
def test_infinite_means_are_infinite(B, ctx, n, V):
    """Terms beyond single precision (200 above: 7e86) and a token that the policy has
    masked since: the means that they enter are infinite, the others what they are."""
    g, x, x64, ch, old, ref = draw(n + V, n, V, "f32")
    adv = np.abs(g.normal(size=n)).astype(np.float32)

    def check(x, x64, old, ref, adv, infinite):
        for want_grad in (True, False):
            st, lp, _ = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), ref_logp=to(ref),
                                         kl_coef=0.1, want_grad=want_grad, **CLIP)
            s, l, _ = L.policy(x64, ch, adv, old, ref, kl_coef=0.1, **CLIP)
            with np.errstate(over="ignore"):
                s = s.astype(np.float32).astype(np.float64)
            got = f64(st)
            assert [i for i in range(6) if np.isinf(s[i])] == infinite
            assert (got[infinite] == s[infinite]).all(), (got, s)
            rest = [i for i in range(6) if i not in infinite]
            check_stats(st[rest], s[rest], 2.0)
            check_rows(lp, l, None, None, "f32")

    far = ref.copy()
    far[1] += 200.0
    check(x, x64, old, far, adv, [B.PR_POL_LOSS, B.PR_POL_KL])
    far = old.copy()
    far[1] -= 200.0  # clipped: the surrogate stays finite
    check(x, x64, far, ref, adv, [B.PR_POL_RATIO, B.PR_POL_OLD_KL])
    minus = adv.copy()
    minus[1] = -1.0  # not clipped
    check(x, x64, far, ref, minus, [B.PR_POL_LOSS, B.PR_POL_SURROGATE, B.PR_POL_RATIO,
                                    B.PR_POL_OLD_KL])
    x = x.clone()
    x[1, ch[1]] = -torch.inf
    check(x, f64(x), old, None, adv, [B.PR_POL_OLD_KL])
    B.pr_ctx_flags(ctx, clear=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(9, 701), (9, 704), (700, 43), (3, 1000003)])
def test_an_answer_without_a_partner_has_no_gradient(B, ctx, n, V, dtype):
    """NaN and infinities in an answer whose partner is empty or masked: zeros, at the emitted
    token (in the row's words or at its ends) as elsewhere."""
    g, x, _, ch, _, ref = draw(n + V, n, V, dtype)
    m = n // 3
    rows = range(m)
    for t in rows:
        x[t, (7 * t) % V] = (torch.nan, torch.inf)[t % 2]
        ch[t] = (0, V // 2, V - 1)[t % 3]
    x64 = f64(x)
    mask = np.ones(n, np.uint8)
    for off in ([0, 0, m, 2 * m, n], [0, m, m, 2 * m, n], [0, m, n]):
        if len(off) == 3:
            mask[m:] = 0  # the partner's rows are all masked
        st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to(off, np.int64), ref_logp=to(ref),
                                             mask=to(mask))
        s, ro, lo, go = L.preference(x64, ch, off, ref, mask)
        assert torch.isnan(lp[:m]).all() and not gr[:m].any()
        check_rows(lp, lo, gr, go, dtype)
        check_stats(st, s, 1.0 + np.nan_to_num(np.abs(ro)).max())
        assert not torch.isnan(st).any()
    B.pr_ctx_flags(ctx, clear=True)


@pytest.mark.parametrize("n", [40, 700, 5000])
def test_offsets_that_decrease(B, ctx, n):
    """Bounds that overlap: each row counts once, for the same request however large the
    batch, and a request's mean is over the rows that it counts."""
    V = 24
    g, x, x64, ch, old, ref = draw(n, n, V, "f32")
    B.pr_ctx_flags(ctx, clear=True)
    for off in ([0, 6, 3, 10], [0, 10, 3, 6, 10], [4, 10, 2, 1, 8], [0, 12, 3, 6, 10], [10, 6, 3, 0, 0],
                [3, -2, 5, 10, 4]):
        off = [v * n // 10 for v in off]
        n_req = len(off) - 1
        adv = g.normal(size=n_req).astype(np.float32)
        for mask in (None, (g.random(n) < 0.7).astype(np.uint8)):
            for norm in (0, 1):
                kw = dict(per_request=True, **CLIP)
                st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), norm=norm,
                                              mask=to(mask), offsets=to(off, np.int64), **kw)
                s, lo, go = L.policy(x64, ch, adv, old, None, mask, off, requests=bool(norm), **kw)
                check_rows(lp, lo, gr, go, "f32")
                check_stats(st, s, 2.0)
                assert B.pr_ctx_flags(ctx, clear=True) & B.PR_FLAG_BAD_OFFSETS
            if n_req % 2:
                continue
            st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to(off, np.int64), ref_logp=to(ref),
                                                 mask=to(mask), length_norm=True)
            s, ro, lo, go = L.preference(x64, ch, off, ref, mask, length_norm=True)
            check_rows(lp, lo, gr, go, "f32")
            assert (np.abs(f64(r) - ro) <= 2e-5 + 1e-6 * np.abs(ro)).all()
            check_stats(st, s, 1.0 + np.abs(ro).max())
            assert B.pr_ctx_flags(ctx, clear=True) & B.PR_FLAG_BAD_OFFSETS
    # nothing of it is left for the next batch
    off = offsets_of(g, n, 6)
    adv = g.normal(size=6).astype(np.float32)
    kw = dict(per_request=True, **CLIP)
    st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), norm=1,
                                  offsets=to(off), **kw)
    s, lo, go = L.policy(x64, ch, adv, old, None, None, off, requests=True, **kw)
    check_rows(lp, lo, gr, go, "f32")
    check_stats(st, s, 2.0)
    B.pr_ctx_flags(ctx, clear=True)


@pytest.mark.parametrize("n_req", [2, 1024, 3000])
def test_batches_without_rows_report_their_bounds(B, ctx, n_req):
    """Both losses raise the same flags for requests of a batch that has no rows."""
    x = torch.zeros(0, 40, device="cuda")
    ch, f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    B.pr_ctx_flags(ctx, clear=True)
    for last, flags in ((0, B.PR_FLAG_EMPTY_REQ), (3, B.PR_FLAG_EMPTY_REQ | B.PR_FLAG_BAD_OFFSETS)):
        off = np.zeros(n_req + 1, np.int64)
        off[-1] = last
        for norm in (0, 1):
            stats = torch.full((6,), 7.0, device="cuda")
            st, lp, gr = B.pr_policy_loss(ctx, x, ch, f, offsets=to(off), norm=norm, stats=stats)
            assert not st.any() and lp.numel() == 0 and gr.shape == (0, 40)
            assert B.pr_ctx_flags(ctx, clear=True) == flags
        st, r, lp, gr = B.pr_preference_loss(ctx, x, ch, to(off))
        assert not st.any() and not r.any()
        assert B.pr_ctx_flags(ctx, clear=True) == flags
    st = B.pr_policy_loss(ctx, x, ch, f)[0]
    assert not st.any() and B.pr_ctx_flags(ctx, clear=True) == 0


def test_a_batch_without_rows_has_its_own_kernel_times(B):
    c = B.pr_ctx_create(0, 1, 1)
    B.pr_ctx_set_option(c, B.PR_OPT_TIMING, 1)
    g, x, _, ch, old, _ = draw(4, 4, 40, "f32")
    B.pr_policy_loss(c, x, to(ch), to(old))
    assert len(B.pr_ctx_kernel_times(c)) == 1
    B.pr_policy_loss(c, x[:0], to(ch), to(old))
    assert len(B.pr_ctx_kernel_times(c)) == 0
    B.pr_policy_loss(c, x[:0], to(ch), to(old), offsets=to([0, 0], np.int64))
    assert len(B.pr_ctx_kernel_times(c)) == 1
    B.pr_ctx_destroy(c)


@pytest.mark.parametrize("n,V", [(12, 701), (700, 43)])
@pytest.mark.parametrize("kind,smooth", [(0, 0.0), (0, 0.1), (0, 1.0), (1, 0.0), (2, 0.0)])
@pytest.mark.parametrize("side", [0, 1])
def test_masked_emitted_token_in_an_answer(B, ctx, n, V, kind, smooth, side):
    """An answer with a token that the model has masked has the log ratio -inf: the loss of its
    pair is 0 or infinite as the formulas say, and no part of it is 0 times infinity."""
    g, x, _, ch, _, ref = draw(n + V, n, V, "f32")
    off = [0, n // 4, n // 2, 3 * n // 4, n]
    t = off[side] + 1
    x[t, ch[t]] = -torch.inf
    kw = dict(loss=kind, label_smoothing=smooth, beta=0.2)
    st, r, lp, gr = B.pr_preference_loss(ctx, x, to(ch), to(off, np.int64), ref_logp=to(ref), **kw)
    s, ro, lo, go = L.preference(f64(x), ch, off, ref, **kw)
    got = f64(st)
    assert not np.isnan(s[:2]).any() and (got[np.isinf(s)] == s[np.isinf(s)]).all()
    fin = torch.from_numpy(np.isfinite(s))
    check_stats(st.cpu()[fin], s[np.isfinite(s)], 1.0 + 0.2 * np.abs(ro[2:]).max() + (
        (3.0 * np.abs(ro[2:]).max() + 25.0) if kind == 1 else 0.0))
    check_rows(lp, lo, None, None, "f32")
    rest = slice(off[2], n)
    check_rows(lp[rest], lo[rest], gr[rest], go[rest], "f32")
    if kind != 1:  # (the squared loss' slope is infinite)
        check_rows(lp, lo, gr, go, "f32")
    assert B.pr_ctx_flags(ctx, clear=True) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", KERNELS)
def test_no_advantage_under_a_ratio_out_of_range(B, ctx, n, V, dtype):
    """r = e^200 is beyond single precision, and r times an advantage of 0 is 0."""
    g, x, x64, ch, old, ref = draw(n + V, n, V, dtype)
    adv = g.normal(size=n).astype(np.float32)
    adv[1] = 0.0
    old[1] -= 200.0
    for beta, r in ((0.0, None), (0.1, ref)):
        for want_grad in (True, False):
            st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old), ref_logp=to(r),
                                          kl_coef=beta, want_grad=want_grad, **CLIP)
            s, l, go = L.policy(x64, ch, adv, old, r, kl_coef=beta, **CLIP)
            check_rows(lp, l, gr, go, dtype)
            check_stats(st[:3], s[:3], 2.0)
            assert f64(st)[B.PR_POL_RATIO] == np.inf
    assert B.pr_ctx_flags(ctx, clear=True) == 0
    # a row of NaN stays NaN whatever its advantage
    x = x.clone()
    x[1, 0] = torch.nan
    st, lp, gr = B.pr_policy_loss(ctx, x, to(ch), to(adv), old_logp=to(old))
    assert torch.isnan(st[0]) and torch.isnan(gr[1]).all() and torch.isfinite(gr[0]).all()
    assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_NONFINITE


@pytest.mark.parametrize("n,V,dtype", [(2100, 262144, "f32"), (2500, 70001, "bf16"), (900, 70001, "bf16")])
def test_the_policy_loss_alone_repeats(B, ctx, n, V, dtype):
    """Without a gradient the ring's places are filled again while rows are summed: time and again the
    bits of the call with one."""
    gen = torch.Generator("cuda").manual_seed(V)
    x = (3 * torch.randn(n, V, generator=gen, device="cuda")).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    ch = torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32)
    adv = torch.randn(n, generator=gen, device="cuda")
    s, logp, _ = B.pr_policy_loss(ctx, x, ch, adv)
    for _ in range(30):
        s1, logp1, _ = B.pr_policy_loss(ctx, x, ch, adv, want_grad=False)
        assert torch.equal(logp, logp1) and torch.equal(s, s1)
