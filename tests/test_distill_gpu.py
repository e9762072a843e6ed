"""GPU parity of pr_distill_loss with the float64 oracle, at the sizes, lists, masks and values
where it can go wrong.

Tolerances (2^-24 = 6e-8 per fp32 rounding), relative to the sizes that the oracle gives:
the sums of the magnitudes of a term's parts.
  kl     a log-probability l carries its row's sum of positive fp32 terms, 2e-5 with
         chains of up to 1,000 terms, and a few roundings, 4e-7 |l|; the terms are products of
         those with probabilities: 2e-5 (1 + size) + 1e-6 size
  grad   probabilities are off by the exponent's error of |z - max| 2^-23 and l's, 8e-5
         together, coefficients by a few of those: 2e-4 of the parts' magnitudes; bf16 adds half a
         step, 2^-8; single precision ends at 1e-38; the oracle's coefficient A is a sum of up to 66 fp64
         terms that cancel in the reverse direction and over lists that are all there is: 66 roundings of 2^-53
         of its parts, below 1e-14 of the row's largest
  stats  weighted means: 5e-5 (1 + mean size)
"""
import numpy as np
import pytest
import torch

from oracle import distill as D

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


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


def draw(seed, n, V, k, dtype, scale=3.0, temperature=1.0, near=0.7):
    """(generator, logits, their float64 values, ids, t_logp, labels): the large model's logits are
    the small one's with noise, its list the first k of them, in any order and some absent."""
    g = np.random.Generator(np.random.PCG64(seed))
    x = torch.from_numpy((scale * g.normal(size=(n, V))).astype(np.float32))
    x[torch.arange(n), torch.from_numpy(g.integers(0, V, n))] += 6.0
    x = x.to(TYPES[dtype])
    x64 = x.double().numpy()
    z = (near * x64 + g.normal(size=(n, V))) / temperature
    z -= z.max(1, keepdims=True)
    lp = z - np.log(np.exp(z).sum(1, keepdims=True))
    m = min(k, V)
    ids = np.full((n, k), -1, np.int32)
    ids[:, :m] = np.argpartition(-lp, m - 1, axis=1)[:, :m]
    sent = np.where(ids >= 0, np.take_along_axis(lp, np.maximum(ids, 0), 1), -np.inf).astype(np.float32)
    gone = g.random((n, k)) < 0.1
    ids[gone & (g.random((n, k)) < 0.5)] = -1
    sent[gone] = -np.inf
    ch = np.where(g.random(n) < 0.6, np.where(ids[:, 0] >= 0, ids[:, 0], 0), g.integers(0, V, n))
    return g, x.cuda(), x64, ids, sent, ch.astype(np.int32)


def offsets_of(g, n, n_req):
    cut = np.sort(g.integers(0, n + 1, n_req - 1)) if n_req > 1 else np.zeros(0, np.int64)
    return np.r_[0, cut, n].astype(np.int64)


def check(got, want, mask, dtype, norm_rows=None):
    stats, kl, grad = (None if t is None else t.double().cpu().numpy() for t in got)
    so, ko, go, size, gsize = want
    with np.errstate(invalid="ignore"):
        ok = (np.abs(kl - ko) <= 2e-5 * (1 + size) + 1e-6 * size) | (kl == ko) | (np.isnan(kl) & np.isnan(ko))
        assert ok.all(), ("kl", np.flatnonzero(~ok)[:5], kl[~ok][:5], ko[~ok][:5])
        if grad is not None:
            tol = 2e-4 * gsize + (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(go) + 1e-37
            tol = tol + 1e-14 * gsize.max(axis=1, initial=0.0, keepdims=True)
            ok = (np.abs(grad - go) <= tol) | (np.isnan(grad) & np.isnan(go))
            assert ok.all(), ("grad", (~ok).sum(), np.argwhere(~ok)[:4].tolist(), grad[~ok][:4], go[~ok][:4],
                              tol[~ok][:4])
        s = np.where(np.isfinite(size), size, 0)
        lim = 5e-5 * (1 + s.max(initial=0.0) + np.abs(so))
        ok = (np.abs(stats - so) <= lim) | (stats == so) | (np.isnan(stats) & np.isnan(so))
        assert ok.all(), ("stats", stats, so)


def same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def both(B, ctx, x, x64, ids, sent, ch, mask, off, dtype, **kw):
    norm = kw.pop("norm", 0)
    got = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), mask=to(mask), offsets=to(off),
                            norm=norm, **kw)
    want = D.distill(x64, ids, sent, ch, mask, off, requests=bool(norm), **kw)
    check(got, want, mask, dtype)
    # the loss alone gives the same bits
    alone = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), mask=to(mask), offsets=to(off),
                              norm=norm, want_grad=False, **kw)
    assert alone[2] is None and same(alone[1], got[1]) and same(alone[0], got[0])
    return got, want


SIZES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (5, 8, 8), (4, 9, 12), (7, 31, 31), (9, 33, 40), (6, 255, 64),
         (3, 1000, 20), (37, 1001, 64), (200, 515, 33), (2, 4096, 1), (3, 8191, 32), (3, 16384, 20),
         (5, 32000, 16), (2, 32003, 50), (170, 2050, 20), (2, 70001, 64), (3, 151936, 32), (2, 262144, 64),
         (1, 393216, 20), (700, 4001, 17), (700, 5000, 64), (640, 12480, 20), (620, 24577, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,k", SIZES)
def test_sizes(B, ctx, n, V, k, dtype):
    T = 1.0 if V % 2 else 0.8
    g, x, x64, ids, sent, ch = draw(V * 7 + n, n, V, k, dtype, temperature=T)
    off = offsets_of(g, n, min(n, 5))
    mask = (g.random(n) < 0.8).astype(np.uint8)
    B.pr_ctx_flags(ctx, clear=True)
    for loss, rest, ce in ((0, 0, 0.0), (1, 0, 0.3), (0, 1, 0.5), (1, 1, 0.0)):
        both(B, ctx, x, x64, ids, sent, ch if ce else None, mask, off, dtype, loss=loss, rest=rest,
             kl_coef=0.8, ce_coef=ce, temperature=T, norm=(n + loss) % 2, grad_scale=1.5)
    assert B.pr_ctx_flags(ctx, clear=True) & ~B.PR_FLAG_EMPTY_REQ == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(24, 40), (24, 1003), (24, 40000), (620, 1003)])
def test_values_that_a_row_can_hold(B, ctx, n, V, dtype):
    """Masked tokens in and out of the list, the type's lowest value, large logits, NaN and
    infinities, in counted and in masked rows."""
    k = 10
    g, x, x64, ids, sent, ch = draw(V, n, V, k, dtype)
    low = torch.finfo(x.dtype).min
    mask = np.ones(n, np.uint8)
    ids[:, 0], ids[:, 1] = 0, V - 1                     # the row's ends are listed
    ids[:, 2:] = 1 + (np.arange(k - 2)[None] * (V // 12) + np.arange(n)[:, None]) % (V - 2)
    sent = np.log(g.dirichlet(np.ones(k + 1), n)[:, :k]).astype(np.float32)
    ch[:] = ids[:, 3]
    ch[::3] = V - 2
    ids_t = torch.from_numpy(ids).long().cuda()
    x[0, : V // 2] = -torch.inf
    x[1] = -torch.inf                                   # nothing left
    x[2] = low                                          # nothing left either
    x[3] = x[3].scatter(0, ids_t[3], 3.0 + torch.zeros(k, device="cuda", dtype=x.dtype))
    x[4, 3] = torch.nan
    x[5, V // 2] = torch.inf
    x[6] = 3e4 + x[6]                                   # large logits
    keep = x[7].gather(0, ids_t[7])
    x[7] = -torch.inf
    x[7] = x[7].scatter(0, ids_t[7], keep)              # the list alone is left
    keep = x[8].gather(0, ids_t[8])
    x[8] = low
    x[8] = x[8].scatter(0, ids_t[8], keep)              # the same, masked by the lowest value
    x[9] = x[9].scatter(0, ids_t[9], torch.full((k,), -torch.inf, device="cuda", dtype=x.dtype))
    x[10, 0] = -torch.inf                               # a listed token is masked
    x[11, V - 1] = low
    x[12], x[13], x[14] = torch.nan, torch.inf, -torch.inf   # rows that do not count
    mask[12:15] = 0
    ids[12, 0], ch[13] = V + 7, -9
    x[15, 0] = torch.nan                                # in a listed place
    x[16, V - 1] = torch.inf
    ids[17, 4] = V                                      # outside the vocabulary
    ids[18, 4] = -2
    ids[19, 5] = ids[19, 6]                             # listed twice
    sent[20, 2], sent[21, 2] = np.nan, np.inf
    ids[22] = -1                                        # no list
    sent[23] = -np.inf
    x64 = x.double().cpu().numpy()
    nan_rows = [1, 2, 4, 5, 15, 16, 17, 18, 19, 20, 21]
    for loss, rest in ((0, 0), (1, 0), (0, 1), (1, 1)):
        for label in (None, ch):
            kw = dict(loss=loss, rest=rest, ce_coef=0.0 if label is None else 0.2)
            B.pr_ctx_flags(ctx, clear=True)
            got, want = both(B, ctx, x, x64, ids, sent, label, mask, None, dtype, **kw)
            assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_NONFINITE | B.PR_FLAG_BAD_CHOSEN
            assert got[1][nan_rows].isnan().all() and not got[2][12:15].any() and not got[1][12:15].any()
            # without the rows that are NaN by right nothing is
            some = mask.copy()
            some[nan_rows + ([9] if loss and rest else [])] = 0
            got, want = both(B, ctx, x, x64, ids, sent, label, some, [0, 4, 9, n], dtype, norm=1, **kw)
            assert not got[2].isnan().any() and not got[0].isnan().any()
            assert B.pr_ctx_flags(ctx, clear=True) == 0


def vectorised(x, ids, sent, mask, reverse):
    """The oracle's (KL, gradient, and what roundings of it are relative to) in torch, fp64, for batches of
    whole rows: a class of the rest, no labels, mean over the counted rows."""
    z = x.double()
    l = z - torch.logsumexp(z, 1, keepdim=True)
    on = (ids >= 0) & (sent > -torch.inf)
    at = torch.where(on, ids, ids.new_tensor(0)).long()
    p = torch.where(on, sent.double().exp(), 0.0)
    t = torch.where(on, sent.double(), 0.0)
    ls = torch.where(on, l.gather(1, at), 0.0)
    out = torch.ones_like(l, dtype=torch.bool)
    r, j = torch.nonzero(on, as_tuple=True)
    out[r, at[r, j]] = False
    l_sigma = torch.logsumexp(l.masked_fill(~out, -torch.inf), 1)
    sigma, rho = l_sigma.exp(), (1 - p.sum(1)).clamp(min=2.0 ** -24)
    if not reverse:
        kl = (p * (t - ls)).sum(1) + rho * (rho.log() - l_sigma)
        a, b = -p, -rho
        size_a, size_b = p, rho
    else:
        q = torch.where(on, ls.exp(), 0.0)
        kl = (q * (ls - t)).sum(1) + sigma * (l_sigma - rho.log())
        a, b = q * (ls - t - kl[:, None]), sigma * (l_sigma - rho.log() - kl)
        size_a = q * (1 + (ls - t).abs() + kl.abs()[:, None] + t.abs())
        size_b = sigma * (1 + l_sigma.abs() + 2 * rho.log().abs() + kl.abs())
    A = a.sum(1) + b
    w = mask.double() / mask.sum()
    g = l.exp() * torch.where(out, (b / sigma - A)[:, None], -A[:, None])
    size = l.exp() * torch.where(out, (size_b / sigma + A.abs())[:, None], A.abs()[:, None])
    g[r, at[r, j]] += a[r, j]
    size[r, at[r, j]] += size_a[r, j]
    return torch.where(mask.bool(), kl, 0.0), g * w[:, None], size * w[:, None]


@pytest.mark.parametrize("n,V,k,dtype", [(600, 151936, 32, "bf16"), (560, 262144, 64, "f32"), (1200, 70001, 50, "bf16"),
                                         (900, 32000, 64, "f32"), (540, 393216, 20, "f32")])
def test_large_batches_of_long_rows(B, ctx, n, V, k, dtype):
    """The launches that fill the GPU: rows over clusters of every size, lists prepared ahead, with
    and without a gradient and in place of the logits.  Against fp64 on the GPU."""
    gen = torch.Generator("cuda").manual_seed(V)
    x = (3 * torch.randn(n, V, generator=gen, device="cuda")).to(TYPES[dtype])
    teacher = (0.8 * x.float() + torch.randn(n, V, generator=gen, device="cuda")).to(TYPES[dtype])
    ids, sent = B.pr_top_logits(ctx, teacher, k)
    del teacher
    ids[::3, -1] = -1
    mask = (torch.rand(n, generator=gen, device="cuda") < 0.85).to(torch.uint8)
    for reverse in (False, True):
        kw = dict(mask=mask, loss=int(reverse))
        s, kl, g = B.pr_distill_loss(ctx, x, ids, sent, **kw)
        s1, kl1, _ = B.pr_distill_loss(ctx, x, ids, sent, want_grad=False, **kw)
        assert torch.equal(s, s1) and torch.equal(kl, kl1)
        y = x.clone()
        B.pr_distill_loss(ctx, y, ids, sent, grad=y, **kw)
        assert torch.equal(y, g)
        del y
        for a in range(0, n, 150):   # 150 rows at a time; the mean is over all counted rows
            b = min(n, a + 150)
            want, gw, size = vectorised(x[a:b], ids[a:b], sent[a:b], mask[a:b], reverse)
            share = float(mask[a:b].sum()) / float(mask.sum())
            assert ((kl[a:b].double() - want).abs() <= 4e-5 * (1 + want.abs())).all()
            tol = 2e-4 * size * share + (2.0 ** -8 if dtype == "bf16" else 0) * gw.abs() * share + 1e-37
            tol += 1e-14 * (size * share).amax(1, keepdim=True)
            assert ((g[a:b].double() - gw * share).abs() <= tol).all()


@pytest.mark.parametrize("n,V,k,dtype", [(2100, 262144, 64, "f32"), (2500, 70001, 64, "bf16"), (3000, 9000, 64, "f32")])
def test_the_loss_alone_repeats(B, ctx, n, V, k, dtype):
    """Places of the ring are filled again right after their listed tokens were left out: time and
    again the bits of the call with a gradient."""
    gen = torch.Generator("cuda").manual_seed(V)
    x = (3 * torch.randn(n, V, generator=gen, device="cuda")).to(TYPES[dtype])
    ids, sent = B.pr_top_logits(ctx, 1.1 * x.float() + torch.randn(n, V, generator=gen, device="cuda"), k)
    s, kl, g = B.pr_distill_loss(ctx, x, ids, sent)
    for _ in range(30):
        s1, kl1, _ = B.pr_distill_loss(ctx, x, ids, sent, want_grad=False)
        assert torch.equal(kl, kl1) and torch.equal(s, s1)
    for _ in range(5):
        g1 = B.pr_distill_loss(ctx, x, ids, sent)[2]
        assert torch.equal(g, g1)


def test_small_rests_and_sure_rows_keep_their_digits(B, ctx):
    """A rest of 1e-9 of the mass, and a label whose probability is 1 - 1e-6: gradients and
    divergences to 2e-3 of themselves (the exponents' error of 30 x 2^-23 in sums of few terms)."""
    V, k = 5000, 8
    x = torch.full((2, V), -30.0, device="cuda")
    x += torch.rand(2, V, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    x[:, :k] = torch.arange(k, device="cuda") / 4
    x[1, 3] = 16.0
    x64 = x.double().cpu().numpy()
    ids = np.tile(np.arange(k, dtype=np.int32), (2, 1))
    p = np.exp(x64[:, :k] - x64[:, :k].max(1, keepdims=True))
    sent = np.log(p / p.sum(1, keepdims=True) * (1 - 1e-3)).astype(np.float32)
    ch = np.array([0, 3], np.int32)
    for kw in (dict(), dict(loss=1), dict(kl_coef=0.0, ce_coef=1.0)):
        s, kl, g = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), **kw)
        so, ko, go, _, _ = D.distill(x64, ids, sent, ch, **kw)
        assert np.abs(kl.double().cpu().numpy() / ko - 1).max() < 2e-3
        big = np.abs(go[:, k:]).max(1, keepdims=True)
        assert (np.abs(g.double().cpu().numpy() - go)[:, k:] <= 2e-3 * np.abs(go[:, k:]) + 1e-6 * big).all()
        if "kl_coef" in kw:
            assert np.abs(g.double().cpu().numpy()[1, :k] / go[1, :k] - 1).max() < 2e-3


@pytest.mark.parametrize("n,V", [(40, 30000), (900, 3000)])
@pytest.mark.parametrize("loss", [0, 1])
def test_lists_that_hold_little_of_a_row(B, ctx, n, V, loss):
    """Soft rows whose lists hold 1e-4 to 1e-2 of the mass.  Exponentials are within 2^-22 and their
    exponents of up to 30 within 30 x 2^-24, so probabilities and listed masses are within 2e-6 of
    themselves and log q within 2e-6: KL, a sum of P (log p - log q) and of logarithms of 1 - P
    and 1 - E, within 4e-6 (P + E); the rest's factor b - A sigma, a difference of E's and P's
    multiples (forward) or of the two logarithms, within as much, and its q within 4e-6."""
    T, k = 8.0, 3
    gen = torch.Generator("cuda").manual_seed(V + loss)
    x = 3 * torch.randn(n, V, generator=gen, device="cuda")
    ids, sent = B.pr_top_logits(ctx, 1.1 * x + torch.randn(n, V, generator=gen, device="cuda"), k, temperature=T)
    _, kl, grad = B.pr_distill_loss(ctx, x, ids, sent, temperature=T, loss=loss, grad_scale=float(n))
    lq = torch.log_softmax(x.double() / T, 1)
    at, q = ids.long(), lq.exp()
    l, t = lq.gather(1, at), sent.double()
    P, E = t.exp().sum(1), l.exp().sum(1)
    l_rho, l_sigma = torch.log1p(-P), torch.log1p(-E)
    if loss == 0:
        want = (t.exp() * (t - l)).sum(1) + (1 - P) * (l_rho - l_sigma)
        a, b = -t.exp(), P - 1
    else:
        want = (l.exp() * (l - t)).sum(1) + (1 - E) * (l_sigma - l_rho)
        a, b = l.exp() * (l - t - want[:, None]), (1 - E) * (l_sigma - l_rho - want)
    assert ((kl.double() - want).abs() <= 4e-6 * (P + E)).all()
    A, sigma = a.sum(1) + b, 1 - E
    g = q * ((b - A * sigma) / sigma)[:, None]
    tol = q * (8e-6 * (P + E) / sigma)[:, None]
    g.scatter_(1, at, a - A[:, None] * l.exp())
    # (reverse: a sums k terms with log q - log p, here below 4 in size)
    tol.scatter_(1, at, 4e-6 * (5 if loss else 1) * (l.exp() + t.exp()))
    assert ((grad.double() * T - g).abs() <= tol + 2. ** -23 * g.abs()).all()


def test_one_listed_token_is_the_whole_distribution(B, ctx):
    gen = torch.Generator("cuda").manual_seed(6)
    for n, V in ((6, 50000), (700, 4001)):
        x = 20 * torch.randn(n, V, generator=gen, device="cuda")
        ids, sent = B.pr_top_logits(ctx, x + torch.randn(n, V, generator=gen, device="cuda"), 1, temperature=0.7)
        _, kl, grad = B.pr_distill_loss(ctx, x, ids, sent, temperature=0.7, loss=B.PR_DISTILL_REVERSE,
                                        rest=B.PR_REST_NONE)
        assert (kl == 0).all() and (grad == 0).all()


def test_coefficients_of_nothing(B, ctx):
    """A term of coefficient 0 is a statistic alone, even an infinite one."""
    n, V, k = 6, 300, 5
    g, x, x64, ids, sent, ch = draw(3, n, V, k, "f32")
    ids[:], sent[:] = np.arange(k), np.log(0.15)
    ch[:] = 50
    x[:, 1] = -torch.inf      # listed: KL infinite
    x64 = x.double().cpu().numpy()
    got, _ = both(B, ctx, x, x64, ids, sent, ch, None, None, "f32", kl_coef=0.0, ce_coef=0.7)
    assert got[0][B.PR_DIS_LOSS].isfinite() and got[0][B.PR_DIS_KL].isinf() and got[1].isinf().all()
    x[:, 1], x[:, 50] = 0.0, -torch.inf   # the label: CE infinite
    x64 = x.double().cpu().numpy()
    got, _ = both(B, ctx, x, x64, ids, sent, ch, None, None, "f32", kl_coef=1.0, ce_coef=0.0)
    assert got[0][B.PR_DIS_LOSS].isfinite() and got[0][B.PR_DIS_CE].isinf() and got[2].isfinite().all()
    got, _ = both(B, ctx, x, x64, ids, sent, ch, None, None, "f32", kl_coef=0.0, ce_coef=0.0)
    assert not got[2].any() and float(got[0][B.PR_DIS_LOSS]) == 0.0
    got, _ = both(B, ctx, x, x64, ids, sent, ch, None, None, "f32", grad_scale=0.0)
    assert not got[2].any()


@pytest.mark.parametrize("rest", [0, 1])
def test_logits_as_lists(B, ctx, rest):
    """A constant drops out of lists that are the whole distribution."""
    n, V, k = 5, 400, 12
    g, x, x64, ids, sent, ch = draw(4, n, V, k, "f32")
    s, kl, grad = B.pr_distill_loss(ctx, x, to(ids), to(sent), rest=B.PR_REST_NONE)
    s2, kl2, grad2 = B.pr_distill_loss(ctx, x, to(ids), to(sent + np.float32(8.0)), rest=B.PR_REST_NONE)
    # (8 takes up to two bits of the sent values)
    assert (kl - kl2).abs().max() < 2e-5 and (grad - grad2).abs().max() < 2e-5
    check((s2, kl2, grad2), D.distill(x64, ids, sent + np.float32(8.0), rest=1), None, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,stride,start,gstride,gstart", [
    (1000, 1003, 1, 1000, 0), (5001, 5001, 3, 5001, 3), (777, 1024, 0, 800, 8),
    (32000, 32001, 5, 32001, 5), (40001, 40008, 8, 40008, 8), (9, 11, 2, 10, 1)])
def test_strides_and_alignments(B, ctx, V, stride, start, gstride, gstart, dtype):
    for n in (3, 700):
        if n * stride > 2e6:
            continue
        k = min(20, V)
        g, xs, x64, ids, sent, ch = draw(V, n, V, k, dtype)
        buf = torch.zeros(start + n * stride + 8, dtype=xs.dtype, device="cuda")
        x = buf[start:start + n * stride].view(n, stride)
        x[:, :V] = xs
        gbuf = torch.full((gstart + n * gstride + 8,), 7.0, dtype=xs.dtype, device="cuda")
        grad = gbuf[gstart:gstart + n * gstride].view(n, gstride)
        mask = (g.random(n) < 0.7).astype(np.uint8)
        got = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), mask=to(mask), ce_coef=0.1,
                                grad=grad, vocab=V)
        want = D.distill(x64, ids, sent, ch, mask, ce_coef=0.1)
        check((got[0], got[1], grad[:, :V]), want, mask, dtype)
        grad[:, :V] = 0
        assert float(gbuf.float().sum()) == 7.0 * (gbuf.numel() - n * V)  # the rest is as it was


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(5, 100), (700, 1001), (9, 32003), (300, 40000), (3, 262144)])
def test_gradient_in_place_of_the_logits(B, ctx, n, V, dtype):
    g, x, x64, ids, sent, ch = draw(n, n, V, 16, dtype)
    mask = (g.random(n) < 0.7).astype(np.uint8)
    kw = dict(chosen=to(ch), mask=to(mask), ce_coef=0.2, loss=1)
    s, kl, grad = B.pr_distill_loss(ctx, x, to(ids), to(sent), **kw)
    s1, kl1, g1 = B.pr_distill_loss(ctx, x, to(ids), to(sent), grad=x, **kw)
    assert g1 is x and torch.equal(g1, grad) and torch.equal(kl, kl1) and torch.equal(s, s1)


def test_gradient_is_the_difference_of_the_loss(B, ctx):
    """Differences of the call's own loss: step 2^-5, whose h^2 / 6 is 2e-4, and roundings of the
    loss of 1e-6 / h: 4e-5; the gradients are of order 1 / n = 0.2."""
    n, V, k, h = 5, 60, 9, 2.0 ** -5
    g, x, x64, ids, sent, ch = draw(6, n, V, k, "f32", scale=1.5)
    for loss, rest in ((0, 0), (1, 0), (0, 1), (1, 1)):
        kw = dict(chosen=to(ch), loss=loss, rest=rest, ce_coef=0.3)
        grad = B.pr_distill_loss(ctx, x, to(ids), to(sent), **kw)[2]
        worst = 0.0
        for v in range(V):
            ks = []
            for sign in (1, -1):
                y = x.clone()
                y[:, v] += sign * h
                # rows one by one: their own loss
                ks.append(torch.stack([B.pr_distill_loss(
                    ctx, y[t:t + 1], to(ids[t:t + 1]), to(sent[t:t + 1]), **{**kw, "chosen": to(ch[t:t + 1])},
                    want_grad=False)[0][0] for t in range(n)]).double())
            d = (ks[0] - ks[1]) / (2 * h) / n
            worst = max(worst, float((d - grad[:, v].double()).abs().max()))
        assert worst < 3e-4, worst


def test_what_top_logits_gives_is_a_list(B, ctx):
    """The calls as they are used together: the large model's rows listed, the small one's trained
    on them; a model distilled from itself has no divergence and no gradient."""
    g, x, x64, _, _, ch = draw(9, 60, 3000, 5, "bf16")
    for k in (20, 64):
        for loss in (0, 1):
            for T in (1.0, 2.0):
                ids, logp = B.pr_top_logits(ctx, x, k, temperature=T)
                s, kl, grad = B.pr_distill_loss(ctx, x, ids, logp, loss=loss, temperature=T)
                # l and t_logp are each off by 2e-5 + 4e-7 |l| at worst
                assert kl.abs().max() < 6e-5 and grad.abs().max() < 6e-5 / 60
                other = (x.float() + torch.randn(x.shape, device="cuda")).bfloat16()
                got = B.pr_distill_loss(ctx, other, ids, logp, loss=loss, temperature=T)
                check(got, D.distill(other.double().cpu().numpy(), ids.cpu().numpy(), logp.cpu().numpy(),
                                     loss=loss, temperature=T), None, "bf16")


def test_batches_without_a_counted_row(B, ctx):
    for n, V in ((4, 100), (3, 40000), (800, 1000)):
        g, x, x64, ids, sent, ch = draw(1, n, V, 8, "f32")
        x[0] = torch.nan
        B.pr_ctx_flags(ctx, clear=True)
        s, kl, grad = B.pr_distill_loss(ctx, x, to(ids), to(sent), mask=to(np.zeros(n, np.uint8)))
        assert not s.any() and not kl.any() and not grad.any()
        s, kl, grad = B.pr_distill_loss(ctx, x, to(ids), to(sent), offsets=to([0, 0, 0], np.int64), norm=1)
        assert not s.any() and not kl.any() and not grad.any()
        assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_EMPTY_REQ
    s, kl, grad = B.pr_distill_loss(ctx, x[:0], to(ids[:0]), to(sent[:0]))
    assert not s.any() and kl.numel() == 0 and grad.shape == (0, 1000)
    B.pr_distill_loss(ctx, x[:0], to(ids[:0]), to(sent[:0]), offsets=to([0, 1], np.int64))
    assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_BAD_OFFSETS


def test_bad_offsets(B, ctx):
    for n in (10, 700):
        g, x, x64, ids, sent, ch = draw(2, n, 500, 8, "f32")
        for off in ([0, 4, 2, n], [-1, 5, n], [0, 5, n + 3], [3, 3, 9, n]):
            off = np.array(off, np.int64)
            got = B.pr_distill_loss(ctx, x, to(ids), to(sent), offsets=to(off), norm=1)
            check(got, D.distill(x64, ids, sent, None, None, off, requests=True), None, "f32")
    assert B.pr_ctx_flags(ctx, clear=True) & B.PR_FLAG_BAD_OFFSETS


def test_results_repeat_on_other_streams_and_in_graphs(B):
    ctx = B.pr_ctx_create(0, 1, 1)
    try:
        for n, V in ((40, 9000), (900, 2000), (6, 151936)):
            g, x, x64, ids, sent, ch = draw(n, n, V, 20, "bf16")
            mask = to((g.random(n) < 0.8).astype(np.uint8))
            ids_t, sent_t = to(ids), to(sent)
            out = dict(stats=torch.empty(5, device="cuda"), kl=torch.empty(n, device="cuda"),
                       grad=torch.empty_like(x))
            s = torch.cuda.Stream()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):  # at first the context's first call
                B.pr_distill_loss(ctx, x, ids_t, sent_t, mask=mask, **out)
            graph.replay()
            torch.cuda.synchronize()
            first = {q: t.clone() for q, t in out.items()}
            for _ in range(3):
                B.pr_distill_loss(ctx, x, ids_t, sent_t, mask=mask, **out)
                assert all(torch.equal(t, first[q]) for q, t in out.items())
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                B.pr_distill_loss(ctx, x, ids_t, sent_t, mask=mask, **out)
            torch.cuda.synchronize()
            assert all(torch.equal(t, first[q]) for q, t in out.items())
            _, y, y64, ids2, sent2, _ = draw(n + 1, n, V, 20, "bf16")
            x.copy_(y), ids_t.copy_(to(ids2)), sent_t.copy_(to(sent2))
            graph.replay()
            check((out["stats"], out["kl"], out["grad"]),
                  D.distill(y64, ids2, sent2, None, mask.cpu().numpy()), None, "bf16")
    finally:
        B.pr_ctx_destroy(ctx)


def test_rows_past_32_bits(B, ctx):
    n, V, stride = 3, 900, (1 << 31) + 24
    g, xs, x64, ids, sent, ch = draw(9, n, V, 20, "bf16")
    far = [torch.as_strided(torch.zeros(2 * stride + V, dtype=torch.bfloat16, device="cuda"), (n, V), (stride, 1))
           for _ in range(2)]
    far[0].copy_(xs)
    want = B.pr_distill_loss(ctx, xs, to(ids), to(sent), chosen=to(ch), ce_coef=0.3)
    got = B.pr_distill_loss(ctx, far[0], to(ids), to(sent), chosen=to(ch), ce_coef=0.3, grad=far[1])
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_refusals(B, ctx):
    g, x, x64, ids, sent, ch = draw(0, 4, 100, 6, "f32")
    i, s, c = to(ids), to(sent), to(ch)
    n0 = B.launch_count()

    def refused(*a, **kw):
        with pytest.raises(B.PRError) as e:
            B.pr_distill_loss(ctx, *a, **kw)
        assert e.value.status == B.PR_ERR_INVALID_ARG

    for T in (0.0, -1.0, 1e-4, 2e3, float("nan")):
        refused(x, i, s, temperature=T)
    for bad in (-0.1, float("nan"), float("inf")):
        refused(x, i, s, kl_coef=bad)
        refused(x, i, s, chosen=c, ce_coef=bad)
    refused(x, i, s, ce_coef=0.5)              # no labels
    refused(x, i, s, grad_scale=float("inf"))
    refused(x, i, s, loss=2)
    refused(x, i, s, rest=2)
    refused(x, i, s, norm=2)
    refused(x.cpu(), i, s)
    refused(x, i.cpu(), s)
    refused(x, i.long(), s)
    refused(x, i, s.double())
    refused(x, i[:3], s)
    refused(x, i, s[:, :5])
    refused(x, i[:, :5], s[:, :5])             # not contiguous
    refused(x, i[:, :0], s[:, :0])
    refused(x, i[0], s[0])
    wide = torch.zeros(4, 65, dtype=torch.int32, device="cuda")
    refused(x, wide, wide.float())
    refused(x, i, s, chosen=c[:3])
    refused(x, i, s, mask=torch.ones(3, dtype=torch.uint8, device="cuda"))
    refused(x, i, s, offsets=torch.zeros(1, dtype=torch.int64, device="cuda"))
    refused(x, i, s, grad=torch.empty(4, 100, dtype=torch.bfloat16, device="cuda"))
    refused(x, i, s, grad=torch.empty(4, 99, device="cuda"))
    refused(x, i, s, kl=torch.empty(3, device="cuda"))
    refused(x, i, s, stats=torch.empty(4, device="cuda"))
    refused(x, i, s, vocab=101)
    big = torch.empty(4, B.PR_DISTILL_MAX_VOCAB + 1, device="cuda")
    refused(big, i, s)
    assert B.launch_count() == n0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(6, 20001), (6, 150000), (640, 20001), (700, 3001)])
@pytest.mark.parametrize("rise", [40.0, 66.0])
def test_gradients_of_rows_that_rise(B, ctx, n, V, rise, dtype):
    """Logits that rise along the row: the sum is against a reference far below the largest, up to
    1e30, and the gradient's factor, a weight over that sum, is to keep its digits all the same.
    Gradients of down to 1e-27 of the ordinary, to `check`'s tolerance of each row's own size."""
    k = 5
    g = np.random.Generator(np.random.PCG64(V + n))
    x = np.linspace(-rise, 0.0, V)[None] + 0.2 * g.normal(size=(n, V))
    x = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])
    x64 = x.double().numpy()
    x = x.cuda()
    ids = np.stack([g.permutation(V // 2)[:k] for _ in range(n)]).astype(np.int32)
    sent = np.log(g.dirichlet(np.ones(k + 1), n)[:, :k]).astype(np.float32)
    ch = g.integers(0, V, n).astype(np.int32)
    for scale in (1.0, 1e-7, 1e-12, 1e-20):
        for loss in (0, 1):
            kw = dict(loss=loss, ce_coef=0.3, grad_scale=scale * n)
            got = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), **kw)
            want = D.distill(x64, ids, sent, ch, **kw)
            grad, go, size = got[2].double().cpu().numpy(), want[2], want[4]
            tol = 2e-4 * size + (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(go) + 1e-37
            tol += 1e-14 * size.max(axis=1, keepdims=True)
            bad = ~(np.abs(grad - go) <= tol)
            assert not bad.any(), (scale, loss, bad.sum(), grad[bad][:4], go[bad][:4], tol[bad][:4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(5, 7), (6, 1003), (6, 40000), (700, 1003), (620, 12011)])
def test_masks_of_any_size(B, ctx, n, V, dtype):
    """What is masked by a large negative number is no part of a row, at any temperature: also where
    nothing else is near."""
    k = 4
    g, x0, _, ids, sent, ch = draw(V, n, V, k, dtype)
    r = np.random.Generator(np.random.PCG64(V))
    hide = r.random((n, V)) < 0.97
    hide[0, : V - 2], hide[1, 2:] = True, True
    hide[0, V - 2:], hide[1, :2], hide[2:, V // 2] = False, False, False
    ch = np.where(np.arange(n) == 0, V - 1, np.where(np.arange(n) == 1, 0, V // 2)).astype(np.int32)
    hide_t = to(hide)
    for low in ("lowest", -1e38, -2.3e38, -1e30, -7e20, -1e12, -6e9):
        x = x0.masked_fill(hide_t, torch.finfo(x0.dtype).min if low == "lowest" else low)
        x64 = x.double().cpu().numpy()
        for T, loss, rest in ((1.0, 0, 0), (1.7, 1, 0), (2.0, 0, 1), (5.0, 0, 0), (5.0, 1, 1)):
            B.pr_ctx_flags(ctx, clear=True)
            some = None
            if loss and rest:  # a row whose whole list is masked is NaN by right
                at = np.maximum(ids, 0)
                listed = (ids >= 0) & (sent > -np.inf)
                left = (listed & (np.take_along_axis(x64, at, 1) > -1e9 * T)).any(1) | ~listed.any(1)
                some = left.astype(np.uint8)
            got, want = both(B, ctx, x, x64, ids, sent, ch, some, None, dtype, loss=loss, rest=rest,
                             temperature=T, ce_coef=0.2)
            assert not got[1].isnan().any() and not got[2].isnan().any(), (low, T, loss, rest)
            assert B.pr_ctx_flags(ctx, clear=True) == 0
