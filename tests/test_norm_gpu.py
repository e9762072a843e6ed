"""GPU parity of pr_layernorm and pr_layernorm_backward with the float64 oracle.

Tolerances (fp32 rounding 2^-24 = 6e-8; u = half a step of the output's type, 2^-8 relative for bf16):
  moments  sums of d terms in chains of at most 64 registers or d / 256 re-read elements, then
           trees: below 64 roundings or so, 1e-5 of mean |h| (mean) and of the variance
  y        |w| (1e-5 mean|h| rstd + 1e-5 |xhat| + 4e-7 |xhat|) + 4e-7 |b| + u |y|
  dx       rstd (4e-7 (|g| + |mean g| + |xhat mean g xhat|) + 1e-5 (mean |g| + |xhat| mean |g xhat|))
           + 4e-7 |dtotal| + u |dx|; given moments are exact inputs
  dw, db   sums over n rows in chains of up to n / 32 terms, 1e-5 of the sum of magnitudes
"""
import numpy as np
import pytest
import torch

from oracle import distill as D

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


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


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def draw(seed, n, d, dtype, wtype=None, offset=0.3):
    g = torch.Generator().manual_seed(seed)

    def rn(*shape):
        return torch.randn(*shape, generator=g)

    x = (rn(n, d) * (0.2 + 2 * torch.rand(n, 1, generator=g)) + offset * rn(n, 1)).to(TYPES[dtype])
    if d > 3:
        x[:, d // 3] *= 30
    r = (0.5 * rn(n, d)).to(TYPES[dtype])
    w = (1 + 0.3 * rn(d)).to(TYPES[wtype or dtype])
    b = (0.2 * rn(d)).to(TYPES[wtype or dtype])
    dy = rn(n, d).to(TYPES[dtype])
    return [t.cuda() for t in (x, r, w, b, dy)]


def check_forward(got, h, w, b, eps, rms, dtype):
    y, mean, rstd = (f64(t) for t in got)
    h, w, b = f64(h), f64(w), f64(b)
    yo, mo, so = D.norm(h, w, b, eps, rms)
    size = np.abs(h).mean(1)
    if mean is not None:
        assert (np.abs(mean - mo) <= 1e-5 * size + 1e-30).all()
    if rstd is not None:
        assert (np.abs(rstd - so) <= (1e-5 * (1 + (0 if rms else 1) * (1e-5 * size * so) ** 2) + 4e-7) * so).all()
    hat = (h - (0 if rms else mo[:, None])) * so[:, None]
    tol = np.abs(w) * (1e-5 * (size * so)[:, None] + 1.04e-5 * np.abs(hat)) + HALF[dtype] * np.abs(yo)
    tol += 1e-30 + (0 if b is None else 4e-7 * np.abs(b))
    bad = ~(np.abs(y - yo) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], y[bad][:4], yo[bad][:4])


def check_backward(got, dy, h, w, mean, rstd, dtotal, rms, dtype, before=(0.0, 0.0)):
    dx, dw, db = (f64(t) for t in got)
    dy, h, w, mean, rstd, dtotal = (f64(t) for t in (dy, h, w, mean, rstd, dtotal))
    xo, wo, bo = D.norm_backward(dy, h, w, mean, rstd, dtotal, rms)
    hat = (h if rms else h - mean[:, None]) * rstd[:, None]
    g = dy * w
    if dx is not None:
        mg = 0.0 if rms else np.abs(g).mean(1, keepdims=True)
        mh = np.abs(g * hat).mean(1, keepdims=True)
        tol = rstd[:, None] * (1e-6 * np.abs(g) + 1.1e-5 * (mg + np.abs(hat) * mh)) + HALF[dtype] * np.abs(xo)
        tol += 1e-30 + (0 if dtotal is None else 4e-7 * np.abs(dtotal))
        bad = ~(np.abs(dx - xo) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:4], dx[bad][:4], xo[bad][:4])
    for v, want, size, was in ((dw, wo, np.abs(dy * hat).sum(0), before[0]),
                               (db, bo, np.abs(dy).sum(0), before[1])):
        if v is not None:
            bad = ~(np.abs(v - want - was) <= 1e-5 * size + 4e-7 * np.abs(was) + 1e-30)
            assert not bad.any(), (np.flatnonzero(bad)[:4], v[bad][:4], want[bad][:4])


SIZES = [(1, 1), (3, 2), (5, 7), (4, 8), (33, 9), (7, 16), (70, 33), (257, 64), (5, 100), (9, 256),
         (400, 257), (17, 512), (3, 1000), (301, 1024), (30, 1025), (650, 2048), (7, 2056), (40, 3584),
         (5, 3585), (160, 4096), (3, 5000), (330, 7168), (2, 8192), (9, 8200), (3, 12288), (4, 16384), (200, 12001), (160, 16384), (170, 8192), (161, 16000),
         (3, 16385), (2, 16392), (2, 40000), (1, 100003), (320, 4288), (330, 5003), (310, 2501), (152, 6144), (153, 6144)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", SIZES)
def test_forward_sizes(B, ctx, n, d, dtype):
    for i, (rms, bias, res, wtype) in enumerate([(False, True, True, dtype), (True, False, False, "f32"),
                                                 (False, False, False, "bf16"), (True, True, True, "f32")]):
        x, r, w, b, _ = draw(n + 3 * d + i, n, d, dtype, wtype)
        b, r = b if bias else None, r if res else None
        y, total, mean, rstd = B.pr_layernorm(ctx, x, w, bias=b, residual=r, eps=1e-5, rms=rms)
        assert (mean is None) == rms
        h = x
        if res:
            h = (x.float() + r.float()).to(x.dtype)
            assert torch.equal(total, h)
        else:
            assert total is None
        check_forward((y, mean, rstd), h, w, b, 1e-5, rms, dtype)
        y2 = B.pr_layernorm(ctx, x, w, bias=b, residual=r, rms=rms, want_stats=False, want_total=False)
        assert torch.equal(y2[0], y) and y2[1:] == (None, None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", SIZES)
def test_backward_sizes(B, ctx, n, d, dtype):
    for i, (rms, bias, res, wtype) in enumerate([(False, True, True, dtype), (True, False, False, "f32"),
                                                 (False, False, False, "bf16"), (True, True, True, "f32")]):
        x, r, w, _, dy = draw(n + 3 * d + i, n, d, dtype, wtype)
        _, _, mean, rstd = B.pr_layernorm(ctx, x, w, rms=rms)
        dt = r if res else None
        got = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, dtotal=dt, rms=rms, want_dbias=bias)
        check_backward(got, dy, x, w, mean, rstd, dt, rms, dtype)
        # one at a time: the same bits
        only = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, dtotal=dt, rms=rms,
                                       want_dweight=False)
        assert torch.equal(only[0], got[0]) and only[1] is None and only[2] is None
        only = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, rms=rms, want_dx=False,
                                       want_dbias=bias)
        assert only[0] is None and torch.equal(only[1], got[1])
        assert not bias or torch.equal(only[2], got[2])


@pytest.mark.parametrize("n,d", [(1000, 64), (5000, 17), (20000, 1), (9000, 130), (3000, 3584), (100000, 64)])
def test_many_rows(B, ctx, n, d):
    x, _, w, b, dy = draw(d, n, d, "f32")
    y, _, mean, rstd = B.pr_layernorm(ctx, x, w, bias=b)
    check_forward((y, mean, rstd), x, w, b, 1e-5, False, "f32")
    got = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, want_dbias=True)
    check_backward(got, dy, x, w, mean, rstd, None, False, "f32")
    again = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, want_dbias=True)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,stride,start", [(64, 67, 1), (100, 104, 0), (3584, 3592, 8), (3584, 3585, 3),
                                            (20000, 20001, 5), (96, 96, 4)])
def test_strides_and_alignments(B, ctx, d, stride, start, dtype):
    n = 37
    g = torch.Generator().manual_seed(d)

    def rows(k):
        buf = torch.randn(n * (stride + k) + start + k, generator=g).to(TYPES[dtype]).cuda()
        return buf[start + k:].view(n, stride + k)[:, :d]

    x, r, y, total, dy, dx = (rows(k) for k in (0, 1, 2, 0, 3, 8))
    _, _, w, b, _ = draw(1, 1, d, dtype)
    out = B.pr_layernorm(ctx, x, w, bias=b, residual=r, y=y, total=total)
    assert out[0] is y and out[1] is total
    assert torch.equal(total, (x.float() + r.float()).to(x.dtype))
    check_forward((y, out[2], out[3]), total, w, b, 1e-5, False, dtype)
    got = B.pr_layernorm_backward(ctx, dy, total, w, out[3], mean=out[2], dtotal=r, dx=dx, want_dbias=True)
    check_backward(got, dy, total, w, out[2], out[3], r, False, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(40, 64), (600, 3584), (5, 3585), (3, 20000)])
def test_outputs_in_place_of_inputs(B, ctx, n, d, dtype):
    x, r, w, b, dy = draw(5, n, d, dtype)
    y, total, mean, rstd = B.pr_layernorm(ctx, x, w, bias=b, residual=r)
    for how in ("y=x", "y=r"):
        x1, r1 = x.clone(), r.clone()
        ys, ts = (x1, r1) if how == "y=x" else (r1, x1)
        B.pr_layernorm(ctx, x1, w, bias=b, residual=r1, y=ys, total=ts)
        assert torch.equal(ys, y) and torch.equal(ts, total)
    x1 = x.clone()
    assert torch.equal(B.pr_layernorm(ctx, x1, w, bias=b, y=x1)[0], B.pr_layernorm(ctx, x, w, bias=b)[0])
    want = B.pr_layernorm_backward(ctx, dy, total, w, rstd, mean=mean, dtotal=r, want_dbias=True)
    for i in range(3):
        ins = [dy.clone(), total.clone(), r.clone()]
        got = B.pr_layernorm_backward(ctx, ins[0], ins[1], w, rstd, mean=mean, dtotal=ins[2],
                                      dx=ins[i], want_dbias=True)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_bytes_around_the_rows_stay(B, ctx):
    for n, d in ((3, 100), (5, 3584), (2, 20000), (3, 7)):
        for dtype in TYPES.values():
            x = torch.randn(n, d, device="cuda").to(dtype)
            w = torch.ones(d, device="cuda")
            out = torch.full((2, n + 2, d + 8), 7.0, device="cuda", dtype=dtype)
            col = torch.full((2, d + 2), 7.0, device="cuda")
            y, dx = out[0, 1:n + 1, :d], out[1, 1:n + 1, :d]
            _, _, mean, rstd = B.pr_layernorm(ctx, x, w, y=y)
            B.pr_layernorm_backward(ctx, x, x, w, rstd, mean=mean, dx=dx, dweight=col[0, 1:d + 1],
                                    dbias=col[1, 1:d + 1], want_dbias=True)
            y.zero_(), dx.zero_()
            col[:, 1:d + 1] = 0
            assert float(out.float().sum()) == 7.0 * 2 * ((n + 2) * (d + 8) - n * d)
            assert float(col.sum()) == 28.0


def test_values(B, ctx):
    """A constant row has deviation 0 (eps is what is left); NaN and infinity stay in their
    rows, and in the columns' sums; large offsets cost nothing but the offset's own rounding."""
    for d in (64, 3584, 20000):
        x = torch.randn(6, d, device="cuda")
        x[0] = 3.25
        x[1, 5] = torch.nan
        x[2, 7] = torch.inf
        x[3] = 0.0
        x[4] += 4096.0
        w = torch.ones(d, device="cuda")
        y, _, mean, rstd = B.pr_layernorm(ctx, x, w, eps=1e-5)
        assert not y[0].any() and not y[3].any()
        assert y[1].isnan().all() and y[2].isnan().any()
        keep = [0, 3, 4, 5]
        check_forward((y[keep], mean[keep], rstd[keep]), x[keep], w, None, 1e-5, False, "f32")
        dy = torch.randn(6, d, device="cuda")
        dx, dw, db = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, want_dbias=True)
        assert dx[keep].isfinite().all() and dx[1].isnan().all() and dw.isnan().all() and db.isfinite().all()
        check_backward((dx[keep], None, None), dy[keep], x[keep], w, mean[keep], rstd[keep], None, False, "f32")
        y, _, _, rstd = B.pr_layernorm(ctx, x, w, rms=True)
        assert y[1].isnan().all() and rstd[1].isnan() and y[2, 7].isnan() and float(rstd[2]) == 0.0
        check_forward((y[keep], None, rstd[keep]), x[keep], w, None, 1e-5, True, "f32")
        y = B.pr_layernorm(ctx, torch.zeros(2, d, device="cuda"), w, eps=0.0)[0]
        assert y.isnan().all()


@pytest.mark.parametrize("n,d", [(0, 8), (1, 40), (300, 3584), (4, 20000)])
def test_accumulate(B, ctx, n, d):
    x, _, w, _, dy = draw(4, n, d, "bf16")
    _, _, mean, rstd = B.pr_layernorm(ctx, x, w)
    dw, db = torch.randn(2, d, device="cuda").unbind()
    was = f64(dw), f64(db)
    B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, dweight=dw, dbias=db, want_dbias=True,
                            accumulate=True)
    check_backward((None, dw, db), dy, x, w, mean, rstd, None, False, "bf16", was)
    B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, dweight=dw, dbias=db, want_dbias=True)
    check_backward((None, dw, db), dy, x, w, mean, rstd, None, False, "bf16")


def test_gradient_is_the_difference_of_the_norm(B, ctx):
    """Differences of the call itself, fp32: h^2 / 6 of a third derivative of order 1 at h = 2^-6,
    4e-5, and roundings of 1e-5 / h: 2e-3 in all."""
    n, d, h = 3, 40, 2.0 ** -6
    x, _, w, b, dy = draw(8, n, d, "f32", offset=0.0)
    for rms in (False, True):
        def f(v, w_=w, b_=b):
            return (B.pr_layernorm(ctx, v, w_, bias=b_, rms=rms)[0].double() * dy.double()).sum()

        _, _, mean, rstd = B.pr_layernorm(ctx, x, w, bias=b, rms=rms)
        dx, dw, db = B.pr_layernorm_backward(ctx, dy, x, w, rstd, mean=mean, rms=rms, want_dbias=True)
        for i in range(0, d, 7):
            e = torch.zeros(d, device="cuda")
            e[i] = h
            for r in range(n):
                m = torch.zeros_like(x)
                m[r] = e
                assert abs(float((f(x + m) - f(x - m)) / (2 * h)) - float(dx[r, i])) < 2e-3 * (1 + abs(float(dx[r, i])))
            assert abs(float((f(x, w + e) - f(x, w - e)) / (2 * h)) - float(dw[i])) < 2e-3 * (1 + abs(float(dw[i])))
            assert abs(float((f(x, w, b + e) - f(x, w, b - e)) / (2 * h)) - float(db[i])) < 2e-3 * (1 + abs(float(db[i])))


def test_streams_and_graphs(B):
    """Another stream, replays on new data, and graphs that outlive a workspace."""
    ctx = B.pr_ctx_create(0, 1, 1)
    try:
        n, d = 700, 1000
        x, r, w, b, dy = draw(3, n, d, "bf16")
        out = [torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda"),
               torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty(d, device="cuda"),
               torch.empty(d, device="cuda")]

        def both():
            B.pr_layernorm(ctx, x, w, bias=b, residual=r, y=out[0], total=out[1], mean=out[2], rstd=out[3])
            B.pr_layernorm_backward(ctx, dy, out[1], w, out[3], mean=out[2], dx=out[4], dweight=out[5],
                                    dbias=out[6], want_dbias=True)

        s = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):  # the context's first call
            both()
        g.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in out]
        big = draw(4, 3000, 5000, "f32")
        _, _, m, rs = B.pr_layernorm(ctx, big[0], big[2])
        B.pr_layernorm_backward(ctx, big[4], big[0], big[2], rs, mean=m)  # the workspace grows
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, first))
        with torch.cuda.stream(s):
            both()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, first))
        x.copy_(draw(6, n, d, "bf16")[0])
        g.replay()
        check_forward((out[0], out[2], out[3]), (x.float() + r.float()).bfloat16(), w, b, 1e-5, False, "bf16")
        check_backward((out[4], out[5], out[6]), dy, out[1], w, out[2], out[3], None, False, "bf16")
    finally:
        B.pr_ctx_destroy(ctx)


def test_rows_past_32_bits(B, ctx):
    n, d, stride = 3, 1000, (1 << 31) + 24
    x, _, w, b, dy = draw(3, n, d, "bf16")
    far = [torch.as_strided(torch.zeros(2 * stride + d, dtype=torch.bfloat16, device="cuda"), (n, d), (stride, 1))
           for _ in range(3)]
    far[0].copy_(x)
    want = B.pr_layernorm(ctx, x, w, bias=b)
    got = B.pr_layernorm(ctx, far[0], w, bias=b, y=far[1])
    assert all(p is None or torch.equal(p, q) for p, q in zip(want, got))
    far[1].copy_(dy)
    want = B.pr_layernorm_backward(ctx, dy, x, w, want[3], mean=want[2])
    got = B.pr_layernorm_backward(ctx, far[1], far[0], w, got[3], mean=got[2], dx=far[2])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_refusals(B, ctx):
    x, r, w, b, dy = draw(0, 4, 32, "f32")
    mean = rstd = torch.ones(4, device="cuda")
    n0 = B.launch_count()

    def refused(f, *a, **kw):
        with pytest.raises(B.PRError) as e:
            f(ctx, *a, **kw)
        assert e.value.status == B.PR_ERR_INVALID_ARG

    fwd, bwd = B.pr_layernorm, B.pr_layernorm_backward
    for eps in (-1e-5, float("nan"), float("inf")):
        refused(fwd, x, w, eps=eps)
    refused(fwd, x.cpu(), w)
    refused(fwd, x, w.cpu())
    refused(fwd, x, w[:31])
    refused(fwd, x, None)
    refused(fwd, None, w)
    refused(fwd, x, w, bias=b.bfloat16())
    refused(fwd, x, w, bias=b[:31])
    refused(fwd, x[0], w)
    refused(fwd, x.t(), w[:4])
    refused(fwd, x, w, residual=r.bfloat16())
    refused(fwd, x, w, residual=r[:3])
    refused(fwd, x, w, residual=r, y=x, total=x)
    refused(fwd, x, w, y=torch.empty(4, 31, device="cuda"))
    refused(fwd, x, w, mean=torch.empty(3, device="cuda"))
    refused(fwd, x.expand(2, 4, 32)[:, 0], w)  # rows that overlap
    refused(fwd, x.half(), w.half())
    refused(bwd, dy, x, w, rstd)               # no mean
    refused(bwd, dy[:3], x, w, rstd, mean=mean)
    refused(bwd, dy.bfloat16(), x, w, rstd, mean=mean)
    refused(bwd, dy, x, w, rstd[:3], mean=mean)
    refused(bwd, dy, x, w, None, mean=mean)
    refused(bwd, None, x, w, rstd, mean=mean)
    refused(bwd, dy, x, w, rstd, mean=mean, dtotal=r[:, :31])
    refused(bwd, dy, x, w, rstd, mean=mean, want_dx=False, want_dweight=False)
    refused(bwd, dy, x, w, rstd, mean=mean, accumulate=True)
    refused(bwd, dy, x, w, rstd, mean=mean, dweight=torch.empty(31, device="cuda"))
    refused(bwd, dy, x, w, rstd, mean=mean, dx=torch.empty(4, 40, device="cuda")[:, :31])
    big = torch.empty(1, (1 << 20) + 1, device="cuda")
    refused(fwd, big, big[0])
    assert B.launch_count() == n0


@pytest.mark.parametrize("n,d,dtype", [(1217, 4104, "bf16"), (1300, 4111, "bf16"), (1400, 5720, "bf16"),
                                       (1300, 6144, "bf16"), (1217, 2056, "f32"), (1521, 2501, "f32")])
def test_backward_of_many_rows_of_three_words_a_thread(B, ctx, n, d, dtype):
    """513 to 768 words a row, two rows on an SM or one."""
    test_backward_sizes(B, ctx, n, d, dtype)
    test_outputs_in_place_of_inputs(B, ctx, n, d, dtype)


def test_rms_norm_has_no_mean(B, ctx):
    x, r, w, b, _ = draw(3, 5, 96, "f32")
    mean = torch.full((5,), 7.0, device="cuda")
    got = B.pr_layernorm(ctx, x, w, bias=b, rms=True, mean=mean)
    assert got[2] is None and (mean == 7).all()
    check_forward((got[0], None, got[3]), x, w, b, 1e-5, True, "f32")
