"""GPU parity of pr_top_logits with the float64 oracle, at the sizes, ties and values where a
selection can go wrong.  Tokens have to be the oracle's, one by one.  Log-probabilities: a
row's sum of positive fp32 terms, each off by 2^-22 and by |z - max| 2^-23 (weighted by
the term itself: below 1e-6), in chains of up to 1,000 terms (6e-5 at worst, the roundings'
mean far less): 2e-5; the roundings of the difference and of its product: 4e-7 |l|."""
import numpy as np
import pytest
import torch

from oracle import distill as D

pytestmark = pytest.mark.gpu


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


TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(seed, n, V, dtype, scale=3.0):
    g = np.random.Generator(np.random.PCG64(seed))
    x = torch.from_numpy((scale * g.normal(size=(n, V))).astype(np.float32))
    x[torch.arange(n), torch.from_numpy(g.integers(0, V, n))] += 6.0
    return x.to(TYPES[dtype]).cuda()


def check(ids, logp, x, k, temperature=1.0):
    want, lw = D.top_logits(x.double().cpu().numpy(), k, temperature)
    got, l = ids.cpu().numpy(), logp.double().cpu().numpy()
    assert (got == want).all(), (np.argwhere(got != want)[:5], got[got != want][:5], want[got != want][:5])
    with np.errstate(invalid="ignore"):
        ok = (np.abs(l - lw) <= 2e-5 + 4e-7 * np.abs(lw)) | (l == lw) | (np.isnan(l) & np.isnan(lw))
    assert ok.all(), (np.argwhere(~ok)[:5], l[~ok][:5], lw[~ok][:5])


SIZES = [(1, 1), (3, 2), (5, 7), (5, 8), (4, 9), (7, 31), (9, 33), (3, 64), (3, 65), (6, 255),
         (3, 1000), (37, 1001), (200, 515), (2, 4096), (3, 8191), (5, 32000), (2, 32003), (170, 2050),
         (700, 4000), (1500, 1), (1300, 40), (1000, 500), (950, 2051), (2000, 5000), (1000, 9001), (2, 70001), (3, 151936), (40, 151936), (1, 262144), (1, 300007), (1, 1000003)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_sizes(B, ctx, n, V, dtype):
    x = rows(3 * n + V, n, V, dtype)
    for k in (1, 20, 32, 33, 64):
        T = 0.7 if k == 20 else 1.0
        check(*B.pr_top_logits(ctx, x, k, temperature=T), x, k, T)
    assert B.pr_ctx_flags(ctx) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(6, 777), (6, 40000), (300, 5000), (1000, 2500), (1000, 333), (6, 151936)])
def test_rows_in_order_and_rows_of_ties(B, ctx, n, V, dtype):
    """What a threshold that rises along the row meets at worst."""
    x = rows(V, n, V, "f32")
    x[0] = torch.sort(x[0])[0]
    x[1] = torch.sort(x[1], descending=True)[0]
    x[2] = 1.5                                             # all alike
    x[3] = (torch.arange(V, device="cuda") % 7).float()    # few values
    x[4] = -torch.arange(V, device="cuda").float() / 64    # the first k
    x = x.to(TYPES[dtype])
    x[-1, V // 2:] = x[-1].max()                           # a tail of ties
    for k in (1, 31, 64):
        check(*B.pr_top_logits(ctx, x, k), x, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(12, 40), (12, 1003), (12, 40000), (400, 1003), (1000, 1003)])
def test_values_that_a_row_can_hold(B, ctx, n, V, dtype):
    x = rows(V + 1, n, V, dtype)
    low = torch.finfo(x.dtype).min
    x[0, : V // 2] = -torch.inf
    x[1] = -torch.inf                      # nothing left
    x[2] = low                             # nothing left either
    x[3, 1:] = low                         # one token left
    x[4, 3] = torch.nan
    x[5, V - 1] = torch.inf
    x[6] = 3e4 + x[6]                      # large logits
    x[7] = torch.where(torch.arange(V, device="cuda") % 3 == 0, 0.0, -0.0).to(x.dtype)
    x[8, 10:] = -torch.inf                 # fewer than k left
    x[9, :-3] = low
    x[10] = -9e8
    x[11, V // 2] = 1.1e9                  # counts as infinite
    for k in (20, 64):
        B.pr_ctx_flags(ctx, clear=True)
        ids, logp = B.pr_top_logits(ctx, x, k)
        check(ids, logp, x, k)
        assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_NONFINITE
        assert (ids[[1, 2, 4, 5, 11]] == -1).all() and logp[[1, 2, 4, 5, 11]].isnan().all()


@pytest.mark.parametrize("dtype,V", [("f32", 6_500_001), ("bf16", 26_000_003)])
def test_vocabularies_beyond_a_cluster(B, ctx, dtype, V):
    x = torch.empty(2, V, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(3))
    x = x.to(TYPES[dtype])
    x[1] = 2.0
    check(*B.pr_top_logits(ctx, x, 40), x, 40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,stride,start", [(1000, 1003, 1), (5001, 5001, 3), (777, 1024, 0),
                                            (32000, 32001, 5), (32000, 32008, 8), (9, 11, 2)])
def test_strides_and_alignments(B, ctx, V, stride, start, dtype):
    for n in (3, 400, 1000):
        if n * stride > 6e6:
            continue
        buf = rows(V, 1, n * stride + start + 8, dtype)[0]
        x = buf[start:start + n * stride].view(n, stride)
        check(*B.pr_top_logits(ctx, x, 24, vocab=V), x[:, :V], 24)
        check(*B.pr_top_logits(ctx, x[:, :V], 24), x[:, :V], 24)


def test_outputs_stay_in_their_place_and_streams_and_graphs(B, ctx):
    n, V, k = 50, 8000, 17
    x = rows(1, n, V, "bf16")
    ids = torch.full((n + 2, k), 77, dtype=torch.int32, device="cuda")
    logp = torch.full((n + 2, k), 7.5, device="cuda")
    B.pr_top_logits(ctx, x, k, ids=ids[1:n + 1], logp=logp[1:n + 1])
    check(ids[1:n + 1], logp[1:n + 1], x, k)
    assert (ids[[0, -1]] == 77).all() and (logp[[0, -1]] == 7.5).all()
    first = ids.clone(), logp.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.pr_top_logits(ctx, x, k, ids=ids[1:n + 1], logp=logp[1:n + 1])
    torch.cuda.synchronize()
    assert torch.equal(ids, first[0]) and torch.equal(logp, first[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.pr_top_logits(ctx, x, k, ids=ids[1:n + 1], logp=logp[1:n + 1])
    x.copy_(rows(2, n, V, "bf16"))
    for _ in range(2):
        g.replay()
        check(ids[1:n + 1], logp[1:n + 1], x, k)


def test_calls_side_by_side(B, ctx):
    """The calls that hold no workspace, of one context on two streams at once."""
    xs = [rows(20 + i, 400, 20000, "bf16") for i in range(2)]
    want = [B.pr_top_logits(ctx, x, 30) for x in xs]
    w = torch.ones(20000, device="cuda", dtype=torch.bfloat16)
    normed = [B.pr_layernorm(ctx, x, w) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append((B.pr_top_logits(ctx, x, 30), B.pr_layernorm(ctx, x, w)))
        torch.cuda.synchronize()
        for (top, norm), t, m in zip(got, want, normed):
            assert torch.equal(top[0], t[0]) and torch.equal(top[1], t[1])
            assert torch.equal(norm[0], m[0]) and torch.equal(norm[3], m[3])


def test_the_first_call_of_a_context_captured(B):
    for n, V in ((3, 9000), (700, 9000), (1200, 800)):
        x = rows(n, n, V, "bf16")
        ctx = B.pr_ctx_create(0, 1, 1)
        try:
            ids = torch.empty(n, 12, dtype=torch.int32, device="cuda")
            logp = torch.empty(n, 12, device="cuda")
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                B.pr_top_logits(ctx, x, 12, ids=ids, logp=logp)
            g.replay()
            check(ids, logp, x, 12)
        finally:
            B.pr_ctx_destroy(ctx)


def test_kernel_times(B):
    ctx = B.pr_ctx_create(0, 1, 1)
    try:
        B.pr_ctx_set_option(ctx, B.PR_OPT_TIMING, 1)
        x = rows(5, 700, 3000, "f32")
        ids, logp = B.pr_top_logits(ctx, x, 8)
        assert len(B.pr_ctx_kernel_times(ctx)) == 1
        B.pr_distill_loss(ctx, x, ids, logp)
        times = B.pr_ctx_kernel_times(ctx)
        assert len(times) == 2 and all(t > 0 for t in times)   # the listing, the rows
        w = torch.ones(3000, device="cuda")
        _, _, mean, rstd = B.pr_layernorm(ctx, x, w)
        assert len(B.pr_ctx_kernel_times(ctx)) == 1
        B.pr_layernorm_backward(ctx, x, x, w, rstd, mean=mean)
        assert len(B.pr_ctx_kernel_times(ctx)) == 2            # the rows, the columns
    finally:
        B.pr_ctx_destroy(ctx)


def test_rows_past_32_bits(B, ctx):
    V, n, stride = 1000, 3, (1 << 31) + 24
    buf = torch.zeros(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (n, V), (stride, 1))
    x.copy_(rows(9, n, V, "bf16"))
    check(*B.pr_top_logits(ctx, x, 20), x, 20)


def test_refusals(B, ctx):
    x = rows(0, 4, 100, "f32")
    n0 = B.launch_count()

    def refused(*a, **kw):
        with pytest.raises(B.PRError) as e:
            B.pr_top_logits(ctx, *a, **kw)
        assert e.value.status == B.PR_ERR_INVALID_ARG

    for k in (0, -1, 65):
        refused(x, k)
    for T in (0.0, -1.0, 1e-4, 2e3, float("nan"), float("inf")):
        refused(x, 5, temperature=T)
    refused(x.cpu(), 5)
    refused(x, 5, vocab=101)
    refused(x, 5, vocab=0)
    refused(x[0], 5)
    refused(x.t(), 5)
    refused(x, 5, ids=torch.empty(3, 5, dtype=torch.int32, device="cuda"))
    refused(x, 5, ids=torch.empty(4, 5, dtype=torch.int64, device="cuda"))
    refused(x, 5, logp=torch.empty(4, 5, dtype=torch.float64, device="cuda"))
    refused(x, 5, logp=torch.empty(4, 5))
    with pytest.raises(TypeError):
        B.pr_top_logits(ctx, x.half(), 5)
    ids, logp = B.pr_top_logits(ctx, x[:0], 5)
    assert ids.shape == (0, 5) and logp.shape == (0, 5)
    assert B.launch_count() == n0


@pytest.mark.parametrize("temperature", [1.0, 0.41, 0.44, 0.47, 1000.0])
@pytest.mark.parametrize("n,V", [(6, 1003), (6, 40000), (1000, 1003), (2, 6_500_001)])
def test_the_border_of_infinity(B, ctx, n, V, temperature):
    """x / T from 1e9 on is infinite, the value before it is not; the same below."""
    big = torch.tensor(1e9 * temperature, dtype=torch.float32)
    below = torch.nextafter(big, torch.zeros(()))
    x = torch.empty(n, V, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(V))
    x[0] = below                           # the largest finite one alone
    x[1, :] = below
    x[1, V - 2] = big                      # one infinite one among those
    if n > 2:
        x[2, 5] = below
        x[3, 5] = big
        x[4] = -big                        # nothing left
        x[5] = -big
        x[5, 7:9] = -below                 # two left
    B.pr_ctx_flags(ctx, clear=True)
    ids, logp = B.pr_top_logits(ctx, x, 20, temperature=temperature)
    check(ids, logp, x, 20, temperature)
    assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_NONFINITE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(64, 151936), (16, 32003), (64, 1001), (1000, 4001), (700, 24001), (2, 6_500_001)])
def test_sure_tokens(B, ctx, n, V, dtype):
    """Rows of which one token, somewhere, has nearly all: its log-probability is never above 0, and as
    near as a sum can be that holds it.  Its term is off by 2^-22 and by its exponent's rounding, of
    up to 16 in size, 2^-21 ln 2; the factor between references by 2^-22; the sum's other roundings
    are of terms below 2^-14 of it, but for those on the way through lanes, warps and CTAs, 13 of
    2^-24, and the thread's own: 2^-24 for each of up to 160 chunks, random, 8 of them (four
    deviations of their mean); the logarithm and its difference 2^-23 (|l| + 1).  The tokens
    after it: the product's rounding as well, 4e-7 |l|."""
    g = torch.Generator("cuda").manual_seed(V)
    for up in (12.0, 17.0, 20.0, 24.0, 40.0):
        x = torch.randn(n, V, generator=g, device="cuda").to(TYPES[dtype])
        at = torch.randint(0, V, (n,), generator=g, device="cuda")
        x[torch.arange(n, device="cuda"), at] = (up + 3 * torch.rand(n, generator=g, device="cuda")).to(x.dtype)
        ids, logp = B.pr_top_logits(ctx, x, 3)
        want = torch.log_softmax(x.double(), 1).gather(1, ids.long())
        tol = (1.4 + 1 + 1) * 2.0 ** -22 + (13 + 8) * 2.0 ** -24 + 2.0 ** -23 + 5e-7 * want.abs()
        off = (logp.double() - want).abs()
        assert (off <= tol).all(), (up, float(off[:, 0].max()), float(off.max()))
        assert (logp <= 0).all() and (up < 12.5 or torch.equal(ids[:, 0].long(), at))


MASKS = ["lowest", -1e38, -2.3e38, -1e30, -7e20, -1e12, -3e9]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(5, 7), (6, 1003), (6, 40000), (1000, 1003), (700, 24001), (2, 6_500_001)])
def test_masks_of_any_size(B, ctx, n, V, dtype):
    """What is masked by a large negative number is no part of a row, at any temperature: also where
    nothing else is near."""
    g = torch.Generator("cuda").manual_seed(V)
    for mask in MASKS:
        x = torch.randn(n, V, generator=g, device="cuda").to(TYPES[dtype])
        low = torch.finfo(x.dtype).min if mask == "lowest" else mask
        x[0, : V - 2] = low
        x[1, 2:] = low
        hide = torch.rand(n, V, generator=g, device="cuda") < 0.97
        hide[:2] = False
        hide[:, V // 2] = False
        x = x.masked_fill(hide, low)
        if n > 3:
            x[3] = low                      # nothing left
        for T in (1e-3, 0.5, 1.0, 1.7, 2.0, 5.0, 100.0):
            B.pr_ctx_flags(ctx, clear=True)
            xt = torch.where(x > -1e3, (x.double() * T).to(x.dtype), x) if T < 1 else x
            ids, logp = B.pr_top_logits(ctx, xt, 5, temperature=T)
            masked = xt.double() <= -float(torch.tensor(1e9 * T, dtype=torch.float32))
            z = (xt.double() / T).masked_fill(masked, -torch.inf)
            top, at = torch.sort(z, dim=1, descending=True, stable=True)
            top, at = top[:, :5], at[:, :5].masked_fill(torch.isinf(top[:, :5]), -1)
            assert torch.equal(ids.long(), at), (mask, T)
            want = top - torch.logsumexp(z, 1, keepdim=True)
            off = (logp.double() - want).abs()
            ok = (off <= 2e-5 + 4e-7 * want.abs()) | (logp == want) | (logp.isnan() & want.isnan())
            assert ok.all(), (mask, T)
            none = bool(masked.all(1).any())
            assert B.pr_ctx_flags(ctx, clear=True) == (B.PR_FLAG_NONFINITE if none else 0)
