"""GPU parity of pr_distill_loss where large batches of rows too long for one warp have their lists
worked out ahead of the rows: every value that a row or a list can hold, little mass, captures and
workspaces that grow, rows off the grid.

Sizes: more than 608 rows (four for each SM), rows above 22 KB.  Tolerances are those of
test_distill_gpu, whose checks are used.
"""
import numpy as np
import pytest
import torch

import test_distill_gpu as M
from oracle import distill as D
from test_distill_gpu import B, TYPES, check, ctx, draw, to  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

LONG = {"bf16": 12011, "f32": 6007}  # 24 KB


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_a_row_can_hold(B, ctx, dtype):
    M.test_values_that_a_row_can_hold(B, ctx, 620, LONG[dtype], dtype)


@pytest.mark.parametrize("V", [6007, 30000])
@pytest.mark.parametrize("loss", [0, 1])
def test_lists_that_hold_little_of_a_row(B, ctx, V, loss):
    M.test_lists_that_hold_little_of_a_row(B, ctx, 640, V, loss)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100001, 250000])
def test_rows_of_clusters_hold_what_small_batches_do(B, ctx, V, dtype):
    """Rows held by clusters: the batch against calls of 24 rows, whose CTAs fetch their lists
    themselves.  Weighted by the number of rows, a row's gradient is the same in both.  Two fp32
    results, each within test_distill_gpu's tolerances of the formula; bf16 gradients each within
    half a step of theirs."""
    n, few, k = 640, 24, 24
    g, x, x64, ids, sent, ch = draw(V, few, V, k, dtype)
    x[0, : V // 2] = -torch.inf
    x[1] = -torch.inf
    x[2, 3] = torch.nan
    x[3, V // 2] = torch.inf
    x[4, 1] = torch.finfo(x.dtype).min
    ids[5, 4], ids[6, 4] = V, -2
    ids[7, 5] = ids[7, 6] = 11
    sent[7, 5] = sent[7, 6] = -4.0
    sent[8, 2], sent[9, 2] = np.nan, np.inf
    ids[10] = -1
    sent[11] = -np.inf
    at = torch.from_numpy(np.maximum(ids[12], 0)).long().cuda()
    x[12, at] = -torch.inf                      # listed tokens are masked
    ch[13], ch[14] = V, -1
    again = np.arange(n) % few
    big = torch.empty(n, V, dtype=x.dtype, device="cuda")
    for a in range(0, n, few):
        big[a:a + few] = x[:min(few, n - a)]
    for loss, rest in ((0, 0), (1, 0), (0, 1), (1, 1)):
        kw = dict(loss=loss, rest=rest, ce_coef=0.2)
        s0, kl0, g0 = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), grad_scale=float(few), **kw)
        s1, kl1, g1 = B.pr_distill_loss(ctx, big, to(ids[again]), to(sent[again]), chosen=to(ch[again]),
                                        grad_scale=float(n), **kw)
        assert B.pr_ctx_flags(ctx, clear=True) == B.PR_FLAG_NONFINITE | B.PR_FLAG_BAD_CHOSEN
        wrong = [1, 2, 3, 5, 6, 7, 8, 9, 13, 14] + ([12] if loss and rest else [])
        assert kl0[wrong].isnan().all() and g0[wrong].isnan().all() and s1.isnan().all()
        assert not g0[[r for r in range(few) if r not in wrong]].isnan().any()
        for a in range(0, n, few):
            m = min(few, n - a)
            p, q = kl1[a:a + m].double(), kl0[:m].double()
            assert ((p == q) | (p.isnan() & q.isnan()) | ((p - q).abs() <= 4e-5 * (1 + q.abs()))).all()
            p, q = g1[a:a + m].double(), g0[:m].double()
            # (a gradient's parts are at most |a| + |A| q: below 30 for these lists)
            tol = (2.0 ** -7 if dtype == "bf16" else 0) * q.abs() + 4e-4 * (q.abs() + 1e-3)
            assert ((p.isnan() & q.isnan()) | ((p - q).abs() <= tol)).all(), (loss, rest, a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("stride,start,gstride,gstart", [(12, 1, 12, 1), (13, 3, 16, 8), (17, 0, 24, 5)])
def test_strides_and_alignments(B, ctx, stride, start, gstride, gstart, dtype):
    n, V, k = 612, LONG[dtype], 20
    stride, gstride = V + stride, V + gstride
    g, xs, x64, ids, sent, ch = draw(V, n, V, k, dtype)
    buf = torch.zeros(start + n * stride + 8, dtype=xs.dtype, device="cuda")
    x = buf[start:start + n * stride].view(n, stride)
    x[:, :V] = xs
    gbuf = torch.full((gstart + n * gstride + 8,), 7.0, dtype=xs.dtype, device="cuda")
    grad = gbuf[gstart:gstart + n * gstride].view(n, gstride)
    mask = (g.random(n) < 0.7).astype(np.uint8)
    got = B.pr_distill_loss(ctx, x, to(ids), to(sent), chosen=to(ch), mask=to(mask), ce_coef=0.1,
                            grad=grad, vocab=V)
    check((got[0], got[1], grad[:, :V]), D.distill(x64, ids, sent, ch, mask, ce_coef=0.1), mask, dtype)
    grad[:, :V] = 0
    assert float(gbuf.double().sum()) == 7.0 * (gbuf.numel() - n * V)  # the rest is as it was
    # in place of the logits
    want = B.pr_distill_loss(ctx, x, to(ids), to(sent), mask=to(mask), vocab=V, grad=grad)[2][:, :V].clone()
    got = B.pr_distill_loss(ctx, x, to(ids), to(sent), mask=to(mask), vocab=V, grad=x)[2][:, :V]
    assert torch.equal(got, want)


def test_lists_in_graphs_whose_workspace_grows(B):
    """The lists' workspace is first made under capture; a graph replays after larger calls have
    grown it, and beside another graph of the same context."""
    ctx = B.pr_ctx_create(0, 1, 1)
    try:
        made = []
        for n, k, dtype in ((612, 7, "f32"), (700, 64, "bf16")):
            V = LONG[dtype]
            g, x, x64, ids, sent, ch = draw(n, n, V, k, dtype)
            mask = to((g.random(n) < 0.8).astype(np.uint8))
            ids_t, sent_t = to(ids), to(sent)
            out = dict(stats=torch.empty(5, device="cuda"), kl=torch.empty(n, device="cuda"),
                       grad=torch.empty_like(x))
            graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            with torch.cuda.graph(graph, stream=s):
                B.pr_distill_loss(ctx, x, ids_t, sent_t, mask=mask, **out)
            made.append((graph, out, x, ids_t, sent_t, mask))
        first = []
        for graph, out, *_ in made:
            graph.replay()
            torch.cuda.synchronize()
            first.append({q: t.clone() for q, t in out.items()})
        g, y, y64, ids, sent, ch = draw(5, 1400, LONG["f32"], 64, "f32")
        B.pr_distill_loss(ctx, y, to(ids), to(sent))     # grows it
        for graph, out, *_ in made:
            for t in out.values():
                t.fill_(7)
        for (graph, out, x, ids_t, sent_t, mask), want in zip(made, first):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(t, want[q]) for q, t in out.items())
            got = B.pr_distill_loss(ctx, x, ids_t, sent_t, mask=mask)
            assert torch.equal(got[0], out["stats"]) and torch.equal(got[1], out["kl"]) and torch.equal(got[2], out["grad"])
            check((out["stats"], out["kl"], out["grad"]),
                  D.distill(x.double().cpu().numpy(), ids_t.cpu().numpy(), sent_t.cpu().numpy(), None,
                            mask.cpu().numpy()), None, "bf16" if x.dtype == torch.bfloat16 else "f32")
    finally:
        B.pr_ctx_destroy(ctx)
