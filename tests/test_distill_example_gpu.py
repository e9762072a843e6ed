"""The distillation operators together, as the example uses them: the gradients of a whole step
against 64-bit differentiation, that it runs, and a step captured in a graph."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "distill_lm_head", os.path.join(ROOT, "examples", "distill_lm_head.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_a_step(example):
    B = example.B
    t = example.Distiller(vocab=1000, dim=64, requests=16, k=24, seed=3)
    try:
        for _ in range(2):  # away from weights of one
            t.step()
        mask = (torch.arange(len(t.row_req), device="cuda") % 5 > 0).to(torch.uint8)
        stats, dtotal, _ = t.gradients(mask)
        # the same in 64 bits, from the rows as the head takes and gives them
        total = (t.block.float() + t.stream.float()).bfloat16().double().requires_grad_()
        w, b = (p.double().clone().requires_grad_() for p in (t.norm_w, t.norm_b))
        head = t.head.double().requires_grad_()
        mid = total - total.mean(1, keepdim=True)
        y = mid / torch.sqrt((mid ** 2).mean(1, keepdim=True) + 1e-5) * w + b
        y = y + (y.detach().bfloat16().double() - y.detach())       # rounded, gradient as it is
        x = y @ head.t()
        x = x + ((y.detach().bfloat16() @ t.head.t()).double() - x.detach())
        x.retain_grad()
        ids, logp = B.pr_top_logits(t.ctx, t.large_logits, t.k)
        lq, lp = torch.log_softmax(x, 1), logp.double()
        out = torch.ones_like(lq, dtype=torch.bool).scatter_(1, ids.long(), False)
        rho = (1 - lp.exp().sum(1)).clamp(min=2.0 ** -24)
        sigma = torch.logsumexp(lq.masked_fill(~out, -torch.inf), 1)
        kl = (lp.exp() * (lp - lq.gather(1, ids.long()))).sum(1) + rho * (rho.log() - sigma)
        term = kl - t.ce_coef * lq.gather(1, ids[:, :1].long())[:, 0]
        keep = mask.bool()
        n_req = len(t.offsets) - 1
        count = torch.zeros(n_req, dtype=torch.float64, device="cuda").index_add_(0, t.row_req, keep.double())
        loss = ((term * keep) / count.clamp(min=1)[t.row_req]).sum() / (count > 0).sum()
        loss.backward()
        assert abs(float(stats[B.PR_DIS_LOSS]) - float(loss.detach())) <= 1e-4 * (1 + abs(float(loss.detach())))
        # bf16, half a step of 2^-8 each: a logit's gradient, each product's result, dx, and y and the
        # head's weights as factors; sums relative to their parts' magnitudes
        u = 2.0 ** -8
        size = x.grad.abs().t() @ y.detach().abs()
        assert ((t.grads[0].double() - head.grad).abs() <= 3 * u * size + 1e-9).all()
        dy = x.grad.abs() @ head.detach().abs()                      # what dy's parts add up to
        hat = (mid / torch.sqrt((mid ** 2).mean(1, keepdim=True) + 1e-5)).detach()
        assert ((t.grads[1].double() - w.grad).abs() <= 3 * u * (dy * hat.abs()).sum(0) + 1e-9).all()
        assert ((t.grads[2].double() - b.grad).abs() <= 3 * u * dy.sum(0) + 1e-9).all()
        g = dy * w.detach().abs()
        rstd = 1 / torch.sqrt((mid ** 2).mean(1, keepdim=True) + 1e-5).detach()
        size = rstd * (g + g.mean(1, keepdim=True) + hat.abs() * (g * hat.abs()).mean(1, keepdim=True))
        assert ((dtotal.double() - total.grad).abs() <= 4 * u * size + 1e-9).all()
        assert float(head.grad.abs().max()) > 0 and float(w.grad.abs().max()) > 0
    finally:
        t.close()


def test_runs_and_repeats(example):
    runs = []
    for _ in range(2):
        t = example.Distiller(vocab=2048, dim=128, requests=24, seed=1)
        try:
            out = [t.step() for _ in range(12)]
            assert example.B.pr_ctx_flags(t.ctx) == 0
            assert torch.isfinite(t.master).all() and torch.isfinite(t.norm_w).all()
            assert torch.equal(t.head, t.master.bfloat16())
            runs.append(out[0][0].clone())
        finally:
            t.close()
    assert torch.equal(runs[0], runs[1])  # (later steps: the example's own sums take any order)


def test_a_captured_step(example):
    t = example.Distiller(vocab=1500, dim=96, requests=12, k=16, seed=5)
    try:
        mask = torch.ones(len(t.row_req), dtype=torch.uint8, device="cuda")
        stats, dtotal, _ = t.gradients(mask)
        want = [stats.clone(), dtotal.clone()] + [g.clone() for g in t.grads]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            t.gradients(mask)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            stats, dtotal, _ = t.gradients(mask)
        for p in t.grads:
            p.zero_()
        for _ in range(2):
            g.replay()
        torch.cuda.synchronize()
        for p, q in zip([stats, dtotal] + t.grads, want):
            assert torch.equal(p, q)
    finally:
        t.close()
