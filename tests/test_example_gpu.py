"""The training example: its gradient against 64-bit differentiation, and that it trains."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "train_lm_head", os.path.join(ROOT, "examples", "train_lm_head.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def logp64(logits, tokens):
    return torch.log_softmax(logits, 1).gather(1, tokens.long()[:, None])[:, 0]


def test_gradient_of_the_weights(example):
    t = example.Trainer(vocab=1000, dim=64, requests=16, seed=3)
    B = example.B
    try:
        for _ in range(3):  # away from the first head, where every log ratio is 0
            t.step()
        tokens, logits = t.answer()
        # some answers on either side, whatever the head makes of them
        scores = B.pr_route(t.ctx, logits, tokens, t.offsets, t.score_w, 0.0, 0.5)[0]
        bias = float(-torch.logit(scores.double().median()))
        route = B.pr_route
        try:
            B.pr_route = lambda c, x, y, o, w, b, tau: route(c, x, y, o, w, bias, tau)
            ship = B.pr_route(t.ctx, logits, tokens, t.offsets, t.score_w, 2.0, 0.5)[1]
            assert 0 < int(ship.sum()) < len(ship)
            x = logits.double().requires_grad_()
            z = logits[t.pair_source].double().requires_grad_()
            policy, pref, _, _ = t.losses(tokens, logits)
        finally:
            B.pr_route = route
        h = t.hidden.double()
        first = (t.hidden @ t.first.t()).double()
        n_req, kept = len(ship), ship.bool()
        # policy: ratio 1, so that the surrogate is r A with r = exp(l - l's value)
        ell = logp64(x, tokens)
        q = logp64(first, tokens) - ell
        grade = torch.zeros(n_req, dtype=torch.float64, device="cuda").index_add_(
            0, t.row_req, (tokens == t.large).double()) / t.offsets.diff()
        adv = grade - grade[kept].mean()
        term = -torch.exp(ell - ell.detach()) * adv[t.row_req] + t.kl_coef * (torch.expm1(q) - q)
        rows = t.offsets.diff().double()
        per = torch.zeros(n_req, dtype=torch.float64, device="cuda").index_add_(0, t.row_req, term)
        loss = (per / rows)[kept].mean()
        loss.backward()
        loss = loss.detach()
        assert abs(float(policy[B.PR_POL_LOSS]) - float(loss)) <= 1e-4 * (1 + abs(float(loss)))
        # pairs
        both = torch.empty(2 * len(tokens), dtype=torch.int64, device="cuda")
        both[t.large_rows], both[t.small_rows] = t.large.long(), tokens.long()
        d = logp64(z, both) - logp64(first[t.pair_source], both)
        s = torch.zeros(n_req, dtype=torch.float64, device="cuda").index_add_(
            0, t.row_req, d[t.large_rows] - d[t.small_rows]) / rows
        pair_loss = -torch.nn.functional.logsigmoid(t.beta * s)[~kept].mean()
        pair_loss.backward()
        pair_loss = pair_loss.detach()
        assert abs(float(pref[B.PR_PREF_LOSS]) - float(pair_loss)) <= 1e-4 * (1 + float(pair_loss))

        src = h[t.pair_source]
        want = x.grad.t() @ h + z.grad.t() @ src
        size = x.grad.abs().t() @ h.abs() + z.grad.abs().t() @ src.abs()
        # bf16: half a unit in the last place, 2^-8, of each logit's gradient, of the first
        # product, of the sum, and of parts that the product may be made of
        assert ((t.grad.double() - want).abs() <= 4 * 2.0 ** -8 * size + 1e-12).all()
        assert float(want.abs().max()) > 0
    finally:
        t.close()


def test_training_moves_the_head_towards_the_large_model(example):
    runs = []
    for _ in range(2):
        t = example.Trainer(vocab=2048, dim=128, requests=24, seed=1)
        try:
            grades = [float(t.step()[3]) for _ in range(40)]
            assert example.B.pr_ctx_flags(t.ctx) == 0
            assert torch.isfinite(t.master).all()
            assert torch.equal(t.weight, t.master.bfloat16())
            runs.append(grades)
        finally:
            t.close()
    grades = runs[0]
    assert sum(grades[-5:]) > sum(grades[:5])
    assert runs[1][0] == grades[0]  # (later steps: the example's own sums take any order)
