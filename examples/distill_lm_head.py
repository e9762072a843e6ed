"""Distil a large model's answers into a small model's LM head: python examples/distill_lm_head.py

Each step the small model's hidden states go through its final layer norm and LM head, and the
verifier ships the answers that it is sure of.  The escalated requests are answered by the large
model, which sends along the first logits of each row (their tokens and log-probabilities) instead
of its whole distribution.  On those rows the small model is distilled: the loss writes its gradient
over the logits, which go through the head's product once more to become the gradients of the
head and of the normalised rows; the norm's backward pass gives those of its weights, and of the
hidden states below (which stay as they are here).  One AdamW step updates all three.
The data are synthetic: random hidden states, and a large model that is a random head.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_28726_gb300 import binding as B  # noqa: E402


class Distiller:
    def __init__(self, vocab=4096, dim=256, requests=48, k=32, seed=0, lr=2e-3, ce_coef=0.1,
                 clip_norm=1.0):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.lr, self.k, self.ce_coef, self.clip_norm = lr, k, ce_coef, clip_norm
        self.steps = 0
        length = torch.randint(1, 40, (requests,), generator=self.gen, device="cuda")
        self.offsets = torch.cat([length.new_zeros(1), length.cumsum(0)])
        n = int(self.offsets[-1])
        self.ctx = B.pr_ctx_create(0, max_rows=n, max_requests=requests)
        self.row_req = torch.repeat_interleave(torch.arange(requests, device="cuda"), length)

        # the last block's output and the residual stream that it is added to
        self.block = self._normal(n, dim).bfloat16()
        self.stream = (3 * self._normal(n, dim) + 0.5).bfloat16()
        total = self.block.float() + self.stream.float()
        teacher = 3 * self._normal(vocab, dim) / dim ** 0.5
        normed = (total - total.mean(1, keepdim=True)) / total.std(1, keepdim=True)
        self.large_logits = (normed @ teacher.t()).bfloat16()
        self.head = (teacher + 2 * self._normal(vocab, dim) / dim ** 0.5).bfloat16()
        self.norm_w, self.norm_b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
        self.master = self.head.float()
        self.grads = [torch.empty_like(self.head), torch.empty_like(self.norm_w), torch.empty_like(self.norm_b)]
        params = [self.head, self.norm_w, self.norm_b]
        moments = [[torch.zeros(p.shape, device="cuda") for p in params] for _ in range(2)]
        self.tensors = B.pr_adamw_tensors(params, self.grads, *moments, master=[self.master, None, None],
                                          weight_decay=[0.01, 0.0, 0.0])
        # the verifier's score: the answer's mean log-probability, sure above -3
        self.score_w = torch.zeros(11, device="cuda")
        self.score_w[0] = 1.0

    def close(self):
        B.pr_ctx_destroy(self.ctx)

    def _normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda")

    def escalated(self, logits, bias=3.0):
        """Rows of the answers that the verifier does not ship (1 for each)."""
        tokens = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=self.gen)[:, 0].int()
        ship = B.pr_route(self.ctx, logits, tokens, self.offsets, self.score_w, bias, 0.5)[1]
        return (1 - ship)[self.row_req]

    def gradients(self, mask=None):
        """(statistics, gradient of the residual stream's sum) of a step; the parameters' in self.grads."""
        y, total, mean, rstd = B.pr_layernorm(self.ctx, self.block, self.norm_w, bias=self.norm_b,
                                              residual=self.stream)
        logits = y @ self.head.t()
        if mask is None:
            mask = self.escalated(logits)
        # what the large model sends: its answer's tokens, and the first logits of each row
        ids, logp = B.pr_top_logits(self.ctx, self.large_logits, self.k)
        answer = ids[:, 0].contiguous()
        stats, _, _ = B.pr_distill_loss(self.ctx, logits, ids, logp, chosen=answer, mask=mask,
                                        offsets=self.offsets, ce_coef=self.ce_coef,
                                        norm=B.PR_NORM_REQUESTS, grad=logits)
        torch.mm(logits.t(), y, out=self.grads[0])
        dtotal, _, _ = B.pr_layernorm_backward(self.ctx, logits @ self.head, total, self.norm_w, rstd, mean=mean,
                                               dweight=self.grads[1], dbias=self.grads[2], want_dbias=True)
        return stats, dtotal, mask

    def step(self):
        """One step: (statistics of the loss, share of the rows that were escalated)."""
        stats, _, mask = self.gradients()
        self.steps += 1
        norm = torch.stack([g.float().norm() for g in self.grads]).norm()
        scale = (self.clip_norm / norm.clamp(min=1e-12)).clamp(max=1.0).reshape(1)
        B.pr_adamw_step(self.ctx, self.tensors, self.lr, beta2=0.95, step=self.steps, grad_scale=scale)
        return stats, mask.float().mean()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--requests", type=int, default=48)
    ap.add_argument("--k", type=int, default=32)
    args = ap.parse_args()
    t = Distiller(args.vocab, args.dim, args.requests, args.k)
    for i in range(args.steps):
        stats, escalated = t.step()
        if i % 10 == 0 or i == args.steps - 1:
            print("step %3d  escalated %.2f  loss %.4f  divergence %.4f  covered %.3f of %.3f" % (
                i, escalated, stats[B.PR_DIS_LOSS], stats[B.PR_DIS_KL], stats[B.PR_DIS_COVERED],
                stats[B.PR_DIS_LISTED]))
    t.close()


if __name__ == "__main__":
    main()
