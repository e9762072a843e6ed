"""Train a small model's LM head on what the verifier decides: python examples/train_lm_head.py

Each step the small model answers a ragged batch of requests, and the verifier ships the
answers that it is sure of and escalates the others:

  - a shipped answer is graded, and its tokens get the grade above the batch's mean as their
    advantage: clipped policy loss with a KL term to the head that training began with;
  - an escalated one is answered by the large model, and the two answers are a pair, the large
    model's above the small one's: loss of paired log ratios against that first head.

Both losses write their gradient over the logits, which go through the head's product once
more to become the gradient of its weights; one AdamW step with 8-bit states and a
single-precision master copy updates it.  The data are synthetic: random hidden states
that stay as they are (the layers below are frozen), and a large model that is a random head.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_28726_gb300 import binding as B  # noqa: E402


class Trainer:
    def __init__(self, vocab=4096, dim=256, requests=48, seed=0, lr=2e-3, beta=0.5, kl_coef=0.02,
                 clip_norm=1.0):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.lr, self.beta, self.kl_coef, self.clip_norm = lr, beta, kl_coef, clip_norm
        self.steps = 0
        length = torch.randint(1, 40, (requests,), generator=self.gen, device="cuda")
        self.offsets = torch.cat([length.new_zeros(1), length.cumsum(0)])
        n = int(self.offsets[-1])
        self.ctx = B.pr_ctx_create(0, max_rows=n, max_requests=requests)
        self.row_req = torch.repeat_interleave(torch.arange(requests, device="cuda"), length)
        # per request the large model's rows, then the small one's
        bounds = torch.stack([length, length], 1).flatten().cumsum(0)
        self.pair_offsets = torch.cat([bounds.new_zeros(1), bounds])
        row = torch.arange(n, device="cuda")
        start = self.offsets[self.row_req]
        self.large_rows = start + row                     # 2 start + (row - start)
        self.small_rows = self.large_rows + length[self.row_req]
        self.pair_source = torch.empty(2 * n, dtype=torch.int64, device="cuda")
        self.pair_source[self.large_rows] = row
        self.pair_source[self.small_rows] = row

        self.hidden = self._normal(n, dim).bfloat16()
        teacher = self._normal(vocab, dim) / dim ** 0.5
        self.large = (self.hidden.float() @ (4 * teacher).t()).argmax(1).int()
        self.weight = (2 * (teacher + self._normal(vocab, dim) / dim ** 0.5)).bfloat16()
        self.first = self.weight.clone()
        self.master = self.weight.float()
        self.grad = torch.empty_like(self.weight)
        blocks = -(-self.weight.numel() // B.PR_ADAMW_BLOCK)
        codes = (torch.zeros_like(self.weight, dtype=torch.int8),
                 torch.zeros_like(self.weight, dtype=torch.uint8))
        scales = torch.zeros(2, blocks, device="cuda")
        self.tensors = B.pr_adamw_tensors([self.weight], [self.grad], [codes[0]], [codes[1]],
                                          master=[self.master], m_scale=[scales[0]],
                                          v_scale=[scales[1]], weight_decay=0.01)
        # the verifier's score: the answer's mean log-probability, sure above -2
        self.score_w = torch.zeros(11, device="cuda")
        self.score_w[0] = 1.0

    def close(self):
        B.pr_ctx_destroy(self.ctx)

    def _normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda")

    def _logp(self, logits, tokens):
        """Log-probabilities of the tokens: the policy loss without a gradient."""
        return B.pr_policy_loss(self.ctx, logits, tokens, torch.zeros(len(tokens), device="cuda"),
                                want_grad=False)[1]

    def answer(self):
        """The small model's answers: (tokens, logits)."""
        logits = self.hidden @ self.weight.t()
        p = torch.softmax(logits.float(), 1)
        return torch.multinomial(p, 1, generator=self.gen)[:, 0].int(), logits

    def losses(self, tokens, logits):
        """Both losses and the gradient of the weights for a batch of answers."""
        first = self.hidden @ self.first.t()
        ship = B.pr_route(self.ctx, logits, tokens, self.offsets, self.score_w, 2.0, 0.5)[1]
        kept = ship[self.row_req]  # the rows of shipped answers
        same = (tokens == self.large).float()
        grade = torch.zeros(len(ship), device="cuda").index_add_(0, self.row_req, same)
        grade /= self.offsets.diff()
        shipped = ship.float()
        advantage = grade - (grade * shipped).sum() / shipped.sum().clamp(min=1)

        # escalated answers, above them the large model's
        both = torch.empty_like(self.pair_source, dtype=torch.int32)
        both[self.large_rows], both[self.small_rows] = self.large, tokens
        escalated = 1 - kept[self.pair_source]
        pairs = logits[self.pair_source]
        ref_pairs = self._logp(first[self.pair_source], both)
        pref, _, _, _ = B.pr_preference_loss(self.ctx, pairs, both, self.pair_offsets,
                                             ref_logp=ref_pairs, mask=escalated, beta=self.beta,
                                             length_norm=True, grad=pairs)

        # shipped ones: old_logp is this head's own, as every answer is used once
        ref = self._logp(first, tokens)
        policy, logp, _ = B.pr_policy_loss(self.ctx, logits, tokens, advantage, ref_logp=ref,
                                           mask=kept, offsets=self.offsets, per_request=True,
                                           kl_coef=self.kl_coef, norm=B.PR_NORM_REQUESTS,
                                           grad=logits)

        torch.mm(logits.t(), self.hidden, out=self.grad)
        self.grad.addmm_(pairs.t(), self.hidden[self.pair_source])
        return policy, pref, shipped.mean(), grade.mean()

    def step(self):
        """One step: (policy statistics, preference statistics, share shipped, mean grade)."""
        out = self.losses(*self.answer())
        self.steps += 1
        scale = (self.clip_norm / self.grad.float().norm()).clamp(max=1.0).reshape(1)
        B.pr_adamw_step(self.ctx, self.tensors, self.lr, beta2=0.95, step=self.steps,
                        grad_scale=scale)
        return out


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--requests", type=int, default=48)
    args = ap.parse_args()
    t = Trainer(args.vocab, args.dim, args.requests)
    for i in range(args.steps):
        policy, pref, shipped, grade = t.step()
        if i % 10 == 0 or i == args.steps - 1:
            print("step %3d  shipped %.2f  grade %.3f  policy loss %+.4f  kl %.4f  pair loss %.4f  "
                  "pairs in order %.2f" % (i, shipped, grade, policy[B.PR_POL_LOSS],
                                           policy[B.PR_POL_KL], pref[B.PR_PREF_LOSS],
                                           pref[B.PR_PREF_ACCURACY]))
    t.close()


if __name__ == "__main__":
    main()
