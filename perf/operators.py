"""The measured cases of the training operators.

The verifier's outcome is a training signal for the small model: a graded
response gives an advantage (policy loss), an escalated one a pair of answers
(preference loss), and the optimiser step ends the update.  A case is one pass
through one operator as a training program makes it, device tensors in hand.

  policy      the clipped policy loss with a KL term over a ragged batch of
              responses, from their logit rows: statistics, token
              log-probabilities and, with `grad`, the gradient of the logits
  preference  the loss of paired log ratios over a ragged batch of answer
              pairs: statistics, the answers' log ratios, token
              log-probabilities and, with `grad`, the gradient of the logits
  adamw       one AdamW step over a program's tensors.  They lie in one arena,
              each from a multiple of 256 elements on, as gradient buckets and
              checkpoints have them.  With 8-bit states the pass also expands
              the states to the values they stand for, as a checkpoint needs

Sizes are those of the project's workloads (vocabularies of 32,000, 70,001,
151,936 and 262,144 tokens, responses of up to 1,024 tokens, the LM head of
width 3,584, the scorer head) and generic ones between them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
V_FULL, V_WIDE, V_TINY, V_ODD = 151936, 262144, 32000, 70001
BUDGET = 2.7e9  # bytes of logits of the largest pass
BLOCK = 256     # elements that share the scale of an 8-bit state
PARAMS = 544538624  # elements of the largest step: the LM head


def listed():
    return [
        # an interactive update on a handful of short replies: latency and launches count
        dict(name="policy_reply", kind="policy", dtype="f32", vocab=V_TINY, n_req=4,
             spread="uniform", lo=1, hi=8, layout=1, grad=True, norm="tokens", ref=False,
             per_request=True, temperature=1.0),
        # monitoring pass over a small batch: the loss and its statistics, no gradient
        dict(name="policy_monitor", kind="policy", dtype="bf16", vocab=V_FULL, n_req=8,
             spread="uniform", lo=16, hi=64, layout=2, grad=False, norm="tokens", ref=True,
             per_request=False, temperature=1.0),
        # the update over a batch of 64 finished responses with a reference model
        dict(name="policy_full", kind="policy", dtype="bf16", vocab=V_FULL, n_req=64,
             spread="uniform", lo=32, hi=256, layout=3, grad=True, norm="tokens", ref=True,
             per_request=False, temperature=1.0),
        # a vocabulary that is no multiple of the vector width, ragged responses that
        # count alike, sampled at a temperature
        dict(name="policy_odd", kind="policy", dtype="bf16", vocab=V_ODD, n_req=24,
             spread="lognormal", lo=8, hi=1024, layout=4, grad=True, norm="requests", ref=True,
             per_request=True, temperature=0.7),
        # two short answer pairs: latency counts
        dict(name="preference_small", kind="preference", dtype="f32", vocab=V_TINY, n_req=4,
             spread="uniform", lo=16, hi=64, layout=5, grad=True, loss="sigmoid",
             length_norm=False, temperature=1.0),
        # the answer pairs of 32 escalated requests
        dict(name="preference_full", kind="preference", dtype="bf16", vocab=V_FULL, n_req=64,
             spread="uniform", lo=32, hi=256, layout=6, grad=True, loss="sigmoid",
             length_norm=False, temperature=1.0),
        # wide fp32 logits, length-normalised log ratios and the squared loss
        dict(name="preference_wide", kind="preference", dtype="f32", vocab=V_WIDE, n_req=8,
             spread="uniform", lo=64, hi=512, layout=7, grad=True, loss="squared",
             length_norm=True, temperature=1.0),
        # evaluation on held-out pairs of an odd vocabulary: no gradient
        dict(name="preference_eval", kind="preference", dtype="bf16", vocab=V_ODD, n_req=16,
             spread="lognormal", lo=8, hi=1024, layout=8, grad=False, loss="sigmoid",
             length_norm=False, temperature=1.0),
        # the scorer head's 28 tensors, all in single precision
        dict(name="adamw_scorer", kind="adamw", dims="scorer", layers=2, d=64, vocab=0,
             param="f32", bits=32),
        # the LM head in bf16 with a master copy and states in single precision
        dict(name="adamw_lm_head", kind="adamw", dims="model", layers=0, d=3584, vocab=V_FULL,
             param="bf16", bits=32),
        # a small transformer's 97 tensors in single precision with 8-bit states
        dict(name="adamw8_stack", kind="adamw", dims="model", layers=8, d=1024, vocab=V_TINY,
             param="f32", bits=8),
        # an LM head in bf16 alone with 8-bit states: the least memory
        dict(name="adamw8_lm_head", kind="adamw", dims="model", layers=0, d=1024, vocab=V_FULL,
             param="bf16", bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["policy", "preference", "adamw"])
    if kind == "adamw":
        c = dict(kind=kind, dims=rng.choice(["scorer", "model", "model"]),
                 layers=rng.randint(1, 8), d=64, vocab=0, param=rng.choice(["f32", "bf16"]),
                 bits=rng.choice([8, 32]))
        if c["dims"] == "model":
            c["d"] = _log_int(rng, 40, 3584)
            c["vocab"] = _log_int(rng, 1000, V_FULL)
        most = PARAMS if c["bits"] == 32 else PARAMS // 3
        while c["layers"] > 0 and sum(n for n, _ in _tensors(c)) > most:
            c["layers"] -= 1
        return c
    c = dict(kind=kind, layout=rng.randrange(100, 1 << 20), dtype=rng.choice(["f32", "bf16"]),
             vocab=_log_int(rng, 4000, V_WIDE), n_req=2 * _log_int(rng, 1, 128),
             spread=rng.choice(["uniform", "lognormal"]), lo=_log_int(rng, 1, 64),
             grad=rng.random() < 0.75, temperature=rng.choice([1.0, 1.0, 0.7, 1.5]))
    c["hi"] = c["lo"] + _log_int(rng, 1, 1024 - c["lo"])
    if rng.random() < 0.4:  # a multiple of 64, as most vocabularies are padded
        c["vocab"] = c["vocab"] // 64 * 64
    if kind == "policy":
        c["norm"] = rng.choice(["tokens", "requests"])
        c["ref"] = rng.random() < 0.5
        c["per_request"] = rng.random() < 0.5
    else:
        c["loss"] = rng.choice(["sigmoid", "sigmoid", "squared", "hinge"])
        c["length_norm"] = rng.random() < 0.3
    while c["n_req"] > 2 and int(_lengths(c).sum()) * c["vocab"] * _esize(c) > BUDGET:
        c["n_req"] -= 2 * max(1, c["n_req"] // 8)
    return c


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _lengths(c):
    g = np.random.Generator(np.random.PCG64(c["layout"]))
    if c["spread"] == "uniform":
        return g.integers(c["lo"], c["hi"], size=c["n_req"], endpoint=True).astype(np.int64)
    raw = np.exp(g.normal(math.log(min(c["hi"], 128)), 0.8, size=c["n_req"]))
    return np.clip(np.round(raw), c["lo"], c["hi"]).astype(np.int64)


def _tensors(c):
    """(elements, whether weight decay applies) of each tensor of a step."""
    d, ff = c["d"], 2 * c["d"] if c["dims"] == "scorer" else 4 * c["d"]
    layer = [(3 * d * d, True), (3 * d, False), (d * d, True), (d, False), (ff * d, True),
             (ff, False), (d * ff, True), (d, False)] + 4 * [(d, False)]
    if c["dims"] == "scorer":
        return [(4 * d, True), (d, False)] + c["layers"] * layer + [(d, True), (1, False)]
    return [(c["vocab"] * d, True)] + c["layers"] * layer


# ---- inputs -------------------------------------------------------------------------------


class State:
    """A program's tensors."""


_context = None


def _ctx():
    """The context that a program keeps."""
    global _context
    if _context is None:
        from paper_2608_28726_gb300 import binding as B
        _context = B.pr_ctx_create(0, 1, 1)
    return _context


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(s, c, n, g):
    """Logit rows (a scale per row, a spike on most rows), tokens drawn from
    their softmax at the case's temperature, and the tokens' log-probabilities."""
    V, T = c["vocab"], c["temperature"]
    s.logits = torch.empty(n, V, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32,
                           device=DEV)
    s.chosen = torch.empty(n, dtype=torch.int32, device=DEV)
    logp = torch.empty(n, device=DEV)
    step = max(1, (1 << 28) // V)
    for a in range(0, n, step):
        b = min(n, a + step)
        k = b - a
        r = torch.arange(k, device=DEV)
        z = torch.randn(k, V, generator=g, device=DEV)
        z.mul_(1.0 + 3.0 * torch.rand(k, 1, generator=g, device=DEV))
        amp = 12.0 * torch.rand(k, generator=g, device=DEV)
        z[r, torch.randint(0, V, (k,), generator=g, device=DEV)] += amp
        s.logits[a:b] = z
        z.copy_(s.logits[a:b]).div_(T)
        u = torch.rand(k, V, generator=g, device=DEV).clamp_(min=1e-30).log_().neg_().log_()
        y = torch.sub(z, u, out=u).argmax(dim=1)
        s.chosen[a:b] = y
        logp[a:b] = z[r, y] - torch.logsumexp(z, dim=1)
        del z, u
    return logp


def prepare(case, seed):
    c, g, s = case, _gen(seed), State()
    s.case = c
    if c["kind"] == "adamw":
        _prepare_adamw(s, c, g)
        return s
    T = _lengths(c)
    n = int(T.sum())
    s.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(T)]).astype(np.int64)).to(DEV)
    logp = _rows(s, c, n, g)
    # tokens that the program inserted (tool results, forced tokens) are not trained on
    s.mask = (torch.rand(n, generator=g, device=DEV) < 0.9).to(torch.uint8)
    s.ref_logp = logp + 0.05 + 0.2 * torch.randn(n, generator=g, device=DEV)
    if c["kind"] == "policy":
        s.old_logp = logp + 0.15 * torch.randn(n, generator=g, device=DEV)
        s.advantage = torch.randn(c["n_req"] if c["per_request"] else n, generator=g, device=DEV)
        if not c["ref"]:
            s.ref_logp = None
    return s


def _prepare_adamw(s, c, g):
    sizes = _tensors(c)
    starts = np.cumsum([0] + [-(-n // BLOCK) * BLOCK for n, _ in sizes]).tolist()
    total = starts[-1]
    dt = torch.bfloat16 if c["param"] == "bf16" else torch.float32
    live = torch.zeros(total // BLOCK, BLOCK, dtype=torch.bool, device=DEV)
    s.decay = torch.zeros(total // BLOCK, 1, device=DEV)  # weight decay of each block
    for (n, wd), a in zip(sizes, starts):
        live.view(-1)[a:a + n] = True
        s.decay[a // BLOCK:(a + n + BLOCK - 1) // BLOCK] = 0.1 if wd else 0.0

    def noise():
        x = torch.randn(total // BLOCK, BLOCK, generator=g, device=DEV)
        return x.mul_(live)

    scale = 1e-3 * torch.exp(torch.randn(total // BLOCK, 1, generator=g, device=DEV))
    p = noise().mul_(0.02)
    s.master = p if c["param"] == "bf16" and c["bits"] == 32 else None
    s.p = p.to(dt)
    s.g = noise().mul_(scale).to(dt)
    m = noise().mul_(scale).mul_(0.3)
    v = noise().mul_(scale).square_()
    s.clip = 0.5 + 0.5 * torch.rand(1, generator=g, device=DEV)  # of the gradient's norm
    s.hyper = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, step=1000)
    if c["bits"] == 8:
        s.m, s.m_scale = _to8(m, True)
        s.v, s.v_scale = _to8(v, False)
    else:
        s.m, s.v, s.m_scale, s.v_scale = m, v, None, None
    if own:  # the program's table of its tensors
        from paper_2608_28726_gb300 import binding as B

        def cut(t):
            return None if t is None else [t.view(-1)[a:a + n] for (n, _), a in zip(sizes, starts)]

        def cut_scales(t):
            return None if t is None else [t.view(-1)[a // BLOCK:(a + n + BLOCK - 1) // BLOCK]
                                           for (n, _), a in zip(sizes, starts)]

        s.table = B.pr_adamw_tensors(cut(s.p), cut(s.g), cut(s.m), cut(s.v), master=cut(s.master),
                                     m_scale=cut_scales(s.m_scale), v_scale=cut_scales(s.v_scale),
                                     weight_decay=[0.1 if wd else 0.0 for _, wd in sizes])


# ---- one pass -----------------------------------------------------------------------------


def run(s):
    if own:
        return {"policy": _own_policy, "preference": _own_preference,
                "adamw": _own_adamw}[s.case["kind"]](s)
    return {"policy": _plain_policy, "preference": _plain_preference,
            "adamw": _plain_adamw}[s.case["kind"]](s)


CLIP_LOW, CLIP_HIGH, KL_COEF, BETA, SMOOTH = 0.2, 0.25, 0.04, 0.1, 0.05


def _own_policy(s):
    from paper_2608_28726_gb300 import binding as B
    c = s.case
    stats, logp, grad = B.pr_policy_loss(
        _ctx(), s.logits, s.chosen, s.advantage, old_logp=s.old_logp, ref_logp=s.ref_logp,
        mask=s.mask, offsets=s.offsets, clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL_COEF,
        temperature=c["temperature"], per_request=c["per_request"], want_grad=c["grad"],
        norm=B.PR_NORM_TOKENS if c["norm"] == "tokens" else B.PR_NORM_REQUESTS)
    return {"stats": stats, "logp": logp, "grad": grad}


def _own_preference(s):
    from paper_2608_28726_gb300 import binding as B
    c = s.case
    loss = {"sigmoid": B.PR_PREF_SIGMOID, "squared": B.PR_PREF_SQUARED,
            "hinge": B.PR_PREF_HINGE}[c["loss"]]
    stats, ratio, logp, grad = B.pr_preference_loss(
        _ctx(), s.logits, s.chosen, s.offsets, ref_logp=s.ref_logp, mask=s.mask, beta=BETA,
        loss=loss, label_smoothing=SMOOTH if c["loss"] == "sigmoid" else 0.0,
        length_norm=c["length_norm"], temperature=c["temperature"], want_grad=c["grad"])
    return {"stats": stats, "ratio": ratio, "logp": logp, "grad": grad}


def _own_adamw(s):
    from paper_2608_28726_gb300 import binding as B
    B.pr_adamw_step(_ctx(), s.table, grad_scale=s.clip, **s.hyper)
    out = {"p": s.p}
    if s.master is not None:
        out["master"] = s.master
    if s.case["bits"] == 8:
        out["m"], out["v"] = B.pr_adamw_unpack(_ctx(), s.table)
    else:
        out["m"], out["v"] = s.m, s.v
    return out


# the plain forms: the formulas in elementary operations, in single precision


def _softmax(s):
    """exp of the shifted rows, their sums, and the tokens' log-probabilities."""
    x = s.logits.float()
    if s.case["temperature"] != 1.0:
        x = x / s.case["temperature"]
    at = s.chosen.long().unsqueeze(1)
    top = x.amax(dim=1, keepdim=True)
    x = x - top  # (logits in single precision stay as they are)
    chosen = x.gather(1, at)
    e = x.exp_()
    total = e.sum(dim=1, keepdim=True)
    return e, total, (chosen - total.log()).squeeze(1), at


def _gradient(s, e, total, at, coef):
    """coef (onehot - p) / temperature, in the logits' type."""
    coef = (coef / s.case["temperature"]).unsqueeze(1)
    e *= -(coef / total)
    e.scatter_add_(1, at, coef)
    return e.to(s.logits.dtype)


def _requests(s):
    """Whether each token counts, its request, and the requests' counted tokens."""
    n = s.logits.shape[0]
    live = s.mask.float()
    req = torch.searchsorted(s.offsets, torch.arange(n, device=DEV), right=True) - 1
    count = torch.zeros(s.offsets.numel() - 1, device=DEV).index_add_(0, req, live)
    return live, req, count


def _plain_policy(s):
    c = s.case
    e, total, logp, at = _softmax(s)
    live, req, count = _requests(s)
    if c["norm"] == "tokens":
        weight = live / count.sum().clamp(min=1.0)
    else:
        weight = live / ((count > 0).sum() * count.clamp(min=1.0))[req]
    adv = s.advantage[req] if c["per_request"] else s.advantage
    ratio = torch.exp(logp - s.old_logp)
    free = ratio * adv
    bound = ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    surrogate = torch.minimum(free, bound)
    clipped = (bound < free).float()
    coef = -free * (1.0 - clipped)
    loss = -surrogate
    kl = torch.zeros_like(logp)
    if s.ref_logp is not None:
        d = s.ref_logp - logp
        kl = torch.exp(d) - d - 1.0
        loss = loss + KL_COEF * kl
        coef = coef + KL_COEF * (1.0 - torch.exp(d))
    old_kl = ratio - (logp - s.old_logp) - 1.0
    stats = torch.stack([(weight * t).sum() for t in (loss, surrogate, kl, ratio, clipped, old_kl)])
    grad = _gradient(s, e, total, at, weight * coef) if c["grad"] else None
    return {"stats": stats, "logp": logp * live, "grad": grad}


def _plain_preference(s):
    c = s.case
    e, total, logp, at = _softmax(s)
    live, req, count = _requests(s)
    ratio = torch.zeros_like(count).index_add_(0, req, live * (logp - s.ref_logp))
    share = live
    if c["length_norm"]:
        ratio = ratio / count.clamp(min=1.0)
        share = live / count.clamp(min=1.0)[req]
    d = ratio[0::2] - ratio[1::2]
    valid = ((count[0::2] > 0) & (count[1::2] > 0)).float()
    pairs = valid.sum().clamp(min=1.0)
    h = BETA * d
    if c["loss"] == "sigmoid":  # -log sigmoid(h) = log(1 + exp(-h))
        up = torch.log1p(torch.exp(-h.abs())) + (-h).clamp(min=0.0)
        down = torch.log1p(torch.exp(-h.abs())) + h.clamp(min=0.0)
        loss = (1.0 - SMOOTH) * up + SMOOTH * down
        slope = BETA * (SMOOTH / (1.0 + torch.exp(-h)) - (1.0 - SMOOTH) / (1.0 + torch.exp(h)))
    elif c["loss"] == "squared":
        loss = (d - 0.5 / BETA) ** 2
        slope = 2.0 * (d - 0.5 / BETA)
    else:
        loss = (1.0 - h).clamp(min=0.0)
        slope = -BETA * (h < 1.0).float()
    stats = torch.stack([(valid * t).sum() / pairs for t in (
        loss, (d > 0).float(), h, BETA * ratio[0::2], BETA * ratio[1::2])])
    grad = None
    if c["grad"]:
        slope = slope * valid / pairs
        side = torch.stack([slope, -slope], dim=1).reshape(-1)
        grad = _gradient(s, e, total, at, share * side[req])
    return {"stats": stats, "ratio": ratio, "logp": logp * live, "grad": grad}


def _to8(x, signed):
    """(codes, scales) of blocks of values: the square root of the ratio to the
    block's largest magnitude in 127 steps with a sign, or its fourth root in 255."""
    top = x.abs().amax(dim=1, keepdim=True)
    top = torch.where(top >= 2.0 ** -126, top, torch.zeros_like(top))
    inv = torch.where(top > 0, 1.0 / top, torch.zeros_like(top))
    r = (x.abs() * inv).sqrt()
    if signed:
        return (torch.round(r * 127.0) * torch.sign(x)).to(torch.int8), top
    return torch.round(r.sqrt() * 255.0).to(torch.uint8), top


def _from8(q, top, signed):
    q = q.float()
    if signed:
        return (q * q.abs()) * (top * (1.0 / 127.0 ** 2))
    q = q * q
    return (q * q) * (top * (1.0 / 255.0 ** 4))


def _plain_adamw(s):
    h, eight = s.hyper, s.case["bits"] == 8
    g = s.g.float() * s.clip
    m = _from8(s.m, s.m_scale, True) if eight else s.m
    v = _from8(s.v, s.v_scale, False) if eight else s.v
    m = m * h["beta1"] + g * (1.0 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1.0 - h["beta2"])
    p = s.p.float() if s.master is None else s.master
    by = (v * (1.0 / (1.0 - h["beta2"] ** h["step"]))).sqrt_().add_(h["eps"])
    by = (m * (1.0 / (1.0 - h["beta1"] ** h["step"]))).div_(by).add_(p * s.decay)
    p = p - h["lr"] * by
    s.p.copy_(p)
    out = {"p": s.p}
    if s.master is not None:
        s.master.copy_(p)
        out["master"] = s.master
    if eight:
        codes, scale = _to8(m, True)
        s.m.copy_(codes), s.m_scale.copy_(scale)
        codes, scale = _to8(v, False)
        s.v.copy_(codes), s.v_scale.copy_(scale)
        out["m"], out["v"] = _from8(s.m, s.m_scale, True), _from8(s.v, s.v_scale, False)
    else:
        s.m.copy_(m), s.v.copy_(v)
        out["m"], out["v"] = s.m, s.v
    return out


# ---- what a pass cannot do without --------------------------------------------------------


def work(case):
    c = case
    if c["kind"] == "adamw":
        n = sum(n for n, _ in _tensors(c))
        e = 2 if c["param"] == "bf16" else 4
        if c["bits"] == 32:  # gradient in, states in and out; parameters in and out, or the
            # master copy in and out and the parameters out
            per = e + 16 + (8 + e if c["param"] == "bf16" else 2 * e)
        else:  # and the two expanded states out
            per = e + 4 + 2 * e + 8
        return {"bytes": n * per, "flops": 14 * n}
    n = int(_lengths(c).sum())
    row = c["vocab"] * _esize(c)
    small = 4 + 4 + 1 + 4 * (2 if c["kind"] == "policy" else 1)
    return {"bytes": 0.9 * n * row + (n * row if c["grad"] else 0) + n * small,
            "flops": 0.9 * n * c["vocab"] * (10 if c["grad"] else 5)}


# ---- the definition in 64 bits ------------------------------------------------------------


def exact(case, seed):
    """The losses from torch's own log-softmax in double precision and their
    gradients by automatic differentiation; the step from its formulas."""
    c, s = case, prepare(case, seed)
    if c["kind"] == "adamw":
        return _exact_adamw(c, s)
    x = s.logits.double().requires_grad_(c["grad"])
    keep = s.mask.bool()
    bounds = s.offsets.tolist()
    lp = torch.log_softmax(x / c["temperature"], dim=1)
    logp = lp[torch.arange(x.shape[0], device=DEV), s.chosen.long()]
    del lp
    spans = [(a, b) for a, b in zip(bounds[:-1], bounds[1:])]
    if c["kind"] == "policy":
        total, used = int(keep.sum()), sum(bool(keep[a:b].any()) for a, b in spans)
        sums = [0.0] * 6
        for r, (a, b) in enumerate(spans):
            k = keep[a:b]
            if not bool(k.any()):
                continue
            l, old = logp[a:b][k], s.old_logp[a:b][k].double()
            adv = s.advantage[r].double() if c["per_request"] else s.advantage[a:b][k].double()
            ratio = torch.exp(l - old)
            low = torch.where(ratio < 1 - CLIP_LOW, torch.full_like(ratio, 1 - CLIP_LOW), ratio)
            cut = torch.where(low > 1 + CLIP_HIGH, torch.full_like(ratio, 1 + CLIP_HIGH), low)
            sur = torch.where(cut * adv < ratio * adv, cut * adv, ratio * adv)
            kl = torch.zeros_like(l)
            if s.ref_logp is not None:
                q = s.ref_logp[a:b][k].double() - l
                kl = torch.expm1(q) - q
            w = 1.0 / total if c["norm"] == "tokens" else 1.0 / (used * int(k.sum()))
            terms = (KL_COEF * kl - sur, sur, kl, ratio, (cut * adv < ratio * adv).double(),
                     torch.expm1(l - old) - (l - old))
            sums = [t + w * u.sum() for t, u in zip(sums, terms)]
        out = {"stats": torch.stack(sums).detach()}
    else:
        terms, ratios = [], []
        for a, b in spans:
            t = (logp[a:b] - s.ref_logp[a:b].double())[keep[a:b]]
            ratios.append(t.mean() if c["length_norm"] and t.numel() else t.sum())
        for r in range(0, len(spans), 2):
            if not all(bool(keep[a:b].any()) for a, b in spans[r:r + 2]):
                continue
            d = ratios[r] - ratios[r + 1]
            if c["loss"] == "sigmoid":
                f = torch.nn.functional.logsigmoid
                loss = -(1 - SMOOTH) * f(BETA * d) - SMOOTH * f(-BETA * d)
            elif c["loss"] == "squared":
                loss = (d - 1 / (2 * BETA)).square()
            else:
                loss = torch.relu(1 - BETA * d)
            terms.append(torch.stack([loss, (d > 0).double(), BETA * d, BETA * ratios[r],
                                      BETA * ratios[r + 1]]))
        sums = torch.stack(terms).mean(dim=0) if terms else torch.zeros(5, dtype=torch.float64)
        out = {"stats": sums.detach(), "ratio": torch.stack(ratios).detach()}
    out["logp"] = torch.where(keep, logp, torch.zeros_like(logp)).detach()
    out["grad"] = None
    if c["grad"]:
        first = sums[0]
        out["grad"] = (torch.autograd.grad(first, x)[0] if first.requires_grad
                       else torch.zeros_like(x))
    return out


def _exact_adamw(c, s):
    h = s.hyper
    g = s.g.double() * s.clip.double()
    m, v = s.m.double(), s.v.double()
    if c["bits"] == 8:
        m = torch.sign(m) * (m / 127) ** 2 * s.m_scale.double()
        v = (v / 255) ** 4 * s.v_scale.double()
    p = (s.p if s.master is None else s.master).double()
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
    mhat, vhat = m / (1 - h["beta1"] ** h["step"]), v / (1 - h["beta2"] ** h["step"])
    p = p - h["lr"] * (mhat / (torch.sqrt(vhat) + h["eps"]) + s.decay.double() * p)
    out = {"p": p}
    if s.master is not None:
        out["master"] = p
    out["m"], out["v"] = (None, None) if c["bits"] == 8 else (m, v)
    return out
