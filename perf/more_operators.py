"""The measured cases of the distillation operators and of the norm before the LM head.

A request that the verifier escalates is answered by the large model.  What it sends along
with the answer, the most likely tokens of each row, trains the small model.  A case is one
pass through one operator as a program makes it, device tensors in hand.

  top      the k largest logits of each row: their tokens in order (ties: lowest token first)
           and their log-probabilities
  distill  the loss of a ragged batch of logit rows against such lists: statistics, the rows'
           divergences and, with `grad`, the gradient of the logits
  norm     layer norm or RMS norm of a batch of rows, a residual added first
  dnorm    its backward pass: the gradients of the rows, the weight and the bias

Sizes are those of the project's workloads (vocabularies of 32,000, 70,001, 151,936 and
262,144 tokens, responses of up to 1,024 tokens, rows of width 3,584, the scorer head's 64) and
generic ones between them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
V_FULL, V_WIDE, V_TINY, V_ODD = 151936, 262144, 32000, 70001
ROWS_FULL = 8847  # rows of the full-response workload
BUDGET = 2.7e9    # bytes of logits of the largest pass
NORM_BUDGET = 7e7  # elements of the largest norm


def listed():
    return [
        # a decode step of 8 requests whose clients asked for the first tokens' log-probabilities
        dict(name="top_step", kind="top", dtype="bf16", vocab=V_FULL, rows=8, k=20,
             temperature=1.0),
        # the large model's answers to a window of escalated requests
        dict(name="top_answers", kind="top", dtype="bf16", vocab=V_FULL, rows=4096, k=32,
             temperature=1.0),
        # wide fp32 logits, the longest lists
        dict(name="top_wide", kind="top", dtype="f32", vocab=V_WIDE, rows=1000, k=64,
             temperature=1.0),
        # rows off the 16-byte grid, softened
        dict(name="top_odd", kind="top", dtype="bf16", vocab=V_ODD, rows=600, k=50,
             temperature=2.0),
        # an interactive update on a handful of short replies: latency and launches count
        dict(name="distill_reply", kind="distill", dtype="f32", vocab=V_TINY, n_req=4,
             spread="uniform", lo=1, hi=8, layout=11, k=16, grad=True, loss="reverse", rest=True,
             kl=1.0, ce=0.0, norm="tokens", temperature=1.0),
        # the update over 64 finished answers
        dict(name="distill_full", kind="distill", dtype="bf16", vocab=V_FULL, n_req=64,
             spread="uniform", lo=32, hi=256, layout=12, k=32, grad=True, loss="forward",
             rest=True, kl=1.0, ce=0.0, norm="tokens", temperature=1.0),
        # an odd vocabulary, lists taken for the whole distribution, hard labels beside them,
        # ragged answers that count alike
        dict(name="distill_odd", kind="distill", dtype="bf16", vocab=V_ODD, n_req=24,
             spread="lognormal", lo=8, hi=1024, layout=13, k=50, grad=True, loss="forward",
             rest=False, kl=2.0, ce=0.5, norm="requests", temperature=2.0),
        # evaluation on held-out answers, wide fp32 logits: no gradient
        dict(name="distill_eval", kind="distill", dtype="f32", vocab=V_WIDE, n_req=8,
             spread="uniform", lo=64, hi=512, layout=14, k=64, grad=False, loss="reverse",
             rest=True, kl=1.0, ce=0.1, norm="tokens", temperature=1.0),
        # the final norm of a decode step of 8 requests: latency
        dict(name="norm_step", kind="norm", dtype="bf16", rows=8, d=3584, rms=True, bias=False,
             residual=True, stats=False),
        # the final norm of a batch in training
        dict(name="norm_forward", kind="norm", dtype="bf16", rows=ROWS_FULL, d=3584, rms=False,
             bias=True, residual=True, stats=True),
        dict(name="norm_backward", kind="dnorm", dtype="bf16", rows=ROWS_FULL, d=3584, rms=False,
             bias=True, residual=True),
        # the scorer head's norm over a pool of short sequences
        dict(name="norm_scorer", kind="dnorm", dtype="f32", rows=30000, d=64, rms=False, bias=True,
             residual=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["top", "distill", "distill", "norm", "dnorm"])
    c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]))
    if kind in ("norm", "dnorm"):
        c.update(d=_log_int(rng, 16, 16384), rms=rng.random() < 0.4, bias=rng.random() < 0.5,
                 residual=rng.random() < 0.5)
        if rng.random() < 0.5:
            c["d"] = max(16, c["d"] // 64 * 64)
        c["rows"] = min(_log_int(rng, 1, 32768), int(NORM_BUDGET) // c["d"])
        if kind == "norm":
            c["stats"] = rng.random() < 0.5
        return c
    c.update(vocab=_log_int(rng, 4000, V_WIDE), k=_log_int(rng, 1, 64),
             temperature=rng.choice([1.0, 1.0, 0.7, 2.0]))
    if rng.random() < 0.4:  # a multiple of 64, as most vocabularies are padded
        c["vocab"] = c["vocab"] // 64 * 64
    if kind == "top":
        c["rows"] = min(_log_int(rng, 1, 8192), int(BUDGET) // (c["vocab"] * _esize(c)))
        return c
    c.update(n_req=_log_int(rng, 1, 256), spread=rng.choice(["uniform", "lognormal"]),
             lo=_log_int(rng, 1, 64), layout=rng.randrange(100, 1 << 20),
             grad=rng.random() < 0.75, loss=rng.choice(["forward", "forward", "reverse"]),
             rest=rng.random() < 0.6, kl=rng.choice([1.0, 0.5]), ce=rng.choice([0.0, 0.3]),
             norm=rng.choice(["tokens", "requests"]))
    c["hi"] = c["lo"] + _log_int(rng, 1, 1024 - c["lo"])
    while c["n_req"] > 1 and int(_lengths(c).sum()) * c["vocab"] * _esize(c) > BUDGET:
        c["n_req"] -= max(1, c["n_req"] // 8)
    return c


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lengths(c):
    g = np.random.Generator(np.random.PCG64(c["layout"]))
    if c["spread"] == "uniform":
        return g.integers(c["lo"], c["hi"], size=c["n_req"], endpoint=True).astype(np.int64)
    raw = np.exp(g.normal(math.log(min(c["hi"], 128)), 0.8, size=c["n_req"]))
    return np.clip(np.round(raw), c["lo"], c["hi"]).astype(np.int64)


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


def _parts(rows, vocab):
    step = max(1, (1 << 28) // vocab)
    return [(a, min(rows, a + step)) for a in range(0, rows, step)]


def _noise_rows(k, V, g):
    """Logits with a scale per row and a spike on most rows."""
    z = torch.randn(k, V, generator=g, device=DEV)
    z.mul_(1.0 + 3.0 * torch.rand(k, 1, generator=g, device=DEV))
    amp = 12.0 * torch.rand(k, generator=g, device=DEV)
    z[torch.arange(k, device=DEV), torch.randint(0, V, (k,), generator=g, device=DEV)] += amp
    return z


def prepare(case, seed):
    c, g, s = case, _gen(seed), State()
    s.case = c
    if c["kind"] in ("norm", "dnorm"):
        _prepare_norm(s, c, g)
    elif c["kind"] == "top":
        s.logits = torch.empty(c["rows"], c["vocab"], dtype=_type(c), device=DEV)
        for a, b in _parts(c["rows"], c["vocab"]):
            s.logits[a:b] = _noise_rows(b - a, c["vocab"], g)
    else:
        _prepare_distill(s, c, g)
    return s


def _prepare_distill(s, c, g):
    V, T, K = c["vocab"], c["temperature"], c["k"]
    lengths = _lengths(c)
    n = int(lengths.sum())
    s.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)).to(DEV)
    s.logits = torch.empty(n, V, dtype=_type(c), device=DEV)
    s.ids = torch.empty(n, K, dtype=torch.int32, device=DEV)
    s.logp = torch.empty(n, K, device=DEV)
    s.chosen = torch.empty(n, dtype=torch.int32, device=DEV)
    for a, b in _parts(n, V):
        k = b - a
        z = _noise_rows(k, V, g)
        s.logits[a:b] = z
        # the large model: the small one's logits, sharper and with others among them
        z.mul_(1.1).add_(torch.randn(k, V, generator=g, device=DEV)).div_(T)
        top, at = z.topk(K, dim=1)
        top = top - torch.logsumexp(z, dim=1, keepdim=True)
        gone = top < math.log(1e-5)  # what is that unlikely is not sent
        gone[:, 0] = False
        s.ids[a:b] = torch.where(gone, -1, at)
        s.logp[a:b] = torch.where(gone, -math.inf, top)
        u = torch.rand(k, K, generator=g, device=DEV).clamp_(min=1e-30).log_().neg_().log_()
        pick = (top - u).argmax(dim=1, keepdim=True)  # its answer: of the list, now and then not
        y = at.gather(1, pick)[:, 0]
        other = torch.randint(0, V, (k,), generator=g, device=DEV)
        s.chosen[a:b] = torch.where(torch.rand(k, generator=g, device=DEV) < 0.05, other, y)
        del z
    # tokens that the program inserted (tool results, forced tokens) are not trained on
    s.mask = (torch.rand(n, generator=g, device=DEV) < 0.9).to(torch.uint8)


def _prepare_norm(s, c, g):
    n, d, dt = c["rows"], c["d"], _type(c)

    def hidden(spread):
        x = torch.randn(n, d, generator=g, device=DEV)
        x.mul_(spread * (0.5 + 1.5 * torch.rand(n, 1, generator=g, device=DEV)))
        x.add_(0.2 * torch.randn(n, 1, generator=g, device=DEV))
        x[:, ::max(1, d // 4)] *= 20.0  # the few columns that carry most of a row
        return x.to(dt)

    s.x = hidden(1.0)
    s.weight = (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(dt)
    s.bias = (0.1 * torch.randn(d, generator=g, device=DEV)).to(dt) if c["bias"] else None
    if c["kind"] == "norm":
        s.residual = hidden(0.5) if c["residual"] else None
        return
    s.dy = (1e-2 * torch.randn(n, d, generator=g, device=DEV)).to(dt)
    s.dtotal = (1e-2 * torch.randn(n, d, generator=g, device=DEV)).to(dt) if c["residual"] else None
    s.mean, s.rstd = _moments(s.x.float(), c["rms"])


# ---- one pass -----------------------------------------------------------------------------

EPS = 1e-5


def run(s):
    kind = s.case["kind"]
    if own:
        return {"top": _own_top, "distill": _own_distill, "norm": _own_norm,
                "dnorm": _own_dnorm}[kind](s)
    return {"top": _plain_top, "distill": _plain_distill, "norm": _plain_norm,
            "dnorm": _plain_dnorm}[kind](s)


def _own_top(s):
    from paper_2608_28726_gb300 import binding as B
    ids, logp = B.pr_top_logits(_ctx(), s.logits, s.case["k"], temperature=s.case["temperature"])
    return {"ids": ids, "logp": logp}


def _own_distill(s):
    from paper_2608_28726_gb300 import binding as B
    c = s.case
    stats, kl, grad = B.pr_distill_loss(
        _ctx(), s.logits, s.ids, s.logp, chosen=s.chosen if c["ce"] > 0 else None, mask=s.mask,
        offsets=s.offsets, kl_coef=c["kl"], ce_coef=c["ce"], temperature=c["temperature"],
        loss=B.PR_DISTILL_FORWARD if c["loss"] == "forward" else B.PR_DISTILL_REVERSE,
        rest=B.PR_REST_CLASS if c["rest"] else B.PR_REST_NONE,
        norm=B.PR_NORM_TOKENS if c["norm"] == "tokens" else B.PR_NORM_REQUESTS,
        want_grad=c["grad"])
    return {"stats": stats, "kl": kl, "grad": grad}


def _own_norm(s):
    from paper_2608_28726_gb300 import binding as B
    c = s.case
    y, total, mean, rstd = B.pr_layernorm(_ctx(), s.x, s.weight, bias=s.bias, residual=s.residual,
                                          eps=EPS, rms=c["rms"], want_stats=c["stats"])
    return {"y": y, "total": total, "mean": mean, "rstd": rstd}


def _own_dnorm(s):
    from paper_2608_28726_gb300 import binding as B
    c = s.case
    dx, dweight, dbias = B.pr_layernorm_backward(_ctx(), s.dy, s.x, s.weight, s.rstd, mean=s.mean,
                                                 dtotal=s.dtotal, rms=c["rms"],
                                                 want_dbias=c["bias"])
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


# the plain forms: the formulas in elementary operations, in single precision


def _plain_top(s):
    c = s.case
    V, K, T = c["vocab"], c["k"], c["temperature"]
    low = torch.arange(V, 0, -1, device=DEV)  # of equal logits the lowest token first
    ids, logp = [], []
    for a, b in _parts(c["rows"], 4 * V):
        x = s.logits[a:b].float() + 0.0
        i = x.view(torch.int32)
        key = (i ^ ((i >> 31) & 0x7fffffff)).long() * (1 << 32) + low
        at = V - (key.topk(K, dim=1)[0] & 0xffffffff)
        z = x / T if T != 1.0 else x
        top = z.amax(dim=1, keepdim=True)
        lse = torch.exp(z - top).sum(dim=1, keepdim=True).log()
        ids.append(at.int())
        logp.append((z.gather(1, at) - top) - lse)
    return {"ids": torch.cat(ids), "logp": torch.cat(logp)}


def _plain_distill(s):
    c = s.case
    n, T = s.logits.shape[0], c["temperature"]
    live = s.mask.double()
    req = torch.searchsorted(s.offsets, torch.arange(n, device=DEV), right=True) - 1
    count = torch.zeros(s.offsets.numel() - 1, dtype=torch.float64, device=DEV)
    count.index_add_(0, req, live)
    if c["norm"] == "tokens":
        weight = live / count.sum().clamp(min=1.0)
    else:
        weight = live / ((count > 0).sum() * count.clamp(min=1.0))[req]

    x = s.logits.float()
    if T != 1.0:
        x = x / T
    top = x.amax(dim=1, keepdim=True)
    x = x - top
    on = s.ids >= 0
    at = torch.where(on, s.ids, s.ids[:, :1]).long()
    listed_x = x.gather(1, at)
    y = s.chosen.long().unsqueeze(1)
    x_y = x.gather(1, y)
    e = x.exp_()
    e_y = e.gather(1, y)
    rest = e.scatter(1, at, 0.0).sum(dim=1, keepdim=True)
    listed_e = torch.where(on, listed_x.exp(), torch.zeros_like(listed_x))
    total = rest + listed_e.sum(dim=1, keepdim=True)

    # the lists are short: in double precision, as a rest next to nothing needs
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    logz = total.double().log()
    ell = listed_x.double() - logz
    logp = torch.where(on, s.logp.double(), zero)
    p = torch.where(on, logp.exp(), zero)
    q = torch.where(on, ell.exp(), zero)
    mass_p, mass_q = p.sum(dim=1, keepdim=True), q.sum(dim=1, keepdim=True)
    sigma = (rest / total).double()
    rho = (1.0 - mass_p).clamp(min=2.0 ** -24)
    if not c["rest"]:
        logp, p = logp - mass_p.log(), p / mass_p
    if c["loss"] == "forward":
        kl = (p * (logp - ell)).sum(dim=1, keepdim=True)
        a, b = -p, torch.zeros_like(rho)
        if c["rest"]:
            kl = kl + rho * (rho.log() - sigma.log())
            b = -rho
    else:
        if not c["rest"]:
            ell, q = ell - mass_q.log(), q / mass_q
        far = ell - logp
        kl = (q * far).sum(dim=1, keepdim=True)
        b = torch.zeros_like(rho)
        if c["rest"]:
            out = sigma.log() - rho.log()
            kl = kl + sigma * out
            b = sigma * (out - kl)
        a = q * (far - kl)
    ce = logz - x_y.double()
    loss = c["kl"] * kl + c["ce"] * ce
    if c["ce"] == 0.0:
        ce = torch.zeros_like(ce)
    stats = torch.stack([(weight * t[:, 0]).sum() for t in (loss, kl, ce, mass_p, mass_q)])
    out = {"stats": stats.float(), "kl": (live * kl[:, 0]).float(), "grad": None}
    if c["grad"]:
        scale = weight.unsqueeze(1) / T
        a, b = c["kl"] * a, c["kl"] * b
        every = a.sum(dim=1, keepdim=True) + b + -c["ce"]
        dense = b / sigma - every
        grad = e.mul_((scale * dense / total).float())
        own_e = (listed_e / total).double()
        # (absent entries: a is 0 for them, and their place is the first token's)
        fixed = torch.where(on, a - every * own_e, (a - every * own_e)[:, :1])
        grad.scatter_(1, at, (scale * fixed).float())
        if c["ce"] > 0.0:
            grad.scatter_add_(1, y, (scale * -c["ce"]).float())
        out["grad"] = grad.to(s.logits.dtype)
    return out


def _moments(h, rms):
    mean = None if rms else h.mean(dim=1)
    v = h if rms else h - mean[:, None]
    return mean, torch.rsqrt((v * v).mean(dim=1) + EPS)


def _plain_norm(s):
    c = s.case
    total, h = None, s.x.float()
    if s.residual is not None:
        total = (h + s.residual.float()).to(s.x.dtype)
        h = total.float()
    mean, rstd = _moments(h, c["rms"])
    y = (h if mean is None else h - mean[:, None]) * rstd[:, None] * s.weight.float()
    if s.bias is not None:
        y = y + s.bias.float()
    if not c["stats"]:
        mean = rstd = None
    return {"y": y.to(s.x.dtype), "total": total, "mean": mean, "rstd": rstd}


def _plain_dnorm(s):
    c = s.case
    dy, h = s.dy.float(), s.x.float()
    hat = (h if c["rms"] else h - s.mean[:, None]) * s.rstd[:, None]
    g = dy * s.weight.float()
    dx = g - hat * (g * hat).mean(dim=1, keepdim=True)
    if not c["rms"]:
        dx = dx - g.mean(dim=1, keepdim=True)
    dx = dx * s.rstd[:, None]
    if s.dtotal is not None:
        dx = dx + s.dtotal.float()
    return {"dx": dx.to(s.x.dtype), "dweight": (dy * hat).sum(dim=0),
            "dbias": dy.sum(dim=0) if c["bias"] else None}


# ---- what a pass cannot do without --------------------------------------------------------


def work(case):
    c = case
    if c["kind"] in ("norm", "dnorm"):
        nd, e = c["rows"] * c["d"], _esize(c)
        if c["kind"] == "norm":
            return {"bytes": nd * e * (4 if c["residual"] else 2) + (1 + c["bias"]) * c["d"] * e
                    + (c["rows"] * (4 if c["rms"] else 8) if c["stats"] else 0), "flops": 8 * nd}
        return {"bytes": nd * e * (4 if c["residual"] else 3) + c["d"] * e
                + 4 * c["d"] * (1 + c["bias"]) + c["rows"] * (4 if c["rms"] else 8),
                "flops": 14 * nd}
    if c["kind"] == "top":
        return {"bytes": c["rows"] * (c["vocab"] * _esize(c) + 8 * c["k"]),
                "flops": 5 * c["rows"] * c["vocab"]}
    n = int(_lengths(c).sum())
    row = c["vocab"] * _esize(c)
    return {"bytes": 0.9 * n * (row + 8 * c["k"]) + (n * row if c["grad"] else 0) + n * 9,
            "flops": 0.9 * n * c["vocab"] * (10 if c["grad"] else 5)}


# ---- the definition in 64 bits ------------------------------------------------------------


def exact(case, seed):
    """Orders from a stable sort, losses and norms from their definitions in double precision,
    gradients by automatic differentiation."""
    c, s = case, prepare(case, seed)
    if c["kind"] == "top":
        ids, logp = [], []
        for a, b in _parts(c["rows"], 8 * c["vocab"]):
            x = s.logits[a:b].double()
            at = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :c["k"]]
            ids.append(at)
            logp.append(torch.log_softmax(x / c["temperature"], dim=1).gather(1, at))
        return {"ids": torch.cat(ids), "logp": torch.cat(logp)}
    if c["kind"] == "distill":
        return _exact_distill(c, s)
    if c["kind"] == "norm":
        h, total = s.x.double(), None
        if s.residual is not None:
            total = h + s.residual.double()
            h = total.to(s.x.dtype).double()
        y, mean, rstd = _exact_norm(c, h, s.weight.double(),
                                    None if s.bias is None else s.bias.double())
        if not c["stats"]:
            mean = rstd = None
        return {"y": y, "total": total, "mean": mean, "rstd": rstd}
    h, w = s.x.double().requires_grad_(), s.weight.double().requires_grad_()
    bias = torch.zeros_like(w).requires_grad_()
    y = _exact_norm(c, h, w, bias)[0]
    dx, dw, db = torch.autograd.grad(y, (h, w, bias), s.dy.double())
    if s.dtotal is not None:
        dx = dx + s.dtotal.double()
    return {"dx": dx, "dweight": dw, "dbias": db if c["bias"] else None}


def _exact_norm(c, h, weight, bias):
    mean = None if c["rms"] else h.mean(dim=1, keepdim=True)
    mid = h if c["rms"] else h - mean
    std = torch.sqrt(torch.mean(mid ** 2, dim=1, keepdim=True) + EPS)
    y = mid / std * weight
    y = y if bias is None else y + bias
    return y, None if mean is None else mean[:, 0], 1.0 / std[:, 0]


def _exact_distill(c, s):
    x = s.logits.double().requires_grad_(c["grad"])
    lp = torch.log_softmax(x / c["temperature"], dim=1)
    rows = torch.arange(x.shape[0], device=DEV)
    out = torch.ones_like(lp, dtype=torch.bool)  # tokens outside a row's list
    r, j = torch.nonzero(s.ids >= 0, as_tuple=True)
    v = s.ids[r, j].long()
    out[r, v] = False
    sent = s.logp[r, j].double()  # entry by entry, with their rows

    def per_row(t):
        return torch.zeros(x.shape[0], dtype=torch.float64, device=DEV).index_add(0, r, t)

    ell = lp[r, v]
    mass_p, mass_q = per_row(sent.exp()), per_row(ell.exp())
    if c["rest"]:
        rest_p = torch.clamp(1.0 - mass_p, min=2.0 ** -24)
        rest_q = torch.logsumexp(lp.masked_fill(~out, -math.inf), dim=1)
        if c["loss"] == "forward":
            kl = per_row(sent.exp() * (sent - ell)) + rest_p * (rest_p.log() - rest_q)
        else:
            kl = per_row(ell.exp() * (ell - sent)) + rest_q.exp() * (rest_q - rest_p.log())
    else:
        sent = sent - mass_p.log()[r]
        if c["loss"] == "forward":
            kl = per_row(sent.exp() * (sent - ell))
        else:
            ell = ell - mass_q.log()[r]
            kl = per_row(ell.exp() * (ell - sent))
    ce = -lp[rows, s.chosen.long()] if c["ce"] > 0 else torch.zeros_like(kl)
    keep = s.mask.bool()
    spans = s.offsets.tolist()
    terms = torch.stack([c["kl"] * kl + c["ce"] * ce, kl, ce, mass_p, mass_q], dim=1)
    parts = [terms[a:b][keep[a:b]] for a, b in zip(spans[:-1], spans[1:])]
    parts = [t for t in parts if t.shape[0] > 0]
    if not parts:
        stats = terms[:0].sum(dim=0)
    elif c["norm"] == "tokens":
        stats = torch.cat(parts).mean(dim=0)
    else:
        stats = torch.stack([t.mean(dim=0) for t in parts]).mean(dim=0)
    grad = None
    if c["grad"]:
        grad = torch.autograd.grad(stats[0], x)[0] if parts else torch.zeros_like(x)
    return {"stats": stats.detach(), "kl": torch.where(keep, kl, torch.zeros_like(kl)).detach(),
            "grad": grad}
