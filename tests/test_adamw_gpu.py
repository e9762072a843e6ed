"""GPU parity of the optimiser step (pr_adamw_step, pr_adamw_unpack) with the
float64 oracle, over tensors of every size, type, alignment and kind of state.

Tolerances: a state is two products and a sum of fp32 values, each within 2^-24,
of constants within 2^-24: 4 x 2^-24 of the larger product, 3e-7 of |b m| + |(1 - b) g|.
The update divides by a root of v: 1e-6 of its size; a parameter adds its own
rounding, 2^-24 (fp32) or half a unit of bf16, 2^-8.  An 8-bit code is the
nearest one up to the rounding of its root (1e-6 of the code); the scale is exact.
"""
import numpy as np
import pytest
import torch

from oracle import loss as L

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, step=7)


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
    return t.double().cpu().numpy()


class Tensors:
    """One step's tensors: sizes, and a start of each buffer in elements."""

    def __init__(self, sizes, param, grad, master, bits, seed, start=0, scale=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        f, pt = torch.float32, torch.bfloat16 if param == "bf16" else torch.float32
        gt = torch.bfloat16 if grad == "bf16" else torch.float32

        def make(n, dtype, values=None):
            buf = torch.zeros(start + n + 8, dtype=dtype, device="cuda")
            t = buf[start:start + n]
            if values is not None:
                t.copy_(values)
            return t

        def noise(n, s=1.0):
            return torch.randn(n, generator=g, device="cuda") * s

        self.p = [make(n, pt, noise(n)) for n in sizes]
        self.g = [make(n, gt, noise(n, scale)) for n in sizes]
        self.master = [make(n, f, t.float()) for n, t in zip(sizes, self.p)] if master else None
        self.m_scale = self.v_scale = None
        if bits == 32:
            self.m = [make(n, f, noise(n, 0.3 * scale)) for n in sizes]
            self.v = [make(n, f, noise(n, scale).square()) for n in sizes]
        else:
            b = [-(-n // 256) for n in sizes]
            self.m = [make(n, torch.int8, torch.randint(-127, 128, (n,), generator=g, device="cuda"))
                      for n in sizes]
            self.v = [make(n, torch.uint8, torch.randint(0, 256, (n,), generator=g, device="cuda"))
                      for n in sizes]
            self.m_scale = [make(k, f, 0.5 * scale * torch.rand(k, generator=g, device="cuda")) for k in b]
            self.v_scale = [make(k, f, scale ** 2 * torch.rand(k, generator=g, device="cuda")) for k in b]
        self.wd = [0.1 * (i % 3) for i in range(len(sizes))]
        self.bits = bits

    def table(self, B):
        return B.pr_adamw_tensors(self.p, self.g, self.m, self.v, master=self.master,
                                  m_scale=self.m_scale, v_scale=self.v_scale, weight_decay=self.wd)

    def states(self):
        if self.bits == 32:
            return [f64(t) for t in self.m], [f64(t) for t in self.v]
        return ([L.held8(f64(q), f64(s), True) for q, s in zip(self.m, self.m_scale)],
                [L.held8(f64(q), f64(s), False) for q, s in zip(self.v, self.v_scale)])


def check_step(B, ctx, t, hyper=HYPER, grad_scale=None):
    gs = 1.0 if grad_scale is None else float(grad_scale.item())
    m0, v0 = t.states()
    p0 = [f64(x) for x in (t.master or t.p)]
    B.pr_adamw_step(ctx, t.table(B), grad_scale=grad_scale, **hyper)
    b1, b2 = hyper["beta1"], hyper["beta2"]
    for i, p in enumerate(p0):
        g = f64(t.g[i])
        want, m, v = L.adamw(p, g, m0[i], v0[i], weight_decay=t.wd[i], grad_scale=gs, **hyper)
        moved = np.abs(want - p) + hyper["lr"] * t.wd[i] * np.abs(p)
        m_off = 3e-7 * (b1 * np.abs(m0[i]) + (1 - b1) * np.abs(gs * g))
        v_off = 3e-7 * (b2 * v0[i] + (1 - b2) * (gs * g) ** 2)
        # m's error moves p by its share of the update
        slack = 2e-6 * moved + hyper["lr"] * m_off * 8 / (np.sqrt(8 * v) + 1e-8) + 1e-7 * np.abs(want)
        if t.master:
            assert (np.abs(f64(t.master[i]) - want) <= slack).all()
            assert torch.equal(t.p[i], t.master[i].bfloat16())
        else:
            slack = slack + (np.abs(want) * 2.0 ** -8 if t.p[i].dtype == torch.bfloat16 else 0.0)
            assert (np.abs(f64(t.p[i]) - want) <= slack).all()
        if t.bits == 32:
            assert (np.abs(f64(t.m[i]) - m) <= m_off).all()
            assert (np.abs(f64(t.v[i]) - v) <= v_off).all()
            continue
        for codes, scale, x, off, signed in ((t.m[i], t.m_scale[i], m, m_off, True),
                                             (t.v[i], t.v_scale[i], v, v_off, False)):
            q, s = L.codes8(x, signed)
            assert np.allclose(f64(scale), s, rtol=1e-6, atol=0)
            # a code follows its value's error by the root's slope, and the scale's
            edge = np.sqrt(np.repeat(s, 256)[:x.size]) + 1e-300
            reach = np.sqrt(np.abs(x) + off) - np.sqrt(np.maximum(np.abs(x) - off, 0.0))
            lim = 0.5 + 1e-4 + 127 * reach / edge
            if not signed:
                lim = 0.5 + 1e-4 + 255 * (np.sqrt(np.sqrt(x + off)) - np.sqrt(np.sqrt(
                    np.maximum(x - off, 0.0)))) / np.sqrt(edge)
            assert (np.abs(f64(codes) - q) <= lim).all()


TYPES = [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", False),
         ("bf16", "f32", False), ("bf16", "bf16", True), ("bf16", "f32", True)]
SIZES = [1, 0, 7, 255, 256, 257, 511, 2048, 2049, 4096, 40000, 300001, 64 * 192]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", TYPES)
@pytest.mark.parametrize("start", [0, 3])
def test_sizes_types_and_alignments(B, ctx, param, grad, master, bits, start):
    t = Tensors(SIZES, param, grad, master, bits, seed=bits + start, start=start)
    check_step(B, ctx, t)
    check_step(B, ctx, t, dict(HYPER, step=8), torch.tensor([0.37], device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
def test_large_tensors_and_many_tensors(B, ctx, bits):
    check_step(B, ctx, Tensors([9_000_001, 5], "f32", "f32", False, bits, seed=1))
    check_step(B, ctx, Tensors([(37 * i) % 600 for i in range(900)], "bf16", "f32", bits == 32,
                               bits, seed=2))


def test_mixed_types_in_one_step(B, ctx):
    parts = [Tensors([300, 1000], p, g, m, b, seed=i) for i, (p, g, m, b) in enumerate(
        [(*ty, b) for ty in TYPES for b in (32, 8)])]
    refs = [Tensors([300, 1000], p, g, m, b, seed=i) for i, (p, g, m, b) in enumerate(
        [(*ty, b) for ty in TYPES for b in (32, 8)])]
    for r in refs:
        check_step(B, ctx, r)

    def cat(name):
        return [x for t in parts for x in (getattr(t, name) or [None] * 2)]

    n0 = B.launch_count()
    B.pr_adamw_step(ctx, B.pr_adamw_tensors(
        cat("p"), cat("g"), cat("m"), cat("v"), master=cat("master"), m_scale=cat("m_scale"),
        v_scale=cat("v_scale"), weight_decay=cat("wd")), **HYPER)
    assert B.launch_count() - n0 == 12
    for t, r in zip(parts, refs):
        for name in ("p", "m", "v", "master", "m_scale", "v_scale"):
            for x, y in zip(getattr(t, name) or [], getattr(r, name) or []):
                assert torch.equal(x, y)


def test_hyperparameters_at_their_ends(B, ctx):
    """The first step (bias corrections of 1 - beta), no momentum, no decay of v, large
    and tiny gradients: squares of 1e-15 are below the normal numbers."""
    for hyper in (dict(HYPER, step=1), dict(HYPER, beta1=0.0), dict(HYPER, beta2=0.0, eps=1e-3),
                  dict(HYPER, step=10 ** 7)):
        for scale in (1.0, 1e-4, 1e4):
            check_step(B, ctx, Tensors([700], "f32", "f32", False, 32, 3, scale=scale), hyper)
            check_step(B, ctx, Tensors([700], "f32", "f32", False, 8, 3, scale=scale), hyper)
    # all-zero states are those before the first step
    t = Tensors([1000], "f32", "f32", False, 8, 5)
    for x in (*t.m, *t.v, *t.m_scale, *t.v_scale):
        x.zero_()
    check_step(B, ctx, t, dict(HYPER, step=1))
    # no gradient: the states stay zero
    t = Tensors([1000], "f32", "f32", False, 8, 5)
    for x in (*t.m, *t.v, *t.m_scale, *t.v_scale, *t.g):
        x.zero_()
    p = t.p[0].clone()
    B.pr_adamw_step(ctx, t.table(B), **HYPER)
    assert not t.m[0].any() and not t.v_scale[0].any() and torch.equal(t.p[0], p)
    t.g[0].fill_(1e-25)  # its square is 0, its first moment is not
    B.pr_adamw_step(ctx, t.table(B), **HYPER)
    assert (t.m[0] == 127).all() and not t.v[0].any() and torch.isfinite(t.p[0]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_nan_and_infinity_stay_in_their_place(B, ctx, bits):
    t = Tensors([256 * 5 + 9], "f32", "f32", False, bits, 6)
    r = Tensors([256 * 5 + 9], "f32", "f32", False, bits, 6)
    t.g[0][300], t.g[0][256 * 5 + 3] = torch.nan, torch.inf
    B.pr_ctx_flags(ctx, clear=True)
    B.pr_adamw_step(ctx, t.table(B), **HYPER)
    assert B.pr_ctx_flags(ctx, clear=True) == (B.PR_FLAG_NONFINITE if bits == 8 else 0)
    B.pr_adamw_step(ctx, r.table(B), **HYPER)
    off = torch.ones(256 * 5 + 9, dtype=torch.bool, device="cuda")
    off[300] = off[256 * 5 + 3] = False
    assert torch.equal(t.p[0][off], r.p[0][off])
    assert torch.isnan(t.p[0][300]) and not torch.isfinite(t.p[0][256 * 5 + 3])
    if bits == 8:
        m, v = B.pr_adamw_unpack(ctx, t.table(B))
        assert torch.isnan(m[1]).all() and torch.isnan(v[1]).all()
        assert torch.isnan(m[5, :9]).all() and not m[5, 9:].any() and not v[5, 9:].any()
        assert torch.isfinite(m[[0, 2, 3, 4]]).all()
        B.pr_ctx_flags(ctx, clear=True)


@pytest.mark.parametrize("start", [0, 1])
def test_unpack_gives_the_held_values(B, ctx, start):
    t = Tensors([1, 300, 0, 256, 70001], "f32", "f32", False, 8, 8, start=start)
    m, v = B.pr_adamw_unpack(ctx, t.table(B))
    assert m.shape == v.shape == (1 + 2 + 1 + 274, 256)
    at = 0
    for qm, sm, qv, sv in zip(t.m, t.m_scale, t.v, t.v_scale):
        n, b = qm.numel(), sm.numel()
        for got, q, s, signed in ((m, qm, sm, True), (v, qv, sv, False)):
            flat = f64(got[at:at + b].reshape(-1))
            want = L.held8(f64(q), f64(s), signed)
            assert np.allclose(flat[:n], want, rtol=3e-7, atol=0) and not flat[n:].any()
        at += b
    # buffers off the 32-byte grid
    buf = torch.full((2 * 278 * 256 + 9,), 7.0, device="cuda")
    m2, v2 = buf[1:1 + 278 * 256], buf[5 + 278 * 256:5 + 2 * 278 * 256]
    B.pr_adamw_unpack(ctx, t.table(B), m=m2, v=v2)
    assert torch.equal(m2, m.reshape(-1)) and torch.equal(v2, v.reshape(-1))
    assert (buf[:1] == 7).all() and (buf[1 + 278 * 256:5 + 278 * 256] == 7).all() and (buf[-4:] == 7).all()


def test_every_code_is_a_fixed_point(B, ctx):
    """beta = 1 - 2^-53 rounds to 1 and its complement to nearly 0: with no gradient a step
    writes back the states that it read."""
    q = torch.arange(256, device="cuda")
    m = [(q - 128).clamp(min=-127).to(torch.int8)]
    v = [q.to(torch.uint8)]
    s = [torch.tensor([0.3], device="cuda")]
    u = [torch.tensor([1.7e-3], device="cuda")]
    p, g = [torch.zeros(256, device="cuda")], [torch.zeros(256, device="cuda")]
    m0, v0 = m[0].clone(), v[0].clone()
    b = 1.0 - 2.0 ** -53
    B.pr_adamw_step(ctx, B.pr_adamw_tensors(p, g, m, v, m_scale=s, v_scale=u), 0.0, beta1=b, beta2=b)
    assert torch.equal(m[0], m0) and torch.equal(v[0], v0)
    assert s[0].item() == np.float32(0.3) and u[0].item() == np.float32(1.7e-3)


def test_bytes_around_the_tensors_stay(B, ctx):
    for bits in (32, 8):
        t = Tensors([301], "bf16", "bf16", False, bits, 9, start=3)
        for x in (t.p, t.m, t.v):
            base = x[0]._base
            base[:3], base[304:] = 5, 5
        B.pr_adamw_step(ctx, t.table(B), **HYPER)
        for x in (t.p, t.m, t.v):
            base = x[0]._base
            assert (base[:3] == 5).all() and (base[304:] == 5).all()


def test_streams_graphs_and_repeats(B, ctx):
    a, b = (Tensors([5000, 77], "bf16", "bf16", True, 32, 4) for _ in range(2))
    c, d = (Tensors([5000, 77], "f32", "f32", False, 8, 4) for _ in range(2))
    ta, tb, tc, td = (t.table(B) for t in (a, b, c, d))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        B.pr_adamw_step(ctx, ta, **HYPER)
        B.pr_adamw_step(ctx, tc, **HYPER)
    with torch.cuda.stream(side):
        B.pr_adamw_step(ctx, tb, **HYPER)
        B.pr_adamw_step(ctx, td, **HYPER)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pr_adamw_step(ctx, tb, **HYPER)
        B.pr_adamw_step(ctx, td, **HYPER)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in ((a, b), (c, d)):
        for name in ("p", "m", "v", "master", "m_scale"):
            for s, t in zip(getattr(x, name) or [], getattr(y, name) or []):
                assert torch.equal(s, t)


def test_refusals(B, ctx):
    t = Tensors([300, 40], "bf16", "bf16", True, 32, 1)
    e = Tensors([300, 40], "f32", "f32", False, 8, 1)
    tab = t.table(B)
    for k in (dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(step=0),
              dict(eps=float("inf"))):
        with pytest.raises(B.PRError) as err:
            B.pr_adamw_step(ctx, tab, **dict(HYPER, **k))
        assert err.value.status == B.PR_ERR_INVALID_ARG
    bad = [
        lambda: B.pr_adamw_tensors(t.p, t.g[:1], t.m, t.v),
        lambda: B.pr_adamw_tensors(t.p, t.g, t.m, t.v, weight_decay=[0.1]),
        lambda: B.pr_adamw_tensors([x.cpu() for x in t.p], t.g, t.m, t.v),
        lambda: B.pr_adamw_tensors([x.half() for x in t.p], t.g, t.m, t.v),
        lambda: B.pr_adamw_tensors(t.p, t.g, [x.double() for x in t.m], t.v),
        lambda: B.pr_adamw_tensors(t.p, t.g, t.m, [x[:-1] for x in t.v]),
        lambda: B.pr_adamw_tensors(e.p, e.g, e.m, e.v),  # codes without scales
        lambda: B.pr_adamw_tensors(e.p, e.g, e.m, t.v, m_scale=e.m_scale, v_scale=e.v_scale),
        lambda: B.pr_adamw_tensors(e.p, e.g, e.m, e.v, m_scale=e.m_scale,
                                   v_scale=[s[:0] for s in e.v_scale]),
        lambda: B.pr_adamw_tensors(e.p, e.g, t.m, t.v, m_scale=e.m_scale, v_scale=e.v_scale),
        lambda: B.pr_adamw_tensors(e.p, e.g, t.m, t.v, master=t.master),
        lambda: B.pr_adamw_tensors([t.p[0].view(30, 10).t()], t.g[:1], t.m[:1], t.v[:1]),
        lambda: B.pr_adamw_step(ctx, [t.p], **HYPER),
        lambda: B.pr_adamw_step(ctx, tab, grad_scale=torch.ones(1), **HYPER),
        lambda: B.pr_adamw_step(ctx, B.pr_adamw_tensors(t.p, t.g, t.m, t.v,
                                                        weight_decay=float("inf")), **HYPER),
        lambda: B.pr_adamw_unpack(ctx, tab),
        lambda: B.pr_adamw_unpack(ctx, e.table(B), m=torch.empty(5, device="cuda")),
    ]
    n0 = B.launch_count()
    for f in bad:
        with pytest.raises(B.PRError) as err:
            f()
        assert err.value.status == B.PR_ERR_INVALID_ARG
    B.pr_adamw_step(ctx, B.pr_adamw_tensors([], [], [], []), **HYPER)
    assert B.launch_count() == n0


@pytest.mark.parametrize("eps", [1e-8, 1e-30])
@pytest.mark.parametrize("scale", [1.0, 1e-10, 1e-12, 3e-13, 1e-13, 3e-14, 1e-15, 1e-17, 1e-18])
def test_codes_of_tiny_second_moments(B, ctx, scale, eps):
    """First steps whose squares go down to the subnormal numbers: v is (1 - beta2) g^2 in two
    rounded products, its code the nearest one.  An IEEE reciprocal, a product and two
    roots put 255 x 2^-22 = 6e-5 onto a code: 1e-4."""
    n = 40 * 256 + 77
    g = torch.Generator(device="cuda").manual_seed(11)
    grad = torch.randn(n, generator=g, device="cuda") * scale
    p = torch.randn(n, generator=g, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    blocks = -(-n // 256)
    ms, vs = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
    t = B.pr_adamw_tensors([p], [grad], [m], [v], m_scale=[ms], v_scale=[vs])
    B.pr_adamw_step(ctx, t, 1e-2, beta1=0.9, beta2=0.95, eps=eps, step=1)
    x = grad.cpu().numpy()
    want = (np.float32(1.0 - 0.95) * (x * x)).astype(np.float64)
    top = np.maximum.reduceat(want, np.arange(0, n, 256))
    top = np.where(top < 2.0 ** -126, 0.0, top)
    assert (f64(vs) == top).all()
    per = np.repeat(top, 256)[:n]
    u = np.where(per > 0, 255.0 * (want / np.where(per > 0, per, 1.0)) ** 0.25, 0.0)
    off = np.abs(f64(v) - u)
    assert (off <= 0.5 + 1e-4).all(), (off.max(), x[off.argmax()])


@pytest.mark.parametrize("bits", [8, 32])
def test_tensor_past_32_bits(B, ctx, bits):
    """Elements beyond the 2^31st take the step that the same elements take by themselves."""
    n, tail = 2 ** 31 + 4096 + 77, 8192 + 77  # the tail begins with a block
    f = torch.float32

    def states(k):
        if bits == 32:
            return [torch.zeros(k, dtype=f, device="cuda") for _ in range(2)], None
        blocks = -(-k // 256)
        return ([torch.zeros(k, dtype=t, device="cuda") for t in (torch.int8, torch.uint8)],
                [torch.zeros(blocks, device="cuda") for _ in range(2)])

    g = torch.Generator(device="cuda").manual_seed(3)
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-tail:] = torch.randn(tail, generator=g, device="cuda").bfloat16()
    grad[-tail:] = torch.randn(tail, generator=g, device="cuda").bfloat16()
    few = [p[-tail:].clone(), grad[-tail:].clone()]
    big_s, big_scale = states(n)
    few_s, few_scale = states(tail)
    for params, gr, (m, v), scale in ((p, grad, big_s, big_scale), (few[0], few[1], few_s, few_scale)):
        t = B.pr_adamw_tensors([params], [gr], [m], [v], weight_decay=0.1,
                               m_scale=[scale[0]] if scale else None,
                               v_scale=[scale[1]] if scale else None)
        for step in (1, 2):
            B.pr_adamw_step(ctx, t, 1e-2, step=step)
    assert torch.equal(p[-tail:], few[0])
    assert not p[:-tail].any()
    for a, b in zip(big_s, few_s):
        assert torch.equal(a[-tail:], b) and not a[:-tail].any()
    if bits == 8:
        for a, b in zip(big_scale, few_scale):
            assert torch.equal(a[-b.numel():], b) and not a[:-b.numel()].any()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("param,grad,master", TYPES)
@pytest.mark.parametrize("start", [8, 16, 24])
def test_starts_on_the_grid_of_the_parameters(B, ctx, param, grad, master, bits, start):
    """Starts at which parameters and gradients fit the wide accesses, and codes, of a byte
    each, may not."""
    t = Tensors(SIZES, param, grad, master, bits, seed=bits + start, start=start)
    check_step(B, ctx, t)
    check_step(B, ctx, t, dict(HYPER, step=8), torch.tensor([0.37], device="cuda"))


@pytest.mark.parametrize("param,grad,master", TYPES)
@pytest.mark.parametrize("off_m,off_v", [(8, 0), (0, 8), (8, 8), (24, 16), (4, 0), (0, 2), (1, 8)])
def test_either_moments_codes_anywhere(B, ctx, param, grad, master, off_m, off_v):
    """Codes at any byte, one moment's or both, give the bits of codes on the grid."""
    a = Tensors([70001, 256, 1000], param, grad, master, 8, 12)
    b = Tensors([70001, 256, 1000], param, grad, master, 8, 12)

    def moved(t, by):
        buf = torch.full((by + t.numel() + 8,), 5, dtype=t.dtype, device="cuda")
        buf[by:by + t.numel()] = t
        return buf[by:by + t.numel()]

    b.m, b.v = [moved(t, off_m) for t in b.m], [moved(t, off_v) for t in b.v]
    for t in (a, b):
        B.pr_adamw_step(ctx, t.table(B), **HYPER)
    for name in ("p", "master", "m", "v", "m_scale", "v_scale"):
        for x, y in zip(getattr(a, name) or [], getattr(b, name) or []):
            assert torch.equal(x, y), name
    for x, y in zip(B.pr_adamw_unpack(ctx, a.table(B)), B.pr_adamw_unpack(ctx, b.table(B))):
        assert torch.equal(x, y)
    for t, by in [(t, off_m) for t in b.m] + [(t, off_v) for t in b.v]:
        assert (t._base[:by] == 5).all() and (t._base[by + t.numel():] == 5).all()


@pytest.mark.parametrize("param,grad,master", TYPES)
def test_tensors_packed_one_behind_the_other(B, ctx, param, grad, master):
    """Tensors of 1,000 elements that share one buffer of each kind: every other one's codes
    lie 8 past a multiple of 16."""
    n, k = 1000, 5
    t = Tensors([n * k], param, grad, master, 8, 13)
    blocks = -(-n // 256)
    g = torch.Generator("cuda").manual_seed(13)
    scales = [0.5 * torch.rand(k * blocks, generator=g, device="cuda") for _ in range(2)]
    t.p, t.g, t.m, t.v = ([x[0][i * n:(i + 1) * n] for i in range(k)] for x in (t.p, t.g, t.m, t.v))
    if t.master:
        t.master = [t.master[0][i * n:(i + 1) * n] for i in range(k)]
    t.m_scale, t.v_scale = ([s[i * blocks:(i + 1) * blocks] for i in range(k)] for s in scales)
    t.wd = [0.1 * (i % 3) for i in range(k)]
    assert t.m[1].data_ptr() % 16 == 8
    check_step(B, ctx, t)
    check_step(B, ctx, t, dict(HYPER, step=8))


@pytest.mark.parametrize("eps", [1e-8, 1e-30])
@pytest.mark.parametrize("top", [1.0e19, 9.2e18, 9.3e18, 1.3e19, 1.84e19])
def test_codes_of_huge_second_moments(B, ctx, top, eps):
    """Gradients whose squares come near the largest number (beta2 0: v is the square, one
    rounded product), among them blocks above 2^126, where the scale's reciprocal is
    subnormal: 21 bits of it are left, which moves a code by 255 x 2^-23 = 3e-5 beside the
    6e-5 of its roots: 1e-4."""
    n = 40 * 256 + 77
    g = torch.Generator(device="cuda").manual_seed(12)
    grad = (top * torch.rand(n, generator=g, device="cuda")).contiguous()
    grad[::256] = top
    p = torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    blocks = -(-n // 256)
    ms, vs = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
    t = B.pr_adamw_tensors([p], [grad], [m], [v], m_scale=[ms], v_scale=[vs])
    B.pr_ctx_flags(ctx, clear=True)
    B.pr_adamw_step(ctx, t, 1e-2, beta1=0.0, beta2=0.0, eps=eps, step=1)
    x = grad.cpu().numpy()
    for got, scale, want, steps, power in ((m, ms, x, 127.0, 0.5), (v, vs, x * x, 255.0, 0.25)):
        want = want.astype(np.float64)
        per = np.maximum.reduceat(want, np.arange(0, n, 256))
        assert (f64(scale) == per).all()
        u = steps * (want / np.repeat(per, 256)[:n]) ** power
        off = np.abs(f64(got) - u)
        assert (off <= 0.5 + 1e-4).all(), (off.max(), x[off.argmax()])
    assert torch.isfinite(p).all() and B.pr_ctx_flags(ctx, clear=True) == 0


def test_states_under_huge_scales_are_kept(B, ctx):
    """States of 3e38 without a gradient: one step gives beta2 v, whatever its code."""
    t = Tensors([2000], "f32", "f32", False, 8, 14)
    t.g[0].zero_()
    t.v_scale[0].fill_(3e38)
    t.v[0][::256] = 255
    for step in (7, 8):
        check_step(B, ctx, t, dict(HYPER, step=step))
    assert (t.v_scale[0] > 2e38).all() and (t.v[0][::256] == 255).all()


@pytest.mark.parametrize("scale", [3e38, 1e-30, 1e-33, 1e-34, 1e-35, 1e-36, 1e-37, 2.0 ** -126])
def test_every_scale_holds_its_values(B, ctx, scale):
    """Every code under scales down to the smallest normal number: the documented value by 3e-7,
    and by what the share of a scale loses where it is subnormal: half of 2^-149 times up to
    (255 / 2^7)^4 = 16 for v, (127 / 2^6)^2 = 4 for m; and the value's own last place."""
    q = torch.arange(256, device="cuda")
    m, v = (q - 128).clamp(min=-127).to(torch.int8), q.to(torch.uint8)
    s = [torch.full((1,), scale, device="cuda") for _ in range(2)]
    z = torch.zeros(256, device="cuda")
    t = B.pr_adamw_tensors([z], [z], [m], [v], m_scale=s[:1], v_scale=s[1:])
    got = B.pr_adamw_unpack(ctx, t)
    for x, codes, signed in ((got[0], m, True), (got[1], v, False)):
        want = L.held8(f64(codes), f64(s[0]), signed)
        assert (np.abs(f64(x[0]) - want) <= 3e-7 * np.abs(want) + 9 * 2.0 ** -149).all()
    # and the step reads the same ones: without a gradient or decay it writes them back
    b = 1.0 - 2.0 ** -53
    m0, v0 = m.clone(), v.clone()
    B.pr_adamw_step(ctx, t, 0.0, beta1=b, beta2=b)
    if scale > 1e-30:  # (below, small codes' values are subnormal)
        assert torch.equal(m, m0) and torch.equal(v, v0)
    assert m[255] == 127 and v[255] == 255
    for x in s:
        assert abs(x.item() / np.float32(scale) - 1.0) <= 1e-6 + (9 * 2.0 ** -149) / scale


def test_tensors_without_elements(B, ctx):
    """They step and expand to nothing, alone and among others."""
    e = Tensors([0, 0], "f32", "f32", False, 8, 1)
    for t in (e.table(B), B.pr_adamw_tensors([], [], [], [])):
        n0 = B.launch_count()
        B.pr_adamw_step(ctx, t, **HYPER)
        m, v = B.pr_adamw_unpack(ctx, t)
        assert m.shape == v.shape == (0, 256) and B.launch_count() == n0
    a, b = Tensors([0, 300, 0], "f32", "f32", False, 8, 1), Tensors([300], "f32", "f32", False, 8, 1)
    a.m[1], a.v[1], a.m_scale[1], a.v_scale[1] = b.m[0], b.v[0], b.m_scale[0], b.v_scale[0]
    for x, y in zip(B.pr_adamw_unpack(ctx, a.table(B)), B.pr_adamw_unpack(ctx, b.table(B))):
        assert x.shape == (2, 256) and torch.equal(x, y)
    # the library itself: no output for tensors that have elements
    t = b.table(B)
    out = torch.empty(2, 256, device="cuda")
    lib, addr = B._lib, B._adamw_table("", 0, t)
    for m, v in ((None, out.data_ptr()), (out.data_ptr(), None)):
        assert lib.pr_adamw_unpack(ctx, addr, 1, m, v, None) == B.PR_ERR_INVALID_ARG
