"""Head norm (ccq_norm_*) against its definition in 64 bits, with autograd for its gradients.

Tolerance, per element: half a step of the stored type plus the fp32 work before it.  A sum over D
channels is formed as a tree (8 in a lane, then halves): its error is below (8 + log2 D) 2^-24
of the sum of sizes; the centred statistics are formed after the subtraction, so a mean that is
large against the spread loses no more than the inputs' own size times 2^-24 over the spread.
n is then off by about 20 2^-24 of max |n| (with |x| / spread < 8 in these inputs: 160 2^-24), and
z, the activation (2^-20 with bf16 io) and the product with the gate keep that order.  The
gradients combine four such factors.  2^-15 of the largest size (bf16 io) and 2^-16 (fp32 io) cover
both; dweight and dbias, fp32 sums of fp32 terms, 2^-15 and 2^-16 of the sum of their terms' sizes."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
KINDS = {"group": 0, "rms": 1, "l2": 2}
ACTS = {"none": 0, "silu": 1, "sigmoid": 2}
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
WORK = {BF: 2.0 ** -15, F32: 2.0 ** -16}


def definition(x, w, b, gate, kind, act, eps):
    if kind == "l2":
        n = x / torch.sqrt(x.square().sum(-1, keepdim=True) + eps)
    else:
        m = x.mean(-1, keepdim=True) if kind == "group" else 0.0
        n = (x - m) / torch.sqrt((x - m).square().mean(-1, keepdim=True) + eps)
    z = n if w is None else n * w
    z = z if b is None else z + b
    u = z if gate is None else gate
    a = {"none": u, "silu": u * torch.sigmoid(u), "sigmoid": torch.sigmoid(u)}[act]
    return (a if gate is None else z * a), n


def make(lead, G, D, dt, kind, affine, shared, gated, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = (r(*lead, G, D) + (2.0 if kind == "group" else 0.0)).to(dt)
    shp = (D,) if shared else (G, D)
    w = 1 + 0.2 * r(*shp) if affine else None
    b = 0.2 * r(*shp) if affine == "bias" else None
    gate = r(*lead, G, D).to(dt) if gated else None
    return x, w, b, gate, r(*lead, G, D).to(dt)


CASES = [  # lead, G, D, dtype, kind, affine, shared, gated, act
    ((1,), 1, 8, BF, "rms", "w", False, True, "silu"),
    ((4,), 8, 256, BF, "rms", "w", True, True, "silu"),
    ((2, 65), 4, 256, BF, "group", "bias", False, False, "silu"),
    ((3, 7), 5, 96, F32, "group", "bias", False, False, "silu"),
    ((1001,), 3, 64, BF, "l2", None, False, False, "none"),
    ((130,), 6, 128, F32, "rms", "bias", True, True, "sigmoid"),
    ((33,), 2, 512, BF, "group", "w", True, True, "silu"),
    ((19,), 1, 520, F32, "rms", "w", False, False, "none"),
    ((9,), 2, 1000, BF, "rms", "bias", True, True, "silu"),
    ((17,), 1, 2048, BF, "rms", "w", False, False, "none"),
    ((5,), 3, 2504, F32, "group", "bias", True, True, "silu"),
    ((6,), 1, 8192, BF, "group", "bias", False, True, "silu"),
    ((4000,), 2, 16, BF, "rms", "bias", False, True, "sigmoid"),
    ((1,), 300, 24, F32, "l2", "w", True, False, "silu"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_forward_and_backward(case):
    lead, G, D, dt, kind, affine, shared, gated, act = case
    x, w, b, gate, dy = make(lead, G, D, dt, kind, affine, shared, gated)
    eps = 1e-5
    leaf = [None if t is None else t.double().requires_grad_() for t in (x, w, b, gate)]
    y, n = definition(*leaf, kind, act, eps)
    names = [m for m, t in zip(("dx", "dweight", "dbias", "dgate"), leaf) if t is not None]
    ref = dict(zip(names, torch.autograd.grad(y, [t for t in leaf if t is not None], dy.double())))
    d = lambda t: None if t is None else t.cuda()  # noqa: E731
    kw = dict(weight=d(w), bias=d(b), gate=d(gate), kind=KINDS[kind], act=ACTS[act], eps=eps)
    got_y = ccq.ccq_norm_fwd(d(x), **kw)
    got = ccq.ccq_norm_bwd(d(x), d(dy), **kw)
    again = ccq.ccq_norm_bwd(d(x), d(dy), **kw)
    torch.cuda.synchronize()
    assert set(got) == set(names)

    def close(a, r, what):
        a = a.cpu().double()
        off = (a - r).abs()
        tol = HALF[dt] * r.abs() + WORK[dt] * r.abs().amax(-1, keepdim=True).clamp_min(
            float(r.abs().max()) / 16)
        print(what, "max off", float(off.max()), "largest", float(r.abs().max()), flush=True)
        assert a.shape == r.shape and bool((off <= tol).all()), (what, float((off - tol).max()))
    close(got_y, y.detach(), "y")
    close(got["dx"], ref["dx"], "dx")
    if gated:
        close(got["dgate"], ref["dgate"], "dgate")
    terms = dy.double().abs()
    if gated:
        terms = terms * gate.double().abs().clamp_min(1)
    over = tuple(range(len(lead) + (1 if shared else 0)))
    for m, f in (("dweight", n.detach().abs()), ("dbias", torch.ones_like(terms))):
        if m in got:
            size = (1.2 * terms * f).sum(over) + 1e-3
            assert bool(((got[m].cpu().double() - ref[m]).abs() <= WORK[dt] * size).all()), m
    assert all(torch.equal(got[m], again[m]) for m in got)  # the same bits every time


@pytest.mark.parametrize("kind", list(KINDS))
def test_rows_of_zeros_and_of_one_value(kind):
    """A head that is zero, or (centred) the same everywhere, has n = 0 exactly and finite
    gradients; NaN stays in its own head."""
    x = torch.zeros(3, 2, 64)
    x[1] = 1.5
    x[2, 0, 5] = float("nan")
    x[2, 1] = torch.randn(64)
    x = x.cuda()
    w = torch.ones(64, device="cuda")
    y = ccq.ccq_norm_fwd(x, weight=w, kind=KINDS[kind], act=0)
    got = ccq.ccq_norm_bwd(x, torch.ones_like(x), weight=w, kind=KINDS[kind], act=0)
    assert bool((y[0] == 0).all()) and bool(torch.isfinite(got["dx"][0]).all())
    if kind == "group":
        assert bool((y[1] == 0).all()) and bool(torch.isfinite(got["dx"][1]).all())
    assert bool(torch.isnan(y[2, 0]).all()) and bool(torch.isfinite(y[2, 1]).all())
    assert bool(torch.isfinite(got["dx"][2, 1]).all())


def test_a_gate_inside_a_wider_projection():
    x, w, b, gate, dy = make((40,), 4, 64, BF, "rms", "w", True, True)
    wide = torch.randn(40, 9, 64, device="cuda").to(BF)
    wide[:, 3:7] = gate.cuda()
    part = wide[:, 3:7]
    xw = torch.zeros(40, 6, 64, device="cuda", dtype=BF)
    xw[:, :4] = x.cuda()
    kw = dict(weight=w.cuda())
    assert torch.equal(ccq.ccq_norm_fwd(xw[:, :4], gate=part, **kw),
                       ccq.ccq_norm_fwd(x.cuda(), gate=gate.cuda(), **kw))
    a = ccq.ccq_norm_bwd(xw[:, :4], dy.cuda(), gate=part, **kw)
    c = ccq.ccq_norm_bwd(x.cuda(), dy.cuda(), gate=gate.cuda(), **kw)
    assert all(torch.equal(a[n], c[n]) for n in a)


def test_no_rows():
    x = torch.zeros(0, 2, 64, device="cuda", dtype=BF)
    w, b = torch.ones(2, 64, device="cuda"), torch.ones(2, 64, device="cuda")
    assert ccq.ccq_norm_fwd(x, weight=w, bias=b).shape == (0, 2, 64)
    got = ccq.ccq_norm_bwd(x, x, weight=w, bias=b)
    assert bool((got["dweight"] == 0).all()) and bool((got["dbias"] == 0).all())


def test_refusals():
    x = torch.zeros(4, 2, 64, device="cuda", dtype=BF)
    w = torch.ones(2, 64, device="cuda")
    with pytest.raises(ValueError):
        ccq.ccq_norm_fwd(x, weight=torch.ones(3, 64, device="cuda"))
    with pytest.raises(TypeError):
        ccq.ccq_norm_fwd(x, weight=w.to(BF))
    with pytest.raises(ValueError):
        ccq.ccq_norm_fwd(x, weight=w, out=x)
    with pytest.raises(ValueError):
        ccq.ccq_norm_fwd(x, gate=x[:3])
    with pytest.raises(ccq.CcqError):
        ccq.ccq_norm_fwd(x, bias=w)
    with pytest.raises(ccq.CcqError):
        ccq.ccq_norm_fwd(x[..., :60].contiguous())


def slope(loss, args, i, v, h=2.0 ** -6):
    """Derivative of the loss along v in args[i] from four points (off by h^4 / 30 of the fifth)."""
    def at(k):
        return loss(*[a + k * h * v if j == i else a for j, a in enumerate(args)])
    return (8 * (at(1) - at(-1)) - (at(2) - at(-2))) / (12 * h)


@pytest.mark.parametrize("kind,gated,act", [("group", False, "silu"), ("rms", True, "silu"),
                                            ("l2", True, "sigmoid"), ("group", True, "none")])
def test_gradient_against_differences(kind, gated, act):
    """fp32 io.  Every y is off by 2^-18 at most (the tolerance above, a quarter of it a step's
    difference), which 18 / 12 over 2^-6 makes 2^-12 of the sum of |dy|; the fifth derivative along
    a step of a hundredth of the inputs adds less than 2^-10 of the slope."""
    x, w, b, gate, dy = [t if t is None else t.cuda() for t in
                         make((3,), 2, 40, F32, kind, "bias", True, gated)]
    args = [x, w, b] + ([gate] if gated else [])
    kw = dict(kind=KINDS[kind], act=ACTS[act])
    got = ccq.ccq_norm_bwd(x, dy, weight=w, bias=b, gate=gate, **kw)

    def loss(x, w, b, gate=None):
        y = ccq.ccq_norm_fwd(x, weight=w, bias=b, gate=gate, **kw)
        return float((y.double() * dy.double()).sum())
    for i, n in enumerate(("dx", "dweight", "dbias", "dgate")[:len(args)]):
        g = torch.Generator(device="cuda").manual_seed(i)
        v = got[n] / got[n].square().mean().sqrt() + torch.randn(args[i].shape, generator=g, device="cuda")
        num, ana = slope(loss, args, i, v), float((got[n].double() * v.double()).sum())
        print(n, num, ana, flush=True)
        assert abs(num - ana) <= 2.0 ** -12 * float(dy.abs().sum()) + 2.0 ** -10 * abs(ana), n
