"""The plain gated delta rule (ccq_delta_*) against the recurrence itself in 64 bits, with
autograd for the gradients.

The bar is the framework's own: max |gpu - ref| / max |ref| per tensor, 1e-4 with fp32 io and
2e-2 with bf16 io, whose products take bf16 operands (a handful of 2^-9 roundings each).  The
final state is held in fp32 whatever the io dtype is: its products take their operands to 2^-17,
four of them a chunk, and the decays are differences of running sums (2^-24 |gamma|, |gamma| < 50
here): 2e-5."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TOL = {BF: 2e-2, F32: 1e-4}
STATE = 2e-5


def recurrence(q, k, v, la, be, S, scale):
    """One sequence, [T, H, d] float64 (q, k already one per value head)."""
    outs = []
    for t in range(q.shape[0]):
        S = S * la[t].exp()[:, None, None]
        u = be[t][:, None] * (v[t] - (S * k[t][:, None]).sum(-1))
        S = S + u[:, :, None] * k[t][:, None]
        outs.append(scale * (S * q[t][:, None]).sum(-1))
    return (torch.stack(outs) if outs else v[:0]), S


def make(lens, HK, HV, dk, dv, dt, state, gates="mild", seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    n = sum(lens)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    d = dict(q=unit(r(n, HK, dk)).to(dt), k=unit(r(n, HK, dk) + 0.5 * r(HK, dk)).to(dt),
             v=r(n, HV, dv).to(dt), la=-torch.nn.functional.softplus(r(n, HV) - 3),
             be=torch.sigmoid(r(n, HV)), dO=r(n, HV, dv).to(dt))
    if gates == "strong":
        d["la"] = -torch.nn.functional.softplus(r(n, HV)) * 0.5
    if gates == "resets":
        d["la"][torch.rand(n, HV, generator=g) < 0.05] = -float("inf")
    if gates == "still":
        d["la"] = torch.zeros(n, HV)
        d["be"] = torch.ones(n, HV)
    d["S"] = 0.2 * r(len(lens), HV, dv, dk) if state else None
    return d


def solve(d, lens, scale, grads):
    HK, HV = d["q"].shape[1], d["v"].shape[1]
    leaf = {n: d[n].double().requires_grad_(grads) for n in ("q", "k", "v", "la", "be")}
    G = HV // HK
    outs, ends, at = [], [], 0
    for b, n in enumerate(lens):
        x = {m: t[at:at + n] for m, t in leaf.items()}
        dv, dk = d["v"].shape[2], d["q"].shape[2]
        S = d["S"][b].double() if d["S"] is not None else torch.zeros(HV, dv, dk).double()
        o, S = recurrence(x["q"].repeat_interleave(G, 1), x["k"].repeat_interleave(G, 1), x["v"],
                          x["la"], x["be"], S, scale)
        outs.append(o)
        ends.append(S)
        at += n
    o = torch.cat(outs)
    res = dict(o=o.detach(), ST=torch.stack(ends).detach())
    if grads:
        got = torch.autograd.grad(o, list(leaf.values()), d["dO"].double(), allow_unused=True,
                                  materialize_grads=True)
        res.update(zip(("dq", "dk", "dv", "dlogalpha", "dbeta"), got))
    return res


def check(got, ref, tol, names=None):
    errs = {}
    for n in names or ref:
        r = ref[n]
        a = got[n].detach().double().cpu().reshape(r.shape)
        assert bool(torch.isfinite(a).all()), n
        big = float(r.abs().max()) if r.numel() else 0.0
        off = float((a - r).abs().max()) if r.numel() else 0.0
        errs[n] = off / big if big else off
    print("  errors", errs, flush=True)
    bad = {n: e for n, e in errs.items() if e > (min(tol, STATE) if n == "ST" else tol)}
    assert not bad, bad


def dev(d, shp=None):
    return [d[n].cuda() if shp is None else d[n].cuda().view(*shp, *d[n].shape[1:])
            for n in ("q", "k", "v", "la", "be")]


FWD = [  # B, T, HK, HV, dk, dv, dtype, state, gates
    (1, 1, 1, 1, 64, 64, BF, True, "mild"),
    (2, 63, 1, 2, 64, 128, BF, False, "mild"),
    (1, 64, 2, 2, 128, 64, BF, True, "mild"),
    (2, 65, 2, 6, 128, 128, BF, True, "strong"),
    (1, 200, 1, 3, 256, 256, BF, True, "mild"),
    (1, 130, 2, 2, 256, 512, BF, False, "resets"),
    (3, 257, 4, 4, 128, 256, BF, False, "still"),
    (2, 130, 3, 3, 64, 64, F32, True, "mild"),
    (1, 70, 1, 2, 128, 128, F32, True, "resets"),
    (17, 66, 2, 4, 64, 512, BF, True, "mild"),
    (9, 129, 4, 8, 128, 256, BF, True, "mild"),
]


@pytest.mark.parametrize("case", FWD, ids=lambda c: "-".join(map(str, c)))
def test_forward(case):
    B, T, HK, HV, dk, dv, dt, state, gates = case
    d = make([T] * B, HK, HV, dk, dv, dt, state, gates)
    ref = solve(d, [T] * B, 0.7, False)
    S0 = d["S"].cuda() if state else None
    got = ccq.ccq_delta_fwd(*dev(d, (B, T)), S0=S0, scale=0.7)
    check(got, ref, TOL[dt])
    if state:  # the final state over the initial one
        again = ccq.ccq_delta_fwd(*dev(d, (B, T)), S0=S0, scale=0.7, want_states=False)
        assert set(again) == {"o"} and torch.equal(again["o"], got["o"])


TRAIN = [
    (1, 1, 1, 1, 64, 64, BF, False, "mild"),
    (2, 65, 1, 3, 64, 64, F32, True, "mild"),
    (1, 130, 2, 2, 128, 128, BF, True, "mild"),
    (2, 100, 2, 4, 128, 256, BF, False, "strong"),
    (1, 129, 1, 2, 256, 256, BF, True, "mild"),
    (2, 70, 2, 2, 64, 512, BF, True, "resets"),
]


@pytest.mark.parametrize("case", TRAIN, ids=lambda c: "-".join(map(str, c)))
def test_training_step(case):
    B, T, HK, HV, dk, dv, dt, state, gates = case
    d = make([T] * B, HK, HV, dk, dv, dt, state, gates)
    ref = solve(d, [T] * B, 0.7, True)
    x = dev(d, (B, T))
    dO = d["dO"].cuda().view(B, T, HV, dv)
    kw = dict(S0=d["S"].cuda() if state else None, scale=0.7)
    got = ccq.ccq_delta_fwd_bwd(*x, dO, want_states=True, **kw)
    check(got, ref, TOL[dt])
    fwd = ccq.ccq_delta_fwd(*x, **kw)
    assert torch.equal(fwd["o"], got["o"]) and torch.equal(fwd["ST"], got["ST"])
    less = ccq.ccq_delta_fwd_bwd(*x, dO, want_o=False, **kw)
    assert set(less) == set(got) - {"o", "ST"}
    assert all(torch.equal(less[n], got[n]) for n in less)


@pytest.mark.parametrize("HK,HV,dk,dv,dt", [(2, 4, 128, 128, BF), (2, 2, 64, 64, F32),
                                            (1, 3, 256, 256, BF)])
def test_packed(HK, HV, dk, dv, dt):
    """Sequences of every awkward length (none, one, a chunk and one) as if each were alone; rows
    behind the last one are left as they were."""
    lens = [65, 0, 1, 64, 130, 0, 3]
    d = make(lens, HK, HV, dk, dv, dt, True)
    ref = solve(d, lens, 1.0, True)
    n, behind = sum(lens), 6
    cu = torch.tensor([0] + [sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32).cuda()
    wide = {m: torch.cat([t, torch.ones(behind, *t.shape[1:], dtype=t.dtype)])
            for m, t in d.items() if m != "S"}
    x = dev(wide)
    o = torch.full_like(x[2], 3.0)
    got = ccq.ccq_delta_fwd_varlen(*x, cu, max(lens), S0=d["S"].cuda(), out=dict(o=o))
    assert bool((got["o"][n:] == 3.0).all())
    check(dict(o=got["o"][:n], ST=got["ST"]), ref, TOL[dt], ("o", "ST"))
    marks = {m: torch.full(s, 3.0, dtype=dt, device="cuda") for m, s in
             (("dq", x[0].shape), ("dk", x[0].shape), ("dv", x[2].shape), ("o", x[2].shape),
              ("dlogalpha", x[3].shape), ("dbeta", x[3].shape))}
    got = ccq.ccq_delta_fwd_bwd_varlen(*x, wide["dO"].cuda(), cu, max(lens), S0=d["S"].cuda(),
                                       out=marks)
    for m in marks:
        assert bool((got[m][n:] == 3.0).all()), m
    check({m: t[:n] for m, t in got.items()}, ref, TOL[dt], list(marks))


@pytest.mark.parametrize("T", [0, 1, 5])
@pytest.mark.parametrize("HK,HV,dk,dv,dt", [(2, 4, 128, 128, BF), (1, 1, 64, 64, F32),
                                            (3, 3, 256, 512, BF), (2, 6, 256, 64, F32)])
def test_step(T, HK, HV, dk, dv, dt):
    B = 3
    d = make([T] * B, HK, HV, dk, dv, dt, True, "resets")
    ref = solve(d, [T] * B, 0.7, False)
    S = d["S"].cuda()
    o = ccq.ccq_delta_step(*dev(d, (B, T)), S, scale=0.7)
    check(dict(o=o, ST=S), ref, TOL[dt])


def test_prefill_then_steps():
    """The chunked form's final state carries no rounding of its own: 40 recurrent steps from it
    stay as near the recurrence as steps from the exact state."""
    B, T, n = 2, 200, 40
    d = make([T + n] * B, 2, 4, 128, 128, BF, False)
    ref = solve(d, [T + n] * B, 1.0, False)
    x = dev(d, (B, T + n))
    S = ccq.ccq_delta_fwd(*[t[:, :T].contiguous() for t in x])["ST"]
    outs = [ccq.ccq_delta_step(*[t[:, i:i + 1].contiguous() for t in x], S) for i in range(T, T + n)]
    got = torch.cat(outs, 1).double().cpu()
    want = ref["o"].view(B, T + n, 4, 128)[:, T:]
    # a stored bf16 value is off by half a step of its own
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + STATE * float(want.abs().max())).all())
    check(dict(ST=S), ref, STATE, ("ST",))


def test_final_state_over_the_initial_one():
    d = make([100], 1, 2, 128, 64, BF, True)
    x = dev(d, (1, 100))
    S = d["S"].cuda()
    want = ccq.ccq_delta_fwd(*x, S0=S)
    shape = ccq.make_delta_shape(1, 100, 1, 2, 128, 64, BF)
    ws = torch.empty(ccq.ccq_delta_workspace_size(shape), dtype=torch.uint8, device="cuda")
    o = torch.empty_like(x[2])
    ccq._launch("ccq_delta_fwd", x[0].device, None, shape, x + [S, o, S], ws)
    assert torch.equal(S, want["ST"]) and torch.equal(o, want["o"])


def test_matches_the_contraction_free_forward():
    """lambda = 0 in the framework's own Gated DeltaNet forward is the same rule."""
    d = make([150, 150], 2, 2, 128, 128, F32, False)
    x = dev(d, (2, 150))
    a = ccq.ccq_delta_fwd(*x)
    b = ccq.ccq_gdn_fwd(*x, torch.zeros(2, 150, 2, device="cuda"))
    assert float((a["o"] - b["o"]).abs().max()) <= 1e-6 and float((a["ST"] - b["ST"]).abs().max()) <= 1e-6


def test_refusals():
    d = make([8], 1, 2, 64, 64, BF, True)
    q, k, v, la, be = dev(d, (1, 8))
    with pytest.raises(TypeError):
        ccq.ccq_delta_fwd(q, k, v, la.to(BF), be)
    with pytest.raises(ValueError):
        ccq.ccq_delta_fwd(q, k, v, la[..., :1].contiguous(), be)
    with pytest.raises(ValueError):
        ccq.ccq_delta_fwd(q, k, v, la, be, out=dict(o=v))
    with pytest.raises(ValueError):
        ccq.ccq_delta_fwd(q, k, v, la, be, S0=d["S"].cuda()[:, :1].contiguous())
    with pytest.raises(ccq.CcqError):
        ccq.ccq_delta_fwd(q, k, v, la, be, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        ccq.ccq_delta_step(q, k, v, la, be, None)


@pytest.mark.parametrize("dk,dv,dt", [(128, 256, BF), (256, 256, BF), (64, 64, F32), (64, 128, BF)])
@pytest.mark.parametrize("poison", [float("nan"), float("inf")])
def test_poison_stays_in_its_sequence(dk, dv, dt, poison):
    """Infinities and NaN in one sequence, in the rows behind the last one, and in another value
    head change no bit of the others' results; ahead of a poisoned token's chunk o is as it was."""
    lens, HK, HV = [70, 33, 130, 5], 2, 4
    d = make(lens, HK, HV, dk, dv, dt, True)
    n = sum(lens)
    cu = torch.tensor([0] + [sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32).cuda()
    clean = {m: torch.cat([t, torch.zeros(7, *t.shape[1:], dtype=t.dtype)])
             for m, t in d.items() if m != "S"}
    dirty = {m: t.clone() for m, t in clean.items()}
    for t in dirty.values():
        t[70:103] = poison
        t[n:] = poison
    S0 = d["S"].cuda()
    kw = dict(S0=S0, want_states=True)
    call = lambda t: ccq.ccq_delta_fwd_bwd_varlen(*dev(t), t["dO"].cuda(), cu, max(lens), **kw)  # noqa: E731
    want, got = call(clean), call(dirty)
    for m in want:
        a, b = (want[m], got[m]) if m == "ST" else (want[m][:n], got[m][:n])
        keep = [0, 2, 3] if m == "ST" else list(range(70)) + list(range(103, n))
        assert torch.equal(a[keep], b[keep]), m
    # a value head of the third sequence, from its token 64 on
    dirty = {m: t.clone() for m, t in clean.items()}
    dirty["v"][103 + 64, 1, 3] = poison
    got = call(dirty)
    heads = [0, 2, 3]
    for m in ("o", "dv", "dlogalpha", "dbeta"):
        assert torch.equal(want[m][:n, heads], got[m][:n, heads]), m
    assert torch.equal(want["ST"][:, heads], got["ST"][:, heads])
    assert torch.equal(want["o"][:103 + 64], got["o"][:103 + 64])
    assert not bool(torch.isfinite(got["o"][103 + 64, 1]).all())


@pytest.mark.parametrize("HK,HV", [(1, 1), (1, 2)])
def test_gradient_against_differences(HK, HV):
    """fp32 io, four points along a direction that holds the gradient itself.  o is off by 1e-6 of
    its norm, which 18 / 12 over a step of 2^-6 makes 2^-13 of |dO| |o|; the fifth derivative
    along a step of a fiftieth of the inputs adds less than 2^-10 of the slope."""
    T, h = 66, 2.0 ** -6
    d = make([T], HK, HV, 64, 64, F32, True)
    args, dO, S0 = dev(d, (1, T)), d["dO"].cuda().view(1, T, HV, 64), d["S"].cuda()
    got = ccq.ccq_delta_fwd_bwd(*args, dO, S0=S0)

    def loss(i, x):
        o = ccq.ccq_delta_fwd(*[x if j == i else a for j, a in enumerate(args)], S0=S0)["o"]
        return float((o.double() * dO.double()).sum())
    size = float(dO.norm() * got["o"].norm())
    for i, n in enumerate(("dq", "dk", "dv", "dlogalpha", "dbeta")):
        g = torch.Generator(device="cuda").manual_seed(i)
        v = got[n] / got[n].square().mean().sqrt() + torch.randn(args[i].shape, generator=g, device="cuda")
        v = v * (0.125 if i < 2 else 0.5 if i > 2 else 1.0)  # a q or k element is 2^-3, a beta 2^-1
        at = {k: loss(i, args[i] + k * h * v) for k in (-2, -1, 1, 2)}
        num = (8 * (at[1] - at[-1]) - (at[2] - at[-2])) / (12 * h)
        ana = float((got[n].double() * v.double()).sum())
        print(n, num, ana, flush=True)
        assert abs(num - ana) <= 2.0 ** -13 * size + 2.0 ** -10 * abs(ana), n


@pytest.mark.parametrize("lens,HK,HV,dk,dv,state,gates", [
    ([1], 1, 1, 64, 64, False, "mild"), ([1], 1, 1, 256, 256, True, "mild"),
    ([1, 1, 1], 2, 6, 128, 64, True, "resets"), ([2], 1, 1, 128, 128, False, "mild"),
    ([3, 3], 1, 2, 64, 512, True, "strong"), ([17], 1, 3, 128, 256, True, "mild"),
    ([16] * 4, 2, 2, 64, 128, False, "still"), ([64], 1, 2, 256, 64, True, "mild"),
    ([7, 0, 1, 9, 2], 1, 2, 128, 128, True, "resets"), ([0, 3], 2, 2, 256, 256, False, "mild")])
def test_gradients_of_a_few_tokens(lens, HK, HV, dk, dv, state, gates):
    """Up to 64 tokens (128 times value heads) the gradients are formed in fp32: half a step of bf16 and
    the sums' own work, a few 2^-22 of their terms, each at most a row of dO against a row of v
    (or of the state, or of both): 2^-18 of the norms' product."""
    d = make(lens, HK, HV, dk, dv, BF, state, gates)
    ref = solve(d, lens, 0.7, True)
    n = sum(lens)
    work = 2.0 ** -18 * float(d["dO"].double().norm(dim=-1).max()) * (
        1 + float(d["v"].double().norm(dim=-1).max()) + (float(d["S"].double().norm(dim=(-2, -1)).max()) if state else 0))
    kw = dict(S0=d["S"].cuda() if state else None, scale=0.7)
    names = ("dq", "dk", "dv", "dlogalpha", "dbeta")

    def held(got):
        for m in names:
            a, r = got[m].double().cpu().reshape(ref[m].shape), ref[m]
            off = (a - r).abs() - 2.0 ** -8 * r.abs()
            print(m, float(off.max()) if n else 0, work, flush=True)
            assert bool((off <= work * (HV // HK)).all()), m
    cu = torch.tensor([0] + [sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32).cuda()
    wide = {m: torch.cat([t, torch.full((4, *t.shape[1:]), float("nan"), dtype=t.dtype)])
            for m, t in d.items() if m != "S"}
    out = {m: torch.full((n + 4, *ref[m].shape[1:]), 3.0, dtype=BF, device="cuda") for m in names}
    ccq.ccq_delta_fwd_bwd_varlen(*dev(wide), wide["dO"].cuda(), cu, max(lens), out=out, want_o=False, **kw)
    assert all(bool((out[m][n:] == 3.0).all()) for m in names)
    held({m: t[:n] for m, t in out.items()})
    if len(set(lens)) == 1:
        B, T = len(lens), lens[0]
        got = ccq.ccq_delta_fwd_bwd(*dev(d, (B, T)), d["dO"].cuda().view(B, T, HV, dv), want_states=True, **kw)
        held(got)
        assert all(torch.equal(got[m].view_as(out[m][:n]), out[m][:n]) for m in names)
        check(got, ref, TOL[BF], ("o", "ST"))
        fwd = ccq.ccq_delta_fwd(*dev(d, (B, T)), **kw)
        assert torch.equal(fwd["o"], got["o"]) and torch.equal(fwd["ST"], got["ST"])
