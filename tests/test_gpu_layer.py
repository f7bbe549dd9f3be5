"""The operators together, as a mixer layer uses them: convolution of q, k and v, l2 norm of q
and k, the delta rule, the gated head norm; forward, backward in the reverse order, and token by
token on the states; on another stream, under capture, and beside the contraction.

Tolerances are norm-wise, max |gpu - ref| / max |ref|: each operator rounds its bf16 outputs
(2^-8) and the delta rule's own bar is 2e-2; five roundings feed it, so 4e-2 for the chain with
bf16 io, 5e-4 with fp32 io (its bar of 1e-4 and the norms' gain, at most 4 here)."""
import pytest
import torch

from paper_2606_01294_amd import ccq

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
B, T, HK, HV, D, W = 2, 100, 2, 4, 64, 4
TOL = {BF: 4e-2, F32: 5e-4}


def params(dt, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    CQ, CV = HK * D, HV * D
    return dict(proj=r(B, T, 2 * CQ + 2 * CV).to(dt),  # q | k | v | output gate
                wq=r(CQ, W) * 0.5, wk=r(CQ, W) * 0.5, wv=r(CV, W) * 0.5, bv=0.1 * r(CV),
                la=-torch.nn.functional.softplus(r(B, T, HV) - 3), be=torch.sigmoid(r(B, T, HV)),
                gn=1 + 0.1 * r(D), dy=r(B, T, HV, D).to(dt))


def split(proj):
    CQ, CV = HK * D, HV * D
    return proj.split([CQ, CQ, CV, CV], -1)


def layer(p, **kw):
    """Forward; the slices of the projection are read where they lie."""
    q, k, v, gate = split(p["proj"])
    q, k, v = (ccq.ccq_conv_fwd(t, p[n], bias=p.get(b), **kw)["y"]
               for t, n, b in ((q, "wq", None), (k, "wk", None), (v, "wv", "bv")))
    q, k = q.view(B, -1, HK, D), k.view(B, -1, HK, D)
    qn, kn = (ccq.ccq_norm_fwd(t, kind=ccq.CCQ_NORM_L2, act=ccq.CCQ_ACT_NONE, **kw) for t in (q, k))
    v = v.view(B, -1, HV, D)
    out = ccq.ccq_delta_fwd(qn, kn, v, p["la"], p["be"], scale=D ** -0.5, **kw)
    gate = gate.unflatten(-1, (HV, D))
    y = ccq.ccq_norm_fwd(out["o"], weight=p["gn"], gate=gate, **kw)
    return y, (q, k, qn, kn, v, out["o"], gate)


def layer_bwd(p, saved, **kw):
    q, k, qn, kn, v, o, gate = saved
    n = ccq.ccq_norm_bwd(o, p["dy"], weight=p["gn"], gate=gate, **kw)
    g = ccq.ccq_delta_fwd_bwd(qn, kn, v, p["la"], p["be"], n["dx"], scale=D ** -0.5, want_o=False, **kw)
    l2 = dict(kind=ccq.CCQ_NORM_L2, act=ccq.CCQ_ACT_NONE)
    dq, dk = (ccq.ccq_norm_bwd(x, d, **l2, **kw)["dx"] for x, d in ((q, g["dq"]), (k, g["dk"])))
    pq, pk, pv, _ = split(p["proj"])
    cq = ccq.ccq_conv_bwd(pq, p["wq"], dq.flatten(2), **kw)
    ck = ccq.ccq_conv_bwd(pk, p["wk"], dk.flatten(2), **kw)
    cv = ccq.ccq_conv_bwd(pv, p["wv"], g["dv"].flatten(2), bias=p["bv"], **kw)
    return dict(proj=torch.cat([cq["dx"], ck["dx"], cv["dx"], n["dgate"].flatten(2)], -1),
                wq=cq["dw"], wk=ck["dw"], wv=cv["dw"], bv=cv["dbias"], la=g["dlogalpha"],
                be=g["dbeta"], gn=n["dweight"])


def reference(p):
    leaf = {n: t.double().requires_grad_() for n, t in p.items() if n != "dy"}

    def conv(x, w, b=0.0):
        e = torch.nn.functional.pad(x, (0, 0, W - 1, 0))
        z = b + sum(w[:, j] * e[:, j:j + T] for j in range(W))
        return z * torch.sigmoid(z)
    q, k, v, gate = split(leaf["proj"])
    q = conv(q, leaf["wq"]).unflatten(-1, (HK, D))
    k = conv(k, leaf["wk"]).unflatten(-1, (HK, D))
    v = conv(v, leaf["wv"], leaf["bv"]).unflatten(-1, (HV, D))
    q, k = (t / torch.sqrt(t.square().sum(-1, keepdim=True) + 1e-5) for t in (q, k))
    q, k = (t.repeat_interleave(HV // HK, 2) for t in (q, k))
    S, outs = torch.zeros(B, HV, D, D).double(), []
    for t in range(T):
        S = S * leaf["la"][:, t].exp()[..., None, None]
        u = leaf["be"][:, t][..., None] * (v[:, t] - (S * k[:, t].unsqueeze(2)).sum(-1))
        S = S + u.unsqueeze(3) * k[:, t].unsqueeze(2)
        outs.append(D ** -0.5 * (S * q[:, t].unsqueeze(2)).sum(-1))
    o = torch.stack(outs, 1)
    gate = gate.unflatten(-1, (HV, D))
    n = o / torch.sqrt(o.square().mean(-1, keepdim=True) + 1e-5)
    y = n * leaf["gn"] * gate * torch.sigmoid(gate)
    grads = torch.autograd.grad(y, list(leaf.values()), p["dy"].double())
    return y.detach(), dict(zip(leaf, grads))


def cuda(p):
    return {n: t.cuda() for n, t in p.items()}


def err(a, r):
    a = a.detach().double().cpu()
    return float((a - r).abs().max() / r.abs().max())


@pytest.mark.parametrize("dt", [BF, F32])
def test_layer_forward_and_backward(dt):
    p = params(dt)
    y, grads = reference(p)
    g = cuda(p)
    got, saved = layer(g)
    back = layer_bwd(g, saved)
    errs = dict({n: err(back[n], grads[n]) for n in grads}, y=err(got, y))
    print("  errors", errs, flush=True)
    assert all(e <= TOL[dt] for e in errs.values()), errs


def test_layer_on_another_stream():
    g = cuda(params(BF))
    want, saved = layer(g)
    back = layer_bwd(g, saved)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for _ in range(3):
        got, sv = layer(g, stream=st)
        st.synchronize()  # (the caller orders what it makes of the outputs between the calls)
        b2 = layer_bwd(g, sv, stream=st)
        st.synchronize()
        assert torch.equal(got, want) and all(torch.equal(b2[n], back[n]) for n in back)


def test_layer_captured_and_replayed():
    """Forward and backward in one graph, replayed over new inputs between eager work; two graphs
    with workspaces of their own do not disturb each other."""
    runs = []
    for seed in (1, 2):
        g = cuda(params(BF, seed))
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            layer_bwd(g, layer(g)[1])
        torch.cuda.current_stream().wait_stream(st)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, saved = layer(g)
            back = layer_bwd(g, saved)
        runs.append((graph, g, y, back))
    for rep in range(3):
        for i, (graph, g, y, back) in enumerate(runs):
            new = cuda(params(BF, 10 + 2 * rep + i))
            for n in g:
                g[n].copy_(new[n])
            graph.replay()
            torch.cuda.synchronize()
            want, saved = layer(new)
            wb = layer_bwd(new, saved)
            torch.cuda.synchronize()
            assert torch.equal(y, want), (rep, i)
            assert all(torch.equal(back[n], wb[n]) for n in wb), (rep, i)


def test_layer_token_by_token():
    """Decoding on the convolutions' and the rule's states against the whole sequence: the
    convolutions and norms give the same bits, the rule's bf16 outputs its bar."""
    g = cuda(params(BF))
    want, saved = layer(g)
    q, k, v, gate = split(g["proj"])
    cs = {n: torch.zeros(B, W - 1, c, dtype=BF, device="cuda")
          for n, c in (("wq", HK * D), ("wk", HK * D), ("wv", HV * D))}
    S = torch.zeros(B, HV, D, D, device="cuda")
    for t in range(T):
        qt, kt, vt = (ccq.ccq_conv_step(x[:, t], g[n], cs[n], bias=g["bv"] if n == "wv" else None)
                      for x, n in ((q, "wq"), (k, "wk"), (v, "wv")))
        assert torch.equal(qt, saved[0][:, t].flatten(1)) and torch.equal(vt, saved[4][:, t].flatten(1))
        qt, kt = (ccq.ccq_norm_fwd(x.view(B, 1, HK, D), kind=ccq.CCQ_NORM_L2, act=ccq.CCQ_ACT_NONE)
                  for x in (qt, kt))
        o = ccq.ccq_delta_step(qt, kt, vt.view(B, 1, HV, D), g["la"][:, t:t + 1].contiguous(),
                               g["be"][:, t:t + 1].contiguous(), S, scale=D ** -0.5)
        y = ccq.ccq_norm_fwd(o, weight=g["gn"], gate=gate[:, t:t + 1].unflatten(-1, (HV, D)))
        ref = want[:, t:t + 1].double()
        assert float((y.double() - ref).abs().max()) <= TOL[BF] * float(want.abs().max())


def test_convolution_and_norm_around_the_contraction():
    """The same neighbours for the framework's CCQ forward: raw q, k from the convolution into
    ccq_fwd_raw, its outputs through the gated norm."""
    H = 4
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = r(B, T, 3 * H * D).cuda()
    w = (r(3 * H * D, W) * 0.5).cuda()
    y = ccq.ccq_conv_fwd(x, w)["y"]
    q, k, v = (t.contiguous().view(B, T, H, D) for t in y.chunk(3, -1))
    wl, bl = (r(H, H * D) * (H * D) ** -0.5).cuda(), r(H).cuda()
    gate = torch.nn.functional.logsigmoid(r(B, T, H, D) + 4).cuda() / 16
    o = ccq.ccq_fwd_raw(q, k, wl, bl, v, gate)["o"]
    og = r(B, T, H, D).cuda()
    z = ccq.ccq_norm_fwd(o, weight=torch.ones(D, device="cuda"), gate=og)
    n = o.double() / torch.sqrt(o.double().square().mean(-1, keepdim=True) + 1e-5)
    ref = n * og.double() * torch.sigmoid(og.double())
    assert float((z.double() - ref).abs().max()) <= 2.0 ** -16 * float(ref.abs().max())
