"""The operators of a Gated DeltaNet / GLA token mixer around its query contraction, as cases.

A mixer layer reads the projections of a token through a short causal convolution, writes and
reads the fast-weight state by the gated delta rule, and normalises every head's output under
an output gate.  Three operators, each forward, backward and for a single token:

* conv   y_t = act(bias + sum_j w_j x_{t-W+1+j}), one filter of W taps per channel, with the
         last W-1 inputs of every sequence as its state;
* delta  S_t = a_t S_{t-1} (I - b_t k_t k_t^T) + b_t v_t k_t^T,  o_t = scale S_t q_t  (the plain
         rule, without the contraction; value heads may share a query/key head);
* norm   group norm over each head's channels, y = n(x) act(gate) or act(n(x)).

With `own` false, run() is the same mathematics in elementary torch operations, 32 bits wide
(the delta rule in chunks, whose corrected values solve a triangular system).  exact() is in 64
bits and by other means: the delta rule one token at a time, with the reverse recurrence for its
gradient; the other gradients by autograd.  Sizes are those of the 500M GLA layer (dk=128,
dv=256) and the 1.3B Gated DeltaNet layer (dk=dv=256) of this repository's benchmark, and odd
ones.
"""
from __future__ import annotations

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
KINDS = {"group": 0, "rms": 1, "l2": 2}
ACTS = {"none": 0, "silu": 1, "sigmoid": 2}
EPS = 1e-5


def listed():
    return [
        # norm ------------------------------------------------------------------------------
        # The output norm of one decode step (batch 4, 1.3B layer): latency.
        _norm("norm_decode", "fwd", 4, 8, 256, "rms", "silu", gate=True, shared=True),
        # The same over a training batch (4 x 4096 tokens), gated, one weight for all heads.
        _norm("norm_t4k", "fwd", 16384, 8, 256, "rms", "silu", gate=True, shared=True),
        # Its backward.
        _norm("norm_bwd_t4k", "bwd", 16384, 8, 256, "rms", "silu", gate=True, shared=True),
        # Group norm with mean and bias, a weight for every channel, activation on the result,
        # full precision, an odd number of tokens and a head size that is no power of two.
        _norm("norm_bwd_group_fp32", "bwd", 4099, 5, 96, "group", "silu", gate=False, shared=False,
              dtype="fp32"),
        # conv ------------------------------------------------------------------------------
        # One decode step of the GLA layer's q, k and v channels (4 heads, batch 8): latency.
        _conv("conv_step", "step", 8, 1, 2048, 4),
        # q, k and v of the 1.3B layer over its 4K context.
        _conv("conv_t4k", "fwd", 4, 4096, 6144, 4),
        # The backward on packed documents of different lengths, with initial states.
        _conv("conv_bwd_packed", "bwd", 8, 2048, 2048, 4, packed=True, state=True),
        # delta -----------------------------------------------------------------------------
        # Full precision, ragged, from a state: checking runs and small models.
        _delta("delta_fp32_ragged", "fwd", 2, 333, 2, 2, 64, 64, dtype="fp32", state=True),
        # Prefill / evaluation of the 1.3B layer at its 4K context.
        _delta("delta_t4k", "fwd", 4, 4096, 8, 8, 256, 256),
        # The training step of that layer.
        _delta("delta_train_t4k", "train", 4, 4096, 8, 8, 256, 256),
        # Training on packed documents, two value heads on every query/key head.
        _delta("delta_train_packed", "train", 8, 2048, 4, 8, 128, 128, packed=True, state=True),
        # One token of a serving batch on its states.
        _delta("delta_step_b64", "step", 64, 1, 8, 8, 256, 256, state=True),
    ]


def _norm(name, call, rows, G, D, kind, act, gate, shared, dtype="bf16"):
    return _named(name, op="norm", call=call, rows=rows, G=G, D=D, kind=kind, act=act, gate=gate,
                  shared=shared, dtype=dtype)


def _conv(name, call, B, T, C, W, act="silu", bias=True, packed=False, state=False, dtype="bf16"):
    return _named(name, op="conv", call=call, B=B, T=T, C=C, W=W, act=act, bias=bias,
                  packed=packed, state=state, dtype=dtype)


def _delta(name, call, B, T, HK, HV, dk, dv, packed=False, state=False, dtype="bf16"):
    return _named(name, op="delta", call=call, B=B, T=T, HK=HK, HV=HV, dk=dk, dv=dv,
                  packed=packed, state=state, dtype=dtype)


def _named(name, **case):
    if name:
        case["name"] = name
    return case


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["norm", "conv", "delta"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if op == "norm":
        D = rng.choice([64, 128, 256, 512, 8 * rng.randint(1, 256)])
        G = rng.choice([1, 2, 3, 4, 5, 8, 16])
        rows = _log_int(rng, 1, max(1, min(16384, 33554432 // (G * D))))
        return _norm(None, rng.choice(["fwd", "bwd"]), rows, G, D, rng.choice(list(KINDS)),
                     rng.choice(list(ACTS)), rng.random() < 0.5, rng.random() < 0.5, dtype)
    if op == "conv":
        call = rng.choice(["fwd", "bwd", "step"])
        C, W = 8 * _log_int(rng, 8, 1024), rng.choice([2, 3, 4, 4])
        act, bias = rng.choice(list(ACTS)), rng.random() < 0.5
        if call == "step":
            return _conv(None, call, _log_int(rng, 1, 256), 1, C, W, act, bias, dtype=dtype)
        B = rng.randint(1, 8)
        T = _log_int(rng, 1, max(1, min(4096, 67108864 // (B * C))))
        return _conv(None, call, B, T, C, W, act, bias, rng.random() < 0.4, rng.random() < 0.5,
                     dtype)
    call = rng.choice(["fwd", "train", "step"])
    dk, dv = rng.choice([(64, 64), (64, 128), (128, 128), (128, 256), (256, 256)])
    if dtype == "fp32" and call != "step":
        dk = 64 if call == "train" else min(dk, 128)
    HK = rng.choice([1, 2, 3, 4, 6, 8])
    HV = HK * rng.choice([1, 1, 2, 3])
    if call == "step":
        B = _log_int(rng, 1, max(1, min(64, 1024 // HV)))
        return _delta(None, call, B, rng.choice([1, 1, 1, 2, 3, 5]), HK, HV, dk, dv, state=True,
                      dtype=dtype)
    B = rng.randint(1, 4)
    T = _log_int(rng, 1, max(1, min(4096, 100000 // (B * HV))))
    if dtype == "fp32":
        T = min(T, 1000)
    return _delta(None, call, B, T, HK, HV, dk, dv, rng.random() < 0.4, rng.random() < 0.5, dtype)


def _lengths(case):
    """Lengths of a packed batch's sequences: the first is T, the others spread down to T / 3;
    the same for every seed."""
    B, T = case["B"], case["T"]
    lens = [max(0, T - (T * 2 // 3) * ((5 * b + 3) % 8) // 8 - b) for b in range(B)]
    lens[0] = T
    return lens


def _tokens(case):
    return sum(_lengths(case)) if case["packed"] else case["B"] * case["T"]


# ---------------------------------------------------------------------------------------
# Inputs.

class _Draw:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)

    def __call__(self, *shape, mul=1.0, add=0.0):
        return torch.randn(*shape, generator=self.gen, device="cuda") * mul + add


def _unit(x):
    return x / x.norm(dim=-1, keepdim=True).clamp_min(1e-12)


def _inputs(case, seed):
    r, dt = _Draw(seed), DTYPES[case["dtype"]]
    s = {}
    if case["op"] == "norm":
        rows, G, D = case["rows"], case["G"], case["D"]
        # Head outputs have scales of their own and, for the centred kind, a mean.
        scale = torch.exp(r(1, G, 1, mul=0.5))
        s["x"] = (r(rows, G, D, add=0.3 if case["kind"] == "group" else 0.0) * scale).to(dt)
        s["gate"] = r(rows, G, D).to(dt) if case["gate"] else None
        wshape = (D,) if case["shared"] else (G, D)
        s["w"] = r(*wshape, mul=0.1, add=1.0) if case["kind"] != "l2" else None
        s["bias"] = r(*wshape, mul=0.1) if case["kind"] == "group" else None
        if case["call"] == "bwd":
            s["dy"] = r(rows, G, D).to(dt)
        return s
    B, T, dev = case["B"], case["T"], "cuda"
    if case["packed"]:
        off = [0]
        for n in _lengths(case):
            off.append(off[-1] + n)
        s["cu"] = torch.tensor(off, dtype=torch.int32, device=dev)
        tok = (off[-1],)
    else:
        tok = (B, T)
    if case["op"] == "conv":
        C, W = case["C"], case["W"]
        if case["call"] == "step":
            tok = (B,)
        s["x"] = r(*tok, C).to(dt)
        s["w"] = r(C, W, mul=W ** -0.5)
        s["bias"] = r(C, mul=0.1) if case["bias"] else None
        state = case["state"] or case["call"] == "step"
        s["state"] = r(B, W - 1, C).to(dt) if state else None
        if case["call"] == "bwd":
            s["dy"] = r(*tok, C).to(dt)
        return s
    HK, HV, dk, dv = case["HK"], case["HV"], case["dk"], case["dv"]
    # Unit queries and keys, keys about a common direction of their head; gates near those of
    # trained layers (alpha about 0.95, beta about 0.5).
    common = 0.5 * dk ** 0.5 * _unit(r(HK, dk))
    s["q"] = _unit(r(*tok, HK, dk)).to(dt)
    s["k"] = _unit(r(*tok, HK, dk) + common).to(dt)
    s["v"] = r(*tok, HV, dv).to(dt)
    s["la"] = -torch.nn.functional.softplus(r(*tok, HV, add=-3.0))
    s["beta"] = torch.sigmoid(r(*tok, HV))
    s["S"] = r(B, HV, dv, dk, mul=0.1) if case["state"] else None
    if case["call"] == "train":
        s["dO"] = r(*tok, HV, dv).to(dt)
    return s


def prepare(case, seed):
    return dict(_inputs(case, seed), case=dict(case))


# ---------------------------------------------------------------------------------------
# One pass.

def run(s):
    return _run_own(s) if own else _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    from paper_2606_01294_amd import ccq
    c = s["case"]
    call = c["call"]
    if c["op"] == "norm":
        kw = dict(weight=s["w"], bias=s["bias"], gate=s["gate"], kind=KINDS[c["kind"]],
                  act=ACTS[c["act"]], eps=EPS)
        if call == "fwd":
            return ccq.ccq_norm_fwd(s["x"], **kw)
        return ccq.ccq_norm_bwd(s["x"], s["dy"], **kw)
    if c["op"] == "conv":
        act = ACTS[c["act"]]
        if call == "step":
            y = ccq.ccq_conv_step(s["x"], s["w"], s["state"], bias=s["bias"], act=act)
            return dict(y=y, state=s["state"])
        pack = (s["cu"], c["T"]) if c["packed"] else ()
        if call == "fwd":
            fwd = ccq.ccq_conv_fwd_varlen if c["packed"] else ccq.ccq_conv_fwd
            return fwd(s["x"], s["w"], *pack, bias=s["bias"], state0=s["state"], act=act,
                       want_state=True)
        bwd = ccq.ccq_conv_bwd_varlen if c["packed"] else ccq.ccq_conv_bwd
        return bwd(s["x"], s["w"], s["dy"], *pack, bias=s["bias"], state0=s["state"], act=act)
    args = [s[n] for n in ("q", "k", "v", "la", "beta")]
    if call == "step":
        o = ccq.ccq_delta_step(*args, s["S"])
        return dict(o=o, S=s["S"])
    pack = (s["cu"], c["T"]) if c["packed"] else ()
    if call == "fwd":
        fwd = ccq.ccq_delta_fwd_varlen if c["packed"] else ccq.ccq_delta_fwd
        return fwd(*args, *pack, S0=s["S"])
    both = ccq.ccq_delta_fwd_bwd_varlen if c["packed"] else ccq.ccq_delta_fwd_bwd
    return both(*args, s["dO"], *pack, S0=s["S"])


def _act(name, z):
    """act(z) and its derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    sg = torch.sigmoid(z)
    if name == "sigmoid":
        return sg, sg * (1 - sg)
    return z * sg, sg * (1 + z * (1 - sg))


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float()
    D = c["D"]
    if c["kind"] == "group":
        x = x - x.mean(-1, keepdim=True)
    n = 1 if c["kind"] == "l2" else D
    rstd = torch.rsqrt((x * x).sum(-1, keepdim=True) / n + EPS)
    xh = x * rstd
    z = xh if s["w"] is None else xh * s["w"]
    if s["bias"] is not None:
        z = z + s["bias"]
    gate = None if s["gate"] is None else s["gate"].float()
    a, da = _act(c["act"], z if gate is None else gate)
    if c["call"] == "fwd":
        return (a if gate is None else z * a).to(dt)
    dy = s["dy"].float()
    res = {}
    if gate is None:
        dz = dy * da
    else:
        dz = dy * a
        res["dgate"] = (dy * z * da).to(dt)
    over = 0 if s["w"] is None or s["w"].dim() == 2 else (0, 1)
    if s["w"] is not None:
        res["dweight"] = (dz * xh).sum(over)
    if s["bias"] is not None:
        res["dbias"] = dz.sum(over)
    g = dz if s["w"] is None else dz * s["w"]
    if c["kind"] == "group":
        g = g - g.mean(-1, keepdim=True)
    res["dx"] = (rstd * (g - xh * ((g * xh).sum(-1, keepdim=True) / n))).to(dt)
    return res


def _plain_conv(s):
    c, dt = s["case"], s["x"].dtype
    B, C, W, call = c["B"], c["C"], c["W"], c["call"]
    w = s["w"]
    bias = 0.0 if s["bias"] is None else s["bias"]
    if call == "step":
        ext = torch.cat([s["state"], s["x"].unsqueeze(1)], 1)
        z = (ext.float() * w.t()).sum(1) + bias
        s["state"].copy_(ext[:, 1:])
        return dict(y=_act(c["act"], z)[0].to(dt), state=s["state"])
    if c["packed"]:
        lens = _lengths(c)
        xs = list(s["x"].split(lens))
        dys = list(s["dy"].split(lens)) if call == "bwd" else None
    else:
        xs = list(s["x"])
        dys = list(s["dy"]) if call == "bwd" else None
    ys, ends, dxs, dstates = [], [], [], []
    dw, db = torch.zeros_like(w), torch.zeros(C, device=w.device)
    for b in range(B):
        n = xs[b].shape[0]
        before = torch.zeros(W - 1, C, dtype=dt, device=w.device) if s["state"] is None \
            else s["state"][b]
        ext = torch.cat([before, xs[b]])
        e = ext.float()
        z = bias + sum(w[:, j] * e[j:j + n] for j in range(W))
        y, dact = _act(c["act"], z)
        if call == "fwd":
            ys.append(y.to(dt))
            ends.append(ext[n:])
            continue
        dz = dys[b].float() * dact
        de = torch.zeros_like(e)
        for j in range(W):
            de[j:j + n] += w[:, j] * dz
            dw[:, j] += (dz * e[j:j + n]).sum(0)
        db += dz.sum(0)
        dxs.append(de[W - 1:].to(dt))
        dstates.append(de[:W - 1].to(dt))
    join = torch.cat if c["packed"] else torch.stack
    if call == "fwd":
        return dict(y=join(ys), stateT=torch.stack(ends))
    res = dict(dx=join(dxs), dw=dw)
    if s["bias"] is not None:
        res["dbias"] = db
    if s["state"] is not None:
        res["dstate0"] = torch.stack(dstates)
    return res


def _padded(c, t):
    """Packed [rows, ...] to padded [B, T, ...], zeros behind every sequence's end."""
    if not c["packed"]:
        return t
    return torch.stack([torch.cat([p, p.new_zeros(c["T"] - p.shape[0], *p.shape[1:])])
                        for p in t.split(_lengths(c))])


def _packed(c, t):
    return torch.cat([t[b, :n] for b, n in enumerate(_lengths(c))]) if c["packed"] else t


def _plain_delta(s):
    """The rule in chunks of 64 tokens: with g the running sum of log a inside a chunk entered
    with the state S, the corrected values solve
    (I + A) U = diag(b) (V - diag(e^g) K S^T),  A_ij = b_i e^{g_i - g_j} (k_i . k_j)  (j < i),
    and o_i = e^{g_i} S q_i + sum_{j<=i} e^{g_i - g_j} (k_j . q_i) u_j.  Tokens behind a
    sequence's end have b = 0 and log a = 0 and change nothing."""
    c, dt = s["case"], s["q"].dtype
    B, T, HK, HV, dk, dv = (c[n] for n in ("B", "T", "HK", "HV", "dk", "dv"))
    if c["call"] == "step":
        return _plain_step(s)
    C = 64
    N = (T + C - 1) // C
    train = c["call"] == "train"
    names = ("q", "k", "v", "la", "beta")
    with torch.set_grad_enabled(train):
        leaf = {n: s[n].float().requires_grad_(train) for n in names}

        def chunks(t):  # [B*HV, N, C, d]
            t = _padded(c, t)
            t = t if t.dim() == 4 else t.unsqueeze(-1)
            t = t.repeat_interleave(HV // t.shape[2], 2).transpose(1, 2)
            t = torch.nn.functional.pad(t, (0, 0, 0, N * C - T))
            return t.reshape(B * HV, N, C, t.shape[-1])

        q, k, v, la, be = (chunks(leaf[n]) for n in names)
        g = la.cumsum(2)
        low = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
        decay = torch.exp((g - g.transpose(2, 3)).masked_fill(~low, 0.0)) * low
        kT = k.transpose(2, 3).contiguous()
        # (I + A)^-1 = (I - A)(I + A^2)(I + A^4) .. (I + A^32), as A^64 = 0; in 64 bits, where
        # the powers cancel
        A = (be * decay * torch.matmul(k, kT)).tril(-1).double()
        eye = torch.eye(C, dtype=A.dtype, device=A.device)
        inv, power = eye - A, A
        for _ in range(5):
            power = torch.matmul(power, power)
            inv = torch.matmul(inv, eye + power)
        inv = inv.float()
        P = decay * torch.matmul(q, kT)
        eg, gl = torch.exp(g), g[:, :, -1:]
        kd, el = k * torch.exp(gl - g), torch.exp(gl)
        S = torch.zeros(B * HV, dv, dk, device=q.device) if s["S"] is None \
            else s["S"].reshape(B * HV, dv, dk)
        outs = []
        for r in range(N):
            ST = S.transpose(1, 2).contiguous()
            U = torch.matmul(inv[:, r], be[:, r] * (v[:, r] - eg[:, r] * torch.matmul(k[:, r], ST)))
            outs.append(eg[:, r] * torch.matmul(q[:, r], ST) + torch.matmul(P[:, r], U))
            S = el[:, r] * S + torch.matmul(U.transpose(1, 2).contiguous(), kd[:, r])
        o = torch.stack(outs, 1).reshape(B, HV, N * C, dv)[:, :, :T].transpose(1, 2)
        o = _packed(c, o)
        if not train:
            return dict(o=o.to(dt), ST=S.view(B, HV, dv, dk))
        grads = torch.autograd.grad(o, list(leaf.values()), s["dO"].float())
    # the gates' gradients in the type of the other gradients
    out = dict(zip(("dq", "dk", "dv", "dlogalpha", "dbeta"), (t.to(dt) for t in grads)))
    return dict(o=o.detach().to(dt), **out)


def _plain_step(s):
    c = s["case"]
    G = c["HV"] // c["HK"]
    S, outs = s["S"], []
    q, k = (s[n].float().repeat_interleave(G, 2) for n in ("q", "k"))
    v, a, be = s["v"].float(), torch.exp(s["la"]), s["beta"]
    for t in range(c["T"]):
        S = S * a[:, t, :, None, None]
        kt = k[:, t].unsqueeze(2)
        u = be[:, t, :, None] * (v[:, t] - (S * kt).sum(-1))
        S = S + u.unsqueeze(3) * kt
        outs.append((S * q[:, t].unsqueeze(2)).sum(-1))
    s["S"].copy_(S)
    return dict(o=torch.stack(outs, 1).to(s["q"].dtype), S=s["S"])


_PLAIN = {"norm": _plain_norm, "conv": _plain_conv, "delta": _plain_delta}


# ---------------------------------------------------------------------------------------
# What one pass cannot do without.

def work(case):
    io = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n = case["rows"] * case["G"] * case["D"]
        par = (case["D"] if case["shared"] else case["G"] * case["D"]) * 4
        par *= (case["kind"] != "l2") + (case["kind"] == "group")
        gate = 1 if case["gate"] else 0
        if case["call"] == "fwd":
            return {"bytes": n * io * (2 + gate) + par, "flops": n * 10}
        return {"bytes": n * io * (3 + 2 * gate) + 2 * par, "flops": n * 25}
    if case["op"] == "conv":
        n, W = _tokens(case) * case["C"], case["W"]
        par = case["C"] * (W + case["bias"]) * 4
        state = case["B"] * (W - 1) * case["C"] * io
        if case["call"] == "step":
            return {"bytes": 2 * n * io + par + 2 * state, "flops": n * (2 * W + 6)}
        if case["call"] == "fwd":
            return {"bytes": 2 * n * io + par + state * (1 + case["state"]),
                    "flops": n * (2 * W + 6)}
        return {"bytes": 3 * n * io + 2 * par + 2 * state * case["state"],
                "flops": n * (6 * W + 12)}
    n, HK, HV, dk, dv = _tokens(case), case["HK"], case["HV"], case["dk"], case["dv"]
    state = case["B"] * HV * dv * dk * 4
    tok = (2 * HK * dk + 2 * HV * dv) * io + HV * 8
    if case["call"] == "train":
        return {"bytes": n * ((4 * HK * dk + 4 * HV * dv) * io + HV * (8 + 2 * io))
                + state * case["state"], "flops": n * HV * 18 * dk * dv}
    return {"bytes": n * tok + state * (1 + case["state"]), "flops": n * HV * 6 * dk * dv}


# ---------------------------------------------------------------------------------------
# The definitions in 64 bits.

def _act64(name, z):
    if name == "none":
        return z
    return z * torch.sigmoid(z) if name == "silu" else torch.sigmoid(z)


def _exact_norm(c, s):
    leaf = {n: s[n].double() for n in ("x", "w", "bias", "gate") if s[n] is not None}
    bwd = c["call"] == "bwd"
    with torch.set_grad_enabled(bwd):
        if bwd:
            leaf = {n: t.requires_grad_() for n, t in leaf.items()}
        x = leaf["x"]
        if c["kind"] == "l2":
            z = x / torch.sqrt(x.square().sum(-1, keepdim=True) + EPS)
        else:
            m = x.mean(-1, keepdim=True) if c["kind"] == "group" else 0.0
            z = (x - m) / torch.sqrt((x - m).square().mean(-1, keepdim=True) + EPS)
        z = z * leaf["w"] if "w" in leaf else z
        z = z + leaf["bias"] if "bias" in leaf else z
        y = z * _act64(c["act"], leaf["gate"]) if "gate" in leaf else _act64(c["act"], z)
        if not bwd:
            return y
        grads = torch.autograd.grad(y, list(leaf.values()), s["dy"].double())
    names = {"x": "dx", "w": "dweight", "bias": "dbias", "gate": "dgate"}
    return {names[n]: g for n, g in zip(leaf, grads)}


def _exact_conv(c, s):
    C, W, call = c["C"], c["W"], c["call"]
    leaf = {n: s[n].double() for n in ("x", "w", "bias", "state") if s[n] is not None}
    bwd = call == "bwd"
    with torch.set_grad_enabled(bwd):
        if bwd:
            leaf = {n: t.requires_grad_() for n, t in leaf.items()}
        x = leaf["x"].unsqueeze(1) if call == "step" else leaf["x"]
        seqs = x.split(_lengths(c)) if c["packed"] else x.unbind(0)
        ys, ends = [], []
        for b, xb in enumerate(seqs):
            head = leaf["state"][b] if "state" in leaf else xb.new_zeros(W - 1, C)
            e = torch.cat([head, xb])
            # [C, n] windows of W inputs against the filters
            z = (e.unfold(0, W, 1) * leaf["w"]).sum(-1)
            z = z + leaf["bias"] if "bias" in leaf else z
            ys.append(_act64(c["act"], z))
            ends.append(e[xb.shape[0]:])
        y = torch.cat(ys) if c["packed"] else torch.stack(ys)
        if call == "step":
            return dict(y=y.squeeze(1), state=torch.stack(ends))
        if not bwd:
            return dict(y=y, stateT=torch.stack(ends))
        grads = torch.autograd.grad(y, list(leaf.values()), s["dy"].double())
    names = {"x": "dx", "w": "dw", "bias": "dbias", "state": "dstate0"}
    return {names[n]: g for n, g in zip(leaf, grads)}


def _exact_delta(c, s):
    """The recurrence itself, one token of every head at a time (a padded token has a = 1 and
    b = 0).  Backwards, with D the adjoint of S_t: dq = S_t^T do, D += do q^T, du = D k,
    db = du . (v - a S k), dv = b du, dk = D^T u - b a S^T du, then with D -= b du k^T the adjoint
    of a S, dlog a = a <D, S> and D = a D for the token before."""
    B, T, HK, HV, dk, dv = (c[n] for n in ("B", "T", "HK", "HV", "dk", "dv"))
    G, n = HV // HK, B * HV

    def rows(t, rep=1):  # [T, B*HV, d] (or [T, B*HV, 1] of a scalar per head)
        t = _padded(c, t).double()
        t = (t if t.dim() == 4 else t.unsqueeze(-1)).repeat_interleave(rep, 2)
        return t.transpose(0, 1).reshape(T, n, t.shape[-1])

    q, k, v = rows(s["q"], G), rows(s["k"], G), rows(s["v"])
    a, be = torch.exp(rows(s["la"])).unsqueeze(-1), rows(s["beta"]).unsqueeze(-1)
    S = s["S"].double().reshape(n, dv, dk) if s["S"] is not None \
        else torch.zeros(n, dv, dk, dtype=torch.float64, device=q.device)

    def write(S, t):
        aS = a[t] * S
        e = v[t].unsqueeze(2) - torch.bmm(aS, k[t].unsqueeze(2))
        u = be[t] * e
        return torch.baddbmm(aS, u, k[t].unsqueeze(1)), u, e

    def back(t, d):  # [T, B*HV, d] to the caller's layout
        return _packed(c, t.reshape(T, B, HV, d).transpose(0, 1))

    train = c["call"] == "train"
    o = torch.empty_like(v)
    seg, kept = 64, []
    for t in range(T):
        if train and t % seg == 0:
            kept.append(S)
        S, _, _ = write(S, t)
        o[t] = torch.bmm(S, q[t].unsqueeze(2)).squeeze(2)
    res = dict(o=back(o, dv))
    if not train:
        res["S" if c["call"] == "step" else "ST"] = S.view(B, HV, dv, dk)
        return res
    do = rows(s["dO"])
    dq, dkk, dvv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dla, dbe = torch.empty_like(v[:, :, :1]), torch.empty_like(v[:, :, :1])
    D = torch.zeros_like(S)
    for r in reversed(range(len(kept))):
        lo, hi = r * seg, min(T, (r + 1) * seg)
        states, us, es = [kept.pop()], [], []
        for t in range(lo, hi):
            S, u, e = write(states[-1], t)
            states.append(S)
            us.append(u)
            es.append(e)
        for t in reversed(range(lo, hi)):
            S0, S, u, e = states[t - lo], states[t - lo + 1], us[t - lo], es[t - lo]
            go = do[t].unsqueeze(2)
            dq[t] = torch.bmm(go.transpose(1, 2), S).squeeze(1)
            D = D + go * q[t].unsqueeze(1)
            du = torch.bmm(D, k[t].unsqueeze(2))
            bdu = be[t] * du
            dvv[t] = bdu.squeeze(2)
            dbe[t] = (du * e).sum(1)
            dkk[t] = torch.bmm(u.transpose(1, 2), D).squeeze(1) \
                - torch.bmm(bdu.transpose(1, 2), a[t] * S0).squeeze(1)
            D = D - bdu * k[t].unsqueeze(1)
            dla[t] = (D * S0).sum((1, 2)).unsqueeze(1) * a[t].view(-1, 1)
            D = a[t] * D
    res["dq"] = back(dq, dk).unflatten(-2, (HK, G)).sum(-2)
    res["dk"] = back(dkk, dk).unflatten(-2, (HK, G)).sum(-2)
    res["dv"] = back(dvv, dv)
    res["dlogalpha"] = back(dla, 1).squeeze(-1)
    res["dbeta"] = back(dbe, 1).squeeze(-1)
    return res


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "conv": _exact_conv, "delta": _exact_delta}[case["op"]](case, s)
