"""Memory of calls on a stream that is not torch's current one (stream=side).

`side` and the current stream take turns at being late.  Blocks that the current stream has freed
while its kernels have yet to write them must not become a call's outputs or workspace; inputs and
outputs that the caller drops while `side` has yet to run must not become the current stream's
tensors."""
import pytest
import torch

from paper_2606_01294_amd import ccq
from paper_2606_01294_amd.inputs import GDN, GLA, make_inputs, to_device

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
LATE = 20_000_000  # clock cycles that a stream is kept busy for


def layer():
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    B, T, H, d = 2, 130, 2, 64
    q, k = (torch.nn.functional.normalize(r(B, T, H, d), dim=-1).to(BF) for _ in range(2))
    rule = [q, k, r(B, T, H, d).to(BF), -0.1 * r(B, T, H).abs(), torch.sigmoid(r(B, T, H))]
    pack = [t.view(B * T, *t.shape[2:]) for t in rule]
    cu = torch.tensor([0, T, 2 * T], dtype=torch.int32, device="cuda")
    one = [t[:, :1].contiguous() for t in rule]
    x, w, b = r(B, T, 256).to(BF), r(256, 4), r(256)
    n = r(B * T, H, d).to(BF)
    wn = r(H, d)
    return {  # name -> (call of (inputs, keywords), inputs)
        "delta_fwd": (ccq.ccq_delta_fwd, rule),
        "delta_fwd_varlen": (lambda *a, **k: ccq.ccq_delta_fwd_varlen(*a, T, **k), pack + [cu]),
        "delta_fwd_bwd": (lambda *a, **k: ccq.ccq_delta_fwd_bwd(*a, want_states=True, **k), rule + [rule[2]]),
        "delta_fwd_bwd_varlen": (lambda *a, **k: ccq.ccq_delta_fwd_bwd_varlen(*a, T, **k),
                                 pack + [pack[2], cu]),
        "delta_step": (ccq.ccq_delta_step, one + [r(B, H, d, d)]),
        "conv_fwd": (lambda *a, **k: ccq.ccq_conv_fwd(*a, want_state=True, **k), [x, w, b]),
        "conv_bwd": (lambda x, w, dy, b, **k: ccq.ccq_conv_bwd(x, w, dy, b, **k), [x, w, x + 1, b]),
        "conv_step": (ccq.ccq_conv_step, [x[:, 0].contiguous(), w, r(B, 3, 256).to(BF), b]),
        "norm_fwd": (lambda x, w, g, **k: ccq.ccq_norm_fwd(x, w, gate=g, **k), [n, wn, n + 1]),
        "norm_bwd": (lambda x, dy, w, g, **k: ccq.ccq_norm_bwd(x, dy, w, gate=g, **k), [n, n - 1, wn, n + 1]),
    }


def mixer():
    def of(backbone, train):
        d = to_device(make_inputs(backbone, 1, 130, 2, 64, 64, BF, seed=5, lam="random", with_dO=True))
        gate = "g" if backbone == GLA else "logalpha"
        if backbone == GLA:
            if train:
                return ccq.ccq_fwd_bwd, [d["q"], d["k"], d["v"], d[gate], d["lam"], d["dO"]]
            return ccq.ccq_gla_fwd, [d["q"], d["k"], d["v"], d[gate], d["lam"]]
        if train:
            f = lambda q, k, v, g, lam, dO, be, **kw: ccq.ccq_fwd_bwd(  # noqa: E731
                q, k, v, g, lam, dO, backbone=ccq.CCQ_GDN, beta=be, **kw)
            return f, [d["q"], d["k"], d["v"], d[gate], d["lam"], d["dO"], d["beta"]]
        return ccq.ccq_gdn_fwd, [d["q"], d["k"], d["v"], d[gate], d["beta"], d["lam"]]
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    H, dk = 2, 64
    raw = [r(2, 70, H, dk).to(BF), r(2, 70, H, dk).to(BF), 0.1 * r(H, H * dk), r(H)]
    return {
        "gla_fwd": of(GLA, False), "gdn_fwd": of(GDN, False), "gla_train": of(GLA, True),
        "gdn_train": of(GDN, True), "prep": (ccq.ccq_prep, raw),
        "fwd_raw": (ccq.ccq_fwd_raw, raw + [r(2, 70, H, 64).to(BF), -r(2, 70, H, dk).abs()]),
        "decode": (lambda *a, **k: ccq.ccq_decode(*a, 0, **k),
                   [r(3, H, dk).to(BF), r(3, H, dk).to(BF), r(3, H, 64).to(BF), -r(3, H, dk).abs(),
                    torch.sigmoid(r(3, H)), r(3, H, 64, dk), torch.zeros(3, H, dk, dk, device="cuda"),
                    torch.zeros(3, H, dk, device="cuda")]),
    }


NAMES = ["delta_fwd", "delta_fwd_varlen", "delta_fwd_bwd", "delta_fwd_bwd_varlen", "delta_step",
         "conv_fwd", "conv_bwd", "conv_step", "norm_fwd", "norm_bwd", "gla_fwd", "gdn_fwd", "gla_train",
         "gdn_train", "prep", "fwd_raw", "decode"]


def tensors(res):
    return dict(res) if isinstance(res, dict) else {"out": res}


def junk(like):
    """One tensor for every size that a call may allocate."""
    return [torch.empty(n, dtype=torch.uint8, device="cuda") for n in like for _ in range(4)]


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_a_call_on_another_stream(name):
    print(name, flush=True)
    f, args = {**layer(), **mixer()}[name]
    cur, side = torch.cuda.current_stream(), torch.cuda.Stream()
    fresh = lambda: [t.clone() for t in args]  # noqa: E731
    ref = {n: t.clone() for n, t in tensors(f(*fresh())).items()}
    sizes = sorted({t.numel() * t.element_size() for t in list(ref.values()) + args} | {1 << 18, 1 << 20, 1 << 22})
    torch.cuda.synchronize()

    # the current stream is late: it has freed blocks that it has yet to write
    mine = fresh()
    torch.cuda.synchronize()
    held = junk(sizes)
    torch.cuda._sleep(LATE)
    for t in held:
        t.fill_(255)
    del held, t
    got = tensors(f(*mine, stream=side))
    side.synchronize()
    early = {n: t.clone() for n, t in got.items()}
    torch.cuda.synchronize()
    for n in ref:
        assert torch.equal(got[n], ref[n]) and torch.equal(early[n], ref[n]), n
    del got, early

    # the side stream is late: the caller drops the inputs, and the current stream allocates
    side.wait_stream(cur)
    with torch.cuda.stream(side):
        torch.cuda._sleep(LATE)
    mine = fresh()
    side.wait_stream(cur)
    got = tensors(f(*mine, stream=side))
    del mine
    held = junk(sizes)
    for t in held:
        t.fill_(255)
    cur.wait_stream(side)
    for n in ref:
        assert torch.equal(got[n], ref[n]), n
    torch.cuda.synchronize()
    del held, t

    # outputs dropped while the current stream still reads them
    cur.wait_stream(side)
    torch.cuda._sleep(LATE)
    read = [t.clone() for t in got.values()]
    names = list(got)
    del got
    with torch.cuda.stream(side):
        held = junk(sizes)
        for t in held:
            t.fill_(255)
    torch.cuda.synchronize()
    for n, t in zip(names, read):
        assert torch.equal(t, ref[n]), n


def test_both_layers_are_covered():
    assert set(NAMES) == set(layer()) | set(mixer())
