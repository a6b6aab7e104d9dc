"""Gated delta rule against its definition in 64 bits.

Tolerances (relative 2-norm).  float storage and states: products run on pairs of bfloat16 (16 mantissa
bits, 2^-17 per rounding, a handful of roundings in a row) or on floats: 1e-5.  bfloat16 outputs: one
storage rounding (at most 2^-8 of a value, 1.7e-3 of the norm) beside up to three factors rounded alike
whose errors add up like independent ones: 5e-3.
"""
import numpy as np
import pytest
import torch

from paper_2604_04250_b200 import binding as cb
from delta_ref import close, delta_inputs, delta_rule, flags_of

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 1e-5, torch.bfloat16: 5e-3}
STATE_TOL = 1e-5


def params(d, scale=None, **kw):
    B, L, Hv, Dv = d["v"].shape
    return cb.make_delta_params(B, L, d["q"].shape[2], Hv, d["q"].shape[3], Dv, scale=scale, flags=flags_of(d["v"].dtype), **kw)


def forward(d, form, with_state=True, in_place=False, prm=None, cuda=None):
    c = cuda or {n: t.cuda() for n, t in d.items()}
    prm = prm or params(d)
    o = torch.full_like(d["v"], float("nan")).cuda()
    si = c["state_in"].clone() if with_state else None
    so = si if in_place else torch.full_like(c["state_in"], float("nan"))
    if form == "step":
        cb.cawn_delta_rule_step(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], o, state_in=si, state_out=so)
    else:
        ws = cb.new_delta_workspace(prm, cb.CAWN_DELTA_FWD)
        ws.fill_(0xFF)                                   # NaN patterns: nothing may be read before it is written
        cb.cawn_delta_rule_fwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], o, ws, state_in=si, state_out=so)
    return o, so


def reference(d, with_state=True):
    w = {n: t.double() for n, t in d.items()}
    return delta_rule(w["q"], w["k"], w["v"], w["g"], w["beta"], d["q"].shape[3] ** -0.5,
                      w["state_in"] if with_state else torch.zeros_like(w["state_in"]))


SHAPES = [  # B, L, Hk, Hv, Dk, Dv
    (1, 1, 1, 1, 64, 64), (2, 2, 1, 3, 64, 64), (1, 7, 2, 2, 128, 128), (3, 15, 1, 1, 8, 8), (1, 63, 2, 4, 40, 24),
    (1, 64, 1, 1, 64, 64), (2, 65, 2, 2, 64, 128), (1, 127, 3, 3, 96, 80), (2, 130, 1, 2, 128, 64), (1, 200, 2, 2, 16, 120),
    (1, 321, 4, 4, 64, 64), (5, 129, 2, 6, 72, 56),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["step", "chunk"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, form, dtype):
    d = delta_inputs(*shape, dtype, seed=sum(shape))
    o, so = forward(d, form)
    want_o, want_s = reference(d)
    close(o, want_o, TOL[dtype], "o")
    close(so, want_s, STATE_TOL, "state")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(100, 3, 2, 6, 40, 72), (160, 1, 4, 4, 128, 40), (80, 2, 8, 8, 64, 64)], ids=str)
def test_step_of_many_streams(shape, dtype):
    d = delta_inputs(*shape, dtype, seed=sum(shape))
    o, so = forward(d, "step")
    want_o, want_s = reference(d)
    close(o, want_o, TOL[dtype])
    close(so, want_s, STATE_TOL)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("L", [16, 17, 32, 33])
def test_either_side_of_the_short_calls(L, dtype):
    d = delta_inputs(2, L, 1, 2, 64, 64, dtype, seed=L)
    o, so = forward(d, "chunk")
    want_o, want_s = reference(d)
    close(o, want_o, TOL[dtype])
    close(so, want_s, STATE_TOL)


@pytest.mark.parametrize("form", ["step", "chunk"])
def test_no_state_in_and_in_place(form):
    d = delta_inputs(2, 150, 2, 2, 64, 64, torch.float32, seed=5)
    o, so = forward(d, form, with_state=False)
    want_o, want_s = reference(d, with_state=False)
    close(o, want_o, 1e-5)
    close(so, want_s, 1e-5)
    o1, s1 = forward(d, form)
    o2, s2 = forward(d, form, in_place=True)
    assert torch.equal(o1, o2) and torch.equal(s1, s2)


@pytest.mark.parametrize("form", ["step", "chunk"])
def test_no_tokens_hand_the_state_on(form):
    d = delta_inputs(2, 0, 1, 2, 64, 64, torch.float32, seed=6)
    _, so = forward(d, form)
    assert torch.equal(so.cpu(), d["state_in"])
    _, so = forward(d, form, with_state=False)
    assert (so == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["step", "chunk"])
def test_slices_of_one_projection(form, dtype):
    """q, k, v side by side in one array, o in a wider one whose other columns stay as they are."""
    B, L, Hk, Hv, Dk, Dv = 2, 99, 2, 4, 64, 72
    d = delta_inputs(B, L, Hk, Hv, Dk, Dv, dtype, seed=7)
    w = torch.cat([d["q"].flatten(2), d["k"].flatten(2), d["v"].flatten(2)], -1).cuda()
    c = {n: t.cuda() for n, t in d.items()}
    c["q"], c["k"], c["v"] = (x.unflatten(-1, s) for x, s in zip(w.split([Hk * Dk, Hk * Dk, Hv * Dv], -1), [(Hk, Dk), (Hk, Dk), (Hv, Dv)]))
    out = torch.full((B, L, Hv * Dv + 16), 7.0, dtype=dtype, device="cuda")
    prm = params(d, q_stride=w.shape[-1], k_stride=w.shape[-1], v_stride=w.shape[-1], o_stride=out.shape[-1])
    so = torch.empty_like(c["state_in"])
    view = out[..., 8:-8]
    args = (prm, c["q"], c["k"], c["v"], c["g"], c["beta"], view)
    if form == "step":
        cb.cawn_delta_rule_step(*args, state_in=c["state_in"], state_out=so)
    else:
        cb.cawn_delta_rule_fwd(*args, cb.new_delta_workspace(prm, cb.CAWN_DELTA_FWD), state_in=c["state_in"], state_out=so)
    want_o, want_s = reference(d)
    close(view.unflatten(-1, (Hv, Dv)), want_o, TOL[dtype])
    close(so, want_s, STATE_TOL)
    assert (out[..., :8] == 7).all() and (out[..., -8:] == 7).all()


@pytest.mark.parametrize("form", ["step", "chunk", "backward"])
def test_slices_of_one_token_with_the_strides_of_the_heads_view(form):
    """One token's slice seen as heads: torch gives the time dimension the slice's width as its stride, batches lie
    the projection's width apart."""
    B, Hk, Hv, Dk, Dv = 3, 2, 4, 64, 72
    d = delta_inputs(B, 1, Hk, Hv, Dk, Dv, torch.bfloat16, seed=8)
    c = {n: t.cuda() for n, t in d.items()}
    w = torch.cat([c["q"].flatten(2), c["k"].flatten(2), c["v"].flatten(2)], -1)
    c["q"], c["k"], c["v"] = (x.unflatten(-1, s) for x, s in zip(w.split([Hk * Dk, Hk * Dk, Hv * Dv], -1), [(Hk, Dk), (Hk, Dk), (Hv, Dv)]))
    assert c["q"].stride(0) == w.shape[-1] and c["q"].stride(1) == Hk * Dk
    prm = params(d, q_stride=c["q"].stride(1), k_stride=c["k"].stride(1), v_stride=c["v"].stride(1))
    if form == "backward":
        return check_grads(backward(d, prm, c), reference_grads(d), torch.bfloat16)
    o, so = forward(d, form, prm=prm, cuda=c)
    want_o, want_s = reference(d)
    close(o, want_o, TOL[torch.bfloat16])
    close(so, want_s, STATE_TOL)


@pytest.mark.parametrize("form", ["step", "chunk"])
def test_state_passing_across_calls(form):
    """A prompt in two calls, of which the second goes token by token, equals one call."""
    d = delta_inputs(2, 203, 2, 2, 64, 64, torch.float32, seed=8)
    want_o, want_s = reference(d)
    first = {n: (t[:, :170].contiguous() if t.dim() > 2 and t.shape[1] == 203 else t) for n, t in d.items()}
    rest = {n: (t[:, 170:].contiguous() if t.dim() > 2 and t.shape[1] == 203 else t) for n, t in d.items()}
    o1, s1 = forward(first, form)
    rest["state_in"] = s1.cpu()
    o2, s2 = forward(rest, "step")
    close(torch.cat([o1, o2], 1), want_o, 1e-5)
    close(s2, want_s, 1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["step", "chunk"])
def test_repeated_tokens(form, dtype):
    """One key over and over with beta = 1 and next to no decay: the chunk's triangular system is the
    all-ones triangle, whose powers grow like binomials (a power series for its inverse would fail)."""
    d = delta_inputs(1, 192, 1, 2, 64, 64, dtype, seed=9)
    d["k"] = d["k"][:, :1].expand_as(d["k"]).contiguous()
    k = d["k"].double()
    d["g"] = torch.full_like(d["g"], -1e-4)
    d["beta"] = torch.ones_like(d["beta"]) / k.square().sum(-1).max().float()
    o, so = forward(d, form)
    want_o, want_s = reference(d)
    close(o, want_o, TOL[dtype])
    close(so, want_s, STATE_TOL)


@pytest.mark.parametrize("form", ["step", "chunk"])
def test_forgetting_and_strong_decay(form):
    """-infinity as log decay starts over (the state before it leaves no trace); very strong and zero
    decays, beta 0 and beta 2 in one call."""
    d = delta_inputs(1, 200, 2, 2, 64, 64, torch.float32, seed=10)
    d["g"][:, 70] = -float("inf")
    d["g"][:, 71] = -float("inf")
    d["g"][:, 100:110] = -90.0
    d["g"][:, 110:120] = -1000.0
    d["g"][:, 120:130] = 0.0
    d["beta"][:, 130:140] = 0.0
    d["beta"][:, 140:145] = 1.9
    o, so = forward(d, form)
    want_o, want_s = reference(d)
    close(o, want_o, 1e-5)
    close(so, want_s, 1e-5)
    late = {n: (t[:, 70:].contiguous() if t.dim() > 2 and t.shape[1] == 200 else t) for n, t in d.items()}
    o2, s2 = forward(late, form)
    close(o2, want_o[:, 70:], 1e-5)
    close(s2, want_s, 1e-5)


def test_bad_values_stay_in_their_stream():
    """NaN and infinity in one batch row's value leave the other rows alone and are not hidden."""
    d = delta_inputs(3, 130, 1, 1, 64, 64, torch.float32, seed=11)
    clean, _ = forward(d, "chunk")
    d["v"][1, 40, 0, 3] = float("nan")
    d["g"][2, 90] = float("nan")
    o, so = forward(d, "chunk")
    assert torch.equal(o[0], clean[0])
    assert torch.isnan(o[1, 40:, 0, 3]).all() and torch.equal(o[1, :, 0, 4:], clean[1, :, 0, 4:])
    assert torch.isnan(o[2, 90:]).all() and torch.isnan(so[2]).all()


@pytest.mark.parametrize("form", ["step", "chunk"])
def test_runs_on_another_stream_and_in_a_graph(form):
    d = delta_inputs(2, 140, 2, 2, 64, 64, torch.bfloat16, seed=12)
    want, want_s = forward(d, form)
    c = {n: t.cuda() for n, t in d.items()}
    prm = params(d)
    o, so = torch.empty_like(want), torch.empty_like(want_s)
    ws = cb.new_delta_workspace(prm, cb.CAWN_DELTA_FWD)
    call = {"step": lambda: cb.cawn_delta_rule_step(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], o, state_in=c["state_in"], state_out=so),
            "chunk": lambda: cb.cawn_delta_rule_fwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], o, ws, state_in=c["state_in"], state_out=so)}[form]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(o, want) and torch.equal(so, want_s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    o.zero_(), so.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(so, want_s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1500, 1, 1, 64, 64), (1, 2100, 2, 4, 128, 72), (2, 769, 1, 2, 40, 128)], ids=str)
def test_long_and_few_heads(shape, dtype):
    """Cut into time segments that run side by side."""
    d = delta_inputs(*shape, dtype, seed=sum(shape))
    o, so = forward(d, "chunk")
    want_o, want_s = reference(d)
    close(o, want_o, TOL[dtype], "o")
    close(so, want_s, STATE_TOL, "state")


# ------------------------------------------------------------------------------------ backward

def backward(d, prm=None, cuda=None, with_states=True):
    c = cuda or {n: t.cuda() for n, t in d.items()}
    prm = prm or params(d)
    nan = lambda t: torch.full(t.shape, float("nan"), dtype=t.dtype, device="cuda")
    out = {n: nan(d[n]) for n in ("q", "k", "v", "g", "beta")}
    gsi = nan(d["state_in"]) if with_states else None
    ws = cb.new_delta_workspace(prm, cb.CAWN_DELTA_BWD)
    ws.fill_(0xFF)
    cb.cawn_delta_rule_bwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], c["grad_o"], out["q"], out["k"], out["v"], out["g"], out["beta"], ws,
                           state_in=c["state_in"] if with_states else None, grad_state_out=c["grad_state_out"] if with_states else None, grad_state_in=gsi)
    if with_states:
        out["state_in"] = gsi
    return out


def loss64(w, scale):
    o, s = delta_rule(w["q"], w["k"], w["v"], w["g"], w["beta"], scale, w["state_in"])
    return (o * w["grad_o"]).sum() + (s * w["grad_state_out"]).sum()


def reference_grads(d, with_states=True):
    w = {n: t.double() for n, t in d.items()}
    if not with_states:
        w["state_in"], w["grad_state_out"] = torch.zeros_like(w["state_in"]), torch.zeros_like(w["state_in"])
    names = ["q", "k", "v", "g", "beta"] + (["state_in"] if with_states else [])
    for n in names:
        w[n].requires_grad_()
    return dict(zip(names, torch.autograd.grad(loss64(w, d["q"].shape[3] ** -0.5), [w[n] for n in names])))


def check_grads(got, want, dtype):
    for n in want:
        close(got[n], want[n], TOL[dtype] if n in "qkv" else STATE_TOL, "grad_" + n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    d = delta_inputs(*shape, dtype, seed=sum(shape) + 1)
    check_grads(backward(d), reference_grads(d), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1100, 1, 1, 64, 64), (1, 900, 1, 2, 128, 72)], ids=str)
def test_backward_long_and_few_heads(shape, dtype):
    d = delta_inputs(*shape, dtype, seed=sum(shape) + 1)
    check_grads(backward(d), reference_grads(d), dtype)


def test_backward_without_states():
    d = delta_inputs(2, 100, 1, 2, 64, 64, torch.float32, seed=20)
    check_grads(backward(d, with_states=False), reference_grads(d, with_states=False), torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward_of_slices(dtype):
    """q, k, v and grad_o with strides; gradients dense."""
    B, L, Hk, Hv, Dk, Dv = 2, 99, 2, 4, 64, 72
    d = delta_inputs(B, L, Hk, Hv, Dk, Dv, dtype, seed=21)
    c = {n: t.cuda() for n, t in d.items()}
    w = torch.cat([c["q"].flatten(2), c["k"].flatten(2), c["v"].flatten(2), c["grad_o"].flatten(2)], -1)
    parts = w.split([Hk * Dk, Hk * Dk, Hv * Dv, Hv * Dv], -1)
    for n, x in zip(("q", "k", "v", "grad_o"), parts):
        c[n] = x
    s = w.shape[-1]
    prm = params(d, q_stride=s, k_stride=s, v_stride=s, o_stride=s)
    check_grads(backward(d, prm, c), reference_grads(d), dtype)


def test_backward_of_shared_heads_sums_them():
    """Hv / Hk value heads on one key head: the same gradients as with the key head written out per value
    head, summed."""
    d = delta_inputs(1, 150, 1, 3, 64, 64, torch.float32, seed=22)
    wide = dict(d)
    wide["q"], wide["k"] = d["q"].repeat_interleave(3, 2), d["k"].repeat_interleave(3, 2)
    a, b = backward(d), backward(wide)
    for n in ("q", "k"):
        close(a[n], b[n].double().sum(2, keepdim=True), 1e-6)
    for n in ("v", "g", "beta", "state_in"):
        assert torch.equal(a[n], b[n])


def test_backward_forgetting_and_repeated_tokens():
    d = delta_inputs(1, 170, 1, 2, 64, 64, torch.float32, seed=23)
    d["k"][:, 20:60] = d["k"][:, 20:21]
    d["g"][:, 64:110] = -1e-4
    d["g"][:, 70] = -float("inf")
    d["g"][:, 120:130] = -60.0
    d["beta"][:, 30:40] = 0.0
    d["beta"][:, 90:100] = 1.0
    got = backward(d)
    want = reference_grads(d)
    assert (got["g"][:, 70] == 0).all()                 # nothing before it reaches past it
    check_grads(got, want, torch.float32)


def test_backward_against_differences():
    """Directional derivatives of the 64-bit loss.  Central differences with h = 1e-5 are good to about
    1e-8 of the gradient's size; the kernel's own 1e-5 dominates."""
    d = delta_inputs(1, 90, 1, 2, 64, 64, torch.float32, seed=24)
    got = backward(d)
    rng = torch.Generator().manual_seed(240)
    for n, grad in got.items():
        way = torch.randn(d[n].shape, generator=rng).double()
        def loss(h):
            w = {m: t.double() for m, t in d.items()}
            w[n] = w[n] + h * way
            return loss64(w, 64 ** -0.5)
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        g = grad.double().cpu()
        assert abs((g * way).sum() - slope) <= 1e-5 * g.norm() * way.norm(), n


def test_backward_is_repeatable_and_runs_in_a_graph():
    d = delta_inputs(2, 200, 2, 4, 64, 64, torch.bfloat16, seed=25)
    want = backward(d)
    again = backward(d)
    assert all(torch.equal(want[n], again[n]) for n in want)
    c = {n: t.cuda() for n, t in d.items()}
    prm = params(d)
    out = {n: torch.empty_like(want[n]) for n in want}
    ws = cb.new_delta_workspace(prm, cb.CAWN_DELTA_BWD)
    call = lambda: cb.cawn_delta_rule_bwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], c["grad_o"], out["q"], out["k"], out["v"], out["g"], out["beta"],
                                          ws, state_in=c["state_in"], grad_state_out=c["grad_state_out"], grad_state_in=out["state_in"])
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in out.values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[n], out[n]) for n in want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(12, 130, 4, 8, 64, 64), (5, 70, 6, 18, 64, 72), (14, 66, 3, 15, 32, 40), (3, 200, 16, 48, 128, 32), (9, 65, 5, 10, 96, 128),
                                   (12, 961, 4, 8, 16, 8), (5, 1000, 6, 18, 8, 8), (13, 1024, 3, 15, 8, 8), (3, 970, 16, 16, 8, 72)], ids=str)
def test_backward_of_many_heads(shape, dtype):
    """More heads than half the SMs, in part more than SMs: some reverse walks run beside the forward ones."""
    d = delta_inputs(*shape, dtype, seed=sum(shape))
    check_grads(backward(d), reference_grads(d), dtype)


def test_backward_of_many_heads_on_streams_and_in_a_graph():
    """The call's second stream is forked from and joined into the caller's, also while that one is captured."""
    d = delta_inputs(12, 1100, 4, 8, 64, 64, torch.bfloat16, seed=27)
    want = backward(d)
    c = {n: t.cuda() for n, t in d.items()}
    prm = params(d)
    side = torch.cuda.Stream()
    out = {n: torch.empty_like(want[n]) for n in want}
    ws = cb.new_delta_workspace(prm, cb.CAWN_DELTA_BWD)
    call = lambda: cb.cawn_delta_rule_bwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], c["grad_o"], out["q"], out["k"], out["v"], out["g"], out["beta"],
                                          ws, state_in=c["state_in"], grad_state_out=c["grad_state_out"], grad_state_in=out["state_in"])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            for t in out.values():
                t.zero_()
            call()
            got = {n: t.clone() for n, t in out.items()}
    side.synchronize()
    assert all(torch.equal(want[n], got[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in out.values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[n], out[n]) for n in want)


def test_backward_of_many_heads_while_a_capture_is_open():
    """A capture that has taken the call's second stream in does not keep another stream from calling."""
    d = delta_inputs(12, 1100, 4, 8, 16, 16, torch.bfloat16, seed=28)
    want = backward(d)
    c = {n: t.cuda() for n, t in d.items()}
    prm = params(d)
    outs = [{n: torch.zeros_like(want[n]) for n in want} for _ in range(2)]
    spaces = [cb.new_delta_workspace(prm, cb.CAWN_DELTA_BWD) for _ in range(2)]

    def call(out, ws):
        cb.cawn_delta_rule_bwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], c["grad_o"], out["q"], out["k"], out["v"], out["g"], out["beta"],
                               ws, state_in=c["state_in"], grad_state_out=c["grad_state_out"], grad_state_in=out["state_in"])

    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        call(outs[0], spaces[0])
        with torch.cuda.stream(other):
            call(outs[1], spaces[1])
        call(outs[0], spaces[0])
    graph.replay()
    torch.cuda.synchronize()
    for out in outs:
        for n in want:
            close(out[n], want[n], 2e-6 if want[n].dtype == torch.float32 else 4e-3, n)      # the sums over both walks in another order


def test_backward_without_tokens():
    d = delta_inputs(2, 0, 1, 1, 64, 64, torch.float32, seed=26)
    got = backward(d)
    assert torch.equal(got["state_in"].cpu(), d["grad_state_out"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 150, 1, 4, 64, 64), (2, 70, 2, 4, 128, 40), (1, 1100, 1, 4, 64, 64)], ids=str)
def test_backward_of_heads_with_short_memory(shape, dtype):
    """One strong decay per head: its gradient carries the factor e^g, and is held to its own size head by head."""
    d = delta_inputs(*shape, dtype, seed=30)
    for h, g in enumerate((-4.0, -8.0, -12.0, -20.0)):
        d["g"][:, :, h] = g
    got, want = backward(d)["g"], reference_grads(d)["g"]
    for h in range(4):
        close(got[:, :, h], want[:, :, h], STATE_TOL, h)


def overwritten(dtype, L=150, size=50.0):
    """A state much larger than the values, which the first tokens overwrite: what is read later is a difference of
    large numbers."""
    d = delta_inputs(1, L, 1, 2, 16, 24, dtype, seed=31)
    d["k"] = torch.eye(16)[torch.arange(L) % 16][None, :, None].to(dtype).contiguous()
    d["g"], d["beta"] = torch.zeros_like(d["g"]), torch.ones_like(d["beta"])
    d["state_in"] *= 2 * size
    return d


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward_of_an_overwritten_state(dtype):
    """Factors of 16 mantissa bits leave 50 x 2^-17 of a few products, 1e-3, beside the rounding of the results (of 8 bits:
    a tenth and more); float storage, with 24 bits, 50 x 1e-5."""
    d = overwritten(dtype)
    got, want = backward(d), reference_grads(d)
    for n in "qkv":
        close(got[n][:, 16:], want[n][:, 16:], 5e-3 if dtype == torch.bfloat16 else 5e-4, n)


def test_backward_of_many_heads_does_not_wait_for_another_stream():
    """Work of one caller's stream stays on it: a call behind a stream that is held up does not hold up another's."""
    d = delta_inputs(12, 1100, 4, 8, 16, 16, torch.bfloat16, seed=32)
    c = {n: t.cuda() for n, t in d.items()}
    prm = params(d)
    outs = [{n: torch.empty_like(c[n]) for n in ("q", "k", "v", "g", "beta")} for _ in range(2)]
    spaces = [cb.new_delta_workspace(prm, cb.CAWN_DELTA_BWD) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]

    def call(i):
        o = outs[i]
        cb.cawn_delta_rule_bwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], c["grad_o"], o["q"], o["k"], o["v"], o["g"], o["beta"], spaces[i],
                               state_in=c["state_in"], stream=streams[i])

    call(0), call(1)                                # first use, before anything is held up
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        torch.cuda._sleep(1 << 30)                  # half a second
    call(0)
    held = torch.cuda.Event()
    held.record(streams[0])
    call(1)
    streams[1].synchronize()
    assert not held.query()
    torch.cuda.synchronize()
    for n in outs[0]:
        assert torch.equal(outs[0][n], outs[1][n])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["step", "chunk"])
def test_overwritten_state(form, dtype):
    """As in the backward: 50 x 2^-17 of a few factors beside the rounding of o; float storage 50 x 1e-5."""
    d = overwritten(dtype)
    o, so = forward(d, form)
    want_o, want_s = reference(d)
    close(o[:, 16:], want_o[:, 16:], 5e-3 if dtype == torch.bfloat16 else 5e-4)
    close(so, want_s, 5e-4)


@pytest.mark.parametrize("shape", [(2, 200, 2, 4, 64, 64), (1, 300, 1, 2, 128, 72)], ids=str)
def test_bfloat16_outputs_are_rounded_once(shape):
    """o, dq, dk, dv against the definition rounded to bfloat16: equal but for values next to a rounding boundary.  With
    factors of 16 bits a result moves by about 1e-5 of its row, and one in a few hundred crosses a boundary by 2^-8 of
    itself: 2^-8 / sqrt(100) = 4e-4 of the norm."""
    d = delta_inputs(*shape, torch.bfloat16, seed=33)
    o, _ = forward(d, "chunk")
    close(o, reference(d)[0].bfloat16(), 4e-4)
    got, want = backward(d), reference_grads(d)
    for n in "qkv":
        close(got[n], want[n].bfloat16(), 4e-4, n)


# ------------------------------------------------------------------------------------ resets, bad values, workspaces

def reset(d):
    """Resets, strong and no decays, beta 0 and almost 2, one key over and over."""
    L = d["g"].shape[1]
    d["g"][:, L // 3] = -float("inf")
    d["g"][:, L // 3 + 1] = -float("inf")
    d["g"][:, L // 2:L // 2 + 10] = -90.0
    d["g"][:, L // 2 + 10:L // 2 + 20] = -1000.0
    d["g"][:, L // 2 + 20:L // 2 + 40] = 0.0
    d["beta"][:, L // 2 + 40:L // 2 + 50] = 0.0
    d["beta"][:, L // 2 + 50:L // 2 + 55] = 1.9
    d["k"][:, L // 4:L // 4 + 20] = d["k"][:, L // 4:L // 4 + 1]
    return d


RESETS = [(1, 200, 2, 2, 64, 64), (2, 230, 1, 2, 128, 72), (1, 1500, 1, 1, 64, 64), (1, 1300, 1, 2, 128, 64)]     # the last two in segments


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("form", ["step", "chunk"])
@pytest.mark.parametrize("shape", RESETS, ids=str)
def test_forgetting_in_both_storages_and_in_segments(shape, form, dtype):
    d = reset(delta_inputs(*shape, dtype, seed=40))
    o, so = forward(d, form)
    want_o, want_s = reference(d)
    close(o, want_o, TOL[dtype])
    close(so, want_s, STATE_TOL)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", RESETS, ids=str)
def test_backward_forgetting_in_both_storages_and_in_segments(shape, dtype):
    d = reset(delta_inputs(*shape, dtype, seed=41))
    got, want = backward(d), reference_grads(d)
    forgotten = d["g"] < -104
    assert (got["g"].cpu()[forgotten] == 0).all()
    check_grads(got, want, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(2, 130, 1, 1, 64, 64), (1, 1500, 1, 1, 64, 64)], ids=str)
def test_bad_values_stay_in_their_row_and_behind_their_chunk(shape, dtype):
    """NaN or infinity in a value: its row of the state from there on, and in the chunk of 64 tokens where it stands; nothing
    else.  A NaN decay: everything behind."""
    d = delta_inputs(*shape, dtype, seed=42)
    L = shape[1]
    at = L // 2 + 9
    first = at // 64 * 64
    clean, clean_s = forward(d, "chunk")
    for bad in (float("nan"), float("inf")):
        x = dict(d, v=d["v"].clone())
        x["v"][0, at, 0, 3] = bad
        o, so = forward(x, "chunk")
        assert torch.equal(o[:, :first], clean[:, :first]) and torch.equal(o[1:], clean[1:])
        assert not torch.isfinite(o[0, at:, 0, 3]).any() and not torch.isfinite(so[0, 0, 3]).any()
        others = [i for i in range(64) if i != 3]
        assert torch.equal(o[..., others], clean[..., others]) and torch.equal(so[:, :, others], clean_s[:, :, others])
    x = dict(d, g=d["g"].clone())
    x["g"][0, at] = float("nan")
    o, so = forward(x, "chunk")
    assert torch.equal(o[:, :first], clean[:, :first]) and torch.isnan(o[0, at:]).all() and torch.isnan(so[0]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1500, 1, 1, 64, 64), (1, 1300, 1, 2, 128, 72), (12, 130, 4, 8, 64, 64), (3, 100, 2, 2, 40, 104), (1, 33, 1, 1, 8, 8)], ids=str)
def test_calls_keep_to_their_workspace(shape, dtype):
    """In segments, with many heads, with values that are no multiple of 64, in both storages: the reported size is enough, and
    nothing behind it is written."""
    d = delta_inputs(*shape, dtype, seed=43)
    c = {n: t.cuda() for n, t in d.items()}
    prm = params(d)
    want_o, want_g = forward(d, "chunk"), backward(d)
    for op in (cb.CAWN_DELTA_FWD, cb.CAWN_DELTA_BWD):
        n = cb.cawn_delta_rule_workspace_bytes(prm, op)
        ws = torch.full((n + (1 << 16),), 0xA5, dtype=torch.uint8, device="cuda")
        if op == cb.CAWN_DELTA_FWD:
            o, so = torch.empty_like(c["v"]), torch.empty_like(c["state_in"])
            cb.cawn_delta_rule_fwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], o, ws[:n], state_in=c["state_in"], state_out=so)
            assert torch.equal(o, want_o[0]) and torch.equal(so, want_o[1])
        else:
            out = {m: torch.empty_like(c[m]) for m in want_g}
            cb.cawn_delta_rule_bwd(prm, c["q"], c["k"], c["v"], c["g"], c["beta"], c["grad_o"], out["q"], out["k"], out["v"], out["g"], out["beta"],
                                   ws[:n], state_in=c["state_in"], grad_state_out=c["grad_state_out"], grad_state_in=out["state_in"])
            assert all(torch.equal(out[m], want_g[m]) for m in out)
        assert (ws[n:] == 0xA5).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward_gradient_of_g_where_little_is_left_of_the_states(dtype):
    """Many short sequences, each head held to its own size: some have a small <state, adjoint>, a difference of large
    terms.  With three terms of both a head's error is that of the other sums, 2^-17 of a few."""
    for seed, shape in ((1, (24, 34, 2, 2, 128, 128)), (2, (16, 63, 4, 4, 64, 64)), (3, (16, 33, 4, 8, 40, 24))):
        d = delta_inputs(*shape, dtype, seed=seed)
        got, want = backward(d)["g"], reference_grads(d)["g"]
        for b in range(shape[0]):
            close(got[b], want[b], STATE_TOL, (seed, b))
