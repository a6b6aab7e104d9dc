"""Short causal convolution against its definition in 64 bits.

Tolerances (relative 2-norm), float: a sum of K + 1 products and two fast exponentials are within 2e-6 of the definition, sums
over rows alike.  bfloat16 results are rounded once, so they are compared with the definition rounded once: 2^-9, equal but
for values that lie next to a rounding boundary.
"""
import pytest
import torch

from delta_ref import close as close64
from paper_2604_04250_b200 import binding as cb
from selective_ref import flags_of, packed_offsets, short_conv, slices

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 2e-6, torch.bfloat16: 2.0 ** -9}
DTYPES = [torch.float32, torch.bfloat16]


def close(got, want, tol, what=""):
    close64(got, want.detach().to(torch.bfloat16) if got.dtype == torch.bfloat16 else want, tol, what)


def case(offsets, C, K, dtype, seed=0, rows=None, pad=0):
    rng = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=rng)
    B, rows = len(offsets) - 1, offsets[-1] if rows is None else rows
    d = {"x": randn(rows, C).to(dtype), "weight": randn(C, K) * K ** -0.5, "bias": 0.3 * randn(C), "state_in": randn(B, K - 1, C),
         "grad_y": randn(rows, C).to(dtype), "grad_state_out": randn(B, K - 1, C)}
    c = {n: t.cuda() for n, t in d.items()}
    c["x"] = slices(d["x"], pad)
    return d, c


def params(offsets, C, K, act, dtype, packed, rows, L=None, pad=0):
    longest = max(b - a for a, b in zip(offsets, offsets[1:]))
    act = cb.CAWN_CONV_ACT_SILU if act == "silu" else cb.CAWN_CONV_ACT_NONE
    return cb.make_conv_params(len(offsets) - 1, longest if L is None else L, C, K, act=act, flags=flags_of(dtype), x_stride=C + 2 * pad if pad else 0,
                               rows=rows if packed else 0)


def check(offsets, C, K, dtype, act, packed=False, rows=None, L=None, pad=0, bias=True, state=True, seed=0):
    rows = offsets[-1] if rows is None else rows
    d, c = case(offsets, C, K, dtype, seed, rows, pad)
    prm = params(offsets, C, K, act, dtype, packed, rows, L, pad)
    off = torch.tensor(offsets, device="cuda") if packed else None
    b, s = (c["bias"] if bias else None), (c["state_in"] if state else None)
    mark = 7.0
    y = torch.full((rows, C), mark, dtype=dtype, device="cuda")
    so = torch.full_like(c["state_in"], float("nan"))
    cb.cawn_short_conv_fwd(prm, c["x"], c["weight"], y, bias=b, state_in=s, state_out=so, offsets=off)

    w = {n: t.double().requires_grad_() for n, t in d.items()}
    want, want_state = short_conv(w["x"], w["weight"], w["bias"] if bias else None, act == "silu", w["state_in"] if state else torch.zeros_like(w["state_in"]),
                                  offsets, prm.L)
    own = torch.zeros(rows, dtype=torch.bool)
    for a, e in zip(offsets, offsets[1:]):
        own[a:min(e, a + prm.L)] = True
    close(y[own], want[own], TOL[dtype], "y")
    assert (y[~own] == mark).all()
    close(so, want_state, TOL[torch.float32], "state_out")

    gx, ws = torch.full((rows, C), mark, dtype=dtype, device="cuda"), cb.new_conv_workspace(prm)
    ws.fill_(0xFF)
    g = {n: torch.full_like(c[n], float("nan")) for n in ("weight", "bias", "state_in")}
    cb.cawn_short_conv_bwd(prm, c["x"], c["weight"], c["grad_y"], gx, ws, bias=b, state_in=s, offsets=off, grad_state_out=c["grad_state_out"],
                           grad_weight=g["weight"], grad_bias=g["bias"], grad_state_in=g["state_in"])
    gy = d["grad_y"].double() * own[:, None]
    names = ["x", "weight"] + (["bias"] if bias else []) + (["state_in"] if state else [])
    got = torch.autograd.grad([want, want_state], [w[n] for n in names], [gy, d["grad_state_out"].double()], allow_unused=True)
    ref = {n: torch.zeros_like(w[n]) if t is None else t for n, t in zip(names, got)}
    close(gx[own], ref["x"][own], TOL[dtype], "grad_x")
    assert (gx[~own] == mark).all()
    for n in names[1:]:
        close(g[n], ref[n], TOL[torch.float32], "grad_" + n)
    # without the sums, and without a gradient of the state: the same grad_x, no workspace
    gx2 = torch.full_like(gx, mark)
    cb.cawn_short_conv_bwd(prm, c["x"], c["weight"], c["grad_y"], gx2, bias=b, state_in=s, offsets=off, grad_state_out=c["grad_state_out"])
    assert torch.equal(gx, gx2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("B, L, C, K", [(1, 1, 8, 4), (3, 1, 64, 4), (2, 2, 24, 4), (2, 3, 40, 3), (1, 16, 8, 2), (2, 17, 256, 4), (3, 64, 264, 4),
                                        (2, 65, 33, 4), (1, 203, 7, 3), (2, 130, 1, 1), (5, 100, 300, 1), (4, 81, 512, 4)])
def test_dense(B, L, C, K, act, dtype):
    check([i * L for i in range(B + 1)], C, K, dtype, act, seed=B + L + C + K)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths, first, behind", [((5, 0, 1, 70, 2), 0, 0), ((0, 0), 3, 4), ((130, 1, 64), 2, 5), ((1,), 0, 1), ((0, 200, 0, 3, 0), 0, 0)])
@pytest.mark.parametrize("C, K", [(40, 4), (13, 3), (256, 2)])
def test_packed(C, K, lengths, first, behind, dtype):
    offsets = packed_offsets(lengths, first)
    if offsets[-1] + behind == 0:
        return
    check(offsets, C, K, dtype, "silu", packed=True, rows=offsets[-1] + behind, seed=len(lengths) + C)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [8, 3, 1])
@pytest.mark.parametrize("bias, state", [(True, False), (False, True), (False, False)])
def test_slices_and_absent_arrays(bias, state, pad, dtype):
    check([0, 70, 140], 48, 4, dtype, "silu", pad=pad, bias=bias, state=state)
    check([0, 1, 2, 3], 48, 4, dtype, "silu", pad=pad, bias=bias, state=state)


def test_longer_sequences_than_said_and_offsets_outside():
    """A sequence of more than L tokens ends there, and whatever the offsets hold nothing outside the rows is touched."""
    check([0, 50, 90], 32, 4, torch.float32, "silu", packed=True, L=40, rows=96)
    d, c = case([0, 50, 90], 32, 4, torch.float32, rows=90)
    prm = params([0, 50, 90], 32, 4, "silu", torch.float32, True, 90)
    y = torch.full((90, 32), 7.0, device="cuda")
    cb.cawn_short_conv_fwd(prm, c["x"], c["weight"], y, offsets=torch.tensor([-5, 30, 10 ** 12], device="cuda"))
    want, _ = short_conv(d["x"].double(), d["weight"].double(), None, True, torch.zeros(2, 3, 32, dtype=torch.double), [0, 30, 90], 50)
    close(y[:80], want[:80], TOL[torch.float32])
    assert (y[80:] == 7).all()
    y.fill_(7)
    cb.cawn_short_conv_fwd(prm, c["x"], c["weight"], y, offsets=torch.tensor([60, 30, -10], device="cuda"))       # they fall: nothing to do
    assert (y == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_tokens_one_by_one_with_the_history_in_place(dtype):
    B, L, C, K = 3, 9, 40, 4
    d, c = case([i * L for i in range(B + 1)], C, K, dtype)
    one = cb.make_conv_params(B, 1, C, K, act=cb.CAWN_CONV_ACT_SILU, flags=flags_of(dtype))
    state, parts = c["state_in"].clone(), []
    for t in range(L):
        y = torch.empty(B, C, dtype=dtype, device="cuda")
        cb.cawn_short_conv_fwd(one, c["x"].view(B, L, C)[:, t].contiguous(), c["weight"], y, bias=c["bias"], state_in=state, state_out=state)
        parts.append(y)
    whole, last = torch.empty(B * L, C, dtype=dtype, device="cuda"), torch.empty_like(state)
    prm = cb.make_conv_params(B, L, C, K, act=cb.CAWN_CONV_ACT_SILU, flags=flags_of(dtype))
    cb.cawn_short_conv_fwd(prm, c["x"], c["weight"], whole, bias=c["bias"], state_in=c["state_in"], state_out=last)
    assert torch.equal(torch.stack(parts, 1).view(B * L, C), whole) and torch.equal(state, last)


def test_no_tokens_pass_the_history_on():
    d, c = case([0, 0, 0], 40, 4, torch.float32, rows=0)
    prm = cb.make_conv_params(2, 0, 40, 4)
    so, g = torch.empty_like(c["state_in"]), torch.empty_like(c["state_in"])
    cb.cawn_short_conv_fwd(prm, None, c["weight"], None, state_in=c["state_in"], state_out=so)
    assert torch.equal(so, c["state_in"])
    gw, ws = torch.full_like(c["weight"], 7.0), cb.new_conv_workspace(prm)
    cb.cawn_short_conv_bwd(prm, None, c["weight"], None, None, ws, state_in=c["state_in"], grad_state_out=c["grad_state_out"], grad_weight=gw, grad_state_in=g)
    assert torch.equal(g, c["grad_state_out"]) and (gw == 0).all()


def test_non_finite_values_stay_where_they_reach():
    d, c = case([0, 40, 80], 32, 4, torch.float32)
    c["x"][50, 3] = float("inf")
    c["x"][60, 5] = float("nan")
    y = torch.empty(80, 32, device="cuda")
    cb.cawn_short_conv_fwd(cb.make_conv_params(2, 40, 32, 4), c["x"], c["weight"], y)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[50:54, 3] = want[60:64, 5] = True
    assert torch.equal(bad, want)


def test_streams_graphs_and_repeats():
    """Captured on another stream and replayed on new inputs, it gives the same bits as a plain call; so do repeats."""
    B, L, C, K = 4, 300, 128, 4
    d, c = case([i * L for i in range(B + 1)], C, K, torch.bfloat16)
    prm = cb.make_conv_params(B, L, C, K, act=cb.CAWN_CONV_ACT_SILU, flags=flags_of(torch.bfloat16))
    ws = cb.new_conv_workspace(prm)
    out = {n: torch.empty_like(c[n]) for n in ("x", "weight", "bias", "state_in")}
    y, so = torch.empty_like(c["x"]), torch.empty_like(c["state_in"])

    def both():
        cb.cawn_short_conv_fwd(prm, c["x"], c["weight"], y, bias=c["bias"], state_in=c["state_in"], state_out=so)
        cb.cawn_short_conv_bwd(prm, c["x"], c["weight"], c["grad_y"], out["x"], ws, bias=c["bias"], state_in=c["state_in"], grad_state_out=c["grad_state_out"],
                               grad_weight=out["weight"], grad_bias=out["bias"], grad_state_in=out["state_in"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        both()
        with torch.cuda.graph(graph, stream=side):
            both()
    torch.cuda.synchronize()
    c["x"].copy_(torch.randn_like(c["x"].float()))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (y, so, *out.values())]
    for _ in range(2):
        for t in (y, so, *out.values()):
            t.zero_()
        ws.fill_(0xFF)
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, so, *out.values())))


def test_gradient_against_differences():
    """A step along the gradient's own direction in x, weight and bias: the difference quotient of a float loss (summed in double)
    is off by its rounding (2^-24 of sums of about 1e3 terms of order one over a step of 1e-2: 1e-5) and its third-order term
    (the step squared, 1e-4, of a slope of order one)."""
    d, c = case([0, 30, 61], 24, 4, torch.float32, seed=4)
    prm = cb.make_conv_params(2, 31, 24, 4, act=cb.CAWN_CONV_ACT_SILU, rows=61)
    off = torch.tensor([0, 30, 61], device="cuda")
    g = {n: torch.empty_like(c[n]) for n in ("x", "weight", "bias", "state_in")}
    cb.cawn_short_conv_bwd(prm, c["x"], c["weight"], c["grad_y"], g["x"], cb.new_conv_workspace(prm), bias=c["bias"], state_in=c["state_in"], offsets=off,
                           grad_weight=g["weight"], grad_bias=g["bias"], grad_state_in=g["state_in"])

    def loss(step):
        y = torch.empty_like(c["x"])
        p = {n: c[n] + step * g[n] / g[n].norm() for n in g}
        cb.cawn_short_conv_fwd(prm, p["x"], p["weight"], y, bias=p["bias"], state_in=p["state_in"], offsets=off)
        return (y.double() * c["grad_y"].double()).sum().item()

    slope = (loss(1e-2) - loss(-1e-2)) / 2e-2
    want = sum(t.norm().item() for t in g.values())
    assert abs(slope - want) < 1e-3 * want


def test_more_than_32_bits_of_elements():
    L, C, dtype = 1_100_000, 2000, torch.bfloat16
    x = torch.randn(L, C, device="cuda", dtype=dtype)
    w, b, y, gx = torch.randn(C, 4, device="cuda"), torch.randn(C, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    prm = cb.make_conv_params(1, L, C, 4, act=cb.CAWN_CONV_ACT_SILU, flags=flags_of(dtype))
    assert x.numel() > 2 ** 31
    cb.cawn_short_conv_fwd(prm, x, w, y, bias=b)
    want, _ = short_conv(x[-203:].cpu().double(), w.cpu().double(), b.cpu().double(), True, torch.zeros(1, 3, C, dtype=torch.double), [0, 203], 203)
    close(y[-200:], want[-200:], TOL[dtype])
    cb.cawn_short_conv_bwd(prm, x, w, y, gx, bias=b)
    tail, gt = x[-203:].contiguous(), torch.empty(203, C, device="cuda", dtype=dtype)
    some = cb.make_conv_params(1, 203, C, 4, act=cb.CAWN_CONV_ACT_SILU, flags=flags_of(dtype))
    cb.cawn_short_conv_bwd(some, tail, w, y[-203:].contiguous(), gt, bias=b)
    assert torch.equal(gx[-200:], gt[-200:])
