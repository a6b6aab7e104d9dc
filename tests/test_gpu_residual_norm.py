"""The norm that adds a branch to its stream, against its definition in 64 bits.

Tolerances (relative 2-norm): float results are a few roundings away from the definition, 1e-6; bfloat16 ones are compared with
the definition rounded once, 2^-9.  8-bit values are compared with the definition's, rounded alike: y / scale is off by four
roundings of 2^-24 at most, so of values whose rounding steps are at least 2^-4 of them at most 2 * 4 * 2^-24 / 2^-4 = 2^-17 lie so near
to a step's middle that they may go the other way, and then by one step (at most 2^-3).
"""
import pytest
import torch

from delta_ref import close as close64
from paper_2604_04250_b200 import binding as cb
from selective_ref import flags_of, residual_norm, slices, to_e4m3

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 1e-6, torch.bfloat16: 2.0 ** -9}
KINDS = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)]


def close(got, want, tol, what=""):
    close64(got, want.detach().to(torch.bfloat16) if got.dtype == torch.bfloat16 else want, tol, what)


def case(N, M, kind, seed=0):
    rng = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=rng)
    dtype, stream = kind
    d = {"x": randn(N, M).to(dtype), "residual": (2 * randn(N, M)).to(stream), "weight": 1 + 0.3 * randn(M), "grad_y": randn(N, M).to(dtype),
         "grad_sum": randn(N, M).to(stream)}
    return d, {n: t.cuda() for n, t in d.items()}


def params(N, M, kind, **kw):
    return cb.make_residual_norm_params(N, M, flags=flags_of(kind[0]), stream_float=kind[0] != kind[1], **kw)


@pytest.mark.parametrize("kind", KINDS, ids=["float", "bf16", "bf16-float-stream"])
@pytest.mark.parametrize("N, M", [(1, 1), (3, 8), (5, 100), (7, 333), (9, 256), (33, 520), (16, 768), (300, 768), (20, 1024), (3, 1025), (5, 2048),
                                  (4, 4100), (2, 8192), (1500, 64), (2, 8191)])
def test_both_directions(N, M, kind):
    d, c = case(N, M, kind, N + M)
    prm = params(N, M, kind)
    y, s = torch.full_like(c["x"], float("nan")), torch.full_like(c["residual"], float("nan"))
    cb.cawn_residual_norm_fwd(prm, c["x"], y, residual=c["residual"], weight=c["weight"], sum_out=s)
    total = (d["x"].double() + d["residual"].double()).to(kind[1])
    assert torch.equal(s.cpu(), total)
    v, w = total.double().requires_grad_(), d["weight"].double().requires_grad_()
    want = residual_norm(v, w, 1e-5)
    close(y, want, TOL[kind[0]], "y")

    ws = cb.new_residual_norm_workspace(prm)
    ws.fill_(0xFF)
    gr, gx, gw = torch.full_like(s, float("nan")), torch.full_like(y, float("nan")), torch.full_like(c["weight"], float("nan"))
    cb.cawn_residual_norm_bwd(prm, s, c["grad_y"], ws, weight=c["weight"], grad_sum=c["grad_sum"], grad_residual=gr, grad_x=gx, grad_weight=gw)
    gv, want_w = torch.autograd.grad(want, [v, w], d["grad_y"].double())
    # differences of sums: of the terms (the gradient through the norm and past it), not of a row in which they cancel
    close(gr, gv + d["grad_sum"].double(), TOL[kind[1]] * 2, "grad_residual")
    close(gx, gv + d["grad_sum"].double(), TOL[kind[0]] * 2, "grad_x")
    close(gw, want_w, 2e-6, "grad_weight")
    # one of the two alone, in place, without what is not given
    g2 = c["grad_sum"].clone()
    cb.cawn_residual_norm_bwd(prm, s, c["grad_y"], weight=c["weight"], grad_sum=g2, grad_residual=g2)
    assert torch.equal(g2, gr)
    g3 = torch.empty_like(gx)
    cb.cawn_residual_norm_bwd(prm, s, c["grad_y"], grad_x=g3)
    if M > 1:       # of a single channel the two terms are equal but for eps, which float rows of order one lose
        close(g3, torch.autograd.grad(residual_norm(v, None, 1e-5), v, d["grad_y"].double())[0], TOL[kind[0]] * 2, "plain grad_x")


@pytest.mark.parametrize("kind", KINDS, ids=["float", "bf16", "bf16-float-stream"])
@pytest.mark.parametrize("block", [0, 32, 64, 128])
@pytest.mark.parametrize("N, M", [(1, 1), (40, 768), (13, 333), (7, 520), (5, 1500), (3, 4096), (130, 72)])
def test_e4m3(N, M, block, kind):
    d, c = case(N, M, kind, N + M + block)
    cols = 1 if block == 0 else -(-M // block)
    prm = params(N, M, kind, out=cb.CAWN_NORM_OUT_E4M3, scale_block=block)
    # one row more than there are: nothing is written behind the last
    y, scales = torch.full((N + 1, M), 0x55, dtype=torch.uint8, device="cuda"), torch.full((N + 1, cols), 7.0, device="cuda")
    s = torch.empty_like(c["residual"])
    cb.cawn_residual_norm_fwd(prm, c["x"], y[:N], residual=c["residual"], weight=c["weight"], sum_out=s, scales=scales[:N])
    assert (y[N] == 0x55).all() and (scales[N] == 7).all()
    total = (d["x"].double() + d["residual"].double()).to(kind[1])
    assert torch.equal(s.cpu(), total)
    want, want_scales = to_e4m3(residual_norm(total.double(), d["weight"].double(), 1e-5), block)
    close64(scales[:N], want_scales, 4e-7, "scales")
    got = y[:N].view(torch.float8_e4m3fn).float().cpu()
    off = got != want
    assert off.sum() <= 1 + want.numel() * 2.0 ** -14                       # 2^-17 of them, eight times that with few values
    assert ((got - want).abs() <= want.abs() / 8 * 1.0001 + 2.0 ** -9).all()


def test_e4m3_rows_of_nothing_and_non_finite_rows():
    N, M = 6, 256
    x = torch.randn(N, M)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 200] = float("inf")
    x[4] *= 1e-25
    x[5, 10] = 3e38
    prm = cb.make_residual_norm_params(N, M, eps=1e-6, out=cb.CAWN_NORM_OUT_E4M3, scale_block=128)
    y, scales = torch.empty(N, M, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(N, 2, device="cuda")
    cb.cawn_residual_norm_fwd(prm, x.cuda(), y, scales=scales)
    y, scales = y.float().cpu(), scales.cpu()
    assert (y[1] == 0).all() and torch.allclose(scales[1], torch.full((2,), 1e-30 / 448))
    assert torch.isnan(y[2]).all() and torch.isnan(scales[2]).all()          # the row's mean square is NaN
    assert torch.isfinite(y[0]).all() and torch.isfinite(y[4]).all()
    want, want_scales = to_e4m3(residual_norm(x[4:5].double(), None, 1e-6), 128)
    assert (y[4] == want[0]).float().mean() > 0.99 and torch.allclose(scales[4].double(), want_scales[0], rtol=1e-5)


def test_in_place_strides_and_absent_arrays():
    N, M = 50, 384
    for kind in KINDS:
        d, c = case(N, M, kind)
        want_sum = (d["x"].double() + d["residual"].double()).to(kind[1])
        y = torch.empty_like(c["x"])
        stream = c["residual"].clone()
        cb.cawn_residual_norm_fwd(params(N, M, kind), c["x"], y, residual=stream, weight=c["weight"], sum_out=stream)
        assert torch.equal(stream.cpu(), want_sum)
        x = c["x"].clone()
        cb.cawn_residual_norm_fwd(params(N, M, kind), x, x, residual=c["residual"], weight=c["weight"])
        assert torch.equal(x, y)
        for pad in (8, 3):
            wide = torch.full((N, M + pad), float("nan"), dtype=kind[0], device="cuda")
            wide[:, :M] = c["x"]
            y2 = torch.empty_like(y)
            cb.cawn_residual_norm_fwd(params(N, M, kind, x_stride=M + pad), wide[:, :M], y2, residual=c["residual"], weight=c["weight"])
            assert torch.equal(y2, y)
        for pad in (8, 3):                      # the middle of wider rows
            x = slices(d["x"], pad)
            y2 = torch.empty_like(y)
            cb.cawn_residual_norm_fwd(params(N, M, kind, x_stride=M + 2 * pad), x, y2, residual=c["residual"], weight=c["weight"])
            assert torch.equal(y2, y)
        y3 = torch.empty_like(y)
        cb.cawn_residual_norm_fwd(params(N, M, kind), c["x"], y3)
        close(y3, residual_norm(d["x"].double(), None, 1e-5), TOL[kind[0]])


def test_no_rows():
    prm, w = cb.make_residual_norm_params(0, 64), torch.full((64,), 7.0, device="cuda")
    cb.cawn_residual_norm_fwd(prm, None, None)
    cb.cawn_residual_norm_bwd(prm, None, None, grad_weight=w)
    assert (w == 0).all()


def test_streams_graphs_and_repeats():
    N, M, kind = 700, 768, KINDS[2]
    d, c = case(N, M, kind)
    prm, ws = params(N, M, kind), None
    ws = cb.new_residual_norm_workspace(prm)
    y, s = torch.empty_like(c["x"]), torch.empty_like(c["residual"])
    gr, gx, gw = torch.empty_like(s), torch.empty_like(y), torch.empty_like(c["weight"])

    def both():
        cb.cawn_residual_norm_fwd(prm, c["x"], y, residual=c["residual"], weight=c["weight"], sum_out=s)
        cb.cawn_residual_norm_bwd(prm, s, c["grad_y"], ws, weight=c["weight"], grad_sum=c["grad_sum"], grad_residual=gr, grad_x=gx, grad_weight=gw)

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
    got = [t.clone() for t in (y, s, gr, gx, gw)]
    for _ in range(2):
        ws.fill_(0xFF)
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, s, gr, gx, gw)))


def test_gradient_against_differences():
    """As for the convolution: rounding 1e-5, third-order term 1e-4 of a slope of order one."""
    d, c = case(20, 96, KINDS[0], 3)
    prm = params(20, 96, KINDS[0])
    s = c["residual"]
    gr, gw = torch.empty_like(s), torch.empty_like(c["weight"])
    cb.cawn_residual_norm_bwd(prm, s, c["grad_y"], cb.new_residual_norm_workspace(prm), weight=c["weight"], grad_residual=gr, grad_weight=gw)

    def loss(step):
        y = torch.empty_like(c["x"])
        cb.cawn_residual_norm_fwd(prm, s + step * gr / gr.norm(), y, weight=c["weight"] + step * gw / gw.norm())
        return (y.double() * c["grad_y"].double()).sum().item()

    slope = (loss(1e-2) - loss(-1e-2)) / 2e-2
    want = (gr.norm() + gw.norm()).item()
    assert abs(slope - want) < 1e-3 * want


def test_more_than_32_bits_of_elements():
    N, M, dtype = 1_100_000, 2000, torch.bfloat16
    x, s, y = torch.randn(N, M, device="cuda", dtype=dtype), None, None
    assert x.numel() > 2 ** 31
    s, y, scales = torch.empty_like(x), torch.empty(N, M, device="cuda", dtype=torch.uint8), torch.empty(N, 16, device="cuda")
    prm = params(N, M, KINDS[1], out=cb.CAWN_NORM_OUT_E4M3, scale_block=128)
    cb.cawn_residual_norm_fwd(prm, x, y, residual=x, sum_out=s, scales=scales)
    some = params(100, M, KINDS[1], out=cb.CAWN_NORM_OUT_E4M3, scale_block=128)
    s2, y2, scales2 = torch.empty_like(s[:100]), torch.empty_like(y[:100]), torch.empty_like(scales[:100])
    cb.cawn_residual_norm_fwd(some, x[-100:], y2, residual=x[-100:], sum_out=s2, scales=scales2)
    assert torch.equal(s2, s[-100:]) and torch.equal(y2, y[-100:]) and torch.equal(scales2, scales[-100:])
    g, g2 = torch.empty_like(x), torch.empty_like(s2)
    cb.cawn_residual_norm_bwd(prm, s, x, grad_residual=g)
    cb.cawn_residual_norm_bwd(some, s2, x[-100:], grad_residual=g2)
    assert torch.equal(g2, g[-100:])
