"""Group norm with an activation, and dropout, against their definitions in 64 bits.

Tolerances (relative 2-norm): float results are a few roundings and two fast exponentials away from the
definition: 2e-6 (sums over positions alike).  bfloat16 results are rounded once, so they are compared
with the definition rounded once to bfloat16: equal but for values that lie next to a rounding boundary.
"""
import numpy as np
import pytest
import torch

from paper_2604_04250_b200 import binding as cb
from delta_ref import PHILOX_ANSWERS, close as close64, flags_of, group_norm, philox_bits, philox_words

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 2e-6, torch.bfloat16: 2.0 ** -9}
SUM_TOL = 2e-6
ACTS = {"none": cb.CAWN_NORM_ACT_NONE, "silu": cb.CAWN_NORM_ACT_SILU, "gate": cb.CAWN_NORM_ACT_GATE}


def close(got, want, tol, what=""):
    close64(got, want.detach().to(torch.bfloat16) if got.dtype == torch.bfloat16 else want, tol, what)


def norm_case(N, G, M, dtype, act, rms=False, affine=True, pad=0, seed=0):
    rng = torch.Generator().manual_seed(seed)
    C = G * M
    wide = torch.randn(N, C + pad, generator=rng) * 1.5 + 0.7
    d = {"x": wide.to(dtype)[:, :C], "gate": torch.randn(N, C + pad, generator=rng).to(dtype)[:, :C], "gy": torch.randn(N, C, generator=rng).to(dtype),
         "w": 1 + 0.3 * torch.randn(C, generator=rng) if affine else None, "b": 0.3 * torch.randn(C, generator=rng) if affine else None}
    if ACTS[act] != cb.CAWN_NORM_ACT_GATE:
        d["gate"] = None
    prm = cb.make_norm_params(N, G, M, eps=1e-5, act=ACTS[act], rms=rms, flags=flags_of(dtype), x_stride=C + pad if pad else 0, gate_stride=C + pad if pad else 0)
    return d, prm


def on_gpu(t):
    if t is None:
        return None
    if not t.is_contiguous():           # keep the row stride
        wide = torch.empty(t.shape[0], t.stride(0), dtype=t.dtype, device="cuda")
        wide[:, :t.shape[1]].copy_(t)
        return wide[:, :t.shape[1]]
    return t.cuda()


def check_norm(d, prm, dtype, rms, act):
    G, N, C = prm.G, prm.N, prm.G * prm.M
    c = {n: on_gpu(t) for n, t in d.items()}
    y = torch.full((N, C), float("nan"), dtype=dtype, device="cuda")
    cb.cawn_group_norm_fwd(prm, c["x"], y, weight=c["w"], bias=c["b"], gate=c["gate"])
    w = {n: (t.double().requires_grad_() if t is not None else None) for n, t in d.items()}
    want = group_norm(w["x"], G, 1e-5, rms, w["w"], w["b"], ACTS[act], w["gate"])
    close(y, want, TOL[dtype], "y")
    gx = torch.full((N, C), float("nan"), dtype=dtype, device="cuda")
    gg = torch.full_like(gx, float("nan")) if d["gate"] is not None else None
    gw, gb = torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    ws = cb.new_norm_workspace(prm)
    ws.fill_(0xFF)
    cb.cawn_group_norm_bwd(prm, c["x"], c["gy"], gx, ws, weight=c["w"], bias=c["b"], gate=c["gate"], grad_gate=gg, grad_weight=gw, grad_bias=gb)
    names = [n for n in ("x", "gate", "w", "b") if w[n] is not None]
    grads = dict(zip(names, torch.autograd.grad(want, [w[n] for n in names], d["gy"].double())))
    close(gx, grads["x"], TOL[dtype], "grad_x")
    if gg is not None:
        close(gg, grads["gate"], TOL[dtype], "grad_gate")
    if d["w"] is not None:
        close(gw, grads["w"], SUM_TOL, "grad_weight")
        close(gb, grads["b"], SUM_TOL, "grad_bias")
    # without the parameter sums the same grad_x comes out, with no workspace
    gx2 = torch.empty_like(gx)
    cb.cawn_group_norm_bwd(prm, c["x"], c["gy"], gx2, weight=c["w"], bias=c["b"], gate=c["gate"], grad_gate=gg)
    assert torch.equal(gx, gx2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 12, 64), (3, 5, 37), (7, 8, 128), (130, 1, 768), (33, 14, 64), (9, 32, 8), (5, 6, 80),
                                   (2, 1, 1000), (4, 2, 4096), (3, 1, 2049), (67, 3, 200), (300, 40, 16), (2, 64, 256)], ids=str)
def test_norm(shape, act, dtype):
    d, prm = norm_case(*shape, dtype, act, seed=sum(shape))
    check_norm(d, prm, dtype, False, act)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("shape", [(5, 8, 1024), (3, 7, 520), (40, 9, 768)], ids=str)
def test_norm_many_wide_groups(shape, act, dtype):
    """A thread holds 32 channels and a block 224 or 256 threads: the sums of the parameters' gradients take more than
    the 48 KB of shared memory that a launch gets unasked."""
    d, prm = norm_case(*shape, dtype, act, seed=sum(shape))
    check_norm(d, prm, dtype, False, act)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("affine", [True, False])
def test_norm_rms_strided(affine, pad, dtype):
    d, prm = norm_case(50, 6, 64, dtype, "gate", rms=True, affine=affine, pad=pad, seed=3)
    check_norm(d, prm, dtype, True, "gate")


def test_norm_many_rows_and_repeatable():
    d, prm = norm_case(5000, 4, 64, torch.float32, "silu", seed=4)
    check_norm(d, prm, torch.float32, False, "silu")
    c = {n: on_gpu(t) for n, t in d.items()}
    got = []
    for _ in range(2):
        gx, gw, gb = torch.empty_like(c["x"]), torch.empty_like(c["w"]), torch.empty_like(c["b"])
        cb.cawn_group_norm_bwd(prm, c["x"], c["gy"], gx, cb.new_norm_workspace(prm), weight=c["w"], bias=c["b"], grad_weight=gw, grad_bias=gb)
        got.append((gx, gw, gb))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("act", sorted(ACTS))
def test_norm_without_eps(act):
    """eps = 0 and a row count that leaves row lanes of the last block without a row."""
    d, _ = norm_case(13, 3, 32, torch.float32, act, seed=8)
    prm = cb.make_norm_params(13, 3, 32, eps=0.0, act=ACTS[act])
    c = {n: on_gpu(t) for n, t in d.items()}
    gx, gw, gb = torch.empty_like(c["x"]), torch.empty_like(c["w"]), torch.empty_like(c["b"])
    gg = torch.empty_like(c["x"]) if act == "gate" else None
    cb.cawn_group_norm_bwd(prm, c["x"], c["gy"], gx, cb.new_norm_workspace(prm), weight=c["w"], bias=c["b"], gate=c["gate"], grad_gate=gg, grad_weight=gw, grad_bias=gb)
    w = {n: (t.double().requires_grad_() if t is not None else None) for n, t in d.items()}
    want = group_norm(w["x"], 3, 0.0, False, w["w"], w["b"], ACTS[act], w["gate"])
    wx, ww, wb = torch.autograd.grad(want, [w["x"], w["w"], w["b"]], d["gy"].double())
    close(gx, wx, 2e-6)
    close(gw, ww, SUM_TOL)
    close(gb, wb, SUM_TOL)


def test_norm_constant_row_and_bad_row():
    """A row without variance gives the bias (rms form excepted); NaN and infinity stay in their group."""
    d, prm = norm_case(3, 2, 64, torch.float32, "none", seed=5)
    d["x"][0] = 3.0
    d["x"][1, 5] = float("nan")
    d["x"][2, 70] = float("inf")
    y = torch.empty(3, 128, device="cuda")
    cb.cawn_group_norm_fwd(prm, d["x"].cuda(), y, weight=d["w"].cuda(), bias=d["b"].cuda())
    close(y[0], d["b"].double(), 2e-6)
    assert torch.isnan(y[1, :64]).all() and torch.isfinite(y[1, 64:]).all()
    assert torch.isfinite(y[2, :64]).all() and not torch.isfinite(y[2, 64:]).any()


def test_norm_gradient_against_differences():
    d, prm = norm_case(6, 3, 32, torch.float32, "gate", seed=6)
    c = {n: on_gpu(t) for n, t in d.items()}
    gx, gg, gw, gb = (torch.empty_like(c[n]) for n in ("x", "gate", "w", "b"))
    cb.cawn_group_norm_bwd(prm, c["x"], c["gy"], gx, cb.new_norm_workspace(prm), weight=c["w"], bias=c["b"], gate=c["gate"], grad_gate=gg, grad_weight=gw, grad_bias=gb)
    rng = torch.Generator().manual_seed(60)
    for name, grad in (("x", gx), ("gate", gg), ("w", gw), ("b", gb)):
        way = torch.randn(d[name].shape, generator=rng).double()
        def loss(h):
            w = {n: t.double() for n, t in d.items()}
            w[name] = w[name] + h * way
            return (group_norm(w["x"], 3, 1e-5, False, w["w"], w["b"], prm.act, w["gate"]) * d["gy"].double()).sum()
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        scale = grad.double().cpu().norm() * way.norm()
        assert abs((grad.double().cpu() * way).sum() - slope) <= 2e-6 * scale, name


def test_norm_in_place_and_empty():
    d, prm = norm_case(20, 4, 64, torch.bfloat16, "gate", seed=7)
    x, gate, w, b = (on_gpu(d[n]) for n in ("x", "gate", "w", "b"))
    y = torch.empty_like(x)
    cb.cawn_group_norm_fwd(prm, x, y, weight=w, bias=b, gate=gate)
    cb.cawn_group_norm_fwd(prm, x, x, weight=w, bias=b, gate=gate)
    assert torch.equal(x, y)
    none = cb.make_norm_params(0, 4, 64, act=cb.CAWN_NORM_ACT_GATE)
    cb.cawn_group_norm_fwd(none, x, y, gate=gate)
    gw, gb = torch.ones(256, device="cuda"), torch.ones(256, device="cuda")
    cb.cawn_group_norm_bwd(none, x, x, y, cb.new_norm_workspace(none), gate=gate, grad_gate=y, grad_weight=gw, grad_bias=gb)
    assert (gw == 0).all() and (gb == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1000, 4099])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9999999])
def test_dropout(p, n, dtype):
    rng = torch.Generator().manual_seed(n)
    x, r = torch.randn(n, generator=rng).to(dtype), torch.randn(n, generator=rng).to(dtype)
    seed, offset = 0x1234567890ABCDEF, 0xFEDCBA9876543210
    prm = cb.make_dropout_params(n, p, seed, offset, flags=flags_of(dtype))
    drop = min(round(p * 65536), 65535)
    keep = torch.from_numpy(philox_bits(n, seed, offset) >= drop)
    branch = torch.where(keep, x.double() * 65536 / (65536 - drop), 0.0)
    guard = torch.full((n + 64,), 5.0, dtype=dtype, device="cuda")
    cb.cawn_dropout(prm, x.cuda(), guard, residual=r.cuda())
    assert (guard[n:] == 5).all()
    close(guard[:n], branch + r.double(), TOL[dtype])
    y = torch.empty(n, dtype=dtype, device="cuda")
    cb.cawn_dropout(prm, x.cuda(), y)
    assert torch.equal((y == 0).cpu(), ~keep | (x == 0))
    if p == 0:
        assert torch.equal(y.cpu(), x)


def test_dropout_is_linear_and_selects():
    """Gradient = the same call; dropped infinities and NaN leave nothing behind; a device-side offset adds."""
    n, seed = 5000, 77
    prm = cb.make_dropout_params(n, 0.5, seed, 3)
    one = torch.empty(n, device="cuda")
    cb.cawn_dropout(prm, torch.ones(n, device="cuda"), one)
    assert set(one.unique().tolist()) == {0.0, 2.0}
    for bad in (float("inf"), float("nan")):
        y = torch.empty(n, device="cuda")
        cb.cawn_dropout(prm, torch.full((n,), bad, device="cuda"), y)
        assert (y[one == 0] == 0).all() and not torch.isfinite(y[one != 0]).any()
    extra = torch.tensor([40], dtype=torch.int64, device="cuda")
    a, b = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    cb.cawn_dropout(prm, torch.ones(n, device="cuda"), a, offset_device=extra)
    cb.cawn_dropout(cb.make_dropout_params(n, 0.5, seed, 43), torch.ones(n, device="cuda"), b)
    assert torch.equal(a, b) and not torch.equal(a, one)


def test_dropout_rate_and_in_place():
    n, p = 1 << 20, 0.25
    prm = cb.make_dropout_params(n, p, 5)
    x = torch.ones(n, device="cuda")
    cb.cawn_dropout(prm, x, x)
    kept = (x != 0).double().mean().item()
    assert abs(kept - (1 - p)) < 6 * (p * (1 - p) / n) ** 0.5       # six standard deviations
    assert abs(x.double().mean().item() - 1) < 6 * (p / (1 - p) / n) ** 0.5


def test_dropout_counter_beyond_32_bits_of_words():
    """The counter's second word: elements past 2^35 cannot be held, so it is checked through the definition
    of the first elements with an offset whose upper half is set."""
    n = 64
    y = torch.empty(n, device="cuda")
    cb.cawn_dropout(cb.make_dropout_params(n, 0.5, 1, 1 << 40), torch.ones(n, device="cuda"), y)
    assert np.array_equal((y != 0).cpu().numpy(), philox_bits(n, 1, 1 << 40) >= 32768)


@pytest.mark.parametrize("between", ["dropout", "norm", "delta step", "scan"])
@pytest.mark.parametrize("writer", ["norm", "dropout", "scan"])
def test_an_independent_input_written_two_calls_before(writer, between):
    """CAWN_FLAG_INPUT_INDEPENDENT says that the call just before does not write the input.  The one before that may:
    it has to be complete when the scan fetches its rows."""
    B, L, C, n = 8, 2048, 768, 4
    rng = torch.Generator(device="cuda").manual_seed(9)
    randn = lambda *s: torch.randn(*s, generator=rng, device="cuda")
    xs = [randn(B * L, 2 * C) for _ in range(n)]
    gamma, theta = torch.full((C,), 0.9, device="cuda"), torch.rand(C, generator=rng, device="cuda")
    p, small, y = torch.empty(B, L, C, dtype=torch.complex64, device="cuda"), randn(4096), torch.empty(4096, device="cuda")
    state, q = torch.zeros(1, 1, 64, 64, device="cuda"), randn(1, 1, 1, 64)
    one, o = torch.ones(1, 1, 1, device="cuda"), torch.empty(1, 1, 1, 64, device="cuda")
    little = torch.view_as_complex(randn(1, 64, 64, 2))
    little_y, little_prm = torch.empty_like(little), cb.make_params(1, 64, 1, 64)
    little_ws = cb.new_workspace(little_prm, cb.CAWN_OP_FWD)
    flat, plain = torch.view_as_real(p).view(B * L, 2 * C), cb.make_params(B, L, 12, 64)
    plain_ws = cb.new_workspace(plain, cb.CAWN_OP_FWD)
    first = {"norm": lambda x: cb.cawn_group_norm_fwd(cb.make_norm_params(B * L, 1, 2 * C), x, flat),
             "dropout": lambda x: cb.cawn_dropout(cb.make_dropout_params(x.numel(), 0.1, 3), x, flat),
             "scan": lambda x: cb.cawn_phase_accumulate_fwd(plain, torch.view_as_complex(x.view(B, L, C, 2)), gamma, theta, p, plain_ws)}[writer]
    second = {"dropout": lambda: cb.cawn_dropout(cb.make_dropout_params(4096, 0.1, 3), small, y),
              "norm": lambda: cb.cawn_group_norm_fwd(cb.make_norm_params(64, 1, 64), small, y),
              "delta step": lambda: cb.cawn_delta_rule_step(cb.make_delta_params(1, 1, 1, 1, 64, 64), q, q, q, -one, one, o, state, state),
              "scan": lambda: cb.cawn_phase_accumulate_fwd(little_prm, little, gamma[:64], theta[:64], little_y, little_ws)}[between]
    outs = []
    for flags in (0, cb.CAWN_FLAG_INPUT_INDEPENDENT):
        prm = cb.make_params(B, L, 12, 64, flags=flags)
        ws, ys = cb.new_workspace(prm, cb.CAWN_OP_FWD), [torch.empty_like(p) for _ in range(n)]
        torch.cuda.synchronize()
        for i in range(n):
            first(xs[i])
            second()
            cb.cawn_phase_accumulate_fwd(prm, p, gamma, theta, ys[i], ws)
            torch.cuda.synchronize()
        assert cb.cawn_poll_status(ws) == 0
        outs.append(ys)
    for a, b in zip(*outs):
        assert torch.equal(torch.view_as_real(a), torch.view_as_real(b))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(20, 4, 64), (3, 2, 4096), (9, 5, 37)], ids=str)
def test_norm_over_its_inputs(shape, dtype):
    """y may take the place of x or of the gate, grad_x that of grad_y (teams of lanes, whole blocks and odd widths)."""
    d, prm = norm_case(*shape, dtype, "gate", seed=70)
    x, gate, gy, w, b = (on_gpu(d[n]) for n in ("x", "gate", "gy", "w", "b"))
    y = torch.empty_like(x)
    cb.cawn_group_norm_fwd(prm, x, y, weight=w, bias=b, gate=gate)
    for n in ("x", "gate"):
        t = {"x": x.clone(), "gate": gate.clone()}
        cb.cawn_group_norm_fwd(prm, t["x"], t[n], weight=w, bias=b, gate=t["gate"])
        assert torch.equal(t[n], y), n
    gx, gg, over = torch.empty_like(x), torch.empty_like(x), gy.clone()
    sums = [torch.empty_like(w) for _ in range(4)]
    cb.cawn_group_norm_bwd(prm, x, gy, gx, cb.new_norm_workspace(prm), weight=w, bias=b, gate=gate, grad_gate=gg, grad_weight=sums[0], grad_bias=sums[1])
    again = torch.empty_like(gg)
    cb.cawn_group_norm_bwd(prm, x, over, over, cb.new_norm_workspace(prm), weight=w, bias=b, gate=gate, grad_gate=again, grad_weight=sums[2], grad_bias=sums[3])
    assert torch.equal(over, gx) and torch.equal(again, gg) and torch.equal(sums[0], sums[2]) and torch.equal(sums[1], sums[3])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(300, 12, 64), (890, 12, 64), (7, 8, 1024), (50, 2, 4096), (5, 5, 37)], ids=str)
def test_norm_keeps_to_its_workspace(shape, dtype):
    d, prm = norm_case(*shape, dtype, "silu", seed=71)
    x, gy, w, b = (on_gpu(d[n]) for n in ("x", "gy", "w", "b"))
    n = cb.cawn_group_norm_workspace_bytes(prm)
    ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    cb.cawn_group_norm_bwd(prm, x, gy, gx, ws[:n], weight=w, bias=b, grad_weight=gw, grad_bias=gb)
    assert (ws[n:] == 0xA5).all()


def test_dropout_over_its_residual():
    n = 4099
    rng = torch.Generator().manual_seed(72)
    x, r = torch.randn(n, generator=rng).cuda(), torch.randn(n, generator=rng).cuda()
    prm = cb.make_dropout_params(n, 0.3, 9, 2)
    y = torch.empty_like(x)
    cb.cawn_dropout(prm, x, y, residual=r)
    cb.cawn_dropout(prm, x, r, residual=r)
    assert torch.equal(y, r)


def test_dropout_draws_the_published_bits():
    """Counter and key of zeros: an element is kept while the threshold is at most its bits."""
    words = PHILOX_ANSWERS[0][2]
    bits = [half for w in words for half in (w & 0xFFFF, w >> 16)]
    y = torch.empty(8, device="cuda")
    for i, b in enumerate(bits):
        for threshold in (b, b + 1):
            cb.cawn_dropout(cb.make_dropout_params(8, threshold / 65536, 0), torch.ones(8, device="cuda"), y)
            assert (y != 0).tolist() == [x >= threshold for x in bits], (i, threshold)


def test_dropout_of_more_than_2_35_elements():
    """The counter's second word is the upper half of element / 8: the last elements of an array of 2^35 + 64 (in place, 69 GB
    of bfloat16)."""
    n = (1 << 35) + 64
    if torch.cuda.mem_get_info()[0] < 90 * (1 << 30):
        pytest.skip("less than 90 GB of device memory free")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    seed, offset = 0x0123456789ABCDEF, 5
    cb.cawn_dropout(cb.make_dropout_params(n, 0.5, seed, offset, flags=flags_of(x.dtype)), x, x)
    tail = (x[-128:] != 0).cpu().numpy()
    del x
    torch.cuda.empty_cache()
    bits = []
    for i in range(n // 8 - 16, n // 8):
        for w in philox_words((i & 0xFFFFFFFF, i >> 32, offset, 0), (seed & 0xFFFFFFFF, seed >> 32)):
            bits += [w & 0xFFFF, w >> 16]
    assert np.array_equal(tail, np.array(bits) >= 32768)
