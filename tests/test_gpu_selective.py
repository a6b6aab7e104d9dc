"""Selective scan against its definition in 64 bits.

Tolerances (relative 2-norm), float storage: a token's decay is off by some 2^-22 (its exponential, the product in front of it, the
product with the state), and a state remembers 1 / (1 - decay) tokens, up to 600 here: as independent errors sqrt(600) 2^-22 = 6e-6,
and as much again for what else is rounded: 1.2e-5, for results and gradients (the sums over channels drop 2^-22 of a term).
bfloat16 storage: results are rounded once and compared with the definition rounded once, 2^-9.  States and parameters' gradients
are float in both.
"""
import pytest
import torch

from delta_ref import close as close64
from paper_2604_04250_b200 import binding as cb
from selective_ref import flags_of, packed_offsets, selective_scan, slices

pytestmark = pytest.mark.gpu
FLOAT = 1.2e-5
TOL = {torch.float32: FLOAT, torch.bfloat16: 2.0 ** -9}
DTYPES = [torch.float32, torch.bfloat16]
LEAVES = ("x", "dt", "A", "B", "C", "skip", "dt_bias", "z", "state_in")
DENSE = ("x", "dt", "z", "B", "C")


def close(got, want, tol, what=""):
    close64(got, want.detach().to(torch.bfloat16) if got.dtype == torch.bfloat16 else want, tol, what)


def case(offsets, D, N, G, dtype, seed=0, rows=None, pad=0, softplus=True):
    rng = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=rng)
    B, rows = len(offsets) - 1, offsets[-1] if rows is None else rows
    step = 0.002 * 50 ** torch.rand(D, generator=rng)
    d = {"x": randn(rows, D).to(dtype), "dt": (0.5 * randn(rows, D)).to(dtype) if softplus else (step * torch.exp(0.5 * randn(rows, D))).to(dtype),
         "A": -torch.arange(1.0, N + 1) * torch.exp(0.2 * randn(D, N)), "B": randn(rows, G, N).to(dtype), "C": randn(rows, G, N).to(dtype),
         "skip": 1 + 0.2 * randn(D), "dt_bias": torch.log(torch.expm1(step)) if softplus else 0.001 * torch.rand(D, generator=rng), "z": randn(rows, D).to(dtype),
         "state_in": 0.5 * randn(B, D, N), "grad_y": randn(rows, D).to(dtype), "grad_state_out": 0.3 * randn(B, D, N)}
    c = {n: t.cuda() for n, t in d.items()}
    for n in ("x", "dt", "z"):
        c[n] = slices(d[n], pad)
    for n in ("B", "C"):
        c[n] = slices(d[n].flatten(1), pad)
    return d, c


def params(offsets, D, N, G, dtype, packed=False, rows=None, L=None, pad=0, softplus=True, z=True):
    longest = max(b - a for a, b in zip(offsets, offsets[1:]))
    p = 2 * pad
    return cb.make_scan_params(len(offsets) - 1, longest if L is None else L, D, N, G, softplus, flags_of(dtype), *((D + p,) * 3 if p else (0, 0, 0)),
                               *((G * N + p,) * 2 if p else (0, 0)), rows=(offsets[-1] if rows is None else rows) if packed else 0)


def forward(prm, c, off=None, absent=(), checkpoints=None, mark=7.0, **kw):
    y, so = torch.full(c["grad_y"].shape, mark, dtype=c["grad_y"].dtype, device="cuda"), torch.full_like(c["state_in"], float("nan"))
    ws = cb.new_scan_workspace(prm, cb.CAWN_SCAN_FWD)
    ws.fill_(0xFF)
    opt = {n: None if n in absent else c[n] for n in ("skip", "dt_bias", "z", "state_in")}
    cb.cawn_selective_scan_fwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y, ws, state_out=so, offsets=off, checkpoints=checkpoints, **opt, **kw)
    return y, so


def backward(prm, c, off=None, absent=(), checkpoints=None, mark=7.0, workspace=None):
    op = cb.CAWN_SCAN_BWD if checkpoints is not None else cb.CAWN_SCAN_BWD_RECOMPUTE
    ws = cb.new_scan_workspace(prm, op) if workspace is None else workspace
    ws.fill_(0xFF)
    rows = c["grad_y"].shape[0]
    dtype = c["grad_y"].dtype
    full = lambda n, *s: torch.full(s, mark if n in DENSE else float("nan"), dtype=dtype if n in DENSE else torch.float32, device="cuda")
    D, N, G = prm.D, prm.N, prm.G
    g = {"x": full("x", rows, D), "dt": full("dt", rows, D), "z": full("z", rows, D), "B": full("B", rows, G, N), "C": full("C", rows, G, N)}
    g.update({n: torch.full_like(c[n], float("nan")) for n in ("A", "skip", "dt_bias", "state_in")})
    opt = {n: None if n in absent else c[n] for n in ("skip", "dt_bias", "z", "state_in")}
    cb.cawn_selective_scan_bwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], c["grad_y"], g["x"], g["dt"], g["A"], g["B"], g["C"], ws, offsets=off,
                               checkpoints=checkpoints, grad_state_out=c["grad_state_out"], grad_skip=g["skip"], grad_dt_bias=g["dt_bias"],
                               grad_z=None if "z" in absent else g["z"], grad_state_in=g["state_in"], **opt)
    return g


def check(offsets, D, N, G, dtype, packed=False, rows=None, L=None, pad=0, absent=(), softplus=True, seed=0, saved=True):
    rows = offsets[-1] if rows is None else rows
    d, c = case(offsets, D, N, G, dtype, seed, rows, pad, softplus)
    prm = params(offsets, D, N, G, dtype, packed, rows, L, pad, softplus)
    off = torch.tensor(offsets, device="cuda") if packed else None
    marks = cb.new_scan_workspace(prm, cb.CAWN_SCAN_CHECKPOINTS) if saved else None
    y, so = forward(prm, c, off, absent, marks)
    w = {n: d[n].double().requires_grad_() for n in LEAVES}
    a = {n: None if n in absent and n != "state_in" else w[n] for n in LEAVES}
    state = torch.zeros_like(w["state_in"]) if "state_in" in absent else w["state_in"]
    want, want_state = selective_scan(a["x"], a["dt"], a["A"], a["B"], a["C"], a["skip"], a["dt_bias"], a["z"], state, offsets, prm.L, softplus)
    own = torch.zeros(rows, dtype=torch.bool)
    for i, e in zip(offsets, offsets[1:]):
        own[i:min(e, i + prm.L)] = True
    close(y[own], want[own], TOL[dtype], "y")
    close(so, want_state, FLOAT, "state_out")
    assert (y[~own] == 7).all()

    g = backward(prm, c, off, absent, marks)
    names = [n for n in LEAVES if n not in absent]
    got = torch.autograd.grad([want, want_state], [w[n] for n in names], [d["grad_y"].double() * own[:, None], d["grad_state_out"].double()], allow_unused=True)
    for n, t in zip(names, got):
        t = torch.zeros_like(w[n]) if t is None else t
        if n in DENSE:
            close(g[n][own], t[own], TOL[dtype], "grad_" + n)
            assert (g[n][~own] == 7).all(), n
        else:
            close(g[n], t, FLOAT, "grad_" + n)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, L, D, N, G", [(1, 1, 8, 16, 1), (2, 1, 40, 16, 1), (1, 2, 32, 4, 1), (2, 15, 32, 16, 1), (1, 16, 64, 16, 2), (3, 17, 33, 5, 1), (2, 31, 96, 24, 1),
                                           (1, 32, 32, 32, 1), (2, 33, 24, 64, 1), (1, 49, 70, 16, 2), (2, 70, 160, 16, 1), (1, 40, 12, 1, 3), (2, 50, 64, 8, 4),
                                           (1, 65, 48, 40, 1), (1, 97, 35, 63, 1), (1, 130, 16, 7, 1)])
def test_dense(B, L, D, N, G, dtype):
    check([i * L for i in range(B + 1)], D, N, G, dtype, seed=B + L + D + N)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D, N, lengths", [(224, 8, 70 * (37,)), (221, 3, 71 * (34,)), (224, 16, 46 * (33,)), (221, 16, 46 * (50,)), (224, 16, 46 * (1,)), (200, 24, 26 * (49,)),
                                           (203, 29, 26 * (17,)), (224, 16, 12 * (37, 0, 50, 16, 1)), (221, 13, 12 * (2, 33, 0, 47, 15)), (200, 32, 6 * (31, 0, 32, 5, 48))])
def test_more_blocks_than_half_of_the_places(D, N, lengths, dtype):
    """Calls that fill the device; those of few blocks have warps of their own for finishing."""
    check(packed_offsets(lengths, 0), D, N, 1, dtype, packed=len(set(lengths)) > 1, seed=D + N)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, L, D, N", [(1, 700, 40, 16), (2, 1100, 24, 4), (1, 800, 16, 64), (1, 523, 33, 24), (1, 1030, 8, 8)])
@pytest.mark.parametrize("saved", [True, False])
def test_segments(B, L, D, N, saved, dtype):
    """Few channels: the time axis is cut, in both directions; with and without the forward's checkpoints."""
    prm = cb.make_scan_params(B, L, D, N)
    assert cb.cawn_selective_scan_workspace_bytes(prm, cb.CAWN_SCAN_FWD) > 0
    check([i * L for i in range(B + 1)], D, N, 1, dtype, seed=L, saved=saved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths, G, N", [((600,), 148, 9), ((600, 3, 0, 40), 90, 12), ((523,), 70, 16), ((1040,), 37, 5), ((385, 385), 30, 20)])
@pytest.mark.parametrize("saved", [True, False])
def test_segments_of_many_blocks(lengths, G, N, saved, dtype):
    """A block a channel: segments that fill the device, so that the backward's pass before them takes them whole."""
    check(packed_offsets(lengths, 0), G, N, G, dtype, packed=len(lengths) > 1, seed=G, saved=saved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths, first, behind", [((5, 0, 1, 70, 2), 0, 0), ((0, 0), 3, 4), ((130, 1, 64), 2, 5), ((1,), 0, 1), ((0, 90, 0, 33, 16), 0, 0),
                                                    ((600, 0, 300, 5), 7, 3)])
@pytest.mark.parametrize("D, N, G, saved", [(40, 16, 1, True), (26, 5, 2, False)])
def test_packed(D, N, G, saved, lengths, first, behind, dtype):
    offsets = packed_offsets(lengths, first)
    check(offsets, D, N, G, dtype, packed=True, rows=offsets[-1] + behind, seed=len(lengths) + D, saved=saved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("absent", [("z",), ("skip", "dt_bias"), ("state_in",), ("z", "skip", "dt_bias", "state_in")])
@pytest.mark.parametrize("pad", [0, 8, 24, 4, 3, 1])
def test_slices_and_absent_arrays(pad, absent, dtype):
    check([0, 40, 80], 48, 16, 1, dtype, pad=pad, absent=absent)


@pytest.mark.parametrize("dtype", DTYPES)
def test_steps_as_they_are(dtype):
    check([0, 40, 80], 40, 16, 1, dtype, softplus=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [1, 3])
def test_rows_of_B_and_C_that_begin_at_any_element(shift, dtype):
    d, c = case([0, 40], 32, 16, 1, dtype)
    prm = params([0, 40], 32, 16, 1, dtype)
    want = forward(prm, c)
    wide = torch.zeros(40, 32 + shift, dtype=dtype, device="cuda")
    wide[:, shift:shift + 16], wide[:, shift + 16:] = c["B"], c["C"]
    prm.b_stride = prm.c_stride = 32 + shift
    c["B"], c["C"] = wide[:, shift:shift + 16], wide[:, shift + 16:]
    got = forward(prm, c)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_longer_sequences_than_said_and_offsets_outside():
    check([0, 50, 90], 40, 16, 1, torch.float32, packed=True, L=40, rows=96)
    d, c = case([0, 50, 90], 32, 16, 1, torch.float32, rows=90)
    prm = params([0, 50, 90], 32, 16, 1, torch.float32, True, 90)
    y, so = forward(prm, c, torch.tensor([-5, 30, 10 ** 12], device="cuda"))
    w = {n: t.double() for n, t in d.items()}
    want, state = selective_scan(*(w[n] for n in LEAVES), [0, 30, 90], 50)
    close(y[:80], want[:80], FLOAT)
    close(so, state, FLOAT)
    assert (y[80:] == 7).all()
    marks = cb.new_scan_workspace(prm, cb.CAWN_SCAN_CHECKPOINTS)
    off = torch.tensor([60, 30, -10], device="cuda")                      # they fall: nothing to do
    y, so = forward(prm, c, off, checkpoints=marks)
    g = backward(prm, c, off, checkpoints=marks)
    assert (y == 7).all() and torch.equal(so, c["state_in"]) and (g["x"] == 7).all() and (g["B"] == 7).all()
    assert torch.equal(g["state_in"], c["grad_state_out"]) and (g["A"] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D, N, G", [(40, 16, 1), (7, 5, 1), (64, 64, 2), (33, 24, 1), (16, 1, 1), (20, 37, 2)])
@pytest.mark.parametrize("B", [3, 5])
def test_tokens_one_by_one(B, D, N, G, dtype):
    """Single tokens with the states in place, several at a time, and the whole sequence: against the definition each."""
    L = 12
    offsets = [i * L for i in range(B + 1)]
    d, c = case(offsets, D, N, G, dtype, seed=D + N)
    w = {n: t.double() for n, t in d.items()}
    want, want_state = selective_scan(*(w[n] for n in LEAVES), offsets, L)
    for some in (1, 4):
        prm, state, parts = cb.make_scan_params(B, some, D, N, G, flags=flags_of(dtype)), c["state_in"].clone(), []
        for t in range(0, L, some):
            now = {n: c[n].view(B, L, -1)[:, t:t + some].contiguous() for n in DENSE}
            y = torch.empty(B, some, D, dtype=dtype, device="cuda")
            cb.cawn_selective_scan_step(prm, now["x"], now["dt"], c["A"], now["B"], now["C"], y, skip=c["skip"], dt_bias=c["dt_bias"], z=now["z"],
                                        state_in=state, state_out=state)
            parts.append(y)
        close(torch.cat(parts, 1).view(B * L, D), want, TOL[dtype], "y")
        close(state, want_state, FLOAT, "state")
    for pad in (1, 8):                              # slices, whose strides the params name
        s = {n: slices(d[n].flatten(1), pad) for n in DENSE}
        prm = cb.make_scan_params(B, L, D, N, G, True, flags_of(dtype), *(s[n].stride(0) for n in ("x", "dt", "z", "B", "C")))
        y, state = torch.empty(B * L, D, dtype=dtype, device="cuda"), c["state_in"].clone()
        cb.cawn_selective_scan_step(prm, s["x"], s["dt"], c["A"], s["B"], s["C"], y, skip=c["skip"], dt_bias=c["dt_bias"], z=s["z"], state_in=state, state_out=state)
        close(y, want, TOL[dtype], "y of slices")
        close(state, want_state, FLOAT, "state of slices")
    y = torch.empty(B * L, D, dtype=dtype, device="cuda")
    cb.cawn_selective_scan_step(cb.make_scan_params(B, L, D, N, G, flags=flags_of(dtype)), c["x"], c["dt"], c["A"], c["B"], c["C"], y)
    want, _ = selective_scan(*(w[n] for n in ("x", "dt", "A", "B", "C")), None, None, None, torch.zeros(B, D, N, dtype=torch.double), offsets, L)
    close(y, want, TOL[dtype], "y from no state")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, D, N", [(70, 300, 16), (61, 1100, 5), (40, 512, 24), (33, 5000, 2), (66, 130, 64)])
def test_single_tokens_of_a_batch(B, D, N, dtype):
    """Enough of them that a thread takes four sequences, the last of which may be fewer."""
    offsets = list(range(B + 1))
    d, c = case(offsets, D, N, 1, dtype, seed=B)
    w = {n: t.double() for n, t in d.items()}
    want, want_state = selective_scan(*(w[n] for n in LEAVES), offsets, 1)
    y, state = torch.empty(B, D, dtype=dtype, device="cuda"), c["state_in"].clone()
    cb.cawn_selective_scan_step(cb.make_scan_params(B, 1, D, N, flags=flags_of(dtype)), c["x"], c["dt"], c["A"], c["B"], c["C"], y, skip=c["skip"], dt_bias=c["dt_bias"],
                                z=c["z"], state_in=state, state_out=state)
    close(y, want, TOL[dtype], "y")
    close(state, want_state, FLOAT, "state")


def test_state_in_place_and_prompts_in_pieces():
    """The state may be written over, also where segments run side by side; a prompt in pieces ends as it does whole."""
    B, L, D, N = 2, 900, 24, 16
    d, c = case([0, L, 2 * L], D, N, 1, torch.float32)
    prm = params([0, L, 2 * L], D, N, 1, torch.float32)
    y, so = forward(prm, c)
    state = c["state_in"].clone()
    ws = cb.new_scan_workspace(prm, cb.CAWN_SCAN_FWD)
    y2 = torch.empty_like(y)
    same = {n: c[n] for n in ("skip", "dt_bias", "z")}
    cb.cawn_selective_scan_fwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y2, ws, state_in=state, state_out=state, **same)
    assert torch.equal(y, y2) and torch.equal(so, state)
    state, parts = c["state_in"].clone(), []
    for a, e in ((0, 1), (1, 700), (700, 900)):
        now = {n: c[n].view(B, L, -1)[:, a:e].contiguous() for n in DENSE}
        part = torch.empty(B, e - a, D, device="cuda")
        cb.cawn_selective_scan_fwd(cb.make_scan_params(B, e - a, D, N), now["x"], now["dt"], c["A"], now["B"], now["C"], part, ws, skip=c["skip"],
                                   dt_bias=c["dt_bias"], z=now["z"], state_in=state, state_out=state)
        parts.append(part)
    close(torch.cat(parts, 1).view(2 * L, D), y, FLOAT)
    close(state, so, FLOAT)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_tokens(dtype):
    d, c = case([0, 0, 0], 40, 16, 1, dtype, rows=0)
    prm = cb.make_scan_params(2, 0, 40, 16, flags=flags_of(dtype))
    so = torch.empty_like(c["state_in"])
    cb.cawn_selective_scan_fwd(prm, None, None, c["A"], None, None, None, state_in=c["state_in"], state_out=so)
    assert torch.equal(so, c["state_in"])
    so.zero_()
    cb.cawn_selective_scan_step(prm, None, None, c["A"], None, None, None, state_in=c["state_in"], state_out=so)
    assert torch.equal(so, c["state_in"])
    gA, gs, ws = torch.full_like(c["A"], 7.0), torch.empty_like(so), cb.new_scan_workspace(prm, cb.CAWN_SCAN_BWD_RECOMPUTE)
    ws.fill_(0xFF)
    cb.cawn_selective_scan_bwd(prm, None, None, c["A"], None, None, None, None, None, gA, None, None, ws, state_in=c["state_in"],
                               grad_state_out=c["grad_state_out"], grad_state_in=gs)
    assert torch.equal(gs, c["grad_state_out"]) and (gA == 0).all()


def test_strong_and_absent_decays():
    """Steps of 0 leave the state as it is, steps that forget everything leave the token's own term alone, and a sum of steps
    whose decay underflows does not turn the state into anything else."""
    d, c = case([0, 60], 32, 16, 1, torch.float32, softplus=False)
    d["dt"][:], d["dt_bias"][:] = 0.0, 0.0
    d["dt"][20:40] = 60.0
    for n in ("dt", "dt_bias"):
        c[n] = d[n].cuda()
    prm = params([0, 60], 32, 16, 1, torch.float32, softplus=False)
    y, so = forward(prm, c)
    w = {n: t.double().requires_grad_() for n, t in d.items()}
    want, state = selective_scan(*(w[n] for n in LEAVES), [0, 60], 60, softplus=False)
    close(y, want, FLOAT)
    close(so, state, FLOAT)
    g = backward(prm, c)
    for n, t in zip(LEAVES, torch.autograd.grad([want, state], [w[n] for n in LEAVES], [d["grad_y"].double(), d["grad_state_out"].double()])):
        close(g[n], t, FLOAT, n)


def test_softplus_over_its_range():
    """Steps from 1e-38 to 1e30: relative error of a few roundings (the exponent's product is rounded: 87 2^-24 at the lower end)."""
    v = torch.cat([torch.linspace(-87, 87, 4096), torch.tensor([1e30, 0.0, -0.0, 1e-30, -1e-30])])
    n = v.numel()
    y = torch.empty(n, 1, device="cuda")
    one = torch.ones(1, 1, device="cuda")
    # h = d x B with x = B = 1, A = 0 and a state of nothing; y = h
    cb.cawn_selective_scan_fwd(cb.make_scan_params(n, 1, 1, 1), torch.ones(n, 1, device="cuda"), v.cuda()[:, None].contiguous(), torch.zeros(1, 1, device="cuda"),
                               torch.ones(n, 1, device="cuda"), torch.ones(n, 1, device="cuda"), y)
    want = torch.nn.functional.softplus(v.double(), threshold=1e300)
    assert ((y[:, 0].double().cpu() - want).abs() <= want * 6e-6).all()
    near = v.abs() < 10
    assert ((y[:, 0].double().cpu() - want).abs()[near] <= want[near] * 1e-6).all()


def test_non_finite_values_stay_in_their_sequence_and_group():
    d, c = case([0, 40, 80], 64, 16, 2, torch.float32)
    prm = params([0, 40, 80], 64, 16, 2, torch.float32)
    clean, state = forward(prm, c)
    gclean = backward(prm, c)
    c["x"][50, 3] = float("inf")
    y, so = forward(prm, c)
    bad = ~torch.isfinite(y)
    assert bad[50:, 3].all() and not bad[:50].any() and not bad[:, :3].any() and not bad[:, 4:].any()
    assert torch.equal(y[:50], clean[:50]) and torch.equal(so[0], state[0])
    g = backward(prm, c)
    assert torch.equal(g["B"][:40], gclean["B"][:40]) and torch.equal(g["B"][:, 1], gclean["B"][:, 1])      # sequence 0; group 1
    assert torch.equal(g["x"][:, 4:], gclean["x"][:, 4:]) and torch.equal(g["A"][4:], gclean["A"][4:])
    assert torch.isfinite(g["C"][40:48]).all()                              # the eight tokens of a selection before it reach no further


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L", [70, 900])
def test_streams_graphs_and_repeats(L, dtype):
    """Captured on another stream and replayed on new inputs, forward and backward give the bits of plain calls; so do repeats."""
    B, D, N = 2, 40, 16
    d, c = case([0, L, 2 * L], D, N, 1, dtype)
    prm = params([0, L, 2 * L], D, N, 1, dtype)
    wf, wb, marks = (cb.new_scan_workspace(prm, op) for op in (cb.CAWN_SCAN_FWD, cb.CAWN_SCAN_BWD, cb.CAWN_SCAN_CHECKPOINTS))
    y, so = torch.empty_like(c["x"]), torch.empty_like(c["state_in"])
    g = {n: torch.empty_like(c[n]) for n in LEAVES}
    same = {n: c[n] for n in ("skip", "dt_bias", "z", "state_in")}

    def both():
        cb.cawn_selective_scan_fwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y, wf, state_out=so, checkpoints=marks, **same)
        cb.cawn_selective_scan_bwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], c["grad_y"], g["x"], g["dt"], g["A"], g["B"], g["C"], wb, checkpoints=marks,
                                   grad_state_out=c["grad_state_out"], grad_skip=g["skip"], grad_dt_bias=g["dt_bias"], grad_z=g["z"],
                                   grad_state_in=g["state_in"], **same)

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
    got = [t.clone() for t in (y, so, *g.values())]
    for _ in range(2):
        for t in (wf, wb, marks):
            t.fill_(0xFF)
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, so, *g.values())))


def test_two_calls_at_once_with_a_workspace_each():
    d, c = case([0, 1500], 64, 16, 1, torch.float32)
    prm = params([0, 1500], 64, 16, 1, torch.float32)
    want = forward(prm, c)[0]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want) for _ in range(2)]
    spaces = [cb.new_scan_workspace(prm, cb.CAWN_SCAN_FWD) for _ in range(2)]
    torch.cuda.synchronize()
    same = {n: c[n] for n in ("skip", "dt_bias", "z", "state_in")}
    for _ in range(4):
        for s, y, ws in zip(streams, outs, spaces):
            cb.cawn_selective_scan_fwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y, ws, stream=s, **same)
    torch.cuda.synchronize()
    assert all(torch.equal(want, y) for y in outs)


def test_a_workspace_of_the_largest_call_serves_smaller_ones():
    big = cb.make_scan_params(3, 1200, 40, 16)
    ws = cb.new_scan_workspace(big, cb.CAWN_SCAN_BWD_RECOMPUTE)
    for B, L in ((1, 1200), (2, 1200), (3, 600), (1, 300), (3, 1200), (3, 20)):
        offsets = [i * L for i in range(B + 1)]
        d, c = case(offsets, 40, 16, 1, torch.float32)
        prm = params(offsets, 40, 16, 1, torch.float32)
        got, want = backward(prm, c, workspace=ws), backward(prm, c)
        assert all(torch.equal(got[n], want[n]) for n in LEAVES)


def test_gradient_against_differences():
    """A step along the gradient's own direction: rounding of a float loss summed in double (2^-24 of about 2e3 terms of order one
    over a step of 1e-2: 2e-5) and the third-order term (1e-4 of a slope of order one; a few times that for the exponentials)."""
    offsets = [0, 50, 83]
    d, c = case(offsets, 24, 8, 2, torch.float32, seed=4)
    prm = params(offsets, 24, 8, 2, torch.float32, True)
    off = torch.tensor(offsets, device="cuda")
    c["grad_state_out"].zero_()
    g = backward(prm, c, off)

    def loss(n, step):
        p = dict(c)
        p[n] = c[n] + step * (g[n] / g[n].norm()).view_as(c[n])
        return (forward(prm, p, off)[0].double() * c["grad_y"].double()).sum().item()

    for n in LEAVES:
        slope, want = (loss(n, 1e-2) - loss(n, -1e-2)) / 2e-2, g[n].norm().item()
        assert abs(slope - want) < 2e-3 * want, n


def test_more_than_32_bits_of_elements():
    """2.2e9 elements an array: the second half alone, from the first half's state, gives the same as the whole call."""
    L, D, N = 1_100_000, 2000, 2
    half, dtype = 560_000, torch.bfloat16
    rng = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(L, D, generator=rng, device="cuda", dtype=dtype)
    dt = torch.full((L, D), -2.0, device="cuda", dtype=dtype)
    dt[:, ::3] = -5.0
    BC = torch.randn(L, 2 * N, generator=rng, device="cuda", dtype=dtype)
    A = -torch.rand(D, N, generator=rng, device="cuda") - 0.1
    y, so = torch.empty(L, D, device="cuda", dtype=dtype), torch.empty(1, D, N, device="cuda")
    assert x.numel() > 2 ** 31

    def forward(a, e, y, state_in, state_out):
        prm = cb.make_scan_params(1, e - a, D, N, flags=flags_of(dtype), b_stride=2 * N, c_stride=2 * N)
        cb.cawn_selective_scan_fwd(prm, x[a:e], dt[a:e], A, BC[a:e, :N], BC[a:e, N:], y[a:e], cb.new_scan_workspace(prm, cb.CAWN_SCAN_FWD), state_in=state_in, state_out=state_out)

    forward(0, L, y, None, so)
    mid, end = torch.empty_like(so), torch.empty_like(so)
    z = torch.empty_like(y)
    forward(0, half, z, None, mid)
    forward(half, L, z, mid, end)
    close(end, so.cpu(), FLOAT, "state")
    close(z[-2000:], y[-2000:].cpu(), 2.0 ** -9, "the last rows")
    close(z[half - 1000:half + 1000], y[half - 1000:half + 1000].cpu(), 2.0 ** -9, "the rows around the middle")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N", [4, 16, 32, 64])
@pytest.mark.parametrize("other", [1, 2, 7, 31, 45])
def test_terms_of_sums_over_channels_keep_their_bits(other, N, dtype):
    """Channel 0 has steps of s + k 2^-23, another one steps of s = 1.3333332539 (all 24 bits in use) and the opposite x; every other channel
    has x = 0, B = C = 1 and decays are 0.  So the terms of dB and dC are these steps with a sign (lam = dy' = 1: dB = sum d x, and h = d x:
    dC = sum d x), and their sums k 2^-23: whole numbers of up to 8 bits times a power of two, which every storage holds and sums of 24
    bits give exactly in any order."""
    D, L = 64, 21
    offsets = [0, L]
    for k in (1, 3, 77, 255, 0x540000):
        d, c = case(offsets, D, N, 1, dtype, softplus=False)
        sign = 1.0 - 2.0 * (torch.arange(L) % 2)
        new = {"x": torch.zeros(L, D), "dt": torch.ones(L, D), "A": torch.full((D, N), -200.0), "B": torch.ones(L, 1, N), "C": torch.ones(L, 1, N),
               "dt_bias": torch.zeros(D), "grad_y": torch.zeros(L, D), "grad_state_out": torch.zeros(1, D, N)}
        new["x"][:, 0], new["x"][:, other] = sign, -sign
        new["grad_y"][:, 0] = new["grad_y"][:, other] = 1.0
        new["dt_bias"][0], new["dt_bias"][other] = (0x2AAAAA + k) * 2.0 ** -23, 0x2AAAAA * 2.0 ** -23
        c.update({n: t.to(c[n].dtype).cuda() for n, t in new.items()})
        g = backward(params(offsets, D, N, 1, dtype, softplus=False, z=False), c, absent=("z", "state_in"))
        want = (sign * k * 2.0 ** -23)[:, None, None].expand(L, 1, N).to(dtype)
        assert torch.equal(g["B"].cpu(), want), (k, (g["B"].cpu().float() - want).abs().max())
        assert torch.equal(g["C"].cpu(), want), (k, (g["C"].cpu().float() - want).abs().max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L, D, N", [(21, 40, 16), (16, 40, 16), (3, 33, 5), (50, 24, 24), (40, 16, 64), (700, 40, 16), (523, 24, 7)])
def test_rates_that_forget_everything(L, D, N, dtype):
    """A of -infinity, and of a size that its product with log2 e does not hold: such a state is its own token's term alone, also behind the last
    token of a tile that is not full.  (The definition's gradient of dt is 0 times infinity there, so that one and dt_bias's are left out.)"""
    offsets = [0, L, 2 * L]
    d, c = case(offsets, D, N, 1, dtype, seed=L)
    d["A"][:, ::3], d["A"][::2, 1] = float("-inf"), -3e38
    c["A"] = d["A"].cuda()
    prm = params(offsets, D, N, 1, dtype)
    marks = cb.new_scan_workspace(prm, cb.CAWN_SCAN_CHECKPOINTS)
    y, so = forward(prm, c, checkpoints=marks)
    w = {n: t.double().requires_grad_() for n, t in d.items()}
    want, state = selective_scan(*(w[n] for n in LEAVES), offsets, L)
    close(y, want, TOL[dtype], "y")
    close(so, state, FLOAT, "state_out")
    names = [n for n in LEAVES if n not in ("dt", "dt_bias")]
    leaves = torch.autograd.grad([want, state], [w[n] for n in names], [d["grad_y"].double(), d["grad_state_out"].double()])
    for saved in (marks, None):
        g = backward(prm, c, checkpoints=saved)
        for n, t in zip(names, leaves):
            close(g[n], t, TOL[dtype] if n in DENSE else FLOAT, "grad_" + n)
    if L < 60:
        y, so = torch.empty_like(y), torch.empty_like(so)
        cb.cawn_selective_scan_step(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y, skip=c["skip"], dt_bias=c["dt_bias"], z=c["z"], state_in=c["state_in"], state_out=so)
        close(y, want, TOL[dtype], "y of single tokens")
        close(so, state, FLOAT, "state of single tokens")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("lengths, first, behind", [((*(30 * (3, 0, 17)), 900, *(20 * (5,))), 0, 0), ((520, *(60 * (1,)), 700, 0, 40), 77, 300), ((*(50 * (0,)), 1100, 16, *(40 * (0,))), 3, 0),
                                                    ((130, 257, 128, 129, 400, 127, 600, 1, 255, 256), 0, 1)])
@pytest.mark.parametrize("D, N, G", [(40, 16, 1), (10, 5, 5), (33, 24, 1)])
def test_many_short_sequences_and_a_long_one(D, N, G, lengths, first, behind, saved, dtype):
    """Cut for the long one: what segments leave is numbered by rows."""
    offsets = packed_offsets(lengths, first)
    check(offsets, D, N, G, dtype, packed=True, rows=offsets[-1] + behind, seed=len(lengths) + D, saved=saved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D, N, G", [(8, 16, 1), (96, 8, 3), (1000, 16, 1), (33, 64, 1), (70, 24, 70)])
def test_calls_take_the_workspace_that_the_query_names(D, N, G, dtype):
    """Each call with as many bytes as the query says, and nothing written behind them; and with those of the largest of the calls."""
    dense = [[i * L for i in range(B + 1)] for B, L in ((1, 1), (1, 300), (3, 600), (7, 130), (1, 2100), (40, 257))]
    packed = [packed_offsets(lengths, first) for lengths, first in (((600, 0, 300, 5), 7), (90 * (3,) + (900,), 0), (20 * (0, 1), 4), ((256, 129) * 9, 0))]
    ops = (cb.CAWN_SCAN_FWD, cb.CAWN_SCAN_BWD, cb.CAWN_SCAN_BWD_RECOMPUTE, cb.CAWN_SCAN_CHECKPOINTS)
    guard, pattern = 4096, 0x5A

    def call(offsets, is_packed, sizes):
        """y, states and gradients (with and without checkpoints) of a call with workspaces of these sizes."""
        rows = offsets[-1]
        _, c = case(offsets, D, N, G, dtype, seed=rows)
        prm = params(offsets, D, N, G, dtype, is_packed, rows)
        off = torch.tensor(offsets, device="cuda") if is_packed else None
        spaces = [torch.full((n + guard,), pattern, dtype=torch.uint8, device="cuda") for n in sizes(prm)]
        wf, wb, wr, marks = (w[:w.numel() - guard] for w in spaces)
        for w in (wf, wb, wr, marks):
            w.fill_(0xFF)
        y, so = torch.full_like(c["grad_y"], 7), torch.empty_like(c["state_in"])
        same = {n: c[n] for n in ("skip", "dt_bias", "z", "state_in")}
        cb.cawn_selective_scan_fwd(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y, wf, state_out=so, offsets=off, checkpoints=marks, **same)
        saved, again = backward(prm, c, off, checkpoints=marks, workspace=wb), backward(prm, c, off, workspace=wr)
        assert all((w[-guard:] == pattern).all() for w in spaces)
        return [y, so, *saved.values(), *again.values()]

    for calls, is_packed in ((dense, False), (packed, True)):
        of = lambda p: [cb.cawn_selective_scan_workspace_bytes(p, op) for op in ops]
        biggest = cb.make_scan_params(max(len(o) - 1 for o in calls), max(b - a for o in calls for a, b in zip(o, o[1:])), D, N, G, flags=flags_of(dtype),
                                      rows=max(o[-1] for o in calls) if is_packed else 0)
        for offsets in calls:
            got, want = call(offsets, is_packed, of), call(offsets, is_packed, lambda p: of(biggest))
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("absent, pad, softplus", [(("z",), 0, True), (("state_in",), 8, True), (("skip", "dt_bias"), 3, True), (("z", "skip", "dt_bias", "state_in"), 8, True),
                                                   ((), 3, False), (("z", "state_in"), 0, False)])
def test_segments_of_slices_and_without_arrays(absent, pad, softplus, saved, dtype):
    check([0, 690, 1380], 40, 16, 2, dtype, pad=pad, absent=absent, softplus=softplus, saved=saved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("absent", [(), ("z", "state_in")])
def test_segments_of_longer_sequences_than_said(absent, dtype):
    """Cut by the L of the params: the rows behind are neither read nor written."""
    check([3, 903, 1203, 1203, 1960], 24, 16, 1, dtype, packed=True, L=600, rows=1965, absent=absent, pad=8)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("absent", [(), ("z",), ("state_in",), ("z", "skip", "dt_bias", "state_in")])
@pytest.mark.parametrize("B, D, N, G, L", [(70, 300, 16, 2, 4), (61, 1100, 5, 2, 3), (40, 512, 24, 4, 2), (33, 5000, 2, 5, 2), (66, 130, 64, 2, 4)])
def test_tokens_of_a_batch_in_groups(B, D, N, G, L, absent, dtype):
    """A thread takes four sequences, several tokens of each, with groups and without what may be absent."""
    offsets = [i * L for i in range(B + 1)]
    d, c = case(offsets, D, N, G, dtype, seed=B + L, pad=8)
    w = {n: t.double() for n, t in d.items()}
    a = [None if n in absent and n != "state_in" else w[n] for n in LEAVES[:-1]]
    want, want_state = selective_scan(*a, torch.zeros_like(w["state_in"]) if "state_in" in absent else w["state_in"], offsets, L)
    y, state = torch.empty(B * L, D, dtype=dtype, device="cuda"), torch.full_like(c["state_in"], float("nan"))
    opt = {n: None if n in absent else c[n] for n in ("skip", "dt_bias", "z", "state_in")}
    prm = cb.make_scan_params(B, L, D, N, G, True, flags_of(dtype), *(c[n].stride(0) for n in ("x", "dt", "z", "B", "C")))
    cb.cawn_selective_scan_step(prm, c["x"], c["dt"], c["A"], c["B"], c["C"], y, state_out=state, **opt)
    close(y, want, TOL[dtype], "y")
    close(state, want_state, FLOAT, "state")
