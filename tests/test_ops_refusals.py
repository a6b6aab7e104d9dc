"""What the operators next to the scan refuse, on the host and before anything is launched (the
addresses are fake and never dereferenced)."""
import ctypes

import pytest

import __graft_entry__ as entry
from paper_2604_04250_b200 import binding as cb

A = 0x10000
N = ctypes.c_size_t()
ref = ctypes.byref


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def test_struct_layouts():
    assert ctypes.sizeof(cb.cawn_delta_params) == 72 and cb.cawn_delta_params.q_stride.offset == 40
    assert ctypes.sizeof(cb.cawn_norm_params) == 56 and cb.cawn_norm_params.x_stride.offset == 40
    assert ctypes.sizeof(cb.cawn_dropout_params) == 40 and cb.cawn_dropout_params.seed.offset == 16


def fwd(prm, q=A, ws=A, n=1 << 40, **kw):
    a = dict(k=A, v=A, g=A, beta=A, state_in=None, o=A, state_out=None)
    a.update(kw)
    return cb.lib().cawn_delta_rule_fwd(None if prm is None else ref(prm), q, a["k"], a["v"], a["g"], a["beta"], a["state_in"], a["o"], a["state_out"], ws, n, None)


def step(prm, q=A, **kw):
    a = dict(k=A, v=A, g=A, beta=A, state_in=None, o=A, state_out=None)
    a.update(kw)
    return cb.lib().cawn_delta_rule_step(None if prm is None else ref(prm), q, a["k"], a["v"], a["g"], a["beta"], a["state_in"], a["o"], a["state_out"], None)


def bwd(prm, ws=A, n=1 << 40, **kw):
    names = ["q", "k", "v", "g", "beta", "state_in", "grad_o", "grad_state_out", "grad_q", "grad_k", "grad_v", "grad_g", "grad_beta", "grad_state_in"]
    return cb.lib().cawn_delta_rule_bwd(None if prm is None else ref(prm), *[kw.get(x, None if "state" in x else A) for x in names], ws, n, None)


def delta(B=2, L=200, Hk=2, Hv=4, Dk=64, Dv=64, **kw):
    return cb.make_delta_params(B, L, Hk, Hv, Dk, Dv, **kw)


INVALID = [dict(B=0), dict(L=-1), dict(Hk=0), dict(Hv=3), dict(Hv=0), dict(Dk=0), dict(flags=cb.CAWN_FLAG_INPUT_BF16), dict(flags=1 << 9),
           dict(q_stride=64), dict(v_stride=300), dict(o_stride=255), dict(k_stride=132), dict(q_stride=-128)]
UNSUPPORTED = [dict(Dk=60), dict(Dv=136), dict(Dk=256), dict(Dv=4), dict(B=1 << 22, Hv=4), dict(L=1 << 60)]


@pytest.mark.parametrize("call", [fwd, step, bwd])
def test_delta_rule_refusals(call):
    assert call(None) == cb.CAWN_ERR_NULL_POINTER
    bad = delta()
    bad.struct_size = 64
    assert call(bad) == cb.CAWN_ERR_INVALID_ARG
    for kw in INVALID:
        assert call(delta(**kw)) == cb.CAWN_ERR_INVALID_ARG, kw
    for kw in UNSUPPORTED:
        assert call(delta(**kw)) == cb.CAWN_ERR_UNSUPPORTED, kw
    for name in ("q", "k", "v", "g", "beta"):
        assert call(delta(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER, name
        assert call(delta(), **{name: A + 8}) == cb.CAWN_ERR_MISALIGNED, name


def test_delta_rule_workspace():
    size = lambda prm, op: cb.cawn_delta_rule_workspace_bytes(prm, op)
    for op in (cb.CAWN_DELTA_FWD, cb.CAWN_DELTA_BWD):
        assert size(delta(L=0), op) >= 0
        assert size(delta(L=300), op) <= size(delta(L=3000), op)
        assert size(delta(L=3000), op) > 0
    lib = cb.lib()
    assert lib.cawn_delta_rule_workspace_bytes(ref(delta()), 2, ref(N)) == cb.CAWN_ERR_INVALID_ARG
    assert lib.cawn_delta_rule_workspace_bytes(ref(delta()), 0, None) == cb.CAWN_ERR_NULL_POINTER
    assert lib.cawn_delta_rule_workspace_bytes(ref(delta(Dk=60)), 0, ref(N)) == cb.CAWN_ERR_UNSUPPORTED
    long = delta(L=4000)
    assert fwd(long, n=256) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL
    assert fwd(long, ws=None) == cb.CAWN_ERR_NULL_POINTER
    assert fwd(long, ws=A + 4) == cb.CAWN_ERR_MISALIGNED
    assert bwd(long, n=256) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL
    assert bwd(long, ws=None) == cb.CAWN_ERR_NULL_POINTER


@pytest.mark.parametrize("op", [cb.CAWN_DELTA_FWD, cb.CAWN_DELTA_BWD])
@pytest.mark.parametrize("flags", [0, cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16])
@pytest.mark.parametrize("Hk, Hv, Dk, Dv", [(12, 12, 64, 64), (1, 1, 128, 128), (2, 6, 128, 64), (1, 3, 40, 72), (4, 8, 64, 96)])
def test_delta_rule_workspace_of_the_largest_call_serves_all(Hk, Hv, Dk, Dv, flags, op):
    """The size never falls as the call grows, in length or in batch."""
    lengths, batches = [*range(0, 4100, 41), *range(4100, 40000, 1013)], [1, 2, 3, 4, 5, 8, 12, 13, 25, 40, 96]
    sizes = [[cb.cawn_delta_rule_workspace_bytes(cb.make_delta_params(B, L, Hk, Hv, Dk, Dv, flags=flags), op) for L in lengths] for B in batches]
    for row in sizes:
        assert all(a <= b for a, b in zip(row, row[1:]))
    for one, more in zip(sizes, sizes[1:]):
        assert all(a <= b for a, b in zip(one, more))
    assert all(row[0] == 0 for row in sizes)                # no tokens, nothing kept


def test_delta_rule_rows_of_tensors():
    """Strides against the tensors they are said of: a batch step that is not L rows is refused, and one token's row
    stride, which torch leaves open, is the batch step."""
    import torch
    for L in (1, 5):
        w = torch.zeros(2, L, 3 * 64)
        q, k, v = (x.unflatten(-1, (1, 64)) for x in w.split(64, -1))
        prm = cb.make_delta_params(2, L, 1, 1, 64, 64, q_stride=q.stride(1), k_stride=192, v_stride=v.stride(1))
        got = cb._delta_rows(prm, q, k, v, torch.zeros(2, L, 1, 64))
        assert (got.q_stride, got.k_stride, got.v_stride, got.o_stride) == (192, 192, 192, 0)
        assert prm.q_stride == q.stride(1)              # the caller's own are left alone
    dense = cb.make_delta_params(2, 5, 1, 1, 64, 64)
    with pytest.raises(ValueError, match="v_stride"):
        cb._delta_rows(dense, torch.zeros(2, 5, 1, 64), torch.zeros(2, 5, 1, 64), v, torch.zeros(2, 5, 1, 64))
    with pytest.raises(ValueError, match="q_stride"):   # the first five tokens of a longer buffer
        cb._delta_rows(dense, torch.zeros(2, 9, 1, 64)[:, :5], k, v, None)


@pytest.mark.parametrize("which", range(4))
def test_delta_rule_one_token_expanded_over_the_batch(which):
    """Its batch step is 0, which the C call would take as dense and read (or write) past the one row there is."""
    import torch
    x = [torch.zeros(4, 1, 1, 64) for _ in range(4)]
    cb._delta_rows(cb.make_delta_params(4, 1, 1, 1, 64, 64), *x)
    x[which] = torch.zeros(1, 1, 1, 64).expand(4, 1, 1, 64)
    with pytest.raises(ValueError, match="qkvo"[which] + "_stride"):
        cb._delta_rows(cb.make_delta_params(4, 1, 1, 1, 64, 64), *x)


def test_delta_rule_layouts():
    """Whatever the batch, rows that are not as the params say and arrays that are not dense are refused."""
    import torch
    B, L, H, D = 2, 5, 3, 64
    dense = lambda B=B: torch.zeros(B, L, H, D)
    make = lambda B=B, **kw: cb.make_delta_params(B, L, H, H, D, D, **kw)
    heads_first = torch.zeros(B, H, L, D).transpose(1, 2)                   # its batch step is that of L rows
    projection = torch.zeros(1, L, 3 * H * D)
    part = projection.split(H * D, -1)[1].unflatten(-1, (H, D))
    wide = projection.shape[-1]
    for i, name in enumerate(("q_stride", "k_stride", "v_stride", "o_stride")):
        def rows(x, params, B=B):
            t = [dense(B) for _ in range(4)]
            t[i] = x
            return cb._delta_rows(params, *t)
        rows(dense(), make())
        rows(dense().flatten(2), make())
        rows(dense().flatten(0, 1), make())
        rows(dense().flatten(), make())
        rows(part, make(1, **{name: wide}), 1)
        rows(part.flatten(2), make(1, **{name: wide}), 1)
        rows(part.flatten(0, 1), make(1, **{name: wide}), 1)
        for x, params, b in ((heads_first, make(), B), (heads_first[:1], make(1), 1), (part, make(1), 1), (part[0], make(1), 1),
                             (dense(1), make(1, **{name: wide}), 1), (dense(1).flatten(), make(1, **{name: wide}), 1),
                             (dense().transpose(2, 3).contiguous().transpose(2, 3), make(), B), (dense()[..., ::2].repeat_interleave(2, 3).mT, make(), B),
                             (torch.zeros(B, 1, H, D).expand(B, L, H, D), make(), B)):
            with pytest.raises(ValueError, match=name):
                rows(x, params, b)
    halves = torch.zeros(B, L, 2 * H).chunk(2, -1)[0]                        # as a projection to decays and betas leaves them
    # every array of every call is looked at, before anything else
    calls = {cb.cawn_delta_rule_fwd: ("g", "beta", "state_in", "state_out"), cb.cawn_delta_rule_step: ("g", "beta", "state_in", "state_out"),
             cb.cawn_delta_rule_bwd: ("g", "beta", "state_in", "grad_state_out", "grad_q", "grad_k", "grad_v", "grad_g", "grad_beta", "grad_state_in")}
    import inspect
    for call, names in calls.items():
        for name in names:
            kw = {n: dense() for n, p in inspect.signature(call).parameters.items() if p.default is p.empty}
            kw.update(params=make(), **{name: halves})
            with pytest.raises(ValueError, match=name):
                call(**kw)


def test_norm_and_dropout_layouts():
    import torch
    N, C = 6, 128
    x, wide = torch.zeros(N, C), torch.zeros(N, 3 * C)[:, C:2 * C]
    prm, strided = cb.make_norm_params(N, 2, 64), cb.make_norm_params(N, 2, 64, x_stride=3 * C, gate_stride=3 * C)
    cb._norm_rows(prm, x, x)
    cb._norm_rows(prm, x.view(2, 3, 2, 64), None)
    cb._norm_rows(strided, wide, wide.unflatten(0, (2, 3)))
    for p, a, g, name in ((prm, wide, None, "x_stride"), (prm, x, wide, "gate_stride"), (strided, x, wide, "x_stride"), (strided, wide, x, "gate_stride"),
                          (prm, torch.zeros(C, N).T, None, "x_stride")):
        with pytest.raises(ValueError, match=name):
            cb._norm_rows(p, a, g)
    for name in ("y", "weight", "bias"):
        with pytest.raises(ValueError, match=name):
            cb.cawn_group_norm_fwd(prm, x, **{"y": x, name: wide})
    for name in ("grad_y", "grad_x", "grad_gate", "grad_weight", "grad_bias", "weight", "bias"):
        with pytest.raises(ValueError, match=name):
            cb.cawn_group_norm_bwd(prm, x, **{"grad_y": x, "grad_x": x, name: wide})
    for name in ("x", "y", "residual"):
        with pytest.raises(ValueError, match=name):
            cb.cawn_dropout(cb.make_dropout_params(N * C, 0.1, 0), **{"x": x, "y": x, name: wide})


def test_delta_rule_backward_pointers():
    for name in ("grad_o", "grad_q", "grad_k", "grad_v", "grad_g", "grad_beta"):
        assert bwd(delta(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER, name
    for name in ("grad_q", "grad_state_out", "grad_state_in", "state_in"):
        assert bwd(delta(), **{name: A + 2}) == cb.CAWN_ERR_MISALIGNED, name


def norm(prm, x=A, gate=None, y=A, w=None):
    return cb.lib().cawn_group_norm_fwd(None if prm is None else ref(prm), x, w, None, gate, y, None)


def norm_bwd(prm, x=A, gate=None, gy=A, gx=A, gg=None, gw=None, ws=None, n=0):
    return cb.lib().cawn_group_norm_bwd(ref(prm), x, None, None, gate, gy, gx, gg, gw, None, ws, n, None)


def test_group_norm_refusals():
    make = cb.make_norm_params
    assert norm(None) == cb.CAWN_ERR_NULL_POINTER
    for prm in (make(-1, 1, 8), make(1, 0, 8), make(1, 1, 0), make(1, 1, 8, eps=-1.0), make(1, 1, 8, eps=float("nan")), make(1, 1, 8, act=3),
                make(1, 1, 8, flags=cb.CAWN_FLAG_OUTPUT_BF16), make(1, 2, 8, x_stride=15), make(1, 2, 8, gate_stride=3)):
        assert norm(prm) == cb.CAWN_ERR_INVALID_ARG
        assert norm_bwd(prm) == cb.CAWN_ERR_INVALID_ARG
    for prm in (make(1, 1, 4097), make(1 << 40, 1, 8), make(1, 65536, 8)):
        assert norm(prm) == cb.CAWN_ERR_UNSUPPORTED
    ok, gated = make(4, 2, 8), make(4, 2, 8, act=cb.CAWN_NORM_ACT_GATE)
    assert norm(ok, x=None) == cb.CAWN_ERR_NULL_POINTER and norm(ok, y=None) == cb.CAWN_ERR_NULL_POINTER
    assert norm(gated) == cb.CAWN_ERR_NULL_POINTER
    assert norm(ok, x=A + 4) == cb.CAWN_ERR_MISALIGNED and norm(ok, w=A + 4) == cb.CAWN_ERR_MISALIGNED
    assert norm_bwd(gated, gate=A) == cb.CAWN_ERR_NULL_POINTER
    assert norm_bwd(ok, gg=A) == cb.CAWN_ERR_INVALID_ARG
    assert norm_bwd(ok, gw=A) == cb.CAWN_ERR_NULL_POINTER
    assert norm_bwd(ok, gw=A, ws=A, n=16) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL
    bad = make(4, 2, 8)
    bad.struct_size = 1
    assert norm(bad) == cb.CAWN_ERR_INVALID_ARG
    assert cb.lib().cawn_group_norm_workspace_bytes(ref(ok), None) == cb.CAWN_ERR_NULL_POINTER


@pytest.mark.parametrize("flags", [0, cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16])
@pytest.mark.parametrize("G, M", [(12, 64), (1, 768), (3, 37), (8, 1024), (40, 16), (2, 4096), (5, 2000)])
def test_group_norm_workspace_of_the_largest_call_serves_all(G, M, flags):
    """The size never falls as the call grows, and is what a call of its own takes."""
    sizes = [cb.cawn_group_norm_workspace_bytes(cb.make_norm_params(N, G, M, flags=flags)) for N in [*range(3000), *range(3000, 200000, 997)]]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_dropout_refusals():
    make = cb.make_dropout_params
    f = lambda prm, x=A, r=None, y=A, d=None: cb.lib().cawn_dropout(None if prm is None else ref(prm), x, r, y, d, None)
    assert f(None) == cb.CAWN_ERR_NULL_POINTER
    for prm in (make(-1, 0.1, 0), make(8, 1.0, 0), make(8, -0.1, 0), make(8, float("nan"), 0), make(8, 0.1, 0, flags=cb.CAWN_FLAG_INPUT_BF16)):
        assert f(prm) == cb.CAWN_ERR_INVALID_ARG
    ok = make(8, 0.1, 0)
    assert f(ok, x=None) == cb.CAWN_ERR_NULL_POINTER and f(ok, y=None) == cb.CAWN_ERR_NULL_POINTER
    assert f(ok, r=A + 2) == cb.CAWN_ERR_MISALIGNED and f(ok, d=A + 4) == cb.CAWN_ERR_MISALIGNED
    assert f(make(1 << 50, 0.1, 0)) == cb.CAWN_ERR_UNSUPPORTED
    assert f(make(0, 0.1, 0), x=None) == cb.CAWN_OK


def test_the_tests_generator_gives_the_published_answers():
    from delta_ref import PHILOX_ANSWERS, philox_bits, philox_words
    for counter, key, answer in PHILOX_ANSWERS:
        assert tuple(philox_words(counter, key)) == answer
    counter, key, answer = PHILOX_ANSWERS[0]
    assert philox_bits(8, 0, 0).tolist() == [half for w in answer for half in (w & 0xFFFF, w >> 16)]
