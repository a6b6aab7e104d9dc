"""What the operators of a selective state space layer refuse, on the host and before anything is launched (the addresses are
fake and never dereferenced), and what their workspaces ask for."""
import ctypes
import inspect

import pytest
import torch

import __graft_entry__ as entry
from paper_2604_04250_b200 import binding as cb

A = 0x10000
BF16 = cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16
N = ctypes.c_size_t()
ref = ctypes.byref


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def call(name, names, prm, optional=(), ws=A, n=1 << 50, workspace=True, **kw):
    """The entry point with fake addresses for `names`, None for the optional ones."""
    args = [kw.get(x, None if x in optional else A) for x in names.split()]
    return getattr(cb.lib(), name)(None if prm is None else ref(prm), *args, *((ws, n) if workspace else ()), None)


def conv_fwd(prm, **kw):
    return call("cawn_short_conv_fwd", "x weight bias state_in offsets y state_out", prm, ("bias", "state_in", "offsets", "state_out"), workspace=False, **kw)


def conv_bwd(prm, **kw):
    return call("cawn_short_conv_bwd", "x weight bias state_in offsets grad_y grad_state_out grad_x grad_weight grad_bias grad_state_in", prm,
                ("bias", "state_in", "offsets", "grad_state_out", "grad_bias", "grad_state_in"), **kw)


def scan_fwd(prm, **kw):
    return call("cawn_selective_scan_fwd", "x dt A B C skip dt_bias z state_in offsets y state_out checkpoints", prm,
                ("skip", "dt_bias", "z", "state_in", "offsets", "state_out", "checkpoints"), **kw)


def scan_step(prm, **kw):
    return call("cawn_selective_scan_step", "x dt A B C skip dt_bias z state_in y state_out", prm, ("skip", "dt_bias", "z", "state_in", "state_out"),
                workspace=False, **kw)


def scan_bwd(prm, **kw):
    return call("cawn_selective_scan_bwd", "x dt A B C skip dt_bias z state_in offsets checkpoints grad_y grad_state_out grad_x grad_dt grad_A grad_B grad_C "
                "grad_skip grad_dt_bias grad_z grad_state_in", prm, ("skip", "dt_bias", "z", "state_in", "offsets", "checkpoints", "grad_state_out",
                                                                     "grad_skip", "grad_dt_bias", "grad_z", "grad_state_in"), **kw)


def norm_fwd(prm, **kw):
    return call("cawn_residual_norm_fwd", "x residual weight sum_out y scales", prm, ("residual", "weight", "sum_out", "scales"), workspace=False, **kw)


def norm_bwd(prm, **kw):
    return call("cawn_residual_norm_bwd", "sum weight grad_y grad_sum grad_residual grad_x grad_weight", prm, ("weight", "grad_sum", "grad_x"), **kw)


def conv(B=2, L=200, C=64, K=4, **kw):
    return cb.make_conv_params(B, L, C, K, **kw)


def scan(B=2, L=200, D=64, N=16, G=1, **kw):
    return cb.make_scan_params(B, L, D, N, G, **kw)


def norm(N=20, M=64, **kw):
    return cb.make_residual_norm_params(N, M, **kw)


def test_struct_layouts():
    assert ctypes.sizeof(cb.cawn_conv_params) == 56 and cb.cawn_conv_params.x_stride.offset == 40
    assert ctypes.sizeof(cb.cawn_scan_params) == 88 and cb.cawn_scan_params.x_stride.offset == 40
    assert ctypes.sizeof(cb.cawn_residual_norm_params) == 48 and cb.cawn_residual_norm_params.x_stride.offset == 40


@pytest.mark.parametrize("entry_point, make", [(conv_fwd, conv), (conv_bwd, conv), (scan_fwd, scan), (scan_step, scan), (scan_bwd, scan), (norm_fwd, norm), (norm_bwd, norm)])
def test_params(entry_point, make):
    assert entry_point(None) == cb.CAWN_ERR_NULL_POINTER
    bad = make()
    bad.struct_size = 12
    assert entry_point(bad) == cb.CAWN_ERR_INVALID_ARG
    for kw in ([dict(B=0), dict(L=-1), dict(rows=-1), dict(rows=77)] if make is not norm else [dict(N=-1), dict(M=0)]) + [dict(flags=1 << 9), dict(flags=cb.CAWN_FLAG_INPUT_BF16),
                                                                                                                         dict(x_stride=63), dict(x_stride=-64)]:
        assert entry_point(make(**kw)) == cb.CAWN_ERR_INVALID_ARG, kw
    bad = make()
    if make is conv:
        bad.reserved[1] = 1
    else:
        bad.reserved = 1
    assert entry_point(bad) == cb.CAWN_ERR_INVALID_ARG


@pytest.mark.parametrize("entry_point", [conv_fwd, conv_bwd])
def test_conv(entry_point):
    for kw in (dict(C=0), dict(K=0), dict(act=2)):
        assert entry_point(conv(**kw)) == cb.CAWN_ERR_INVALID_ARG, kw
    for kw in (dict(K=5), dict(C=1 << 23), dict(B=1 << 30, L=100), dict(L=1 << 60)):
        assert entry_point(conv(**kw)) == cb.CAWN_ERR_UNSUPPORTED, kw
    assert entry_point(conv(), offsets=A) == cb.CAWN_ERR_INVALID_ARG              # packed, and how many rows is not said
    assert entry_point(conv(rows=300), offsets=A + 4) == cb.CAWN_ERR_MISALIGNED
    for name in ("x", "weight"):
        assert entry_point(conv(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER, name
    for name in ("weight", "bias", "state_in"):
        assert entry_point(conv(), **{name: A + 8}) == cb.CAWN_ERR_MISALIGNED, name
    assert entry_point(conv(), x=A + 2) == cb.CAWN_ERR_MISALIGNED and entry_point(conv(flags=BF16), x=A + 1) == cb.CAWN_ERR_MISALIGNED


def test_conv_pointers_of_one_direction():
    assert conv_fwd(conv(), y=None) == cb.CAWN_ERR_NULL_POINTER and conv_fwd(conv(), state_out=A + 4) == cb.CAWN_ERR_MISALIGNED
    for name in ("grad_y", "grad_x"):
        assert conv_bwd(conv(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER, name
    for name in ("grad_y", "grad_x", "grad_weight", "grad_bias", "grad_state_out", "grad_state_in"):
        assert conv_bwd(conv(), **{name: A + 4}) == cb.CAWN_ERR_MISALIGNED, name
    assert conv_bwd(conv(), ws=None) == cb.CAWN_ERR_NULL_POINTER and conv_bwd(conv(), ws=A + 8) == cb.CAWN_ERR_MISALIGNED
    assert conv_bwd(conv(), n=64) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("entry_point", [scan_fwd, scan_step, scan_bwd])
def test_scan(entry_point):
    for kw in (dict(D=0), dict(N=0), dict(G=0), dict(G=3), dict(softplus=2), dict(dt_stride=63), dict(z_stride=5), dict(b_stride=15), dict(c_stride=-16), dict(G=2, c_stride=31)):
        assert entry_point(scan(**kw)) == cb.CAWN_ERR_INVALID_ARG, kw
    for kw in (dict(N=65), dict(D=1 << 23), dict(B=1 << 30), dict(L=1 << 60), dict(B=1 << 20, L=1 << 20), dict(D=1 << 20, G=1 << 20)):
        assert entry_point(scan(**kw)) == cb.CAWN_ERR_UNSUPPORTED, kw
    for name in ("x", "dt", "A", "B", "C"):
        assert entry_point(scan(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER, name
    for name in ("A", "skip", "dt_bias", "state_in"):
        assert entry_point(scan(), **{name: A + 8}) == cb.CAWN_ERR_MISALIGNED, name
    for name in ("x", "dt", "z", "B", "C"):         # aligned to their elements is enough
        more = {"grad_z": A} if name == "z" and entry_point is scan_bwd else {}
        assert entry_point(scan(), **{name: A + 2, **more}) == cb.CAWN_ERR_MISALIGNED, name
        assert entry_point(scan(flags=BF16), **{name: A + 1, **more}) == cb.CAWN_ERR_MISALIGNED, name
    if entry_point is not scan_step:
        assert entry_point(scan(), offsets=A) == cb.CAWN_ERR_INVALID_ARG
        assert entry_point(scan(rows=300), offsets=A + 4) == cb.CAWN_ERR_MISALIGNED


def test_scan_pointers_of_one_direction():
    long = scan(B=1, L=5000)                            # few channels: segments, which need a workspace
    assert scan_fwd(scan(), y=None) == cb.CAWN_ERR_NULL_POINTER and scan_step(scan(), y=None) == cb.CAWN_ERR_NULL_POINTER
    for name in ("y", "state_out", "checkpoints"):
        assert scan_fwd(scan(), **{name: A + 4}) == cb.CAWN_ERR_MISALIGNED, name
    assert scan_fwd(long, ws=None) == cb.CAWN_ERR_NULL_POINTER and scan_fwd(long, n=256) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL
    assert scan_fwd(long, ws=A + 8) == cb.CAWN_ERR_MISALIGNED
    for name in ("grad_y", "grad_x", "grad_dt", "grad_A", "grad_B", "grad_C"):
        assert scan_bwd(scan(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER, name
        assert scan_bwd(scan(), **{name: A + 4}) == cb.CAWN_ERR_MISALIGNED, name
    for name in ("grad_skip", "grad_dt_bias", "grad_state_in", "grad_state_out", "checkpoints"):
        assert scan_bwd(scan(), **{name: A + 4}) == cb.CAWN_ERR_MISALIGNED, name
    assert scan_bwd(scan(), z=A) == cb.CAWN_ERR_NULL_POINTER and scan_bwd(scan(), grad_z=A) == cb.CAWN_ERR_INVALID_ARG
    assert scan_bwd(scan(), ws=None) == cb.CAWN_ERR_NULL_POINTER and scan_bwd(scan(), n=256) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL
    need = cb.cawn_selective_scan_workspace_bytes(long, cb.CAWN_SCAN_BWD)
    assert need < cb.cawn_selective_scan_workspace_bytes(long, cb.CAWN_SCAN_BWD_RECOMPUTE)
    assert scan_bwd(long, n=need - 256 * 1024) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL
    lib = cb.lib()
    assert lib.cawn_selective_scan_workspace_bytes(ref(scan()), 4, ref(N)) == cb.CAWN_ERR_INVALID_ARG
    assert lib.cawn_selective_scan_workspace_bytes(ref(scan()), 0, None) == cb.CAWN_ERR_NULL_POINTER
    assert lib.cawn_selective_scan_workspace_bytes(ref(scan(N=65)), 0, ref(N)) == cb.CAWN_ERR_UNSUPPORTED


def test_residual_norm():
    for p in (norm(eps=-1.0), norm(eps=float("nan")), norm(out=2), norm(scale_block=32), norm(out=1, scale_block=48), norm(out=1, scale_block=256)):
        assert norm_fwd(p, scales=A if p.out == 1 else None) == cb.CAWN_ERR_INVALID_ARG
    bad = norm()
    bad.stream_float = 2
    assert norm_fwd(bad) == cb.CAWN_ERR_INVALID_ARG
    for p in (norm(M=8193), norm(N=1 << 31), norm(N=1 << 30, x_stride=1 << 40)):
        assert norm_fwd(p) == cb.CAWN_ERR_UNSUPPORTED
    assert norm_fwd(norm(), scales=A) == cb.CAWN_ERR_INVALID_ARG and norm_fwd(norm(out=1)) == cb.CAWN_ERR_NULL_POINTER
    for name in ("x", "y"):
        assert norm_fwd(norm(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER
    for name in ("y", "residual", "weight", "sum_out"):
        assert norm_fwd(norm(), **{name: A + 4}) == cb.CAWN_ERR_MISALIGNED, name
    assert norm_fwd(norm(), x=A + 2) == cb.CAWN_ERR_MISALIGNED
    assert norm_fwd(norm(out=1), scales=A + 4) == cb.CAWN_ERR_MISALIGNED
    for name in ("sum", "grad_y"):
        assert norm_bwd(norm(), **{name: None}) == cb.CAWN_ERR_NULL_POINTER
    assert norm_bwd(norm(), grad_residual=None) == cb.CAWN_ERR_NULL_POINTER
    for name in ("sum", "grad_y", "weight", "grad_sum", "grad_residual", "grad_x", "grad_weight"):
        assert norm_bwd(norm(), **{name: A + 4}) == cb.CAWN_ERR_MISALIGNED, name
    assert norm_bwd(norm(), ws=None) == cb.CAWN_ERR_NULL_POINTER and norm_bwd(norm(), n=16) == cb.CAWN_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("flags", [0, BF16])
def test_a_workspace_of_the_largest_call_serves_all(flags):
    """The sizes never fall as a call grows, in length, batch or rows."""
    lengths, batches = [*range(0, 4100, 41), *range(4100, 40000, 1013)], [1, 2, 3, 4, 5, 8, 12, 13, 25, 40, 96]

    def grows(size):
        table = [[size(B, L) for L in lengths] for B in batches]
        for row in table:
            assert all(a <= b for a, b in zip(row, row[1:]))
        for one, more in zip(table, table[1:]):
            assert all(a <= b for a, b in zip(one, more))

    for D, n, G in ((8, 16, 1), (768, 16, 1), (2048, 64, 2), (100, 5, 4)):
        for op in range(4):
            grows(lambda B, L: cb.cawn_selective_scan_workspace_bytes(cb.make_scan_params(B, L, D, n, G, flags=flags), op))
            rows = [cb.cawn_selective_scan_workspace_bytes(cb.make_scan_params(3, 500, D, n, G, flags=flags, rows=r), op) for r in range(1, 3000, 7)]
            assert all(a <= b for a, b in zip(rows, rows[1:]))
    for C in (8, 768, 5000):
        grows(lambda B, L: cb.cawn_short_conv_workspace_bytes(cb.make_conv_params(B, L, C, 4, flags=flags)))
    for M in (8, 768, 5000):
        sizes = [cb.cawn_residual_norm_workspace_bytes(cb.make_residual_norm_params(r, M, flags=flags)) for r in range(0, 5000, 13)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_a_call_needs_no_more_than_the_query_says():
    """Fake addresses: a call that finds its workspace too small says so before anything else can happen."""
    for B, L in ((1, 300), (1, 5000), (3, 5000), (7, 700), (40, 5000)):
        for D, n in ((8, 16), (768, 16), (100, 5)):
            p = scan(B=B, L=L, D=D, N=n)
            assert cb.cawn_selective_scan_workspace_bytes(p, cb.CAWN_SCAN_BWD) >= B * D * (n + 2) * 4


def test_layouts_of_tensors():
    B, L, D, n, G = 2, 5, 48, 8, 2
    dense = {"x": torch.zeros(B, L, D), "dt": torch.zeros(B, L, D), "z": torch.zeros(B, L, D), "B": torch.zeros(B, L, G, n), "C": torch.zeros(B, L, G * n)}
    prm = cb.make_scan_params(B, L, D, n, G)
    cb._scan_rows(prm, None, **dense)
    cb._scan_rows(prm, None, **{k: v.flatten(0, 1) for k, v in dense.items()})
    for name, width, stride in (("x", D, "x_stride"), ("dt", D, "dt_stride"), ("z", D, "z_stride"), ("B", G * n, "b_stride"), ("C", G * n, "c_stride")):
        wide = torch.zeros(B, L, 3 * width)[..., width:2 * width]
        good = cb.make_scan_params(B, L, D, n, G, **{stride: 3 * width})
        cb._scan_rows(good, None, **{**dense, name: wide})
        for p, x in ((prm, wide), (good, dense[name]), (prm, torch.zeros(B, L + 1, width)[:, :L]), (prm, torch.zeros(L, B, width).transpose(0, 1)),
                     (prm, torch.zeros(B, 1, width).expand(B, L, width)), (prm, torch.zeros(B, L + 1, width)), (prm, torch.zeros(B * L * width // 2))):
            with pytest.raises(ValueError, match=stride):
                cb._scan_rows(p, None, **{**dense, name: x})
    packed = cb.make_scan_params(3, 6, D, n, G, rows=B * L)
    cb._scan_rows(packed, torch.tensor([0, 1, 4, 10]), **dense)
    for offsets in (torch.tensor([0, 1, 10]), torch.tensor([0, 1, 4, 10], dtype=torch.int32), torch.zeros(8, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError, match="offsets"):
            cb._scan_rows(packed, offsets, **dense)
    # a single row: torch leaves its step open, but its elements have to be neighbours
    one = cb.make_scan_params(1, 1, D, n, G)
    with pytest.raises(ValueError, match="dt_stride"):
        cb._scan_rows(one, None, torch.zeros(1, D), torch.zeros(1, 2 * D)[:, ::2], None, torch.zeros(1, G * n), torch.zeros(1, G * n))
    with pytest.raises(ValueError, match="checkpoints"):
        cb._scan_checkpoints(prm, torch.zeros(8))


def test_every_dense_array_of_every_call_is_looked_at():
    halves = torch.zeros(4, 96).chunk(2, -1)[0]
    dense = torch.zeros(4, 48)
    calls = {cb.cawn_short_conv_fwd: ("weight", "y", "bias", "state_in", "state_out"),
             cb.cawn_short_conv_bwd: ("weight", "grad_y", "grad_x", "bias", "state_in", "grad_state_out", "grad_weight", "grad_bias", "grad_state_in"),
             cb.cawn_selective_scan_fwd: ("A", "y", "skip", "dt_bias", "state_in", "state_out", "checkpoints"),
             cb.cawn_selective_scan_step: ("A", "y", "skip", "dt_bias", "state_in", "state_out"),
             cb.cawn_selective_scan_bwd: ("A", "grad_y", "grad_x", "grad_dt", "grad_A", "grad_B", "grad_C", "skip", "dt_bias", "state_in", "checkpoints",
                                          "grad_state_out", "grad_skip", "grad_dt_bias", "grad_z", "grad_state_in"),
             cb.cawn_residual_norm_fwd: ("y", "residual", "weight", "sum_out", "scales"),
             cb.cawn_residual_norm_bwd: ("sum", "grad_y", "weight", "grad_sum", "grad_residual", "grad_x", "grad_weight")}
    for f, names in calls.items():
        prm = {"s": cb.make_scan_params(1, 4, 48, 48), "c": cb.make_conv_params(1, 4, 48, 4), "r": cb.make_residual_norm_params(4, 48)}
        prm = prm["s" if "scan" in f.__name__ else "c" if "conv" in f.__name__ else "r"]
        for name in names:
            kw = {k: dense for k, p in inspect.signature(f).parameters.items() if p.default is p.empty}
            kw.update(params=prm, **{name: halves})
            with pytest.raises(ValueError, match=name):
                f(**kw)


@pytest.mark.parametrize("N, fewer", [(5, True), (8, True), (9, True), (16, True), (24, False), (64, False)])
def test_the_backward_is_cut_for_the_blocks_that_are_resident(N, fewer):
    """A block of the walk keeps fetched rows as they are stored, so with up to 16 states fewer blocks of float are resident than of bfloat16
    (4 and 5, with 9 or more states 3 and 4): fewer segments, whose states and sums are the workspace of this call but for parts
    that are float in both."""
    of = lambda flags: cb.cawn_selective_scan_workspace_bytes(scan(B=1, L=8192, D=60, N=N, G=60, flags=flags), cb.CAWN_SCAN_BWD)
    assert (of(0) < of(BF16)) if fewer else (of(0) == of(BF16))


B_, L_, D_, N_, G_, K_ = 2, 3, 48, 8, 2, 4


def arrays_of(f, dtype, wide=False):
    """Arguments of a call with every array it takes, of the sizes and types that its params say."""
    rows, z = B_ * L_, lambda n, t: torch.zeros(n, dtype=t)
    flags = BF16 if dtype == torch.bfloat16 else 0
    if "norm" in f.__name__:
        stream = torch.float32 if wide else dtype
        prm = cb.make_residual_norm_params(rows, D_, flags=flags, stream_float=wide)
        of = {"x": dtype, "y": dtype, "grad_y": dtype, "grad_x": dtype, "residual": stream, "sum_out": stream, "sum": stream, "grad_sum": stream, "grad_residual": stream}
        sizes = {**{n: (rows * D_, t) for n, t in of.items()}, "weight": (D_, torch.float32), "grad_weight": (D_, torch.float32)}
    elif "conv" in f.__name__:
        prm = cb.make_conv_params(B_, L_, D_, K_, flags=flags)
        sizes = {**{n: (rows * D_, dtype) for n in ("x", "y", "grad_y", "grad_x")}, "weight": (D_ * K_, torch.float32), "bias": (D_, torch.float32)}
        sizes.update({"grad_" + n: sizes[n] for n in ("weight", "bias")})
        sizes.update({n: (B_ * (K_ - 1) * D_, torch.float32) for n in ("state_in", "state_out", "grad_state_out", "grad_state_in")})
    else:
        prm = cb.make_scan_params(B_, L_, D_, N_, G_, flags=flags)
        sizes = {**{n: (rows * D_, dtype) for n in ("x", "dt", "z", "y")}, **{n: (rows * G_ * N_, dtype) for n in ("B", "C")}, "A": (D_ * N_, torch.float32),
                 "skip": (D_, torch.float32), "dt_bias": (D_, torch.float32), "state_in": (B_ * D_ * N_, torch.float32)}
        sizes.update({"grad_" + n: s for n, s in sizes.items()})
        sizes.update({n: sizes["state_in"] for n in ("state_out", "grad_state_out")})
    takes = inspect.signature(f).parameters
    return {"params": prm, **{n: z(*s) for n, s in sizes.items() if n in takes}, **({"workspace": torch.zeros(4096, dtype=torch.uint8)} if "workspace" in takes else {})}


@pytest.mark.parametrize("dtype, wide", [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True)])
@pytest.mark.parametrize("f", [cb.cawn_short_conv_fwd, cb.cawn_short_conv_bwd, cb.cawn_selective_scan_fwd, cb.cawn_selective_scan_step, cb.cawn_selective_scan_bwd,
                               cb.cawn_residual_norm_fwd, cb.cawn_residual_norm_bwd])
def test_arrays_that_are_short_or_of_another_type(f, dtype, wide, monkeypatch):
    """Each array one element short, and of each other type: refused before the library is called, which would read or write past it."""
    class Reached(Exception):
        pass

    def lib():
        raise Reached

    good = arrays_of(f, dtype, wide)
    checked = [n for n, t in good.items() if isinstance(t, torch.Tensor) and n != "workspace"]
    assert len(checked) >= 5
    monkeypatch.setattr(cb, "lib", lib)
    with pytest.raises(Reached):
        f(**good)
    for n in checked:
        t = good[n]
        for bad in (t[:-1], *(t.to(k) for k in (torch.float32, torch.bfloat16, torch.float16, torch.float64) if k != t.dtype)):
            with pytest.raises(ValueError, match="(?i)^" + n):         # B's rows go by the name of their stride
                f(**{**good, n: bad})


def test_scales_and_8_bit_rows(monkeypatch):
    def lib():
        raise KeyError
    monkeypatch.setattr(cb, "lib", lib)
    x, rows = torch.zeros(6, 200), torch.zeros(6, 200, dtype=torch.uint8)
    for block, cols in ((0, 1), (32, 7), (64, 4), (128, 2)):
        prm = norm(N=6, M=200, out=cb.CAWN_NORM_OUT_E4M3, scale_block=block)
        for y in (rows, rows.view(torch.float8_e4m3fn)):
            with pytest.raises(KeyError):
                cb.cawn_residual_norm_fwd(prm, x, y, scales=torch.zeros(6, cols))
        for y, scales, name in ((rows, torch.zeros(6 * cols - 1), "scales"), (rows, torch.zeros(6, cols, dtype=torch.float64), "scales"), (rows[:5], torch.zeros(6, cols), "y"),
                                (x, torch.zeros(6, cols), "y"), (x.bfloat16(), torch.zeros(6, cols), "y")):
            with pytest.raises(ValueError, match=name):
                cb.cawn_residual_norm_fwd(prm, x, y, scales=scales)
    with pytest.raises(ValueError, match="x"):          # a slice of rows, one of them missing
        cb.cawn_residual_norm_fwd(norm(N=6, M=200, x_stride=400), torch.zeros(5, 400)[:, :200], x)


@pytest.mark.parametrize("B, rows, L, D, N", [(256, 65536, 2048, 2048, 16), (1000, 30000, 4000, 512, 8), (64, 100000, 20000, 64, 24)])
def test_packed_workspaces_are_counted_by_their_rows(B, rows, L, D, N):
    """Many sequences shorter than the longest: what the dense call of as many rows in sequences of L takes, and for each sequence a state (forward)
    or a row of parameters' gradients (backward) more."""
    packed, dense = cb.make_scan_params(B, L, D, N, rows=rows), cb.make_scan_params(-(-rows // L), L, D, N)
    size = cb.cawn_selective_scan_workspace_bytes
    assert size(packed, cb.CAWN_SCAN_FWD) <= size(dense, cb.CAWN_SCAN_FWD) + B * D * N * 4 + 1024
    assert size(packed, cb.CAWN_SCAN_BWD) <= size(dense, cb.CAWN_SCAN_BWD) + B * D * (N + 2) * 4 + 1024
