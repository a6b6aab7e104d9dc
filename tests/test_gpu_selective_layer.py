"""The example's layer: residual norm, short convolution and selective scan as they are used together, against the same layer written
with torch in 64 bits.

Tolerance, float storage: the scan is within 1.2e-5 of its norm, the norm, the convolution and each product of up to 128 terms in
float32 within 2e-6; the three products and the gate behind and in front of the scan may each double an error that reaches them: 1e-4.
"""
import importlib.util
import os

import pytest
import torch

from delta_ref import close
from selective_ref import residual_norm, selective_scan, short_conv, to_e4m3

pytestmark = pytest.mark.gpu
TOL = 1e-4


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "selective_scan_layer.py")
    spec = importlib.util.spec_from_file_location("selective_scan_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_layer(layer, w, branch, stream, history, state, offsets, L, eight_bit=False):
    """The layer in the type of its arguments, on the CPU; w: its parameters."""
    D, N = layer.D, layer.N
    total = branch + stream
    h = residual_norm(total, w["norm"], 1e-6)
    if eight_bit:
        q, scales = to_e4m3(h, 128)
        h = q.double() * scales.repeat_interleave(128, 1)[:, :h.shape[1]]
    x, z = (h @ w["w_in"].T).chunk(2, -1)
    x, history = short_conv(x, w["conv_w"], w["conv_b"], True, history, offsets, L)
    low, B, C = (x @ w["w_x"].T).split([layer.rank, N, N], -1)
    y, state = selective_scan(x, low @ w["w_dt"].T, -torch.exp(w["A_log"]), B[:, None], C[:, None], w["skip"], w["dt_bias"], z, state, offsets, L)
    return y @ w["w_out"].T, total, history, state


@pytest.mark.parametrize("lengths", [(40, 40), (70, 0, 3, 21)], ids=["dense", "packed"])
def test_layer_and_its_gradients(example, lengths):
    width, D, N, rows, B = 96, 128, 16, sum(lengths), len(lengths)
    packed = len(set(lengths)) > 1
    offsets = [0, *torch.tensor(lengths).cumsum(0).tolist()]
    layer = example.SelectiveLayer(width, D, N, rank=8, seed=5, dtype=torch.float32)
    rng = torch.Generator().manual_seed(1)
    ins = [torch.randn(s, generator=rng) for s in ((rows, width), (rows, width), (B, 3, D), (B, D, N))]
    outs = [torch.randn(s, generator=rng) for s in ((rows, width), (rows, width), (B, 3, D), (B, D, N))]
    c = [t.cuda().requires_grad_() for t in ins]
    y, total, (history, state) = layer(c[0], c[1], (c[2], c[3]), torch.tensor(offsets, device="cuda") if packed else None, max(lengths))
    torch.autograd.backward([y, total, history, state], [g.cuda() for g in outs])

    w = {n: t.detach().double().cpu().requires_grad_() for n, t in layer.named_parameters()}
    d = [t.double().requires_grad_() for t in ins]
    want = plain_layer(layer, w, *d, offsets, max(lengths))
    torch.autograd.backward(list(want), [g.double() for g in outs])
    for got, ref, name in zip((y, total, history, state), want, ("y", "stream", "history", "state")):
        close(got, ref, TOL, name)
    for got, ref, name in zip(c, d, ("branch", "stream", "history", "state")):
        close(got.grad, ref.grad, TOL, "grad of " + name)
    for n, t in layer.named_parameters():
        close(t.grad, w[n].grad, TOL, n)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, TOL), (torch.bfloat16, 2e-2)])
def test_prompt_then_single_tokens(example, dtype, tol):
    """A prompt at once and its continuation token by token give what the whole sequence gives (bfloat16: each side rounds its
    activations to 8 bits six times over)."""
    B, L, width = 3, 60, 96
    layer = example.SelectiveLayer(width, 128, 16, rank=8, seed=3, dtype=dtype)
    branch = torch.randn(B, L, width, generator=torch.Generator().manual_seed(2)).cuda().to(dtype)
    stream = torch.zeros(B, L, width, device="cuda")
    rows = lambda t, a, e: t[:, a:e].reshape(-1, width)
    with torch.no_grad():
        whole, _, last = layer(rows(branch, 0, L), rows(stream, 0, L), layer.new_state(B))
        y, _, state = layer(rows(branch, 0, 50), rows(stream, 0, 50), layer.new_state(B))
        parts = [y.view(B, 50, width)]
        for t in range(50, L):
            y, _, state = layer(rows(branch, t, t + 1), rows(stream, t, t + 1), state)
            parts.append(y.view(B, 1, width))
    close(torch.cat(parts, 1), whole.view(B, L, width), tol, "y")
    close(state[0], last[0], tol, "history")
    close(state[1], last[1], tol, "state")


def test_norm_in_eight_bits(example):
    """The same layer with 8-bit rows in front of its first product, against the definition with rows rounded alike.  A few of the
    5,000 values may be rounded the other way (see the norm's own test): by an eighth of themselves, so 1 of 5,000 is 2e-3 of the
    rows' norm."""
    rows, width = 40, 128
    layer = example.SelectiveLayer(width, 64, 16, rank=8, seed=4, dtype=torch.float32)
    rng = torch.Generator().manual_seed(6)
    branch, stream = torch.randn(rows, width, generator=rng), torch.randn(rows, width, generator=rng)
    with torch.no_grad():
        y, total, state = layer(branch.cuda(), stream.cuda(), layer.new_state(2), eight_bit=True)
    w = {n: t.detach().double().cpu() for n, t in layer.named_parameters()}
    want = plain_layer(layer, w, branch.float().double(), stream.double(), torch.zeros(2, 3, 64).double(), torch.zeros(2, 64, 16).double(), [0, 20, 40], 20, True)
    close(y, want[0], 5e-3, "y")
    close(state[1], want[3], 5e-3, "state")
