"""The example's layer: norm, delta rule, gated norm and dropout as they are used together, against the same layer
written with torch in 64 bits.

Tolerance, float storage: the delta rule is within 1e-5 of its norm, each norm and each product of up to 128 terms in
float32 within 1e-6; the two norms and two products behind it may each double an error that reaches them: 5e-5.
"""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

from delta_ref import close, delta_rule, philox_bits

pytestmark = pytest.mark.gpu
TOL = 5e-5


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "gated_delta_layer.py")
    spec = importlib.util.spec_from_file_location("gated_delta_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_layer(layer, w, x, state, mask):
    """The layer in the type of its arguments, on the CPU; w: its parameters."""
    B, L, width = x.shape
    Hk, Hv, Dk, Dv = layer.Hk, layer.Hv, layer.Dk, layer.Dv
    rms = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    h = rms(x) * w["norm_in"]
    qk, v, gate = (h @ w["w_in"].T).split([2 * Hk * Dk, Hv * Dv, Hv * Dv], -1)
    decay, step = (h @ w["w_rates"].T).chunk(2, -1)
    qk = rms(qk.unflatten(-1, (2 * Hk, Dk))) * Dk ** -0.5
    g = -torch.exp(w["log_rate"]) * F.softplus(decay)
    o, state = delta_rule(qk[:, :, :Hk], qk[:, :, Hk:], v.unflatten(-1, (Hv, Dv)), g, torch.sigmoid(step), Dk ** -0.5, state)
    y = rms(o).flatten(2) * w["norm_out"] * F.silu(gate)
    return x + mask * (y @ w["w_out"].T), state


def test_layer_and_its_gradients(example):
    B, L, width, p = 2, 70, 128, 0.25
    layer = example.GatedDeltaLayer(width, 2, 4, 64, 32, p=p, seed=5, dtype=torch.float32)
    rng = torch.Generator().manual_seed(1)
    x, state, gy, gs = (torch.randn(s, generator=rng) for s in ((B, L, width), (B, 4, 32, 64), (B, L, width), (B, 4, 32, 64)))
    xc, sc = x.cuda().requires_grad_(), (0.3 * state).cuda().requires_grad_()
    y, s = layer(xc, sc)
    torch.autograd.backward([y, s], [gy.cuda(), gs.cuda()])

    w = {n: t.detach().double().cpu().requires_grad_() for n, t in layer.named_parameters()}
    xd, sd = x.double().requires_grad_(), (0.3 * state).double().requires_grad_()
    keep = torch.from_numpy(philox_bits(x.numel(), 5, 1) >= round(p * 65536)).view(x.shape)      # first call: offset 1
    want_y, want_s = plain_layer(layer, w, xd, sd, keep / (1 - p))
    torch.autograd.backward([want_y, want_s], [gy.double(), gs.double()])
    close(y, want_y, TOL, "y")
    close(s, want_s, TOL, "state")
    close(xc.grad, xd.grad, TOL, "x")
    close(sc.grad, sd.grad, TOL, "state_in")
    for n, t in layer.named_parameters():
        close(t.grad, w[n].grad, TOL, n)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, TOL), (torch.bfloat16, 2e-2)])
def test_prompt_then_single_tokens(example, dtype, tol):
    """A prompt at once and its continuation token by token give what the whole sequence gives (bfloat16: each side
    rounds its activations to 8 bits five times over)."""
    B, L, width = 3, 90, 128
    layer = example.GatedDeltaLayer(width, 2, 2, 64, 64, seed=3, dtype=dtype).eval()
    x = torch.randn(B, L, width, generator=torch.Generator().manual_seed(2)).cuda().to(dtype)
    with torch.no_grad():
        whole, last = layer(x, layer.new_state(B))
        y, state = layer(x[:, :80], layer.new_state(B))
        parts = [y]
        for t in range(80, L):
            y, state = layer(x[:, t:t + 1], state)
            parts.append(y)
    close(torch.cat(parts, 1) - x, whole - x, tol, "y")
    close(state, last, tol, "state")
