"""A residual layer around the gated delta rule, trained and then run token by token.

    x -> rms norm -> projection (q | k | v | gate) and (decay, step)
      -> q, k to unit rows -> gated delta rule -> per-head norm times SiLU(gate) -> projection
      -> dropout, added to x

All of it but the matrix products is the library's: cawn_group_norm_* (three times, once on slices of
the projection), cawn_delta_rule_* (prompt, single tokens, gradient), cawn_dropout (mask drawn from a
seed and a call number, never stored).

    python examples/gated_delta_layer.py        # a few training steps, then a prompt and its continuation
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2604_04250_b200 import binding as cb


def _flags(x):
    return cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16 if x.dtype == torch.bfloat16 else 0


class GroupNorm(torch.autograd.Function):
    """x and gate [N, G*M]: rows may be slices of wider ones."""

    @staticmethod
    def forward(ctx, x, weight, gate, G, rms, eps):
        act = cb.CAWN_NORM_ACT_NONE if gate is None else cb.CAWN_NORM_ACT_GATE
        ctx.prm = cb.make_norm_params(x.shape[0], G, x.shape[1] // G, eps=eps, act=act, rms=rms, flags=_flags(x),
                                      x_stride=x.stride(0), gate_stride=0 if gate is None else gate.stride(0))
        ctx.save_for_backward(x, weight, gate)
        y = x.new_empty(x.shape)
        cb.cawn_group_norm_fwd(ctx.prm, x, y, weight=weight, gate=gate)
        return y

    @staticmethod
    def backward(ctx, grad_y):
        x, weight, gate = ctx.saved_tensors
        grad_x = x.new_empty(x.shape)
        grad_gate = None if gate is None else x.new_empty(x.shape)
        grad_weight, workspace = None, None
        if ctx.needs_input_grad[1]:
            grad_weight, workspace = torch.empty_like(weight), cb.new_norm_workspace(ctx.prm)
        cb.cawn_group_norm_bwd(ctx.prm, x, grad_y.contiguous(), grad_x, workspace, weight=weight, gate=gate,
                               grad_gate=grad_gate, grad_weight=grad_weight)
        return grad_x, grad_weight, grad_gate, None, None, None


class DeltaRule(torch.autograd.Function):
    """q, k [B, L, Hk, Dk], v [B, L, Hv, Dv], g, beta [B, L, Hv] float, state [B, Hv, Dv, Dk] float -> o, state."""

    @staticmethod
    def forward(ctx, q, k, v, g, beta, state):
        B, L, Hk, Dk = q.shape
        Hv, Dv = v.shape[2:]
        ctx.prm = cb.make_delta_params(B, L, Hk, Hv, Dk, Dv, flags=_flags(v), q_stride=q.stride(1), k_stride=k.stride(1),
                                       v_stride=v.stride(1))
        ctx.save_for_backward(q, k, v, g, beta, state)
        o, state_out = v.new_empty(v.shape), torch.empty_like(state)
        if L == 1:
            cb.cawn_delta_rule_step(ctx.prm, q, k, v, g, beta, o, state_in=state, state_out=state_out)
        else:
            cb.cawn_delta_rule_fwd(ctx.prm, q, k, v, g, beta, o, cb.new_delta_workspace(ctx.prm, cb.CAWN_DELTA_FWD),
                                   state_in=state, state_out=state_out)
        return o, state_out

    @staticmethod
    def backward(ctx, grad_o, grad_state_out):
        q, k, v, g, beta, state = ctx.saved_tensors
        grads = [x.new_empty(x.shape) for x in (q, k, v, g, beta, state)]
        cb.cawn_delta_rule_bwd(ctx.prm, q, k, v, g, beta, grad_o.contiguous(), *grads[:5],
                               cb.new_delta_workspace(ctx.prm, cb.CAWN_DELTA_BWD), state_in=state,
                               grad_state_out=grad_state_out.contiguous(), grad_state_in=grads[5])
        return tuple(grads)


class DropoutAdd(torch.autograd.Function):
    """residual + dropout(x); (seed, offset) name the mask, and the gradient draws it again."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        ctx.prm = cb.make_dropout_params(x.numel(), p, seed, offset, flags=_flags(x))
        y = torch.empty_like(x)
        cb.cawn_dropout(ctx.prm, x, y, residual=residual)
        return y

    @staticmethod
    def backward(ctx, grad_y):
        grad_y = grad_y.contiguous()
        grad_x = torch.empty_like(grad_y)
        cb.cawn_dropout(ctx.prm, grad_y, grad_x)
        return grad_x, grad_y, None, None, None


class GatedDeltaLayer(torch.nn.Module):
    def __init__(self, width, Hk, Hv, Dk, Dv, p=0.1, seed=0, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.Hk, self.Hv, self.Dk, self.Dv, self.p, self.seed, self.calls = Hk, Hv, Dk, Dv, p, seed, 0
        rng = torch.Generator(device=device).manual_seed(seed)
        parameter = lambda rows, cols, type: torch.nn.Parameter(
            (torch.randn(rows, cols, generator=rng, device=device) * cols ** -0.5).to(type))
        ones = lambda n: torch.nn.Parameter(torch.ones(n, device=device))
        self.w_in = parameter(2 * Hk * Dk + 2 * Hv * Dv, width, dtype)
        self.w_rates = parameter(2 * Hv, width, torch.float32)
        self.w_out = parameter(width, Hv * Dv, dtype)
        self.norm_in, self.norm_out = ones(width), ones(Hv * Dv)
        self.log_rate = torch.nn.Parameter(torch.linspace(-4.0, 0.0, Hv, device=device))
        self.register_buffer("unit", torch.full((2 * Hk * Dk,), Dk ** -0.5, device=device))

    def new_state(self, B):
        return torch.zeros(B, self.Hv, self.Dv, self.Dk, device=self.w_in.device)

    def forward(self, x, state):
        """x [B, L, width] -> the stream behind the layer, and the state behind its last token."""
        x = x.contiguous()
        B, L, width = x.shape
        Hk, Hv, Dk, Dv = self.Hk, self.Hv, self.Dk, self.Dv
        h = GroupNorm.apply(x.reshape(B * L, width), self.norm_in, None, 1, True, 1e-6)
        qk, v, gate = (h @ self.w_in.T).split([2 * Hk * Dk, Hv * Dv, Hv * Dv], -1)
        decay, step = (h.float() @ self.w_rates.T).view(B, L, 2 * Hv).chunk(2, -1)
        qk = GroupNorm.apply(qk, self.unit, None, 2 * Hk, True, 1e-6).view(B, L, 2 * Hk, Dk)
        g = -torch.exp(self.log_rate) * F.softplus(decay)
        o, state = DeltaRule.apply(qk[:, :, :Hk], qk[:, :, Hk:], v.unflatten(0, (B, L)).unflatten(-1, (Hv, Dv)), g,
                                   torch.sigmoid(step).contiguous(), state)
        y = GroupNorm.apply(o.view(B * L, Hv * Dv), self.norm_out, gate, Hv, True, 1e-6) @ self.w_out.T
        self.calls += 1
        return DropoutAdd.apply(y.view(B, L, width), x, self.p if self.training else 0.0, self.seed, self.calls), state


def main():
    torch.manual_seed(0)
    B, L, width = 4, 512, 768
    layer = GatedDeltaLayer(width, 12, 12, 64, 64)
    opt = torch.optim.Adam(layer.parameters(), lr=3e-3)
    x = torch.randn(B, L, width, device="cuda").bfloat16()
    want = torch.cat([torch.zeros_like(x[:, :8]), x[:, :-8]], 1)          # recall the token eight steps back
    for i in range(20):
        y, _ = layer(x, layer.new_state(B))
        loss = F.mse_loss((y - x).float(), want.float())
        opt.zero_grad()
        loss.backward()
        opt.step()
        if i % 5 == 0 or i == 19:
            print(f"step {i:2d}  loss {loss.item():.4f}")
    layer.eval()
    with torch.no_grad():
        whole, last = layer(x, layer.new_state(B))
        y, state = layer(x[:, :500], layer.new_state(B))                   # the prompt at once ...
        parts = [y]
        for t in range(500, L):                                            # ... then a token at a time
            y, state = layer(x[:, t:t + 1], state)
            parts.append(y)
    d = (torch.cat(parts, 1) - whole).float().abs().max().item()
    print(f"prompt + single tokens against the whole sequence: largest difference {d:.3g}, state "
          f"{((state - last).norm() / last.norm()).item():.2g} of its norm")


if __name__ == "__main__":
    main()
