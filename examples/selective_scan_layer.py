"""A residual layer around the selective scan, trained on packed sequences and then run token by token.

    stream + branch -> rms norm -> projection (x | z) -> short causal convolution with SiLU
      -> projection (step factor | B | C) -> step sizes -> selective scan, gated by z -> projection: the next branch

All of it but the matrix products is the library's: cawn_residual_norm_* (which adds the branch of the layer before to the
stream), cawn_short_conv_* and cawn_selective_scan_* (sequences of unequal lengths behind one another, prompt, single tokens,
gradient).  With eight_bit=True the norm hands 8-bit values and their scales to the first projection.

    python examples/selective_scan_layer.py     # a few training steps, then a prompt and its continuation
"""
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2604_04250_b200 import binding as cb


def _flags(x):
    return cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16 if x.dtype == torch.bfloat16 else 0


class ResidualNorm(torch.autograd.Function):
    """x [rows, width], stream [rows, width] (float, or of x's type) -> normed rows, x + stream."""

    @staticmethod
    def forward(ctx, x, stream, weight, eps):
        ctx.prm = cb.make_residual_norm_params(x.shape[0], x.shape[1], eps=eps, stream_float=stream.dtype != x.dtype, flags=_flags(x))
        y, total = torch.empty_like(x), torch.empty_like(stream)
        cb.cawn_residual_norm_fwd(ctx.prm, x, y, residual=stream, weight=weight, sum_out=total)
        ctx.save_for_backward(total, weight)
        return y, total

    @staticmethod
    def backward(ctx, grad_y, grad_total):
        total, weight = ctx.saved_tensors
        grad_stream, grad_weight = torch.empty_like(total), torch.empty_like(weight)
        grad_x = torch.empty_like(grad_y, memory_format=torch.contiguous_format) if grad_y.dtype != total.dtype else None
        cb.cawn_residual_norm_bwd(ctx.prm, total, grad_y.contiguous(), cb.new_residual_norm_workspace(ctx.prm), weight=weight,
                                  grad_sum=grad_total.contiguous(), grad_residual=grad_stream, grad_x=grad_x, grad_weight=grad_weight)
        return grad_stream if grad_x is None else grad_x, grad_stream, grad_weight, None


class ShortConv(torch.autograd.Function):
    """x [rows, C] (may be a slice of wider rows), history [B, K-1, C] float -> y, history."""

    @staticmethod
    def forward(ctx, x, weight, bias, history, offsets, longest):
        B, C, K = history.shape[0], x.shape[1], weight.shape[1]
        ctx.prm = cb.make_conv_params(B, longest, C, K, act=cb.CAWN_CONV_ACT_SILU, flags=_flags(x), x_stride=x.stride(0),
                                      rows=0 if offsets is None else x.shape[0])
        ctx.offsets = offsets
        ctx.save_for_backward(x, weight, bias, history)
        y, out = x.new_empty(x.shape), torch.empty_like(history)
        cb.cawn_short_conv_fwd(ctx.prm, x, weight, y, bias=bias, state_in=history, state_out=out, offsets=offsets)
        return y, out

    @staticmethod
    def backward(ctx, grad_y, grad_out):
        x, weight, bias, history = ctx.saved_tensors
        grads = [t.new_empty(t.shape) for t in (x, weight, bias, history)]
        cb.cawn_short_conv_bwd(ctx.prm, x, weight, grad_y.contiguous(), grads[0], cb.new_conv_workspace(ctx.prm), bias=bias, state_in=history,
                               offsets=ctx.offsets, grad_state_out=grad_out.contiguous(), grad_weight=grads[1], grad_bias=grads[2], grad_state_in=grads[3])
        return (*grads, None, None)


class SelectiveScan(torch.autograd.Function):
    """x, dt, z [rows, D], A [D, N], B, C [rows, N], state [B, D, N] float -> y, state."""

    @staticmethod
    def forward(ctx, x, dt, A, B, C, skip, dt_bias, z, state, offsets, longest):
        n, D, N = state.shape
        ctx.prm = prm = cb.make_scan_params(n, longest, D, N, flags=_flags(x), x_stride=x.stride(0), dt_stride=dt.stride(0), z_stride=z.stride(0),
                                            b_stride=B.stride(0), c_stride=C.stride(0), rows=0 if offsets is None else x.shape[0])
        ctx.offsets = offsets
        y, out = x.new_empty(x.shape), torch.empty_like(state)
        same = dict(skip=skip, dt_bias=dt_bias, z=z, state_in=state)
        if longest == 1 and offsets is None:
            cb.cawn_selective_scan_step(prm, x, dt, A, B, C, y, state_out=out, **same)
            ctx.checkpoints = None
        else:
            ctx.checkpoints = cb.new_scan_workspace(prm, cb.CAWN_SCAN_CHECKPOINTS) if any(ctx.needs_input_grad) else None
            cb.cawn_selective_scan_fwd(prm, x, dt, A, B, C, y, cb.new_scan_workspace(prm, cb.CAWN_SCAN_FWD), state_out=out, offsets=offsets,
                                       checkpoints=ctx.checkpoints, **same)
        ctx.save_for_backward(x, dt, A, B, C, skip, dt_bias, z, state)
        return y, out

    @staticmethod
    def backward(ctx, grad_y, grad_out):
        x, dt, A, B, C, skip, dt_bias, z, state = ctx.saved_tensors
        g = [t.new_empty(t.shape) for t in (x, dt, A, B, C, skip, dt_bias, z, state)]
        op = cb.CAWN_SCAN_BWD_RECOMPUTE if ctx.checkpoints is None else cb.CAWN_SCAN_BWD
        cb.cawn_selective_scan_bwd(ctx.prm, x, dt, A, B, C, grad_y.contiguous(), *g[:5], cb.new_scan_workspace(ctx.prm, op), skip=skip, dt_bias=dt_bias, z=z,
                                   state_in=state, offsets=ctx.offsets, checkpoints=ctx.checkpoints, grad_state_out=grad_out.contiguous(),
                                   grad_skip=g[5], grad_dt_bias=g[6], grad_z=g[7], grad_state_in=g[8])
        return (*g, None, None)


class SelectiveLayer(torch.nn.Module):
    def __init__(self, width, D, N, K=4, rank=16, seed=0, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.D, self.N, self.K, self.rank = D, N, K, rank
        rng = torch.Generator(device=device).manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=rng, device=device)
        product = lambda rows, cols: torch.nn.Parameter((randn(rows, cols) * cols ** -0.5).to(dtype))
        self.norm = torch.nn.Parameter(torch.ones(width, device=device))
        self.w_in, self.w_x, self.w_dt, self.w_out = product(2 * D, width), product(rank + 2 * N, D), product(D, rank), product(width, D)
        self.conv_w, self.conv_b = torch.nn.Parameter(randn(D, K) * K ** -0.5), torch.nn.Parameter(torch.zeros(D, device=device))
        self.A_log = torch.nn.Parameter(torch.log(torch.arange(1.0, N + 1, device=device)).expand(D, N).contiguous())
        self.skip = torch.nn.Parameter(torch.ones(D, device=device))
        step = torch.exp(torch.rand(D, generator=rng, device=device) * math.log(100.0)) * 0.001         # 0.001 to 0.1
        self.dt_bias = torch.nn.Parameter(torch.log(torch.expm1(step)))

    def new_state(self, B):
        new = lambda *s: torch.zeros(B, *s, device=self.w_in.device)
        return new(self.K - 1, self.D), new(self.D, self.N)

    def rows_of_norm(self, branch, stream, eight_bit):
        """The normed rows and the stream; in 8 bits as the values that they stand for, which an 8-bit product would take as they are."""
        if not eight_bit:
            return ResidualNorm.apply(branch, stream, self.norm, 1e-6)
        rows, width = branch.shape
        prm = cb.make_residual_norm_params(rows, width, eps=1e-6, out=cb.CAWN_NORM_OUT_E4M3, scale_block=128, stream_float=stream.dtype != branch.dtype,
                                           flags=_flags(branch))
        q, total = torch.empty(rows, width, dtype=torch.float8_e4m3fn, device=branch.device), torch.empty_like(stream)
        scales = torch.empty(rows, -(-width // 128), device=branch.device)
        cb.cawn_residual_norm_fwd(prm, branch, q, residual=stream, weight=self.norm, sum_out=total, scales=scales)
        return (q.float() * scales.repeat_interleave(128, 1)[:, :width]).to(branch.dtype), total

    def forward(self, branch, stream, state, offsets=None, longest=None, eight_bit=False):
        """branch, stream [rows, width] -> the next branch, the stream, the states.  Dense: B sequences of `longest` rows each."""
        longest = branch.shape[0] // state[0].shape[0] if longest is None else longest
        h, stream = self.rows_of_norm(branch.contiguous(), stream.contiguous(), eight_bit)
        x, z = (h @ self.w_in.T).chunk(2, -1)
        x, history = ShortConv.apply(x, self.conv_w, self.conv_b, state[0], offsets, longest)
        low, B, C = (x @ self.w_x.T).split([self.rank, self.N, self.N], -1)
        y, last = SelectiveScan.apply(x, low @ self.w_dt.T, -torch.exp(self.A_log), B, C, self.skip, self.dt_bias, z, state[1], offsets, longest)
        return y @ self.w_out.T, stream, (history, last)


def main():
    torch.manual_seed(0)
    width, lengths = 768, [700, 37, 1200, 111]
    layer = SelectiveLayer(width, 1024, 16, rank=48)
    opt = torch.optim.Adam(layer.parameters(), lr=3e-3)
    offsets = torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], device="cuda")
    rows = sum(lengths)
    branch, stream = torch.randn(rows, width, device="cuda").bfloat16(), torch.zeros(rows, width, device="cuda")
    want = torch.cat([torch.zeros_like(branch[:2]), branch[:-2]]).float()           # recall the token two steps back
    for i in range(20):
        y, total, _ = layer(branch, stream, layer.new_state(len(lengths)), offsets, max(lengths))
        loss = F.mse_loss(y.float(), want)
        opt.zero_grad()
        loss.backward()
        opt.step()
        if i % 5 == 0 or i == 19:
            print(f"step {i:2d}  loss {loss.item():.4f}")
    with torch.no_grad():
        B, L = 4, 512
        branch, stream = branch[:B * L].view(B, L, width), stream[:B * L].view(B, L, width)
        rows_of = lambda t, a, e: t[:, a:e].reshape(-1, width)
        whole, _, last = layer(rows_of(branch, 0, L), rows_of(stream, 0, L), layer.new_state(B))
        y, _, state = layer(rows_of(branch, 0, 500), rows_of(stream, 0, 500), layer.new_state(B))       # the prompt at once ...
        parts = [y.view(B, 500, width)]
        for t in range(500, L):                                                                         # ... then a token at a time
            y, _, state = layer(rows_of(branch, t, t + 1), rows_of(stream, t, t + 1), state)
            parts.append(y.view(B, 1, width))
        d = (torch.cat(parts, 1) - whole.view(B, L, width)).float().abs().max().item()
        print(f"prompt + single tokens against the whole sequence: largest difference {d:.3g}, state "
              f"{((state[1] - last[1]).norm() / last[1].norm()).item():.2g} of its norm")


if __name__ == "__main__":
    main()
