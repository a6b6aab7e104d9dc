"""Plain 64-bit forms of the operators of a selective state space layer: the definitions, a sequence and a token at a
time, on the CPU.  Gradients come from automatic differentiation of the same definitions."""
import torch

from delta_ref import BF16


def spans(offsets, L):
    """(first row, length) of each sequence, as the device clamps them to L tokens."""
    return [(a, min(b - a, L)) for a, b in zip(offsets, offsets[1:])]


def short_conv(x, weight, bias, silu, state, offsets, L):
    """x [rows, C], weight [C, K], state [B, K-1, C] -> y (rows that no sequence has: 0), state."""
    K = weight.shape[1]
    y, states = torch.zeros_like(x), []
    for b, (a, n) in enumerate(spans(offsets, L)):
        e = torch.cat([state[b], x[a:a + n]])
        z = sum(e[k:k + n] * weight[:, k] for k in range(K)) + (0 if bias is None else bias)
        y = torch.cat([y[:a], z * torch.sigmoid(z) if silu else z, y[a + n:]])
        states.append(e[n:])
    return y, torch.stack(states)


def selective_scan(x, dt, A, B, C, skip, dt_bias, z, state, offsets, L, softplus=True):
    """x, dt, z [rows, D]; A [D, N]; B, C [rows, G, N]; state [B, D, N] -> y (rows that no sequence has: 0), state."""
    rows, D = x.shape
    rep = D // B.shape[1]
    d = dt if dt_bias is None else dt + dt_bias
    d = torch.nn.functional.softplus(d, threshold=1e9) if softplus else d
    B, C = B.repeat_interleave(rep, 1), C.repeat_interleave(rep, 1)
    out, states = [torch.zeros_like(x[0])] * rows, []
    for b, (a, n) in enumerate(spans(offsets, L)):
        h = state[b]
        for t in range(a, a + n):
            h = torch.exp(d[t][:, None] * A) * h + (d[t] * x[t])[:, None] * B[t]
            out[t] = (C[t] * h).sum(-1) + (0 if skip is None else skip * x[t])
        states.append(h)
    y = torch.stack(out) if out else torch.zeros_like(x)
    return (y if z is None else y * z * torch.sigmoid(z)), torch.stack(states)


def residual_norm(s, weight, eps):
    y = s / torch.sqrt((s ** 2).mean(1, keepdim=True) + eps)
    return y if weight is None else y * weight


def to_e4m3(y, block):
    """(stored, scales) of rows y in 64 bits."""
    M = y.shape[1]
    block = block or M
    scales, parts = [], []
    for c in range(0, M, block):
        part = y[:, c:c + block]
        scale = part.abs().amax(1).clamp_min(1e-30) / 448
        scales.append(scale)
        parts.append((part / scale[:, None]).to(torch.float8_e4m3fn))
    return torch.cat([p.float() for p in parts], 1), torch.stack(scales, 1)


def packed_offsets(lengths, first=0):
    out = [first]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def slices(x, pad, device="cuda"):
    """x [rows, width] on the device as the middle of rows that are 2 pad wider (NaN around it), or dense."""
    if not pad:
        return x.to(device)
    wide = torch.full((x.shape[0], x.shape[1] + 2 * pad), float("nan"), dtype=x.dtype, device=device)
    wide[:, pad:pad + x.shape[1]] = x.to(device)
    return wide[:, pad:pad + x.shape[1]]


def flags_of(dtype):
    return BF16 if dtype == torch.bfloat16 else 0
