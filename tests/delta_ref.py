"""Plain 64-bit forms of the operators next to the scan: the definitions, one token / row / element at
a time, on the CPU.  Gradients come from automatic differentiation of the same definitions."""
import numpy as np
import torch

from paper_2604_04250_b200 import binding as cb

BF16 = cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16


def flags_of(dtype):
    return BF16 if dtype == torch.bfloat16 else 0


def delta_rule(q, k, v, g, beta, scale, state):
    """Gated delta rule by its recurrence; state [B, Hv, Dv, Dk].  Returns (o, state)."""
    rep = v.shape[2] // q.shape[2]
    q, k = q.repeat_interleave(rep, 2), k.repeat_interleave(rep, 2)
    S, out = state, []
    for t in range(v.shape[1]):
        S = torch.exp(g[:, t])[..., None, None] * S
        u = beta[:, t][..., None] * (v[:, t] - torch.einsum("bhvk,bhk->bhv", S, k[:, t]))
        S = S + torch.einsum("bhv,bhk->bhvk", u, k[:, t])
        out.append(scale * torch.einsum("bhvk,bhk->bhv", S, q[:, t]))
    return (torch.stack(out, 1) if out else torch.zeros_like(v)), S


def delta_inputs(B, L, Hk, Hv, Dk, Dv, dtype, seed, rate=(0.002, 1.0), lean=0.4):
    """Unit queries and keys leaning towards a common direction, decays from long to short memory."""
    rng = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=rng)
    unit = lambda x: torch.nn.functional.normalize(x, dim=-1)
    d = {"q": unit(randn(B, L, Hk, Dk) + lean * randn(1, 1, Hk, Dk)).to(dtype),
         "k": unit(randn(B, L, Hk, Dk) + lean * randn(1, 1, Hk, Dk)).to(dtype),
         "v": randn(B, L, Hv, Dv).to(dtype)}
    rates = torch.exp(torch.linspace(np.log(rate[0]), np.log(rate[1]), Hv))
    d["g"] = -rates * torch.nn.functional.softplus(randn(B, L, Hv))
    d["beta"] = torch.sigmoid(randn(B, L, Hv))
    d["state_in"] = 0.5 * randn(B, Hv, Dv, Dk)
    d["grad_o"] = randn(B, L, Hv, Dv).to(dtype)
    d["grad_state_out"] = 0.1 * randn(B, Hv, Dv, Dk)
    return d


def group_norm(x, G, eps, rms, w, b, act, gate):
    N, C = x.shape
    xs = x.reshape(N, G, C // G)
    if not rms:
        xs = xs - xs.mean(2, keepdim=True)
    z = (xs / torch.sqrt((xs ** 2).mean(2, keepdim=True) + eps)).reshape(N, C)
    z = z if w is None else z * w
    z = z if b is None else z + b
    if act == cb.CAWN_NORM_ACT_SILU:
        return z * torch.sigmoid(z)
    return z * gate * torch.sigmoid(gate) if act == cb.CAWN_NORM_ACT_GATE else z


def philox_bits(n, seed, offset):
    """16 bits per element, Python integers throughout."""
    out = []
    for i in range((n + 7) // 8):
        c, k = [i & 0xFFFFFFFF, i >> 32, offset & 0xFFFFFFFF, offset >> 32], [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        for w in c:
            out += [w & 0xFFFF, w >> 16]
    return np.array(out[:n])


def philox_words(counter, key):
    """The published generator on four counter words and two key words."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


# Known answers of Philox4x32-10 as its authors publish them: counter, key, result
PHILOX_ANSWERS = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


def errors(got, want):
    """(relative 2-norm, largest difference over max(|want|, rms)); non-finite values have to agree."""
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    assert got.shape == want.shape
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), "finite where the definition is not, or the other way round"
    got, want = got[fine], want[fine]
    if want.numel() == 0:
        return 0.0, 0.0
    rms = want.square().mean().sqrt()
    if rms == 0:
        return (0.0, 0.0) if (got == 0).all() else (float("inf"), float("inf"))
    d = (got - want).abs()
    return (d.square().mean().sqrt() / rms).item(), (d / want.abs().clamp_min(rms)).max().item()


def close(got, want, tol, what=""):
    """2-norm within tol, single elements within 40 tol (they are measured against the rms, and the
    largest of many normal errors is several times their root mean square)."""
    norm, worst = errors(got, want)
    assert norm <= tol and worst <= 40 * tol, (what, norm, worst, tol)
