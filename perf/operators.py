"""Workloads of the operators that stand next to the phase accumulation in a layer: the gated delta
rule (prefill, single tokens, backward), the group norm with activation of its heads (forward,
backward) and the counter-based dropout that adds a branch to the stream (either direction).

``run`` computes them with elementary torch operations in float32 where ``own`` is false and with
the library's entry points where it is true; ``exact`` follows the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
CHUNK = 64


# ------------------------------------------------------------------------------------ cases

def _delta(name, op, B, L, Hk, Hv, Dk, Dv, type, fused=False):
    return {"name": name, "op": op, "B": B, "L": L, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv, "type": type, "fused": fused}


def _norm(name, op, N, G, M, type, act, rms=False):
    return {"name": name, "op": op, "N": N, "G": G, "M": M, "type": type, "act": act, "rms": rms}


def _drop(name, op, n, p, type):
    return {"name": name, "op": op, "n": n, "p": p, "type": type}


def listed():
    return [
        # one stream generating: a single token through one layer's state, latency alone counts
        _delta("step-one-stream", "delta_step", 1, 1, 12, 12, 64, 64, "bf16"),
        # a serving batch, one token each: every state is read and written once
        _delta("step-batch", "delta_step", 96, 1, 8, 16, 128, 128, "bf16", fused=True),
        # prompt processing / training forward at the shape of the library's headline forward
        _delta("prefill", "delta_fwd", 8, 2048, 12, 12, 64, 64, "bf16"),
        # float32 tensors, shared key heads, a ragged length, unequal head widths
        _delta("prefill-fp32-ragged", "delta_fwd", 2, 1021, 4, 8, 64, 96, "fp32"),
        # one long prompt in the 32,768-token chunks of the paper's prefill: few rows, long time axis
        _delta("prefill-one-long", "delta_fwd", 1, 32768, 12, 12, 64, 64, "bf16", fused=True),
        # wide heads
        _delta("prefill-wide", "delta_fwd", 4, 4096, 8, 8, 128, 128, "bf16"),
        # training backward at the same shape as the forward
        _delta("backward", "delta_bwd", 8, 2048, 12, 12, 64, 64, "bf16"),
        # backward in float32 with shared key heads and a ragged length
        _delta("backward-fp32-shared", "delta_bwd", 2, 777, 2, 6, 128, 64, "fp32"),
        # head norm and output gate of a decode step for a small batch
        _norm("norm-decode", "norm_fwd", 24, 12, 64, "bf16", "gate"),
        # head norm, gate and their gradients over a training batch
        _norm("norm-backward", "norm_bwd", 32768, 12, 64, "bf16", "gate"),
        # the largest stream of the library's configurations: 16 x 8192 tokens of width 768
        _drop("dropout-residual", "drop_fwd", 16 * 8192 * 768, 0.1, "bf16"),
        # gradient through the same mask, float32, an odd count
        _drop("dropout-backward", "drop_bwd", 1021 * 895, 0.25, "fp32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["delta_step", "delta_fwd", "delta_fwd", "delta_bwd", "delta_bwd", "norm_fwd", "norm_bwd", "drop_fwd", "drop_bwd"])
    type = rng.choice(["bf16", "bf16", "fp32"])
    if op.startswith("delta"):
        Hk = rng.choice([1, 2, 3, 4, 8, 12])
        Hv = Hk * rng.choice([1, 1, 2, 3])
        Dk, Dv = rng.choice([(64, 64), (64, 64), (128, 128), (64, 128), (32, 64), (96, 80), (40, 24)])
        if op == "delta_step":
            L, B = rng.choice([1, 1, 2, 3, 4]), _log(rng, 1, 96)
        else:
            L = _log(rng, 33, 32768)
            B = _log(rng, 1, max(1, min(16, 16384 // L)))
            while B * L * Hv * Dk * Dv > 8 * 2048 * 12 * 64 * 64:       # no more than the largest listed one
                Hv, L = (Hv - Hk, L) if Hv > Hk else (Hv, L // 2)
        return {"op": op, "B": B, "L": L, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv, "type": type, "fused": rng.random() < 0.5}
    if op.startswith("norm"):
        G, M = rng.choice([(12, 64), (8, 128), (14, 64), (1, 768), (6, 80), (32, 8), (5, 37), (1, 896)])
        return {"op": op, "N": _log(rng, 1, 32768), "G": G, "M": M, "type": type, "act": rng.choice(["none", "silu", "gate"]), "rms": rng.random() < 0.3}
    return {"op": op, "n": _log(rng, 1000, 16 * 8192 * 768 // 2), "p": rng.choice([0.05, 0.1, 0.25, 0.5]), "type": type}


# ------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    rng = torch.Generator(device="cuda")
    rng.manual_seed(seed)
    dt = TYPES[case["type"]]

    def randn(*shape):
        return torch.randn(shape, generator=rng, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=rng, device="cuda")

    op = case["op"]
    s = {"case": case, "dt": dt}
    if op.startswith("delta"):
        B, L, Hk, Hv, Dk, Dv = (case[n] for n in ("B", "L", "Hk", "Hv", "Dk", "Dv"))
        # unit queries and keys that lean towards a common direction, as a trained layer's do
        unit = torch.nn.functional.normalize
        q = unit(randn(B, L, Hk, Dk) + 0.4 * randn(1, 1, Hk, Dk), dim=-1).to(dt)
        k = unit(randn(B, L, Hk, Dk) + 0.4 * randn(1, 1, Hk, Dk), dim=-1).to(dt)
        v = randn(B, L, Hv, Dv).to(dt)
        if case["fused"]:       # slices of one projection's output, [B, L, (q | k | v)]
            w = torch.cat([q.flatten(2), k.flatten(2), v.flatten(2)], dim=-1)
            q, k, v = w.split([Hk * Dk, Hk * Dk, Hv * Dv], dim=-1)
            q, k, v = q.unflatten(-1, (Hk, Dk)), k.unflatten(-1, (Hk, Dk)), v.unflatten(-1, (Hv, Dv))
        # log decay -rate * softplus(x): heads from long memory (rate 0.002) to short (rate 1)
        rate = torch.exp(torch.linspace(math.log(0.002), 0.0, Hv, device="cuda"))
        s.update(q=q, k=k, v=v, g=-rate * torch.nn.functional.softplus(randn(B, L, Hv)), beta=torch.sigmoid(randn(B, L, Hv)),
                 scale=Dk ** -0.5, state_in=0.5 * randn(B, Hv, Dv, Dk))
        if op == "delta_bwd":
            s.update(grad_o=randn(B, L, Hv, Dv).to(dt), grad_state_out=0.1 * randn(B, Hv, Dv, Dk))
    elif op.startswith("norm"):
        N, C = case["N"], case["G"] * case["M"]
        s.update(x=(randn(N, C) * (0.2 + rand(N, 1)) + 0.3).to(dt), weight=1 + 0.1 * randn(C), bias=0.1 * randn(C), eps=1e-5)
        if case["act"] == "gate":
            s["gate"] = randn(N, C).to(dt)
        if op == "norm_bwd":
            s["grad_y"] = randn(N, C).to(dt)
    else:
        words = np.random.RandomState(seed % (1 << 32)).randint(0, 1 << 32, 4, dtype=np.uint64)
        s.update(x=randn(case["n"]).to(dt), seed=int(words[0] << np.uint64(32) | words[1]), offset=int(words[2] << np.uint64(20) | words[3] >> np.uint64(12)))
        if op == "drop_fwd":
            s["residual"] = randn(case["n"]).to(dt)
    return s


# ------------------------------------------------------------------------------------ plain forms

def _chunks(x, H):
    """[B, L, h, ...] in chunks along time, shared heads repeated: [B, H, L/64, 64, ...] float32."""
    B, L, h = x.shape[:3]
    x = x.float().repeat_interleave(H // h, dim=2)
    x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, -L % CHUNK))
    return x.unflatten(1, (-1, CHUNK)).movedim(3, 1)


def _joined(x, L):
    """Inverse of _chunks for as many heads as there are: [B, L, H, ...]."""
    return x.movedim(1, 3).flatten(1, 2)[:, :L]


def _delta_pieces(s):
    Hv = s["v"].shape[2]
    q, k, v, g, beta = (_chunks(s[n], Hv) for n in ("q", "k", "v", "g", "beta"))
    G = g.cumsum(-1)
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=G.device).tril()
    gam = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~low, -math.inf))
    kk = (k @ k.mT * gam).tril(-1)
    qk = s["scale"] * (q @ k.mT) * gam
    A = kk * beta[..., None, :]
    T = torch.eye(CHUNK, device=G.device).expand_as(A).contiguous()
    for i in range(1, CHUNK):       # forward substitution, a row of every chunk at a time
        T[..., i, :i] = -(A[..., i, None, :i] @ T[..., :i, :i])[..., 0, :]
    return q, k, v, beta, G, gam, kk, qk, T


def _delta_forward(s, with_output=True):
    q, k, v, beta, G, gam, kk, qk, T = pieces = _delta_pieces(s)
    S = s["state_in"].mT                                       # [B, H, Dk, Dv]
    eG, left = torch.exp(G)[..., None], torch.exp(G[..., -1:] - G)[..., None]
    states, rs, outs = [], [], []
    for c in range(q.shape[2]):
        states.append(S)
        r = T[:, :, c] @ (v[:, :, c] - eG[:, :, c] * (k[:, :, c] @ S))
        u = beta[:, :, c, :, None] * r
        if with_output:
            outs.append(s["scale"] * eG[:, :, c] * (q[:, :, c] @ S) + qk[:, :, c] @ u)
        S = eG[:, :, c, -1:] * S + k[:, :, c].mT @ (left[:, :, c] * u)
        rs.append(r)
    return pieces, states, rs, outs, S, eG, left


def _delta_plain(s):
    L = s["v"].shape[1]
    _, _, _, outs, S, _, _ = _delta_forward(s)
    return {"o": _joined(torch.stack(outs, 2), L).to(s["dt"]), "state_out": S.mT.contiguous()}


def _delta_plain_backward(s):
    B, L, Hv, Dv = s["v"].shape
    Hk = s["q"].shape[2]
    (q, k, v, beta, G, gam, kk, qk, T), states, rs, _, _, eG, left = _delta_forward(s, False)
    do = _chunks(s["grad_o"], Hv)
    D = s["grad_state_out"].mT
    ends, rbs = [], []
    qs, PdO = (s["scale"] * eG * q).mT @ do, qk.mT @ do
    for c in reversed(range(q.shape[2])):
        ends.append(D)
        dU = PdO[:, :, c] + left[:, :, c] * (k[:, :, c] @ D)
        rb = T[:, :, c].mT @ (beta[:, :, c, :, None] * dU)
        D = eG[:, :, c, -1:] * D + qs[:, :, c] - (eG[:, :, c] * k[:, :, c]).mT @ rb
        rbs.append(rb)
    S, r, rb, E = torch.stack(states, 2), torch.stack(rs, 2), torch.stack(rbs[::-1], 2), torch.stack(ends[::-1], 2)
    D1, M = do @ r.mT, rb @ r.mT
    dP = s["scale"] * gam * beta[..., None, :] * D1
    dA = -(gam * beta[..., None, :] * M).tril(-1)
    dq_state = s["scale"] * eG * (do @ S.mT)
    rE = left * (r @ E.mT)
    dk_state = -eG * (rb @ S.mT)
    dq = dq_state + dP @ k
    dk = dP.mT @ q + beta[..., None] * rE + dk_state + (dA + dA.mT) @ k
    dbeta = (qk * D1).sum(-2) + (k * rE).sum(-1) - (kk * M).sum(-2)
    both = (qk * beta[..., None, :] * D1).tril(-1) - kk * beta[..., None, :] * M
    z = beta * (k * rE).sum(-1)
    dG = both.sum(-1) - both.sum(-2) + (q * dq_state).sum(-1) + (k * dk_state).sum(-1) - z
    end = z.sum(-1) + eG[..., -1, 0] * (S * E).sum((-1, -2))
    dg = dG.flip(-1).cumsum(-1).flip(-1) + end[..., None]
    dq, dk = (_joined(x, L).unflatten(2, (Hk, -1)).sum(3).to(s["dt"]) for x in (dq, dk))
    return {"grad_q": dq, "grad_k": dk, "grad_v": _joined(rb, L).to(s["dt"]), "grad_g": _joined(dg, L), "grad_beta": _joined(dbeta, L),
            "grad_state_in": D.mT.contiguous()}


def _step_plain(s):
    Hv = s["v"].shape[2]
    rep = Hv // s["q"].shape[2]
    q, k = (s[n].float().repeat_interleave(rep, dim=2) for n in ("q", "k"))
    v, S, outs = s["v"].float(), s["state_in"], []
    for t in range(v.shape[1]):
        S = torch.exp(s["g"][:, t, :, None, None]) * S
        u = s["beta"][:, t, :, None] * (v[:, t] - (S * k[:, t, :, None, :]).sum(-1))
        S = S + u[..., None] * k[:, t, :, None, :]
        outs.append(s["scale"] * (S * q[:, t, :, None, :]).sum(-1))
    return {"o": torch.stack(outs, 1).to(s["dt"]), "state_out": S}


def _norm_parts(s):
    case = s["case"]
    x = s["x"].float().unflatten(1, (case["G"], case["M"]))
    mean = 0.0 if case["rms"] else x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + s["eps"]).rsqrt()
    xh = (x - mean) * rstd
    return xh, rstd, xh.flatten(1) * s["weight"] + s["bias"]


def _norm_plain(s):
    z = _norm_parts(s)[2]
    if s["case"]["act"] == "silu":
        z = z / (1 + torch.exp(-z))
    elif s["case"]["act"] == "gate":
        gate = s["gate"].float()
        z = z * gate / (1 + torch.exp(-gate))
    return z.to(s["dt"])


def _norm_plain_backward(s):
    case = s["case"]
    xh, rstd, z = _norm_parts(s)
    dz = s["grad_y"].float()
    out = {}
    if case["act"] == "silu":
        sg = 1 / (1 + torch.exp(-z))
        dz = dz * sg * (1 + z * (1 - sg))
    elif case["act"] == "gate":
        gate = s["gate"].float()
        sg = 1 / (1 + torch.exp(-gate))
        out["grad_gate"] = (dz * z * sg * (1 + gate * (1 - sg))).to(s["dt"])
        dz = dz * gate * sg
    out["grad_weight"], out["grad_bias"] = (dz * xh.flatten(1)).sum(0), dz.sum(0)
    d = (dz * s["weight"]).unflatten(1, (case["G"], case["M"]))
    dx = d - xh * (d * xh).mean(-1, keepdim=True)
    if not case["rms"]:
        dx = dx - d.mean(-1, keepdim=True)
    out["grad_x"] = (rstd * dx).flatten(1).to(s["dt"])
    return out


def _mul32(a, b):
    """High and low 32 bits of a * b, a an int below 2^32, b int64 values below 2^32."""
    lo, hi = a * (b & 0xFFFF), a * (b >> 16)
    return (hi + (lo >> 16)) >> 16, (((hi & 0xFFFF) << 16) + lo) & 0xFFFFFFFF


def _bits(n, seed, offset, device):
    """16 random bits an element: Philox4x32-10 (Salmon et al. 2011) on counter (i / 8, offset), key seed."""
    i = torch.arange((n + 7) // 8, device=device)
    c = [i & 0xFFFFFFFF, i >> 32, torch.full_like(i, offset & 0xFFFFFFFF), torch.full_like(i, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = _mul32(0xD2511F53, c[0]), _mul32(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = torch.stack(c, -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).flatten()[:n]


def _drop_plain(s):
    drop = round(s["case"]["p"] * 65536)
    keep = _bits(s["case"]["n"], s["seed"], s["offset"], s["x"].device) >= drop
    y = torch.where(keep, s["x"].float() * (65536 / (65536 - drop)), 0.0)
    return (y + s["residual"].float() if "residual" in s else y).to(s["dt"])


# ------------------------------------------------------------------------------------ the library's calls

def _own_flags(s):
    from paper_2604_04250_b200 import binding as cb
    return cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16 if s["dt"] == torch.bfloat16 else 0


def _own_delta(s):
    from paper_2604_04250_b200 import binding as cb
    q, k, v = s["q"], s["k"], s["v"]
    B, L, Hv, Dv = v.shape
    prm = cb.make_delta_params(B, L, q.shape[2], Hv, q.shape[3], Dv, scale=s["scale"], flags=_own_flags(s),
                               q_stride=q.stride(1), k_stride=k.stride(1), v_stride=v.stride(1))
    op = s["case"]["op"]
    new = lambda x: torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if op == "delta_step":
        o, state = new(v), new(s["state_in"])
        cb.cawn_delta_rule_step(prm, q, k, v, s["g"], s["beta"], o, state_in=s["state_in"], state_out=state)
        return {"o": o, "state_out": state}
    if "workspace" not in s:        # kept by the program for its later calls, as all of the library's workspaces
        s["workspace"] = cb.new_delta_workspace(prm, cb.CAWN_DELTA_FWD if op == "delta_fwd" else cb.CAWN_DELTA_BWD)
    if op == "delta_fwd":
        o, state = new(v), new(s["state_in"])
        cb.cawn_delta_rule_fwd(prm, q, k, v, s["g"], s["beta"], o, s["workspace"], state_in=s["state_in"], state_out=state)
        return {"o": o, "state_out": state}
    out = {"grad_q": new(q), "grad_k": new(k), "grad_v": new(v), "grad_g": new(s["g"]), "grad_beta": new(s["beta"]), "grad_state_in": new(s["state_in"])}
    cb.cawn_delta_rule_bwd(prm, q, k, v, s["g"], s["beta"], s["grad_o"], out["grad_q"], out["grad_k"], out["grad_v"], out["grad_g"], out["grad_beta"],
                           s["workspace"], state_in=s["state_in"], grad_state_out=s["grad_state_out"], grad_state_in=out["grad_state_in"])
    return out


def _own_norm(s):
    from paper_2604_04250_b200 import binding as cb
    case, x = s["case"], s["x"]
    act = {"none": cb.CAWN_NORM_ACT_NONE, "silu": cb.CAWN_NORM_ACT_SILU, "gate": cb.CAWN_NORM_ACT_GATE}[case["act"]]
    prm = cb.make_norm_params(case["N"], case["G"], case["M"], eps=s["eps"], act=act, rms=case["rms"], flags=_own_flags(s))
    gate = s.get("gate")
    if case["op"] == "norm_fwd":
        y = torch.empty_like(x)
        cb.cawn_group_norm_fwd(prm, x, y, weight=s["weight"], bias=s["bias"], gate=gate)
        return y
    if "workspace" not in s:
        s["workspace"] = cb.new_norm_workspace(prm)
    out = {}
    if gate is not None:
        out["grad_gate"] = torch.empty_like(x)
    out["grad_weight"], out["grad_bias"], out["grad_x"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"]), torch.empty_like(x)
    cb.cawn_group_norm_bwd(prm, x, s["grad_y"], out["grad_x"], s["workspace"], weight=s["weight"], bias=s["bias"], gate=gate,
                           grad_gate=out.get("grad_gate"), grad_weight=out["grad_weight"], grad_bias=out["grad_bias"])
    return out


def _own_drop(s):
    from paper_2604_04250_b200 import binding as cb
    y = torch.empty_like(s["x"])
    prm = cb.make_dropout_params(s["case"]["n"], s["case"]["p"], s["seed"], s["offset"], flags=_own_flags(s))
    cb.cawn_dropout(prm, s["x"], y, residual=s.get("residual"))
    return y


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_delta(state) if op.startswith("delta") else _own_norm(state) if op.startswith("norm") else _own_drop(state)
    if op == "delta_step":
        return _step_plain(state)
    if op.startswith("delta"):
        return _delta_plain(state) if op == "delta_fwd" else _delta_plain_backward(state)
    if op.startswith("norm"):
        return _norm_plain(state) if op == "norm_fwd" else _norm_plain_backward(state)
    return _drop_plain(state)


# ------------------------------------------------------------------------------------ work

def work(case):
    e = 2 if case["type"] == "bf16" else 4
    op = case["op"]
    if op.startswith("delta"):
        B, L, Hk, Hv, Dk, Dv = (case[n] for n in ("B", "L", "Hk", "Hv", "Dk", "Dv"))
        row = 2 * Hk * Dk * e + Hv * Dv * e + 2 * Hv * 4      # q, k, v, g, beta
        state = B * Hv * Dk * Dv * 4
        cell = B * L * Hv * Dk * Dv
        if op == "delta_bwd":       # and the same again as gradients, dO in; states and their gradients end to end
            return {"bytes": B * L * (2 * row + Hv * Dv * e) + 3 * state, "flops": 21 * cell}
        return {"bytes": B * L * (row + Hv * Dv * e) + 2 * state, "flops": 7 * cell}
    if op.startswith("norm"):
        n = case["N"] * case["G"] * case["M"]
        gated = case["act"] == "gate"
        arrays = (3 if gated else 2) if op == "norm_fwd" else (5 if gated else 3)
        return {"bytes": n * e * arrays + case["G"] * case["M"] * (8 if op == "norm_fwd" else 16), "flops": n * (12 if op == "norm_fwd" else 25)}
    return {"bytes": case["n"] * e * (3 if op == "drop_fwd" else 2), "flops": 3 * case["n"]}


# ------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("delta"):
        return _exact_delta_backward(s) if op == "delta_bwd" else _exact_delta(s)
    if op.startswith("norm"):
        return _exact_norm(s)
    return _exact_drop(s)


def _walk(s, S, t):
    """One token of the recurrence: (decayed state, read-out error, correction, new state), states [B, H, Dk, Dv]."""
    Sd = S * s["a"][:, t, :, None, None]
    miss = s["v"][:, t] - torch.einsum("bhkv,bhk->bhv", Sd, s["k"][:, t])
    u = s["beta"][:, t, :, None] * miss
    return Sd, miss, u, Sd + torch.einsum("bhk,bhv->bhkv", s["k"][:, t], u)


def _wide(s):
    rep = s["v"].shape[2] // s["q"].shape[2]
    d = {n: s[n].double().contiguous() for n in ("q", "k", "v", "beta")}
    for n in ("q", "k"):
        d[n] = torch.repeat_interleave(d[n], rep, 2)
    d["a"] = torch.exp(s["g"].double())
    return d


def _exact_delta(s):
    d = _wide(s)
    S, o = s["state_in"].double().mT.contiguous(), torch.empty_like(d["v"])
    for t in range(o.shape[1]):
        S = _walk(d, S, t)[3]
        o[:, t] = s["scale"] * torch.einsum("bhkv,bhk->bhv", S, d["q"][:, t])
    return {"o": o, "state_out": S.mT.contiguous()}


def _exact_delta_backward(s):
    d = _wide(s)
    L, do, sc = d["v"].shape[1], s["grad_o"].double(), s["scale"]
    S = s["state_in"].double().mT.contiguous()
    marks = []
    for t in range(L):              # every 48th state is kept, the ones between are walked again
        if t % 48 == 0:
            marks.append(S)
        S = _walk(d, S, t)[3]
    dq, dk, dv = torch.empty_like(d["q"]), torch.empty_like(d["k"]), torch.empty_like(d["v"])
    dg, db = torch.empty_like(d["beta"]), torch.empty_like(d["beta"])
    lam = s["grad_state_out"].double().mT.contiguous()
    for m in reversed(range(len(marks))):
        S, steps = marks[m], []
        for t in range(48 * m, min(L, 48 * m + 48)):
            steps.append(_walk(d, S, t))
            S = steps[-1][3]
        for t in reversed(range(48 * m, min(L, 48 * m + 48))):
            Sd, miss, u, S1 = steps.pop()
            k = d["k"][:, t]
            lam = lam + sc * torch.einsum("bhk,bhv->bhkv", d["q"][:, t], do[:, t])
            dq[:, t] = sc * torch.einsum("bhkv,bhv->bhk", S1, do[:, t])
            du = torch.einsum("bhkv,bhk->bhv", lam, k)
            dv[:, t] = d["beta"][:, t, :, None] * du
            db[:, t] = (du * miss).sum(-1)
            dk[:, t] = torch.einsum("bhkv,bhv->bhk", lam, u) - torch.einsum("bhkv,bhv->bhk", Sd, dv[:, t])
            lam = lam - torch.einsum("bhk,bhv->bhkv", k, dv[:, t])
            dg[:, t] = (lam * Sd).sum((-1, -2))
            lam = lam * d["a"][:, t, :, None, None]
    Hk = s["q"].shape[2]
    dq, dk = dq.unflatten(2, (Hk, -1)).sum(3), dk.unflatten(2, (Hk, -1)).sum(3)
    return {"grad_q": dq, "grad_k": dk, "grad_v": dv, "grad_g": dg, "grad_beta": db, "grad_state_in": lam.mT.contiguous()}


def _exact_norm(s):
    case = s["case"]
    x = s["x"].double().requires_grad_()
    w, b = s["weight"].double().requires_grad_(), s["bias"].double().requires_grad_()
    gate = s["gate"].double().requires_grad_() if "gate" in s else None
    xs = x.view(case["N"], case["G"], case["M"])
    if case["rms"]:
        xh = xs / torch.sqrt((xs ** 2).mean(2, keepdim=True) + s["eps"])
    else:
        xh = (xs - xs.mean(2, keepdim=True)) / torch.sqrt(xs.var(2, unbiased=False, keepdim=True) + s["eps"])
    y = xh.reshape(case["N"], -1) * w + b
    if case["act"] == "silu":
        y = y * torch.sigmoid(y)
    elif gate is not None:
        y = y * gate * torch.sigmoid(gate)
    if case["op"] == "norm_fwd":
        return y.detach()
    names = [("grad_gate", gate)] if gate is not None else []
    names += [("grad_weight", w), ("grad_bias", b), ("grad_x", x)]
    got = torch.autograd.grad(y, [t for _, t in names], s["grad_y"].double())
    return {n: t for (n, _), t in zip(names, got)}


def _exact_drop(s):
    n, u = s["case"]["n"], np.uint64
    low = u(0xFFFFFFFF)
    i = np.arange((n + 7) // 8, dtype=u)
    x0, x1 = i & low, i >> u(32)
    x2, x3 = np.full_like(i, s["offset"] & 0xFFFFFFFF), np.full_like(i, s["offset"] >> 32)
    k0, k1 = s["seed"] & 0xFFFFFFFF, s["seed"] >> 32
    for _ in range(10):
        p0, p1 = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (p1 >> u(32)) ^ x1 ^ u(k0), p1 & low, (p0 >> u(32)) ^ x3 ^ u(k1), p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    r = np.empty((i.size, 4), np.uint32)
    r[:, 0], r[:, 1], r[:, 2], r[:, 3] = x0, x1, x2, x3
    r = r.view(np.uint16).reshape(-1)[:n]       # little endian: the low half of each word first
    drop = round(s["case"]["p"] * 65536)
    keep = torch.from_numpy((r >= drop).copy()).to(s["x"].device)
    y = torch.where(keep, s["x"].double() * (65536.0 / (65536 - drop)), torch.zeros((), dtype=torch.float64, device=keep.device))
    return y + s["residual"].double() if "residual" in s else y
