"""Workloads of the operators of a selective state space layer: the short causal convolution (prompt,
gradient, single tokens), the selective scan behind it (prompt, training step, single tokens), and the
root-mean-square norm in front of both, which adds the branch to the stream and may write 8-bit values
for the projection (forward, gradient).

Sequences lie one after the other as rows: B sequences of L tokens, or, in the packed cases, B of
unequal lengths (one may be empty) that are named by their offsets.

``run`` computes them with elementary torch operations in float32 where ``own`` is false and with
the library's entry points where it is true; ``exact`` follows the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------ cases

def _conv(name, op, B, L, C, K, type, act="silu", packed=False, fused=True):
    return {"name": name, "op": op, "B": B, "L": L, "C": C, "K": K, "type": type, "act": act, "packed": packed, "fused": fused}


def _scan(name, op, B, L, D, N, type, G=1, gate=True, packed=False):
    return {"name": name, "op": op, "B": B, "L": L, "D": D, "N": N, "G": G, "type": type, "gate": gate, "packed": packed}


def _norm(name, op, rows, M, type, out="same", block=0, wide=False):
    return {"name": name, "op": op, "rows": rows, "M": M, "type": type, "out": out, "block": block, "wide": wide}


def listed():
    return [
        # a serving batch, one token each: the convolution's history moves on by one row
        _conv("conv-step", "conv_fwd", 96, 1, 2048, 4, "bf16"),
        # training forward at the headline forward's 8 x 2048 tokens, channels that are a slice of the projection
        _conv("conv-prompt", "conv_fwd", 8, 2048, 2048, 4, "bf16"),
        # gradient with packed documents of unequal lengths, float32 tensors
        _conv("conv-grad-packed", "conv_bwd", 7, 1021, 768, 4, "fp32", packed=True),
        # one stream generating: latency alone counts
        _scan("scan-step-one", "scan_step", 1, 1, 2048, 16, "bf16"),
        # a serving batch, one token each: every state is read and written once
        _scan("scan-step-batch", "scan_step", 256, 1, 2048, 16, "bf16"),
        # training forward / prompts of a batch
        _scan("scan-prompt", "scan_fwd", 8, 2048, 2048, 16, "bf16"),
        # one long prompt in the 32,768-token chunks of the paper's prefill: few channels, long time axis
        _scan("scan-long", "scan_fwd", 1, 32768, 768, 16, "bf16"),
        # prompts of unequal lengths behind one another, two groups of rows B and C, float32, no gate
        _scan("scan-packed-fp32", "scan_fwd", 6, 333, 520, 24, "fp32", G=2, gate=False, packed=True),
        # a training step: forward with what the gradient needs, then the gradient of everything
        _scan("scan-train", "scan_train", 8, 2048, 1024, 16, "bf16"),
        # the norm in front of a layer for a decoding batch
        _norm("norm-step", "norm_fwd", 96, 768, "bf16"),
        # the same for a prompt, with e4m3 values and a scale per 128 channels for the projection, a float32 stream
        _norm("norm-8bit", "norm_fwd", 32768, 768, "bf16", out="e4m3", block=128, wide=True),
        # its gradient in training
        _norm("norm-grad", "norm_bwd", 32768, 768, "bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["conv_fwd", "conv_fwd", "conv_bwd", "scan_step", "scan_fwd", "scan_fwd", "scan_train", "scan_train", "norm_fwd", "norm_fwd", "norm_bwd"])
    type = rng.choice(["bf16", "bf16", "fp32"])
    widths = [512, 768, 1024, 1280, 2048, 520, 1000, 333]
    if op.startswith("conv"):
        L = _log(rng, 1, 32768)
        B, C = _log(rng, 1, max(1, min(256, 16384 // L))), rng.choice(widths)
        return {"op": op, "B": B, "L": L, "C": C, "K": rng.choice([2, 3, 4, 4]), "type": type, "act": rng.choice(["none", "silu", "silu"]),
                "packed": B > 1 and L > 1 and rng.random() < 0.4, "fused": rng.random() < 0.5}
    if op.startswith("scan"):
        D, N, G = rng.choice(widths), rng.choice([8, 16, 16, 16, 24, 32, 64, 5]), rng.choice([1, 1, 2])
        G = G if D % G == 0 else 1
        if op == "scan_step":
            B, L = _log(rng, 1, 256), rng.choice([1, 1, 2, 4])
        else:
            L = _log(rng, 2, 32768)
            B = _log(rng, 1, max(1, min(32, 16384 // L)))
            cells = 8 * 2048 * 1024 * 16
            while B * L * D * N > cells:            # no more than the largest listed one
                B, L = (B - 1, L) if B > 1 else (B, L // 2)
        return {"op": op, "B": B, "L": L, "D": D, "N": N, "G": G, "type": type, "gate": rng.random() < 0.7,
                "packed": op != "scan_step" and B > 1 and rng.random() < 0.4}
    out = rng.choice(["same", "e4m3"]) if op == "norm_fwd" else "same"
    return {"op": op, "rows": _log(rng, 1, 32768), "M": rng.choice([768, 768, 512, 520, 333]), "type": type, "out": out,
            "block": rng.choice([0, 64, 128]) if out == "e4m3" else 0, "wide": type == "bf16" and rng.random() < 0.5}


# ------------------------------------------------------------------------------------ inputs

def _offsets(case):
    """Where the sequences of a case begin and end: B + 1 whole numbers, the same for every seed."""
    B, L = case["B"], case["L"]
    if not case["packed"]:
        return [i * L for i in range(B + 1)]
    cuts = np.random.RandomState(1000003 * B + L).randint(0, B * L + 1, B - 1)
    if B > 3:
        cuts[1] = cuts[0]           # an empty sequence
    return [0, *sorted(int(c) for c in cuts), B * L]


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
    if op.startswith("norm"):
        rows, M = case["rows"], case["M"]
        stream = torch.float32 if case["wide"] else dt
        s.update(weight=1 + 0.1 * randn(M), eps=1e-5)
        residual = randn(rows, M) * (0.5 + 2 * rand(rows, 1))
        if op == "norm_fwd":
            s.update(x=randn(rows, M).to(dt), residual=residual.to(stream))
        else:                       # the stream that the forward left, what comes back through the norm and past it
            s.update(sum=residual.to(stream), grad_y=randn(rows, M).to(dt), grad_sum=randn(rows, M).to(stream))
        return s
    offsets = _offsets(case)
    B, rows = case["B"], offsets[-1]
    s.update(rows=rows, longest=max(b - a for a, b in zip(offsets, offsets[1:])), offsets=torch.tensor(offsets, device="cuda"))
    if op.startswith("conv"):
        C, K = case["C"], case["K"]
        x = randn(rows, 2 * C if case["fused"] else C).to(dt)[:, :C]          # the front half of (x | z)
        s.update(x=x, weight=randn(C, K) * K ** -0.5, bias=0.1 * randn(C), state_in=randn(B, K - 1, C).to(dt).float())
        if op == "conv_bwd":
            s.update(grad_y=randn(rows, C).to(dt), grad_state_out=randn(B, K - 1, C))
        return s
    D, N, G = case["D"], case["N"], case["G"]
    rank = -(-D // 32 // 8) * 8
    proj = randn(rows, rank + 2 * G * N).to(dt)                             # (step sizes' factor | B | C)
    # rates of -1 to -N as these layers begin with, moved as training does; steps of 0.001 to 0.1 (log-uniform) times e^noise
    step = torch.exp(rand(D) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
    s.update(x=torch.nn.functional.silu(randn(rows, D)).to(dt), dt_raw=(0.5 * randn(rows, D)).to(dt),
             A=-torch.arange(1, N + 1, device="cuda") * torch.exp(0.2 * randn(D, N)),
             Bm=proj[:, rank:rank + G * N], Cm=proj[:, rank + G * N:], skip=1 + 0.1 * randn(D),
             dt_bias=step + torch.log(-torch.expm1(-step)), state_in=0.3 * randn(B, D, N))
    if case["gate"]:
        s["z"] = randn(rows, 2 * D).to(dt)[:, D:]                           # the back half of (x | z)
    if op == "scan_train":
        s.update(grad_y=randn(rows, D).to(dt), grad_state_out=0.1 * randn(B, D, N))
    return s


# ------------------------------------------------------------------------------------ plain forms

def _place(s):
    """Per row: its sequence and its place in it."""
    offsets = s["offsets"]
    row = torch.arange(s["rows"], device=offsets.device)
    seq = torch.searchsorted(offsets, row, right=True) - 1
    return seq, row - offsets[seq]


def _silu(x):
    return x / (1 + torch.exp(-x))


def _silu_slope(x):
    sg = 1 / (1 + torch.exp(-x))
    return sg * (1 + x * (1 - sg))


def _shifted(s, x, n, seq, place):
    """Row t gets row t - n of its sequence, from the history before its first."""
    K = s["case"]["K"]
    rows = torch.arange(x.shape[0], device=x.device)
    if K == 1:
        return x
    old = s["state_in"][seq, (K - 1 - n + place).clamp(0, K - 2)]
    return torch.where((place >= n)[:, None], x[(rows - n).clamp_min(0)], old)


def _conv_pre(s, seq, place):
    K, x = s["case"]["K"], s["x"].float()
    taps = [_shifted(s, x, K - 1 - k, seq, place) for k in range(K)]
    return taps, s["bias"] + sum(t * s["weight"][:, k] for k, t in enumerate(taps))


def _history(s):
    """The last K - 1 rows of (history, sequence): where they are among the rows, or else among the histories."""
    K, offsets = s["case"]["K"], s["offsets"]
    back = torch.arange(K - 1, device=offsets.device)
    length = offsets[1:] - offsets[:-1]
    at = length[:, None] - (K - 1) + back                                   # below 0: before the sequence
    return at, (offsets[:-1, None] + at).clamp_min(0), (K - 1 + at).clamp(0, K - 2)


def _conv_plain(s):
    seq, place = _place(s)
    _, pre = _conv_pre(s, seq, place)
    y = _silu(pre) if s["case"]["act"] == "silu" else pre
    at, row, old = _history(s)
    x = s["x"].float()
    state = torch.where((at >= 0)[..., None], x[row], torch.gather(s["state_in"], 1, old[..., None].expand(-1, -1, x.shape[1])))
    return {"y": y.to(s["dt"]), "state_out": state}


def _conv_plain_backward(s):
    K, C, B = s["case"]["K"], s["case"]["C"], s["case"]["B"]
    seq, place = _place(s)
    taps, pre = _conv_pre(s, seq, place)
    dz = s["grad_y"].float()
    if s["case"]["act"] == "silu":
        dz = dz * _silu_slope(pre)
    dx, dstate = torch.zeros_like(dz), torch.zeros_like(s["state_in"])
    for k in range(K):              # tap k of row t is row t - (K - 1 - k)
        n = K - 1 - k
        term, rows = dz * s["weight"][:, k], torch.arange(s["rows"], device=dz.device)
        dx.index_add_(0, (rows - n).clamp_min(0), torch.where((place >= n)[:, None], term, 0.0))
        before = (place < n).nonzero()[:, 0]
        dstate.index_put_((seq[before], K - 1 - n + place[before]), term[before], accumulate=True)
    at, row, old = _history(s)
    inside = at >= 0
    dx.index_add_(0, row.flatten(), torch.where(inside[..., None], s["grad_state_out"], 0.0).flatten(0, 1))
    dstate.scatter_add_(1, old[..., None].expand(-1, -1, C), torch.where(inside[..., None], 0.0, s["grad_state_out"]))
    return {"grad_x": dx.to(s["dt"]), "grad_weight": torch.stack([(dz * t).sum(0) for t in taps], 1), "grad_bias": dz.sum(0), "grad_state_in": dstate}


def _doubled(a, b, longest):
    """h_t = a_t h_{t-1} + b_t along the first axis, by doubling the stretch that a row sums up (a is 0 at a sequence's first row)."""
    n = 1
    while n < longest:
        b = torch.cat([b[:n], b[n:] + a[n:] * b[:-n]])
        a = torch.cat([a[:n], a[n:] * a[:-n]])
        n *= 2
    return b


def _scan_parts(s):
    case, D = s["case"], s["case"]["D"]
    N, rep = case["N"], D // case["G"]
    seq, place = _place(s)
    first = (place == 0)[:, None, None]
    raw = s["dt_raw"].float() + s["dt_bias"]
    delta = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp_max(20.0))))
    x = s["x"].float()
    Bm, Cm = (s[n].float().unflatten(1, (case["G"], N)).repeat_interleave(rep, 1) for n in ("Bm", "Cm"))       # [rows, D, N]
    a = torch.exp(delta[..., None] * s["A"])
    old = s["state_in"][seq]
    b = (delta * x)[..., None] * Bm
    h = _doubled(torch.where(first, 0.0, a), b + torch.where(first, a * old, 0.0), s["longest"])
    return seq, first, raw, delta, x, Bm, Cm, a, old, h


def _ends(s, h):
    """Each sequence's last row of h, its given state where it has no rows."""
    offsets = s["offsets"]
    return torch.where((offsets[1:] > offsets[:-1])[:, None, None], h[(offsets[1:] - 1).clamp_min(0)], s["state_in"])


def _scan_out(s, x, Cm, h):
    pre = (Cm * h).sum(-1) + s["skip"] * x
    return pre, (pre * _silu(s["z"].float()) if "z" in s else pre).to(s["dt"])


def _scan_plain(s):
    _, _, _, _, x, _, Cm, _, _, h = _scan_parts(s)
    return {"y": _scan_out(s, x, Cm, h)[1], "state_out": _ends(s, h)}


def _scan_plain_train(s):
    case = s["case"]
    seq, first, raw, delta, x, Bm, Cm, a, old, h = _scan_parts(s)
    pre, y = _scan_out(s, x, Cm, h)
    out = {"y": y, "state_out": _ends(s, h)}
    dy = s["grad_y"].float()
    if "z" in s:
        z = s["z"].float()
        out["grad_z"] = (dy * pre * _silu_slope(z)).to(s["dt"])
        dy = dy * _silu(z)
    offsets = s["offsets"]
    full = offsets[1:] > offsets[:-1]
    lam = Cm * dy[..., None]
    lam.index_add_(0, (offsets[1:] - 1).clamp_min(0), torch.where(full[:, None, None], s["grad_state_out"], 0.0))
    after = torch.cat([torch.where(first, 0.0, a)[1:], torch.zeros_like(a[:1])])
    lam = _doubled(after.flip(0), lam.flip(0), s["longest"]).flip(0)
    w = a * torch.where(first, old, torch.cat([h[:1], h[:-1]]))
    G, N = case["G"], case["N"]
    flow, drift = (lam * Bm).sum(-1), lam * w
    draw_ = (drift * s["A"]).sum(-1) + flow * x
    draw_ = draw_ / (1 + torch.exp(-raw))
    out.update(grad_x=(delta * flow + s["skip"] * dy).to(s["dt"]), grad_dt=draw_.to(s["dt"]), grad_A=(drift * delta[..., None]).sum(0),
               grad_B=(lam * (delta * x)[..., None]).unflatten(1, (G, -1)).sum(2).flatten(1).to(s["dt"]),
               grad_C=(h * dy[..., None]).unflatten(1, (G, -1)).sum(2).flatten(1).to(s["dt"]),
               grad_skip=(dy * x).sum(0), grad_dt_bias=draw_.sum(0),
               grad_state_in=torch.where(full[:, None, None], (a * lam)[offsets[:-1].clamp_max(s["rows"] - 1)], s["grad_state_out"]))
    return out


def _step_plain(s):
    case = s["case"]
    B, D, N, rep = case["B"], case["D"], case["N"], case["D"] // case["G"]
    raw = s["dt_raw"].float() + s["dt_bias"]
    delta = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp_max(20.0)))).view(B, -1, D)
    x = s["x"].float().view(B, -1, D)
    Bm, Cm = (s[n].float().view(B, -1, case["G"], N).repeat_interleave(rep, 2) for n in ("Bm", "Cm"))
    h, outs = s["state_in"], []
    for t in range(x.shape[1]):
        h = torch.exp(delta[:, t, :, None] * s["A"]) * h + (delta[:, t] * x[:, t])[..., None] * Bm[:, t]
        outs.append((h * Cm[:, t]).sum(-1) + s["skip"] * x[:, t])
    y = torch.stack(outs, 1).view(-1, D)
    return {"y": (y * _silu(s["z"].float()) if "z" in s else y).to(s["dt"]), "state_out": h}


def _norm_plain(s):
    case = s["case"]
    total = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    v = total.float()
    y = v * (v.square().mean(1, keepdim=True) + s["eps"]).rsqrt() * s["weight"]
    if case["out"] == "same":
        return {"sum": total, "y": y.to(s["dt"])}
    M, block = case["M"], case["block"] or case["M"]
    parts = torch.nn.functional.pad(y, (0, -M % block)).unflatten(1, (-1, block))
    scale = parts.abs().amax(2).clamp_min(1e-30) / E4M3_MAX
    return {"sum": total, "y": (parts / scale[..., None]).flatten(1)[:, :M].to(torch.float8_e4m3fn), "scale": scale}


def _norm_plain_backward(s):
    v, dy = s["sum"].float(), s["grad_y"].float()
    rstd = (v.square().mean(1, keepdim=True) + s["eps"]).rsqrt()
    vh = v * rstd
    d = dy * s["weight"]
    dx = rstd * (d - vh * (d * vh).mean(1, keepdim=True)) + s["grad_sum"].float()
    out = {"grad_residual": dx.to(s["sum"].dtype), "grad_weight": (dy * vh).sum(0)}
    if s["case"]["wide"]:
        out["grad_x"] = dx.to(s["dt"])
    return out


# ------------------------------------------------------------------------------------ the library's calls

def _flags(s):
    from paper_2604_04250_b200 import binding as cb
    return cb.CAWN_FLAG_INPUT_BF16 | cb.CAWN_FLAG_OUTPUT_BF16 if s["dt"] == torch.bfloat16 else 0


def _new(x, *shape, dtype=None):
    return torch.empty(shape or x.shape, dtype=dtype or x.dtype, device=x.device)


def _own_conv(s):
    from paper_2604_04250_b200 import binding as cb
    case, x = s["case"], s["x"]
    packed = case["packed"]
    act = cb.CAWN_CONV_ACT_SILU if case["act"] == "silu" else cb.CAWN_CONV_ACT_NONE
    prm = cb.make_conv_params(case["B"], s["longest"], case["C"], case["K"], act=act, flags=_flags(s), x_stride=x.stride(0), rows=s["rows"] if packed else 0)
    offsets = s["offsets"] if packed else None
    if case["op"] == "conv_fwd":
        out = {"y": _new(x), "state_out": _new(s["state_in"])}
        cb.cawn_short_conv_fwd(prm, x, s["weight"], out["y"], bias=s["bias"], state_in=s["state_in"], state_out=out["state_out"], offsets=offsets)
        return out
    if "workspace" not in s:        # kept by the program for its later calls, as all of the library's workspaces
        s["workspace"] = cb.new_conv_workspace(prm)
    out = {"grad_x": _new(x), "grad_weight": _new(s["weight"]), "grad_bias": _new(s["bias"]), "grad_state_in": _new(s["state_in"])}
    cb.cawn_short_conv_bwd(prm, x, s["weight"], s["grad_y"], out["grad_x"], s["workspace"], bias=s["bias"], state_in=s["state_in"], offsets=offsets,
                           grad_state_out=s["grad_state_out"], grad_weight=out["grad_weight"], grad_bias=out["grad_bias"], grad_state_in=out["grad_state_in"])
    return out


def _own_scan(s):
    from paper_2604_04250_b200 import binding as cb
    case, x, z = s["case"], s["x"], s.get("z")
    op, packed = case["op"], case["packed"]
    prm = cb.make_scan_params(case["B"], s["longest"], case["D"], case["N"], G=case["G"], softplus=True, flags=_flags(s), x_stride=x.stride(0),
                              dt_stride=s["dt_raw"].stride(0), b_stride=s["Bm"].stride(0), c_stride=s["Cm"].stride(0),
                              z_stride=0 if z is None else z.stride(0), rows=s["rows"] if packed else 0)
    out = {"y": _new(x), "state_out": _new(s["state_in"])}
    args = (x, s["dt_raw"], s["A"], s["Bm"], s["Cm"])
    same = {"skip": s["skip"], "dt_bias": s["dt_bias"], "z": z, "state_in": s["state_in"]}
    if op == "scan_step":
        cb.cawn_selective_scan_step(prm, *args, out["y"], state_out=out["state_out"], **same)
        return out
    same["offsets"] = s["offsets"] if packed else None
    if "workspace" not in s:
        s["workspace"] = cb.new_scan_workspace(prm, cb.CAWN_SCAN_FWD)
        if op == "scan_train":
            s["workspace_bwd"], s["checkpoints"] = cb.new_scan_workspace(prm, cb.CAWN_SCAN_BWD), cb.new_scan_workspace(prm, cb.CAWN_SCAN_CHECKPOINTS)
    cb.cawn_selective_scan_fwd(prm, *args, out["y"], s["workspace"], state_out=out["state_out"], checkpoints=s.get("checkpoints"), **same)
    if op == "scan_train":
        out.update(grad_x=_new(x), grad_dt=_new(x), grad_A=_new(s["A"]), grad_B=_new(x, *s["Bm"].shape), grad_C=_new(x, *s["Cm"].shape),
                   grad_skip=_new(s["skip"]), grad_dt_bias=_new(s["dt_bias"]), grad_state_in=_new(s["state_in"]))
        if z is not None:
            out["grad_z"] = _new(x)
        cb.cawn_selective_scan_bwd(prm, *args, s["grad_y"], out["grad_x"], out["grad_dt"], out["grad_A"], out["grad_B"], out["grad_C"], s["workspace_bwd"],
                                   checkpoints=s["checkpoints"], grad_state_out=s["grad_state_out"], grad_skip=out["grad_skip"],
                                   grad_dt_bias=out["grad_dt_bias"], grad_z=out.get("grad_z"), grad_state_in=out["grad_state_in"], **same)
    return out


def _own_norm(s):
    from paper_2604_04250_b200 import binding as cb
    case = s["case"]
    rows, M = case["rows"], case["M"]
    e4m3 = case["out"] == "e4m3"
    prm = cb.make_residual_norm_params(rows, M, eps=s["eps"], out=cb.CAWN_NORM_OUT_E4M3 if e4m3 else cb.CAWN_NORM_OUT_SAME, scale_block=case["block"],
                                       stream_float=case["wide"], flags=_flags(s))
    if case["op"] == "norm_fwd":
        out = {"sum": _new(s["residual"]), "y": _new(s["x"], dtype=torch.float8_e4m3fn if e4m3 else None)}
        if e4m3:
            out["scale"] = _new(s["weight"], rows, -(-M // (case["block"] or M)))
        cb.cawn_residual_norm_fwd(prm, s["x"], out["y"], residual=s["residual"], weight=s["weight"], sum_out=out["sum"], scales=out.get("scale"))
        return out
    if "workspace" not in s:
        s["workspace"] = cb.new_residual_norm_workspace(prm)
    out = {"grad_residual": _new(s["sum"]), "grad_weight": _new(s["weight"])}
    if case["wide"]:
        out["grad_x"] = _new(s["grad_y"])
    cb.cawn_residual_norm_bwd(prm, s["sum"], s["grad_y"], workspace=s["workspace"], weight=s["weight"], grad_sum=s["grad_sum"],
                              grad_residual=out["grad_residual"], grad_x=out.get("grad_x"), grad_weight=out["grad_weight"])
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_conv(state) if op.startswith("conv") else _own_scan(state) if op.startswith("scan") else _own_norm(state)
    return {"conv_fwd": _conv_plain, "conv_bwd": _conv_plain_backward, "scan_step": _step_plain, "scan_fwd": _scan_plain,
            "scan_train": _scan_plain_train, "norm_fwd": _norm_plain, "norm_bwd": _norm_plain_backward}[op](state)


# ------------------------------------------------------------------------------------ work

def work(case):
    e = 2 if case["type"] == "bf16" else 4
    op = case["op"]
    if op.startswith("conv"):
        n, K = case["B"] * case["L"] * case["C"], case["K"]
        state = case["B"] * (K - 1) * case["C"] * 4
        if op == "conv_fwd":
            return {"bytes": 2 * n * e + 2 * state + case["C"] * (K + 1) * 4, "flops": n * (2 * K + 4)}
        return {"bytes": 3 * n * e + 3 * state + 2 * case["C"] * (K + 1) * 4, "flops": n * (6 * K + 12)}
    if op.startswith("scan"):
        rows, D, N = case["B"] * case["L"], case["D"], case["N"]
        row = D * e * (3 + case["gate"]) + 2 * case["G"] * N * e        # x, dt, y (z), B, C
        state, fixed = case["B"] * D * N * 4, D * (N + 2) * 4
        if op != "scan_train":      # a decay's product and exponential, the term, the state, the read-out
            return {"bytes": rows * row + 2 * state + fixed, "flops": rows * D * (7 * N + 15)}
        back = D * e * (5 + 2 * case["gate"]) + 4 * case["G"] * N * e   # x, dt, dy (z) in, and the gradients of x, dt (z); B, C and theirs
        return {"bytes": rows * (row + back) + 5 * state + 3 * fixed, "flops": rows * D * (27 * N + 40)}
    n, wide = case["rows"] * case["M"], 4 if case["wide"] else e
    if op == "norm_fwd":
        block = case["block"] or case["M"]
        out = n * e if case["out"] == "same" else n + 4 * case["rows"] * -(-case["M"] // block)
        return {"bytes": n * (e + 2 * wide) + out + case["M"] * 4, "flops": n * 6}
    return {"bytes": n * (e + 3 * wide + (e if case["wide"] else 0)) + case["M"] * 8, "flops": n * 12}


# ------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("conv"):
        return _exact_conv(s)
    if op.startswith("scan"):
        return _exact_scan(s)
    return _exact_norm(s)


def _exact_conv(s):
    case, K = s["case"], s["case"]["K"]
    offsets = s["offsets"].tolist()
    names = ("x", "weight", "bias", "state_in")
    x, w, b, old = (s[n].double().requires_grad_(case["op"] == "conv_bwd") for n in names)
    ys, states = [], []
    for i in range(case["B"]):      # a sequence at a time, its history in front of it
        whole = torch.cat([old[i], x[offsets[i]:offsets[i + 1]]])
        n = offsets[i + 1] - offsets[i]
        pre = b + sum(whole[k:k + n] * w[:, k] for k in range(K))
        ys.append(pre * torch.sigmoid(pre) if case["act"] == "silu" else pre)
        states.append(whole[n:])
    y, state = torch.cat(ys), torch.stack(states)
    if case["op"] == "conv_fwd":
        return {"y": y, "state_out": state}
    got = torch.autograd.grad([y, state], [x, w, b, old], [s["grad_y"].double(), s["grad_state_out"].double()], allow_unused=True)
    return {"grad_" + n: torch.zeros_like(t) if g is None else g for n, t, g in zip(names, (x, w, b, old), got)}


def _exact_scan(s):
    case = s["case"]
    B, D, N, G, op = case["B"], case["D"], case["N"], case["G"], case["op"]
    train = op == "scan_train"
    offsets = s["offsets"].tolist()
    lengths = [b - a for a, b in zip(offsets, offsets[1:])]
    order = sorted(range(B), key=lambda i: -lengths[i])         # the longest first: those still running are the first ones
    begin = torch.tensor([offsets[i] for i in order], device="cuda")
    d = {n: s[n].double() for n in ("x", "A", "skip", "dt_bias", "state_in")}
    raw = s["dt_raw"].double() + d["dt_bias"]
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    Bm, Cm = s["Bm"].double().view(-1, G, 1, N), s["Cm"].double().view(-1, G, 1, N)
    gate = None if "z" not in s else s["z"].double() * torch.sigmoid(s["z"].double())
    grouped = lambda v: v.view(v.shape[0], G, D // G, N)
    h = grouped(d["state_in"][order].clone())
    A = d["A"].view(G, D // G, N)
    pre, kept = torch.zeros_like(d["x"]), []
    live = [sum(n > t for n in lengths) for t in range(max(lengths))]
    for t in range(max(lengths)):
        m = live[t]
        at = begin[:m] + t
        a = torch.exp(delta[at].view(m, G, -1, 1) * A)
        if train:
            kept.append(h[:m].clone())
        new = a * h[:m] + (delta[at] * d["x"][at]).view(m, G, -1, 1) * Bm[at]
        h[:m] = new
        pre[at] = (new * Cm[at]).sum(-1).view(m, D) + d["skip"] * d["x"][at]
    back = torch.empty(B, dtype=torch.long, device="cuda")
    back[torch.tensor(order, device="cuda")] = torch.arange(B, device="cuda")
    out = {"y": pre if gate is None else pre * gate, "state_out": h.view(B, D, N)[back]}
    if not train:
        return out
    dy = s["grad_y"].double()
    if gate is not None:
        z = s["z"].double()
        out["grad_z"] = dy * pre * torch.sigmoid(z) * (1 + z * (1 - torch.sigmoid(z)))
        dy = dy * gate
    lam = grouped(s["grad_state_out"].double()[order].clone())
    gx, gdt = d["skip"] * dy, torch.zeros_like(raw)
    gA, gB, gC = torch.zeros_like(A), torch.zeros(s["rows"], G, N, device="cuda", dtype=torch.float64), torch.zeros(s["rows"], G, N, device="cuda", dtype=torch.float64)
    for t in reversed(range(max(lengths))):
        m = live[t]
        at = begin[:m] + t
        de, xv, dyv = (v[at].view(m, G, -1, 1) for v in (delta, d["x"], dy))
        a, old = torch.exp(de * A), kept.pop()
        now = a * old + de * xv * Bm[at]
        cur = lam[:m] + Cm[at] * dyv
        gC[at], gB[at] = (now * dyv).sum(2), (cur * de * xv).sum(2)
        through = cur * a * old
        flow = (cur * Bm[at]).sum(-1).view(m, D)
        gx[at] += delta[at] * flow
        gdt[at] = (through * A).sum(-1).view(m, D) + flow * d["x"][at]
        gA += (through * de).sum(0)
        lam[:m] = cur * a
    gdt = gdt * torch.sigmoid(raw)
    out.update(grad_x=gx, grad_dt=gdt, grad_A=gA.view(D, N), grad_B=gB.flatten(1), grad_C=gC.flatten(1), grad_skip=(dy * d["x"]).sum(0),
               grad_dt_bias=gdt.sum(0), grad_state_in=lam.reshape(B, D, N)[back])
    return out


def _exact_norm(s):
    case = s["case"]
    w = s["weight"].double().requires_grad_()
    if case["op"] == "norm_fwd":
        total = (s["x"].double() + s["residual"].double()).to(s["residual"].dtype)         # the stream holds its own type
    else:
        total = s["sum"]
    v = total.double().requires_grad_()
    y = v / torch.sqrt((v ** 2).mean(1, keepdim=True) + s["eps"]) * w
    if case["op"] == "norm_bwd":
        gv, gw = torch.autograd.grad(y, [v, w], s["grad_y"].double())
        gv = gv + s["grad_sum"].double()
        return {"grad_residual": gv, "grad_weight": gw} | ({"grad_x": gv} if case["wide"] else {})
    y = y.detach()
    if case["out"] == "same":
        return {"sum": total, "y": y}
    M = case["M"]
    scales, parts = [], []
    for c in range(0, M, case["block"] or M):
        part = y[:, c:c + (case["block"] or M)]
        scales.append(part.abs().max(1).values.clamp(min=1e-30) / E4M3_MAX)
        parts.append((part / scales[-1][:, None]).to(torch.float8_e4m3fn))
    return {"sum": total, "y": torch.cat([p.double() for p in parts], 1), "scale": torch.stack(scales, 1)}
