"""Cases of the operators of a selective memory and its training step: the layer norm with the residual's addition, the
short causal convolution over channels, the selective scan (a diagonal state space whose step, input and output maps
come with every token), and the norm of all gradients with its clipping.

`own` False: the operators written out with elementary torch operations in 32 bits.  `own` True: the calls of this
package.  The layer norm's tensors are (outer, channels, inner): inner = 1 is a token-major row, inner > 1 a
channels-first field.  Convolution and scan work on token-major tensors (batch, length, channels); a ragged batch has a
length of its own for each entry, and what lies behind it is not used (outputs there are zero).
"""
import math

import torch

own = False

EPS = 1e-5
CLIP_EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "c64": 8}
CHUNK = 64                      # steps of the plain scan that are in memory at once


def listed():
    return [
        # one new frame of four running rollouts: latency
        {"name": "layer_norm_step", "op": "norm", "type": "bf16", "outer": 4, "channels": 2048, "inner": 1, "residual": True},
        # a training step on token-major latents
        {"name": "layer_norm_train_rows", "op": "norm_train", "type": "bf16", "outer": 16384, "channels": 2048, "inner": 1,
         "residual": True},
        # a training step on channels-first fields: width 20, a grid with a time axis of 30, rows off a vector's multiple
        {"name": "layer_norm_train_field", "op": "norm_train", "type": "f32", "outer": 1, "channels": 20,
         "inner": 64 * 64 * 32 * 30, "residual": False},
        # one new frame: the convolution's window moves on by one
        {"name": "conv_step", "op": "conv", "type": "bf16", "batch": 4, "length": 1, "channels": 4096, "width": 4,
         "ragged": False, "strided": True},
        # a training step; the input is one half of a projection's output
        {"name": "conv_train", "op": "conv_train", "type": "bf16", "batch": 4, "length": 4096, "channels": 4096, "width": 4,
         "ragged": False, "strided": True},
        # one new frame of four rollouts: one step of the scan
        {"name": "scan_step", "op": "scan", "type": "bf16", "batch": 4, "length": 1, "channels": 4096, "states": 16,
         "groups": 1, "gated": True, "ragged": False, "strided": True},
        # one long history read in at once: a single sequence
        {"name": "scan_history", "op": "scan", "type": "bf16", "batch": 1, "length": 16384, "channels": 4096, "states": 16,
         "groups": 1, "gated": True, "ragged": False, "strided": True},
        # a training step on full sequences
        {"name": "scan_train", "op": "scan_train", "type": "bf16", "batch": 4, "length": 2048, "channels": 4096, "states": 16,
         "groups": 1, "gated": True, "ragged": False, "strided": True},
        # a training step on a ragged batch, sizes that fill no tile, two groups of channels, no output gate
        {"name": "scan_train_ragged", "op": "scan_train", "type": "f32", "batch": 3, "length": 1027, "channels": 1002,
         "states": 12, "groups": 2, "gated": False, "ragged": True, "strided": False},
        # the gradients of a small spectral network: many small tensors
        {"name": "clip_network", "op": "clip", "set": "fno", "type": "f32", "layers": 4, "width": 16, "modes": 512},
        # those of a selective memory's layers in 16 bits
        {"name": "clip_memory", "op": "clip", "set": "memory", "type": "bf16", "layers": 5, "width": 2048, "modes": 0},
        # those of a large four-dimensional spectral network: half a gigabyte a layer
        {"name": "clip_large", "op": "clip", "set": "fno", "type": "f32", "layers": 2, "width": 16, "modes": 32 * 32 * 32 * 8},
    ]


def _spread(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_train", "conv", "conv_train", "scan", "scan", "scan_train", "scan_train", "clip"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_train"):
        if rng.random() < 0.4:                                    # channels-first fields
            c, outer = rng.choice([4, 8, 16, 20, 32, 64, 128]), rng.choice([1, 2, 4])
            inner = _spread(rng, 1024, (1 << 26) // (c * outer))
        else:
            c, inner = _spread(rng, 64, 8192), 1
            outer = _spread(rng, 1, max(1, (1 << 25) // c))
        return {"op": op, "type": kind, "outer": outer, "channels": c, "inner": inner, "residual": rng.random() < 0.5}
    if op in ("conv", "conv_train"):
        c = _spread(rng, 64, 8192)
        n = _spread(rng, 1, 16384)
        return {"op": op, "type": kind, "batch": _spread(rng, 1, max(1, min(32, (1 << 25) // (c * n)))), "length": min(n, (1 << 25) // c),
                "channels": c, "width": rng.choice([2, 3, 4, 4]), "ragged": rng.random() < 0.3, "strided": rng.random() < 0.5}
    if op in ("scan", "scan_train"):
        groups = rng.choice([1, 1, 1, 2, 4])
        c = _spread(rng, 64, 8192) // groups * groups
        states = rng.choice([4, 8, 12, 16, 16, 16, 32])
        most = (1 << 24) * 16 // max(16, states) * (2 if op == "scan" else 1)
        n = min(_spread(rng, 1, 16384), most // c)
        return {"op": op, "type": kind, "batch": _spread(rng, 1, max(1, min(32, most // (c * n)))), "length": n, "channels": c,
                "states": states, "groups": groups, "gated": rng.random() < 0.7, "ragged": rng.random() < 0.3,
                "strided": rng.random() < 0.5}
    if rng.random() < 0.5:
        width = rng.choice([8, 16, 20])
        return {"op": "clip", "set": "fno", "type": "f32", "layers": rng.randint(1, 6), "width": width,
                "modes": _spread(rng, 32, 65536)}
    return {"op": "clip", "set": "memory", "type": kind, "layers": rng.randint(1, 5), "width": _spread(rng, 65, 2048), "modes": 0}


# ---------------------------------------------------------------- inputs
def _tensors(case):
    """Shapes and types of one network's gradients."""
    w, kind = case["width"], case["type"]
    if case["set"] == "fno":                     # lifting, per layer the modes' weights and the bypass, projection
        out = [((w, 3), "f32"), ((w,), "f32")]
        for _ in range(case["layers"]):
            out += [((w, w, case["modes"]), "c64"), ((w, w), "f32")]
        return out + [((1, w), "f32"), ((1,), "f32")]
    out = []
    for _ in range(case["layers"]):              # projections in their type, the rest in 32 bits
        h, r = 2 * w, max(1, w // 16)
        out += [((2 * h, w), kind), ((r + 32, h), kind), ((h, r), kind), ((w, h), kind), ((h, 4), "f32"), ((h,), "f32"),
                ((h, 16), "f32"), ((h,), "f32"), ((h,), "f32"), ((w,), "f32"), ((w,), "f32")]
    return out


def _token_rows(rn, case, dt, part=0):
    """(batch, length, channels); strided: one half of a projection's output of twice the channels."""
    b, n, c = case["batch"], case["length"], case["channels"]
    if not case["strided"]:
        return rn(b, n, c).to(dt)
    return rn(b, n, 2 * c).to(dt)[..., part * c:(part + 1) * c]


def _lengths(case, gen):
    if not case["ragged"]:
        return None
    return torch.randint(0, case["length"] + 1, (case["batch"],), device="cuda", generator=gen, dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    ru = lambda *s: torch.rand(s, device="cuda", generator=gen)
    st = {"case": dict(case)}
    op = case["op"]
    if op == "clip":
        grads = []
        for shape, kind in _tensors(case):
            if kind == "c64":
                grads.append(torch.view_as_complex(rn(*shape, 2)))
            else:
                grads.append((3.0 * rn(*shape)).to(TYPES[kind]))
        st["grads"], st["max_norm"] = grads, 1.0
        if own:
            from paper_2607_14394_b200 import GradNorm
            # clipped copies: the gradients as they were stay for another use
            st["out"] = [torch.empty_like(g) for g in grads]
            st["plan"] = GradNorm(grads, out=st["out"])
        return st
    dt = TYPES[case["type"]]
    if op in ("norm", "norm_train"):
        shape = (case["outer"], case["channels"], case["inner"])
        shape = shape[:2] if case["inner"] == 1 else shape
        # latents with a common offset: their mean is not small next to their spread
        st["x"] = (0.7 + rn(*shape)).to(dt)
        st["residual"] = (2.0 * rn(*shape)).to(dt) if case["residual"] else None
        st["weight"], st["bias"] = 1.0 + 0.2 * rn(case["channels"]), 0.3 * rn(case["channels"])
        if op == "norm_train":
            st["grad_y"] = rn(*shape).to(dt)
            st["grad_s"] = rn(*shape).to(dt) if case["residual"] else None
        if own:
            from paper_2607_14394_b200 import LayerNorm
            st["plan"] = LayerNorm(shape, 1, dtype=dt, eps=EPS)
        return st
    b, n, c = case["batch"], case["length"], case["channels"]
    st["x"] = _token_rows(rn, case, dt)
    st["lengths"] = _lengths(case, gen)
    if op in ("conv", "conv_train"):
        k = case["width"]
        st["weight"], st["bias"] = rn(c, k) / k ** 0.5, 0.2 * rn(c)
        st["state"] = rn(b, k - 1, c).to(dt)
        if op == "conv_train":
            st["grad_y"], st["grad_state"] = rn(b, n, c).to(dt), rn(b, k - 1, c).to(dt)
        if own:
            from paper_2607_14394_b200 import CausalConv
            st["plan"] = CausalConv((b, n, c), k, dtype=dt, activation="silu")
        return st
    s, g = case["states"], case["groups"]
    # steps of 0.001 to 0.1 around each channel's own, decays of 1 to `states` a unit of time
    step = torch.exp(math.log(1e-3) + (math.log(0.1) - math.log(1e-3)) * ru(c))
    st["dt_bias"] = step + torch.log(-torch.expm1(-step))
    st["dt"] = (0.5 * rn(b, n, c)).to(dt)
    st["A"] = -(torch.arange(1, s + 1, device="cuda", dtype=torch.float32) * torch.exp(0.1 * rn(c, s)))
    both = rn(b, n, 2 * g * s).to(dt)                             # one projection gives both maps
    st["B"], st["C"] = both[..., :g * s].unflatten(-1, (g, s)), both[..., g * s:].unflatten(-1, (g, s))
    st["D"] = 1.0 + 0.1 * rn(c)
    st["z"] = _token_rows(rn, case, dt, 1) if case["gated"] else None
    st["h0"] = rn(b, c, s)
    if op == "scan_train":
        st["grad_y"], st["grad_last"] = rn(b, n, c).to(dt), rn(b, c, s)
    if own:
        from paper_2607_14394_b200 import SelectiveScan
        st["plan"] = SelectiveScan((b, n, c), s, groups=g, dtype=dt, softplus=True)
        if op == "scan_train":
            st["checkpoints"] = st["plan"].new_checkpoints()
    return st


# ---------------------------------------------------------------- plain forms, in 32 bits
def _plain_norm(st):
    case, dt = st["case"], TYPES[st["case"]["type"]]
    s = st["x"].float()
    if st["residual"] is not None:
        s = s + st["residual"].float()
    view = (1, -1) + (1,) * (s.dim() - 2)
    w, b = st["weight"].view(view), st["bias"].view(view)
    d = s - s.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    n = d * rstd
    out = {"y": (n * w + b).to(dt)}
    if st["residual"] is not None:
        out["s"] = s.to(dt)
    if case["op"] == "norm":
        return out
    gy = st["grad_y"].float()
    gn = w * gy
    gx = rstd * (gn - gn.mean(dim=1, keepdim=True) - n * (gn * n).mean(dim=1, keepdim=True))
    if st["residual"] is not None:
        gx = gx + st["grad_s"].float()
    rest = [d for d in range(s.dim()) if d != 1]
    out.update(grad_x=gx.to(dt), grad_weight=(gy * n).sum(dim=rest), grad_bias=gy.sum(dim=rest))
    return out


def _keep(st):
    """(batch, length, 1) of the steps that exist, or None."""
    if st["lengths"] is None:
        return None
    steps = torch.arange(st["x"].shape[1], device="cuda")
    return (steps[None, :] < st["lengths"][:, None])[..., None]


def _plain_conv(st):
    case, dt = st["case"], TYPES[st["case"]["type"]]
    k, n, keep = case["width"], case["length"], _keep(st)
    x = st["x"].float()
    if keep is not None:
        x = torch.where(keep, x, torch.zeros_like(x))
    w = st["weight"]
    u = torch.cat([st["state"].float(), x], dim=1)                # u[:, t + j] is tap j of step t
    pre = st["bias"] + sum(w[:, j] * u[:, j:j + n] for j in range(k))
    sig = torch.sigmoid(pre)
    y = pre * sig
    if keep is not None:
        y = torch.where(keep, y, torch.zeros_like(y))
    if st["lengths"] is None:
        last = u[:, n:]
    else:
        at = st["lengths"].long()[:, None] + torch.arange(k - 1, device="cuda")
        last = torch.gather(u, 1, at[..., None].expand(-1, -1, u.shape[2]))
    out = {"y": y.to(dt), "state": last.to(dt)}
    if case["op"] == "conv":
        return out
    gp = st["grad_y"].float() * (sig + pre * sig * (1 - sig))
    if keep is not None:
        gp = torch.where(keep, gp, torch.zeros_like(gp))
    gu = torch.zeros_like(u)
    for j in range(k):
        gu[:, j:j + n] += w[:, j] * gp
    if st["lengths"] is None:
        gu[:, n:] += st["grad_state"].float()
    else:
        gu.scatter_add_(1, at[..., None].expand(-1, -1, u.shape[2]), st["grad_state"].float())
    gx = gu[:, k - 1:]
    if keep is not None:
        gx = torch.where(keep, gx, torch.zeros_like(gx))
    gw = torch.stack([(gp * u[:, j:j + n]).sum(dim=(0, 1)) for j in range(k)], dim=1)
    out.update(grad_x=gx.to(dt), grad_state=gu[:, :k - 1].to(dt), grad_weight=gw, grad_bias=gp.sum(dim=(0, 1)))
    return out


def _prefix(a, u, h0):
    """h_t = a_t h_{t-1} + u_t along dimension 1, in log2(length) doublings of whole-tensor operations."""
    h, d, n = torch.cat([a[:, :1] * h0[:, None] + u[:, :1], u[:, 1:]], dim=1), 1, a.shape[1]
    while d < n:
        h = torch.cat([h[:, :d], h[:, d:] + a[:, d:] * h[:, :-d]], dim=1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], dim=1)
        d *= 2
    return h


def _plain_scan(st):
    case, dt = st["case"], TYPES[st["case"]["type"]]
    n, c, s, g = case["length"], case["channels"], case["states"], case["groups"]
    keep, A, b = _keep(st), st["A"], case["batch"]
    rows = lambda m, t: m[:, t].float().repeat_interleave(c // g, dim=2)             # (batch, steps, channels, states)

    def terms(t):
        raw = st["dt"][:, t].float() + st["dt_bias"]
        x, delta = st["x"][:, t].float(), raw.clamp_min(0) + torch.log1p(torch.exp(-raw.abs()))
        if keep is not None:
            x, delta = torch.where(keep[:, t], x, torch.zeros_like(x)), torch.where(keep[:, t], delta, torch.zeros_like(x))
        return raw, x, delta, torch.exp(delta[..., None] * A), rows(st["B"], t), rows(st["C"], t)

    h0, h, starts, ys = st["h0"], st["h0"], [], []
    for t0 in range(0, n, CHUNK):
        t = slice(t0, min(n, t0 + CHUNK))
        raw, x, delta, a, B, C = terms(t)
        starts.append(h)
        hs = _prefix(a, (delta * x)[..., None] * B, h)
        h = hs[:, -1].contiguous()
        y = (hs * C).sum(dim=3) + st["D"] * x
        if st["z"] is not None:
            z = st["z"][:, t].float()
            y = y * z * torch.sigmoid(z)
        ys.append(y if keep is None else torch.where(keep[:, t], y, torch.zeros_like(y)))
    out = {"y": torch.cat(ys, dim=1).to(dt), "h_last": h}
    if case["op"] == "scan":
        return out
    del ys
    carry, grads = st["grad_last"], {k: [] for k in ("x", "dt", "B", "C", "z")}
    gA, gD, gbias = torch.zeros_like(A), torch.zeros_like(st["D"]), torch.zeros_like(st["D"])
    per_group = lambda m: m.view(m.shape[0], m.shape[1], g, c // g, s).sum(dim=3)
    for i in reversed(range(len(starts))):
        t = slice(i * CHUNK, min(n, (i + 1) * CHUNK))
        raw, x, delta, a, B, C = terms(t)
        hs = _prefix(a, (delta * x)[..., None] * B, starts[i])
        gy = st["grad_y"][:, t].float()
        if keep is not None:
            gy = torch.where(keep[:, t], gy, torch.zeros_like(gy))
        if st["z"] is not None:
            z = st["z"][:, t].float()
            sig = torch.sigmoid(z)
            core = (hs * C).sum(dim=3) + st["D"] * x
            grads["z"].append(gy * core * (sig + z * sig * (1 - sig)))
            gy = gy * z * sig
        # gradient of every state: what its own output and the next state pass back
        back = torch.cat([torch.ones_like(a[:, :1]), a[:, 1:].flip(1)], dim=1)
        gh = _prefix(back, (gy[..., None] * C).flip(1), carry).flip(1)
        before = torch.cat([starts[i][:, None], hs[:, :-1]], dim=1)
        ga = gh * before * a
        through = (gh * B).sum(dim=3)
        gdelta = (ga * A).sum(dim=3) + through * x
        graw = gdelta * torch.sigmoid(raw)
        gx = through * delta + gy * st["D"]
        if keep is not None:
            graw, gx = torch.where(keep[:, t], graw, torch.zeros_like(gx)), torch.where(keep[:, t], gx, torch.zeros_like(gx))
        grads["x"].append(gx)
        grads["dt"].append(graw)
        grads["B"].append(per_group(gh * (delta * x)[..., None]))
        grads["C"].append(per_group(hs * gy[..., None]))
        gA += (ga * delta[..., None]).sum(dim=(0, 1))
        gD += (gy * x).sum(dim=(0, 1))
        gbias += graw.sum(dim=(0, 1))
        carry = a[:, 0] * gh[:, 0]
    for k, v in grads.items():
        if v:
            out["grad_" + k] = torch.cat(v[::-1], dim=1).to(dt)
    out.update(grad_A=gA, grad_D=gD, grad_dt_bias=gbias, grad_h0=carry)
    return out


def _real(t):
    return torch.view_as_real(t) if t.is_complex() else t


def _plain_clip(st):
    parts = [_real(g).float() for g in st["grads"]]
    norm = torch.sqrt(torch.stack([(p * p).sum() for p in parts]).sum())
    coef = (st["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    return {"norm": norm, "grads": [(p * coef).to(_real(g).dtype) for p, g in zip(parts, st["grads"])]}


def _plain(st):
    op = st["case"]["op"]
    if op in ("norm", "norm_train"):
        return _plain_norm(st)
    if op in ("conv", "conv_train"):
        return _plain_conv(st)
    return _plain_clip(st) if op == "clip" else _plain_scan(st)


def _framework(st):
    op, plan = st["case"]["op"], st["plan"]
    if op == "norm":
        y, s, _ = plan.forward(st["x"], st["weight"], st["bias"], residual=st["residual"], need_backward=False)
        return {"y": y} if st["residual"] is None else {"y": y, "s": s}
    if op == "norm_train":
        y, s, stats = plan.forward(st["x"], st["weight"], st["bias"], residual=st["residual"])
        gx, gw, gb = plan.backward(st["grad_y"], s, st["weight"], stats, grad_s=st["grad_s"])
        out = {"y": y}
        if st["residual"] is not None:
            out["s"] = s
        out.update(grad_x=gx, grad_weight=gw, grad_bias=gb)
        return out
    if op in ("conv", "conv_train"):
        y, last = plan.forward(st["x"], st["weight"], st["bias"], state=st["state"], lengths=st["lengths"])
        out = {"y": y, "state": last}
        if op == "conv_train":
            gx, gw, gb, gs = plan.backward(st["grad_y"], st["x"], st["weight"], st["bias"], state=st["state"],
                                           lengths=st["lengths"], grad_state_out=st["grad_state"])
            out.update(grad_x=gx, grad_state=gs, grad_weight=gw, grad_bias=gb)
        return out
    if op == "clip":
        return {"norm": plan.clip(st["max_norm"], eps=CLIP_EPS), "grads": [_real(g) for g in st["out"]]}
    maps = {"D": st["D"], "z": st["z"], "dt_bias": st["dt_bias"], "h0": st["h0"], "lengths": st["lengths"]}
    if op == "scan":
        y, last = plan.forward(st["x"], st["dt"], st["A"], st["B"], st["C"], **maps)
        return {"y": y, "h_last": last}
    y, last = plan.forward(st["x"], st["dt"], st["A"], st["B"], st["C"], checkpoints=st["checkpoints"], **maps)
    gr = plan.backward(st["grad_y"], st["x"], st["dt"], st["A"], st["B"], st["C"], st["checkpoints"], grad_last=st["grad_last"], **maps)
    out = {"y": y, "h_last": last}
    for k in ("x", "dt", "B", "C", "z", "A", "D", "dt_bias", "h0"):
        if k != "z" or st["z"] is not None:
            out["grad_" + k] = gr[k]
    return out


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------- work and the definition in 64 bits
def work(case):
    op = case["op"]
    if op == "clip":
        n = [(math.prod(s) * SIZE[k], math.prod(s) * (2 if k == "c64" else 1)) for s, k in _tensors(case)]
        return {"bytes": 2 * sum(a for a, _ in n), "flops": 3 * sum(b for _, b in n)}
    b = SIZE[case["type"]]
    if op in ("norm", "norm_train"):
        n, c = case["outer"] * case["channels"] * case["inner"], case["channels"]
        r = case["residual"]
        if op == "norm":
            return {"bytes": n * b * (4 if r else 2) + 8 * c, "flops": 8 * n}
        return {"bytes": n * b * (7 if r else 4) + 16 * c, "flops": 20 * n}
    t, c = case["batch"] * case["length"], case["channels"]
    n = t * c
    if op in ("conv", "conv_train"):
        k = case["width"]
        edge = case["batch"] * (k - 1) * c * b
        if op == "conv":
            return {"bytes": 2 * n * b + 2 * edge + 4 * c * (k + 1), "flops": n * (2 * k + 6)}
        return {"bytes": 4 * n * b + 4 * edge + 8 * c * (k + 1), "flops": n * (6 * k + 20)}
    s, g, z = case["states"], case["groups"], 1 if case["gated"] else 0
    maps, state = 2 * t * g * s * b, 4 * case["batch"] * c * s
    if op == "scan":
        return {"bytes": n * b * (3 + z) + maps + 2 * state + 4 * c * (s + 2), "flops": n * (7 * s + 12)}
    return {"bytes": n * b * (6 + 2 * z) + 2 * maps + 4 * state + 8 * c * (s + 2), "flops": n * (26 * s + 40)}


def _exact_norm(case, st):
    s = st["x"].double()
    if st["residual"] is not None:
        s += st["residual"].double()
    c = s.shape[1]
    shape = [1, c] + [1] * (s.dim() - 2)
    w, b = st["weight"].double().reshape(shape), st["bias"].double().reshape(shape)
    mean = torch.einsum("oc...->o...", s).unsqueeze(1) / c
    n = s - mean
    sd = torch.sqrt(torch.einsum("oc...,oc...->o...", n, n) / c + EPS).unsqueeze(1)
    n /= sd
    out = {"y": n * w + b}
    if st["residual"] is not None:
        out["s"] = s
    if case["op"] == "norm":
        return out
    gy = st["grad_y"].double()
    out_w, out_b = torch.einsum("oc...,oc...->c", gy, n), torch.einsum("oc...->c", gy)
    gn = gy * w
    gx = gn - torch.einsum("oc...->o...", gn).unsqueeze(1) / c
    gx -= n * (torch.einsum("oc...,oc...->o...", gn, n) / c).unsqueeze(1)
    gx /= sd
    if st["grad_s"] is not None:
        gx += st["grad_s"].double()
    out.update(grad_x=gx, grad_weight=out_w, grad_bias=out_b)
    return out


def _exact_conv(case, st):
    b, n, c, k = case["batch"], case["length"], case["channels"], case["width"]
    w, bias = st["weight"].double(), st["bias"].double()
    train = case["op"] == "conv_train"
    y = torch.zeros((b, n, c), dtype=torch.float64, device="cuda")
    last = torch.empty((b, k - 1, c), dtype=torch.float64, device="cuda")
    gx, gs = torch.zeros_like(y), torch.empty_like(last)
    gw, gb = torch.zeros_like(w), torch.zeros_like(bias)
    ends = [n] * b if st["lengths"] is None else st["lengths"].tolist()
    for i, e in enumerate(ends):                                  # one sequence after the other, without its padding
        seq = torch.cat([st["state"][i].double(), st["x"][i, :e].double()])
        last[i] = seq[e:]
        pre = bias.expand(e, c).clone()
        for j in range(k):
            pre += w[:, j] * seq[j:j + e]
        sig = 1 / (1 + torch.exp(-pre))
        y[i, :e] = pre * sig
        if train:
            gp = st["grad_y"][i, :e].double() * sig * (1 + pre * (1 - sig))
            gseq = torch.zeros_like(seq)
            gseq[e:] = st["grad_state"][i].double()
            for j in range(k):
                gseq[j:j + e] += w[:, j] * gp
                gw[:, j] += torch.einsum("tc,tc->c", gp, seq[j:j + e])
            gb += torch.einsum("tc->c", gp)
            gs[i], gx[i, :e] = gseq[:k - 1], gseq[k - 1:]
    out = {"y": y, "state": last}
    if train:
        out.update(grad_x=gx, grad_state=gs, grad_weight=gw, grad_bias=gb)
    return out


def _exact_scan(case, st):
    b, n, c, s, g = (case[k] for k in ("batch", "length", "channels", "states", "groups"))
    A, D, bias = st["A"].double().view(g, c // g, s), st["D"].double(), st["dt_bias"].double()
    end = torch.full((b,), n, device="cuda") if st["lengths"] is None else st["lengths"].long()
    train = case["op"] == "scan_train"
    raw = st["dt"].double() + bias
    delta = torch.logaddexp(raw, torch.zeros((), dtype=torch.float64, device="cuda"))
    x = st["x"].double()
    grouped = lambda m: m.reshape(b, g, c // g)
    state = st["h0"].double().view(b, g, c // g, s)
    y = torch.zeros((b, n, c), dtype=torch.float64, device="cuda")
    core = torch.zeros_like(y) if train else None
    before = torch.empty((n, b, g, c // g, s), dtype=torch.float64, device="cuda") if train else None
    gate = st["z"].double() if st["z"] is not None else None
    for t in range(n):                                            # one step after the other, as the definition says
        live = (t < end)[:, None, None, None]
        if train:
            before[t] = state
        d, u = grouped(delta[:, t]), grouped(delta[:, t] * x[:, t])
        new = torch.exp(d[..., None] * A) * state + torch.einsum("bgc,bgs->bgcs", u, st["B"][:, t].double())
        state = torch.where(live, new, state)
        o = torch.einsum("bgcs,bgs->bgc", state, st["C"][:, t].double()).reshape(b, c) + D * x[:, t]
        if train:
            core[:, t] = o
        if gate is not None:
            o = o * gate[:, t] / (1 + torch.exp(-gate[:, t]))
        y[:, t] = torch.where((t < end)[:, None], o, torch.zeros_like(o))
    out = {"y": y, "h_last": state.reshape(b, c, s)}
    if not train:
        return out
    out.update(grad_x=torch.zeros_like(y), grad_dt=torch.zeros_like(y))
    out.update(grad_B=torch.zeros(st["B"].shape, dtype=torch.float64, device="cuda"),
               grad_C=torch.zeros(st["C"].shape, dtype=torch.float64, device="cuda"))
    gA, gD, gbias = torch.zeros_like(A), torch.zeros_like(D), torch.zeros_like(bias)
    carry, gyz = st["grad_last"].double().view(b, g, c // g, s), st["grad_y"].double()
    if gate is not None:
        sig = 1 / (1 + torch.exp(-gate))
        alive = (torch.arange(n, device="cuda")[None, :] < end[:, None])[..., None]
        out["grad_z"] = torch.where(alive, gyz * core * sig * (1 + gate * (1 - sig)), torch.zeros_like(gate))
        gyz = gyz * gate * sig
    slope = 1 / (1 + torch.exp(-raw))
    for t in range(n - 1, -1, -1):
        live = (t < end)
        gy, d = grouped(gyz[:, t]), grouped(delta[:, t])
        B, C, xt = st["B"][:, t].double(), st["C"][:, t].double(), grouped(x[:, t])
        a = torch.exp(d[..., None] * A)
        now = a * before[t] + torch.einsum("bgc,bgs->bgcs", d * xt, B)
        gh = carry + torch.einsum("bgc,bgs->bgcs", gy, C)
        ga = gh * before[t] * a
        through = torch.einsum("bgcs,bgs->bgc", gh, B)
        gd = torch.einsum("bgcs,gcs->bgc", ga, A) + through * xt
        m2, m3, m4 = live[:, None].double(), live[:, None, None].double(), live[:, None, None, None]
        out["grad_x"][:, t] = m2 * (through * d + gy * D.view(g, c // g)).reshape(b, c)
        graw = m2 * gd.reshape(b, c) * slope[:, t]
        out["grad_dt"][:, t] = graw
        out["grad_B"][:, t] = m3 * torch.einsum("bgcs,bgc->bgs", gh, d * xt)
        out["grad_C"][:, t] = m3 * torch.einsum("bgcs,bgc->bgs", now, gy)
        gA += torch.einsum("bgcs,bgc->gcs", ga, d * m3)
        gD += torch.einsum("bgc,bgc->gc", gy * m3, xt).reshape(c)
        gbias += torch.einsum("bc->c", graw)
        carry = torch.where(m4, a * gh, carry)
    out.update(grad_A=gA.reshape(c, s), grad_D=gD, grad_dt_bias=gbias, grad_h0=carry.reshape(b, c, s))
    order = ["y", "h_last"] + ["grad_" + k for k in ("x", "dt", "B", "C", "z", "A", "D", "dt_bias", "h0")]
    return {k: out[k] for k in order if k in out}


def _exact_clip(case, st):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in st["grads"]:
        v = _real(g).double().flatten()
        total += torch.dot(v, v)
    norm = torch.sqrt(total)
    coef = torch.minimum(st["max_norm"] / (norm + CLIP_EPS), torch.ones_like(norm))
    return {"norm": norm, "grads": [_real(g).double() * coef for g in st["grads"]]}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(case, st)
    if case["op"] in ("conv", "conv_train"):
        return _exact_conv(case, st)
    return _exact_clip(case, st) if case["op"] == "clip" else _exact_scan(case, st)
