"""Cases of the recurrent-memory operators: the root-mean-square norm with the residual's addition (and its output
in 8 bits), the matrix product of 8-bit operands with a scale for each block of 128, and the gated linear recurrence.

`own` False: the operators written out with elementary torch operations in 32 bits.  `own` True: the calls of this
package.  Tensors of an operator that works along one dimension are (outer, that dimension, inner): inner = 1 is a
token-major row (norm) or a field whose last axis is time (recurrence); inner > 1 a channels-first field (norm) or a
token-major sequence (recurrence).
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128
E4M3_MAX = 448.0
AMAX_FLOOR = 2.0 ** -100        # a block of zeros: its scale stays finite
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one new frame of four running rollouts: latency
        {"name": "norm_step_fp8", "op": "norm_fp8", "type": "bf16", "rows": 4, "channels": 2048, "residual": True},
        # a long history read in at once
        {"name": "norm_history_fp8", "op": "norm_fp8", "type": "bf16", "rows": 16384, "channels": 2048, "residual": True},
        # a training step on channels-first fields: width 20, a grid with a time axis of 30
        {"name": "norm_train_field", "op": "norm_train", "type": "f32", "outer": 1, "channels": 20,
         "inner": 64 * 64 * 32 * 30, "residual": True},
        # a training step on token-major latents, sizes that fill no tile, no residual
        {"name": "norm_train_odd", "op": "norm_train", "type": "f16", "outer": 5003, "channels": 1001, "inner": 1,
         "residual": False},
        # the projections of one new frame: the weights' bytes and latency
        {"name": "matmul_step", "op": "matmul", "type": "bf16", "m": 4, "n": 4096, "k": 2048},
        # ragged in every dimension
        {"name": "matmul_odd", "op": "matmul", "type": "f32", "m": 1000, "n": 1111, "k": 1360},
        # the projections of a long history
        {"name": "matmul_history", "op": "matmul", "type": "bf16", "m": 16384, "n": 4096, "k": 2048},
        # one step of the recurrence for the running rollouts
        {"name": "scan_step", "op": "scan", "type": "bf16", "gate": "sigmoid", "outer": 4, "length": 1, "inner": 2048,
         "ragged": False},
        # one long history: few independent sequences
        {"name": "scan_history", "op": "scan", "type": "bf16", "gate": "sigmoid", "outer": 1, "length": 65536,
         "inner": 1024, "ragged": False},
        # a training step along the time axis of channels-first fields
        {"name": "scan_train_field", "op": "scan_train", "type": "f32", "gate": "sigmoid", "outer": 20 * 64 * 64 * 32,
         "length": 30, "inner": 1, "ragged": False},
        # a training step on a ragged batch of token-major latents, odd sizes
        {"name": "scan_train_ragged", "op": "scan_train", "type": "bf16", "gate": "sigmoid", "outer": 6, "length": 4097,
         "inner": 1000, "ragged": True},
        # a training step with given decays along the first axis of a grid
        {"name": "scan_train_axis", "op": "scan_train", "type": "f32", "gate": "decay", "outer": 32, "length": 256,
         "inner": 63 * 33, "ragged": False},
    ]


def _spread(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_fp8", "norm_train", "matmul", "scan", "scan_train"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "norm_fp8":
        c = _spread(rng, 64, 8192)
        return {"op": op, "type": kind, "rows": _spread(rng, 1, max(1, min(16384, (1 << 25) // c))), "channels": c,
                "residual": rng.random() < 0.7}
    if op == "norm_train":
        if rng.random() < 0.5:                                    # channels-first fields
            c, outer = rng.choice([4, 8, 16, 20, 32, 64, 128]), rng.choice([1, 2, 4])
            inner = _spread(rng, 1024, (1 << 26) // (c * outer))
        else:
            c, inner = _spread(rng, 64, 8192), 1
            outer = _spread(rng, 1, max(1, (1 << 25) // c))
        return {"op": op, "type": kind, "outer": outer, "channels": c, "inner": inner, "residual": rng.random() < 0.5}
    if op == "matmul":
        n, k = _spread(rng, 64, 8192), _spread(rng, 64, 8192)
        most = min(16384, (1 << 37) // (n * k))
        return {"op": op, "type": kind, "m": _spread(rng, 1, max(1, most)), "n": n, "k": k}
    if rng.random() < 0.4:                                        # fields whose last axis is time
        length, inner = rng.choice([_spread(rng, 1, 64), _spread(rng, 1, 4096)]), 1
        outer = _spread(rng, 16, max(16, (1 << 25) // length))
    else:                                                         # token-major, or another axis of a grid
        length, inner = _spread(rng, 1, 16384), _spread(rng, 16, 4096)
        outer = _spread(rng, 1, max(1, min(64, (1 << 25) // (length * inner))))
    return {"op": op, "type": kind, "gate": rng.choice(["sigmoid", "sigmoid", "decay"]), "outer": outer,
            "length": length, "inner": inner, "ragged": rng.random() < 0.3}


# ---------------------------------------------------------------- inputs
def _quantised(shape, gen):
    """Normal numbers, quantised by rows of blocks of 128: what an earlier step of the same program left."""
    m, k = shape
    x = torch.randn(shape, device="cuda", generator=gen)
    return _quantise(x)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["type"]]
    rn = lambda *s: torch.randn(s, device="cuda", generator=gen)
    st = {"case": dict(case)}
    op = case["op"]
    if op in ("norm_fp8", "norm_train"):
        if op == "norm_fp8":
            shape, dim = (case["rows"], case["channels"]), 1
        else:
            shape, dim = (case["outer"], case["channels"], case["inner"]), 1
            shape = shape[:2] if case["inner"] == 1 else shape
        st["x"] = rn(*shape).to(dt)
        st["residual"] = (2.0 * rn(*shape)).to(dt) if case["residual"] else None
        st["weight"] = 1.0 + 0.2 * rn(case["channels"])
        if op == "norm_train":
            st["grad_y"] = rn(*shape).to(dt)
            st["grad_s"] = rn(*shape).to(dt) if case["residual"] else None
        if own:
            from paper_2607_14394_b200 import RmsNorm
            st["plan"] = RmsNorm(shape, dim, dtype=dt, eps=EPS)
    elif op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        kb, nb, ld = -(-k // BLOCK), -(-n // BLOCK), -(-k // 16) * 16
        # rows of 8-bit values start on 16-byte boundaries
        x = torch.zeros((m, ld), dtype=torch.float8_e4m3fn, device="cuda")
        q, st["x_scale"] = _quantised((m, k), gen)
        x[:, :k] = q
        w = torch.zeros((n, ld), dtype=torch.float8_e4m3fn, device="cuda")
        # weights: one scale for a block of 128 x 128
        full = torch.nn.functional.pad(rn(n, k) / k ** 0.5, (0, kb * BLOCK - k, 0, nb * BLOCK - n))
        full = full.view(nb, BLOCK, kb, BLOCK)
        amax = full.abs().amax(dim=(1, 3)).clamp_min(AMAX_FLOOR)
        wq = (full * (E4M3_MAX / amax)[:, None, :, None]).view(nb * BLOCK, kb * BLOCK)[:n, :k]
        w[:, :k] = wq.to(torch.float8_e4m3fn)
        st["x"], st["w"], st["w_scale"] = x[:, :k], w[:, :k], (amax / E4M3_MAX).contiguous()
        if own:
            from paper_2607_14394_b200 import Fp8Linear
            st["plan"] = Fp8Linear(st["w"], st["w_scale"], out_dtype=dt)
    else:
        o, n, i = case["outer"], case["length"], case["inner"]
        shape = (o, n) if i == 1 else (o, n, i)
        st["v"] = rn(*shape).to(dt)
        # gates of a memory that holds for a few to a few hundred steps
        g = 2.0 + 1.5 * rn(*shape)
        st["g"] = (torch.sigmoid(g) if case["gate"] == "decay" else g).to(dt)
        st["h0"] = rn(*((o,) if i == 1 else (o, i)))
        st["lengths"] = None
        if case["ragged"]:
            st["lengths"] = torch.randint(0, n + 1, (o,), device="cuda", generator=gen, dtype=torch.int32)
        if op == "scan_train":
            st["grad_h"] = rn(*shape).to(dt)
            st["grad_last"] = rn(*st["h0"].shape)
        if own:
            from paper_2607_14394_b200 import GatedScan
            st["plan"] = GatedScan(shape, 1, dtype=dt, gate=case["gate"])
            if op == "scan_train":
                st["checkpoints"] = st["plan"].new_checkpoints()
    return st


# ---------------------------------------------------------------- plain forms, in 32 bits
def _quantise(y):
    """Rows [m, k] -> 8-bit values [m, k] and scales [blocks of 128 along k, m]."""
    m, k = y.shape
    kb = -(-k // BLOCK)
    yp = torch.nn.functional.pad(y, (0, kb * BLOCK - k)).view(m, kb, BLOCK)
    amax = yp.abs().amax(dim=2).clamp_min(AMAX_FLOOR)
    q = (yp * (E4M3_MAX / amax)[..., None]).view(m, kb * BLOCK)[:, :k].to(torch.float8_e4m3fn)
    return q, (amax / E4M3_MAX).t().contiguous()


def _norm(x, residual, weight):
    s = x.float()
    if residual is not None:
        s = s + residual.float()
    rstd = torch.rsqrt((s * s).mean(dim=1, keepdim=True) + EPS)
    w = weight.view((1, -1) + (1,) * (x.dim() - 2))
    return s, rstd, w


def _prefix(a, u, h0):
    """h_t = a_t h_{t-1} + u_t along dimension 1, in log2(length) doublings of whole-tensor operations."""
    first = (a[:, :1] * h0[:, None] + u[:, :1])
    h, d, n = torch.cat([first, u[:, 1:]], dim=1), 1, a.shape[1]
    while d < n:
        h = torch.cat([h[:, :d], h[:, d:] + a[:, d:] * h[:, :-d]], dim=1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], dim=1)
        d *= 2
    return h


def _scan_terms(st):
    """(a, u, v, keep): masked steps carry the state on (a = 1, u = 0); keep is None or the steps that exist."""
    v, g = st["v"].float(), st["g"].float()
    keep = None
    if st["lengths"] is not None:
        steps = torch.arange(v.shape[1], device=v.device)
        keep = (steps[None, :] < st["lengths"][:, None]).view(v.shape[:2] + (1,) * (v.dim() - 2))
        v = torch.where(keep, v, torch.zeros_like(v))
    if st["case"]["gate"] == "sigmoid":
        a, u = torch.sigmoid(g), torch.sigmoid(-g) * v
    else:
        a, u = g, v
    if keep is not None:
        a = torch.where(keep, a, torch.ones_like(a))
    return a, u, v, keep


def _plain_scan(st, train):
    dt = TYPES[st["case"]["type"]]
    a, u, v, keep = _scan_terms(st)
    h = _prefix(a, u, st["h0"])
    out = {"h": h if keep is None else torch.where(keep, h, torch.zeros_like(h)), "h_last": h[:, -1].contiguous()}
    out["h"] = out["h"].to(dt)
    if not train:
        return out
    gh = st["grad_h"].float()
    if keep is not None:
        gh = torch.where(keep, gh, torch.zeros_like(gh))
    back = torch.cat([torch.ones_like(a[:, :1]), a[:, 1:].flip(1)], dim=1)      # the decay that leads into each step
    delta = _prefix(back, gh.flip(1), st["grad_last"]).flip(1)
    before = torch.cat([st["h0"][:, None], h[:, :-1]], dim=1)
    if st["case"]["gate"] == "sigmoid":
        gv, gg = delta * torch.sigmoid(-st["g"].float()), delta * (before - v) * a * torch.sigmoid(-st["g"].float())
    else:
        gv, gg = delta, delta * before
    if keep is not None:
        gv, gg = torch.where(keep, gv, torch.zeros_like(gv)), torch.where(keep, gg, torch.zeros_like(gg))
    out.update(grad_v=gv.to(dt), grad_g=gg.to(dt), grad_h0=(a[:, 0] * delta[:, 0]).contiguous())
    return out


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    dt = TYPES[case["type"]]
    if op == "norm_fp8":
        s, rstd, w = _norm(st["x"], st["residual"], st["weight"])
        q, scale = _quantise(s * rstd * w)
        out = {"q": q, "scale": scale}
        if st["residual"] is not None:
            out["s"] = s.to(dt)
        return out
    if op == "norm_train":
        s, rstd, w = _norm(st["x"], st["residual"], st["weight"])
        out = {"y": (s * rstd * w).to(dt)}
        gy = st["grad_y"].float()
        n = s * rstd
        gx = rstd * (w * gy - n * (w * gy * n).mean(dim=1, keepdim=True))
        if st["residual"] is not None:
            out["s"] = s.to(dt)
            gx = gx + st["grad_s"].float()
        out["grad_x"] = gx.to(dt)
        out["grad_weight"] = (gy * n).sum(dim=[d for d in range(s.dim()) if d != 1])
        return out
    if op == "matmul":
        k = case["k"]
        x = st["x"].float() * st["x_scale"].t().repeat_interleave(BLOCK, dim=1)[:, :k]
        ws = st["w_scale"].repeat_interleave(BLOCK, dim=0).repeat_interleave(BLOCK, dim=1)
        w = st["w"].float() * ws[:case["n"], :k]
        return {"out": (x @ w.t()).to(dt)}
    return _plain_scan(st, op == "scan_train")


def _framework(st):
    op, plan = st["case"]["op"], st["plan"]
    if op == "norm_fp8":
        q, scale, s = plan.forward_fp8(st["x"], st["weight"], residual=st["residual"])
        out = {"q": q, "scale": scale}
        if st["residual"] is not None:
            out["s"] = s
        return out
    if op == "norm_train":
        y, s, rstd = plan.forward(st["x"], st["weight"], residual=st["residual"])
        gx, gw = plan.backward(st["grad_y"], s, st["weight"], rstd, grad_s=st["grad_s"])
        out = {"y": y, "grad_x": gx, "grad_weight": gw}
        if st["residual"] is not None:
            out["s"] = s
        return out
    if op == "matmul":
        return {"out": plan.forward(st["x"], st["x_scale"])}
    if op == "scan":
        h, last = plan.forward(st["v"], st["g"], st["h0"], lengths=st["lengths"])
        return {"h": h, "h_last": last}
    h, last = plan.forward(st["v"], st["g"], st["h0"], lengths=st["lengths"], checkpoints=st["checkpoints"])
    gv, gg, g0 = plan.backward(st["grad_h"], st["v"], st["g"], st["checkpoints"], st["h0"], lengths=st["lengths"],
                               grad_last=st["grad_last"])
    return {"h": h, "h_last": last, "grad_v": gv, "grad_g": gg, "grad_h0": g0}


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------- work and the definition in 64 bits
def work(case):
    op, b = case["op"], SIZE[case["type"]]
    if op == "norm_fp8":
        r, c = case["rows"], case["channels"]
        n = r * c
        return {"bytes": n * b * (3 if case["residual"] else 1) + n + 4 * r * -(-c // BLOCK) + 4 * c, "flops": 6 * n}
    if op == "norm_train":
        n = case["outer"] * case["channels"] * case["inner"]
        return {"bytes": n * b * (7 if case["residual"] else 4) + 8 * case["channels"], "flops": 14 * n}
    if op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // BLOCK)
        return {"bytes": m * k + n * k + m * n * b + 4 * kb * (m + -(-n // BLOCK)), "flops": 2 * m * n * k}
    rows = case["outer"] * case["inner"]
    n = rows * case["length"]
    if op == "scan":
        return {"bytes": 3 * n * b + 8 * rows, "flops": 8 * n}
    return {"bytes": 6 * n * b + 16 * rows, "flops": 20 * n}


def _to_e4m3(x):
    """The nearest number with 4 significant bits and an exponent of at least -6, ties to even."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp_min(-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_norm(case, st):
    s = st["x"].double()
    if st["residual"] is not None:
        s += st["residual"].double()
    c = s.shape[1]
    ms = torch.einsum("oc...,oc...->o...", s, s) / c + EPS
    n = s / torch.sqrt(ms).unsqueeze(1)
    w = st["weight"].double().reshape([1, c] + [1] * (s.dim() - 2))
    out = {} if st["residual"] is None else {"s": s}
    if case["op"] == "norm_fp8":
        y, kb = n * w, -(-c // BLOCK)
        q = torch.empty_like(y)
        scale = torch.empty((kb, y.shape[0]), dtype=torch.float64, device=y.device)
        for j in range(kb):
            part = y[:, j * BLOCK:(j + 1) * BLOCK]
            scale[j] = part.abs().max(dim=1).values.clamp_min(AMAX_FLOOR) / E4M3_MAX
            q[:, j * BLOCK:(j + 1) * BLOCK] = _to_e4m3(part / scale[j][:, None])
        out.update(q=q, scale=scale)
        return out
    out["y"] = n * w
    gy = st["grad_y"].double()
    out["grad_weight"] = torch.einsum("oc...,oc...->c", gy, n)
    gn = gy * w
    gx = gn - n * (torch.einsum("oc...,oc...->o...", gn, n) / c).unsqueeze(1)
    gx /= torch.sqrt(ms).unsqueeze(1)
    if st["grad_s"] is not None:
        gx += st["grad_s"].double()
    out["grad_x"] = gx
    return out


def _exact_scan(case, st):
    v, g = st["v"].double(), st["g"].double()
    o, n = v.shape[:2]
    end = st["lengths"].long() if st["lengths"] is not None else torch.full((o,), n, device=v.device)
    end = end.view([o] + [1] * (v.dim() - 2))
    sig = case["gate"] == "sigmoid"
    a = 1 / (1 + torch.exp(-g)) if sig else g
    b = 1 / (1 + torch.exp(g)) if sig else torch.ones_like(g)
    state, before, h = st["h0"].double(), torch.empty_like(v), torch.empty_like(v)
    for t in range(n):                                            # one step after the other, as the definition says
        live = t < end
        before[:, t] = state
        state = torch.where(live, a[:, t] * state + b[:, t] * v[:, t], state)
        h[:, t] = torch.where(live, state, torch.zeros_like(state))
    out = {"h": h, "h_last": state}
    if case["op"] == "scan":
        return out
    carry, gh = st["grad_last"].double(), st["grad_h"].double()
    gv, gg = torch.empty_like(v), torch.empty_like(v)
    zero = torch.zeros_like(carry)
    for t in range(n - 1, -1, -1):
        live = t < end
        delta = carry + gh[:, t]
        da = delta * (before[:, t] - v[:, t]) * a[:, t] * b[:, t] if sig else delta * before[:, t]
        gv[:, t], gg[:, t] = torch.where(live, delta * b[:, t], zero), torch.where(live, da, zero)
        carry = torch.where(live, delta * a[:, t], carry)
    out.update(grad_v=gv, grad_g=gg, grad_h0=carry)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("norm_fp8", "norm_train"):
        return _exact_norm(case, st)
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        acc = torch.zeros((m, n), dtype=torch.float64, device="cuda")
        rows = torch.arange(n, device="cuda") // BLOCK
        for j, k0 in enumerate(range(0, k, BLOCK)):               # block by block, the scales outside the sums
            part = st["x"][:, k0:k0 + BLOCK].double() @ st["w"][:, k0:k0 + BLOCK].double().t()
            acc += part * st["x_scale"][j].double()[:, None] * st["w_scale"][rows, j].double()[None, :]
        return {"out": acc}
    return _exact_scan(case, st)
