"""Measured cases of the operators of a stage whose blocks mix positions by a recurrence, as calls of their own.

  conv   a causal convolution of few taps along the positions, each channel by itself, and SiLU behind it: forward pass (with the inputs before the first
         position, for programs that go on from a prompt a token at a time) and backward pass
  scan   a selective state space: per head S_t = exp(-delta_t e^a) S_{t-1} + delta_t x_t B_t', y_t = S_t C_t + skip x_t, delta = softplus(dt + bias), over rows
         [x | B | C]: forward pass over prompts and single tokens, and backward pass
  norm   group norm over channels-last maps (or each token's groups of features) with its activation: forward and backward pass
  clip   the norm of all gradients of a stage together, and the gradients scaled to at most a given norm

With `own` false, `run` computes them from elementary operations in 32 bits (decays and sums of many values in 64), with it true through the library.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64   # positions that the scan's plain form takes at a time


# ------------------------------------------------------------------------------------------------ the cases
def _conv(**kw):
    return dict({"op": "conv", "dtype": "bf16", "backward": False, "taps": 4, "carried": False, "silu": True, "bias": True}, **kw)


def _scan(**kw):
    return dict({"op": "scan", "dtype": "bf16", "backward": False, "groups": 1, "carried": False}, **kw)


def _norm(**kw):
    return dict({"op": "norm", "dtype": "bf16", "backward": False, "act": "relu", "rms": False}, **kw)


def _clip(**kw):
    return dict({"op": "clip", "dtype": "f32", "limit": 0.5}, **kw)


def listed():
    return [
        # one new token for each of 8 sequences, in fp32: a launch and one latency
        _conv(name="conv_token_f32", dtype="f32", samples=8, positions=1, channels=1664, carried=True),
        # the benchmark's mini-batch of 16 sequences of 512 positions, a mixer of twice its width, back
        _conv(name="conv_text_grad", samples=16, positions=512, channels=1664, backward=True),
        # serving 64 sequences, one new token each: the states are read and written
        _scan(name="scan_token", samples=64, positions=1, heads=24, dh=64, n=64, carried=True),
        # the benchmark's mini-batch, forward and backward
        _scan(name="scan_text", samples=16, positions=512, heads=24, dh=64, n=64),
        _scan(name="scan_text_grad", samples=16, positions=512, heads=24, dh=64, n=64, backward=True),
        # one long prompt with states of twice the features
        _scan(name="scan_prompt", samples=1, positions=32768, heads=24, dh=64, n=128, carried=True),
        # odd sizes in fp32, heads in two groups, from a given state, back
        _scan(name="scan_odd_f32_grad", dtype="f32", samples=3, positions=333, heads=6, dh=40, n=24, groups=2, carried=True, backward=True),
        # the norm behind the mixer: each token's 24 groups of 64 features, without means
        _norm(name="norm_text", samples=8192, positions=1, channels=1536, groups=24, act="silu", rms=True),
        # the test suite's small maps
        _norm(name="norm_small_f32", dtype="f32", samples=8, positions=64, channels=64, groups=8),
        # a residual network's first maps, a mini-batch of 32 images, back
        _norm(name="norm_maps_grad", samples=32, positions=3136, channels=256, groups=32, backward=True),
        # a small multi-layer network's gradients
        _clip(name="clip_small", width=256, layers=2, vocab=0, limit=0.1),
        # all gradients of a stage of 24 mixers at the benchmark's width, with its vocabulary
        _clip(name="clip_stage", width=768, layers=24, vocab=32000, limit=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm", "norm", "clip"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "conv":
        channels = _log_int(rng, 8, 4096)
        if rng.random() < 0.6:
            channels = (channels + 31) // 32 * 32
        positions = rng.choice([1, _log_int(rng, 2, 16384), _log_int(rng, 2, 16384)])
        samples = _log_int(rng, 1, max(1, min(256, 16 * 512 * 1664 // (2 if dtype == "f32" else 1) // (positions * channels))))
        return _conv(dtype=dtype, samples=samples, positions=positions, channels=channels, taps=rng.randint(2, 8) if rng.random() < 0.4 else 4,
                     carried=rng.random() < 0.5, silu=rng.random() < 0.8, bias=rng.random() < 0.8, backward=positions > 1 and rng.random() < 0.5)
    if op == "scan":
        dh, n = rng.choice([16, 32, 64, 64, 128, rng.randint(4, 128)]), rng.choice([16, 32, 64, 128, rng.randint(4, 128)])
        groups = rng.choice([1, 1, 1, 2, 4])
        heads = groups * _log_int(rng, 1, 48 // groups)
        positions = rng.choice([1, _log_int(rng, 2, 16384), _log_int(rng, 2, 16384)])
        most = 16 * 512 * 24 * 64 // (4 if dtype == "f32" else 2)
        samples = _log_int(rng, 1, max(1, min(128, most // (max(positions, 64) * heads * dh * max(1, n // 64)))))
        backward = 1 < positions <= 2048 and rng.random() < 0.5
        return _scan(dtype=dtype, samples=samples, positions=positions, heads=heads, dh=dh, n=n, groups=groups, carried=rng.random() < 0.5 or positions == 1, backward=backward)
    if op == "norm":
        size = _log_int(rng, 1, 128)
        if rng.random() < 0.6:
            size = (size + 7) // 8 * 8
        groups = _log_int(rng, 1, max(1, min(64, 8192 // size)))
        positions = rng.choice([1, rng.randint(2, 80) ** 2, _log_int(rng, 2, 6400)])
        size = max(size, -(-16 // positions))   # (of very few values a norm leaves next to nothing but their signs)
        most = 32 * 3136 * 256 // (2 if dtype == "f32" else 1)
        samples = _log_int(rng, 1, max(1, min(16384, most // (positions * groups * size))))
        return _norm(dtype=dtype, samples=samples, positions=positions, channels=groups * size, groups=groups, act=rng.choice(["none", "relu", "gelu", "silu"]),
                     rms=rng.random() < 0.3, backward=rng.random() < 0.5)
    return _clip(dtype=dtype, width=_log_int(rng, 16, 1024), layers=rng.randint(1, 24), vocab=rng.choice([0, 1000, rng.randint(2, 32000)]), limit=rng.choice([0.05, 1.0, 1e9]))


def _clip_shapes(case):
    """A mixer's parameters, layer by layer: the product before it, its convolution, its heads' numbers, the norm, the product behind it; and a token table."""
    d = case["width"]
    inner, n, heads = 2 * d, 64, max(1, d // 32)
    layer = [(inner + 2 * n + heads, d), (inner + 2 * n, 4), (inner + 2 * n,), (heads,), (heads,), (heads,), (inner,), (d, inner), (d,)]
    return ([(case["vocab"], d)] if case["vocab"] else []) + layer * case["layers"]


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 1000003 + 29)
    t, f32 = TYPES[case["dtype"]], torch.float32

    def normal(*shape, to=None):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(t if to is None else to)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=DEVICE)

    st = {"case": case}
    if case["op"] == "conv":
        rows, c = case["samples"] * case["positions"], case["channels"]
        st["x"] = normal(rows, c)
        st["weight"] = normal(c, case["taps"], to=f32) / math.sqrt(case["taps"])
        st["bias"] = 0.1 * normal(c, to=f32) if case["bias"] else None
        st["tail"] = normal(case["samples"], case["taps"] - 1, c) if case["carried"] else None
        if case["backward"]:
            st["dy"] = normal(rows, c)
            st["dtail"] = normal(case["samples"], case["taps"] - 1, c) if case["carried"] else None
        return st
    if case["op"] == "scan":
        rows, h, p, n = case["samples"] * case["positions"], case["heads"], case["dh"], case["n"]
        x = normal(rows, h * p + 2 * case["groups"] * n, to=f32)
        st["x"] = (x / (1.0 + torch.exp(-x))).to(t)   # behind SiLU
        st["dt"] = 0.5 * normal(rows, h)
        step = torch.exp(math.log(1e-3) + uniform(h) * math.log(1e2))   # steps of 0.001 to 0.1
        st["dt_bias"] = step + torch.log(-torch.expm1(-step))
        st["a_log"] = torch.log(1.0 + 15.0 * uniform(h))
        st["skip"] = 1.0 + 0.1 * normal(h, to=f32)
        st["state"] = 0.3 * normal(case["samples"], h, p, n, to=f32) if case["carried"] else None
        if case["backward"]:
            st["dy"] = normal(rows, h * p)
            st["dstate"] = 0.3 * normal(case["samples"], h, p, n, to=f32) if case["carried"] else None
        return st
    if case["op"] == "norm":
        rows, c = case["samples"] * case["positions"], case["channels"]
        st["x"] = normal(rows, c) + 0.5
        st["gain"] = 1.0 + 0.2 * normal(c, to=f32)
        st["shift"] = None if case["rms"] else 0.2 * normal(c, to=f32)
        if case["backward"] and case["act"] == "relu":
            # 32 bits do not say on which side of the border a number next to it lies: it is moved off
            mean, rstd = _norm_stats(case, st["x"])[:, None, :, None].unbind(4)
            z = ((_norm_groups(case, st["x"].float()) - mean) * rstd).reshape(rows, c) * st["gain"]
            if st["shift"] is not None:
                z += st["shift"]
            st["x"] = torch.where(z.abs() < 1e-5, st["x"] + 0.25, st["x"])
        if case["backward"]:
            st["stats"] = _norm_stats(case, st["x"])   # as the forward pass has left them
            st["dy"] = normal(rows, c)
        return st
    shapes = _clip_shapes(case)
    st["grads"] = [normal(*s) * 0.01 for s in shapes]
    st["sent"] = torch.empty(sum(math.prod(s) for s in shapes), dtype=t, device=DEVICE)   # one array that leaves the stage, and a view of it for each gradient
    st["out"] = [v.view(s) for v, s in zip(st["sent"].split([math.prod(s) for s in shapes]), shapes)]
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _conv_sums(st):
    """The inputs with those before the first position, and the sums of taps and bias."""
    case, w = st["case"], st["weight"]
    b, s, c, k = case["samples"], case["positions"], case["channels"], case["taps"]
    tail = st["tail"].float() if case["carried"] else torch.zeros(b, k - 1, c, device=DEVICE)
    u = torch.cat([tail, st["x"].float().reshape(b, s, c)], 1)
    z = sum(u[:, j:j + s] * w[:, j] for j in range(k))
    return u, z if st["bias"] is None else z + st["bias"]


def _conv_plain(st):
    case, t = st["case"], st["x"].dtype
    s, c, k = case["positions"], case["channels"], case["taps"]
    u, z = _conv_sums(st)
    if not case["backward"]:
        y = z * _sigmoid(z) if case["silu"] else z
        out = {"y": y.reshape(-1, c).to(t)}
        if case["carried"]:
            out["tail"] = u[:, s:].to(t)
        return out
    dz = st["dy"].float().reshape(z.shape)
    if case["silu"]:
        g = _sigmoid(z)
        dz = dz * (g * (1.0 + z * (1.0 - g)))
    du = torch.zeros_like(u)
    if case["carried"]:
        du[:, s:] = st["dtail"].float()
    for j in range(k):
        du[:, j:j + s] += dz * st["weight"][:, j]
    out = {"dx": du[:, k - 1:].reshape(-1, c).to(t), "dweight": torch.stack([(dz * u[:, j:j + s]).sum((0, 1)) for j in range(k)], 1)}
    if st["bias"] is not None:
        out["dbias"] = dz.sum((0, 1))
    if case["carried"]:
        out["dtail"] = du[:, :k - 1].to(t)
    return out


def _scan_parts(case, x):
    """x [samples, positions, heads, dh], B and C [samples, positions, heads, n] of rows [x | B | C]."""
    b, s, h, p, g, n = case["samples"], case["positions"], case["heads"], case["dh"], case["groups"], case["n"]
    xs = x[:, :h * p].reshape(b, s, h, p)
    bs = x[:, h * p:h * p + g * n].reshape(b, s, g, 1, n).expand(b, s, g, h // g, n).reshape(b, s, h, n)
    cs = x[:, h * p + g * n:].reshape(b, s, g, 1, n).expand(b, s, g, h // g, n).reshape(b, s, h, n)
    return xs, bs, cs


def _scan_forward(case, x, dt, a_log, skip, dt_bias, state):
    """Positions in chunks: inside one by its matrix of decayed products C_t B_s, from chunk to chunk by the chunks' states.  Decays are formed in 64 bits."""
    b, s, h, p, n = case["samples"], case["positions"], case["heads"], case["dh"], case["n"]
    q = min(CHUNK, s)
    m = -(-s // q)
    xs, bs, cs = _scan_parts(case, x)
    u = dt.reshape(b, s, h) + dt_bias
    delta = torch.clamp(u, min=0.0) + torch.log1p(torch.exp(-u.abs()))

    def chunks(v):   # [b, s, h, ...] -> [b, h, m, q, ...], zeros behind the last position
        v = torch.cat([v, v.new_zeros(b, m * q - s, *v.shape[2:])], 1)
        return v.reshape(b, m, q, *v.shape[2:]).movedim(3, 1)

    xc, bc, cc, dc = chunks(xs), chunks(bs), chunks(cs), chunks(delta)
    total = torch.cumsum(-dc.double() * torch.exp(a_log.double())[None, :, None, None], 3)   # [b, h, m, q]
    past = torch.ones(q, q, dtype=torch.bool, device=x.device).tril()
    decay = torch.exp((total[..., :, None] - total[..., None, :]).masked_fill(~past, -math.inf)).float()
    y = ((cc @ bc.transpose(-1, -2)) * decay * dc[..., None, :]) @ xc
    end = total[..., -1]                                                                     # [b, h, m]
    own_states = (xc * (dc * torch.exp(end[..., None] - total).float())[..., None]).transpose(-1, -2) @ bc   # [b, h, m, p, n]
    # the state behind chunk j is the sum of the states that chunks i <= j have left, decayed by the chunks between
    ends = torch.cumsum(end, 2)
    lower = torch.ones(m, m, dtype=torch.bool, device=x.device).tril()
    between = torch.exp((ends[..., :, None] - ends[..., None, :]).masked_fill(~lower, -math.inf)).float()
    states = (between @ own_states.reshape(b, h, m, p * n)).reshape(b, h, m, p, n)
    first = state if state is not None else torch.zeros(b, h, p, n, device=x.device)
    states = states + torch.exp(ends).float()[..., None, None] * first[:, :, None]
    before = torch.cat([first[:, :, None], states[:, :, :-1]], 2)
    y = y + (cc @ before.transpose(-1, -2)) * torch.exp(total).float()[..., None]
    y = y.movedim(1, 3).reshape(b, m * q, h, p)[:, :s] + skip[:, None] * xs
    return y.reshape(b * s, h * p), states[:, :, -1]


def _scan_plain(st):
    case, t = st["case"], st["x"].dtype
    leaves = [st["x"].float(), st["dt"].float(), st["a_log"], st["skip"], st["dt_bias"], st["state"]]
    if not case["backward"]:
        y, state = _scan_forward(case, *leaves)
        return {"y": y.to(t), "state": state} if case["carried"] else {"y": y.to(t)}
    with torch.enable_grad():
        leaves = [v.detach().requires_grad_(True) if v is not None else None for v in leaves]
        y, state = _scan_forward(case, *leaves)
        results, given = [y], [st["dy"].float()]
        if case["carried"]:
            results, given = results + [state], given + [st["dstate"]]
        grads = torch.autograd.grad(results, [v for v in leaves if v is not None], given)
    out = {"dx": grads[0].to(t), "ddt": grads[1].to(t), "da_log": grads[2], "dskip": grads[3], "ddt_bias": grads[4]}
    if case["carried"]:
        out["dstate"] = grads[5]
    return out


def _norm_groups(case, v):
    """Rows as [samples, positions, groups, features of a group]."""
    return v.reshape(case["samples"], case["positions"], case["groups"], case["channels"] // case["groups"])


def _norm_stats(case, x):
    """Mean (0 without means) and 1 / standard deviation of each sample's groups: [samples, groups, 2]."""
    v = _norm_groups(case, x.float())
    mean = torch.zeros_like(v[:, :1, :, :1]) if case["rms"] else v.mean((1, 3), keepdim=True)
    var = ((v - mean) ** 2).mean((1, 3), keepdim=True)
    return torch.stack([mean[:, 0, :, 0], 1.0 / torch.sqrt(var[:, 0, :, 0] + 1e-5)], 2).contiguous()


def _norm_plain(st):
    case, t = st["case"], st["x"].dtype
    size = case["channels"] // case["groups"]
    stats = st["stats"] if case["backward"] else _norm_stats(case, st["x"])
    mean, rstd = stats[:, None, :, None, 0], stats[:, None, :, None, 1]
    xhat = (_norm_groups(case, st["x"].float()) - mean) * rstd
    gain = st["gain"].reshape(-1, size)
    z = gain * xhat
    if st["shift"] is not None:
        z = z + st["shift"].reshape(-1, size)
    act = case["act"]
    if not case["backward"]:
        if act == "relu":
            z = torch.clamp(z, min=0.0)
        elif act == "gelu":
            z = z * (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))))
        elif act == "silu":
            z = z * _sigmoid(z)
        return {"y": z.reshape(-1, case["channels"]).to(t), "stats": stats}
    dz = _norm_groups(case, st["dy"].float())
    if act == "relu":
        dz = dz * (z > 0)
    elif act == "gelu":
        dz = dz * (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi))
    elif act == "silu":
        g = _sigmoid(z)
        dz = dz * (g * (1.0 + z * (1.0 - g)))
    out = {"dgain": (dz * xhat).sum((0, 1)).reshape(-1)}
    if not case["rms"]:
        out["dshift"] = dz.sum((0, 1)).reshape(-1)
    dz = dz * gain
    d = dz - xhat * (dz * xhat).mean((1, 3), keepdim=True)
    if not case["rms"]:
        d = d - dz.mean((1, 3), keepdim=True)
    out["dx"] = (d * rstd).reshape(-1, case["channels"]).to(t)
    return out


def _clip_plain(st):
    grads, limit = st["grads"], st["case"]["limit"]
    norm = torch.sqrt(torch.stack([g.double().square().sum() for g in grads]).sum())
    scale = torch.where(norm > limit, limit / norm, torch.ones_like(norm)).float()
    for g, o in zip(grads, st["out"]):
        torch.mul(g, scale, out=o) if g.dtype == torch.float32 else o.copy_(g.float() * scale)
    return {"norm": norm.float(), "grads": st["sent"]}


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if not own:
        return {"conv": _conv_plain, "scan": _scan_plain, "norm": _norm_plain, "clip": _clip_plain}[case["op"]](st)
    import paper_2410_14312_amd as tmps
    if case["op"] == "conv":
        if not case["backward"]:
            y, tail = tmps.short_conv(st["x"], st["weight"], st["bias"], positions=case["positions"], tail=st["tail"], want_tail=case["carried"], silu=case["silu"])
            return {"y": y, "tail": tail} if case["carried"] else {"y": y}
        dx, dweight, dbias, dtail = tmps.short_conv_backward(st["dy"], st["x"], st["weight"], st["bias"], positions=case["positions"], tail=st["tail"],
                                                             dtail=st["dtail"], silu=case["silu"])
        return {k: v for k, v in {"dx": dx, "dweight": dweight, "dbias": dbias, "dtail": dtail}.items() if v is not None}
    if case["op"] == "scan":
        shape = {"positions": case["positions"], "groups": case["groups"], "state_features": case["n"], "state": st["state"]}
        if not case["backward"]:
            y, state = tmps.selective_scan(st["x"], st["dt"], st["a_log"], st["skip"], st["dt_bias"], want_state=case["carried"], **shape)
            return {"y": y, "state": state} if case["carried"] else {"y": y}
        dx, ddt, da_log, dskip, ddt_bias, dstate = tmps.selective_scan_backward(st["dy"], st["x"], st["dt"], st["a_log"], st["skip"], st["dt_bias"],
                                                                                dstate=st["dstate"], **shape)
        out = {"dx": dx, "ddt": ddt, "da_log": da_log, "dskip": dskip, "ddt_bias": ddt_bias}
        return dict(out, dstate=dstate) if case["carried"] else out
    if case["op"] == "norm":
        act = None if case["act"] == "none" else case["act"]
        if not case["backward"]:
            y, stats = tmps.group_norm(st["x"], st["gain"], st["shift"], groups=case["groups"], positions=case["positions"], act=act, rms=case["rms"])
            return {"y": y, "stats": stats}
        dx, dgain, dshift = tmps.group_norm_backward(st["dy"], st["x"], st["stats"], st["gain"], st["shift"], groups=case["groups"], positions=case["positions"],
                                                     act=act, rms=case["rms"])
        return {"dx": dx, "dgain": dgain} if case["rms"] else {"dx": dx, "dgain": dgain, "dshift": dshift}
    norm = tmps.clip_gradients(st["grads"], case["limit"], out=st["out"])
    return {"norm": norm, "grads": st["sent"]}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "conv":
        n, c, k = case["samples"] * case["positions"] * case["channels"], case["channels"], case["taps"]
        tails = case["samples"] * (k - 1) * c * size * case["carried"]
        if not case["backward"]:
            return {"bytes": 2 * n * size + 2 * tails + 4 * c * (k + case["bias"]), "flops": n * (2 * k + 4 * case["silu"])}
        return {"bytes": 3 * n * size + 3 * tails + 8 * c * (k + case["bias"]), "flops": n * (6 * k + 8 * case["silu"])}
    if case["op"] == "scan":
        rows, h, p, n, g = case["samples"] * case["positions"], case["heads"], case["dh"], case["n"], case["groups"]
        wide, states = h * p + 2 * g * n, 4 * case["samples"] * h * p * n * case["carried"]
        if not case["backward"]:   # a position's state: decayed, added to, read
            return {"bytes": rows * (wide + h + h * p) * size + 2 * states, "flops": rows * h * (5 * p * n + 10)}
        return {"bytes": rows * (2 * wide + 2 * h + h * p) * size + 3 * states, "flops": rows * h * (16 * p * n + 30)}
    if case["op"] == "norm":
        rows, c = case["samples"] * case["positions"], case["channels"]
        stats, act = 8 * case["samples"] * case["groups"], 6 if case["act"] in ("gelu", "silu") else 1
        if not case["backward"]:
            return {"bytes": 2 * rows * c * size + stats + 8 * c, "flops": rows * c * (7 + act)}
        return {"bytes": 3 * rows * c * size + stats + 16 * c, "flops": rows * c * (14 + 2 * act)}
    n = sum(math.prod(s) for s in _clip_shapes(case))
    return {"bytes": 2 * n * size, "flops": 3 * n}


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "conv":
        return _exact_conv(case, st)
    if case["op"] == "scan":
        return _exact_scan(case, st) if case["positions"] <= 40000 else None
    if case["op"] == "norm":
        return _exact_norm(case, st)
    grads = [g.double() for g in st["grads"]]
    norm = math.sqrt(sum(float((g * g).sum()) for g in grads))
    return {"norm": norm, "grads": torch.cat([g.reshape(-1) * min(1.0, case["limit"] / norm) for g in grads])}


def _exact_conv(case, st):
    b, s, c, k = case["samples"], case["positions"], case["channels"], case["taps"]
    leaf = {n: st[n].double().requires_grad_(True) for n in ("x", "weight", "bias", "tail") if st[n] is not None}
    with torch.enable_grad():
        tail = leaf["tail"] if case["carried"] else torch.zeros(b, k - 1, c, dtype=torch.float64, device=DEVICE)
        u = torch.cat([tail, leaf["x"].view(b, s, c)], 1)
        z = (u.unfold(1, k, 1) * leaf["weight"]).sum(3)   # [b, s, c, k]
        if "bias" in leaf:
            z = z + leaf["bias"]
        y = (z * torch.sigmoid(z) if case["silu"] else z).reshape(-1, c)
        if not case["backward"]:
            out = {"y": y.detach()}
            if case["carried"]:
                out["tail"] = u[:, s:].detach()
            return out
        results, given = [y], [st["dy"].double()]
        if case["carried"]:
            results, given = [y, u[:, s:]], given + [st["dtail"].double()]
        grads = torch.autograd.grad(results, list(leaf.values()), given)
    return {"d" + n: g for n, g in zip(leaf, grads)}


def _exact_scan(case, st):
    """Position by position; the gradients by the recurrence's own adjoint, from the last position to the first."""
    b, s, h, p, n, g = case["samples"], case["positions"], case["heads"], case["dh"], case["n"], case["groups"]
    f64 = torch.float64
    xs, bs, cs = _scan_parts(case, st["x"].double())
    u = st["dt"].double().view(b, s, h) + st["dt_bias"].double()
    delta = torch.logaddexp(u, torch.zeros_like(u))
    rate = torch.exp(st["a_log"].double())
    decay = torch.exp(-delta * rate)
    state = st["state"].double() if case["carried"] else torch.zeros(b, h, p, n, dtype=f64, device=DEVICE)
    if case["backward"] and s * state.numel() * 8 > (48 << 30):
        return None
    y, kept = torch.empty(b, s, h, p, dtype=f64, device=DEVICE), []
    for t in range(s):
        if case["backward"]:
            kept.append(state)
        state = decay[:, t, :, None, None] * state + (delta[:, t, :, None] * xs[:, t])[..., None] * bs[:, t, :, None]
        y[:, t] = (state * cs[:, t, :, None]).sum(3)
    skip = st["skip"].double()[:, None]
    if not case["backward"]:
        out = {"y": (y + skip * xs).reshape(b * s, h * p)}
        return dict(out, state=state) if case["carried"] else out
    dy = st["dy"].double().view(b, s, h, p)
    gs = st["dstate"].double() if case["carried"] else torch.zeros_like(state)
    dx, db, dc, ddelta, drate = skip * dy, torch.empty_like(bs), torch.empty_like(cs), torch.empty_like(delta), torch.zeros_like(rate)
    for t in reversed(range(s)):
        dc[:, t] = (state * dy[:, t, ..., None]).sum(2)
        gs = gs + dy[:, t, ..., None] * cs[:, t, :, None]
        through = (gs * bs[:, t, :, None]).sum(3)
        dx[:, t] += delta[:, t, :, None] * through
        db[:, t] = (gs * (delta[:, t, :, None] * xs[:, t])[..., None]).sum(2)
        state = kept.pop()
        lost = (gs * state).sum((2, 3)) * decay[:, t]
        ddelta[:, t] = (through * xs[:, t]).sum(2) - rate * lost
        drate -= (delta[:, t] * lost).sum(0)
        gs = decay[:, t, :, None, None] * gs
    du = ddelta * torch.sigmoid(u)
    shared = [v.view(b, s, g, h // g, n).sum(3).reshape(b * s, g * n) for v in (db, dc)]
    out = {"dx": torch.cat([dx.reshape(b * s, h * p)] + shared, 1), "ddt": du.reshape(b * s, h), "da_log": drate * rate, "dskip": (dy * xs).sum((0, 1, 3)),
           "ddt_bias": du.sum((0, 1))}
    return dict(out, dstate=gs) if case["carried"] else out


def _exact_norm(case, st):
    rows, c, g = case["samples"] * case["positions"], case["channels"], case["groups"]
    leaf = {n: st[n].double().requires_grad_(True) for n in ("x", "gain", "shift") if st[n] is not None}
    with torch.enable_grad():
        v = leaf["x"].view(case["samples"], case["positions"], g, c // g).transpose(1, 2).flatten(2)   # [samples, groups, values]
        mean = torch.zeros_like(v[:, :, :1]) if case["rms"] else v.mean(2, keepdim=True)
        rstd = (v - mean).square().mean(2, keepdim=True).add(1e-5).rsqrt()
        z = ((v - mean) * rstd).unflatten(2, (case["positions"], c // g)).transpose(1, 2).reshape(rows, c) * leaf["gain"]
        if "shift" in leaf:
            z = z + leaf["shift"]
        y = {"none": lambda w: w, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]](z)
        if not case["backward"]:
            return {"y": y.detach(), "stats": torch.cat([mean, rstd], 2).detach()}
        grads = torch.autograd.grad(y, list(leaf.values()), st["dy"].double())
    return {"d" + n: grad for n, grad in zip(leaf, grads)}
