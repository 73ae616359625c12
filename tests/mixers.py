"""Plain forms, in 64 bits, of the operators of blocks that mix positions by a recurrence, with what each result is a sum of: next to a value stands the sum of the absolute values of its
terms, which roundings are counted against."""
import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
F32 = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def generator(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, size, relative, name=""):
    """|got - want| <= half a step of the type at `want`, and `relative` of the terms' sizes."""
    g, step = got.double().cpu(), half_step(got.dtype)
    want, size = want.double().cpu(), size.double().cpu()
    bound = step * want.abs() + relative * size + 1e-37
    off = (g - want).abs() / bound
    assert g.shape == want.shape and bool(torch.isfinite(g).all()), name
    assert float(off.max() if off.numel() else 0.0) <= 1.0, "%s: %.3g times the bound" % (name, float(off.max()))


# ------------------------------------------------------------------------------------------------ short convolution
def conv(x, weight, bias, positions, tail, silu, dy=None, dtail=None):
    """Values, and sizes of their sums, of y and the tail, or of the gradients."""
    rows, c = x.shape
    k, b = weight.shape[1], rows // positions
    leaf = {"x": x, "weight": weight, "bias": bias, "tail": tail}
    leaf = {n: v.double().cpu().requires_grad_(True) for n, v in leaf.items() if v is not None}

    def forward(leaf, act):
        u = torch.cat([leaf["tail"] if "tail" in leaf else torch.zeros(b, k - 1, c, dtype=torch.float64), leaf["x"].view(b, positions, c)], 1)
        z = sum(u[:, j:j + positions] * leaf["weight"][:, j] for j in range(k)) + leaf.get("bias", 0.0)
        return (z * torch.sigmoid(z) if act and silu else z).reshape(rows, c), u[:, positions:]

    with torch.enable_grad():
        y, after = forward(leaf, True)
        sizes, _ = forward({n: v.detach().abs() for n, v in leaf.items()}, False)
        if dy is None:
            return {"y": y.detach(), "tail": after.detach()}, {"y": sizes}
        given = [dy.double().cpu()] + ([dtail.double().cpu()] if dtail is not None else [])
        grads = torch.autograd.grad([y, after][:len(given)], list(leaf.values()), given, allow_unused=True)
        # sizes: SiLU's slope is at most 1.1, and off by what z is off by at most
        plain = {n: v.detach().abs().requires_grad_(True) for n, v in leaf.items()}
        s, t = forward(plain, False)
        of = torch.autograd.grad([s, t][:len(given)], list(plain.values()), [1.1 * given[0].abs() * (1.0 + sizes)] + [g.abs() for g in given[1:]], allow_unused=True)
    zero = {n: torch.zeros_like(v) for n, v in leaf.items()}
    return ({"d" + n: g if g is not None else zero[n] for n, g in zip(leaf, grads)}, {"d" + n: g if g is not None else zero[n] for n, g in zip(leaf, of)})


# ------------------------------------------------------------------------------------------------ selective scan
def scan_inputs(seed, samples, positions, heads, dh, groups, n, t, carried, backward=False):
    g = generator(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g)
    rows = samples * positions
    out = {"x": normal(rows, heads * dh + 2 * groups * n).to(t), "dt": (0.5 * normal(rows, heads)).to(t), "a_log": torch.log(1.0 + 15.0 * torch.rand(heads, generator=g)),
           "skip": 1.0 + 0.1 * normal(heads), "dt_bias": -4.0 + 2.0 * torch.rand(heads, generator=g), "state": 0.5 * normal(samples, heads, dh, n) if carried else None}
    if backward:
        out.update(dy=normal(rows, heads * dh).to(t), dstate=0.5 * normal(samples, heads, dh, n) if carried else None)
    return {k: v.to(DEV) if v is not None else None for k, v in out.items()}


def scan(i, samples, positions, heads, dh, groups, n, backward=False, size=False, across=False):
    """Position by position.  size: every product and sum of absolute values in its place.  across: of the gradient of an exponent those terms alone that pass through its position."""
    b, s, h, p, g = samples, positions, heads, dh, groups
    mag = (lambda v: v.abs()) if size else (lambda v: v)
    x = mag(i["x"].double())
    xs = x[:, :h * p].reshape(b, s, h, p)
    bs = x[:, h * p:h * p + g * n].reshape(b, s, g, 1, n).expand(b, s, g, h // g, n).reshape(b, s, h, n)
    cs = x[:, h * p + g * n:].reshape(b, s, g, 1, n).expand(b, s, g, h // g, n).reshape(b, s, h, n)
    u = i["dt"].double().reshape(b, s, h) + i["dt_bias"].double()
    delta = torch.logaddexp(u, torch.zeros_like(u))
    rate = torch.exp(i["a_log"].double())
    decay = torch.exp(-delta * rate)
    zero = torch.zeros(b, h, p, n, dtype=torch.float64, device=x.device)
    state = mag(i["state"].double()) if i["state"] is not None else zero
    y, kept = torch.empty_like(xs), []
    for t in range(s):
        kept.append(state)
        state = decay[:, t, :, None, None] * state + (delta[:, t, :, None] * xs[:, t])[..., None] * bs[:, t, :, None]
        y[:, t] = (state * cs[:, t, :, None]).sum(3)
    skip = mag(i["skip"].double())[:, None]
    if not backward:
        return {"y": (y + skip * xs).reshape(b * s, h * p), "state": state}
    dy = mag(i["dy"].double()).reshape(b, s, h, p)
    gs = mag(i["dstate"].double()) if i.get("dstate") is not None else zero
    dx, db, dc, ddelta, drate = skip * dy, torch.empty_like(bs), torch.empty_like(cs), torch.empty_like(delta), torch.zeros_like(rate)
    running = torch.zeros_like(rate).expand(b, h).clone()
    sign = 1.0 if size else -1.0
    for t in reversed(range(s)):
        dc[:, t] = (state * dy[:, t, ..., None]).sum(2)
        gs = gs + dy[:, t, ..., None] * cs[:, t, :, None]
        through = (gs * bs[:, t, :, None]).sum(3)
        dx[:, t] += delta[:, t, :, None] * through
        db[:, t] = (gs * (delta[:, t, :, None] * xs[:, t])[..., None]).sum(2)
        of_x = (through * xs[:, t]).sum(2)
        if size:
            # the gradient of an exponent is formed as a sum over the positions of a chunk from its own on: dy y and delta of_x of each, and <S, G> behind the chunk
            if t % 64 == 63 or t == s - 1:
                running = (gs * state).sum((2, 3))
            running = running + (dy[:, t] * y[:, t]).sum(2) + delta[:, t] * of_x
            lost = running
        state = kept[t]
        if not size or across:
            lost = (gs * state).sum((2, 3)) * decay[:, t]
        ddelta[:, t] = of_x + sign * rate * lost
        drate += sign * (delta[:, t] * lost).sum(0)
        gs = decay[:, t, :, None, None] * gs
    du = ddelta * torch.sigmoid(u)
    shared = [v.view(b, s, g, h // g, n).sum(3).reshape(b * s, g * n) for v in (db, dc)]
    out = {"dx": torch.cat([dx.reshape(b * s, h * p)] + shared, 1), "ddt": du.reshape(b * s, h), "da_log": drate * rate, "dskip": (dy * xs).sum((0, 1, 3)), "ddt_bias": du.sum((0, 1))}
    if i["state"] is not None:
        out["dstate"] = gs
    return out


# ------------------------------------------------------------------------------------------------ group norm
ACTS = {None: lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


def group_norm(x, gain, shift, groups, positions, act, rms, dy=None):
    rows, c = x.shape
    b = rows // positions
    leaf = {n: v.double().cpu().requires_grad_(True) for n, v in (("x", x), ("gain", gain), ("shift", shift)) if v is not None}
    with torch.enable_grad():
        v = leaf["x"].view(b, positions, groups, c // groups).transpose(1, 2).flatten(2)
        mean = torch.zeros_like(v[:, :, :1]) if rms else v.mean(2, keepdim=True)
        rstd = (v - mean).square().mean(2, keepdim=True).add(1e-5).rsqrt()
        xhat = ((v - mean) * rstd).unflatten(2, (positions, c // groups)).transpose(1, 2).reshape(rows, c)
        z = xhat * leaf["gain"]
        if "shift" in leaf:
            z = z + leaf["shift"]
        y = ACTS[act](z)
        if dy is None:
            return {"y": y.detach(), "stats": torch.cat([mean, rstd], 2).detach(), "z": z.detach(), "xhat": xhat.detach()}
        grads = torch.autograd.grad(y, list(leaf.values()), dy.double().cpu())
    return dict({"d" + n: g for n, g in zip(leaf, grads)}, z=z.detach(), xhat=xhat.detach(), rstd=rstd.detach())
