"""Measured cases of the operators that stand between a decoder stage's contractions, as calls of their own.

  rotary   the query and key heads of packed rows [q | k | v], turned by positions of up to three axes (time, height, width);
           `inverse` is the way back, which the gradient takes
  join     a block's result behind its norm, under its gate, joined with the scaled residual, and the norm in front of the next
           block: forward pass, and backward pass with the gradients of all parameters
  distill  the loss of a row of logits against a teacher's largest logits and the row's label, and its gradient

With `own` false, `run` computes them from elementary operations in 32 bits (angles in 64), with it true through the library.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------ the cases
def _rotary(**kw):
    return dict({"op": "rotary", "dtype": "bf16", "inverse": False, "interleaved": False, "own_ladders": False, "pt": 0, "ph": 0, "pw": 0, "far": 0, "base": 10000.0}, **kw)


def _join(**kw):
    return dict({"op": "join", "dtype": "bf16", "backward": False, "rms": True, "gate": False, "pre": True, "dy": True}, **kw)


def _distill(**kw):
    return dict({"op": "distill", "dtype": "bf16", "temperature": 2.0, "alpha": 0.9}, **kw)


def listed():
    return [
        # one new token far behind the others, in fp32: a launch and one latency
        _rotary(name="rotary_one_token", dtype="f32", rows=1, q=12, kv=12, dh=64, pt=32, far=1000000),
        # the benchmark's transformer: a mini-batch of 16 sequences of 512 positions of text
        _rotary(name="rotary_text", rows=8192, q=12, kv=12, dh=64, pt=32),
        # video: 16 frames of 32 x 32 patches, queries in groups that share a key head, the gradient's way
        _rotary(name="rotary_video_grad", rows=16384, q=32, kv=8, dh=128, pt=16, ph=24, pw=24, inverse=True),
        # an image of 50 x 50 patches in fp32, neighbours in pairs, a ladder for each axis, features behind the pairs left as they are
        _rotary(name="rotary_image_f32", dtype="f32", rows=2500, q=16, kv=16, dh=72, ph=16, pw=16, interleaved=True, own_ladders=True),
        # the test suite's small transformer: 8 sequences of 32 positions of 64 features
        _join(name="join_small_f32", dtype="f32", rows=256, d=64, gate=True),
        # the benchmark's transformer width, gate beside the block's result, forward and backward
        _join(name="join_768", rows=8192, d=768, gate=True),
        _join(name="join_768_grad", rows=8192, d=768, gate=True, backward=True),
        # a wide model's long batch
        _join(name="join_4096_grad", rows=16384, d=4096, backward=True),
        # an odd width in fp32 with means, the last block of a stage (nobody reads its result but the norm)
        _join(name="join_odd_f32_grad", dtype="f32", rows=2999, d=1001, rms=False, backward=True, dy=False),
        # a student's classifier of a hundred classes on a small batch
        _distill(name="distill_small_f32", dtype="f32", rows=64, classes=100, k=10, temperature=1.0, alpha=0.5),
        # the benchmark's vocabulary and mini-batch against a teacher's 64 largest logits
        _distill(name="distill_32000", rows=8192, classes=32000, k=64),
        # few rows of a large vocabulary, its size no multiple of anything
        _distill(name="distill_few_wide", rows=48, classes=131071, k=100, temperature=1.5, alpha=1.0),
    ]


def _pairs(case):
    """Pairs of features that turn with time, height and width."""
    return [case["pt"], case["ph"], case["pw"]]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "join", "join", "distill"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "rotary":
        dh = 2 * _log_int(rng, 4, 128)
        if rng.random() < 0.5:
            dh = (dh + 15) // 16 * 16
        kv = rng.randint(1, 12)
        q = kv * rng.choice([1, 1, 2, 4])
        rows = _log_int(rng, 1, max(1, min(32768, 16384 * 40 * 128 // (2 if dtype == "f32" else 1) // ((q + kv) * dh))))
        half = dh // 2 if rng.random() < 0.7 else rng.randint(1, dh // 2)
        a = rng.randint(0, half)
        b = rng.randint(0, half - a)
        pt, ph, pw = (half, 0, 0) if rng.random() < 0.4 else (a, b, half - a - b)
        return _rotary(dtype=dtype, rows=rows, q=q, kv=kv, dh=dh, pt=pt, ph=ph, pw=pw, inverse=rng.random() < 0.5, interleaved=rng.random() < 0.4,
                       own_ladders=rng.random() < 0.4, far=rng.choice([0, 0, 100000]), base=rng.choice([10000.0, 500000.0]))
    if op == "join":
        d = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            d = (d + 63) // 64 * 64
        rows = _log_int(rng, 1, max(1, min(32768, 16384 * 4096 // (2 if dtype == "f32" else 1) // d)))
        gate, pre = rng.random() < 0.4, rng.random() < 0.8
        if gate:
            rows = max(1, rows * 2 // 3)
        return _join(dtype=dtype, rows=rows, d=d, backward=rng.random() < 0.6, rms=rng.random() < 0.6, gate=gate, pre=pre,
                     dy=True if not pre else rng.random() < 0.7)
    classes = _log_int(rng, 16, 131072)
    rows = _log_int(rng, 1, max(1, min(16384, 8192 * 32000 // (2 if dtype == "f32" else 1) // classes)))
    return _distill(dtype=dtype, rows=rows, classes=classes, k=min(classes, _log_int(rng, 1, 256)), temperature=rng.choice([1.0, 1.0, 0.7, 1.5, 2.0, 4.0]),
                    alpha=rng.choice([1.0, 0.9, 0.5, 0.2]))


# ------------------------------------------------------------------------------------------------ inputs
def _distill_kind(r):
    """Rows of a mini-batch: some are padding or part of the question (nothing to learn), some have a label or a teacher alone."""
    return {5: "none", 13: "none", 9: "label", 12: "teacher"}.get(r % 16, "both")


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 1000003 + 17)
    t = TYPES[case["dtype"]]

    def normal(*shape, to=None):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(t if to is None else to)

    st = {"case": case}
    if case["op"] == "rotary":
        heads, rows = case["q"] + case["kv"], case["rows"]
        st["x"] = normal(rows, (heads + case["kv"]) * case["dh"])   # rows [q | k | v]
        n = torch.arange(rows, device=DEVICE)
        first = int(torch.randint(0, 64, (1,), generator=gen, device=DEVICE).item()) + case["far"]
        if case["ph"] or case["pw"]:
            pos = torch.stack([n // 1024 + first, n // 32 % 32, n % 32], 1)
        else:
            pos = torch.stack([n % 8192 + first] * 3, 1)
        st["positions"] = pos.to(torch.int32).contiguous()
        return st
    if case["op"] == "join":
        rows, d = case["rows"], case["d"]
        f32 = torch.float32
        st["x"] = normal(rows, d * (2 if case["gate"] else 1))
        st["r"] = normal(rows, d)
        st["gain"] = 1.0 + 0.2 * normal(d, to=f32)
        st["scale"] = 1.0 + 0.1 * normal(d, to=f32)
        st["pre_gain"] = 1.0 + 0.2 * normal(d, to=f32) if case["pre"] else None
        st["pre_shift"] = 0.1 * normal(d, to=f32) if case["pre"] and not case["rms"] else None
        if case["backward"]:
            # what the forward pass has left: its result and the rows' statistics, and the gradients that come in
            y, _, stats = _join_forward(st)
            st["y"], st["stats"] = y, stats
            st["dy"] = normal(rows, d) if case["dy"] else None
            st["du"] = normal(rows, d) if case["pre"] else None
        return st
    rows, classes, k = case["rows"], case["classes"], case["k"]
    st["logits"] = torch.randn(rows, classes, generator=gen, device=DEVICE) * 2.0
    st["ids"] = torch.empty(rows, k, dtype=torch.int32, device=DEVICE)
    st["teacher"] = torch.empty(rows, k, device=DEVICE)
    st["labels"] = torch.empty(rows, dtype=torch.int32, device=DEVICE)
    step = max(1, (1 << 26) // classes)
    for r in range(0, rows, step):
        z = st["logits"][r:r + step]
        teacher, ids = (z + torch.randn(z.shape, generator=gen, device=DEVICE)).topk(k, dim=1)
        st["teacher"][r:r + step] = teacher
        st["ids"][r:r + step] = ids.to(torch.int32)
        st["labels"][r:r + step] = ids[:, 0].to(torch.int32)
    kinds = [_distill_kind(r) for r in range(rows)]
    no_teacher = torch.tensor([w in ("none", "label") for w in kinds], device=DEVICE)
    no_label = torch.tensor([w in ("none", "teacher") for w in kinds], device=DEVICE)
    st["ids"][no_teacher] = -1
    st["labels"][no_label] = -1
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _turn_angles(case, pos):
    """Angles of every row and pair in 64 bits."""
    pairs, out, first = _pairs(case), [], 0
    for axis, n in enumerate(pairs):
        j = torch.arange(n, device=pos.device, dtype=torch.float64)
        theta = case["base"] ** (-(j / max(n, 1) if case["own_ladders"] else (first + j) / sum(pairs)))
        out.append(pos[:, axis:axis + 1].double() * theta)
        first += n
    return torch.cat(out, 1)


def _rotary_plain(st):
    case, x = st["case"], st["x"]
    heads, dh, n = case["q"] + case["kv"], case["dh"], sum(_pairs(case))
    angle = _turn_angles(case, st["positions"])
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if case["inverse"]:
        s = -s
    h = x[:, :heads * dh].reshape(-1, heads, dh).float()
    if case["interleaved"]:
        a, b = h[:, :, 0:2 * n:2], h[:, :, 1:2 * n:2]
    else:
        a, b = h[:, :, :n], h[:, :, n:2 * n]
    turned = torch.empty_like(h)
    if case["interleaved"]:
        turned[:, :, 0:2 * n:2] = a * c - b * s
        turned[:, :, 1:2 * n:2] = b * c + a * s
    else:
        turned[:, :, :n] = a * c - b * s
        turned[:, :, n:2 * n] = b * c + a * s
    turned[:, :, 2 * n:] = h[:, :, 2 * n:]
    return turned.reshape(-1, heads * dh).to(x.dtype)


def _stats(v, rms):
    m = torch.zeros_like(v[:, :1]) if rms else v.mean(1, keepdim=True)
    return m, 1.0 / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + 1e-5)


def _join_forward(st):
    case = st["case"]
    d = case["d"]
    x = st["x"].float()
    f = x[:, :d]
    m1, i1 = _stats(f, case["rms"])
    v = st["gain"] * ((f - m1) * i1)
    if case["gate"]:
        v = v / (1.0 + torch.exp(-x[:, d:]))
    y = (st["scale"] * st["r"].float() + v).to(st["x"].dtype)
    if not case["pre"]:
        return y, None, torch.cat([m1, i1, torch.zeros_like(m1), torch.zeros_like(m1)], 1)
    w = y.float()   # the next block's norm reads the result as it is stored
    m2, i2 = _stats(w, case["rms"])
    u = (w - m2) * i2 * st["pre_gain"]
    if not case["rms"]:
        u = u + st["pre_shift"]
    return y, u.to(y.dtype), torch.cat([m1, i1, m2, i2], 1)


def _norm_back(t, xhat, rstd, rms):
    t = t - xhat * (t * xhat).mean(1, keepdim=True) - (0.0 if rms else t.mean(1, keepdim=True))
    return t * rstd


def _join_backward(st):
    case, stats, t = st["case"], st["stats"], st["x"].dtype
    d, rms = case["d"], case["rms"]
    out = {}
    dh = st["dy"].float() if st["dy"] is not None else 0.0
    if case["pre"]:
        du = st["du"].float()
        yhat = (st["y"].float() - stats[:, 2:3]) * stats[:, 3:4]
        out["dpre_gain"] = (du * yhat).sum(0)
        if not rms:
            out["dpre_shift"] = du.sum(0)
        dh = dh + _norm_back(du * st["pre_gain"], yhat, stats[:, 3:4], rms)
    r = st["r"].float()
    out["dr"] = (dh * st["scale"]).to(t)
    out["dscale"] = (dh * r).sum(0)
    x = st["x"].float()
    fhat = (x[:, :d] - stats[:, 0:1]) * stats[:, 1:2]
    if case["gate"]:
        g = 1.0 / (1.0 + torch.exp(-x[:, d:]))
        da = dh * st["gain"] * fhat * (g * (1.0 - g))
        dh = dh * g
    out["dgain"] = (dh * fhat).sum(0)
    df = _norm_back(dh * st["gain"], fhat, stats[:, 1:2], rms)
    out["dx"] = (torch.cat([df, da], 1) if case["gate"] else df).to(t)
    return out


def _distill_plain(st):
    case, z = st["case"], st["logits"]
    T, alpha, rows = case["temperature"], case["alpha"], case["rows"]
    ids, teacher, labels = st["ids"].long(), st["teacher"], st["labels"].long()
    entry = ids >= 0
    taught, labelled = entry.any(1), labels >= 0
    at = ids.clamp(min=0)
    # the teacher's probabilities of its entries
    tl = torch.where(entry, teacher / T, torch.full_like(teacher, -math.inf))
    tm = torch.where(taught, tl.max(1).values, torch.zeros_like(tl[:, 0]))[:, None]
    e = torch.exp(tl - tm)
    total = torch.where(taught, e.sum(1), torch.ones_like(e[:, 0]))[:, None]
    p = e / total
    log_p = torch.where(entry, tl - tm - torch.log(total), torch.zeros_like(tl))
    zm = z - z.max(1, keepdim=True).values
    eq = torch.exp(zm / T)
    sq = eq.sum(1, keepdim=True)
    log_q = zm.gather(1, at) / T - torch.log(sq)
    loss = alpha * T * T * (p * (log_p - log_q)).sum(1)
    weight = (alpha * T) * taught.float()[:, None]
    g = eq * (weight / sq)
    g.scatter_add_(1, at, p * -(alpha * T))
    if alpha < 1.0:
        es = torch.exp(zm)
        ss = es.sum(1, keepdim=True)
        mine = labels.clamp(min=0)[:, None]
        on = labelled.float()[:, None]
        loss = loss + (1.0 - alpha) * (on * (torch.log(ss) - zm.gather(1, mine)))[:, 0]
        g += es * ((1.0 - alpha) * on / ss)
        g.scatter_add_(1, mine, -(1.0 - alpha) * on)
    return {"loss": loss, "dlogits": (g / rows).to(TYPES[case["dtype"]])}


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if not own:
        if case["op"] == "rotary":
            return _rotary_plain(st)
        if case["op"] == "distill":
            return _distill_plain(st)
        if case["backward"]:
            return _join_backward(st)
        y, u, _ = _join_forward(st)
        return {"y": y, "u": u} if case["pre"] else {"y": y}
    import paper_2410_14312_amd as tmps
    if case["op"] == "rotary":
        return tmps.rotary(st["x"], st["positions"], case["q"] + case["kv"], case["dh"], _pairs(case), base=case["base"],
                           interleaved=case["interleaved"], own_ladders=case["own_ladders"], inverse=case["inverse"])
    if case["op"] == "distill":
        loss, dlogits = tmps.distill(st["logits"], st["labels"], st["ids"], st["teacher"], temperature=case["temperature"], alpha=case["alpha"],
                                     grad_scale=1.0 / case["rows"], dtype=case["dtype"])
        return {"loss": loss, "dlogits": dlogits}
    if not case["backward"]:
        y, u, _ = tmps.norm_join(st["x"], st["r"], st["gain"], st["scale"], pre_gain=st["pre_gain"], pre_shift=st["pre_shift"],
                                 rms=case["rms"], gate=case["gate"])
        return {"y": y, "u": u} if case["pre"] else {"y": y}
    dx, dr, dgain, dscale, dpre_gain, dpre_shift = tmps.norm_join_backward(
        st["dy"], st["du"], st["x"], st["r"], st["y"], st["stats"], st["gain"], st["scale"], pre_gain=st["pre_gain"], rms=case["rms"],
        gate=case["gate"])
    out = {"dx": dx, "dr": dr, "dgain": dgain, "dscale": dscale}
    if case["pre"]:
        out["dpre_gain"] = dpre_gain
        if not case["rms"]:
            out["dpre_shift"] = dpre_shift
    return out


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotary":
        n = case["rows"] * (case["q"] + case["kv"])
        return {"bytes": 2 * n * case["dh"] * size + 12 * case["rows"], "flops": 6 * n * sum(_pairs(case))}
    rows = case["rows"]
    if case["op"] == "join":
        n, wide = rows * case["d"], 2 if case["gate"] else 1
        vectors = 2 + (case["pre"] and (1 if case["rms"] else 2))
        if not case["backward"]:   # x, r in; y, u and the statistics out
            return {"bytes": n * size * (wide + 2 + case["pre"]) + 16 * rows + 4 * vectors * case["d"], "flops": n * (8 + 4 * case["gate"] + 6 * case["pre"])}
        read = wide + 1 + 2 * case["pre"] + case["dy"]   # x, r; y and du; dy
        return {"bytes": n * size * (read + wide + 1) + 16 * rows + 8 * vectors * case["d"], "flops": n * (14 + 8 * case["gate"] + 12 * case["pre"])}
    live = sum(_distill_kind(r) != "none" and (case["alpha"] < 1.0 or _distill_kind(r) != "label") for r in range(rows))
    n = live * case["classes"]
    return {"bytes": 4 * n + rows * case["classes"] * size + rows * (8 * case["k"] + 8), "flops": n * (8 if case["alpha"] == 1.0 else 14)}


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        # a pair is a complex number, a turn a product with exp(i angle)
        heads, dh, n = case["q"] + case["kv"], case["dh"], sum(_pairs(case))
        turn = []
        for i in range(n):
            axis = 0 if i < _pairs(case)[0] else 1 if i < _pairs(case)[0] + _pairs(case)[1] else 2
            exponent = (i - sum(_pairs(case)[:axis])) / _pairs(case)[axis] if case["own_ladders"] else i / n
            turn.append(st["positions"][:, axis].double() * math.exp(-exponent * math.log(case["base"])))
        turn = torch.stack(turn, 1)
        turn = torch.polar(torch.ones_like(turn), -turn if case["inverse"] else turn)[:, None]
        out = st["x"][:, :heads * dh].double().view(-1, heads, dh).clone()
        if case["interleaved"]:
            v = torch.view_as_complex(out[:, :, :2 * n].reshape(-1, heads, n, 2)) * turn
            out[:, :, :2 * n] = torch.view_as_real(v).reshape(-1, heads, 2 * n)
        else:
            v = torch.complex(out[:, :, :n].contiguous(), out[:, :, n:2 * n].contiguous()) * turn
            out[:, :, :n], out[:, :, n:2 * n] = v.real, v.imag
        return out.reshape(-1, heads * dh)
    if case["op"] == "join":
        return _exact_join(case, st)
    return _exact_distill(case, st)


def _exact_norm(v, rms):
    if not rms:
        v = v - v.mean(1, keepdim=True)
    return v * (v.square().mean(1, keepdim=True) + 1e-5).rsqrt()


def _exact_join(case, st):
    d, t = case["d"], TYPES[case["dtype"]]
    leaf = {k: st[k].double().requires_grad_(case["backward"]) for k in ("x", "r", "gain", "scale", "pre_gain", "pre_shift") if st[k] is not None}
    with torch.enable_grad():
        y = leaf["gain"] * _exact_norm(leaf["x"][:, :d], case["rms"])
        if case["gate"]:
            y = y * torch.sigmoid(leaf["x"][:, d:])
        y = y + leaf["scale"] * leaf["r"]
        if not case["backward"]:
            out = {"y": y}
            if case["pre"]:
                out["u"] = leaf["pre_gain"] * _exact_norm(y.to(t).double(), case["rms"])
                if not case["rms"]:
                    out["u"] = out["u"] + leaf["pre_shift"]
            return out
        dh = st["dy"].double() if case["dy"] else torch.zeros_like(y)
        out = {}
        if case["pre"]:   # the norm read the stored result
            stored = st["y"].double().requires_grad_(True)
            u = leaf["pre_gain"] * _exact_norm(stored, case["rms"])
            if not case["rms"]:
                u = u + leaf["pre_shift"]
            wanted = [stored, leaf["pre_gain"]] + ([] if case["rms"] else [leaf["pre_shift"]])
            grads = torch.autograd.grad(u, wanted, st["du"].double())
            dh = dh + grads[0]
        dx, dr, dgain, dscale = torch.autograd.grad(y, [leaf["x"], leaf["r"], leaf["gain"], leaf["scale"]], dh)
    out.update(dx=dx, dr=dr, dgain=dgain, dscale=dscale)
    if case["pre"]:
        out["dpre_gain"] = grads[1]
        if not case["rms"]:
            out["dpre_shift"] = grads[2]
    return out


def _exact_distill(case, st):
    T, alpha, rows = case["temperature"], case["alpha"], case["rows"]
    loss = torch.zeros(rows, dtype=torch.float64, device=DEVICE)
    grad = torch.zeros(rows, case["classes"], dtype=torch.float64, device=DEVICE)
    step = max(1, (1 << 26) // case["classes"])
    for a in range(0, rows, step):
        part = slice(a, min(rows, a + step))
        ids, labels = st["ids"][part].long(), st["labels"][part].long()
        with torch.enable_grad():
            z = st["logits"][part].double().requires_grad_(True)
            log_q = torch.log_softmax(z / T, 1)
            log_p = torch.log_softmax(st["teacher"][part].double() / T, 1)
            kl = (log_p.exp() * (log_p - log_q.gather(1, ids.clamp(min=0)))).sum(1)
            ce = -torch.log_softmax(z, 1).gather(1, labels.clamp(min=0)[:, None])[:, 0]
            part_loss = alpha * T * T * torch.where(ids[:, 0] >= 0, kl, torch.zeros_like(kl)) + (1.0 - alpha) * torch.where(labels >= 0, ce, torch.zeros_like(ce))
            (g,) = torch.autograd.grad(part_loss.sum() / rows, [z])
        loss[part], grad[part] = part_loss.detach(), g
    return {"loss": loss, "dlogits": grad}
