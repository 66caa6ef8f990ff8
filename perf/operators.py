"""The operators of a softmax head trained on region descriptors, as cases to be measured: root-mean-square norm (with the
residual's addition, in 16, 32 or 8 bits) and its gradient, softmax cross entropy over a large vocabulary and its gradients,
and AdamW steps over many tensors (states in 32 or 8 bits).

``run`` computes the plain form (elementary torch operations in 32 bits, rounded once at the end), or calls the library's
operators where ``own`` is true.  ``exact`` is the same from the definitions in 64 bits.
"""
import math

import torch

own = False

F8_MAX = 448.0            # largest value of e4m3
EPS = 1e-6                # of the norm
BLOCK = 256               # values that share a scale in 8-bit optimiser states
ADAM = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "step": 100}
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
DN = {"f32": 0, "f16": 1, "bf16": 2, "f8": 3}

MAX_NORM = 32000 * 4096
MAX_LOSS = 16384 * 2048 * 65536
MAX_ADAM = 64_000_000


def listed():
    return [
        # one new row through a block's norm: latency only
        {"name": "norm_one_row", "op": "norm", "n": 1, "C": 4096, "dt": "bf16", "out": "bf16", "res": True, "block": 0, "pad": 0},
        # the descriptors of one image's 2000 regions (6 x 6 x 256, fp32), normalised and stored in 8 bits, one scale a row
        {"name": "norm_regions_8bit", "op": "norm", "n": 2000, "C": 9216, "dt": "f32", "out": "f8", "res": False, "block": 0, "pad": 0},
        # an odd number of rows of odd length, not aligned to vectors
        {"name": "norm_odd_f16", "op": "norm", "n": 8191, "C": 2047, "dt": "f16", "out": "f16", "res": True, "block": 0, "pad": 0},
        # gradient of the norm over a batch of 16 images' regions
        {"name": "norm_back_batch", "op": "norm_back", "n": 32000, "C": 4096, "dt": "bf16", "out": "bf16", "res": True, "pad": 0},
        # the loss of a single token: serving, a candidate answer scored
        {"name": "loss_one_token", "op": "loss", "n": 1, "C": 4096, "V": 32000, "dt": "bf16", "pad": 0, "masked": 0.0},
        # evaluation: one image's regions against an odd vocabulary, a tenth of them without a label
        {"name": "loss_eval_f16", "op": "loss", "n": 2000, "C": 2048, "V": 50257, "dt": "f16", "pad": 0, "masked": 0.1},
        # a training batch's gradients
        {"name": "loss_back_bf16", "op": "loss_back", "n": 4096, "C": 2048, "V": 32000, "dt": "bf16", "pad": 0, "masked": 0.1, "rows": False},
        # fp32 descriptors and weights, odd numbers of rows and words, a weight for each row
        {"name": "loss_back_f32", "op": "loss_back", "n": 1001, "C": 1024, "V": 10007, "dt": "f32", "pad": 0, "masked": 0.1, "rows": True},
        # the largest gradient: a long batch over a large vocabulary
        {"name": "loss_back_large", "op": "loss_back", "n": 16384, "C": 2048, "V": 65536, "dt": "bf16", "pad": 0, "masked": 0.0, "rows": False},
        # a head's few small tensors, stepped alone
        {"name": "adamw_small", "op": "adamw", "tensors": 4, "total": 40000, "dt": "f32", "grad": "bf16", "copy": True, "bits": 32, "align": 64},
        # a model's tensors, weights in fp32 with a bf16 copy for the products
        {"name": "adamw_32bit", "op": "adamw", "tensors": 160, "total": 64_000_000, "dt": "f32", "grad": "bf16", "copy": True, "bits": 32, "align": 64},
        # the same with states in 8 bits
        {"name": "adamw_8bit", "op": "adamw", "tensors": 160, "total": 64_000_000, "dt": "f32", "grad": "bf16", "copy": True, "bits": 8, "align": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_back", "loss", "loss_back", "adamw"])
    dt = rng.choice(["bf16", "f16", "f32"])
    if op == "adamw":
        return {"op": op, "tensors": _log(rng, 1, 200), "total": _log(rng, 1000, MAX_ADAM), "dt": rng.choice(["f32", "f32", "bf16", "f16"]),
                "grad": dt, "copy": rng.random() < 0.5, "bits": rng.choice([32, 8]), "align": rng.choice([64, 64, 1])}
    n = _log(rng, 1, 32000 if op.startswith("norm") else 16384)
    C = _log(rng, 16, 9216)
    if rng.random() < 0.5:  # half of them whole numbers of vectors
        C = (C + 15) // 16 * 16
    pad = rng.choice([0, 0, 8, 3])
    if op.startswith("norm"):
        n = max(1, min(n, MAX_NORM // C))
        case = {"op": op, "n": n, "C": C, "dt": dt, "out": rng.choice(["bf16", "f16", "f32"]), "res": rng.random() < 0.6, "pad": pad}
        if op == "norm":
            case["out"] = rng.choice([case["out"], "f8"])
            case["block"] = rng.choice([0, 32, 128]) if case["out"] == "f8" else 0
        return case
    V = max(2, min(_log(rng, 100, 131072), MAX_LOSS // (n * C)))
    case = {"op": op, "n": n, "C": C, "V": V, "dt": dt, "pad": pad, "masked": rng.choice([0.0, 0.1, 0.5])}
    if op == "loss_back":
        case["rows"] = rng.random() < 0.5
    return case


def _sizes(case):
    """Sizes of a case's tensors: every fourth a short vector, the rest matrices of uneven sizes, adding up to about `total`."""
    k, total = case["tensors"], case["total"]
    share = [0.01 if i % 4 == 3 else 1.0 + (i * 7 % 5) for i in range(k)]
    return [max(1, int(total * s / sum(share)) - i % 3) for i, s in enumerate(share)]


def _offsets(sizes, align):
    at, offs = 0, []
    for n in sizes:
        offs.append(at)
        at += (n + align - 1) // align * align
    return offs, at


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, n, C, dt, pad, scale=1.0):
    """[n][C] of normal values in a buffer whose rows are C + pad apart."""
    return (torch.randn(n, C + pad, generator=g, device="cuda") * scale).to(DT[dt])[:, :C]


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op in ("norm", "norm_back"):
        n, C, dt, pad = case["n"], case["C"], case["dt"], case["pad"]
        s = {"case": case, "x": _rows(g, n, C, dt, pad, 2.0), "gamma": 1 + 0.2 * torch.randn(C, generator=g, device="cuda")}
        if op == "norm":
            s["res"] = _rows(g, n, C, dt, pad) if case["res"] else None
        else:
            s["dy"] = _rows(g, n, C, case["out"], pad)
            s["dsum"] = _rows(g, n, C, dt, pad) if case["res"] else None
        return s
    if op in ("loss", "loss_back"):
        n, C, V, dt, pad = case["n"], case["C"], case["V"], case["dt"], case["pad"]
        s = {"case": case, "h": _rows(g, n, C, dt, pad), "w": _rows(g, V, C, dt, pad, 2.0 / math.sqrt(C))}
        labels = torch.randint(0, V, (n,), generator=g, device="cuda")
        s["labels"] = torch.where(torch.rand(n, generator=g, device="cuda") < case["masked"], -1, labels)
        if op == "loss_back":  # the forward pass has been there: its log-sums are in hand
            s["lse"] = torch.cat([torch.logsumexp(a.double() @ s["w"].T.double(), 1).float() for a in s["h"].split(max(1, (1 << 28) // V))])
            s["dloss"] = torch.rand(n, generator=g, device="cuda") / n if case["rows"] else None
        return s
    sizes = _sizes(case)
    offs, total = _offsets(sizes, case["align"])
    blocks, held = _offsets(sizes, BLOCK)
    views = lambda flat: [flat[o:o + n] for o, n in zip(offs, sizes)]  # noqa: E731
    s = {"case": case, "sizes": sizes, "blocks": blocks, "seed": seed & 0x7FFFFFFF}
    s["flat_p"] = (0.05 * torch.randn(total, generator=g, device="cuda")).to(DT[case["dt"]])
    s["flat_g"] = (0.01 * torch.randn(total, generator=g, device="cuda")).to(DT[case["grad"]])
    s["flat_copy"] = s["flat_p"].to(torch.bfloat16) if case["copy"] else None
    s["p"], s["g"] = views(s["flat_p"]), views(s["flat_g"])
    s["copy"] = views(s["flat_copy"]) if case["copy"] else None
    inside = torch.zeros(held, dtype=torch.bool, device="cuda")
    for o, n in zip(blocks, sizes):
        inside[o:o + n] = True
    m = torch.where(inside, 0.003 * torch.randn(held, generator=g, device="cuda"), 0.0)
    r = torch.where(inside, 0.01 * torch.rand(held, generator=g, device="cuda") + 1e-4, 0.0)
    if case["bits"] == 32:
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, r * r, None, None
    else:
        s["m_scale"], s["v_scale"] = (t.view(-1, BLOCK).abs().amax(1) / F8_MAX for t in (m, r))
        s["m"], s["v"] = ((t.view(-1, BLOCK) / k[:, None]).to(DT["f8"]).view(-1) for t, k in ((m, s["m_scale"]), (r, s["v_scale"])))
    if own:  # the handle that a training program keeps beside its tensors: their addresses and sizes
        from paper_1404_1869_amd import densenet as D
        s["plan"] = D.AdamWPlan(s["p"], s["g"], s["m"], s["v"], m_scale=s["m_scale"], v_scale=s["v_scale"], copies=s["copy"])
    return s


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _norm(s):
    case = s["case"]
    a = s["x"].float()
    if s["res"] is not None:
        a = a + s["res"].float()
    y = a * torch.rsqrt(a.square().mean(1, keepdim=True) + EPS) * s["gamma"]
    out = {"sum": a.to(DT[case["dt"]]) if s["res"] is not None else None}
    if case["out"] != "f8":
        return {**out, "y": y.to(DT[case["out"]])}
    n, C = y.shape
    b = case["block"] or C
    k = -(-C // b)
    y = torch.nn.functional.pad(y, (0, k * b - C)).view(n, k, b)
    scale = y.abs().amax(2) / F8_MAX
    q = (y / torch.where(scale > 0, scale, 1.0)[:, :, None]).clamp(-F8_MAX, F8_MAX)
    return {**out, "y": q.view(n, k * b)[:, :C].to(DT["f8"]), "scale": scale}


def _norm_back(s):
    x, dy = s["x"].float(), s["dy"].float()
    q = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    a = dy * s["gamma"]
    dx = q * (a - x * (q * q) * (a * x).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * x * q).sum(0)}


def _loss(s):
    logits = s["h"].float() @ s["w"].float().T
    top = logits.amax(1, keepdim=True)
    lse = (logits - top).exp().sum(1).log() + top[:, 0]
    has = s["labels"] >= 0
    at = logits.gather(1, s["labels"].clamp(min=0)[:, None])[:, 0]
    return {"loss": torch.where(has, lse - at, 0.0), "lse": torch.where(has, lse, 0.0)}


def _loss_back(s):
    has = s["labels"] >= 0
    h, w = s["h"].float(), s["w"].float()
    p = (h @ w.T).sub_(s["lse"][:, None]).exp_()
    p.scatter_add_(1, s["labels"].clamp(min=0)[:, None], torch.full_like(p[:, :1], -1.0))
    c = s["dloss"] if s["dloss"] is not None else 1.0 / has.sum().clamp(min=1)
    p *= torch.where(has, c, 0.0)[:, None]
    return {"dh": (p @ w).to(s["h"].dtype), "dw": (p.T @ h).to(s["w"].dtype)}


def _noise(count, seed, device):
    """32 bits for each index 0 .. count - 1: a multiplicative hash of the index and the seed."""
    x = (torch.arange(count, dtype=torch.int64, device=device) * 0x9E3779B1 + seed) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF
    x = ((x ^ (x >> 12)) * 0x297A2D39) & 0xFFFFFFFF
    return x ^ (x >> 15)


def _round8(a, bits):
    """a in [0, 448] to the e4m3 value below or above it, above with the chance of its place between them; bits: 16 random ones."""
    small = torch.floor(a * 512 + bits.float() * 2.0 ** -16) * 2.0 ** -9
    large = ((a.view(torch.int32) + (bits.int() << 4)) & ~0xFFFFF).view(torch.float32)
    return torch.where(a < 2.0 ** -6, small, large)


def _store8(t, bits, floor):
    """[blocks][256] to e4m3 values and scales; floor: what is above 0 stays above 0."""
    top = t.abs().amax(1)
    scale = top / F8_MAX
    q = _round8((t.abs() * torch.where(top > 0, F8_MAX / top, 0.0)[:, None]).clamp(max=F8_MAX), bits)
    if floor:
        q = torch.where(t > 0, q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, t).to(DT["f8"]), scale


def _adamw(s):
    case, sizes, k = s["case"], s["sizes"], ADAM
    rate, root = k["lr"] / (1 - k["beta1"] ** k["step"]), 1 / math.sqrt(1 - k["beta2"] ** k["step"])
    if case["bits"] == 32:
        g = [t.float() for t in s["g"]]
        m, v = ([t[o:o + n] for o, n in zip(s["blocks"], sizes)] for t in (s["m"], s["v"]))
        torch._foreach_mul_(m, k["beta1"])
        torch._foreach_add_(m, g, alpha=1 - k["beta1"])
        torch._foreach_mul_(v, k["beta2"])
        torch._foreach_addcmul_(v, g, g, value=1 - k["beta2"])
        d = torch._foreach_sqrt(v)
        torch._foreach_mul_(d, root)
        torch._foreach_add_(d, k["eps"])
        p = [t.float() for t in s["p"]] if case["dt"] != "f32" else s["p"]
        torch._foreach_mul_(p, 1 - k["lr"] * k["weight_decay"])
        torch._foreach_addcdiv_(p, m, d, value=-rate)
    else:
        blocks = lambda ts: torch.cat([torch.nn.functional.pad(t.float(), (0, -t.numel() % BLOCK)) for t in ts]).view(-1, BLOCK)  # noqa: E731
        g, p = blocks(s["g"]), blocks(s["p"])
        m = s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]
        r = s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]
        m = m * k["beta1"] + g * (1 - k["beta1"])
        v = r * r * k["beta2"] + g * g * (1 - k["beta2"])
        r = v.sqrt()
        p = p * (1 - k["lr"] * k["weight_decay"]) - rate * m / (r * root + k["eps"])
        bits = _noise(m.numel(), s["seed"], m.device).view(-1, BLOCK)
        for name, t, b, floor in (("m", m, bits >> 16, False), ("v", r, bits & 0xFFFF, True)):
            q, scale = _store8(t, b, floor)
            s[name].copy_(q.view(-1))
            s[name + "_scale"].copy_(scale)
        p = p.view(-1)
        p = [p[o:o + n] for o, n in zip(s["blocks"], sizes)]
    if p is not s["p"]:
        torch._foreach_copy_(s["p"], p)
    if s["copy"] is not None:
        torch._foreach_copy_(s["copy"], p)
    return _state(s)


def _state(s):
    return {"p": s["flat_p"], "copy": s["flat_copy"], "m": s["m"], "v": s["v"], "m_scale": s["m_scale"], "v_scale": s["v_scale"]}


def _own(s):
    from paper_1404_1869_amd import densenet as D
    case = s["case"]
    op = case["op"]
    if op == "norm":
        y, total, scale = D.densenet_rms_norm(s["x"], s["gamma"], residual=s["res"], eps=EPS, out_dtype=DN[case["out"]], block=case["block"])
        return {"y": y, "sum": total, "scale": scale}
    if op == "norm_back":
        dx, dgamma = D.densenet_rms_norm_backward(s["dy"], s["x"], s["gamma"], dsum=s["dsum"], eps=EPS)
        return {"dx": dx, "dgamma": dgamma}
    if op == "loss":
        loss, lse = D.densenet_softmax_loss(s["h"], s["w"], s["labels"])
        return {"loss": loss, "lse": lse}
    if op == "loss_back":
        dh, dw = D.densenet_softmax_loss_backward(s["h"], s["w"], s["labels"], s["lse"], dloss=s["dloss"])
        return {"dh": dh, "dw": dw}
    D.densenet_adamw(s["plan"], lr=ADAM["lr"], beta1=ADAM["beta1"], beta2=ADAM["beta2"], eps=ADAM["eps"],
                     weight_decay=ADAM["weight_decay"], step=ADAM["step"], seed=s["seed"])
    return _state(s)


def run(state):
    if own:
        return _own(state)
    return {"norm": _norm, "norm_back": _norm_back, "loss": _loss, "loss_back": _loss_back, "adamw": _adamw}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# The work of a pass, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}
    op = case["op"]
    if op in ("norm", "norm_back"):
        nC, e, o = case["n"] * case["C"], size[case["dt"]], size[case["out"]]
        if op == "norm":
            scales = case["n"] * -(-case["C"] // (case["block"] or case["C"])) if case["out"] == "f8" else 0
            return {"bytes": nC * (e * (3 if case["res"] else 1) + o) + 4 * (case["C"] + scales), "flops": 5 * nC}
        return {"bytes": nC * (e * (3 if case["res"] else 2) + o) + 8 * case["C"], "flops": 12 * nC}
    if op in ("loss", "loss_back"):
        n, C, V, e = case["n"], case["C"], case["V"], size[case["dt"]]
        if op == "loss":
            return {"bytes": (n + V) * C * e + 16 * n, "flops": 2 * n * V * C}
        return {"bytes": 2 * (n + V) * C * e + (16 if case["rows"] else 12) * n, "flops": 6 * n * V * C}
    count = sum(_sizes(case))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": count * (2 * size[case["dt"]] + size[case["grad"]] + state + (2 if case["copy"] else 0)), "flops": 16 * count}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        a = s["x"].double() if s["res"] is None else s["x"].double() + s["res"].double()
        y = s["gamma"].double() * a / (EPS + (a * a).sum(1, keepdim=True) / case["C"]).sqrt()
        out = {"sum": None if s["res"] is None else a, "y": y}
        if case["out"] == "f8":
            b, C = case["block"] or case["C"], case["C"]
            parts = [y[:, i:i + b] for i in range(0, C, b)]
            tops = [t.abs().max(1, keepdim=True).values for t in parts]
            out["y"] = torch.cat([torch.nan_to_num(t / (k / F8_MAX)) for t, k in zip(parts, tops)], 1).to(DT["f8"])
            out["scale"] = torch.cat(tops, 1) / F8_MAX
        return out
    if op == "norm_back":
        x, dy, w = s["x"].double(), s["dy"].double(), s["gamma"].double()
        C = case["C"]
        size = (EPS + (x * x).sum(1, keepdim=True) / C).sqrt()
        unit = x / size
        dx = (dy * w - unit * ((dy * w * unit).sum(1, keepdim=True) / C)) / size
        return {"dx": dx if s["dsum"] is None else dx + s["dsum"].double(), "dgamma": (dy * unit).sum(0)}
    if op == "loss":
        w, found = s["w"].double(), []
        for h, t in zip(s["h"].split(4096), s["labels"].split(4096)):
            logits = h.double() @ w.T
            lse = torch.logsumexp(logits, 1)
            rows = torch.arange(len(t), device=t.device)
            found.append(torch.stack([lse - logits[rows, t.clamp(min=0)], lse]) * (t >= 0))
        found = torch.cat(found, 1)
        return {"loss": found[0], "lse": found[1]}
    if op == "loss_back":
        w, h, t = s["w"].double(), s["h"].double(), s["labels"]
        has = t >= 0
        weight = (s["dloss"].double() if s["dloss"] is not None else torch.ones_like(t, dtype=torch.float64) / max(1, int(has.sum()))) * has
        dh, dw, lse = torch.empty_like(h), torch.zeros_like(w), s["lse"].double()
        step = 4096
        for i in range(0, case["n"], step):
            p = (h[i:i + step] @ w.T - lse[i:i + step, None]).exp()
            rows = torch.arange(len(p), device=t.device)
            p[rows, t[i:i + step].clamp(min=0)] -= 1
            p *= weight[i:i + step, None]
            dh[i:i + step] = p @ w
            dw += p.T @ h[i:i + step]
        return {"dh": dh, "dw": dw}
    k = {a: float(b) for a, b in ADAM.items()}
    out = {"p": s["flat_p"].double(), "copy": None, "m": s["m"].double(), "v": s["v"].double(), "m_scale": None, "v_scale": None}
    bits8 = case["bits"] == 8
    if bits8:
        out["m_scale"], out["v_scale"] = s["m_scale"].double(), s["v_scale"].double()
        hashed = torch.arange(s["m"].numel(), dtype=torch.int64, device="cuda").mul(0x9E3779B1).add(s["seed"]).bitwise_and(0xFFFFFFFF)
        for shift, factor in ((15, 0x2C1B3C6D), (12, 0x297A2D39)):
            hashed = hashed.bitwise_xor(hashed >> shift).mul(factor).bitwise_and(0xFFFFFFFF)
        hashed = hashed.bitwise_xor(hashed >> 15)
        chance = {"m": (hashed >> 16).double() / 65536, "v": (hashed & 0xFFFF).double() / 65536}
    offs, _ = _offsets(s["sizes"], case["align"])
    for o, b, n, g in zip(offs, s["blocks"], s["sizes"], s["g"]):
        g, held = g.double(), -(-n // BLOCK)
        at, own_blocks = slice(b, b + n), slice(b // BLOCK, b // BLOCK + held)
        m, v = out["m"][at], out["v"][at]
        if bits8:
            wide = lambda name: out[name][own_blocks].repeat_interleave(BLOCK)[:n]  # noqa: E731
            m, v = m * wide("m_scale"), (v * wide("v_scale")) ** 2
        m, v = m + (1 - k["beta1"]) * (g - m), v + (1 - k["beta2"]) * (g * g - v)
        p = out["p"][o:o + n]
        step = m / (1 - k["beta1"] ** k["step"]) / ((v / (1 - k["beta2"] ** k["step"])).sqrt() + k["eps"])
        out["p"][o:o + n] = p - k["lr"] * (step + k["weight_decay"] * p)
        if not bits8:
            out["m"][at], out["v"][at] = m, v
            continue
        for name, t in (("m", m), ("v", v.sqrt())):
            whole = torch.zeros(held * BLOCK, dtype=torch.float64, device="cuda")
            whole[:n] = t
            top = whole.view(-1, BLOCK).abs().max(1).values
            a = whole.abs() / (top / F8_MAX).clamp(min=1e-300).repeat_interleave(BLOCK)
            fine = 2.0 ** (torch.frexp(a.clamp(min=2.0 ** -6))[1].double() - 4)
            q = torch.floor(a / fine + chance[name][b:b + held * BLOCK]) * fine
            if name == "v":
                q = torch.where(whole > 0, q.clamp(min=2.0 ** -9), q)
            out[name][b:b + held * BLOCK] = q.clamp(max=F8_MAX) * whole.sign()
            out[name + "_scale"][own_blocks] = top / F8_MAX
    if case["copy"]:
        out["copy"] = s["flat_copy"].double()
        for o, n in zip(offs, s["sizes"]):
            out["copy"][o:o + n] = out["p"][o:o + n]
    return out
