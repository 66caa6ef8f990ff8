"""The operators of a head that learns and answers in 8 bits, as cases to be measured: rows and weights to e4m3 with a scale for
every block of 128, along both axes at once; matrix products of such operands; log probability of a given token, entropy and best
alternatives of each row of logits, with their gradient; and Muon steps, which orthogonalise a matrix's update by Newton-Schulz
products.

``run`` computes the plain form (elementary torch operations in 32 bits, rounded once at the end), or calls the library's
operators where ``own`` is true.  ``exact`` is the same from the definitions in 64 bits.
"""
import math

import torch

own = False

F8_MAX = 448.0            # largest value of e4m3
BLOCK = 128               # values, or rows and values, that share a scale
MUON = {"lr": 0.02, "momentum": 0.95, "weight_decay": 0.01, "eps": 1e-7, "a": 3.4445, "b": -4.7750, "c": 2.0315, "steps": 5}
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
DN = {"f32": 0, "f16": 1, "bf16": 2, "f8": 3}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}

MAX_QUANT = 32000 * 8192
MAX_PRODUCT = 16384 * 4096 * 16384
MAX_SCORES = 4096 * 65536
MAX_MUON = 6 * (3 * 2048 * 2048 * 8192 + 2048 ** 3)


def listed():
    return [
        # the words of a large head, quantised after each step: squares of 128 x 128, along rows for the logits and turned for dh
        {"name": "quant_words", "op": "quant", "n": 32000, "C": 4096, "dt": "bf16", "rows": 128, "turned": True, "pad": 0},
        # an odd batch's gradient of odd rows, in blocks along the row for dh and, turned, along the batch for dw
        {"name": "quant_grad_odd", "op": "quant", "n": 2001, "C": 10007, "dt": "bf16", "rows": 1, "turned": True, "pad": 3},
        # serving: the logits of one row
        {"name": "product_one_row", "op": "product", "n": 1, "C": 4096, "V": 32000, "out": "bf16"},
        # the descriptors of one image's 2000 regions (6 x 6 x 256) over an odd vocabulary
        {"name": "product_regions", "op": "product", "n": 2000, "C": 9216, "V": 10007, "out": "bf16"},
        # a training batch's product, the largest
        {"name": "product_large", "op": "product", "n": 16384, "C": 4096, "V": 16384, "out": "bf16"},
        # serving: the answer of one row, with 20 alternatives
        {"name": "scores_one_row", "op": "scores", "n": 1, "V": 131072, "dt": "bf16", "top": 20, "scale": 1.25, "masked": 0.1, "pad": 0},
        # evaluation: one image's 2000 regions over an odd vocabulary, with 5 alternatives
        {"name": "scores_eval_f16", "op": "scores", "n": 2000, "V": 50257, "dt": "f16", "top": 5, "scale": 1.0, "masked": 0.0, "pad": 0},
        # a training batch's gradient: of log probabilities and entropy, as a policy is trained
        {"name": "scores_back_bf16", "op": "scores_back", "n": 4096, "V": 32000, "dt": "bf16", "top": 0, "scale": 1.0, "masked": 0.1, "pad": 0},
        # fp32 logits, an odd vocabulary, and a gradient of the alternatives too, as one model learns from another's
        {"name": "scores_back_f32", "op": "scores_back", "n": 333, "V": 50257, "dt": "f32", "top": 8, "scale": 0.5, "masked": 0.0, "pad": 0},
        # a few small matrices, stepped together
        {"name": "muon_small", "op": "muon", "tensors": 4, "R": 96, "C": 256, "dt": "f32", "grad": "bf16", "copy": True},
        # the weights of a head of 1000 classes on region descriptors, in fp32 with a bf16 copy for the products
        {"name": "muon_head", "op": "muon", "tensors": 1, "R": 1000, "C": 9216, "dt": "f32", "grad": "bf16", "copy": True},
        # a model's matrices, kept in bf16
        {"name": "muon_model", "op": "muon", "tensors": 6, "R": 2048, "C": 8192, "dt": "bf16", "grad": "bf16", "copy": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quant", "product", "product", "scores", "scores_back", "muon"])
    dt = rng.choice(["bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 8, 3])
    if op == "muon":
        R, C, k = _log(rng, 16, 4096), _log(rng, 16, 9216), _log(rng, 1, 16)
        case = {"op": op, "tensors": k, "R": R, "C": C, "dt": rng.choice(["f32", "f32", "bf16", "f16"]), "grad": dt, "copy": rng.random() < 0.5}
        while _muon_flops(case) > MAX_MUON:
            case["tensors" if case["tensors"] > 1 else "C" if case["C"] > case["R"] else "R"] //= 2
        return case
    if op in ("scores", "scores_back"):
        V = _log(rng, 100, 200000)
        n = max(1, min(_log(rng, 1, 16384), MAX_SCORES // V))
        return {"op": op, "n": n, "V": V, "dt": dt, "top": rng.choice([0, 1, 5, 20, 64]), "scale": rng.choice([1.0, 0.5, 1.25]),
                "masked": rng.choice([0.0, 0.1, 0.5]), "pad": pad}
    C = _log(rng, 16, 9216)
    if rng.random() < 0.5:  # half of them whole numbers of vectors
        C = (C + 15) // 16 * 16
    if op == "quant":
        n = max(1, min(_log(rng, 1, 65536), MAX_QUANT // C))
        return {"op": op, "n": n, "C": C, "dt": dt, "rows": rng.choice([1, 128]), "turned": rng.random() < 0.7, "pad": pad}
    n = _log(rng, 1, 16384)
    return {"op": op, "n": n, "C": C, "V": max(1, min(_log(rng, 16, 65536), MAX_PRODUCT // (n * C))), "out": dt}


def _shapes(case):
    """Shapes of a case's matrices: every second lies on its side, and each is a little smaller than the one before."""
    k = case["tensors"]
    sides = [(max(1, case["R"] - 3 * i), max(1, case["C"] - 5 * i)) for i in range(k)]
    return [s if i % 2 == 0 else s[::-1] for i, s in enumerate(sides)]


def _muon_flops(case):
    total = 0
    for s in _shapes(case):
        r, c = sorted(s)
        total += 3 * r * r * c + r ** 3  # X X', of which half is the other half's mirror, its square, likewise, and B X
    return total


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, n, C, dt, pad, scale=1.0):
    """[n][C] of normal values in a buffer whose rows are C + pad apart, rows and columns of uneven size."""
    x = torch.randn(n, C + pad, generator=g, device="cuda") * scale
    x *= torch.exp(0.5 * torch.randn(n, 1, generator=g, device="cuda"))
    x *= torch.exp(0.5 * torch.randn(C + pad, generator=g, device="cuda"))
    return x.to(DT[dt])[:, :C]


def _grid(x, rows):
    """x, with zeros around it, as [blocks of rows][rows][blocks of values][BLOCK]."""
    n, C = x.shape
    x = torch.nn.functional.pad(x, (0, -C % BLOCK, 0, -n % rows))
    return x.view(x.shape[0] // rows, rows, x.shape[1] // BLOCK, BLOCK)


def _quantize(x, rows):
    """Codes and scales of x [n][C], a scale for every `rows` x BLOCK values."""
    n, C = x.shape
    b = _grid(x.float(), rows)
    scale = b.abs().amax((1, 3)) / F8_MAX
    q = (b / torch.where(scale > 0, scale, 1.0)[:, None, :, None]).clamp(-F8_MAX, F8_MAX)
    return q.reshape(-1, q.shape[2] * BLOCK)[:n, :C].to(DT["f8"]), scale


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "quant":
        return {"case": case, "x": _rows(g, case["n"], case["C"], case["dt"], case["pad"], 0.02)}
    if op == "product":
        n, C, V = case["n"], case["C"], case["V"]
        a, a_scale = _quantize(_rows(g, n, C, "bf16", 0), 1)
        w, w_scale = _quantize(_rows(g, V, C, "bf16", 0, 2.0 / math.sqrt(C)), BLOCK)
        row = -(-C // 16) * 16  # codes lie in rows of whole vectors, as a program that quantises them keeps them
        lay = lambda t: torch.nn.functional.pad(t.view(torch.uint8), (0, row - C)).view(DT["f8"])[:, :C]  # noqa: E731
        return {"case": case, "a": lay(a), "a_scale": a_scale, "w": lay(w), "w_scale": w_scale}
    if op in ("scores", "scores_back"):
        n, V, k, pad = case["n"], case["V"], case["top"], case["pad"]
        x = 2.5 * torch.randn(n, V + pad, generator=g, device="cuda")
        x[torch.rand(n, V + pad, generator=g, device="cuda") < case["masked"]] = -math.inf  # words that may not be said
        keep = torch.randint(0, V, (n,), generator=g, device="cuda")
        x[torch.arange(n, device="cuda"), keep] = 3.0 + torch.randn(n, generator=g, device="cuda")  # one that may
        s = {"case": case, "x": x.to(DT[case["dt"]])[:, :V]}
        token = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, keep, torch.randint(0, V, (n,), generator=g, device="cuda"))
        token = torch.where(s["x"].gather(1, token[:, None])[:, 0] == -math.inf, keep, token)
        s["token"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, -1, token)  # rows without a given token
        if op == "scores_back":  # the forward pass has been there
            z = torch.cat([_answer(t, case) for t in s["x"].split(max(1, (1 << 26) // V))])
            s["lse"], s["entropy"] = z[:, 0].contiguous(), z[:, 1].contiguous()
            s["dlogp"] = torch.randn(n, generator=g, device="cuda") / n
            s["dentropy"] = 0.01 * torch.randn(n, generator=g, device="cuda") / n
            s["top_id"] = s["dtop"] = None
            if k:
                s["top_id"], s["dtop"] = _top(s["x"], k), torch.rand(n, k, generator=g, device="cuda") / n
        return s
    shapes = _shapes(case)
    s = {"case": case, "shapes": shapes, "rates": [0.2 * math.sqrt(max(r)) for r in shapes]}
    s["p"] = [(0.02 * torch.randn(r, generator=g, device="cuda")).to(DT[case["dt"]]) for r in shapes]
    # gradients of a few strong directions and noise, as a batch gives them
    s["g"], s["m"] = [], []
    for r, c in shapes:
        k = min(r, c, 16)
        strong = torch.randn(r, k, generator=g, device="cuda") @ torch.randn(k, c, generator=g, device="cuda")
        s["g"].append((1e-4 * strong + 1e-4 * torch.randn(r, c, generator=g, device="cuda")).to(DT[case["grad"]]))
        s["m"].append(1e-3 * strong + 5e-4 * torch.randn(r, c, generator=g, device="cuda"))
    s["copy"] = [t.to(torch.bfloat16) for t in s["p"]] if case["copy"] else None
    if own:  # the handle that a training program keeps beside its tensors: their addresses, sizes and workspace
        from paper_1404_1869_amd import densenet as D
        s["plan"] = D.MuonPlan(s["p"], s["g"], s["m"], copies=s["copy"], rates=s["rates"])
    return s


def _answer(x, case):
    """[n][2]: log of the sum of exponentials, and entropy, in 64 bits, of a few rows."""
    x = x.double() * case["scale"]
    lse = torch.logsumexp(x, 1, keepdim=True)
    return torch.cat([lse, -torch.special.xlogy((x - lse).exp(), (x - lse).exp()).sum(1, keepdim=True)], 1).float()


def _top(x, k):
    """Places of the k largest values of each row, the lower place first among equals; -1 where only -infinity is left."""
    found = []
    for t in x.split(max(1, (1 << 27) // x.shape[1])):
        v, at = t.sort(dim=1, descending=True, stable=True)
        at = torch.where(v == -math.inf, -1, at)[:, :k]
        found.append(torch.nn.functional.pad(at, (0, k - at.shape[1]), value=-1))
    return torch.cat(found).contiguous()


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _quant(s):
    case = s["case"]
    x = s["x"].float()
    codes, scale = _quantize(x, case["rows"])
    out = {"codes": codes, "scale": scale, "turned": None, "turned_scale": None}
    if case["turned"] and case["rows"] == 1:
        out["turned"], out["turned_scale"] = _quantize(x.T, 1)
    elif case["turned"]:
        out["turned"], out["turned_scale"] = codes.view(torch.uint8).T.contiguous().view(DT["f8"]), scale.T.contiguous()
    return out


def _wide(q, scale, rows):
    """Codes times their scales in 32 bits."""
    n, C = q.shape
    return (_grid(q.float(), rows) * scale[:, None, :, None]).view(-1, scale.shape[1] * BLOCK)[:n, :C]


def _product(s):
    y = _wide(s["a"], s["a_scale"], 1) @ _wide(s["w"], s["w_scale"], BLOCK).T
    return {"y": y.to(DT[s["case"]["out"]])}


def _scores(s):
    case = s["case"]
    x = s["x"].float() * case["scale"]
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    z = e.sum(1)
    lse = z.log() + top[:, 0]
    mean = torch.where(e > 0, e * (x - top), 0.0).sum(1) / z
    has = s["token"] >= 0
    at = x.gather(1, s["token"].clamp(min=0)[:, None])[:, 0]
    out = {"logp": torch.where(has, at - lse, 0.0), "entropy": z.log() - mean, "lse": lse, "top_id": None, "top_logp": None}
    if case["top"]:
        out["top_id"] = _top(s["x"], case["top"])
        got = x.gather(1, out["top_id"].clamp(min=0)) - lse[:, None]
        out["top_logp"] = torch.where(out["top_id"] >= 0, got, -math.inf)
    return out


def _scores_back(s):
    case = s["case"]
    logp = s["x"].float() * case["scale"] - s["lse"][:, None]
    p = logp.exp()
    has = s["token"] >= 0
    dlogp = torch.where(has, s["dlogp"], 0.0)[:, None]
    held = dlogp
    if s["dtop"] is not None:
        dtop = torch.where(s["top_id"] >= 0, s["dtop"], 0.0)
        held = held + dtop.sum(1, keepdim=True)
    d = torch.where(p > 0, -p * (held + s["dentropy"][:, None] * (logp + s["entropy"][:, None])), 0.0)
    d.scatter_add_(1, s["token"].clamp(min=0)[:, None], dlogp)
    if s["dtop"] is not None:
        d.scatter_add_(1, s["top_id"].clamp(min=0), dtop)
    return {"dx": (d * case["scale"]).to(s["x"].dtype)}


def _orthogonal(u):
    """Newton-Schulz steps towards the nearest matrix of orthogonal rows (or columns, where those are fewer)."""
    k = MUON
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (x.square().sum().sqrt() + k["eps"])
    for _ in range(k["steps"]):
        a = x @ x.T
        x = k["a"] * x + (k["b"] * a + k["c"] * (a @ a)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def _muon(s):
    k = MUON
    for i, (p, g, m) in enumerate(zip(s["p"], s["g"], s["m"])):
        m.mul_(k["momentum"]).add_(g.float())
        o = _orthogonal(g.float() + k["momentum"] * m)
        new = p.float() * (1 - k["lr"] * k["weight_decay"]) - (k["lr"] * s["rates"][i]) * o
        p.copy_(new)
        if s["copy"] is not None:
            s["copy"][i].copy_(new)
    return _state(s)


def _state(s):
    return {"p": s["p"], "m": s["m"], "copy": s["copy"]}


def _own(s):
    from paper_1404_1869_amd import densenet as D
    case = s["case"]
    op = case["op"]
    if op == "quant":
        codes, scale, turned, turned_scale = D.densenet_quantize_blocks(s["x"], rows=case["rows"], turned=case["turned"])
        return {"codes": codes, "scale": scale, "turned": turned, "turned_scale": turned_scale}
    if op == "product":
        return {"y": D.densenet_block_product(s["a"], s["a_scale"], s["w"], s["w_scale"], out_dtype=DN[case["out"]])}
    if op == "scores":
        logp, entropy, lse, top_id, top_logp = D.densenet_token_scores(s["x"], s["token"], top=case["top"], scale=case["scale"])
        return {"logp": logp, "entropy": entropy, "lse": lse, "top_id": top_id, "top_logp": top_logp}
    if op == "scores_back":
        dx = D.densenet_token_scores_backward(s["x"], s["token"], s["lse"], entropy=s["entropy"], dlogp=s["dlogp"],
                                              dentropy=s["dentropy"], top_id=s["top_id"], dtop=s["dtop"], scale=case["scale"])
        return {"dx": dx}
    k = MUON
    D.densenet_muon(s["plan"], lr=k["lr"], momentum=k["momentum"], weight_decay=k["weight_decay"], eps=k["eps"], steps=k["steps"],
                    coefficients=(k["a"], k["b"], k["c"]))
    return _state(s)


def run(state):
    if own:
        return _own(state)
    return {"quant": _quant, "product": _product, "scores": _scores, "scores_back": _scores_back, "muon": _muon}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# The work of a pass, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    up = lambda v: -(-v // BLOCK)  # noqa: E731
    if op == "quant":
        n, C = case["n"], case["C"]
        forms = 2 if case["turned"] else 1
        scales = (up(n) if case["rows"] > 1 else n) * up(C) + (forms - 1) * up(n) * (up(C) if case["rows"] > 1 else C)
        return {"bytes": n * C * (SIZE[case["dt"]] + forms) + 4 * scales, "flops": 3 * n * C}
    if op == "product":
        n, C, V = case["n"], case["C"], case["V"]
        return {"bytes": (n + V) * C + 4 * (n + up(V)) * up(C) + n * V * SIZE[case["out"]], "flops": 2 * n * V * C}
    if op in ("scores", "scores_back"):
        n, V, e, k = case["n"], case["V"], SIZE[case["dt"]], case["top"]
        if op == "scores":
            return {"bytes": n * V * e + n * (20 + 12 * k), "flops": 8 * n * V}
        return {"bytes": 2 * n * V * e + n * (24 + 12 * k), "flops": 8 * n * V}
    values = sum(r * c for r, c in _shapes(case))
    each = 2 * SIZE[case["dt"]] + SIZE[case["grad"]] + 8 + (2 if case["copy"] else 0)
    return {"bytes": values * each, "flops": MUON["steps"] * _muon_flops(case)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        x, rows = s["x"].double(), case["rows"]
        n, C = x.shape

        def codes(t, rows):
            """Block by block of columns, each against its rows' (or squares') largest."""
            q, tops = torch.empty_like(t), []
            for j in range(0, t.shape[1], BLOCK):
                part = t[:, j:j + BLOCK].abs().amax(1)
                if rows > 1:
                    part = torch.nn.functional.pad(part, (0, -t.shape[0] % rows)).view(-1, rows).amax(1)
                tops.append(part)
                held = part.repeat_interleave(rows)[:t.shape[0]] if rows > 1 else part
                q[:, j:j + BLOCK] = torch.nan_to_num(t[:, j:j + BLOCK] / (held / F8_MAX)[:, None])
            return q.to(DT["f8"]), torch.stack(tops, 1) / F8_MAX

        out = dict(zip(("codes", "scale"), codes(x, rows)), turned=None, turned_scale=None)
        if case["turned"]:
            out["turned"], out["turned_scale"] = codes(x.T.contiguous(), rows)
        return out
    if op == "product":
        y = torch.zeros(case["n"], case["V"], dtype=torch.float64, device="cuda")
        wide = s["w_scale"].double().repeat_interleave(BLOCK, 0)[:case["V"]]
        step = 8 * BLOCK  # a few blocks of the sum at a time
        for j in range(0, case["C"], step):
            k = slice(j // BLOCK, (j + step) // BLOCK)
            factor = lambda t: t[:, k].repeat_interleave(BLOCK, 1)[:, :min(step, case["C"] - j)]  # noqa: E731
            y += (s["a"][:, j:j + step].double() * factor(s["a_scale"].double())) @ (s["w"][:, j:j + step].double() * factor(wide)).T
        return {"y": y}
    if op in ("scores", "scores_back"):
        n, V, k = case["n"], case["V"], case["top"]
        parts = []
        step = max(1, (1 << 27) // V)
        for i in range(0, n, step):
            x, t = s["x"][i:i + step].double() * case["scale"], s["token"][i:i + step]
            rows = torch.arange(len(t), device="cuda")
            if op == "scores":
                logp = torch.log_softmax(x, 1)
                p = logp.exp()
                found = {"logp": logp[rows, t.clamp(min=0)] * (t >= 0), "entropy": -torch.special.xlogy(p, p).sum(1),
                         "lse": torch.logsumexp(x, 1), "top_id": None, "top_logp": None}
                if k:
                    best = logp.sort(1, descending=True).values[:, :k]
                    found["top_logp"] = torch.nn.functional.pad(best, (0, k - best.shape[1]), value=-math.inf)
            else:
                logp = x - s["lse"][i:i + step].double()[:, None]
                p, c = logp.exp(), (s["dlogp"][i:i + step].double() * (t >= 0))[:, None]
                held = torch.zeros_like(p)
                held[rows, t.clamp(min=0)] += c[:, 0]
                total = c
                if k:
                    ids, dt = s["top_id"][i:i + step], s["dtop"][i:i + step].double()
                    dt = dt * (ids >= 0)
                    for j in range(k):
                        held[rows, ids[:, j].clamp(min=0)] += dt[:, j]
                    total = total + dt.sum(1, keepdim=True)
                grow = torch.nan_to_num(logp, neginf=0.0) + s["entropy"][i:i + step].double()[:, None]
                found = {"dx": case["scale"] * (held - p * total - p * grow * s["dentropy"][i:i + step].double()[:, None])}
            parts.append(found)
        return {name: None if parts[0][name] is None else torch.cat([q[name] for q in parts]) for name in parts[0]}
    k = MUON
    out = {"p": [], "m": [], "copy": [] if case["copy"] else None}
    for p, g, m, rate in zip(s["p"], s["g"], s["m"], s["rates"]):
        m = m.double() * k["momentum"] + g.double()
        u = m * k["momentum"] + g.double()
        tall = u.shape[0] > u.shape[1]
        x = (u.T if tall else u).contiguous()
        x = x / (torch.linalg.vector_norm(x) + k["eps"])
        for _ in range(k["steps"]):
            gram = x @ x.T
            poly = k["c"] * gram
            poly.diagonal().add_(k["b"])
            x = k["a"] * x + poly @ (gram @ x)
        p = p.double() * (1 - k["lr"] * k["weight_decay"]) - k["lr"] * rate * (x.T if tall else x)
        out["p"].append(p)
        out["m"].append(m)
        if case["copy"]:
            out["copy"].append(p)
    return out
