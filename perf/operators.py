"""The operators of a training step around the quantised layers, as a program runs them: the layer
norm between two layers, the loss of a linear classifier behind the last one, and the
orthogonalised update made of a layer's weight gradient.

Shapes are those of the benchmark's layers (a ResNet18 for 32x32 images: 64 to 512 channels, 32x32
to 4x4 pixels), generic wide ones, and ragged ones between them.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
NORM_EPS = 1e-5
UPDATE_EPS = 1e-7


def _norm(name, rows, channels, kind, x="f32", y="f32", g="f32"):
    c = dict(kind=kind, rows=rows, channels=channels, x=x, y=y, g=g)
    return dict(name=name, **c) if name else c


def _loss(name, rows, features, classes, kind, type="f32", bias=False, ignored=0.0):
    c = dict(kind=kind, rows=rows, features=features, classes=classes, type=type, bias=bias,
             ignored=ignored)
    return dict(name=name, **c) if name else c


def _update(name, batch, rows, cols, type="f32"):
    c = dict(kind="update", batch=batch, rows=rows, cols=cols, type=type)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # behind the smallest layer of the benchmark: one 8x8 image, 16 channels
        _norm("norm_smallest_c16", 64, 16, "norm"),
        # between two layers of the network's first stage, a batch of 128: fp32 in, the int8 codes
        # that the next layer takes out
        _norm("norm_codes_c64", 128 * 32 * 32, 64, "norm", y="i8"),
        # gradients behind the third stage, the headline layer's batch
        _norm("norm_backward_c256", 256 * 8 * 8, 256, "norm_backward"),
        # a wide network in bf16, many rows: throughput
        _norm("norm_backward_wide", 8192, 4096, "norm_backward", x="bf16", y="bf16", g="bf16"),
        # the classifier of the ResNet18: ten classes, a training step's loss and gradients
        _loss("loss_classifier_10", 256, 512, 10, "loss_train", bias=True),
        # unquantised training over some ten thousand classes, no size a multiple of anything
        _loss("loss_ragged_f32", 1001, 515, 10007, "loss_train", bias=True, ignored=0.05),
        # one row scored against a large vocabulary: the weights are read once
        _loss("loss_one_row", 1, 4096, 131072, "loss", type="bf16"),
        # a training step over a large vocabulary
        _loss("loss_train_large", 4096, 2048, 65536, "loss_train", type="bf16", ignored=0.05),
        # updates of the four layers of the first stage: launches and latency
        _update("update_c64", 4, 64, 9 * 64),
        # the three layers of the third stage
        _update("update_c256", 3, 256, 9 * 256),
        # the three layers of the last stage, gradients kept in bf16
        _update("update_c512_bf16", 3, 512, 9 * 512, type="bf16"),
        # one large matrix, taller than wide
        _update("update_large", 1, 6144, 1536),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    """Any operator, type and direction; from one row to the largest listed case's work."""
    kind = rng.choice(("norm", "norm", "norm_backward", "loss", "loss_train", "loss_train", "update", "update"))
    while True:
        t = rng.choice(("f32", "bf16"))
        if kind.startswith("norm"):
            c = _norm(None, _log_int(rng, 1, 262144), _log_int(rng, 8, 16384), kind, x=t,
                      y=rng.choice(("i8", t)) if kind == "norm" else t, g=t)
            size = 4 if t == "f32" else 2
            if c["rows"] * c["channels"] * size <= 8192 * 4096 * 2:
                return c
        elif kind.startswith("loss"):
            c = _loss(None, _log_int(rng, 1, 8192), _log_int(rng, 16, 4096), _log_int(rng, 2, 131072),
                      kind, type=t, bias=rng.random() < 0.5, ignored=rng.choice((0.0, 0.05)))
            work = c["rows"] * c["features"] * c["classes"]
            if work * (6 if t == "f32" else 1) <= 4096 * 2048 * 65536 and \
                    max(c["rows"] * c["classes"], c["features"] * c["classes"]) <= 4096 * 131072:
                return c
        else:
            c = _update(None, rng.randint(1, 8), _log_int(rng, 8, 2048), _log_int(rng, 8, 8192), type=t)
            r, w = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
            if c["batch"] * r * r * w <= 1536 * 1536 * 6144:
                return c


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _matrices(case, g):
    """Gradients of a layer's weights: a few strong directions over noise, small numbers."""
    b, r, c = case["batch"], case["rows"], case["cols"]
    few = min(8, r, c)
    fall = 0.5 ** torch.arange(few, device="cuda", dtype=torch.float32)
    strong = torch.matmul(_normal(g, b, r, few) * fall, _normal(g, b, few, c))
    return ((strong + 0.3 * _normal(g, b, r, c)) * 1e-3).to(DTYPES[case["type"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case}
    if case["kind"].startswith("norm"):
        R, C = case["rows"], case["channels"]
        # a layer's output: channels with means and spreads of their own
        s["x"] = (_normal(g, R, C) * (0.5 + _normal(g, C).abs()) + _normal(g, C)).to(DTYPES[case["x"]])
        s["gamma"], s["beta"] = 1 + 0.2 * _normal(g, C), 0.2 * _normal(g, C)
        s["s_y"] = 4.0 / 127  # codes saturate beyond four
        if case["kind"] == "norm_backward":
            s["dy"] = (_normal(g, R, C) * 1e-2).to(DTYPES[case["g"]])
            x = s["x"].float()
            s["mean"] = x.mean(1)  # what the forward pass has kept
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + NORM_EPS)
    elif case["kind"].startswith("loss"):
        T, D, V = case["rows"], case["features"], case["classes"]
        t = DTYPES[case["type"]]
        w = _normal(g, V, D) / math.sqrt(D)
        target = torch.randint(0, V, (T,), generator=g, device="cuda")
        s["w"] = w.to(t)
        # features of a partly trained network: they lean towards their class
        s["h"] = (_normal(g, T, D) + 2 * w[target]).to(t)
        s["bias"] = 0.1 * _normal(g, V) if case["bias"] else None
        out = torch.rand(T, generator=g, device="cuda") < case["ignored"]
        s["target"] = torch.where(out, torch.full_like(target, -100), target)
        kept = s["target"] >= 0
        s["dloss"] = kept.float() / kept.sum().clamp(min=1)  # of the mean over the rows that count
    else:
        s["grad"] = _matrices(case, g)
    if own:
        import paper_2004_11077_amd as wn
        code = {"f32": wn.TYPE_F32, "bf16": wn.TYPE_BF16, "i8": wn.TYPE_I8}
        if case["kind"].startswith("norm"):
            s["desc"] = wn.NormDesc(case["rows"], case["channels"], x_type=code[case["x"]],
                                    y_type=code[case["y"]], g_type=code[case["g"]], eps=NORM_EPS,
                                    s_y=s["s_y"])
            size = (wn.wino_layer_norm_backward_workspace_bytes(s["desc"])
                    if case["kind"] == "norm_backward" else 256)
        elif case["kind"].startswith("loss"):
            s["desc"] = wn.LossDesc(case["rows"], case["features"], case["classes"],
                                    type=code[case["type"]], ignore_index=-100)
            size = wn.wino_linear_cross_entropy_workspace_bytes(s["desc"])
            if case["kind"] == "loss_train":
                size = max(size, wn.wino_linear_cross_entropy_backward_workspace_bytes(s["desc"]))
        else:
            a, b, c = COEFFICIENTS
            s["desc"] = wn.OrthogonaliseDesc(case["batch"], case["rows"], case["cols"],
                                             g_type=code[case["type"]], o_type=code[case["type"]],
                                             steps=STEPS, a=a, b=b, c=c, eps=UPDATE_EPS)
            size = wn.wino_orthogonalise_workspace_bytes(s["desc"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


def _plain_norm(s):
    case = s["case"]
    # codes lie next to borders between two whole numbers: 64 bits there
    x = s["x"].double() if case["y"] == "i8" else s["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + NORM_EPS)
    y = (x - mean) * rstd * s["gamma"] + s["beta"]
    if case["y"] == "i8":
        y = torch.clamp(torch.round(y / _f32(s["s_y"])), -127, 127).to(torch.int8)
    else:
        y = y.to(DTYPES[case["y"]])
    return {"y": y, "mean": mean[:, 0].float(), "rstd": rstd[:, 0].float()}


def _f32(v):
    """A number as a 32-bit field of a descriptor holds it."""
    return torch.tensor(v, dtype=torch.float32).item()


def _plain_norm_backward(s):
    case = s["case"]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return {"dx": dx.to(DTYPES[case["g"]]), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _plain_loss(s):
    case = s["case"]
    h, w = s["h"].float(), s["w"].float()
    kept = s["target"] >= 0
    at = s["target"].clamp(min=0)[:, None]
    logits = h @ w.t()
    if s["bias"] is not None:
        logits = logits + s["bias"]
    top = logits.max(1, keepdim=True).values
    p = torch.exp(logits - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    loss = torch.where(kept, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    r = {"loss": loss, "lse": lse}
    if case["kind"] == "loss_train":
        t = DTYPES[case["type"]]
        scale = torch.where(kept, s["dloss"], torch.zeros_like(lse))[:, None]
        dl = p.div_(total).mul_(scale)
        dl.scatter_add_(1, at, -scale)
        r["dh"], r["dw"] = (dl @ w).to(t), (dl.t() @ h).to(t)
        if s["bias"] is not None:
            r["dbias"] = dl.sum(0)
    return r


def _step(x):
    a, b, c = COEFFICIENTS
    m = torch.matmul(x, x.transpose(1, 2))
    return a * x + torch.matmul(b * m + c * torch.matmul(m, m), x)


def _plain_update(s):
    g = s["grad"].float()
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + UPDATE_EPS)
    x = _step(_step(_step(_step(_step(x)))))
    return {"update": (x.transpose(1, 2) if tall else x).contiguous().to(s["grad"].dtype)}


def _own_norm(s):
    import paper_2004_11077_amd as wn
    case = s["case"]
    dtype = torch.int8 if case["y"] == "i8" else DTYPES[case["y"]]
    y = torch.empty(case["rows"], case["channels"], dtype=dtype, device="cuda")
    mean, rstd = (torch.empty(case["rows"], device="cuda") for _ in range(2))
    wn.wino_layer_norm(s["desc"], s["x"], s["gamma"], s["beta"], y, mean, rstd)
    return {"y": y, "mean": mean, "rstd": rstd}


def _own_norm_backward(s):
    import paper_2004_11077_amd as wn
    dx = torch.empty_like(s["dy"])
    dgamma, dbeta = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    wn.wino_layer_norm_backward(s["desc"], s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], dx,
                                dgamma, dbeta, s["workspace"])
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_loss(s):
    import paper_2004_11077_amd as wn
    loss, lse = (torch.empty(s["case"]["rows"], device="cuda") for _ in range(2))
    wn.wino_linear_cross_entropy(s["desc"], s["h"], s["w"], s["bias"], s["target"], loss, lse,
                                 s["workspace"])
    r = {"loss": loss, "lse": lse}
    if s["case"]["kind"] == "loss_train":
        dh, dw = torch.empty_like(s["h"]), torch.empty_like(s["w"])
        dbias = None if s["bias"] is None else torch.empty_like(s["bias"])
        wn.wino_linear_cross_entropy_backward(s["desc"], s["h"], s["w"], s["bias"], s["target"], lse,
                                              s["dloss"], dh, dw, dbias, s["workspace"])
        r["dh"], r["dw"] = dh, dw
        if dbias is not None:
            r["dbias"] = dbias
    return r


def _own_update(s):
    import paper_2004_11077_amd as wn
    o = torch.empty_like(s["grad"])
    wn.wino_orthogonalise(s["desc"], s["grad"], o, s["workspace"])
    return {"update": o}


def run(state):
    kind = state["case"]["kind"]
    if own:
        f = {"norm": _own_norm, "norm_backward": _own_norm_backward, "loss": _own_loss,
             "loss_train": _own_loss, "update": _own_update}
    else:
        f = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "loss": _plain_loss,
             "loss_train": _plain_loss, "update": _plain_update}
    return f[kind](state)


def work(case):
    size = {"f32": 4, "bf16": 2, "i8": 1}
    if case["kind"].startswith("norm"):
        R, C = case["rows"], case["channels"]
        if case["kind"] == "norm":
            return {"bytes": R * C * (size[case["x"]] + size[case["y"]]) + 8 * R + 8 * C, "flops": 8 * R * C}
        return {"bytes": R * C * (size[case["x"]] + 2 * size[case["g"]]) + 8 * R + 12 * C, "flops": 15 * R * C}
    if case["kind"].startswith("loss"):
        T, D, V = case["rows"], case["features"], case["classes"]
        b = size[case["type"]]
        once = (T * D + V * D) * b + (4 * V if case["bias"] else 0) + 16 * T
        if case["kind"] == "loss":
            return {"bytes": once, "flops": 2 * T * D * V}
        return {"bytes": once + (T * D + V * D) * b + (4 * V if case["bias"] else 0) + 4 * T,
                "flops": 6 * T * D * V}
    n, r, c = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # X X^T and its square are symmetric: half of their entries
    return {"bytes": 2 * n * r * c * size[case["type"]],
            "flops": STEPS * n * (r * (r + 1) * c + r * (r + 1) * r + 2 * r * r * c)}


def exact(case, seed):
    s = prepare(case, seed)
    wide = torch.float64
    if case["kind"] == "norm":
        x = s["x"].to(wide)
        centred = x - x.sum(1, keepdim=True) / case["channels"]
        var = (centred ** 2).sum(1, keepdim=True) / case["channels"]
        inv = 1 / torch.sqrt(var + NORM_EPS)
        y = centred * inv * s["gamma"].to(wide) + s["beta"].to(wide)
        if case["y"] == "i8":
            y = torch.round(y / _f32(s["s_y"])).clamp(-127, 127).to(torch.int8)
        return {"y": y, "mean": (x - centred)[:, 0], "rstd": inv[:, 0]}
    if case["kind"] == "norm_backward":
        # dx as the product of dy with the derivative of y, whose three terms are the unit matrix,
        # the mean's and the spread's
        C = case["channels"]
        inv = s["rstd"].to(wide).unsqueeze(1)
        z = (s["x"].to(wide) - s["mean"].to(wide).unsqueeze(1)) * inv
        dy = s["dy"].to(wide)
        dz = dy * s["gamma"].to(wide)
        along = (dz * z).sum(1, keepdim=True) / C
        return {"dx": inv * dz - inv * (dz.sum(1, keepdim=True) / C) - inv * along * z,
                "dgamma": torch.einsum("rc,rc->c", dy, z), "dbeta": dy.sum(0)}
    if case["kind"].startswith("loss"):
        h, w = s["h"].to(wide), s["w"].to(wide)
        logits = torch.mm(h, w.t().contiguous())
        if s["bias"] is not None:
            logits += s["bias"].to(wide)
        lse = torch.logsumexp(logits, 1)
        rows = torch.nonzero(s["target"] >= 0)[:, 0]
        cls = s["target"][rows]
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - logits[rows, cls]
        r = {"loss": loss, "lse": lse}
        if case["kind"] == "loss_train":
            d = logits.sub_(lse.unsqueeze(1)).exp_()
            d[rows, cls] -= 1
            weight = torch.zeros_like(lse)
            weight[rows] = s["dloss"][rows].to(wide)
            d *= weight.unsqueeze(1)
            r["dh"], r["dw"] = torch.mm(d, w), torch.mm(d.t().contiguous(), h)
            if s["bias"] is not None:
                r["dbias"] = d.sum(0)
        return r
    a, b, c = COEFFICIENTS
    g = s["grad"].to(wide)
    out = torch.empty_like(g)
    for i in range(case["batch"]):
        x = g[i] if case["rows"] <= case["cols"] else g[i].t().contiguous()
        x = x / (torch.linalg.norm(x) + UPDATE_EPS)
        for _ in range(STEPS):
            m = x @ x.t()
            # (a + b m + c m^2) x, from the right: two products with m
            mx = m @ x
            x = a * x + b * mx + c * (m @ mx)
        out[i] = x if case["rows"] <= case["cols"] else x.t()
    return {"update": out}
