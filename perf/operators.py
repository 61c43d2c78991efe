"""Cases of the operators of a worker's training step: layer norm, matrix product with its epilogue, distillation loss.

`run` computes a case either with the library's kernels (`own` true) or in plain torch operations in 32 bits,
rounded once to the output's type.  `exact` restates each operator in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

LARGEST_FLOPS = 2.0 * 8192 * 4096 * 16384     # of the products
LARGEST_ROWS_DIM = 16384 * 8192               # elements of a layer norm's matrix
LARGEST_ROWS_VOCAB = 4096 * 131072            # elements of the logits


def listed():
    return [
        # one token through a norm of the smallest transformer widths: latency alone
        {"name": "layernorm fwd, one row", "op": "layernorm_fwd", "rows": 1, "dim": 1024, "dtype": "bf16"},
        # a worker's batch of tokens in a wide model
        {"name": "layernorm fwd, batch", "op": "layernorm_fwd", "rows": 16384, "dim": 4096, "dtype": "bf16"},
        # fp32 training on an odd width: rows and parameter slices that start off a 16-byte boundary
        {"name": "layernorm bwd, odd width", "op": "layernorm_bwd", "rows": 1531, "dim": 1003, "dtype": "f32"},
        # the widest model's batch, gradients of both parameters reduced over all rows
        {"name": "layernorm bwd, largest", "op": "layernorm_bwd", "rows": 16384, "dim": 8192, "dtype": "bf16"},
        # a handful of tokens through a layer: the weight's bytes and the launch are what counts
        {"name": "linear fwd, few rows", "op": "linear_fwd", "m": 5, "n": 4096, "k": 1024, "dtype": "f16",
         "act": "gelu", "residual": False, "save_z": False, "pad": 0},
        # the widening product of a feed-forward block in training: the pre-activation is kept for the gradient
        {"name": "linear fwd, widening", "op": "linear_fwd", "m": 8192, "n": 16384, "k": 4096, "dtype": "bf16",
         "act": "gelu", "residual": False, "save_z": True, "pad": 0},
        # fp32 training, the 4096 x 4096 layer of the VGG-16-shaped workload, as a residual branch
        {"name": "linear fwd, fp32 residual", "op": "linear_fwd", "m": 2048, "n": 4096, "k": 4096, "dtype": "f32",
         "act": "none", "residual": True, "save_z": False, "pad": 0},
        # the narrowing product's gradients: input gradient through the activation, weight and bias gradient in fp32
        {"name": "linear bwd, narrowing", "op": "linear_bwd", "m": 8192, "n": 4096, "k": 4096, "dtype": "bf16",
         "act": "gelu", "add": False, "pad": 0},
        # odd sizes and padded rows, the residual's gradient added
        {"name": "linear bwd, odd sizes", "op": "linear_bwd", "m": 1537, "n": 1000, "k": 515, "dtype": "f16",
         "act": "relu", "add": True, "pad": 3},
        # a few images with 1000 classes, hard labels beside the teacher's five best
        {"name": "distill, 1000 classes", "op": "distill", "rows": 32, "vocab": 1000, "top": 5, "dtype": "f32",
         "temperature": 4.0, "kd": 0.9, "ce": 0.1, "masked": 0.0},
        # an odd vocabulary, part of it masked out
        {"name": "distill, odd vocabulary", "op": "distill", "rows": 1024, "vocab": 50021, "top": 37, "dtype": "f16",
         "temperature": 2.0, "kd": 1.0, "ce": 0.5, "masked": 0.1},
        # a worker's batch of tokens over a large vocabulary
        {"name": "distill, largest", "op": "distill", "rows": 4096, "vocab": 131072, "top": 64, "dtype": "bf16",
         "temperature": 2.0, "kd": 1.0, "ce": 0.0, "masked": 0.0},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["layernorm_fwd", "layernorm_bwd", "linear_fwd", "linear_bwd", "distill"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op.startswith("layernorm"):
        dim = _log(rng, 64, 8192)
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        most = min(16384, LARGEST_ROWS_DIM // dim * 2 // BYTES[dtype])
        return {"op": op, "rows": _log(rng, 1, most), "dim": dim, "dtype": dtype}
    if op.startswith("linear"):
        n, k = _log(rng, 64, 16384), _log(rng, 64, 16384)
        if rng.random() < 0.6:
            n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
        most = LARGEST_FLOPS / (2.0 * n * k) / (2 if op == "linear_bwd" else 1) / (6 if dtype == "f32" else 1)
        case = {"op": op, "m": _log(rng, 1, max(1, min(16384, most))), "n": n, "k": k, "dtype": dtype,
                "act": rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), "pad": rng.choice([0, 0, 0, 8, 3])}
        if op == "linear_fwd":
            return {**case, "residual": rng.random() < 0.5, "save_z": rng.random() < 0.5}
        return {**case, "add": rng.random() < 0.5}
    vocab = _log(rng, 1000, 131072)
    if rng.random() < 0.5:
        vocab = vocab // 8 * 8
    most = min(8192, LARGEST_ROWS_VOCAB // vocab * 2 // BYTES[dtype])
    kd, ce = rng.choice([(1.0, 0.0), (0.9, 0.1), (0.5, 0.5)])
    return {"op": op, "rows": _log(rng, 1, most), "vocab": vocab, "top": _log(rng, 1, 128), "dtype": dtype,
            "temperature": rng.choice([1.0, 2.0, 3.5]), "kd": kd, "ce": ce, "masked": rng.choice([0.0, 0.0, 0.3])}


# ---------------------------------------------------------------------------------------------- inputs


def _matrix(rows, cols, pad, dtype, gen, scale):
    """[rows, cols] with a row stride of cols + pad."""
    wide = torch.randn(rows, cols + pad, generator=gen, device="cuda", dtype=torch.float32)
    return wide.mul_(scale).to(dtype)[:, :cols]


def _out(rows, cols, pad, dtype):
    return torch.empty(rows, cols + pad, device="cuda", dtype=dtype)[:, :cols]


def _prepare_layernorm(case, gen):
    rows, dim, dtype = case["rows"], case["dim"], TYPES[case["dtype"]]
    x = _matrix(rows, dim, 0, dtype, gen, 1.5)
    x += torch.randn(rows, 1, generator=gen, device="cuda").to(dtype)
    model = torch.randn(2 * dim, generator=gen, device="cuda") * 0.1      # gamma and beta: slices of the flat model
    model[:dim] += 1.0
    s = {"x": x, "gamma": model[:dim], "beta": model[dim:], "eps": 1e-5}
    if case["op"] == "layernorm_fwd":
        s["y"] = _out(rows, dim, 0, dtype)
        s["mean"], s["rstd"] = torch.empty(2, rows, device="cuda").unbind(0)
        return s
    s["dy"] = _matrix(rows, dim, 0, dtype, gen, 0.01)
    x32 = x.float()
    s["mean"] = x32.mean(1)
    s["rstd"] = torch.rsqrt((x32 - s["mean"][:, None]).square().mean(1) + s["eps"])
    s["dx"] = _out(rows, dim, 0, dtype)
    delta = torch.empty(2 * dim, device="cuda")                            # the worker's flat update
    s["dgamma"], s["dbeta"] = delta[:dim], delta[dim:]
    return s


def _prepare_linear(case, gen):
    m, n, k, pad, dtype = case["m"], case["n"], case["k"], case["pad"], TYPES[case["dtype"]]
    s = {"act": case["act"], "w": _matrix(n, k, pad, dtype, gen, 1.0 / math.sqrt(k))}
    if case["op"] == "linear_fwd":
        s["x"] = _matrix(m, k, pad, dtype, gen, 1.0)
        s["bias"] = torch.randn(n, generator=gen, device="cuda") * 0.1
        s["residual"] = _matrix(m, n, pad, dtype, gen, 1.0) if case["residual"] else None
        s["y"] = _out(m, n, pad, dtype)
        s["z"] = _out(m, n, pad, dtype) if case["save_z"] else None
        return s
    s["z"] = _matrix(m, k, pad, dtype, gen, 1.0) if case["act"] != "none" else None
    s["x"] = _matrix(m, k, pad, dtype, gen, 1.0) if s["z"] is None else _act(s["z"].float(), case["act"]).to(dtype)
    s["dy"] = _matrix(m, n, pad, dtype, gen, 0.01)
    s["add"] = _matrix(m, k, pad, dtype, gen, 0.01) if case["add"] else None
    s["dx"] = _out(m, k, pad, dtype)
    delta = torch.empty(n * k + n, device="cuda")
    s["dw"], s["db"] = delta[: n * k].view(n, k), delta[n * k:]
    return s


def _prepare_distill(case, gen):
    rows, vocab, top, dtype = case["rows"], case["vocab"], min(case["top"], case["vocab"]), TYPES[case["dtype"]]
    logits = torch.randn(rows, vocab, generator=gen, device="cuda") * 2.0
    first = torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda")
    step = torch.randint(1, max(2, vocab // top), (rows, 1), generator=gen, device="cuda")
    idx = (first + step * torch.arange(top, device="cuda")) % vocab        # distinct in a row
    teacher = torch.sort(torch.randn(rows, top, generator=gen, device="cuda") * 2.0 + 8.0, 1, descending=True)[0]
    logits.scatter_add_(1, idx, teacher * 0.5)                             # a student that partly agrees
    if case["masked"]:
        out = torch.rand(vocab, generator=gen, device="cuda") < case["masked"]
        held = torch.gather(logits, 1, idx)
        logits.masked_fill_(out[None, :], float("-inf"))                   # entries that no row may choose
        logits.scatter_(1, idx, held)                                      # but for those the teacher names
    label = idx[:, 0].clone()
    count = torch.randint(1, top + 1, (rows, 1), generator=gen, device="cuda")
    some = torch.rand(rows, 1, generator=gen, device="cuda") < 0.1         # rows whose teacher kept fewer entries
    idx = torch.where(some & (torch.arange(top, device="cuda") >= count), -1, idx)
    u = torch.rand(rows, generator=gen, device="cuda")
    label = torch.where(u < 0.05, -100, label)                             # positions without a label
    scale = 1024.0 if case["dtype"] == "f16" else 1.0                      # fp16 training scales its loss
    weight = torch.where(u > 0.95, 0.0, scale / rows)                      # zero at padded positions
    return {"logits": logits.to(dtype), "idx": idx.to(torch.int32), "teacher": teacher,
            "label": label.to(torch.int32) if case["ce"] else None, "weight": weight,
            "temperature": case["temperature"], "kd": case["kd"], "ce": case["ce"],
            "loss": torch.empty(rows, device="cuda"), "dlogits": _out(rows, vocab, 0, dtype)}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    make = _prepare_distill if case["op"] == "distill" else \
        _prepare_layernorm if case["op"].startswith("layernorm") else _prepare_linear
    state = make(case, gen)
    state["op"] = case["op"]
    if own:                                   # the scratch that a caller of the library keeps beside its buffers
        import paper_1709_09393_b200 as P
        size = 16
        if case["op"] == "layernorm_bwd":
            size = P.layernorm_workspace_bytes(case["rows"], case["dim"])
        elif case["op"].startswith("linear"):
            size = P.linear_workspace_bytes(case["m"], case["n"], case["k"], TYPES[case["dtype"]])
        state["ws"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    return state


# ---------------------------------------------------------------------------------------------- one pass


def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _plain(s):
    op = s["op"]
    if op == "layernorm_fwd":
        x = s["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = torch.rsqrt((c * c).mean(1) + s["eps"])
        y = c * rstd[:, None] * s["gamma"] + s["beta"]
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if op == "layernorm_bwd":
        h = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * s["rstd"][:, None]
        return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}
    if op == "linear_fwd":
        z = s["x"].float() @ s["w"].float().t() + s["bias"]
        y = _act(z, s["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(s["x"].dtype), "z": z.to(s["x"].dtype) if s["z"] is not None else None}
    if op == "linear_bwd":
        dy = s["dy"].float()
        dx = dy @ s["w"].float()
        if s["z"] is not None:
            dx = dx * _act_slope(s["z"].float(), s["act"])
        if s["add"] is not None:
            dx = dx + s["add"].float()
        return {"dx": dx.to(s["x"].dtype), "dw": dy.t() @ s["x"].float(), "db": dy.sum(0)}
    # distillation
    T, kd, ce, w = s["temperature"], s["kd"], s["ce"], s["weight"]
    z = s["logits"].float()
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z / T)
    total = e.sum(1, keepdim=True)
    there = s["idx"] >= 0
    at = s["idx"].clamp_min(0).long()
    t = torch.where(there, s["teacher"], float("-inf")) / T
    t = t - t.amax(1, keepdim=True)
    q = torch.exp(t)
    logq = t - torch.log(q.sum(1, keepdim=True))
    q = q / q.sum(1, keepdim=True)
    logp = torch.gather(z, 1, at) / T - torch.log(total)
    loss = kd * T * T * torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    grad = e.mul_(kd * T / total)
    grad.scatter_add_(1, at, -kd * T * q)
    if s["label"] is not None:
        has = (s["label"] >= 0)[:, None]
        y = s["label"].clamp_min(0).long()[:, None]
        e = torch.exp(z)
        total = e.sum(1, keepdim=True)
        loss = loss + ce * torch.where(has, torch.log(total) - torch.gather(z, 1, y), 0.0)[:, 0]
        grad += e * torch.where(has, ce / total, 0.0)
        grad.scatter_add_(1, y, torch.where(has, -ce, 0.0))
    return {"loss": w * loss, "dlogits": (grad * w[:, None]).to(s["logits"].dtype)}


def _own(s):
    import paper_1709_09393_b200 as P
    op = s["op"]
    if op == "layernorm_fwd":
        P.slimdp_layernorm_forward(s["x"], s["gamma"], s["beta"], s["eps"], s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "layernorm_bwd":
        P.slimdp_layernorm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"],
                                    s["dbeta"], s["ws"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if op == "linear_fwd":
        P.slimdp_linear_forward(s["x"], s["w"], s["bias"], s["y"], s["ws"], activation=s["act"],
                                residual=s["residual"], z=s["z"])
        return {"y": s["y"], "z": s["z"]}
    if op == "linear_bwd":
        P.slimdp_linear_backward_input(s["dy"], s["w"], s["dx"], s["ws"], activation=s["act"], z=s["z"], add=s["add"])
        P.slimdp_linear_backward_weight(s["dy"], s["x"], s["dw"], s["db"], s["ws"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    P.slimdp_distill(s["logits"], s["idx"], s["teacher"], s["loss"], s["dlogits"], label=s["label"],
                     row_weight=s["weight"], temperature=s["temperature"], kd_weight=s["kd"], ce_weight=s["ce"])
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- bounds


def work(case):
    op, size = case["op"], BYTES[case["dtype"]]
    if op.startswith("layernorm"):
        rows, dim = case["rows"], case["dim"]
        if op == "layernorm_fwd":
            return {"bytes": 2 * rows * dim * size + 8 * dim + 8 * rows, "flops": 8 * rows * dim}
        return {"bytes": 3 * rows * dim * size + 12 * dim + 8 * rows, "flops": 14 * rows * dim}
    if op.startswith("linear"):
        m, n, k = case["m"], case["n"], case["k"]
        if op == "linear_fwd":
            tensors = m * k + n * k + m * n * (1 + case["residual"] + case["save_z"])
            return {"bytes": tensors * size + 4 * n, "flops": 2 * m * n * k}
        tensors = m * n + n * k + m * k * (2 + (case["act"] != "none") + case["add"])
        return {"bytes": tensors * size + 4 * n * k + 4 * n, "flops": 4 * m * n * k}
    rows, vocab, top = case["rows"], case["vocab"], min(case["top"], case["vocab"])
    both = 2 if case["ce"] else 1
    return {"bytes": 2 * rows * vocab * size + rows * (8 * top + 8 + 4 * (both - 1)), "flops": (2 + 4 * both) * rows * vocab}


# ---------------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    d = {name: v.double() for name, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()
         and name not in ("y", "dx", "dw", "db", "loss", "dlogits", "dgamma", "dbeta")}
    if op == "layernorm_fwd":
        var, mean = torch.var_mean(d["x"], 1, correction=0, keepdim=True)
        rstd = (var + s["eps"]) ** -0.5
        y = (d["x"] - mean) * rstd * d["gamma"] + d["beta"]
        return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "layernorm_bwd":
        r = d["rstd"][:, None]
        h = (d["x"] - d["mean"][:, None]) * r
        g = d["dy"] * d["gamma"]
        n = case["dim"]
        along = torch.einsum("rd,rd->r", g, h)[:, None] / n
        dx = r * (g - g.sum(1, keepdim=True) / n - h * along)
        return {"dx": dx, "dgamma": torch.einsum("rd,rd->d", d["dy"], h), "dbeta": torch.einsum("rd->d", d["dy"])}
    functions = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
                 "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}
    if op == "linear_fwd":
        z = torch.addmm(d["bias"], d["x"], d["w"].t())
        y = functions[case["act"]](z)
        if case["residual"]:
            y = y + d["residual"]
        return {"y": y, "z": z if case["save_z"] else None}
    if op == "linear_bwd":
        dx = torch.mm(d["dy"], d["w"])
        if case["act"] != "none":
            with torch.enable_grad():
                z = d["z"].clone().requires_grad_(True)
                slope, = torch.autograd.grad(functions[case["act"]](z).sum(), z)
            dx = dx * slope
        if case["add"]:
            dx = dx + d["add"]
        return {"dx": dx, "dw": torch.mm(d["dy"].t(), d["x"]), "db": d["dy"].sum(0)}
    T = case["temperature"]
    rows = torch.arange(case["rows"], device="cuda")[:, None]
    there = s["idx"] >= 0
    at = torch.where(there, s["idx"], 0).long()
    q = torch.where(there, torch.softmax(torch.where(there, d["teacher"] / T, -math.inf), 1), 0.0)
    scaled = d["logits"] / T
    logp = torch.log_softmax(scaled, 1)
    loss = case["kd"] * T * T * (torch.special.xlogy(q, q) - torch.where(q > 0, q * logp[rows, at], 0.0)).sum(1)
    soft = torch.zeros_like(logp).index_put_((rows, at), q, accumulate=True)
    grad = case["kd"] * T * (logp.exp_() - soft)
    del soft, scaled, logp
    if case["ce"]:
        has = s["label"] >= 0
        y = torch.where(has, s["label"], 0).long()
        loss = loss + case["ce"] * torch.where(has, torch.logsumexp(d["logits"], 1) - d["logits"][rows[:, 0], y], 0.0)
        p = torch.softmax(d["logits"], 1)
        p[rows[:, 0], y] -= 1.0
        grad += p.mul_(case["ce"] * has.double()[:, None])
    return {"loss": d["weight"] * loss, "dlogits": grad.mul_(d["weight"][:, None])}
