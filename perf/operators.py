"""The layer operators beside the convolutions, as measurable cases.

A case is one call on n-h-w-c activations seen as rows (one per pixel) of
channels, in the paper's notation (i_c channels in, k_c out):

  linear       Y = act(X K + bias) + R, or act(X K + bias + R); Z, the activation's
               argument, is kept where a training step will need it
  linear_grad  dX, dK, dbias and dZ from G = dloss/dY and Z
  norm         layer norm of every row, with its mean and 1/deviation
  norm_grad    its input's and its weights' gradients
  orth         Newton-Schulz orthogonalisation of a stack of kernel gradients, each the
               (k_h*k_w*i_c) x k_c matrix that K is viewed as

`dtype` is the type of the activations and of K; bias, gamma, beta and the row
statistics are fp32. `gap` is what lies between two rows of X (and R) when they
are a slice of the channels of a wider tensor, in elements.
"""
import math

import torch

own = False

STEPS, COEFFICIENTS, ORTH_EPS, NORM_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7, 1e-5


def _linear(name, dtype, rows, i_c, k_c, act, residual, save, gap=0, op="linear"):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "i_c": i_c, "k_c": k_c,
            "act": act, "residual": residual, "save": save, "gap": gap}


def _norm(name, op, dtype, rows, channels, gap=0):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "channels": channels, "gap": gap}


def _orth(name, dtype, batch, rows, cols):
    return {"name": name, "op": "orth", "dtype": dtype, "batch": batch, "rows": rows, "cols": cols}


def listed():
    return [
        # the classifier of a residual network on one image: latency, the weights read once
        _linear("linear_one", "bf16", 1, 2048, 1000, "none", "none", False),
        # sizes that are multiples of nothing (an 11x11x3 patch in), rows cut out of a wider tensor
        _linear("linear_odd", "f32", 333, 363, 131, "silu", "last", False, gap=5),
        # the widening 1x1 of a residual block at batch 32: relu(X K + bias + shortcut)
        _linear("linear_expand", "f32", 32 * 56 * 56, 64, 256, "relu", "first", True),
        # a large product in 16 bits, throughput inference: the most arithmetic of all
        _linear("linear_large", "bf16", 16384, 4096, 4096, "gelu", "last", False),
        # gradients of a middle layer in 32 bits
        _linear("linear_grad_mid", "f32", 32 * 14 * 14, 1024, 256, "silu", "none", True, op="linear_grad"),
        # gradients of a widening layer at a full batch (256 images of 14x14) in 16 bits
        _linear("linear_grad_wide", "bf16", 256 * 14 * 14, 512, 2048, "gelu", "none", True, op="linear_grad"),
        # one image's last layer: 49 pixels
        _norm("norm_few", "norm", "f32", 49, 2048),
        # a full batch in 16 bits: bytes only
        _norm("norm_wide", "norm", "bf16", 32 * 56 * 56, 512),
        # an odd width, gradients
        _norm("norm_grad_odd", "norm_grad", "f32", 256 * 7 * 7, 1001),
        # the gradients of a full batch
        _norm("norm_grad_wide", "norm_grad", "bf16", 32 * 56 * 56, 512),
        # the update of a first layer: 11x11x3 -> 96
        _orth("orth_first", "f32", 1, 363, 96),
        # the 23 equal 3x3 layers of a residual network's third stage, in one call
        _orth("orth_stack", "f32", 23, 2304, 256),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng, lo, hi):
    c = _log_int(rng, lo, hi)
    if rng.random() < 0.6 and c >= 16:  # most networks round their channels
        c = 16 * round(c / 16)
    return c


def draw(rng):
    """Any of the operators over the ranges of the listed cases, odd sizes among them."""
    op = rng.choice(["linear", "linear", "linear_grad", "linear_grad", "norm", "norm_grad", "orth"])
    dtype = rng.choice(["f32", "bf16"])
    gap = rng.choice([0, 0, 0, rng.randint(1, 64)])
    most = max(work(c)["bytes"] for c in listed())
    while True:
        if op in ("linear", "linear_grad"):
            case = _linear("", dtype, _log_int(rng, 1, 131072), _channels(rng, 16, 4096), _channels(rng, 16, 4096),
                           rng.choice(["none", "relu", "silu", "gelu"]), rng.choice(["none", "last", "first"]),
                           rng.random() < 0.5, gap, op)
            if op == "linear_grad":
                case["residual"], case["save"] = "none", True
            limit = 5.5e11 if dtype == "bf16" else 1e11
        elif op in ("norm", "norm_grad"):
            case = _norm("", op, dtype, _log_int(rng, 1, 131072), _channels(rng, 16, 8192), gap)
            limit = 1e12
        else:
            k_c = _channels(rng, 16, 1024)
            case = _orth("", dtype, _log_int(rng, 1, 32), rng.choice([1, 3, 9]) * _channels(rng, 16, 1024), k_c)
            limit = 2e11
        w = work(case)
        if w["bytes"] <= most and w["flops"] <= limit:
            return case


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("linear", "linear_grad"):
        rows, i_c, k_c = case["rows"], case["i_c"], case["k_c"]
        x, k, y = rows * i_c, i_c * k_c, rows * k_c
        if case["op"] == "linear":
            return {"bytes": e * (x + k + y * (1 + (case["residual"] != "none") + case["save"])) + 4 * k_c,
                    "flops": 2 * rows * i_c * k_c}
        acts = case["act"] != "none"
        return {"bytes": e * (2 * x + 2 * k + y * (1 + 2 * acts)) + 4 * k_c, "flops": 4 * rows * i_c * k_c}
    if case["op"] == "norm":
        rows, c = case["rows"], case["channels"]
        return {"bytes": 2 * e * rows * c + 8 * rows + 8 * c, "flops": 8 * rows * c}
    if case["op"] == "norm_grad":
        rows, c = case["rows"], case["channels"]
        return {"bytes": 3 * e * rows * c + 8 * rows + 12 * c, "flops": 13 * rows * c}
    # the two symmetric products of a step need half their multiplications
    m, n = sorted((case["rows"], case["cols"]))
    return {"bytes": 2 * e * case["batch"] * m * n, "flops": case["batch"] * STEPS * (3 * m * m * n + m * m * m)}


def _rows(case, width, make):
    """rows x width, `gap` elements between two rows."""
    wide = make(case["rows"], width + case["gap"])
    return wide[:, :width]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    state = {"case": case}
    if case["op"] in ("linear", "linear_grad"):
        rows, i_c, k_c = case["rows"], case["i_c"], case["k_c"]
        # activations: channels of different size and offset
        scale, shift = 0.5 + randn(i_c + case["gap"]).abs(), 0.3 * randn(i_c + case["gap"])
        state["X"] = _rows(case, i_c, lambda r, c: (randn(r, c) * scale + shift).to(dtype))
        state["K"] = (randn(i_c, k_c) / math.sqrt(i_c)).to(dtype)
        state["bias"] = 0.1 * randn(k_c)
        state["R"] = None
        if case["residual"] != "none":
            state["R"] = _rows(case, k_c, lambda r, c: randn(r, c).to(dtype))
        if case["op"] == "linear_grad":
            state["Z"] = (state["X"].float() @ state["K"].float() + state["bias"]).to(dtype)
            state["G"] = (randn(rows, k_c) * 1e-3).to(dtype)
    elif case["op"] in ("norm", "norm_grad"):
        rows, c = case["rows"], case["channels"]
        # a residual stream: offsets and sizes by channel, a few channels far larger
        scale, shift = 0.5 + randn(c + case["gap"]).abs(), randn(c + case["gap"])
        scale[torch.randint(c, (max(1, c // 256),), generator=g, device="cuda")] *= 20.0
        state["X"] = _rows(case, c, lambda r, w: (randn(r, w) * scale + shift).to(dtype))
        state["gamma"], state["beta"] = 1.0 + 0.2 * randn(c), 0.2 * randn(c)
        if case["op"] == "norm_grad":
            x = state["X"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = 1.0 / torch.sqrt((x - state["mean"][:, None]).square().mean(1) + NORM_EPS)
            state["G"] = (randn(rows, c) * 1e-3).to(dtype)
    else:
        b, m, n = case["batch"], case["rows"], case["cols"]
        # a gradient: a few strong directions over noise
        rank = max(1, min(m, n) // 8)
        strong = torch.bmm(randn(b, m, rank), randn(b, rank, n)) / math.sqrt(rank)
        state["U"] = (1e-3 * (strong + 0.3 * randn(b, m, n))).to(dtype)
    if own:
        import paper_1706_06873_amd as mec
        # training programs keep their workspaces between calls
        need = 0
        if case["op"] == "linear_grad":
            need = mec.linear_grad_workspace_bytes(case["rows"], case["i_c"], case["k_c"], _code(mec, case))
        elif case["op"] == "norm_grad":
            need = mec.layer_norm_grad_workspace_bytes(case["rows"], case["channels"], _code(mec, case))
        elif case["op"] == "orth":
            need = mec.orthogonalize_workspace_bytes(case["batch"], case["rows"], case["cols"], _code(mec, case))
        state["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    return state


def _code(mec, case):
    return mec.F32 if case["dtype"] == "f32" else mec.BF16


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_1706_06873_amd as mec
    case = state["case"]
    op = case["op"]
    if op == "linear":
        Z = None
        if case["save"]:
            Z = torch.empty((case["rows"], case["k_c"]), dtype=state["X"].dtype, device="cuda")
        Y = mec.linear(state["X"], state["K"], state["bias"], residual=state["R"], act=case["act"],
                       residual_first=case["residual"] == "first", Z=Z)
        return [Y, Z] if case["save"] else [Y]
    if op == "linear_grad":
        dX, dK, dbias, dZ = mec.linear_grad(state["G"], state["X"], state["K"], Z=state["Z"], act=case["act"],
                                            workspace=state["workspace"])
        return [dX, dK, dbias, dZ]
    if op == "norm":
        return list(mec.layer_norm(state["X"], state["gamma"], state["beta"], eps=NORM_EPS))
    if op == "norm_grad":
        return list(mec.layer_norm_grad(state["G"], state["X"], state["mean"], state["rstd"], state["gamma"],
                                        workspace=state["workspace"]))
    return [mec.orthogonalize(state["U"], steps=STEPS, coefficients=COEFFICIENTS, eps=ORTH_EPS,
                              workspace=state["workspace"])]


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _run_plain(state):
    case = state["case"]
    op = case["op"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    if op == "linear":
        z = torch.matmul(state["X"].float(), state["K"].float()) + state["bias"]
        if case["residual"] == "first":
            z = z + state["R"].float()
        if case["act"] == "relu":
            y = torch.where(z > 0, z, torch.zeros_like(z))
        elif case["act"] == "silu":
            y = z * _sigmoid(z)
        elif case["act"] == "gelu":
            y = z * _sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        else:
            y = z
        if case["residual"] == "last":
            y = y + state["R"].float()
        return [y.to(dtype), z.to(dtype)] if case["save"] else [y.to(dtype)]
    if op == "linear_grad":
        g, z = state["G"].float(), state["Z"].float()
        if case["act"] == "relu":
            dz = torch.where(z > 0, g, torch.zeros_like(g))
        elif case["act"] == "silu":
            s = _sigmoid(z)
            dz = g * s * (1.0 + z * (1.0 - s))
        elif case["act"] == "gelu":
            c = math.sqrt(2.0 / math.pi)
            s = _sigmoid(2.0 * c * (z + 0.044715 * z * z * z))
            dz = g * (s + z * s * (1.0 - s) * 2.0 * c * (1.0 + 3.0 * 0.044715 * z * z))
        else:
            dz = g
        dX = torch.matmul(dz, state["K"].float().t())
        dK = torch.matmul(state["X"].float().t(), dz)
        return [dX.to(dtype), dK.to(dtype), dz.sum(0), dz.to(dtype)]
    if op == "norm":
        x = state["X"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((d * d).mean(1) + NORM_EPS)
        return [(d * rstd[:, None] * state["gamma"] + state["beta"]).to(dtype), mean, rstd]
    if op == "norm_grad":
        g, x = state["G"].float(), state["X"].float()
        xh = (x - state["mean"][:, None]) * state["rstd"][:, None]
        w = g * state["gamma"]
        dx = state["rstd"][:, None] * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
        return [dx.to(dtype), (g * xh).sum(0), g.sum(0)]
    u = state["U"].float()
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u  # the Gram matrix on the smaller side
    norm = torch.sqrt((x * x).sum((1, 2), keepdim=True))
    x = x / (norm + ORTH_EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        poly = b * gram + c * torch.bmm(gram, gram)
        x = a * x + torch.bmm(poly, x)
    if tall:
        x = x.transpose(1, 2).contiguous()
    return [x.to(dtype)]


def exact(case, seed):
    """The definitions in 64 bits. Row statistics that are inputs are taken as they are."""
    state = prepare(case, seed)
    t = {k: v.double() for k, v in state.items() if torch.is_tensor(v) and v.is_floating_point()}
    c = math.sqrt(2.0 / math.pi)
    if case["op"] == "linear":
        z = torch.addmm(t["bias"], t["X"], t["K"])
        if case["residual"] == "first":
            z += t["R"]
        if case["act"] == "relu":
            y = z.clamp(min=0.0)
        elif case["act"] == "silu":
            y = z / (1.0 + torch.exp(-z))
        elif case["act"] == "gelu":
            y = 0.5 * z * (1.0 + torch.tanh(c * (z + 0.044715 * z ** 3)))
        else:
            y = z
        if case["residual"] == "last":
            y = y + t["R"]
        return [y, z] if case["save"] else [y]
    if case["op"] == "linear_grad":
        z = t["Z"]
        if case["act"] == "relu":
            slope = (z > 0).double()
        elif case["act"] == "silu":
            e = torch.exp(-z)
            slope = (1.0 + e + z * e) / (1.0 + e) ** 2
        elif case["act"] == "gelu":
            h = torch.tanh(c * (z + 0.044715 * z ** 3))
            slope = 0.5 * (1.0 + h) + 0.5 * z * (1.0 - h * h) * c * (1.0 + 0.134145 * z * z)
        else:
            slope = torch.ones_like(z)
        dz = t["G"] * slope
        return [dz @ t["K"].t().contiguous(), t["X"].t().contiguous() @ dz, dz.sum(0), dz]
    if case["op"] == "norm":
        var, mean = torch.var_mean(t["X"], 1, correction=0, keepdim=True)
        rstd = (var + NORM_EPS) ** -0.5
        return [torch.addcmul(t["beta"], (t["X"] - mean) * rstd, t["gamma"]), mean[:, 0], rstd[:, 0]]
    if case["op"] == "norm_grad":
        n = case["channels"]
        xh = (t["X"] - t["mean"][:, None]) * t["rstd"][:, None]
        w = t["G"] * t["gamma"]
        dots = (w * xh).sum(1, keepdim=True)
        return [t["rstd"][:, None] / n * (n * w - w.sum(1, keepdim=True) - xh * dots), (t["G"] * xh).sum(0), t["G"].sum(0)]
    a, b, c5 = COEFFICIENTS
    out = []
    for u in t["U"]:
        x = u / (torch.linalg.vector_norm(u) + ORTH_EPS)
        for _ in range(STEPS):  # p(X) = a X + b (X X^T) X + c (X X^T)^2 X, from the right or from the left
            if x.shape[0] > x.shape[1]:
                y = x @ (x.t().contiguous() @ x)
                x = a * x + b * y + c5 * (y @ (x.t().contiguous() @ x))
            else:
                y = (x @ x.t().contiguous()) @ x
                x = a * x + b * y + c5 * ((x @ x.t().contiguous()) @ y)
        out.append(x)
    return [torch.stack(out)]
