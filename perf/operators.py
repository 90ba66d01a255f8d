"""The operators of a training step behind the gathered feature blocks, and the calls they are timed by: layer norm with its
gradients, and the orthogonalised update of the weights.

A case is a dict of plain values.  "op" says what one pass runs:

  norm       layer norm of every row: y and the rows' mean and 1 / deviation
  norm_step  the same, then its gradients from dy: y, dx, dweight, dbias ("input": rows that are data, so no dx)
  orth       the orthogonalised form of each of the matrices named by "shapes" (Newton-Schulz products)
  muon       one step of an optimiser on them: momentum, orthogonalised update, decay, new weights

own = False computes each in elementary torch operations in 32 bits, rounded once at the end; own = True calls the library.
"""
import math

import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
EPS_NORM, EPS_ORTH, STEPS = 1e-5, 1e-7, 5
A, B, C = 3.4445, -4.7750, 2.0315            # the quintic's coefficients
LR, DECAY, MOMENTUM = 0.02, 0.01, 0.95


def _norm(name, op, rows, cols, dtype, weight="float32", pad=0, **kw):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, weight=weight, pad=pad, **dict(dict(input=False), **kw))


def _mats(name, op, shapes, dtype, nesterov=True):
    return dict(name=name, op=op, shapes=shapes, dtype=dtype, nesterov=nesterov)


def listed():
    return [
        # The input block of a small graph's batch: one call among many small ones, so its latency counts.
        _norm("norm_small", "norm", 256, 64, "float32"),
        # The input block of a batch of the dense graph as it was gathered: 602 features in rows padded to 16 bytes.  The
        # rows are data, so only the weight's and the bias' gradients are wanted.
        _norm("norm_features", "norm_step", 199_000, 602, "float32", pad=2, input=True),
        # Hidden rows of the graph with large fan-outs, bf16 between layers, the norm's weights in fp32.
        _norm("norm_hidden", "norm_step", 150_000, 256, "bfloat16"),
        # Rows of a wide model.
        _norm("norm_wide", "norm_step", 8192, 8192, "bfloat16", weight="bfloat16"),
        # An odd width, rows back to back: no row but the first starts at a multiple of four bytes.
        _norm("norm_odd", "norm_step", 10_007, 1001, "float16"),
        # Few long rows.
        _norm("norm_long_rows", "norm", 61, 131_071, "float32"),
        # The classifier of a node classification model alone: the smallest matrix.
        _mats("orth_classifier", "orth", "47x256", "bfloat16"),
        # All weights of a GraphSAGE model over the dense graph's features: self and neighbours side by side.
        _mats("muon_sage", "muon", "256x1204,256x512,41x512", "float32"),
        # The matrices of one size of a stack of layers.
        _mats("muon_stack", "muon", ",".join(["1024x4096"] * 6), "bfloat16"),
        # A tall matrix of odd sides.
        _mats("orth_tall", "orth", "1999x517", "float32"),
        # A square matrix in fp32, plain momentum.
        _mats("muon_square", "muon", "2048x2048", "float32", nesterov=False),
        # The largest.
        _mats("orth_large", "orth", "4096x4096", "bfloat16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["float32", "float32", "bfloat16", "bfloat16", "float16"])
    if rng.random() < 0.5:
        cols = _log_int(rng, 1, 16_384) if rng.random() < 0.9 else _log_int(rng, 16_384, 131_072)
        rows = min(_log_int(rng, 1, 300_000), 100_000_000 // cols)
        case = _norm("", rng.choice(["norm", "norm_step", "norm_step"]), rows, cols, dtype, weight=rng.choice(["float32", dtype]),
                     pad=rng.choice([0, 0, rng.randint(1, 16), -cols % 8]), input=rng.random() < 0.2)
        if case["op"] == "norm":
            case["input"] = False
    else:
        shapes, left = [], 1.3e12 if dtype != "float32" else 3e11
        for _ in range(rng.choice([1, 1, 2, 3, 6, 12])):
            r, c = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
            while _products(r, c) > left:
                r, c = r // 2 + 1, c // 2 + 1
            left -= _products(r, c)
            shapes.append(f"{r}x{c}")
            if left < 1e11:
                break
        case = _mats("", rng.choice(["orth", "muon"]), ",".join(shapes), dtype, nesterov=rng.random() < 0.5)
    del case["name"]
    return case


def _shapes(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["shapes"].split(",")]


def _products(r, c):
    """Operations of the Newton-Schulz products: of the two symmetric ones only one half is needed."""
    n, m = min(r, c), max(r, c)
    return STEPS * (n * (n + 1) * m + n * (n + 1) * n + 2 * n * n * m)


def work(case):
    if case["op"] in ("norm", "norm_step"):
        n, d, b, wb = case["rows"], case["cols"], _BYTES[case["dtype"]], _BYTES[case["weight"]]
        if case["op"] == "norm":
            return {"bytes": 2 * n * d * b + 8 * n + 2 * d * wb, "flops": 8 * n * d}
        tensors = 3 if case["input"] else 4                              # x, dy, y, dx
        return {"bytes": tensors * n * d * b + 16 * n + 5 * d * wb, "flops": (8 + 12) * n * d}
    b = _BYTES[case["dtype"]]
    elements = sum(r * c for r, c in _shapes(case))
    flops = sum(_products(r, c) for r, c in _shapes(case))
    return {"bytes": elements * (2 * b if case["op"] == "orth" else 3 * b + 8), "flops": flops}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + 29) & 0x7FFFFFFF)
    t = _TYPES[case["dtype"]]

    def normal(*size):
        return torch.randn(size, generator=g, device="cuda", dtype=torch.float32)

    if case["op"] in ("norm", "norm_step"):
        n, d, wt = case["rows"], case["cols"], _TYPES[case["weight"]]
        # rows of different sizes around a mean that is not zero, in a buffer of longer rows where "pad" says so
        buffer = torch.zeros((n, d + case["pad"]), dtype=t, device="cuda")
        x = buffer[:, :d]
        x.copy_(normal(n, d) * torch.exp(0.5 * normal(n, 1)) + 0.3 * normal(1, d) + 0.5 * normal(n, 1))
        s = dict(case=case, x=x, weight=(1 + 0.2 * normal(d)).to(wt), bias=(0.1 * normal(d)).to(wt))
        if case["op"] == "norm_step":
            s["dy"] = (normal(n, d) * torch.exp(0.5 * normal(n, 1))).to(t)         # of a scaled loss
        return s

    def gradient(r, c):
        # error rows times activations that are never negative, of columns of different sizes, summed over samples
        k = max(1024, 2 * max(r, c))
        h = torch.relu(normal(k, c) + 0.5) * torch.exp(0.5 * normal(1, c))
        return (normal(k, r) * torch.exp(0.5 * normal(k, 1))).t() @ h / k

    sh = _shapes(case)
    s = dict(case=case, grad=[gradient(r, c).to(t) for r, c in sh])
    if case["op"] == "muon":
        s["momentum"] = [8 * gradient(r, c) for r, c in sh]
        s["weight"] = [(normal(r, c) / math.sqrt(c)).to(t) for r, c in sh]
    return s


# ---------------------------------------------------------------- the plain form
def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(dim=1, keepdim=True) + EPS_NORM)
    xhat = c * rstd
    w = s["weight"].float()
    y = (xhat * w + s["bias"].float()).to(s["x"].dtype)
    if s["case"]["op"] == "norm":
        return dict(y=y, mean=mean[:, 0], rstd=rstd[:, 0])
    dy = s["dy"].float()
    out = dict(y=y, dweight=(dy * xhat).sum(dim=0).to(s["weight"].dtype), dbias=dy.sum(dim=0).to(s["bias"].dtype))
    if not s["case"]["input"]:
        q = dy * w
        out["dx"] = (rstd * (q - q.mean(dim=1, keepdim=True) - xhat * (q * xhat).mean(dim=1, keepdim=True))).to(s["x"].dtype)
    return out


def _plain_orth(u):
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / (x.square().sum().sqrt() + EPS_ORTH)
    for _ in range(STEPS):
        gram = x @ x.t()
        x = A * x + (B * gram + C * (gram @ gram)) @ x
    return x.t() if tall else x


def _plain_muon(weight, momentum, grad, nesterov):
    g, w = grad.float(), weight.float()
    m = MOMENTUM * momentum + g
    o = _plain_orth(g + MOMENTUM * m if nesterov else m)
    scale = math.sqrt(max(1.0, w.shape[0] / w.shape[1]))
    return (w - LR * DECAY * w - LR * scale * o).to(weight.dtype), m


def run(s):
    case = s["case"]
    if not own:
        if case["op"] in ("norm", "norm_step"):
            return _plain_norm(s)
        if case["op"] == "orth":
            return [_plain_orth(u.float()).to(u.dtype).contiguous() for u in s["grad"]]
        new = [_plain_muon(w, m, u, case["nesterov"]) for w, m, u in zip(s["weight"], s["momentum"], s["grad"])]
        return dict(weight=[w for w, _ in new], momentum=[m for _, m in new])

    from paper_2509_05207_amd import binding as rg
    if case["op"] in ("norm", "norm_step"):
        y, mean, rstd = rg.rg_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS_NORM)
        if case["op"] == "norm":
            return dict(y=y, mean=mean, rstd=rstd)
        dx, dweight, dbias = rg.rg_layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd, want_dx=not case["input"])
        out = dict(y=y, dweight=dweight, dbias=dbias)
        if not case["input"]:
            out["dx"] = dx
        return out
    if case["op"] == "orth":
        return rg.rg_orthogonalize(s["grad"], steps=STEPS, eps=EPS_ORTH)
    # a step that leaves the weights and momenta that it started from (a program that can go back to them keeps both)
    weight = [torch.empty_like(w) for w in s["weight"]]
    momentum = [torch.empty_like(m) for m in s["momentum"]]
    rg.rg_muon_step(s["weight"], s["grad"], s["momentum"], lr=LR, weight_decay=DECAY, momentum=MOMENTUM, nesterov=case["nesterov"],
                    steps=STEPS, eps=EPS_ORTH, out_weights=weight, out_momenta=momentum)
    return dict(weight=weight, momentum=momentum)


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _exact_norm(case, s):
    x = s["x"].double()
    d = case["cols"]
    mean = x.sum(dim=1) / d
    x -= mean[:, None]
    rstd = 1 / torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / d + EPS_NORM)
    x *= rstd[:, None]                                                     # xhat
    out = dict(y=torch.addcmul(s["bias"].double(), x, s["weight"].double()))
    if case["op"] == "norm":
        return dict(out, mean=mean, rstd=rstd)
    dy = s["dy"].double()
    out["dbias"] = torch.ones(case["rows"], dtype=torch.float64, device=x.device) @ dy
    out["dweight"] = torch.linalg.vecdot(dy, x, dim=0)
    if not case["input"]:
        # the Jacobian of xhat is rstd (I - 1 1^T / d - xhat xhat^T / d)
        dy *= s["weight"].double()
        along = torch.linalg.vecdot(dy, x, dim=1) / d
        dy -= dy.sum(dim=1, keepdim=True) / d
        dy -= x * along[:, None]
        out["dx"] = dy * rstd[:, None]
    return out


def _exact_orth(u):
    """The same polynomial from the right: x (a + s (b + c s)) with s = x^T x of the narrower side."""
    x = u if u.shape[0] >= u.shape[1] else u.t()
    x = x / (torch.linalg.vector_norm(x) + EPS_ORTH)
    eye = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        s = x.t().contiguous() @ x.contiguous()
        x = x @ (A * eye + s @ (B * eye + C * s))
    return x if u.shape[0] >= u.shape[1] else x.t()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_step"):
        return _exact_norm(case, s)
    if case["op"] == "orth":
        return [_exact_orth(u.double()).contiguous() for u in s["grad"]]
    weight, momentum = [], []
    for w, m, u in zip(s["weight"], s["momentum"], s["grad"]):
        w, u = w.double(), u.double()
        m = m.double() * MOMENTUM + u
        o = _exact_orth(u + m * MOMENTUM if case["nesterov"] else m)
        weight.append((1 - LR * DECAY) * w - LR * max(1.0, w.shape[0] / w.shape[1]) ** 0.5 * o)
        momentum.append(m)
    return dict(weight=weight, momentum=momentum)
