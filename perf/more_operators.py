"""Rows held in 8 bits and the products on them, and the calls they are timed by.

A held row is its codes (int8), zeros, and its scale (fp32) in the last four of 16 ceil((cols + 4) / 16) bytes, so that a gather moves it as
it moves any row.  A case is a dict of plain values.  "op" says what one pass runs:

  hold      rows are quantised as they are written to a buffer ("pick": those of some positions of a table), and read back
  read      rows of a held table, picked by their positions, read back
  product   y = x w^T + bias of held rows x and held weights w, a scale for each row of either
  backward  what dy gives of it: dx, dweight, dbias ("input": rows that are data, so no dx)

own = False computes each in elementary torch operations in 32 bits, rounded once at the end (quotients next to a border in 64); own = True
calls the library.
"""
import math

import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
LEAST = 2.0 ** -126


def _rows(name, op, rows, cols, dtype, pick=0, pad=0):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, pick=pick, pad=pad)


def _product(name, op, rows, cols, outs, dtype, bias=True, input=False):
    return dict(name=name, op=op, rows=rows, cols=cols, outs=outs, dtype=dtype, bias=bias, input=input)


def listed():
    return [
        # The activations of a small batch held for the backward pass: one call among many small ones, so its latency counts.
        _rows("hold_small", "hold", 256, 64, "float32"),
        # The input block of a batch of the dense graph, as it was gathered: 602 features in rows padded to 16 bytes.
        _rows("hold_features", "hold", 199_000, 602, "float32", pad=2),
        # A cache of hot rows as it is written: 200,000 of a table's million.
        _rows("hold_hot", "hold", 200_000, 256, "bfloat16", pick=1_000_000),
        # A batch's rows out of a table that is held in 8 bits.
        _rows("read_block", "read", 199_000, 602, "bfloat16", pick=233_000),
        # A few rows for an answer.
        _rows("read_few", "read", 1_000, 100, "float32", pick=100_000),
        # One row through a wide layer: serving.
        _product("product_one", "product", 1, 4096, 4096, "bfloat16"),
        # A hidden layer of the graph with large fan-outs: self and neighbours side by side.
        _product("product_hidden", "product", 150_000, 512, 256, "bfloat16"),
        # Odd sides.
        _product("product_odd", "product", 10_007, 1001, 517, "float32"),
        # The largest.
        _product("product_large", "product", 8192, 8192, 8192, "bfloat16", bias=False),
        # The first layer over the dense graph's features: data, so no dx.
        _product("backward_features", "backward", 199_000, 602, 256, "float32", input=True),
        # The hidden layer's backward pass.
        _product("backward_hidden", "backward", 150_000, 512, 256, "bfloat16"),
        # A wide layer's.
        _product("backward_wide", "backward", 8192, 4096, 4096, "bfloat16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["float32", "float32", "bfloat16", "bfloat16", "float16"])
    op = rng.choice(["hold", "read", "product", "product", "backward", "backward"])
    if op in ("hold", "read"):
        cols = _log_int(rng, 1, 16_384) if rng.random() < 0.9 else _log_int(rng, 16_384, 131_072)
        rows = min(_log_int(rng, 1, 300_000), 100_000_000 // cols)
        pick = min(_log_int(rng, 1, 1_000_000), 200_000_000 // cols) if op == "read" or rng.random() < 0.3 else 0
        case = _rows("", op, rows, cols, dtype, pick=pick, pad=0 if pick else rng.choice([0, 0, rng.randint(1, 16), -cols % 8]))
    else:
        rows = _log_int(rng, 1, 64) if rng.random() < 0.2 else _log_int(rng, 1, 300_000)
        cols, outs = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
        if op == "product" and rng.random() < 0.05:
            cols = _log_int(rng, 8192, 131_072)
        most = 2e11 if op == "product" else 1e11 if dtype != "float32" else 3e10
        while rows * cols * outs > most or rows * max(cols, outs) > 130_000_000:
            rows, cols, outs = rows * 2 // 3 + 1, cols * 4 // 5 + 1, outs * 4 // 5 + 1
        case = _product("", op, rows, cols, outs, dtype, bias=rng.random() < 0.7, input=op == "backward" and rng.random() < 0.2)
    del case["name"]
    return case


def _held_bytes(cols):
    return (cols + 4 + 15) // 16 * 16


def work(case):
    n, d, b = case["rows"], case["cols"], _BYTES[case["dtype"]]
    if case["op"] == "hold":
        return {"bytes": n * d * b + 2 * n * (d + 4) + n * d * b + (8 * n if case["pick"] else 0), "flops": 4 * n * d}
    if case["op"] == "read":
        return {"bytes": n * (d + 4) + n * d * b + 8 * n, "flops": n * d}
    m = case["outs"]
    if case["op"] == "product":
        return {"bytes": (n + m) * (d + 4) + n * m * b + (4 * m if case["bias"] else 0), "flops": 2 * n * m * d}
    if case["input"]:
        return {"bytes": n * m * b + n * (d + 4) + m * d * b + m * b, "flops": 2 * n * m * d}
    return {"bytes": n * m * b + (n + m) * (d + 4) + (n + m) * d * b + m * b, "flops": 4 * n * m * d}


# ---------------------------------------------------------------- held rows in plain operations
def _codes_and_scale(x):
    """Quotients in 64 bits: what lies next to the border between two codes goes where the exact quotient says."""
    scale = (x.float().abs().amax(dim=1) / 127).clamp(min=LEAST)
    return torch.round(x.double() / scale.double()[:, None]), scale


def _pack(x):
    codes, scale = _codes_and_scale(x)
    held = torch.zeros((x.shape[0], _held_bytes(x.shape[1])), dtype=torch.uint8, device=x.device)
    held[:, : x.shape[1]] = codes.to(torch.int8).view(torch.uint8)
    held.view(torch.float32)[:, -1] = scale
    return held


def _values(held, cols):
    return held[:, :cols].view(torch.int8).float() * held.view(torch.float32)[:, -1:]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + 47) & 0x7FFFFFFF)
    t, n, d = _TYPES[case["dtype"]], case["rows"], case["cols"]

    def normal(*size):
        return torch.randn(size, generator=g, device="cuda", dtype=torch.float32)

    def activations(r, c):
        # columns and rows of different sizes, as features and hidden layers have them
        return normal(r, c).mul_(torch.exp(0.5 * normal(r, 1))).mul_(torch.exp(0.3 * normal(1, c)))

    if case["op"] in ("hold", "read"):
        table = case["pick"] or n
        s = dict(case=case, pick=torch.randint(table, (n,), generator=g, device="cuda") if case["pick"] else None)
        if case["op"] == "read":
            s["held"] = _pack(activations(table, d))
        else:
            x = torch.zeros((table, d + case["pad"]), dtype=t, device="cuda")[:, :d]
            s["x"] = x.copy_(activations(table, d))
        return s
    m = case["outs"]
    s = dict(case=case, x=_pack(torch.relu_(activations(n, d) + 0.5)), w=_pack(normal(m, d) / math.sqrt(d)))
    if case["op"] == "product":
        s["bias"] = 0.1 * normal(m) if case["bias"] else None
    else:
        s["dy"] = (normal(n, m) * torch.exp(0.5 * normal(n, 1)) / math.sqrt(n)).to(t)
    return s


# ---------------------------------------------------------------- the plain form
def _plain(s):
    case = s["case"]
    t, d = _TYPES[case["dtype"]], case["cols"]
    if case["op"] == "hold":
        codes, scale = _codes_and_scale(s["x"] if s["pick"] is None else s["x"][s["pick"]])
        return dict(values=(codes.float() * scale[:, None]).to(t), scale=scale)
    if case["op"] == "read":
        return _values(s["held"][s["pick"]], d).to(t)
    if case["op"] == "product":
        y = _values(s["x"], d) @ _values(s["w"], d).t()
        return (y + s["bias"] if case["bias"] else y).to(t)
    dy = s["dy"].float()
    out = dict(dweight=(dy.t() @ _values(s["x"], d)).to(t), dbias=dy.sum(dim=0).to(t))
    if not case["input"]:
        out["dx"] = (dy @ _values(s["w"], d)).to(t)
    return out


def run(s):
    if not own:
        return _plain(s)
    from paper_2509_05207_amd import binding as rg
    case = s["case"]
    t, d = _TYPES[case["dtype"]], case["cols"]
    if case["op"] == "hold":
        held = rg.rg_quantize_rows(s["x"], rows=s["pick"])
        return dict(values=rg.rg_dequantize_rows(held, d, dtype=t), scale=held.view(torch.float32)[:, -1])
    if case["op"] == "read":
        return rg.rg_dequantize_rows(s["held"], d, dtype=t, rows=s["pick"])
    if case["op"] == "product":
        return rg.rg_rows8_product(s["x"], s["w"], d, bias=s["bias"], dtype=t)
    dx, dweight, dbias = rg.rg_rows8_product_backward(s["dy"], s["x"], s["w"], d, want_dx=not case["input"])
    out = dict(dweight=dweight, dbias=dbias)
    if not case["input"]:
        out["dx"] = dx
    return out


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _exact_values(held, cols):
    scale = held[:, -4:].contiguous().view(torch.float32).double()
    codes = held[:, :cols].to(torch.float64)
    return torch.where(codes > 127, codes - 256, codes).mul_(scale)


def exact(case, seed):
    s = prepare(case, seed)
    d = case["cols"]
    if case["op"] == "hold":
        x = (s["x"] if s["pick"] is None else torch.index_select(s["x"], 0, s["pick"])).double()
        scale = torch.linalg.vector_norm(x, ord=math.inf, dim=1).div_(127).float().double().clamp_(min=LEAST)
        q = x.div_(scale[:, None])
        low = torch.floor(q)
        part = q - low
        up = (part > 0.5) | ((part == 0.5) & (torch.remainder(low, 2) == 1))
        return dict(values=(low + up).mul_(scale[:, None]), scale=scale)
    if case["op"] == "read":
        return _exact_values(torch.index_select(s["held"], 0, s["pick"]), d)
    if case["op"] == "product":
        y = torch.mm(_exact_values(s["x"], d), _exact_values(s["w"], d).t().contiguous())
        return y.add_(s["bias"].double()) if case["bias"] else y
    dy = s["dy"].double()
    out = dict(dweight=torch.mm(dy.t().contiguous(), _exact_values(s["x"], d)), dbias=torch.mv(dy.t().contiguous(), torch.ones(case["rows"], dtype=torch.float64, device=dy.device)))
    if not case["input"]:
        out["dx"] = torch.mm(dy, _exact_values(s["w"], d))
    return out
