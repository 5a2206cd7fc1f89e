"""Layers on top of states, as measurable cases: linear layers on every cell in
microscaled 4 bits, their gradients, and dropout without a stored mask.

  call "quantise"  ``runtime.MX4Matrix``: rows of values to 4 bits and back
  call "linear"    ``runtime.CellLayer.forward``: rows quantised and multiplied
                   with 4-bit weights
  call "product"   the same from rows that are held in 4 bits already
  call "backward"  ``runtime.CellLayer.backward``: gradients of a layer's input,
                   weights and bias
  call "dropout"   ``runtime.Dropout``: forward (x dropped, or added to another
                   tensor) and gradient (gated by the layer's output)

Rows are cells: the features of a state (C, 2C or H values of the package's
models), or of generic layers.  ``pad`` is the distance from a row's end to the
next one's start.
"""
import math

import torch

own = False

BLOCK = 32
_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _quantise(name, rows, cols, dtype, pad=0):
    return {"name": name, "call": "quantise", "rows": rows, "cols": cols, "dtype": dtype,
            "pad": pad}


def _layer(name, call, rows, cols, outs, dtype, out, bias=True, relu=False, pad=0):
    """rows x cols inputs of `dtype` (or 4 bits), `outs` outputs of type `out`.
    Gradients: `dtype` is the type of both the outputs' and the inputs'."""
    return {"name": name, "call": call, "rows": rows, "cols": cols, "outs": outs, "dtype": dtype,
            "out": out, "bias": bias, "relu": relu, "pad": pad}


def _dropout(name, rows, cols, dtype, rate, gate=False, add=False, pad=0):
    return {"name": name, "call": "dropout", "rows": rows, "cols": cols, "dtype": dtype,
            "rate": rate, "gate": gate, "add": add, "pad": pad}


def listed():
    return [
        # perception features (2C) of a 320 x 320 training patch, kept for a backward
        _quantise("quantise_patch_320", 320 * 320, 32, "f32"),
        # hidden units of the large model's cells in a volume: odd rows, a part of a block
        _quantise("quantise_volume_100", 1_228_811, 100, "f16", pad=4),
        # one cell through a wide layer: all latency
        _layer("linear_one_4096", "linear", 1, 4096, 4096, "bf16", "bf16", relu=True),
        # the features of a 1024 x 1024 image to the model's hidden units
        _layer("linear_cells_1024", "linear", 1024 * 1024, 32, 64, "f32", "f16", relu=True),
        # the largest layer
        _layer("linear_large", "linear", 16384, 8192, 8192, "bf16", "bf16"),
        # hidden units kept in 4 bits to scores of 19 classes, for every cell of an image
        _layer("product_classes_19", "product", 1024 * 1024, 64, 19, "mx4", "f32"),
        # a few rows of odd sizes
        _layer("product_ragged", "product", 1000, 517, 1003, "mx4", "f32"),
        # gradients of the patch's layer
        _layer("backward_patch_320", "backward", 320 * 320, 32, 64, "f32", "f32"),
        # gradients of a large layer
        _layer("backward_large", "backward", 8192, 4096, 4096, "bf16", "bf16"),
        # hidden units of a 64 x 64 image, as they leave a ReLU: a launch
        _dropout("dropout_tiny_64", 64 * 64, 64, "f32", 0.1, gate=True),
        # gradients of odd rows, gated
        _dropout("dropout_odd_rows", 102_403, 517, "f16", 0.5, gate=True, pad=3),
        # a large activation dropped and added to what it updates
        _dropout("dropout_large_add", 131_072, 4096, "bf16", 0.1, add=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds, sizes over the whole range."""
    call = rng.choice(["quantise", "linear", "linear", "product", "backward", "dropout"])
    pad = rng.choice([0, 0, 0, 1, 8])
    dtype = rng.choice(["f32", "f16", "bf16"])
    cols = _log(rng, 1, 8192)
    if call in ("quantise", "dropout"):
        values = _log(rng, 1000, 3e8)
        rows = max(1, values // cols)
        if call == "quantise":
            case = _quantise(None, rows, cols, dtype, pad)
        else:
            case = _dropout(None, rows, cols, dtype, rng.choice([0.0, 0.1, 0.5, rng.random()]),
                            rng.random() < 0.5, rng.random() < 0.3, pad)
    else:
        outs = _log(rng, 1, 8192)
        # rows within 2^28 values on either side, and half the largest products
        most = min(2e6, 2 ** 28 / max(cols, outs), 5e11 / cols / outs)
        rows = _log(rng, 1, max(1.0, most))
        out = rng.choice([dtype, "f32"]) if call != "backward" else dtype
        case = _layer(None, call, rows, cols, outs, "mx4" if call == "product" else dtype, out,
                      rng.random() < 0.7, rng.random() < 0.5 and call != "backward", pad)
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rows(x, pad):
    """x with its rows `pad` values apart."""
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _features(gen, rows, cols):
    """Values of cells: channels of very different magnitude, a part of the
    cells all zero (background)."""
    x = torch.empty((rows, cols), device="cuda").normal_(generator=gen)
    x.mul_(torch.exp2(torch.rand(cols, generator=gen, device="cuda") * 8 - 5))
    empty = torch.rand(rows, generator=gen, device="cuda") < 0.1
    return x.mul_((~empty)[:, None])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, call = case["rows"], case["cols"], case["call"]
    st = {}
    if call == "quantise":
        st["x"] = _rows(_features(gen, rows, cols).to(_TYPES[case["dtype"]]), case["pad"])
    elif call == "dropout":
        x = torch.empty((rows, cols), device="cuda").normal_(generator=gen)
        st["x"] = _rows(x.to(_TYPES[case["dtype"]]), case["pad"])
        for k in ("gate", "add"):
            if case[k]:
                x.normal_(generator=gen)
                if k == "gate":     # what a ReLU has left of it
                    x.clamp_(min=0.0)
                st[k] = _rows(x.to(_TYPES[case["dtype"]]), case["pad"])
            else:
                st[k] = None
        st["seed"] = 1_000_003 * seed + 12_345_678_901
        st["index"] = (seed * 7919) % 100_000
    else:
        outs = case["outs"]
        w = torch.empty((outs, cols), device="cuda").normal_(generator=gen)
        w.mul_(1.0 / math.sqrt(cols))
        st["w"] = _plain_quantise(w)     # the values that 4-bit weights stand for
        st["bias"] = (torch.randn(outs, generator=gen, device="cuda") * 0.1 if case["bias"]
                      else None)
        if call == "backward":
            g = torch.empty((rows, outs), device="cuda").normal_(generator=gen)
            # most of a gradient is small; some cells have none
            g.mul_(torch.exp2(torch.rand(rows, 1, generator=gen, device="cuda") * 10 - 10))
            g.mul_(torch.rand(rows, 1, generator=gen, device="cuda") < 0.9)
            st["grad"] = _rows(g.to(_TYPES[case["dtype"]]), case["pad"])
            del g
        x = _features(gen, rows, cols)
        if call == "linear":
            st["x"] = _rows(x.to(_TYPES[case["dtype"]]), case["pad"])
        else:
            st["kept"] = _plain_quantise(x)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    rows, cols, call = case["rows"], case["cols"], case["call"]
    if call in ("quantise", "dropout"):
        st["out"] = _rows(torch.zeros_like(st["x"], memory_format=torch.contiguous_format),
                          case["pad"])
    elif call == "backward":
        st["out"] = torch.zeros((rows, cols), dtype=_TYPES[case["dtype"]], device="cuda")
    else:
        st["out"] = _rows(torch.zeros((rows, case["outs"]), dtype=_TYPES[case["out"]],
                                      device="cuda"), case["pad"])
    if own:
        from paper_2508_06993_amd.runtime import CellLayer, Dropout, MX4Matrix
        if call == "quantise":
            st["mx"] = MX4Matrix(rows, cols)
        elif call == "dropout":
            st["drop"] = Dropout(case["rate"], st["seed"])
        else:
            bias = st["bias"]
            if call == "backward":      # a layer without a bias has no gradient of it
                bias = torch.zeros(case["outs"], device="cuda")
            st["layer"] = CellLayer(st["w"], bias, rows=rows, train=call == "backward")
            if "kept" in st:
                st["mx"] = MX4Matrix(rows, cols).quantise(st["kept"])
    st["case"] = case
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _plain_quantise(x):
    """The values that 4 bits hold of x [rows][cols], in fp32."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    x = x.float()
    if cols % BLOCK:
        x = torch.cat([x, x.new_zeros(rows, blocks * BLOCK - cols)], 1)
    x = x.reshape(rows, blocks, BLOCK)
    # a = f 2^e with f in [1/2, 1): a <= 6 * 2^k from k = e - 3 on if f <= 3/4
    frac, exp = torch.frexp(x.abs().amax(2, keepdim=True))
    exp = torch.where(frac > 0.75, exp - 2, exp - 3).clamp_(min=-127)
    x = torch.ldexp(x, -exp)
    # steps of 1/2 below 2, of 1 below 4, of 2 above (round takes ties to even)
    mag = x.abs()
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    x = torch.ldexp((x / step).round_().mul_(step), exp)
    x = x.reshape(rows, blocks * BLOCK)
    return x[:, :cols].contiguous() if cols % BLOCK else x


def _plain_layer(st, case):
    x = st["kept"] if case["call"] == "product" else _plain_quantise(st["x"])
    y = x @ st["w"].t()
    if st["bias"] is not None:
        y += st["bias"]
    if case["relu"]:
        y.clamp_(min=0.0)
    st["out"].copy_(y)
    return {"out": st["out"]}


def _plain_backward(st):
    g = st["grad"].float()
    st["out"].copy_(g @ st["w"])
    return {"input": st["out"], "weight": g.t() @ st["kept"], "bias": g.sum(0)}


_MASK = 0xFFFFFFFF


def _plain_draws(n, seed, index):
    """The first n 32-bit draws of Philox4x32-10 with counter (e >> 2, index)."""
    group = torch.arange((n + 3) // 4, device="cuda")
    c = [group & _MASK, group >> 32, torch.full_like(group, index & _MASK),
         torch.full_like(group, index >> 32)]
    k0, k1 = seed & _MASK, seed >> 32 & _MASK
    for _ in range(10):
        # products modulo 2^64: the low 64 bits do not depend on the sign
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32 & _MASK) ^ c[1] ^ k0, q & _MASK, (p >> 32 & _MASK) ^ c[3] ^ k1, p & _MASK]
        k0, k1 = k0 + 0x9E3779B9 & _MASK, k1 + 0xBB67AE85 & _MASK
    return torch.stack(c, 1).reshape(-1)[:n]


def _plain_dropout(st, case):
    shape = st["x"].shape
    threshold = min(2 ** 32, math.floor(_f32(case["rate"]) * 2.0 ** 32))
    kept = (_plain_draws(shape.numel(), st["seed"], st["index"]) >= threshold).reshape(shape)
    if st["gate"] is not None:
        kept &= st["gate"] > 0
    y = torch.where(kept, st["x"].float() * _f32(2.0 ** 32 / (2 ** 32 - threshold)), 0.0)
    if st["add"] is not None:
        y += st["add"]
    st["out"].copy_(y)
    return {"out": st["out"]}


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def run(state):
    case, call = state["case"], state["case"]["call"]
    if call == "quantise":
        if own:
            state["mx"].quantise(state["x"])
            return {"values": state["mx"].dequantise(state["out"])}
        state["out"].copy_(_plain_quantise(state["x"]))
        return {"values": state["out"]}
    if call == "dropout":
        if own:
            return {"out": state["drop"](state["x"], state["out"], gate=state["gate"],
                                         add=state["add"], index=state["index"])}
        return _plain_dropout(state, case)
    if call == "backward":
        if own:
            layer = state["layer"]
            layer.backward(state["grad"], state["out"], kept=state["mx"])
            return {"input": state["out"], "weight": layer.grad_weight, "bias": layer.grad_bias}
        return _plain_backward(state)
    if own:
        x = state["mx"] if call == "product" else state["x"]
        return {"out": state["layer"].forward(x, state["out"], relu=case["relu"])}
    return _plain_layer(state, case)


# ---------------------------------------------------------------------------
# work, and the definition in 64 bits
# ---------------------------------------------------------------------------

def _mx4_bytes(rows, cols):
    return rows * -(-cols // BLOCK) * 17


def work(case):
    rows, cols, call = case["rows"], case["cols"], case["call"]
    held = _mx4_bytes(rows, cols)
    if call == "quantise":
        return {"bytes": 2 * (rows * cols * _SIZE[case["dtype"]] + held), "flops": 2 * rows * cols}
    if call == "dropout":
        arrays = 2 + case["gate"] + case["add"]
        return {"bytes": rows * cols * _SIZE[case["dtype"]] * arrays, "flops": rows * cols}
    outs = case["outs"]
    n = rows * cols * outs
    weights = _mx4_bytes(outs, cols)
    if call == "backward":
        size = _SIZE[case["dtype"]]
        return {"bytes": rows * (outs + cols) * size + held + weights + 4 * outs * (cols + 1),
                "flops": 4 * n}
    read = held if call == "product" else held + rows * cols * _SIZE[case["dtype"]]
    return {"bytes": read + weights + rows * outs * _SIZE[case["out"]] + 4 * outs * case["bias"],
            "flops": 2 * n}


def _exact_values(x):
    """Each value to the nearest of the 15 values of its block's scale, by
    comparison with the borders between them (ties to the even one)."""
    rows, cols = x.shape
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    borders = (values[1:] + values[:-1]) / 2
    out = torch.empty((rows, cols), dtype=torch.float64, device=x.device)
    for at in range(0, cols, BLOCK):
        part = x[:, at:at + BLOCK].double()
        top = part.abs().max(1, keepdim=True).values
        e = torch.ceil(torch.log2((top / 6).clamp(min=2.0 ** -127)))
        e = torch.where(6 * torch.exp2(e - 1) >= top, e - 1, e)
        e = torch.where(6 * torch.exp2(e) < top, e + 1, e).clamp(min=-127)
        mag = part.abs() / torch.exp2(e)
        # below an even code a border belongs to it, above one too
        low = torch.bucketize(mag, borders)                # borders strictly below mag
        high = torch.bucketize(mag, borders, right=True)   # borders at or below mag
        code = torch.where(high % 2 == 0, high, low)
        out[:, at:at + BLOCK] = values[code] * torch.exp2(e) * torch.sign(part)
    return out


def _exact_draws(n, seed, index):
    """Philox4x32-10, its products from 16-bit halves."""
    def mul(a, m):
        low, high = a * (m & 0xFFFF), a * (m >> 16)
        p = (low & 0xFFFFFFFF) + ((high & 0xFFFF) << 16)
        return (high >> 16) + (low >> 32) + (p >> 32), p & _MASK
    e = torch.arange((n + 3) // 4, dtype=torch.int64, device="cuda")
    x0, x1 = e % 2 ** 32, e // 2 ** 32
    x2, x3 = torch.zeros_like(e) + index % 2 ** 32, torch.zeros_like(e) + index // 2 ** 32
    for i in range(10):
        ka = (seed + i * 0x9E3779B9) % 2 ** 32
        kb = ((seed >> 32) + i * 0xBB67AE85) % 2 ** 32
        h0, l0 = mul(x0, 0xD2511F53)
        h2, l2 = mul(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = torch.bitwise_xor(h2 ^ x1, torch.full_like(e, ka)), l2, \
            torch.bitwise_xor(h0 ^ x3, torch.full_like(e, kb)), l0
    return torch.stack([x0, x1, x2, x3]).t().flatten()[:n]


def exact(case, seed):
    if case["rows"] * max(case["cols"], case.get("outs", 0)) > 600_000_000:
        return None
    st = _inputs(case, seed)
    call = case["call"]
    if call == "quantise":
        return {"values": _exact_values(st["x"])}
    if call == "dropout":
        x = st["x"]
        t = int(_f32(case["rate"]) * 4294967296.0)
        drop = _exact_draws(x.numel(), st["seed"], st["index"]).view(x.shape) < t
        if st["gate"] is not None:
            drop = drop | (st["gate"] <= 0)
        y = x.double() / (1 - t / 4294967296.0)
        y = y.masked_fill(drop, 0.0)
        return {"out": y if st["add"] is None else y + st["add"].double()}
    w = st["w"].double()
    if call == "backward":
        g = st["grad"].double()
        return {"input": torch.matmul(g, w), "weight": torch.matmul(g.t(), st["kept"].double()),
                "bias": g.sum(0)}
    x = st["kept"].double() if call == "product" else _exact_values(st["x"])
    y = torch.matmul(x, w.t())
    if st["bias"] is not None:
        y = y + st["bias"].double()
    return {"out": torch.relu(y) if case["relu"] else y}
