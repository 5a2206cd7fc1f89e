"""The operators around a training step, as measurable cases.

  call "clip"    ``runtime.Parameters.clip``: the global norm of many gradient
                 tensors and their clipped copies
  call "adamw"   ``runtime.Parameters.adamw``: clipped AdamW update of many
                 tensors, with a running average of the weights
  call "keep"    ``runtime.StateCache``: states quantised to 8 bits as they are
                 written into the cache, and read back
  call "gather"  ``runtime.StateCache.read`` of states that the cache holds

Tensor lists are the weights of OctreeNCA models (five tensors per level), of
an ensemble of them, or lists of generic sizes.  Their tensors are views of one
flat buffer, which the outputs show whole: ``gap`` 1 packs them one after the
other (most then start at an odd place), ``gap`` 64 starts each at a multiple of
64 values.  States are those of the package's workloads and of sizes between.
"""
import math
import random

import torch

own = False

SCALES = {"f16": 1.0 / 1024.0}     # fp16 gradients come from a loss times 1024
BETA1, BETA2, EPS, LR = 0.9, 0.99, 1e-8, 1.6e-3
EMA = 0.99
TINY = 2.0 ** -100                 # smallest magnitude that sets a block's scale


def _tensors(name, call, kind, tensors, elements, gap, grad, gnorm, out="f32", ema=False,
             decay=0.0):
    """kind "model 16/64/3": levels of five tensors (channels, hidden, dims);
    "mixed": `tensors` sizes of all magnitudes that add up to `elements`."""
    return {"name": name, "call": call, "kind": kind, "tensors": tensors, "elements": elements,
            "gap": gap, "grad": grad, "gnorm": gnorm, "out": out, "ema": ema, "decay": decay}


def _states(name, call, d, h, w, channels, dtype, code, block, n, slots=0):
    """n states of d x h x w cells, in a cache of `slots` (0: of n)."""
    return {"name": name, "call": call, "d": d, "h": h, "w": w, "channels": channels,
            "dtype": dtype, "code": code, "block": block, "n": n, "slots": slots or n}


def listed():
    return [
        # the gradients of one 5-level pathology model: 25 tensors, all latency
        _tensors("clip_model_5x5", "clip", "model 16/64/2", 25, 0, 64, "f32", 4.0),
        # an ensemble of 16 large volume models, gradients of a scaled loss in fp16
        _tensors("clip_ensemble_320", "clip", "model 20/100/3", 320, 0, 64, "f16", 4.0),
        # many tensors of all sizes packed at odd places, nothing to clip
        _tensors("clip_packed_1000", "clip", "mixed", 1000, 30_000_001, 1, "f32", 0.5),
        # a large list, bf16 in and out
        _tensors("clip_large_bf16", "clip", "mixed", 400, 250_000_000, 64, "bf16", 4.0, out="bf16"),
        # one model's update with the running average, as each training step ends
        _tensors("adamw_model_5x5", "adamw", "model 16/64/2", 25, 0, 64, "f32", 4.0, ema=True),
        # a packed list of odd sizes, fp16 gradients, weight decay
        _tensors("adamw_packed_f16", "adamw", "mixed", 150, 3_000_017, 1, "f16", 4.0, decay=0.01),
        # a large list with everything
        _tensors("adamw_large", "adamw", "mixed", 300, 100_000_000, 64, "bf16", 4.0, ema=True,
                 decay=0.01),
        # one state of a 320 x 320 training patch, kept for its backward step
        _states("keep_patch_320", "keep", 1, 320, 320, 16, "f32", "i8", 64, 1),
        # the ten states of a volume patch of the small model
        _states("keep_volume_12x10", "keep", 12, 96, 96, 12, "f32", "f8", 32, 10),
        # the state of one minute of surgery video, fp16
        _states("keep_video_1min", "keep", 1800, 240, 432, 16, "f16", "i8", 128, 1),
        # the state of a whole slide, the largest call
        _states("keep_slide_184mp", "keep", 1, 11264, 16384, 16, "f32", "i8", 64, 1),
        # a batch of 32 states of the large model drawn from a pool of 256, odd extents
        _states("gather_pool_61x67", "gather", 1, 61, 67, 20, "f32", "i8", 64, 32, 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds, sizes over the whole range."""
    call = rng.choice(["clip", "adamw", "keep", "keep", "gather"])
    if call in ("clip", "adamw"):
        grad = rng.choice(["f32", "f32", "f16", "bf16"])
        out = rng.choice(["f32", grad]) if grad != "f16" else "f32"
        more = dict(out=out) if call == "clip" else dict(ema=rng.random() < 0.5,
                                                         decay=rng.choice([0.0, 0.01]))
        gap, gnorm = rng.choice([1, 64]), rng.choice([0.5, 4.0, 50.0])
        if rng.random() < 0.4:
            kind = rng.choice(["model 16/64/2", "model 16/64/3", "model 12/48/3",
                               "model 20/100/2", "model 20/100/3"])
            case = _tensors(None, call, kind, 5 * _log(rng, 1, 400), 0, gap, grad, gnorm, **more)
        else:
            elements = _log(rng, 1000, 2e8 if call == "clip" else 8e7)
            tensors = min(_log(rng, 1, 2000), elements // 4)
            case = _tensors(None, call, "mixed", tensors, elements, gap, grad, gnorm, **more)
    else:
        cells = _log(rng, 1000, 6e7 if call == "keep" else 2e6)
        d = rng.choice([1, 1, _log(rng, 2, 48)])
        h = max(1, int(math.sqrt(cells / d) * rng.uniform(0.7, 1.4)))
        w = max(1, cells // (d * h))
        n = min(_log(rng, 1, 64), max(1, int(6e7 // cells)))
        slots = n + _log(rng, 1, 64) if call == "gather" else n
        case = _states(None, call, d, h, w, rng.choice([16, 16, 12, 20]),
                       rng.choice(["f32", "f32", "f16"]), rng.choice(["i8", "f8"]),
                       rng.choice([32, 64, 128]), n, min(slots, 120_000_000 // cells + n))
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# shapes
# ---------------------------------------------------------------------------

def _counts(case):
    if case["kind"].startswith("model"):
        c, h, dims = (int(v) for v in case["kind"].split()[1].split("/"))
        level = [c * 3 ** dims, c, 2 * c * h, h, c * h]
        return [level[i % 5] for i in range(case["tensors"])]
    # sizes over four decades, scaled to the total; the last takes the remainder
    n, total = case["tensors"], case["elements"]
    rng = random.Random(n * 1_000_003 + total)
    share = [10.0 ** rng.uniform(0, 4) for _ in range(n)]
    unit = (total - n) / sum(share)
    counts = [1 + int(s * unit) for s in share]
    counts[-1] += total - sum(counts)
    return counts


def _offsets(case):
    """Where each tensor starts in its flat buffer, and the buffer's length."""
    at, gap, starts = 0, case["gap"], []
    for n in _counts(case):
        at = -(-at // gap) * gap
        starts.append(at)
        at += n
    return starts, at


def _cells(case):
    return case["d"] * case["h"] * case["w"]


def _blocks(case):
    return -(-_cells(case) // case["block"])


_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _flat(case, gen, scale, spread=True):
    """A flat buffer of N(0, scale) values; with `spread` each tensor has a
    magnitude of its own.  What lies between the tensors is 0."""
    starts, total = _offsets(case)
    out = torch.randn(total, generator=gen, device="cuda").mul_(scale)
    counts = torch.tensor(_counts(case), device="cuda")
    mag = torch.rand(len(starts), generator=gen, device="cuda") * 1.5 + 0.25
    if not spread:
        mag.fill_(1.0)
    begin = torch.tensor(starts, device="cuda")
    edge = torch.zeros(total + 1, device="cuda")
    edge.index_add_(0, begin, mag)
    edge.index_add_(0, begin + counts, -mag)
    step = torch.cumsum(edge[:total], 0, dtype=torch.float64)
    return out.mul_(torch.where(step > 0.1, step, torch.zeros_like(step)).float())


def _gradient(case, gen):
    g = _flat(case, gen, 1.0)
    norm = torch.linalg.vector_norm(g, dtype=torch.float64)
    g.mul_((case["gnorm"] / norm / SCALES.get(case["grad"], 1.0)).float())
    return g.to(_TYPES[case["grad"]])


def _split(case, flat):
    starts, _ = _offsets(case)
    return [flat[s:s + n] for s, n in zip(starts, _counts(case))]


def _tensor_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"grad": _gradient(case, gen)}
    if case["call"] == "clip":
        st["out"] = torch.zeros(st["grad"].shape, dtype=_TYPES[case["out"]], device="cuda")
    else:
        # moments of a run that has gone on for a while
        typical = case["gnorm"] / math.sqrt(sum(_counts(case)))
        st["param"] = _flat(case, gen, 0.1)
        st["m"] = _flat(case, gen, 0.3 * typical)
        st["v"] = _flat(case, gen, typical).square_()
        st["ema"] = st["param"] * 0.99 if case["ema"] else None
        st["step"] = torch.full((1,), 117, dtype=torch.int64, device="cuda")
    return st


def _state_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, n, slots = case["channels"], case["n"], case["slots"]
    st = {"slots": torch.randperm(slots, generator=gen, device="cuda")[:n].contiguous()}
    out = torch.zeros((n, case["d"], case["h"], case["w"], c), dtype=_TYPES[case["dtype"]],
                      device="cuda")
    if case["call"] == "gather":
        # a pool that earlier steps have filled; one state is drawn twice and one
        # entry asks for a state that does not exist yet (an empty one)
        lo, hi = (-127, 128) if case["code"] == "i8" else (0, 256)
        codes = torch.randint(lo, hi, (slots, _cells(case), c), generator=gen, device="cuda",
                              dtype=torch.int16)
        if case["code"] == "f8":    # the two codes of NaN do not occur
            codes = torch.where((codes & 127) == 127, codes - 1, codes)
        st["codes"] = codes.to(torch.int8 if case["code"] == "i8" else torch.uint8)
        st["scales"] = torch.exp2(torch.randint(-12, 4, (slots, _blocks(case), c), generator=gen,
                                                device="cuda").float())
        if case["code"] == "i8":
            st["scales"] *= 1.0 + torch.rand(st["scales"].shape, generator=gen, device="cuda")
        if n > 2:
            st["slots"][1] = st["slots"][0]
            st["slots"][2] = -1
    else:
        # image channels in [0, 1], hidden channels of very different magnitude
        x = torch.empty(out.shape, dtype=out.dtype, device="cuda").normal_(generator=gen)
        mag = torch.exp2(torch.linspace(-3, 6, c, device="cuda"))
        x.mul_(mag.to(x.dtype))
        x[..., :3] = torch.rand(out.shape[:-1] + (3,), generator=gen, device="cuda",
                                dtype=torch.float32).to(x.dtype)
        st["states"] = x
        code = torch.int8 if case["code"] == "i8" else torch.uint8
        st["codes"] = torch.zeros((slots, _cells(case), c), dtype=code, device="cuda")
        st["scales"] = torch.zeros((slots, _blocks(case), c), device="cuda")
    st["out"] = out
    return st


def prepare(case, seed):
    if case["call"] in ("keep", "gather"):
        st = _state_inputs(case, seed)
        if own:
            import paper_2508_06993_amd as octnca
            from paper_2508_06993_amd.runtime import StateCache
            model = octnca.Model(ndim=3, n_in=3, dtype=case["dtype"], channels=case["channels"],
                                 hidden={12: 48, 16: 64, 20: 100}[case["channels"]])
            st["cache"] = StateCache(model, (case["d"], case["h"], case["w"]), case["slots"],
                                     code=case["code"], block=case["block"], codes=st["codes"],
                                     scales=st["scales"])
    else:
        st = _tensor_inputs(case, seed)
        if own:
            from paper_2508_06993_amd.runtime import Parameters
            views = {k: _split(case, v) for k, v in st.items() if k != "step" and v is not None}
            if case["call"] == "clip":
                st["list"] = Parameters(views["grad"], clipped=views["out"])
            else:
                st["list"] = Parameters(views["grad"], views["param"], views["m"], views["v"],
                                        ema=views.get("ema"), step=st["step"])
    st["case"] = case
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _plain_norm(g, scale, max_norm):
    """(norm, factor of the gradients) of fp32 gradients."""
    norm = g.square().sum().sqrt() * scale
    return norm, torch.where(norm > max_norm, max_norm / norm, torch.ones_like(norm)) * scale


def _plain_clip(st, scale):
    g = st["grad"].float()
    norm, factor = _plain_norm(g, scale, 1.0)
    st["out"].copy_(g * factor)
    return {"norm": norm, "clipped": st["out"]}


def _plain_adamw(st, scale, decay):
    g = st["grad"].float()
    norm, factor = _plain_norm(g, scale, 1.0)
    g = g * factor
    st["step"].add_(1)
    t = st["step"].float()
    p, m, v = st["param"], st["m"], st["v"]
    m.mul_(BETA1).add_(g, alpha=1 - BETA1)
    v.mul_(BETA2).add_(g * g, alpha=1 - BETA2)
    update = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    p.sub_(LR * (update + decay * p))
    if st["ema"] is not None:
        st["ema"].mul_(EMA).add_(p, alpha=1 - EMA)
    return {"norm": norm, "param": p, "m": m, "v": v, "ema": st["ema"], "step": st["step"]}


def _plain_write(st, case):
    n, c, block = case["n"], case["channels"], case["block"]
    cells, blocks = _cells(case), _blocks(case)
    x = st["states"].reshape(n, cells, c).float()
    if blocks * block != cells:
        x = torch.cat([x, x.new_zeros(n, blocks * block - cells, c)], 1)
    x = x.reshape(n, blocks, block, c)
    top = x.abs().amax(2).clamp_min(TINY)
    if case["code"] == "i8":
        limit = torch.full_like(top, 127.0)
        scale, inverse = top / limit, limit / top
        codes = (x * inverse[:, :, None]).round_().to(torch.int8)
    else:
        frac, exp = torch.frexp(top)
        exp = torch.where(frac > 0.875, exp - 8, exp - 9)
        scale, inverse = torch.exp2(exp.float()), torch.exp2(-exp.float())
        codes = (x * inverse[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    st["codes"][st["slots"]] = codes.reshape(n, blocks * block, c)[:, :cells]
    st["scales"][st["slots"]] = scale


def _plain_read(st, case):
    n, c, block = case["n"], case["channels"], case["block"]
    cells, blocks = _cells(case), _blocks(case)
    there = (st["slots"] >= 0) & (st["slots"] < case["slots"])
    at = st["slots"].clamp(0, case["slots"] - 1)
    codes = st["codes"][at]
    x = codes.float() if case["code"] == "i8" else codes.view(torch.float8_e4m3fn).float()
    if blocks * block != cells:
        x = torch.cat([x, x.new_zeros(n, blocks * block - cells, c)], 1)
    x = x.reshape(n, blocks, block, c) * st["scales"][at][:, :, None]
    x = x.reshape(n, blocks * block, c)[:, :cells]
    st["out"].copy_(torch.where(there[:, None, None], x, 0.0).reshape(st["out"].shape))
    return st["out"]


def run(state):
    case = state["case"]
    if case["call"] == "keep":
        if own:
            state["cache"].write(state["states"], state["slots"])
            state["cache"].read(state["out"], state["slots"])
        else:
            _plain_write(state, case)
            _plain_read(state, case)
        return {"states": state["out"]}
    if case["call"] == "gather":
        if own:
            state["cache"].read(state["out"], state["slots"])
        else:
            _plain_read(state, case)
        return {"states": state["out"]}
    scale = SCALES.get(case["grad"], 1.0)
    if case["call"] == "clip":
        if own:
            return {"norm": state["list"].clip(1.0, scale), "clipped": state["out"]}
        return _plain_clip(state, scale)
    if own:
        norm = state["list"].adamw(LR, (BETA1, BETA2), EPS, case["decay"], max_norm=1.0,
                                   scale=scale, ema_decay=EMA)
        return {"norm": norm, "param": state["param"], "m": state["m"], "v": state["v"],
                "ema": state["ema"], "step": state["step"]}
    return _plain_adamw(state, scale, case["decay"])


# ---------------------------------------------------------------------------
# work, and the definition in 64 bits
# ---------------------------------------------------------------------------

_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def work(case):
    if case["call"] in ("clip", "adamw"):
        n = sum(_counts(case))
        if case["call"] == "clip":
            return {"bytes": n * (_SIZE[case["grad"]] + _SIZE[case["out"]]), "flops": 3 * n}
        return {"bytes": n * (_SIZE[case["grad"]] + 24 + (8 if case["ema"] else 0)),
                "flops": n * (17 + (3 if case["ema"] else 0))}
    values = case["n"] * _cells(case) * case["channels"]
    held = values + 4 * case["n"] * _blocks(case) * case["channels"]
    one = values * _SIZE[case["dtype"]] + held
    return ({"bytes": 2 * one, "flops": 4 * values} if case["call"] == "keep"
            else {"bytes": one, "flops": values})


def _exact_tensors(case, seed):
    st = _tensor_inputs(case, seed)
    g = st["grad"].double()
    scale = SCALES.get(case["grad"], 1.0)
    norm = float(torch.dot(g, g)) ** 0.5 * scale
    g *= scale * min(1.0, 1.0 / norm)
    if case["call"] == "clip":
        return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "clipped": g}
    t = int(st["step"]) + 1
    m = BETA1 * st["m"].double() + (1 - BETA1) * g
    v = BETA2 * st["v"].double() + (1 - BETA2) * g ** 2
    root = torch.sqrt(v / (1 - BETA2 ** t)) + EPS
    p = st["param"].double()
    p = p - LR * case["decay"] * p - LR / (1 - BETA1 ** t) * m / root
    ema = EMA * st["ema"].double() + (1 - EMA) * p if case["ema"] else None
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "param": p, "m": m,
            "v": v, "ema": ema, "step": None}


def _e4m3(x):
    """Nearest value of 1 sign, 4 exponent and 3 mantissa bits (bias 7)."""
    mag = x.abs()
    e = torch.floor(torch.log2(mag.clamp_min(2.0 ** -6)))
    e = torch.where(torch.exp2(e) > mag.clamp_min(2.0 ** -6), e - 1, e)
    unit = torch.exp2(e - 3)
    return torch.round(x / unit) * unit


def _exact_state(case, st, k):
    """State k as the cache gives it back."""
    cells, c, block = _cells(case), case["channels"], case["block"]
    pad = _blocks(case) * block - cells

    def split(x):
        x = torch.nn.functional.pad(x.reshape(cells, c).double(), (0, 0, 0, pad))
        return x.reshape(-1, block, c)
    if case["call"] == "gather":
        slot = int(st["slots"][k])
        if not 0 <= slot < case["slots"]:
            return torch.zeros((cells, c), dtype=torch.float64, device="cuda")
        codes = st["codes"][slot].short()
        if case["code"] == "f8":
            mag, sign = codes & 127, 1.0 - 2.0 * (codes >> 7).double()
            e, frac = (mag >> 3).double(), (mag & 7).double()
            x = sign * torch.where(e > 0, (8 + frac) * torch.exp2(e - 10), frac * 2.0 ** -9)
        else:
            x = codes
        x = split(x) * st["scales"][slot].double()[:, None]
    else:
        x = split(st["states"][k])
        top = torch.clamp(x.abs().max(1, keepdim=True).values, min=TINY)
        if case["code"] == "i8":
            x = torch.round(x * 127 / top) * (top / 127)
        else:
            e = torch.ceil(torch.log2(top / 448))
            e = torch.where(448 * torch.exp2(e - 1) >= top, e - 1, e)
            e = torch.where(448 * torch.exp2(e) < top, e + 1, e)
            x = _e4m3(x / torch.exp2(e)) * torch.exp2(e)
    return x.reshape(-1, c)[:cells]


def exact(case, seed):
    if case["call"] in ("clip", "adamw"):
        return _exact_tensors(case, seed)
    if case["n"] * _cells(case) * case["channels"] > 1_200_000_000:
        return None
    st = _state_inputs(case, seed)
    out = torch.stack([_exact_state(case, st, k) for k in range(case["n"])])
    return {"states": out.reshape(st["out"].shape)}
