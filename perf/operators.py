"""The products around a layer's quantisation, measured: their plain forms and the library's kernels.

Rows (tokens) of all experts come together, sorted by expert; expert e has the rows
offsets[e] .. offsets[e + 1] - 1.  One expert is a plain linear layer.  The operators:

* ``forward``: y = x W_e^T, with the layer's 16-bit weights.
* ``backward``: dx = dy W_e and dW_e = dy^T x over the expert's rows.
* ``gram``: H_e = X_e^T X_e in fp32, what a layer's optimisation starts from.
* ``int8``: the rows of x in 8-bit integers with a scale each (absolute maximum / 127), times 8-bit
  weights with a scale per output channel.
* ``packed``: y = x W_e^T with the bytes that a hardened layer is packed into, each weight being
  scale * level in fp32, rounded to the type of x.

Sizes are those of the layers in ``paper_2604_18556_amd/inputs.py`` (linear layers of 8B and 70B
models, routed experts under a Zipf profile of tokens) and generic ones: small, odd, ragged.
"""
import math

import torch

own = False

LEVELS = {2: (-0.5, 0.5), 3: (-1.0, 0.0, 1.0), 4: (-1.5, -0.5, 0.5, 1.5),
          8: (-3.5, -2.5, -1.5, -0.5, 0.5, 1.5, 2.5, 3.5), 16: tuple(k - 7.5 for k in range(16))}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(kind, groups, rows, out_features, in_features, dtype="bf16", spread="zipf", levels=0,
          layout="", group=0):
    return {"kind": kind, "groups": groups, "rows": rows, "out": out_features, "in": in_features,
            "dtype": dtype, "spread": spread, "levels": levels, "layout": layout, "group": group}


def listed():
    out = []

    def add(name, *args, **kw):
        out.append(dict(_case(*args, **kw), name=name))

    # eight tokens of a generation step, each routed to eight of 64 experts: weights are read, little else
    add("forward-decode-64x2048x7168", "forward", 64, 64, 2048, 7168)
    # the same experts over a batch of 16384 routed rows, as a calibration pass sends them
    add("forward-batch-64x2048x7168", "forward", 64, 16384, 2048, 7168)
    # training smaller experts on a ragged batch
    add("backward-16x1408x2048", "backward", 16, 6011, 1408, 2048, dtype="fp16")
    # a toy layer of odd sizes: launches, latency, tails in every direction
    add("backward-5x77x203", "backward", 5, 131, 77, 203)
    # H of a block's experts, and of one attention projection, from calibration tokens
    add("gram-8x7168", "gram", 8, 4099, 0, 7168)
    add("gram-1x4096", "gram", 1, 8192, 0, 4096, dtype="fp16")
    # a projection kept at 8 bits: one token, a long prompt, and ragged rows of small experts
    add("int8-token-4096x4096", "int8", 1, 1, 4096, 4096)
    add("int8-prompt-14336x4096", "int8", 1, 4096, 14336, 4096)
    add("int8-ragged-8x1000x2056", "int8", 8, 777, 1000, 2056, dtype="fp16")
    # packed layers: one token through a 3-bit down projection, a generation step through the experts'
    # super-blocks, and a prompt through a ternary projection
    add("packed-token-4096x14336-k8", "packed", 1, 1, 4096, 14336, levels=8, layout="group", group=128)
    add("packed-decode-64x2048x7168-superblock", "packed", 64, 64, 2048, 7168, levels=8,
        layout="superblock", group=16)
    add("packed-prompt-4096x4096-base3", "packed", 1, 2001, 4096, 4096, dtype="fp16", levels=3,
        layout="base3", group=128)
    return out


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("forward", "backward", "gram", "int8", "packed"))
    dtype = rng.choice(("bf16", "bf16", "fp16"))
    levels, layout, group, unit = 0, "", 0, rng.choice((1, 8, 64, 128))
    if kind == "packed":
        layout = rng.choice(("group", "group", "base3", "superblock"))
        levels = {"base3": 3, "superblock": 8}.get(layout) or rng.choice((2, 3, 4, 8, 16))
        group = 16 if layout == "superblock" else rng.choice((16, 32, 64, 128, 128, 256))
        unit = 256 if layout == "superblock" else group
    while True:
        groups = rng.choice((1, 1, _log(rng, 2, 64)))
        rows = _log(rng, 1, 16384)
        o = _log(rng, 64, 16384)
        o = max(1, o // 16 * 16) if rng.random() < 0.7 else o
        i = max(unit, _log(rng, 64, 16384) // unit * unit)
        if kind == "gram":
            i, o = min(i, 8192), 0
        case = _case(kind, groups, rows, o, i, dtype, rng.choice(("zipf", "zipf", "even")), levels,
                     layout, group)
        w = work(case)
        # within the largest listed cases, in what is kept as well as in what a pass does
        if w["flops"] <= 4.5e11 and w["bytes"] <= 1.5e9 and groups * max(o, i) * i <= 9e8:
            return case


def _counts(case):
    """Rows of each expert, largest first: 1 / rank^1.2, or all alike."""
    n, rows = case["groups"], case["rows"]
    share = [(k + 1) ** -1.2 if case["spread"] == "zipf" else 1.0 for k in range(n)]
    total = sum(share)
    counts = [int(rows * s / total) for s in share]
    for k in range(rows - sum(counts)):
        counts[k % n] += 1
    return counts


def work(case):
    counts = _counts(case)
    used = sum(c > 0 for c in counts)
    n, r, o, i = case["groups"], case["rows"], case["out"], case["in"]
    kind = case["kind"]
    if kind == "gram":
        return {"bytes": 2.0 * r * i + 4.0 * n * i * i, "flops": 1.0 * r * i * (i + 1)}
    if kind == "backward":
        return {"bytes": 2.0 * (2 * r * i + r * o + used * o * i + n * o * i), "flops": 4.0 * r * o * i}
    if kind == "forward":
        weights = 2.0 * used * o * i
    elif kind == "int8":
        weights = used * o * (i + 4.0)
    else:
        bits = {"base3": 1.6, "superblock": 110 / 32}.get(case["layout"])
        if bits is None:
            bits = math.ceil(math.log2(case["levels"]))
        weights = used * o * i * (bits / 8 + (0 if case["layout"] == "superblock" else 2 / case["group"]))
    return {"bytes": weights + 2.0 * r * (i + o), "flops": 2.0 * r * o * i}


# ------------------------------------------------------------------ inputs
def _activations(rows, width, dtype, gen, device):
    """Heavy-tailed rows (Student-t, 4 degrees of freedom) with a scale per channel."""
    x = torch.randn(rows, width, generator=gen, device=device)
    chi = torch.zeros_like(x)
    for _ in range(4):
        chi.add_(torch.randn(rows, width, generator=gen, device=device).square_())
    x.div_(chi.mul_(0.25).sqrt_().clamp_min_(0.05))
    return x.mul_(torch.randn(width, generator=gen, device=device).mul_(0.5).exp_()).to(dtype)


def _weights(shape, gen, device):
    """N(0, 0.02^2) with a thousandth of outliers, ten times larger."""
    w = torch.randn(shape, generator=gen, device=device).mul_(0.02)
    w[torch.rand(shape, generator=gen, device=device) < 1e-3] *= 10.0
    return w


def _codes(case, gen, device):
    """A hardened layer: level indices, and the scales in the parts that the layout keeps."""
    n, o, i, group = case["groups"], case["out"], case["in"], case["group"]
    mids = torch.tensor(LEVELS[case["levels"]], device=device)
    top = float(mids.abs().max())
    mids = (mids[1:] + mids[:-1]) * 0.5
    codes = torch.empty(n, o, i, dtype=torch.uint8, device=device)
    parts = []
    for e in range(n):
        w = _weights((o, i // group, group), gen, device)
        s = w.abs().amax(-1) / top
        if case["layout"] == "superblock":
            s = s.reshape(o, i // 256, 16)
            d = (s.amax(-1, keepdim=True) / 63.0).half()
            sc = (s / d.float()).round_().clamp_(1, 63).to(torch.uint8)
            parts.append((d, sc))
            s = (d.float() * sc).reshape(o, i // group)
        else:
            s = s.half()
            parts.append((s,))
            s = s.float()
        codes[e] = torch.bucketize(w / s[..., None], mids, out_int32=True).reshape(o, i)
    return codes, tuple(torch.stack(p) for p in zip(*parts))


def _pack(case, codes, parts):
    """The bytes of the layer: little-endian code bits then fp16 scales, five base-3 digits a byte then
    fp16 scales, or records of 110 bytes (fp16 d, 16 6-bit scales, 256 3-bit codes)."""

    def bits(values, width):           # a last dimension of 8 values becomes `width` bytes
        word = torch.zeros(values.shape[:-1], dtype=torch.int64, device=values.device)
        for k in range(8):
            word |= values[..., k].long() << (width * k)
        return torch.stack([(word >> (8 * k)) & 255 for k in range(width)], -1).to(torch.uint8)

    n, o, i = codes.shape
    if case["layout"] == "superblock":
        d, sc = parts
        out = torch.empty(n, o * i // 256, 110, dtype=torch.uint8, device=codes.device)
        for e in range(n):
            out[e, :, 0:2] = d[e].reshape(-1, 1).view(torch.uint8)
            out[e, :, 2:14] = bits(sc[e].reshape(-1, 2, 8), 6).reshape(-1, 12)
            out[e, :, 14:110] = bits(codes[e].reshape(-1, 32, 8), 3).reshape(-1, 96)
        return out.reshape(-1)
    scales = parts[0].reshape(-1).view(torch.uint8)
    if case["layout"] == "base3":
        flat = torch.nn.functional.pad(codes.reshape(-1), (0, -codes.numel() % 5)).reshape(-1, 5)
        byte = flat[:, 0].clone()
        for k in range(1, 5):
            byte += flat[:, k] * 3 ** k
        return torch.cat((byte, scales))
    width = math.ceil(math.log2(case["levels"]))
    return torch.cat([bits(c.reshape(-1, 8), width).reshape(-1) for c in codes] + [scales])


def _inputs(case, seed):
    device = torch.device("cuda:0")
    gen = torch.Generator(device=device).manual_seed(int(seed))
    n, r, o, i = case["groups"], case["rows"], case["out"], case["in"]
    dtype, kind = DTYPES[case["dtype"]], case["kind"]
    order = torch.randperm(n, generator=torch.Generator().manual_seed(int(seed))).tolist()
    counts = _counts(case)
    counts = [counts[k] for k in order]
    data = {"counts": counts, "x": _activations(r, i, dtype, gen, device)}
    if kind in ("forward", "backward", "int8"):
        w = torch.empty(n, o, i, dtype=torch.int8 if kind == "int8" else dtype, device=device)
        if kind == "int8":
            data["w_scales"] = torch.empty(n, o, device=device)
        for e in range(n):
            we = _weights((o, i), gen, device)
            if kind == "int8":
                s = we.abs().amax(-1) / 127.0
                data["w_scales"][e] = s
                we = (we / s[:, None]).round_().clamp_(-127, 127)
            w[e] = we
        data["w"] = w
    if kind == "backward":
        data["dy"] = torch.randn(r, o, generator=gen, device=device).mul_(0.1).to(dtype)
    if kind == "packed":
        data["codes"], data["parts"] = _codes(case, gen, device)
    return data


def prepare(case, seed):
    state = _inputs(case, seed)
    device = state["x"].device
    n, r, o, i = case["groups"], case["rows"], case["out"], case["in"]
    dtype, kind = DTYPES[case["dtype"]], case["kind"]
    ends = torch.tensor([0] + state["counts"]).cumsum(0)
    state["offsets"] = ends.to(device)
    state["bounds"] = ends.tolist()
    if kind == "backward":
        state["dx"] = torch.empty(r, i, dtype=dtype, device=device)
        state["dw"] = torch.empty(n, o, i, dtype=dtype, device=device)
    elif kind == "gram":
        state["h"] = torch.empty(n, i, i, device=device)
    else:
        state["y"] = torch.empty(r, o, dtype=dtype, device=device)
    if kind == "int8":
        state["q"] = torch.empty(r, i, dtype=torch.int8, device=device)
        state["q_scales"] = torch.empty(r, device=device)
    if kind == "packed":
        state["packed"] = _pack(case, state.pop("codes"), state.pop("parts"))
        state["levels"] = torch.tensor(LEVELS[case["levels"]], device=device)
    if own:
        from paper_2604_18556_amd import binding as B
        state["B"] = B
        if kind == "packed":
            layout = {"group": B.LAYOUT_GROUP, "base3": B.LAYOUT_BASE3,
                      "superblock": B.LAYOUT_SUPERBLOCK}[case["layout"]]
            cfg = B.LayerConfig(o, i, LEVELS[case["levels"]], case["group"], n, layout,
                                relaxation=B.RELAX_SHIFT if case["levels"] > 8 else B.RELAX_GRID)
            state["linear"] = B.Linear(cfg, state["packed"])
    state["case"] = case
    torch.cuda.synchronize()
    return state


# ------------------------------------------------------------------ one pass
def _run_own(state):
    B, kind, off = state["B"], state["case"]["kind"], state["offsets"]
    if kind == "forward":
        B.grouped_forward(state["x"], state["w"], state["y"], offsets=off)
        return state["y"]
    if kind == "backward":
        B.grouped_input_grad(state["dy"], state["w"], state["dx"], offsets=off)
        B.grouped_weight_grad(state["dy"], state["x"], state["dw"], offsets=off)
        return {"dx": state["dx"], "dw": state["dw"]}
    if kind == "gram":
        B.gram(state["x"], state["h"], offsets=off)
        return state["h"]
    if kind == "int8":
        B.quantize_rows(state["x"], state["q"], state["q_scales"])
        B.grouped_forward_i8(state["q"], state["q_scales"], state["w"], state["w_scales"], state["y"],
                             offsets=off)
        return state["y"]
    state["linear"].forward(state["x"], state["y"], offsets=off)
    return state["y"]


def _unpack(case, packed, levels, e, dtype):
    """Expert e's weights from the packed bytes, as fp32 values of the type `dtype`."""
    n, o, i, group = case["groups"], case["out"], case["in"], case["group"]
    total, size = n * o * i, o * i

    def fields(data, width, count):    # `count` fields of `width` bits in the last dimension's bytes
        word = torch.zeros(data.shape[:-1], dtype=torch.int64, device=data.device)
        for k in range(data.shape[-1]):
            word |= data[..., k].long() << (8 * k)
        shifts = torch.arange(count, device=data.device) * width
        return (word[..., None] >> shifts) & ((1 << width) - 1)

    if case["layout"] == "superblock":
        rec = packed[e * size // 256 * 110:(e + 1) * size // 256 * 110].reshape(-1, 110)
        d = rec[:, 0:2].contiguous().view(torch.float16).float()
        sc = fields(rec[:, 2:14].reshape(-1, 2, 6), 6, 8).reshape(-1, 16)
        codes = fields(rec[:, 14:110].reshape(-1, 32, 3), 3, 8)
        scales = d * sc.float()
    else:
        if case["layout"] == "base3":
            nbytes = (total + 4) // 5
            first, last = e * size // 5, ((e + 1) * size + 4) // 5
            digits = packed[first:last].to(torch.int32)[:, None]
            power = torch.tensor([1, 3, 9, 27, 81], dtype=torch.int32, device=packed.device)
            codes = (torch.div(digits, power, rounding_mode="floor") % 3).reshape(-1)
            codes = codes[e * size - first * 5:][:size]
        else:
            width = math.ceil(math.log2(case["levels"]))
            nbytes = total * width // 8
            data = packed[e * size * width // 8:(e + 1) * size * width // 8]
            codes = fields(data.reshape(-1, width), width, 8)
        scales = packed[nbytes:].clone().view(torch.float16)
        scales = scales[e * size // group:(e + 1) * size // group].float()
    values = levels[codes.reshape(-1, group).long()] * scales.reshape(-1, 1)
    return values.to(dtype).float().reshape(o, i)


def run(state):
    if own:
        return _run_own(state)
    case, bounds = state["case"], state["bounds"]
    kind, x = case["kind"], state["x"]
    dtype = x.dtype
    if kind == "int8":
        xf = x.float()
        s = xf.abs().amax(-1, keepdim=True) / torch.full((1, 1), 127.0, device=x.device)
        # the quotient in 64 bits: whole numbers may not turn over at a half
        q = torch.where(s > 0, xf.double() / s.double(), 0.0).round().clamp(-127, 127)
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        if kind == "forward" and b > a:
            state["y"][a:b] = (x[a:b].float() @ state["w"][e].float().t()).to(dtype)
        elif kind == "backward":
            dy = state["dy"][a:b].float()
            if b > a:
                state["dx"][a:b] = (dy @ state["w"][e].float()).to(dtype)
            state["dw"][e] = (dy.t() @ x[a:b].float()).to(dtype)
        elif kind == "gram":
            xf = x[a:b].float()
            state["h"][e] = xf.t() @ xf
        elif kind == "int8" and b > a:
            # 32 bits hold no sum beyond 2^24
            dot = q[a:b] @ state["w"][e].double().t()
            state["y"][a:b] = (dot.float() * s[a:b] * state["w_scales"][e]).to(dtype)
        elif kind == "packed" and b > a:
            w = _unpack(case, state["packed"], state["levels"], e, dtype)
            state["y"][a:b] = (x[a:b].float() @ w.t()).to(dtype)
    if kind == "backward":
        return {"dx": state["dx"], "dw": state["dw"]}
    return state["h"] if kind == "gram" else state["y"]


# ------------------------------------------------------------------ the same in 64 bits
def _value(x):
    return x.to(torch.float64)


def exact(case, seed):
    data = _inputs(case, seed)
    x, kind = _value(data["x"]), case["kind"]
    ends = [sum(data["counts"][:k]) for k in range(case["groups"] + 1)]
    rows = [slice(ends[k], ends[k + 1]) for k in range(case["groups"])]
    if kind == "gram":
        return torch.stack([torch.matmul(x[k].mT, x[k]) for k in rows])
    if kind == "backward":
        dy = _value(data["dy"])
        return {"dx": torch.cat([torch.matmul(dy[k], _value(w)) for k, w in zip(rows, data["w"])]),
                "dw": torch.stack([torch.matmul(dy[k].mT, x[k]) for k in rows])}
    if kind == "int8":
        # the scale is kept in 32 bits; everything after it is exact
        scale = (x.abs().max(dim=1).values / 127.0).float().double()
        q = torch.round(x / torch.where(scale == 0, 1.0, scale)[:, None])
        x = torch.clamp(q, -127.0, 127.0)
    parts = []
    for e, k in enumerate(rows):
        if kind == "packed":
            # the weight's own definition rounds: scale * level in 32 bits, then to the type of x
            s = data["parts"][0][e].float()
            if case["layout"] == "superblock":
                s = s * data["parts"][1][e].float()
            level = torch.tensor(LEVELS[case["levels"]], device=x.device)[data["codes"][e].int()]
            w = s.reshape(case["out"], -1).repeat_interleave(case["group"], dim=1) * level
            w = _value(w.to(data["x"].dtype))
        else:
            w = _value(data["w"][e])
        y = torch.matmul(x[k], w.mT)
        if kind == "int8":
            y = y * scale[k, None] * _value(data["w_scales"][e])
        parts.append(y)
    return torch.cat(parts)
