"""Routing to experts and low-rank adapters, measured: their plain forms and the library's kernels.

What stands beside the products of grouped rows.  The operators:

* ``route``: the experts and weights of each token from its logits, and the order in which the rows of
  all experts come together (offsets, where each row goes, and where it comes from).
* ``route-grad``: the gradient of the logits from that of the weights.
* ``exchange``: tokens copied into the experts' order, and the experts' rows summed back with weights.
* ``exchange-grad``: the gradients of both.
* ``adapter``: y = base + s B (A x), the adapter being that of the row's request, beside a shared
  projection's output.
* ``adapter-grad``: the gradients of x, A and B, beside the shared projection's gradient of x.

Sizes are those of the layers in ``paper_2604_18556_amd/inputs.py`` (linear layers, 64 routed experts of
2048 x 7168) and generic ones: small, odd, ragged.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _routing(kind, tokens, experts, top_k, score="softmax", bias=False, groups=1, top_groups=1,
             group_score="top2", renormalise=True, scale=1.0, dtype="bf16", padded=0):
    return {"kind": kind, "tokens": tokens, "experts": experts, "top_k": top_k, "score": score, "bias": bias,
            "groups": groups, "top_groups": top_groups, "group_score": group_score, "renormalise": renormalise,
            "scale": scale, "dtype": dtype, "padded": padded}


def _exchange(kind, tokens, experts, top_k, width, dtype="bf16", padded=0):
    return {"kind": kind, "tokens": tokens, "experts": experts, "top_k": top_k, "width": width, "dtype": dtype,
            "padded": padded}


def _adapter(kind, rows, segments, adapters, out_features, in_features, rank, dtype="bf16", spread="zipf",
             indexed=True):
    return {"kind": kind, "rows": rows, "segments": segments, "adapters": adapters, "out": out_features,
            "in": in_features, "rank": rank, "dtype": dtype, "spread": spread, "indexed": indexed}


def listed():
    out = []

    def add(name, case):
        out.append(dict(case, name=name))

    # a generation step of 64 requests: sigmoid scores with a bias for balance, four of eight groups
    add("route-decode-64x256", _routing("route", 64, 256, 8, score="sigmoid", bias=True, groups=8, top_groups=4,
                                        scale=2.5, dtype="fp32"))
    # a prompt of 16384 tokens over 64 experts, its last tokens padding
    add("route-prompt-16384x64", _routing("route", 16384, 64, 8, renormalise=False, padded=133))
    # the same sizes in training, and an odd batch of grouped experts
    add("route-grad-16384x64", _routing("route-grad", 16384, 64, 8, renormalise=False))
    add("route-grad-1001x162", _routing("route-grad", 1001, 162, 6, score="sigmoid", bias=True, groups=9,
                                        top_groups=4, dtype="fp32"))
    # eight tokens of a generation step through eight of 64 experts, and a batch of 16384 routed rows
    add("exchange-decode-8x7168", _exchange("exchange", 8, 64, 8, 7168))
    add("exchange-batch-2048x7168", _exchange("exchange", 2048, 64, 8, 7168))
    # the batch in training; smaller experts on a ragged batch with padding
    add("exchange-grad-2048x7168", _exchange("exchange-grad", 2048, 64, 8, 7168))
    add("exchange-grad-1003x2048", _exchange("exchange-grad", 1003, 16, 6, 2048, dtype="fp16", padded=40))
    # a generation step of 64 requests, most with an adapter of their own, beside an attention projection
    add("adapter-decode-64x4096x4096-r16", _adapter("adapter", 64, 64, 48, 4096, 4096, 16))
    # the prompts of eight requests beside an up projection
    add("adapter-prompt-4096x14336x4096-r64", _adapter("adapter", 4096, 8, 6, 14336, 4096, 64))
    # one batch that trains four adapters beside a down projection, and a toy layer of odd sizes
    add("adapter-grad-4096x4096x14336-r32", _adapter("adapter-grad", 4096, 4, 4, 4096, 14336, 32, indexed=False))
    add("adapter-grad-131x77x203-r5", _adapter("adapter-grad", 131, 7, 5, 77, 203, 5, dtype="fp16"))
    return out


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("route", "route-grad", "exchange", "exchange-grad", "adapter", "adapter-grad"))
    dtype = rng.choice(("bf16", "bf16", "fp16"))
    while True:
        if kind.startswith("route"):
            groups = rng.choice((1, 1, 4, 8, rng.randint(2, 12)))
            experts = max(1, _log(rng, 8, 384) // groups) * groups
            top_groups = rng.randint((groups + 1) // 2, groups)
            top_k = rng.randint(1, min(10, top_groups * (experts // groups)))
            tokens = _log(rng, 1, 16384)
            case = _routing(kind, tokens, experts, top_k, rng.choice(("softmax", "sigmoid")), rng.random() < 0.5,
                            groups, top_groups, rng.choice(("top2", "max")), rng.random() < 0.5,
                            rng.choice((1.0, 2.5)), rng.choice((dtype, "fp32")), tokens // 50 * rng.randint(0, 1))
        elif kind.startswith("exchange"):
            tokens, experts = _log(rng, 1, 8192), _log(rng, 4, 256)
            width = _log(rng, 64, 8192)
            width = width // 8 * 8 if rng.random() < 0.7 else width
            case = _exchange(kind, tokens, experts, rng.randint(1, min(8, experts)), width,
                             rng.choice((dtype, dtype, "fp32")), tokens // 50 * rng.randint(0, 1))
        else:
            rows = _log(rng, 1, 8192)
            segments = min(rows, _log(rng, 1, 64)) if rng.random() < 0.7 else min(rows, 256)
            indexed = rng.random() < 0.7
            o, i = _log(rng, 64, 16384), _log(rng, 64, 16384)
            if rng.random() < 0.7:
                o, i = max(64, o // 16 * 16), max(64, i // 16 * 16)
            case = _adapter(kind, rows, segments, rng.randint(1, segments) if indexed else segments, o, i,
                            rng.choice((8, 16, 16, 32, 64, _log(rng, 1, 128))), dtype,
                            rng.choice(("zipf", "even")), indexed)
        w = work(case)
        # no more than the largest listed cases of the operator do
        if w["bytes"] <= (6e8 if kind == "exchange-grad" else 3.3e8) and w["flops"] <= 9.6e9:
            return case


def _rows(case):
    """Rows that experts get: those of tokens that are not padding."""
    return (case["tokens"] - case["padded"]) * case["top_k"]


def _counts(case):
    """Rows of each request, largest first: 1 / rank^1.2, or all alike; one at least."""
    n, rows = case["segments"], case["rows"]
    share = [(k + 1) ** -1.2 if case["spread"] == "zipf" else 1.0 for k in range(n)]
    total = sum(share)
    counts = [1 + int((rows - n) * s / total) for s in share]
    for k in range(rows - sum(counts)):
        counts[k % n] += 1
    return counts


def _adapter_of(case, seed):
    """The adapter of each request: mostly drawn, -1 (none) for some of many requests."""
    n = case["segments"]
    if not case["indexed"]:
        return list(range(n))
    gen = torch.Generator().manual_seed(int(seed) + 1)
    index = torch.randint(0, case["adapters"], (n,), generator=gen)
    if n > 8:
        index[torch.rand(n, generator=gen) < 0.1] = -1
    return index.tolist()


def work(case):
    kind, size = case["kind"], {"fp32": 4.0}.get(case["dtype"], 2.0)
    if kind.startswith("route"):
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        if kind == "route":
            return {"bytes": size * t * e + 4.0 * e * case["bias"] + 16.0 * t * k + 8.0 * (e + 1),
                    "flops": 5.0 * t * e}
        return {"bytes": 2 * size * t * e + 8.0 * t * k, "flops": 5.0 * t * e}
    if kind.startswith("exchange"):
        t, r, c = case["tokens"], _rows(case), case["width"]
        slots = 4.0 * t * case["top_k"]
        if kind == "exchange":
            return {"bytes": size * c * (2.0 * t + 2.0 * r) + 2 * slots + 4.0 * t * case["top_k"], "flops": 2.0 * r * c}
        return {"bytes": size * c * (2.0 * t + 3.0 * r) + 3 * slots, "flops": 4.0 * r * c}
    r, o, i, q = case["rows"], case["out"], case["in"], case["rank"]
    used = min(case["adapters"], case["segments"])
    if kind == "adapter":
        return {"bytes": 2.0 * (r * i + 2 * r * o + used * q * (i + o)), "flops": 2.0 * r * q * (i + o)}
    return {"bytes": 2.0 * (3 * r * i + r * o + used * q * (i + o)) + 4.0 * (r * q + case["adapters"] * q * (i + o)),
            "flops": 4.0 * r * q * (i + o)}


# ------------------------------------------------------------------ inputs
def _activations(rows, width, dtype, gen, device):
    """Heavy-tailed rows (Student-t, 4 degrees of freedom) with a scale per channel."""
    x = torch.randn(rows, width, generator=gen, device=device)
    chi = torch.zeros_like(x)
    for _ in range(4):
        chi.add_(torch.randn(rows, width, generator=gen, device=device).square_())
    x.div_(chi.mul_(0.25).sqrt_().clamp_min_(0.05))
    return x.mul_(torch.randn(width, generator=gen, device=device).mul_(0.5).exp_()).to(dtype)


def _chosen(case, gen, device):
    """Distinct experts of each token, popular ones more often; -1 for padding."""
    t, e = case["tokens"], case["experts"]
    popular = torch.randn(e, generator=gen, device=device)
    noise = -torch.log(-torch.log(torch.rand(t, e, generator=gen, device=device).clamp(1e-7, 1 - 1e-7)))
    ids = torch.argsort(popular + noise, dim=1, descending=True, stable=True)[:, :case["top_k"]]
    ids = ids.to(torch.int32).contiguous()
    if case["padded"]:
        ids[t - case["padded"]:] = -1
    return ids


def _order(ids):
    """Where each (token, choice) goes when all are sorted by expert, and what stands there."""
    flat = ids.reshape(-1).long()
    n, some = flat.numel(), int((flat >= 0).sum())
    order = torch.argsort(torch.where(flat < 0, 1 << 30, flat), stable=True)
    slots = torch.full((n,), -1, dtype=torch.int32, device=ids.device)
    slots[order[:some]] = torch.arange(some, dtype=torch.int32, device=ids.device)
    sources = order.to(torch.int32)
    sources[some:] = -1
    return slots.reshape(ids.shape), sources


def _inputs(case, seed):
    device = torch.device("cuda:0")
    gen = torch.Generator(device=device).manual_seed(int(seed))
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind.startswith("route"):
        t, e = case["tokens"], case["experts"]
        logits = torch.randn(t, e, generator=gen, device=device).mul_(1.5)
        logits.add_(torch.randn(e, generator=gen, device=device))
        data = {"logits": logits.to(dtype), "bias": None}
        if case["padded"]:
            data["logits"][t - case["padded"]:] = float("-inf")
        if case["bias"]:
            data["bias"] = torch.randn(e, generator=gen, device=device).mul_(0.1)
        if kind == "route-grad":
            data["ids"] = _choice(case, data["logits"], data["bias"])[0]
            data["dw"] = torch.randn(t, case["top_k"], generator=gen, device=device)
        return data
    if kind.startswith("exchange"):
        t, k, c = case["tokens"], case["top_k"], case["width"]
        ids = _chosen(case, gen, device)
        slots, sources = _order(ids)
        data = {"slots": slots, "sources": sources,
                "weights": torch.rand(t, k, generator=gen, device=device).add_(0.05)}
        data["weights"].div_(data["weights"].sum(-1, keepdim=True))
        data["ys"] = torch.randn(t * k, c, generator=gen, device=device).to(dtype)
        if kind == "exchange":
            data["x"] = _activations(t, c, dtype, gen, device)
        else:
            data["dy"] = torch.randn(t, c, generator=gen, device=device).mul_(0.1).to(dtype)
            data["dxs"] = torch.randn(t * k, c, generator=gen, device=device).mul_(0.1).to(dtype)
        return data
    r, o, i, q, n = case["rows"], case["out"], case["in"], case["rank"], case["adapters"]
    order = torch.randperm(case["segments"], generator=torch.Generator().manual_seed(int(seed))).tolist()
    counts = _counts(case)
    data = {"counts": [counts[k] for k in order], "index": _adapter_of(case, seed),
            "x": _activations(r, i, dtype, gen, device),
            "a": torch.randn(n, q, i, generator=gen, device=device).mul_(i ** -0.5).to(dtype),
            "b": torch.randn(n, o, q, generator=gen, device=device).mul_(0.05).to(dtype),
            "scales": torch.rand(n, generator=gen, device=device).mul_(1.5).add_(0.5)}
    if kind == "adapter":
        data["base"] = torch.randn(r, o, generator=gen, device=device).to(dtype)
    else:
        data["dy"] = torch.randn(r, o, generator=gen, device=device).mul_(0.1).to(dtype)
        data["base"] = torch.randn(r, i, generator=gen, device=device).mul_(0.1).to(dtype)
    return data


def prepare(case, seed):
    state = _inputs(case, seed)
    kind, dtype, device = case["kind"], DTYPES[case["dtype"]], torch.device("cuda:0")

    def empty(*shape, of=dtype):
        return torch.zeros(*shape, dtype=of, device=device)

    if kind.startswith("route"):
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        if kind == "route":
            state["ids"], state["weights"] = empty(t, k, of=torch.int32), empty(t, k, of=torch.float32)
            state["offsets"] = empty(e + 1, of=torch.int64)
            state["slots"], state["sources"] = empty(t, k, of=torch.int32), empty(t * k, of=torch.int32)
        else:
            state["dlogits"] = empty(t, e)
    elif kind.startswith("exchange"):
        t, k, c = case["tokens"], case["top_k"], case["width"]
        if kind == "exchange":
            state["xs"], state["y"] = empty(t * k, c), empty(t, c)
        else:
            state["dys"], state["dw"], state["dx"] = empty(t * k, c), empty(t, k, of=torch.float32), empty(t, c)
    else:
        r, o, i, q, n = case["rows"], case["out"], case["in"], case["rank"], case["adapters"]
        ends = torch.tensor([0] + state["counts"]).cumsum(0)
        state["offsets"], state["bounds"] = ends.to(device), ends.tolist()
        state["which"] = state["index"]
        state["index"] = torch.tensor(state["which"], dtype=torch.int32, device=device) if case["indexed"] else None
        state["h"] = empty(r, q, of=torch.float32)
        if kind == "adapter":
            state["y"] = empty(r, o)
        else:
            # what the forward pass has kept
            for e, a, b in zip(state["which"], state["bounds"], state["bounds"][1:]):
                if e >= 0:
                    state["h"][a:b] = state["x"][a:b].float() @ state["a"][e].float().t()
            state["dh"], state["dx"] = empty(r, q, of=torch.float32), empty(r, i)
            state["da"], state["db"] = empty(n, q, i, of=torch.float32), empty(n, o, q, of=torch.float32)
    if own:
        from paper_2604_18556_amd import binding as B
        state["B"] = B
        if kind.startswith("route"):
            state["routing"] = B.Routing(
                case["experts"], case["top_k"], case["groups"], case["top_groups"],
                {"softmax": B.SCORE_SOFTMAX, "sigmoid": B.SCORE_SIGMOID}[case["score"]],
                {"top2": B.GROUP_TOP2, "max": B.GROUP_MAX}[case["group_score"]], case["renormalise"], case["scale"])
    state["case"] = case
    torch.cuda.synchronize()
    return state


# ------------------------------------------------------------------ one pass
def _run_own(state):
    B, case = state["B"], state["case"]
    kind = case["kind"]
    if kind == "route":
        B.route(state["routing"], state["logits"], state["ids"], state["weights"], bias=state["bias"])
        B.group_rows(state["ids"], state["offsets"], state["slots"], state["sources"])
        return {k: state[k] for k in ("ids", "weights", "offsets", "slots", "sources")}
    if kind == "route-grad":
        B.route_grad(state["routing"], state["logits"], state["ids"], state["dw"], state["dlogits"])
        return state["dlogits"]
    if kind == "exchange":
        B.dispatch_rows(state["x"], state["slots"], state["xs"])
        B.combine_rows(state["ys"], state["slots"], state["y"], weights=state["weights"])
        return {"xs": state["xs"], "y": state["y"]}
    if kind == "exchange-grad":
        B.combine_rows_grad(state["dy"], state["ys"], state["slots"], state["weights"], state["dys"], state["dw"])
        B.combine_rows(state["dxs"], state["slots"], state["dx"])
        return {"dys": state["dys"], "dw": state["dw"], "dx": state["dx"]}
    where = {"offsets": state["offsets"], "index": state["index"], "scales": state["scales"]}
    if kind == "adapter":
        B.adapter_forward(state["x"], state["a"], state["b"], state["h"], state["y"], base=state["base"], **where)
        return state["y"]
    B.adapter_input_grad(state["dy"], state["a"], state["b"], state["dh"], state["dx"], base=state["base"], **where)
    B.adapter_weight_grad(state["dy"], state["x"], state["h"], state["dh"], state["da"], state["db"], **where)
    return {"dx": state["dx"], "da": state["da"], "db": state["db"]}


def _scores(case, logits):
    """In 64 bits: what chooses stands next to borders."""
    l = logits.double()
    if case["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    top = l.amax(-1, keepdim=True)
    e = torch.exp(l - torch.where(torch.isinf(top), 0.0, top))
    return e / e.sum(-1, keepdim=True).clamp_min(1e-300)


def _first_best(key):
    """The best of the last dimension and the lowest place that has it."""
    best = key.amax(-1, keepdim=True)
    place = torch.arange(key.shape[-1], device=key.device)
    return best, torch.where(key == best, place, key.shape[-1]).amin(-1, keepdim=True)


def _choice(case, logits, bias):
    """The experts of each token and the scores of all: iterated maxima."""
    t, e, g = case["tokens"], case["experts"], case["groups"]
    low = float("-inf")
    scores = _scores(case, logits)
    value = scores if bias is None else scores + bias.double()
    key = logits.double() if bias is None else value
    key = torch.where(logits == low, low, key)
    if g > 1:
        value = torch.where(logits == low, low, value).reshape(t, g, e // g)
        best, at = _first_best(value)
        group = best[..., 0]
        if case["group_score"] == "top2" and e > g:
            second, _ = _first_best(value.scatter(-1, at, low))
            group = group + torch.where(second == low, 0.0, second)[..., 0]
        keep = torch.zeros(t, g, dtype=torch.bool, device=key.device)
        for _ in range(case["top_groups"]):
            _, at = _first_best(group)
            keep.scatter_(-1, at, True)
            group = torch.where(keep, low, group)
        key = torch.where(keep.repeat_interleave(e // g, dim=1), key, low)
    ids = torch.empty(t, case["top_k"], dtype=torch.int32, device=key.device)
    for j in range(case["top_k"]):
        best, at = _first_best(key)
        ids[:, j:j + 1] = torch.where(best == low, -1, at).to(torch.int32)
        key = key.scatter(-1, at, low)
    return ids, scores


def _weights(case, ids, scores):
    w = scores.gather(-1, ids.long().clamp_min(0)) * (ids >= 0)
    if case["renormalise"]:
        w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
    return w * case["scale"]


def _run_route(state):
    case = state["case"]
    ids, scores = _choice(case, state["logits"], state["bias"])
    state["ids"].copy_(ids)
    state["weights"].copy_(_weights(case, ids, scores))
    slots, sources = _order(ids)
    state["slots"].copy_(slots)
    state["sources"].copy_(sources)
    experts = torch.arange(case["experts"], device=ids.device)
    counts = (ids.reshape(-1, 1) == experts).sum(0)
    state["offsets"][0] = 0
    state["offsets"][1:] = counts.cumsum(0)
    return {k: state[k] for k in ("ids", "weights", "offsets", "slots", "sources")}


def _run_route_grad(state):
    case, ids = state["case"], state["ids"]
    s = _scores(case, state["logits"]).float()
    at, some = ids.long().clamp_min(0), ids >= 0
    chosen = s.gather(-1, at) * some
    g = state["dw"] * some * case["scale"]
    if case["renormalise"]:
        total = chosen.sum(-1, keepdim=True).clamp_min(1e-30)
        g = (g - (g * chosen).sum(-1, keepdim=True) / total) / total
    ds = torch.zeros_like(s).scatter_add(-1, at, g)
    if case["score"] == "sigmoid":
        dl = ds * s * (1.0 - s)
    else:
        dl = s * (ds - (ds * s).sum(-1, keepdim=True))
    state["dlogits"].copy_(dl)
    return state["dlogits"]


def _run_exchange(state):
    case, slots, dtype = state["case"], state["slots"], state["ys"].dtype
    k, some = case["top_k"], slots >= 0

    def combined(rows, weights):
        total = torch.zeros(case["tokens"], case["width"], device=rows.device)
        for j in range(k):
            part = rows[slots[:, j].long().clamp_min(0)].float() * some[:, j:j + 1]
            total += part if weights is None else part * weights[:, j:j + 1]
        return total.to(dtype)

    if case["kind"] == "exchange":
        n = _rows(case)
        state["xs"][:n] = state["x"][state["sources"][:n].long() // k]
        state["y"].copy_(combined(state["ys"], state["weights"]))
        return {"xs": state["xs"], "y": state["y"]}
    dy = state["dy"].float()
    for j in range(k):
        at, w = slots[:, j].long(), state["weights"][:, j:j + 1]
        t = _rows(case) // k                     # padding comes last
        state["dys"][at[:t]] = (dy[:t] * w[:t]).to(dtype)
        state["dw"][:, j] = (dy * state["ys"][at.clamp_min(0)].float()).sum(-1) * some[:, j]
    state["dx"].copy_(combined(state["dxs"], None))
    return {"dys": state["dys"], "dw": state["dw"], "dx": state["dx"]}


def _run_adapter(state):
    case, dtype, bounds = state["case"], state["x"].dtype, state["bounds"]
    if case["kind"] == "adapter":
        for e, lo, hi in zip(state["which"], bounds, bounds[1:]):
            y = state["base"][lo:hi].float()
            if e >= 0:
                h = state["x"][lo:hi].float() @ state["a"][e].float().t()
                y = y + (h @ state["b"][e].float().t()) * state["scales"][e]
            state["y"][lo:hi] = y.to(dtype)
        return state["y"]
    state["da"].zero_()
    state["db"].zero_()
    for e, lo, hi in zip(state["which"], bounds, bounds[1:]):
        dx, dy, x = state["base"][lo:hi].float(), state["dy"][lo:hi].float(), state["x"][lo:hi].float()
        if e >= 0:
            dh = (dy @ state["b"][e].float()) * state["scales"][e]
            dx = dx + dh @ state["a"][e].float()
            state["da"][e] += dh.t() @ x
            state["db"][e] += (dy.t() @ state["h"][lo:hi]) * state["scales"][e]
        state["dx"][lo:hi] = dx.to(dtype)
    return {"dx": state["dx"], "da": state["da"], "db": state["db"]}


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "route":
        return _run_route(state)
    if kind == "route-grad":
        return _run_route_grad(state)
    return (_run_exchange if kind.startswith("exchange") else _run_adapter)(state)


# ------------------------------------------------------------------ the same in 64 bits
def _value(x):
    return x.to(torch.float64)


def _exact_route(case, data):
    """Choices by stable sorts."""
    t, e, g, k = case["tokens"], case["experts"], case["groups"], case["top_k"]
    logits, low = _value(data["logits"]), -math.inf
    if case["score"] == "sigmoid":
        scores = torch.sigmoid(logits)
    else:
        scores = torch.softmax(logits, dim=1).nan_to_num(nan=0.0)
    absent = torch.isneginf(logits)
    if case["kind"] == "route":
        shifted = scores if data["bias"] is None else scores + _value(data["bias"])[None]
        order_by = (logits if data["bias"] is None else shifted).masked_fill(absent, low)
        if g > 1:
            inside = shifted.masked_fill(absent, low).view(t, g, -1).sort(dim=2, descending=True, stable=True).values
            total = inside[:, :, 0].clone()
            if case["group_score"] == "top2" and inside.shape[2] > 1:
                total += inside[:, :, 1].masked_fill(torch.isneginf(inside[:, :, 1]), 0.0)
            kept = total.sort(dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
            allowed = torch.zeros_like(total).scatter_(1, kept, 1.0).bool()
            order_by = order_by.masked_fill(~allowed[:, torch.arange(e, device=logits.device) // (e // g)], low)
        best = order_by.sort(dim=1, descending=True, stable=True)
        ids = best.indices[:, :k].masked_fill(torch.isneginf(best.values[:, :k]), -1)
    else:
        ids = data["ids"].to(torch.int64)
    hit = ids >= 0
    picked = torch.take_along_dim(scores, torch.relu(ids), 1).masked_fill(~hit, 0.0)
    if case["kind"] == "route":
        w = picked / picked.sum(1, keepdim=True) if case["renormalise"] else picked
        flat = ids.flatten()
        by_expert = [torch.nonzero(flat == x).flatten() for x in range(e)]
        sources = torch.full((t * k,), -1, dtype=torch.int32, device=logits.device)
        slots, ends, done = sources.clone(), [0], 0
        for where in by_expert:
            n = where.numel()
            sources[done:done + n] = where.int()
            slots[where] = torch.arange(done, done + n, dtype=torch.int32, device=logits.device)
            done += n
            ends.append(done)
        return {"ids": ids.int(), "weights": (w * case["scale"]).nan_to_num(nan=0.0),
                "offsets": torch.tensor(ends, device=logits.device), "slots": slots.view(t, k), "sources": sources}
    gw = _value(data["dw"]).masked_fill(~hit, 0.0) * case["scale"]
    if case["renormalise"]:
        mass = picked.sum(1, keepdim=True)
        gw = ((gw - (gw * picked / mass).sum(1, keepdim=True)) / mass).nan_to_num(nan=0.0)
    member = torch.zeros_like(scores).scatter_add_(1, torch.relu(ids), gw)
    if case["score"] == "sigmoid":
        return member * scores * (1 - scores)
    return scores * member - scores * (scores * member).sum(1, keepdim=True)


def _exact_exchange(case, data):
    t, k, c = case["tokens"], case["top_k"], case["width"]
    live = _rows(case)
    slots = data["slots"].long()[:live // k]

    def back(rows, weights):
        picked = _value(rows[slots.flatten()]).view(-1, k, c)
        total = (picked * weights[..., None]).sum(1)
        return torch.cat((total, total.new_zeros(t - len(total), c)))

    one = torch.ones(len(slots), k, dtype=torch.float64, device=slots.device)
    w = _value(data["weights"])[:len(slots)]
    if case["kind"] == "exchange":
        xs = torch.zeros(t * k, c, dtype=torch.float64, device=slots.device)
        xs[slots.flatten()] = _value(data["x"])[:len(slots)].repeat_interleave(k, 0)
        return {"xs": xs, "y": back(data["ys"], w)}
    dy = _value(data["dy"])[:len(slots)]
    dys = torch.zeros(t * k, c, dtype=torch.float64, device=slots.device)
    dw = torch.zeros(t, k, dtype=torch.float64, device=slots.device)
    for j in range(k):
        dys[slots[:, j]] = w[:, j, None] * dy
        dw[:len(slots), j] = torch.linalg.vecdot(dy, _value(data["ys"][slots[:, j]]))
    return {"dys": dys, "dw": dw, "dx": back(data["dxs"], one)}


def _exact_adapter(case, data):
    ends = [sum(data["counts"][:k]) for k in range(case["segments"] + 1)]
    x, base, s = _value(data["x"]), _value(data["base"]), _value(data["scales"]).tolist()
    out = base.clone()
    da, db = _value(torch.zeros_like(data["a"])), _value(torch.zeros_like(data["b"]))
    for k, e in enumerate(data["index"]):
        if e < 0:
            continue
        rows = slice(ends[k], ends[k + 1])
        a, b = _value(data["a"][e]), _value(data["b"][e])
        low = torch.matmul(x[rows], a.mT)
        if case["kind"] == "adapter":
            out[rows] += s[e] * torch.matmul(low, b.mT)
            continue
        dy = _value(data["dy"][rows])
        dlow = s[e] * torch.matmul(dy, b)
        out[rows] += torch.matmul(dlow, a)
        da[e] += torch.matmul(dlow.mT, x[rows])
        db[e] += s[e] * torch.matmul(dy.mT, low)
    return out if case["kind"] == "adapter" else {"dx": out, "da": da, "db": db}


def exact(case, seed):
    data = _inputs(case, seed)
    if case["kind"].startswith("route"):
        return _exact_route(case, data)
    return (_exact_exchange if case["kind"].startswith("exchange") else _exact_adapter)(case, data)
