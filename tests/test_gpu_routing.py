"""The routing to experts against 64-bit references.

Choices, places and copies are whole numbers: they must be equal.  Bounds of the others, from the roundings on the way
(u = 2^-24, half a step of fp32):
* weights: 64 bits throughout, but for softmax's sum without bias, groups and renormalising, which is in fp32.  An
  exponential of x = logit - largest, as 2^(x log2 e), is off by at most (1.5 |x| + 3) 2u (the product's rounding and the
  function's), the sum of E terms by (PER + 4) u <= 20 u in the order of the lanes; then one rounding u.
* the logits' gradient: a score is off by a relative (|x| + mean of |x| + 32) 2u, and the difference of two such
  products by the sum of their magnitudes times that; then half a step of the output's type.
* weighted sums of K rows: (K + 1) u of the sum of magnitudes, and half a step; products over C columns C 2u of it.
"""
import pytest

from paper_2604_18556_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
U = 2.0 ** -24
INF = float("inf")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load()
    return torch.device("cuda:0")


def rng_of(*seed):
    return torch.Generator().manual_seed(hash(seed) % (1 << 31))


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


# ------------------------------------------------------------------ references
def scores_ref(r, logits):
    l = logits.double()
    if r.score == B.SCORE_SIGMOID:
        return torch.sigmoid(l)
    return torch.softmax(l, -1).nan_to_num(nan=0.0)


def route_ref(r, logits, bias=None):
    """ids, weights in 64 bits."""
    t, e = logits.shape
    l, s = logits.double(), scores_ref(r, logits)
    value = s if bias is None else s + bias.double()
    gone = torch.isinf(l) & (l < 0) | torch.isnan(value) | (value == -INF)
    value = value.masked_fill(gone, -INF)
    key = (l if bias is None else value).masked_fill(gone, -INF)
    if r.groups > 1:
        best = value.view(t, r.groups, -1).sort(dim=-1, descending=True).values
        group = best[..., 0].clone()
        if r.group_score == B.GROUP_TOP2 and best.shape[-1] > 1:
            group += best[..., 1].masked_fill(best[..., 1] == -INF, 0.0)
        kept = group.sort(dim=-1, descending=True, stable=True).indices[:, :r.top_groups]
        keep = torch.zeros(t, r.groups, dtype=torch.bool).scatter_(1, kept, True)
        key = key.masked_fill(~keep.repeat_interleave(e // r.groups, 1), -INF)
    order = key.sort(dim=-1, descending=True, stable=True)
    ids = order.indices[:, :r.top_k].masked_fill(order.values[:, :r.top_k] == -INF, -1)
    w = s.gather(1, ids.clamp_min(0)).masked_fill(ids < 0, 0.0)
    if r.renormalise:
        w = (w / w.sum(-1, keepdim=True)).nan_to_num(nan=0.0)
    wrong = torch.isnan(l).any(-1) | ((l == INF).any(-1) if r.score == B.SCORE_SOFTMAX else torch.zeros(t).bool())
    ids[wrong] = -1
    w[wrong] = float("nan")
    return ids.int(), w * r.scale


def weights_of(r, logits, ids):
    """The weights of given experts in 64 bits, as a function that can be differentiated."""
    s = torch.sigmoid(logits) if r.score == B.SCORE_SIGMOID else torch.softmax(logits, -1)
    w = s.gather(1, ids.long().clamp_min(0)) * (ids >= 0)
    if r.renormalise:
        w = w / w.sum(-1, keepdim=True)
    return w * r.scale


def group_ref(ids, groups):
    flat = ids.reshape(-1).long()
    flat = torch.where((flat < 0) | (flat >= groups), groups, flat)
    order = torch.argsort(flat, stable=True)
    some = int((flat < groups).sum())
    offsets = torch.zeros(groups + 1, dtype=torch.int64)
    offsets[1:] = torch.bincount(flat, minlength=groups + 1)[:groups].cumsum(0)
    slots = torch.full(flat.shape, -1, dtype=torch.int32)
    slots[order[:some]] = torch.arange(some, dtype=torch.int32)
    sources = order.int()
    sources[some:] = -1
    return offsets, slots.view(ids.shape), sources


def route(r, logits, bias, dev):
    t = logits.shape[0]
    ids = torch.full((t, r.top_k), 77, dtype=torch.int32, device=dev)
    w = torch.full((t, r.top_k), 7.0, device=dev)
    B.route(r, logits.to(dev), ids, w, bias=None if bias is None else bias.to(dev))
    return ids.cpu(), w.cpu()


def weight_bound(r, logits, w, bias):
    if r.score == B.SCORE_SOFTMAX and not r.renormalise and bias is None and r.groups == 1:
        x = (logits.double() - logits.double().amax(-1, keepdim=True)).clamp_min(-1e4)
        mean = (torch.softmax(logits.double(), -1).nan_to_num(nan=0.0) * x.abs()).sum(-1, keepdim=True).nan_to_num(nan=0.0)
        rel = (1.5 * mean + 3) * 2 * U + 20 * U + U
    else:
        rel = 2 * U
    return w.abs() * rel + 1e-44


def group_of(ids, groups, dev):
    n = ids.numel()
    off = torch.full((groups + 1,), 7, dtype=torch.int64, device=dev)
    slots, sources = torch.full(ids.shape, 7, dtype=torch.int32, device=dev), torch.full((n,), 7, dtype=torch.int32, device=dev)
    B.group_rows(ids.to(dev), off, slots, sources)
    return off.cpu(), slots.cpu(), sources.cpu()


# ------------------------------------------------------------------ the choice
R = B.Routing
SOFT, SIG, MAX, TOP2 = B.SCORE_SOFTMAX, B.SCORE_SIGMOID, B.GROUP_MAX, B.GROUP_TOP2
ROUTINGS = [(1, R(1, 1)), (1, R(8, 2)), (5, R(7, 7, score=SIG)), (64, R(64, 8, renormalise=False)), (3, R(65, 5)),
            (9, R(64, 6, 4, 2)), (70, R(256, 8, 8, 4, SIG, TOP2, True, 2.5)), (33, R(160, 6, 8, 3, SOFT, MAX, False, 16.0)),
            (17, R(100, 10, 10, 4, SIG, MAX)), (6, R(162, 6, 9, 4)), (4, R(384, 8)), (5, R(1024, 32, 64, 16, SIG)),
            (3, R(1000, 20, 40, 1, SOFT, TOP2)), (2, R(36, 32, 3, 3, SIG, TOP2, False)), (1001, R(128, 4, 4, 4)),
            (13, R(12, 5, 12, 6, SOFT, TOP2)), (8, R(255, 9, renormalise=False, scale=-0.5)), (3, R(16, 16, 16, 16, SIG)),
            # many tokens, four to a wavefront; more choices than a token has lanes
            (2500, R(64, 20)), (2049, R(100, 6, 10, 4, SIG)), (3001, R(128, 8, 16, 5)), (2100, R(250, 17, renormalise=False)),
            (2053, R(7, 3, score=SIG)), (2200, R(30, 6, 3, 2, SOFT, MAX)), (2070, R(256, 8, 8, 4, SIG, TOP2, True, 2.5)),
            (2060, R(300, 32))]


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("t,r", ROUTINGS, ids=lambda v: str(v) if isinstance(v, int) else f"{v.experts}-{v.top_k}-{v.groups}")
def test_route(dev, t, r, biased, dtype):
    """16-bit logits hold many equal ones; half of the biased cases have a bias of zeros, which leaves them so."""
    print(f"route {t} {r} {biased} {dtype}", flush=True)
    gen = rng_of(t, r.experts, biased)
    logits = torch.randn(t, r.experts, generator=gen).mul_(2).to(dtype)
    bias = torch.randn(r.experts, generator=gen) * 0.1 * (t % 2) if biased else None
    ids, w = route(r, logits, bias, dev)
    idr, wr = route_ref(r, logits, bias)
    assert torch.equal(ids, idr)
    assert ((w.double() - wr).abs() <= weight_bound(r, logits, wr, bias)).all()


@pytest.mark.parametrize("times", [1, 130])
@pytest.mark.parametrize("biased", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("score", [SOFT, SIG], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top_groups,renorm", [(1, 1, True), (1, 1, False), (6, 2, True), (6, 6, False)])
def test_route_rows_that_masks_leave_little_of(dev, groups, top_groups, renorm, score, biased, times):
    """Rows without an expert, with fewer than top_k, with equal logits, huge and tiny ones, and rows that are not
    finite beside fine ones; few and many of them (a token by all lanes of a wavefront, and by a quarter)."""
    e, k = 48, 6
    r = R(e, k, groups, top_groups, score, TOP2, renorm, 1.5)
    gen = rng_of(groups, renorm, score)
    logits = torch.randn(16, e, generator=gen)
    logits[1] = -INF
    logits[2, 3:] = -INF
    logits[3, :47] = -INF
    logits[4] = 0.25
    logits[5, 7] = float("nan")
    logits[6, 20] = INF
    logits[7] = -INF
    logits[7, 13] = float("nan")
    logits[8] *= 40.0
    logits[9] = -200.0 + logits[9]
    logits[10, ::2] = -INF
    logits[11] = torch.finfo(torch.float32).min
    logits[12] = torch.finfo(torch.float32).min
    logits[12, 40] = 3.0
    logits[13, 1:] = -0.0
    logits[13, 0] = 0.0
    bias = None
    if biased:
        bias = torch.randn(e, generator=gen) * 0.2
        bias[11], bias[12], bias[33] = -INF, float("nan"), 5.0
    logits = logits.repeat(times, 1)
    ids, w = route(r, logits, bias, dev)
    idr, wr = route_ref(r, logits, bias)
    assert torch.equal(ids, idr)
    assert torch.equal(torch.isnan(w), torch.isnan(wr))
    fine = ~torch.isnan(wr)
    assert ((w.double() - wr).abs() <= weight_bound(r, logits, wr, bias))[fine].all()
    assert (ids[1] == -1).all() and (w[1] == 0).all() and torch.isnan(w[5]).all() and (ids[5] == -1).all()
    if not biased:
        assert ids[4].tolist() == list(range(6)) and ids[13].tolist() == list(range(6))


def test_route_keys_that_32_bits_do_not_tell_apart(dev):
    """Scores that differ by less than fp32 holds beside a bias, and scores that are equal where logits are not."""
    r = R(4, 2, score=SIG)
    logits = torch.tensor([[0.0, 1e-7, 0.0, -3.0], [30.0, 31.0, 32.0, 29.0]])
    for bias in (torch.tensor([7.0, 7.0, 7.0, 7.0]), torch.tensor([0.0, 0.0, 1e-30, 0.0])):
        ids, _ = route(r, logits, bias, dev)
        assert torch.equal(ids, route_ref(r, logits, bias)[0])
    assert route(r, logits, None, dev)[0].tolist() == [[1, 0], [2, 1]]


@pytest.mark.parametrize("times", [1, 1200])
@pytest.mark.parametrize("score,scale", [(SOFT, 1.5), (SIG, 2.5)], ids=["softmax", "sigmoid"])
def test_route_weights_of_subnormal_scores(dev, score, scale, times):
    """A bias chooses experts whose scores in 64 bits are below the smallest normal one: weights are still their shares.
    One expert's is the scale itself.  Others: scores of at least 2^-1041 are whole numbers of 2^-1074, off by up to two of
    them, 2^-32 of a score, here and in the reference: 2^-30 of a share with the sum's, beside half a step of fp32."""
    low = 720.0 if score == SOFT else 709.0
    logits = torch.tensor([[low, 0.0, 0.25, -0.5, 1.0, 0.0, 0.0, 0.0], [0.0, 3.0, -0.25, -1.0, low, 0.5, 0.0, 0.0]]) - low
    if score == SIG:
        logits = logits.clamp_min(-709.5)
    bias = torch.tensor([0.0, 9.0, 8.0, 7.0, 0.0, 6.0, 0.0, 0.0])
    logits = logits.repeat(times, 1)
    for k in (1, 2, 4):
        r = R(8, k, score=score, scale=scale)
        ids, w = route(r, logits, bias, dev)
        idr, wr = route_ref(r, logits, bias)
        assert torch.equal(ids, idr) and ids[0].tolist() == [1, 2, 3, 5][:k]
        assert torch.isfinite(w).all() and ((w.double() - wr).abs() <= wr * (U + 2.0 ** -30)).all()
        if k == 1:
            assert (w == scale).all()
    if score == SOFT:                              # the smallest score that there is, and none at all
        r = R(8, 1, scale=scale)
        for down, want in ((744.0, scale), (800.0, 0.0)):
            _, w = route(r, torch.cat((logits[:1, :1] * 0 + down, logits[:1, 1:] * 0), 1).repeat(times, 1), bias, dev)
            assert (w == want).all()


def test_route_from_any_address(dev):
    gen = rng_of(4)
    for e in (33, 64, 255):
        r = R(e, 4, renormalise=False)
        for dtype in (BF16, FP32):
            logits = torch.randn(9, e, generator=gen).to(dtype)
            pool = torch.zeros(9 * e + 3, dtype=dtype, device=dev)
            moved = pool[3:].view(9, e)
            moved.copy_(logits)
            ids, w = torch.zeros(9, 4, dtype=torch.int32, device=dev), torch.zeros(9, 4, device=dev)
            B.route(r, moved, ids, w)
            ref = route(r, logits, None, dev)
            assert torch.equal(ids.cpu(), ref[0]) and torch.equal(w.cpu(), ref[1])
            d, out = torch.ones(9, 4, device=dev), torch.zeros(9 * e + 1, dtype=dtype, device=dev)[1:].view(9, e)
            B.route_grad(r, moved, ids, d, out)
            want = torch.empty(9, e, dtype=dtype, device=dev)
            B.route_grad(r, logits.to(dev), ids, d, want)
            assert torch.equal(out, want)


# ------------------------------------------------------------------ its gradient
def grad_ref(r, logits, ids, dw):
    l = logits.double().requires_grad_()
    (weights_of(r, l, ids) * dw.double()).sum().backward()
    return l.grad


def grad_bound(r, logits, ids, dw, dtype, ref):
    l, s = logits.double(), scores_ref(r, logits)
    x = (l - l.amax(-1, keepdim=True)).abs() if r.score == SOFT else l.abs()
    chosen = torch.zeros_like(s).scatter_add_(1, ids.long().clamp_min(0), (ids >= 0).double()) > 0
    g = torch.zeros_like(s).scatter_add_(1, ids.long().clamp_min(0), dw.double().abs() * (ids >= 0)) * abs(r.scale)
    p = s * chosen if r.renormalise else s
    if r.renormalise:
        p = p / p.sum(-1, keepdim=True)
    near = x.masked_fill(~chosen, 0.0).amax(-1, keepdim=True) if r.renormalise else (s * x).sum(-1, keepdim=True)
    mag = p * (g + (g * p).sum(-1, keepdim=True))
    # the reference's own: experts that are not chosen have a gradient of zero, which 64 bits form as a difference
    own = (l.shape[-1] + 16) * 2.0 ** -52 * g.sum(-1, keepdim=True)
    err = mag * (x + near + 32) * 2 * U + own
    return err + half_step(dtype) * (ref.abs() + err) + smallest(dtype)


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("t,r", ROUTINGS, ids=lambda v: str(v) if isinstance(v, int) else f"{v.experts}-{v.top_k}-{v.groups}")
def test_route_grad(dev, t, r, dtype):
    gen = rng_of(t, r.experts, 3)
    logits = torch.randn(t, r.experts, generator=gen).mul_(2).to(dtype)
    ids, _ = route_ref(r, logits)
    if t > 2:
        ids[1, r.top_k // 2:] = -1                # a token with fewer experts
    dw = torch.randn(t, r.top_k, generator=gen)
    out = torch.full((t, r.experts), 7.0, dtype=dtype, device=dev)
    B.route_grad(r, logits.to(dev), ids.to(dev), dw.to(dev), out)
    if t > 2 and r.top_k // 2 == 0 and r.renormalise:
        ids, dw, logits, out = (torch.cat((v[:1], v[2:])) for v in (ids, dw, logits, out))   # 0 / 0 in the reference
    ref = grad_ref(r, logits, ids, dw)
    assert ((out.cpu().double() - ref).abs() <= grad_bound(r, logits, ids, dw, dtype, ref)).all()


def test_route_grad_is_the_weights_differences(dev):
    """Central differences of the 64-bit weights, step h: off by h^2 / 6 times the third derivative (below 24 for
    products of scores) and by 2^-52 / h."""
    h, gen = 1e-4, rng_of(8)
    for r in (R(12, 4), R(12, 4, renormalise=False), R(12, 4, score=SIG), R(12, 4, score=SIG, renormalise=False, scale=2.5)):
        logits, dw = torch.randn(3, 12, generator=gen), torch.randn(3, 4, generator=gen)
        ids, _ = route_ref(r, logits)
        out = torch.empty(3, 12, device=dev)
        B.route_grad(r, logits.to(dev), ids.to(dev), dw.to(dev), out)
        for e in range(12):
            step = torch.zeros(12, dtype=torch.float64)
            step[e] = h
            d = (weights_of(r, logits.double() + step, ids) - weights_of(r, logits.double() - step, ids)) / (2 * h)
            lim = 4 * h * h * r.scale * dw.abs().double().sum(-1) + 1e-11 + 64 * U * r.scale * dw.abs().double().sum(-1)
            assert ((out[:, e].cpu().double() - (d * dw).sum(-1)).abs() <= lim).all()


def test_route_grad_with_ids_that_are_not_experts_or_come_twice(dev):
    r = R(10, 3, renormalise=False)
    gen = rng_of(2)
    logits, dw = torch.randn(4, 10, generator=gen), torch.randn(4, 3, generator=gen)
    ids = torch.tensor([[1, 10, 2], [-5, 3, 1 << 30], [4, 4, 9], [-1, -1, -1]], dtype=torch.int32)
    out = torch.empty(4, 10, device=dev)
    B.route_grad(r, logits.to(dev), ids.to(dev), dw.to(dev), out)
    clean = torch.where((ids < 0) | (ids >= 10), -1, ids)
    ref = grad_ref(r, logits, clean, dw)
    assert ((out.cpu().double() - ref).abs() <= grad_bound(r, logits, clean, dw, FP32, ref)).all()
    assert not out[3].any()
    for s in (SOFT, SIG):                          # padding: no logit is finite, no expert is chosen
        for renorm in (False, True):
            B.route_grad(R(10, 3, score=s, renormalise=renorm), torch.full((4, 10), -INF, device=dev),
                         torch.full((4, 3), -1, dtype=torch.int32, device=dev), dw.to(dev), out)
            assert not out.any()


# ------------------------------------------------------------------ the order of rows
@pytest.mark.parametrize("groups", [1, 2, 7, 64, 257, 4096])
@pytest.mark.parametrize("count", [0, 1, 63, 64, 65, 1000, 4097, 8192, 8193, 20000, 200003])
def test_group_rows(dev, count, groups):
    """Even ids, and ids of which most are one; some belong to no group."""
    print(f"group {count} {groups}", flush=True)
    gen = rng_of(count, groups)
    for skewed in (False, True):
        ids = torch.randint(0, groups, (count,), generator=gen, dtype=torch.int32)
        if skewed:
            ids[torch.rand(count, generator=gen) < 0.7] = groups - 1
            ids[torch.rand(count, generator=gen) < 0.1] = -1
            ids[torch.rand(count, generator=gen) < 0.02] = groups
            ids[torch.rand(count, generator=gen) < 0.02] = -(1 << 31)
            ids[torch.rand(count, generator=gen) < 0.02] = (1 << 31) - 1
        for got, ref in zip(group_of(ids, groups, dev), group_ref(ids, groups)):
            assert torch.equal(got, ref)


def test_group_rows_of_none_and_of_many(dev):
    ids = torch.full((3000, 4), -1, dtype=torch.int32)
    off, slots, sources = group_of(ids, 5, dev)
    assert not off.any() and (slots == -1).all() and (sources == -1).all()
    ids = torch.randint(0, 300, (1 << 20, 3), generator=rng_of(6), dtype=torch.int32)
    for got, ref in zip(group_of(ids, 300, dev), group_ref(ids, 300)):
        assert torch.equal(got, ref)


# ------------------------------------------------------------------ rows there and back
def exchange_case(t, k, drop, gen):
    """Distinct slots among a few rows more than needed, some of them naming no row."""
    n = t * k + 3
    slots = torch.randperm(n, generator=gen)[:t * k].view(t, k).int()
    if drop:
        gone = torch.rand(t, k, generator=gen) < 0.3
        slots[gone] = torch.tensor([-1, n, -(1 << 31), (1 << 31) - 1], dtype=torch.int32)[
            torch.randint(0, 4, (int(gone.sum()),), generator=gen)]
    return slots, n


def combine_ref(rows, slots, weights):
    some = (slots >= 0) & (slots < rows.shape[0])
    picked = rows.double()[torch.where(some, slots, 0).long()] * some[..., None]
    w = weights.double()[..., None]
    return (picked * w).sum(1), (picked * w).abs().sum(1), picked


EXCHANGES = [(1, 1, 1), (3, 2, 7), (5, 3, 8), (70, 8, 64), (33, 9, 203), (2, 33, 24), (19, 4, 1000), (9, 8, 7168),
             (300, 6, 72), (4, 2, 20001), (17, 1, 2048),
             (7, 8, 520), (5, 8, 516), (3, 10, 2056), (6, 8, 264), (40, 1, 3), (9, 2, 5)]


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("t,k,c", EXCHANGES)
def test_exchange(dev, t, k, c, shift, dtype):
    """Dispatch, combine and their gradients; rows that no slot names stay; arrays that begin `shift` elements in."""
    print(f"exchange {t} {k} {c} {shift} {dtype}", flush=True)
    gen = rng_of(t, k, c)

    def moved(x):
        m = torch.zeros(x.numel() + shift, dtype=x.dtype, device=dev)[shift:].view(x.shape)
        return m.copy_(x)

    for drop in (False, True):
        slots, n = exchange_case(t, k, drop, gen)
        some = (slots >= 0) & (slots < n)
        x, dy = torch.randn(t, c, generator=gen).to(dtype), torch.randn(t, c, generator=gen).to(dtype)
        rows, w = torch.randn(n, c, generator=gen).to(dtype), torch.randn(t, k, generator=gen)
        xd, dyd, rowsd, wd, sd = moved(x), moved(dy), moved(rows), moved(w), moved(slots)
        out = moved(torch.full((n, c), 7.0, dtype=dtype))
        B.dispatch_rows(xd, sd, out)
        ref = torch.full((n, c), 7.0, dtype=dtype)
        ref[slots[some].long()] = x[:, None].expand(t, k, c)[some]
        assert torch.equal(out.cpu(), ref)
        for weights in (w, None):
            y = moved(torch.full((t, c), 7.0, dtype=dtype))
            B.combine_rows(rowsd, sd, y, weights=None if weights is None else wd)
            ref, mag, picked = combine_ref(rows, slots, torch.ones(t, k) if weights is None else w)
            err = (k + 1) * U * mag
            assert ((y.cpu().double() - ref).abs() <= err + half_step(dtype) * (ref.abs() + err) + smallest(dtype)).all()
        drows, dw = moved(torch.full((n, c), 7.0, dtype=dtype)), moved(torch.full((t, k), 7.0))
        B.combine_rows_grad(dyd, rowsd, sd, wd, drows, dw)
        # w dy, rounded to fp32 or not before it is rounded to the type: u of the product and half a step at most
        ref = torch.full((n, c), 7.0, dtype=torch.float64)
        ref[slots[some].long()] = (w.double()[..., None] * dy.double()[:, None])[some]
        lim = ref.abs() * (U + half_step(dtype) * (1 + U)) + smallest(dtype)
        named = torch.zeros(n, dtype=torch.bool)
        named[slots[some].long()] = True
        assert ((drows.cpu().double() - ref).abs() <= lim).all() and (drows.cpu()[~named] == 7).all()
        picked = combine_ref(rows, slots, w)[2]
        prod = picked * dy.double()[:, None]
        assert ((dw.cpu().double() - prod.sum(-1)).abs() <= c * 2 * U * prod.abs().sum(-1)).all()
        assert not dw.cpu()[~some].any()


@pytest.mark.parametrize("t,k,c", [(1100, 4, 4096), (5000, 1, 4104)])
def test_exchanges_that_no_cache_holds(dev, t, k, c):
    """Against the same sums by torch on the GPU, from the bounds above; rows that no slot names stay."""
    gen = torch.Generator(device=dev).manual_seed(t)
    n = t * k + 5
    slots = torch.randperm(n, generator=gen, device=dev)[:t * k].view(t, k).int()
    slots[3, 0], slots[t - 1, k - 1] = -1, n
    some = (slots >= 0) & (slots < n)
    at = torch.where(some, slots, 0).long()
    x, rows = (torch.randn(m, c, generator=gen, device=dev).to(BF16) for m in (t, n))
    w = torch.randn(t, k, generator=gen, device=dev)
    out, y = torch.full((n, c), 7.0, dtype=BF16, device=dev), torch.empty(t, c, dtype=BF16, device=dev)
    B.dispatch_rows(x, slots, out)
    B.combine_rows(rows, slots, y, weights=w)
    drows, dw = torch.full((n, c), 7.0, dtype=BF16, device=dev), torch.empty(t, k, device=dev)
    B.combine_rows_grad(x, rows, slots, w, drows, dw)
    named = torch.zeros(n, dtype=torch.bool, device=dev)
    named[slots[some].long()] = True
    assert (out[~named] == 7).all() and (drows[~named] == 7).all()
    ref, mag = torch.zeros(t, c, dtype=torch.float64, device=dev), torch.zeros(t, c, dtype=torch.float64, device=dev)
    for j in range(k):
        on = some[:, j]
        assert torch.equal(out[at[on, j]], x[on])
        got, want = drows[at[on, j]].double(), w[on, j:j + 1].double() * x[on].double()
        assert ((got - want).abs() <= want.abs() * (U + half_step(BF16) * (1 + U)) + smallest(BF16)).all()
        part = rows[at[:, j]].double() * on[:, None]
        ref += part * w[:, j:j + 1]
        mag += (part * w[:, j:j + 1]).abs()
        prod = part * x.double()
        assert ((dw[:, j].double() - prod.sum(-1)).abs() <= c * 2 * U * prod.abs().sum(-1)).all()
    err = (k + 1) * U * mag
    assert ((y.double() - ref).abs() <= err + half_step(BF16) * (ref.abs() + err) + smallest(BF16)).all()


@pytest.mark.parametrize("c", [5, 40, 1001, 7168])
def test_rows_that_several_slots_name(dev, c):
    """Each value of such a row is one of theirs; other rows, sums and the weights' gradients are as ever."""
    gen, t, n = rng_of(c), 300, 900
    slots = torch.arange(2 * t, dtype=torch.int32).view(t, 2)
    slots[7] = 500                                 # twice by one token, and by token 250
    slots[100:200, 0] = 700                        # by a hundred
    slots[250, 1] = 3                              # by token 1 too
    x, rows, w = torch.randn(t, c, generator=gen), torch.randn(n, c, generator=gen), torch.randn(t, 2, generator=gen)
    sd, out = slots.to(dev), torch.full((n, c), 7.0, device=dev)
    B.dispatch_rows(x.to(dev), sd, out)
    out = out.cpu()
    for row in (3, 500, 700):
        tokens = (slots == row).any(1).nonzero().flatten()
        assert (out[row] == x[tokens]).any(0).all()
    ref = torch.full((n, c), 7.0)
    ref[slots.flatten().long()] = x.repeat_interleave(2, 0)
    alone = torch.ones(n, dtype=torch.bool)
    alone[[3, 500, 700]] = False
    assert torch.equal(out[alone], ref[alone])
    y, drows, dw = torch.empty(t, c, device=dev), torch.full((n, c), 7.0, device=dev), torch.empty(t, 2, device=dev)
    B.combine_rows(rows.to(dev), sd, y, weights=w.to(dev))
    want, mag, picked = combine_ref(rows, slots, w)
    assert ((y.cpu().double() - want).abs() <= 3 * U * mag + U * want.abs() + smallest(FP32)).all()
    B.combine_rows_grad(x.to(dev), rows.to(dev), sd, w.to(dev), drows, dw)
    prod = picked * x.double()[:, None]
    assert ((dw.cpu().double() - prod.sum(-1)).abs() <= c * 2 * U * prod.abs().sum(-1)).all()
    drows = drows.cpu().double()
    for row in (3, 500, 700):
        token, place = (slots == row).nonzero(as_tuple=True)
        each = w[token, place, None].double() * x[token].double()
        assert ((drows[row] - each).abs() <= each.abs() * 2 * U + smallest(FP32)).any(0).all()


def test_exchange_gradients_are_differences(dev):
    """f = <dy, combine(rows, w)> is linear in each: with small whole numbers its differences are exact."""
    gen, t, k, c = rng_of(3), 6, 3, 40
    slots, n = exchange_case(t, k, True, gen)
    whole = [torch.randint(-3, 4, s, generator=gen).float().to(dev) for s in ((n, c), (t, k), (t, c))]
    rows, w, dy = whole
    sd = slots.to(dev)
    drows, dw = torch.zeros(n, c, device=dev), torch.empty(t, k, device=dev)
    B.combine_rows_grad(dy, rows, sd, w, drows, dw)

    def f(rows_, w_):
        y = torch.empty(t, c, device=dev)
        B.combine_rows(rows_, sd, y, weights=w_)
        return (y * dy).sum().item()

    for p, q in ((0, 0), (7, 39), (n - 1, 5), (4, 11)):
        step = rows.clone()
        step[p, q] += 1
        assert f(step, w) - f(rows, w) == drows[p, q].item()
    for p, q in ((0, 0), (5, 2), (3, 1)):
        step = w.clone()
        step[p, q] += 1
        assert f(rows, step) - f(rows, w) == dw[p, q].item()


def test_values_that_are_not_finite_stay_in_their_rows(dev):
    t, k, c = 5, 2, 72
    slots = torch.arange(10, dtype=torch.int32).view(t, k).to(dev)
    slots[4, 1] = -1
    rows, w = torch.ones(10, c, dtype=BF16, device=dev), torch.ones(t, k, device=dev)
    rows[3, 7] = float("nan")
    rows[4, 71] = INF
    w[0, 1], w[4, 1] = INF, float("nan")
    y = torch.empty(t, c, dtype=BF16, device=dev)
    B.combine_rows(rows, slots, y, weights=w)
    bad = torch.zeros(t, c, dtype=torch.bool)
    bad[0], bad[4], bad[1, 7], bad[2, 71] = True, True, True, True
    assert torch.equal(~torch.isfinite(y.cpu()), bad)


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("c", [3, 67, 72, 523, 528, 4099])
@pytest.mark.parametrize("k", [2, 3])
def test_gradients_of_weights_with_values_that_are_not_finite(dev, k, c, dtype):
    """A weight whose slot names no row has gradient 0 whatever dout is; infinities in one place of a row give infinities,
    also in the last columns, and stay with their slots."""
    t = 2 * c if c < 8 else 40
    slots = torch.arange(t * k, dtype=torch.int32).view(t, k)
    dout, rows = torch.ones(t, c, dtype=dtype), torch.ones(t * k, c, dtype=dtype)
    want = torch.full((t, k), float(c))
    for i in range(0, t - 1, 2):                      # infinities from the last column on backwards
        at = c - 1 - i // 2 % c
        rows[i * k + 1, at], want[i, 1] = -INF, -INF
        dout[i + 1, at], want[i + 1] = INF, INF
    slots[1, 0], slots[3, k - 1], want[1, 0], want[3, k - 1] = -1, t * k, 0, 0
    slots[5], want[5], dout[5] = -1, 0, float("nan")
    w, drows, dw = torch.ones(t, k, device=dev), torch.zeros(t * k, c, dtype=dtype, device=dev), torch.empty(t, k, device=dev)
    B.combine_rows_grad(dout.to(dev), rows.to(dev), slots.to(dev), w, drows, dw)
    assert torch.equal(dw.cpu(), want)
    some = (slots >= 0) & (slots < t * k)
    assert torch.equal(drows.cpu()[slots[some].long()], dout[:, None].expand(t, k, c)[some])


def test_no_tokens(dev):
    r = R(8, 2)
    none, ids, w = torch.empty(0, 8, device=dev), torch.empty(0, 2, dtype=torch.int32, device=dev), torch.empty(0, 2, device=dev)
    B.route(r, none, ids, w)
    B.route_grad(r, none, ids, w, none)
    rows = torch.full((3, 16), 7.0, device=dev)
    B.dispatch_rows(torch.empty(0, 16, device=dev), ids, rows)
    B.combine_rows(rows, ids, torch.empty(0, 16, device=dev))
    B.combine_rows_grad(torch.empty(0, 16, device=dev), rows, ids, w, rows.clone(), w)
    assert (rows == 7).all()
    # no rows: every slot names none
    x, s = torch.ones(2, 16, device=dev), torch.zeros(2, 2, dtype=torch.int32, device=dev)
    B.dispatch_rows(x, s, torch.empty(0, 16, device=dev))
    B.combine_rows(torch.empty(0, 16, device=dev), s, x)
    assert not x.any()


def test_more_tokens_than_a_grid_has_workgroups(dev):
    """Each workgroup goes through several tokens, one after another."""
    c, t = 264, (1 << 24) + 5000
    x = (torch.arange(t, device=dev) % 199).to(BF16)[:, None].expand(t, c).contiguous()
    slots = torch.arange(t - 1, -1, -1, dtype=torch.int32, device=dev)[:, None].contiguous()
    out = torch.zeros(t, c, dtype=BF16, device=dev)
    B.dispatch_rows(x, slots, out)
    assert torch.equal(out, x.flip(0))
    y = torch.zeros_like(x)
    B.combine_rows(out, slots, y)
    assert torch.equal(y, x)
    del y
    t = (1 << 22) + 5000
    x, out, slots = x[:t], out[-t:], slots[-t:].contiguous()      # slots t - 1 .. 0
    w, dw, drows = torch.full((t, 1), 0.5, device=dev), torch.zeros(t, 1, device=dev), torch.zeros(t, c, dtype=BF16, device=dev)
    B.combine_rows_grad(x, out.contiguous(), slots, w, drows, dw)
    assert torch.equal(drows, (x * 0.5).flip(0))
    assert torch.equal(dw[:, 0], x[:, 0].float() ** 2 * c)        # whole numbers below 2^24


def test_rows_beyond_32_bits(dev):
    """Elements past 2^31 of the rows' array."""
    c, n = 8192, (1 << 18) + 9
    rows = torch.zeros(n, c, dtype=BF16, device=dev)
    x = torch.randn(2, c, generator=rng_of(1)).to(BF16).to(dev)
    slots = torch.tensor([[n - 1, 0], [n - 3, -1]], dtype=torch.int32, device=dev)
    B.dispatch_rows(x, slots, rows)
    assert torch.equal(rows[n - 1], x[0]) and torch.equal(rows[0], x[0]) and torch.equal(rows[n - 3], x[1])
    assert not rows[1:n - 3].any() and not rows[n - 2].any()
    y, dw = torch.empty_like(x), torch.empty(2, 2, device=dev)
    B.combine_rows(rows, slots, y)
    assert torch.equal(y[1], x[1]) and torch.equal(y[0], (2 * x[0].float()).to(BF16))
    B.combine_rows_grad(x, rows.clone(), slots, torch.ones(2, 2, device=dev), rows, dw)
    assert dw[1, 1] == 0 and torch.equal(rows[n - 3], x[1])


# ------------------------------------------------------------------ as they are used
def moe(dev, r, x, logits, w, linear=None):
    """One layer of routed experts by the library's calls, and what its backward needs."""
    t, k, o, n = x.shape[0], r.top_k, w.shape[1], x.shape[0] * r.top_k
    s = {"ids": torch.empty(t, k, dtype=torch.int32, device=dev), "w": torch.empty(t, k, device=dev),
         "off": torch.empty(r.experts + 1, dtype=torch.int64, device=dev),
         "slots": torch.empty(t, k, dtype=torch.int32, device=dev), "src": torch.empty(n, dtype=torch.int32, device=dev),
         "xs": torch.zeros(n, x.shape[1], dtype=x.dtype, device=dev), "ys": torch.zeros(n, o, dtype=x.dtype, device=dev),
         "y": torch.empty(t, o, dtype=x.dtype, device=dev)}

    def forward():
        B.route(r, logits, s["ids"], s["w"])
        B.group_rows(s["ids"], s["off"], s["slots"], s["src"])
        B.dispatch_rows(x, s["slots"], s["xs"])
        if linear is None:
            B.grouped_forward(s["xs"], w, s["ys"], offsets=s["off"])
        else:
            linear.forward(s["xs"], s["ys"], offsets=s["off"])
        B.combine_rows(s["ys"], s["slots"], s["y"], weights=s["w"])

    return s, forward


def test_experts_from_logits_to_gradients(dev):
    """Routing, the experts' products and the way back, and all gradients, with padded tokens, against one expression
    in 64 bits.  Bounds: each 16-bit rounding on the way (the experts' outputs and their gradients) is half a step of
    its magnitude, sums as in the products' own tests."""
    gen, t, e, k, o, i = rng_of(12), 50, 8, 3, 40, 72
    r = R(e, k, renormalise=True)
    logits = torch.randn(t, e, generator=gen)
    logits[47:] = -INF
    x, w = torch.randn(t, i, generator=gen).to(BF16), torch.randn(e, o, i, generator=gen).mul_(0.1).to(BF16)
    dy = torch.randn(t, o, generator=gen).to(BF16)
    xd, wd, ld, dyd = x.to(dev), w.to(dev), logits.to(dev), dy.to(dev)
    s, forward = moe(dev, r, xd, ld, wd)
    forward()
    n = t * k
    dys, dxs = torch.zeros(n, o, dtype=BF16, device=dev), torch.zeros(n, i, dtype=BF16, device=dev)
    dw_, dx, dwt = torch.empty(t, k, device=dev), torch.empty(t, i, dtype=BF16, device=dev), torch.empty(e, o, i, device=dev)
    dl = torch.empty(t, e, device=dev)
    B.combine_rows_grad(dyd, s["ys"], s["slots"], s["w"], dys, dw_)
    B.grouped_input_grad(dys, wd, dxs, offsets=s["off"])
    B.grouped_weight_grad(dys, s["xs"], dwt, offsets=s["off"])
    B.combine_rows(dxs, s["slots"], dx)
    B.route_grad(r, ld, s["ids"], dw_, dl)

    live = slice(0, 47)
    l64, x64, w64 = logits[live].double().requires_grad_(), x[live].double().requires_grad_(), w.double().requires_grad_()
    ids = route_ref(r, logits)[0]
    assert torch.equal(s["ids"].cpu(), ids) and (s["off"][-1] == 47 * k).item()
    rw = weights_of(r, l64, ids[live])
    per = torch.stack([x64 @ w64[j].t() for j in range(e)], 1)                      # t x e x o
    picked = per.gather(1, ids[live].long()[..., None].expand(-1, -1, o))
    y = (picked * rw[..., None]).sum(1)
    y.backward(dy[live].double())
    h = half_step(BF16)
    # |x| |w| of every product, weighted: what roundings are relative to
    mag = torch.stack([x64.abs() @ w64[j].abs().t() for j in range(e)], 1)
    mag = mag.gather(1, ids[live].long()[..., None].expand(-1, -1, o)).detach()
    ymag = (mag * rw.detach()[..., None]).sum(1)
    assert ((s["y"][live].cpu().double() - y.detach()).abs() <= ymag * (2 * h + 200 * U) + 1e-30).all()
    assert not s["y"][47:].any() and not dx[47:].any() and not dl[47:].any()
    # a gradient through two 16-bit roundings (dys, dxs) and its own
    ad = dy[live].double().abs()
    dxmag = sum((rw.detach()[:, j:j + 1] * torch.einsum("to,toi->ti", ad, w.double().abs()[ids[live][:, j].long()]))
                for j in range(k))
    assert ((dx[live].cpu().double() - x64.grad).abs() <= dxmag * (3 * h + 200 * U) + 1e-30).all()
    dwmag = torch.zeros(e, o, i, dtype=torch.float64)
    for j in range(k):
        for row in range(47):
            dwmag[ids[row, j]] += torch.outer(rw.detach()[row, j] * ad[row], x[row].double().abs())
    assert ((dwt.cpu().double() - w64.grad).abs() <= dwmag * (2 * h + 200 * U) + 1e-30).all()
    # dl = sum_j p_j (g_j - D), and each g is a product with the rounded outputs
    gmag = (mag * ad[:, None]).sum(-1)
    p = rw.detach()
    part = p * (gmag + (gmag * p).sum(-1, keepdim=True)) * (h + 300 * U)
    lim = torch.zeros(47, e, dtype=torch.float64).scatter_add_(1, ids[live].long(), part)
    own = (e + 16) * 2.0 ** -52 * gmag.sum(-1, keepdim=True)     # the reference's own, as in grad_bound
    assert ((dl[live].cpu().double() - l64.grad).abs() <= lim + own).all()


def test_experts_with_packed_weights_in_a_graph(dev):
    """Logits to outputs through a packed layer, captured once and replayed for other tokens, with eager runs of the
    same calls between; and the same calls on two streams at once."""
    gen, t, e, k, o, i = rng_of(13), 24, 4, 2, 48, 128
    r = R(e, k, 2, 1, SIG, TOP2)
    cfg = B.LayerConfig(o, i, (-1.5, -0.5, 0.5, 1.5), 64, e)
    packed = torch.randint(0, 256, (B.packed_size(cfg),), generator=gen, dtype=torch.uint8)
    ng = e * o * (i // 64)
    packed[-2 * ng:] = (torch.rand(ng, generator=gen) * 0.1).half().view(torch.uint8)
    lin = B.Linear(cfg, packed.to(dev))
    x, logits = torch.zeros(t, i, dtype=BF16, device=dev), torch.zeros(t, e, device=dev)
    s, forward = moe(dev, r, x, logits, torch.empty(e, o, i, device=dev), lin)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        forward()
    for n in range(4):
        x.copy_(torch.randn(t, i, generator=gen).to(BF16))
        new = torch.randn(t, e, generator=gen)
        new[t - n:] = -INF
        logits.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = {name: v.clone() for name, v in s.items()}
        for name in ("ids", "w", "slots", "src", "y", "off"):
            s[name].fill_(3)
        forward()
        torch.cuda.synchronize()
        total = int(s["off"][-1])
        assert total == (t - n) * k
        for name, v in s.items():
            a, b = (got[name][:total], v[:total]) if name in ("xs", "ys") else (got[name], v)
            assert torch.equal(a, b), name
        assert torch.equal(s["ids"].cpu(), route_ref(r, new)[0])
    pairs = [moe(dev, r, x, logits, torch.empty(e, o, i, device=dev), lin) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(5):
        for (_, call), stream in zip(pairs, streams):
            with torch.cuda.stream(stream):
                call()
    torch.cuda.synchronize()
    for other, _ in pairs:
        assert torch.equal(other["y"], s["y"]) and torch.equal(other["src"], s["src"])
