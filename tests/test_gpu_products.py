"""The products of grouped rows, the 8-bit product and the packed layer against 64-bit references.

Two kinds of inputs:
* small whole numbers, whose products and sums are exact in every type on the way (sums below 2^24, results
  rounded once): the outputs must be the reference's, rounded once, bit for bit;
* random ones, with a bound for each element: the sum of K products in fp32, in any order, is off by at
  most K 2^-23 sum |a b| (a full unit in the last place for each addition, as the matrix cores need not
  round to nearest), and the output's rounding by half a unit, finfo.eps / 2 of the value.
"""
import numpy as np
import pytest

from oracle import pack as refpack
from paper_2604_18556_amd import binding as B
from paper_2604_18556_amd import inputs

from gpu_common import layer_inputs

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load()
    return torch.device("cuda:0")


def rng_of(*seed):
    return torch.Generator().manual_seed(hash(seed) % (1 << 31))


def whole(shape, gen, top=3):
    return torch.randint(-top, top + 1, shape, generator=gen).double()


def offsets_of(counts, dev, first=0):
    return torch.tensor([first] + list(counts)).cumsum(0).to(dev)


def split(off):
    o = off.tolist()
    return list(zip(o, o[1:]))


def forward_ref(x, w, off):
    y = torch.full((x.shape[0], w.shape[1]), float("nan"), dtype=torch.float64)
    for e, (a, b) in enumerate(split(off)):
        y[a:b] = x[a:b] @ w[e].t()
    return y


def assert_close(got, ref, mag, k, dtype, label=""):
    """The bound of the head comment; `mag` is the sum of |a b|."""
    got = got.double().cpu()
    delta = k * 2.0 ** -23 * mag
    half = 0.0 if dtype == FP32 else torch.finfo(dtype).eps / 2
    smallest = 0.0 if dtype == FP32 else torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    bound = delta + half * (ref.abs() + delta) + smallest
    worst = ((got - ref).abs() - bound).max().item() if ref.numel() else -1.0
    assert not torch.isnan(got).any() and worst <= 0, f"{label}: {worst:.3e} beyond the bound"


# rows of each group, out, in: one row; empty groups; sizes around the tiles; odd; many small groups;
# a large group beside tiny ones
SHAPES = [([1], 1, 1), ([1], 16, 8), ([1], 64, 4096), ([3], 40, 72), ([17], 100, 264), ([64], 64, 64),
          ([0, 5, 0, 1, 70], 96, 136), ([65], 257, 130), ([130, 3], 77, 203), ([0], 8, 8),
          ([2] * 70, 24, 48), ([300, 0, 1, 33], 272, 520), ([257], 520, 264), ([1000, 24, 9], 1000, 712),
          ([12, 0, 7], 512, 1032), ([1, 1, 2, 0, 4], 1024, 2048), ([40], 2048, 1024), ([700], 640, 1096),
          ([4, 40, 100, 200], 384, 256), ([2000], 256, 64)]


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,o,i", SHAPES)
def test_products_of_whole_numbers_are_exact(dev, counts, o, i, dtype):
    """All four products; rows before the first and behind the last group stay as they were."""
    print(f"exact {counts} {o}x{i} {dtype}", flush=True)
    gen = rng_of(len(counts), o, i)
    first, e = 2, len(counts)
    rows = first + sum(counts) + 3
    off = offsets_of(counts, dev, first)
    x, w, dy = whole((rows, i), gen), whole((e, o, i), gen, 2), whole((rows, o), gen, 2)
    xd, wd, dyd = (t.to(dtype).to(dev) for t in (x, w, dy))
    y = torch.full((rows, o), 7.0, dtype=dtype, device=dev)
    dx = torch.full((rows, i), 7.0, dtype=dtype, device=dev)
    B.grouped_forward(xd, wd, y, offsets=off)
    B.grouped_input_grad(dyd, wd, dx, offsets=off)
    yr, dxr = torch.full((rows, o), 7.0).double(), torch.full((rows, i), 7.0).double()
    dwr, hr = torch.zeros(e, o, i).double(), torch.zeros(e, i, i).double()
    for k, (a, b) in enumerate(split(off)):
        yr[a:b], dxr[a:b] = x[a:b] @ w[k].t(), dy[a:b] @ w[k]
        dwr[k], hr[k] = dy[a:b].t() @ x[a:b], x[a:b].t() @ x[a:b]
    assert torch.equal(y.cpu(), yr.to(dtype))
    assert torch.equal(dx.cpu(), dxr.to(dtype))
    for out_dtype in (dtype, FP32):
        dw = torch.full((e, o, i), 7.0, dtype=out_dtype, device=dev)
        B.grouped_weight_grad(dyd, xd, dw, offsets=off)
        assert torch.equal(dw.cpu(), dwr.to(out_dtype))
    B.grouped_weight_grad(dyd, xd, dw, offsets=off, accumulate=True)
    assert torch.equal(dw.cpu(), (2 * dwr).float())
    h = torch.full((e, i, i), 7.0, device=dev)
    B.gram(xd, h, offsets=off)
    assert torch.equal(h.cpu(), hr.float())
    B.gram(xd, h, offsets=off, accumulate=True)
    assert torch.equal(h.cpu(), (2 * hr).float())


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,o,i", [([1], 512, 4096), ([33, 0, 200], 264, 1000), ([9], 77, 203),
                                        ([600, 1], 520, 768), ([5, 5, 6], 1024, 7168)])
def test_products_of_random_values(dev, counts, o, i, dtype):
    gen = rng_of(o, i, 5)
    e, rows = len(counts), sum(counts)
    off = offsets_of(counts, dev)
    x = torch.randn(rows, i, generator=gen).mul_(torch.randn(i, generator=gen).mul_(0.5).exp_()).to(dtype)
    w, dy = torch.randn(e, o, i, generator=gen).mul_(0.02).to(dtype), torch.randn(rows, o, generator=gen).to(dtype)
    xd, wd, dyd = (t.to(dev) for t in (x, w, dy))
    x, w, dy = x.double(), w.double(), dy.double()
    y, dx = torch.empty(rows, o, dtype=dtype, device=dev), torch.empty(rows, i, dtype=dtype, device=dev)
    dw, h = torch.empty(e, o, i, dtype=dtype, device=dev), torch.empty(e, i, i, device=dev)
    B.grouped_forward(xd, wd, y, offsets=off)
    B.grouped_input_grad(dyd, wd, dx, offsets=off)
    B.grouped_weight_grad(dyd, xd, dw, offsets=off)
    B.gram(xd, h, offsets=off)
    for k, (a, b) in enumerate(split(off)):
        assert_close(y[a:b], x[a:b] @ w[k].t(), x[a:b].abs() @ w[k].abs().t(), i, dtype, "y")
        assert_close(dx[a:b], dy[a:b] @ w[k], dy[a:b].abs() @ w[k].abs(), o, dtype, "dx")
        assert_close(dw[k], dy[a:b].t() @ x[a:b], dy[a:b].abs().t() @ x[a:b].abs(), b - a, dtype, "dw")
        assert_close(h[k], x[a:b].t() @ x[a:b], x[a:b].abs().t() @ x[a:b].abs(), b - a, FP32, "h")
    assert torch.equal(h, h.mT.contiguous())


# sizes that fill the GPU: whole workgroups on 256, 128 and 64 rows, on 128 x 128 tiles, from unaligned arrays
LARGE = [([2048], 8192, 520), ([1000], 8192, 1032), ([520], 8192, 2056), ([700, 0, 300, 90, 20], 4096, 1032),
         ([4000], 4096, 4104), ([300] * 5, 2048, 2048), ([4100], 2050, 514), ([600, 40], 1030, 3001)]


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,o,i", LARGE)
def test_large_products_of_whole_numbers_are_exact(dev, counts, o, i, dtype):
    """As above, against 64-bit products on the GPU.  Values up to 1, so that 8192 of them stay exact in fp16."""
    print(f"large {counts} {o}x{i} {dtype}", flush=True)
    gen = torch.Generator(device=dev).manual_seed(o + i)
    e, first = len(counts), 5
    rows, off = first + sum(counts) + 9, offsets_of(counts, dev, first)

    def numbers(*shape):
        return torch.randint(-1, 2, shape, generator=gen, device=dev, dtype=torch.int8)

    x, w, dy = numbers(rows, i), numbers(e, o, i), numbers(rows, o)
    y, dx = torch.full((rows, o), 7.0, dtype=dtype, device=dev), torch.full((rows, i), 7.0, dtype=dtype, device=dev)
    dw, h = torch.empty(e, o, i, dtype=dtype, device=dev), torch.empty(e, i, i, device=dev)
    y8, ones = torch.full((rows, o), 7.0, dtype=dtype, device=dev), torch.ones(max(rows, e * o), device=dev)
    B.grouped_forward(x.to(dtype), w.to(dtype), y, offsets=off)
    B.grouped_input_grad(dy.to(dtype), w.to(dtype), dx, offsets=off)
    B.grouped_weight_grad(dy.to(dtype), x.to(dtype), dw, offsets=off)
    B.gram(x.to(dtype), h, offsets=off)
    B.grouped_forward_i8(x, ones[:rows], w, ones[:e * o].view(e, o), y8, offsets=off)
    for k, (a, b) in enumerate(split(off)):
        xe, we, de = x[a:b].double(), w[k].double(), dy[a:b].double()
        ref = (xe @ we.t()).to(dtype)
        assert torch.equal(y[a:b], ref) and torch.equal(y8[a:b], ref)
        assert torch.equal(dx[a:b], (de @ we).to(dtype))
        assert torch.equal(dw[k], (de.t() @ xe).to(dtype))
        assert torch.equal(h[k], (xe.t() @ xe).float())
    for t in (y, y8, dx):
        assert (t[:first] == 7).all() and (t[rows - 9:] == 7).all()


def test_many_groups(dev):
    """More groups than a wavefront has lanes, most of them empty, several times over."""
    gen, e, o, i = rng_of(21), 1000, 72, 136
    counts = torch.randint(0, 4, (e,), generator=gen) * (torch.rand(e, generator=gen) < 0.3)
    counts[777] = 150
    rows, off = int(counts.sum()), offsets_of(counts.tolist(), dev)
    x, w, dy = whole((rows, i), gen, 2), whole((e, o, i), gen, 2), whole((rows, o), gen, 2)
    y, dx = torch.empty(rows, o, dtype=BF16, device=dev), torch.empty(rows, i, dtype=BF16, device=dev)
    dw = torch.empty(e, o, i, device=dev)
    xd, wd, dyd = (t.to(BF16).to(dev) for t in (x, w, dy))
    B.grouped_forward(xd, wd, y, offsets=off)
    B.grouped_input_grad(dyd, wd, dx, offsets=off)
    B.grouped_weight_grad(dyd, xd, dw, offsets=off)
    group = torch.arange(e).repeat_interleave(counts)
    assert torch.equal(y.cpu(), torch.stack([x[r] @ w[group[r]].t() for r in range(rows)]).to(BF16))
    assert torch.equal(dx.cpu(), torch.stack([dy[r] @ w[group[r]] for r in range(rows)]).to(BF16))
    ref = torch.zeros(e, o, i).double()
    for r in range(rows):
        ref[group[r]] += torch.outer(dy[r], x[r])
    assert torch.equal(dw.cpu(), ref.float())


def test_gradients_are_the_forwards_differences(dev):
    """f = <dy, y(x, w)> is linear in x and in w: with whole numbers its differences are exact."""
    gen, counts, o, i = rng_of(1), [6, 0, 11], 40, 56
    rows, off = sum(counts), offsets_of(counts, dev)
    x, w, dy = (whole(s, gen, 2).to(BF16).to(dev) for s in ((rows, i), (3, o, i), (rows, o)))
    dx, dw = torch.empty_like(x), torch.empty(3, o, i, device=dev)
    B.grouped_input_grad(dy, w, dx, offsets=off)
    B.grouped_weight_grad(dy, x, dw, offsets=off)

    def f(x_, w_):
        # y beyond 2^8 would round in bf16: whole numbers up to 2^11 are exact in fp16
        y = torch.empty(rows, o, dtype=FP16, device=dev)
        B.grouped_forward(x_.to(FP16), w_.to(FP16), y, offsets=off)
        return (y.double() * dy.double()).sum().item()

    assert dx.abs().max() <= 256
    base = f(x, w)
    for r, k in ((0, 0), (5, 55), (6, 17), (16, 31)):
        step = x.clone()
        step[r, k] += 1
        assert f(step, w) - base == dx[r, k].item()
    for e, n, k in ((0, 0, 0), (0, 39, 55), (1, 3, 3), (2, 20, 9)):
        step = w.clone()
        step[e, n, k] += 1
        assert f(x, step) - base == dw[e, n, k].item()


@pytest.mark.parametrize("shift", [1, 3, 4])
def test_addresses_of_any_element_alignment(dev, shift):
    """Arrays that begin `shift` elements into their memory."""
    gen, counts, o, i = rng_of(shift), [5, 90], 72, 136
    rows, off = 95, offsets_of(counts, dev)
    x, w, dy = whole((rows, i), gen), whole((2, o, i), gen), whole((rows, o), gen)

    def moved(t, dtype):
        m = torch.zeros(t.numel() + shift, dtype=dtype, device=dev)
        m[shift:] = t.reshape(-1).to(dtype).to(dev)
        return m[shift:].view(t.shape)

    xd, wd, dyd = moved(x, BF16), moved(w, BF16), moved(dy, BF16)
    y, dx = moved(torch.zeros(rows, o), BF16), moved(torch.zeros(rows, i), BF16)
    dw, h = moved(torch.zeros(2, o, i), FP32), moved(torch.zeros(2, i, i), FP32)
    B.grouped_forward(xd, wd, y, offsets=off)
    B.grouped_input_grad(dyd, wd, dx, offsets=off)
    B.grouped_weight_grad(dyd, xd, dw, offsets=off)
    B.gram(xd, h, offsets=off)
    for k, (a, b) in enumerate(split(off)):
        assert torch.equal(y[a:b].cpu(), (x[a:b] @ w[k].t()).to(BF16))
        assert torch.equal(dx[a:b].cpu(), (dy[a:b] @ w[k]).to(BF16))
        assert torch.equal(dw[k].cpu(), (dy[a:b].t() @ x[a:b]).float())
        assert torch.equal(h[k].cpu(), (x[a:b].t() @ x[a:b]).float())
    q, s = moved(torch.zeros(rows, i), torch.int8), moved(torch.zeros(rows), FP32)
    B.quantize_rows(xd, q, s)
    wq, ws = moved(w, torch.int8), moved(torch.ones(2, o), FP32)
    B.grouped_forward_i8(q, s, wq, ws, y, offsets=off)
    for k, (a, b) in enumerate(split(off)):
        ref = (q[a:b].cpu().double() @ w[k].t()).float() * s[a:b].cpu()[:, None]
        assert torch.equal(y[a:b].cpu(), ref.to(BF16))


@pytest.mark.parametrize("counts,o,i", [([4, 20], 48, 72), ([3, 0, 2], 1024, 520), ([300, 40], 300, 200),
                                        ([30, 7], 33, 35)])
def test_values_that_are_not_finite_stay_where_they_belong(dev, counts, o, i):
    """An infinity or NaN in one row (or channel) reaches that row's outputs only: not its neighbours in a
    tile, nor another group's."""
    gen, e, rows = rng_of(o, i), len(counts), sum(counts)
    off = offsets_of(counts, dev)
    x, w, dy = whole((rows, i), gen), whole((e, o, i), gen, 2), whole((rows, o), gen, 2)
    bad_row = counts[0] - 1                      # the last of the first group
    xb, wb, dyb = x.clone(), w.clone(), dy.clone()
    xb[bad_row, i - 1], dyb[bad_row, o - 1] = float("nan"), float("inf")
    wb[e - 1, o - 1, 0] = float("nan")
    xd, wd, dyd = (t.to(BF16).to(dev) for t in (xb, wb, dyb))
    y, dx = torch.empty(rows, o, dtype=BF16, device=dev), torch.empty(rows, i, dtype=BF16, device=dev)
    dw, h = torch.empty(e, o, i, device=dev), torch.empty(e, i, i, device=dev)
    B.grouped_forward(xd, wd, y, offsets=off)
    B.grouped_input_grad(dyd, wd, dx, offsets=off)
    B.grouped_weight_grad(dyd, xd, dw, offsets=off)
    B.gram(xd, h, offsets=off)
    for k, (a, b) in enumerate(split(off)):
        for got, ref in ((y[a:b], (xb[a:b] @ wb[k].t()).to(BF16)), (dx[a:b], (dyb[a:b] @ wb[k]).to(BF16)),
                         (dw[k], (dyb[a:b].t() @ xb[a:b]).float()), (h[k], (xb[a:b].t() @ xb[a:b]).float())):
            got = got.cpu()
            finite = torch.isfinite(ref)
            assert torch.equal(torch.isfinite(got), finite)
            assert torch.equal(got[finite], ref[finite])


def test_offsets_beyond_32_bits(dev):
    """Rows and weights whose element offsets pass 2^31; only the last ones are used."""
    i, rows = 1024, (1 << 21) + 40
    x = torch.zeros(rows, i, dtype=BF16, device=dev)
    gen = rng_of(3)
    tail, w = whole((5, i), gen), whole((1, 24, i), gen)
    x[rows - 6:rows - 1] = tail.to(BF16).to(dev)
    off = torch.tensor([rows - 6, rows - 1], device=dev)
    y = torch.full((rows, 24), 7.0, dtype=BF16, device=dev)
    B.grouped_forward(x, w.to(BF16).to(dev), y, offsets=off)
    assert torch.equal(y[rows - 6:rows - 1].cpu(), (tail @ w[0].t()).to(BF16))
    assert (y[:rows - 6] == 7).all() and (y[rows - 1] == 7).all()
    h = torch.empty(1, i, i, device=dev)
    B.gram(x, h, offsets=off)
    assert torch.equal(h[0].cpu(), (tail.t() @ tail).float())
    dx = torch.full((rows, i), 7.0, dtype=BF16, device=dev)
    dy = torch.zeros(rows, 24, dtype=BF16, device=dev)
    t2 = whole((5, 24), gen)
    dy[rows - 6:rows - 1] = t2.to(BF16).to(dev)
    B.grouped_input_grad(dy, w.to(BF16).to(dev), dx, offsets=off)
    assert torch.equal(dx[rows - 6:rows - 1].cpu(), (t2 @ w[0]).to(BF16))
    assert (dx[rows - 1] == 7).all() and (dx[rows - 7] == 7).all()
    del x, y, dx, dy
    e, o, i = 33, 8192, 8192
    w = torch.zeros(e, o, i, dtype=BF16, device=dev)
    last, x = whole((o, i), gen, 1), whole((2, i), gen, 1)
    w[e - 1] = last.to(BF16).to(dev)
    off = torch.tensor([0] * e + [2], device=dev)
    y = torch.empty(2, o, dtype=BF16, device=dev)
    B.grouped_forward(x.to(BF16).to(dev), w, y, offsets=off)
    assert torch.equal(y.cpu(), (x @ last.t()).to(BF16))
    dy = whole((2, o), gen, 1)
    B.grouped_weight_grad(dy.to(BF16).to(dev), x.to(BF16).to(dev), w, offsets=off)
    assert torch.equal(w[e - 1].cpu(), (dy.t() @ x).to(BF16))
    assert not w[:e - 1].any()


def test_offsets_that_are_wrong_touch_nothing_outside(dev):
    """Offsets beyond the rows or falling: rows outside every reading of them stay as they were."""
    gen, o, i = rng_of(8), 24, 40
    x, w = whole((20, i), gen).to(BF16).to(dev), whole((3, o, i), gen).to(BF16).to(dev)
    pool = torch.full((22, o), 7.0, dtype=BF16, device=dev)
    B.grouped_forward(x, w, pool[1:21], offsets=torch.tensor([-5, 4, 3, 99], device=dev))
    assert (pool[0] == 7).all() and (pool[21] == 7).all()
    B.grouped_forward(x, w, pool[1:21], offsets=torch.tensor([1 << 40, -(1 << 62), 1 << 62, 7], device=dev))
    assert (pool[0] == 7).all() and (pool[21] == 7).all()
    dw = torch.empty(3, o, i, device=dev)
    dy = whole((20, o), gen).to(BF16).to(dev)
    B.grouped_weight_grad(dy, x, dw, offsets=torch.tensor([-5, 30, 2, 1 << 40], device=dev))
    assert torch.isfinite(dw).all()


def test_captured_products_follow_the_offsets(dev):
    """One graph of a layer's products and its backward, on a stream of its own, replayed for other batches,
    with eager calls between."""
    gen, e, o, i, rows = rng_of(9), 4, 136, 264, 60
    w = whole((e, o, i), gen, 2)
    wd = w.to(BF16).to(dev)
    x, dy = torch.zeros(rows, i, dtype=BF16, device=dev), torch.zeros(rows, o, dtype=BF16, device=dev)
    off = offsets_of([15] * 4, dev)
    y, dx = torch.empty(rows, o, dtype=BF16, device=dev), torch.empty(rows, i, dtype=BF16, device=dev)
    dw, h = torch.empty(e, o, i, device=dev), torch.empty(e, i, i, device=dev)
    q, qs = torch.empty(rows, i, dtype=torch.int8, device=dev), torch.empty(rows, device=dev)
    y8, ws = torch.empty(rows, o, dtype=FP16, device=dev), torch.ones(e, o, device=dev)
    w8 = w.to(torch.int8).to(dev)

    def calls():
        B.grouped_forward(x, wd, y, offsets=off)
        B.grouped_input_grad(dy, wd, dx, offsets=off)
        B.grouped_weight_grad(dy, x, dw, offsets=off)
        B.gram(x, h, offsets=off)
        B.quantize_rows(x, q, qs)
        B.grouped_forward_i8(q, qs, w8, ws, y8, offsets=off)

    outs = (y, dx, dw, h, q, qs, y8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for counts in ([60, 0, 0, 0], [1, 2, 50, 7], [0, 0, 0, 60], [20, 0, 39, 1]):
        xr, dyr = whole((rows, i), gen), whole((rows, o), gen, 2)
        x.copy_(xr.to(BF16))
        dy.copy_(dyr.to(BF16))
        off.copy_(offsets_of(counts, dev))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.fill_(3)
        calls()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b)
        for k, (a, b) in enumerate(split(off)):
            assert torch.equal(got[0][a:b].cpu(), (xr[a:b] @ w[k].t()).to(BF16))
            assert torch.equal(got[2][k].cpu(), (dyr[a:b].t() @ xr[a:b]).float())


def test_two_streams_at_once(dev):
    """The calls keep no scratch: the same products on two streams, into outputs of their own."""
    gen, o, i, rows = rng_of(10), 512, 1024, 300
    x, w = whole((rows, i), gen), whole((1, o, i), gen, 2)
    xd, wd = x.to(BF16).to(dev), w.to(BF16).to(dev)
    ref, href = (x @ w[0].t()).to(BF16), (x.t() @ x).float()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [(torch.empty(rows, o, dtype=BF16, device=dev), torch.empty(1, i, i, device=dev)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (y, h) in zip(streams, outs):
            B.grouped_forward(xd, wd, y, stream=s)
            B.gram(xd, h, stream=s)
    torch.cuda.synchronize()
    for y, h in outs:
        assert torch.equal(y.cpu(), ref) and torch.equal(h[0].cpu(), href)


# ------------------------------------------------------------------ 8-bit integers
def quantize_ref(x):
    """Scale in fp32, then the exact quotient in 64 bits, to the nearest, ties to even."""
    x = x.double()
    top = x.abs().amax(-1)
    s = (top / 127.0).float()
    q = torch.where(s[:, None] > 0, x / s.double()[:, None], torch.zeros(()).double()).round().clamp(-127, 127)
    return q.to(torch.int8), s


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 64), (5, 1000), (4, 4096), (3, 20011), (70, 264)])
def test_quantized_rows(dev, rows, cols, dtype):
    gen = rng_of(rows, cols, 2)
    x = torch.randn(rows, cols, generator=gen)
    x = (x / torch.randn(rows, cols, generator=gen).abs().clamp_min(0.05)).to(dtype)
    q = torch.empty(rows, cols, dtype=torch.int8, device=dev)
    s = torch.empty(rows, device=dev)
    B.quantize_rows(x.to(dev), q, s)
    qr, sr = quantize_ref(x)
    assert torch.equal(s.cpu(), sr)
    assert torch.equal(q.cpu(), qr)


@pytest.mark.parametrize("cols", [16, 131, 4096])
def test_quantized_rows_at_the_borders(dev, cols):
    """Exact halves go to even; zeros, the smallest numbers, and rows that are not finite."""
    x = torch.zeros(8, cols)
    halves = torch.arange(-12, 4).double() + 0.5
    x[0, :16] = halves
    x[0, 0] = 127.0                                # scale 1: the halves are ties
    x[1, :16] = halves * 0.25
    x[1, 0] = -127.0 * 0.25
    x[2, cols - 1] = 2.0 ** -126                   # its scale is subnormal
    x[3, :] = 2.0 ** -149
    x[5, 3] = float("inf")
    x[6, cols - 1] = float("nan")
    x[7, 0], x[7, cols - 1] = 3.0e38, -3.4e38
    q, s = torch.full((8, cols), 9, dtype=torch.int8, device=dev), torch.empty(8, device=dev)
    B.quantize_rows(x.to(dev), q, s)
    qr, sr = quantize_ref(x)
    fine = [0, 1, 2, 3, 4, 7]
    assert torch.equal(s.cpu()[fine], sr[fine]) and torch.equal(q.cpu()[fine], qr[fine])
    assert q.cpu()[0, 1:16].tolist() == [-10, -10, -8, -8, -6, -6, -4, -4, -2, -2, 0, 0, 2, 2, 4][:15]
    assert torch.isnan(s[5:7]).all() and not q[5:7].any()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,o,i", SHAPES)
def test_integer_products(dev, counts, o, i, dtype):
    """Full-range integers.  The sum is exact; it, and its two scalings, are rounded to fp32 once each, and
    then to the output's type: three roundings of 2^-24 and one of eps / 2."""
    print(f"int8 {counts} {o}x{i} {dtype}", flush=True)
    gen = rng_of(o, i, 4)
    first, e = 1, len(counts)
    rows = first + sum(counts) + 2
    off = offsets_of(counts, dev, first)
    x = torch.randint(-128, 128, (rows, i), generator=gen, dtype=torch.int8)
    w = torch.randint(-128, 128, (e, o, i), generator=gen, dtype=torch.int8)
    xs, ws = torch.rand(rows, generator=gen) * 0.01, torch.rand(e, o, generator=gen) * 0.01
    y = torch.full((rows, o), 7.0, dtype=dtype, device=dev)
    B.grouped_forward_i8(x.to(dev), xs.to(dev), w.to(dev), ws.to(dev), y, offsets=off)
    y = y.cpu()
    half = torch.finfo(dtype).eps / 2
    small = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for k, (a, b) in enumerate(split(off)):
        dot = x[a:b].double() @ w[k].double().t()
        ref = dot * xs[a:b].double()[:, None] * ws[k].double()
        assert ((y[a:b].double() - ref).abs() <= ref.abs() * (half + 4 * 2.0 ** -24) + small).all()
    rest = torch.ones(rows, dtype=torch.bool)
    rest[first:rows - 2] = False
    assert (y[rest] == 7).all()


def test_integer_sums_at_their_limit(dev):
    """The largest sums that fit: 131071 products of -128 and -128, and a row that is not finite."""
    i = 131071
    x = torch.full((3, i), -128, dtype=torch.int8, device=dev)
    x[1] = 127
    w = torch.full((1, 17, i), -128, dtype=torch.int8, device=dev)
    xs = torch.tensor([2.0 ** -31, 2.0 ** -31, float("nan")], device=dev)
    y = torch.empty(3, 17, dtype=BF16, device=dev)
    B.grouped_forward_i8(x, xs, w, torch.ones(1, 17, device=dev), y)
    assert (y[0].cpu() == torch.tensor(i * 128.0 * 128.0 / 2 ** 31).to(BF16)).all()
    assert (y[1].cpu() == torch.tensor(-i * 128.0 * 127.0 / 2 ** 31).to(BF16)).all()
    assert torch.isnan(y[2]).all()


# ------------------------------------------------------------------ the packed layer
PACKED = [  # layout, levels, group, batch, O, I
    ("group", (-0.5, 0.5), 16, 1, 5, 16), ("group", (-0.5, 0.5), 128, 2, 40, 384),
    ("group", inputs.L3, 32, 1, 17, 96), ("group", inputs.L4, 64, 3, 33, 192),
    ("group", inputs.L4, 128, 1, 256, 1024), ("group", inputs.L4, 256, 2, 48, 768),
    ("group", (-2.0, -1.0, 0.0, 1.0, 2.0), 16, 2, 31, 176), ("group", inputs.L8, 32, 1, 70, 160),
    ("group", inputs.L8, 64, 1, 64, 320), ("group", inputs.L8, 128, 2, 300, 640),
    ("group", inputs.L8, 256, 1, 100, 1280), ("group", tuple(k - 7.5 for k in range(16)), 16, 1, 20, 208),
    ("group", tuple(k - 7.5 for k in range(16)), 128, 2, 272, 512),
    ("group", tuple(round(1.3 ** k - 5, 3) for k in range(11)), 64, 1, 48, 256),
    ("base3", inputs.L3, 16, 3, 7, 48), ("base3", inputs.L3, 128, 1, 256, 512),
    ("base3", (-1.37, 0.11, 0.93), 64, 2, 41, 320),
    ("superblock", inputs.L8, 16, 1, 3, 256), ("superblock", inputs.L8, 16, 3, 50, 768),
    ("superblock", inputs.L4, 16, 1, 256, 512), ("superblock", (-3.3, -1.0, 0.2, 0.7, 2.9), 16, 2, 19, 256)]
LAYOUTS = {"group": B.LAYOUT_GROUP, "base3": B.LAYOUT_BASE3, "superblock": B.LAYOUT_SUPERBLOCK}


def packed_layer(layout, levels, group, batch, o, i, gen):
    """Random codes and scales, their packed bytes (by the oracle), and the effective scales per group."""
    codes = torch.randint(0, len(levels), (batch, o, i), generator=gen).numpy().astype(np.uint8)
    cfg = B.LayerConfig(o, i, levels, group, batch, LAYOUTS[layout],
                        relaxation=B.RELAX_SHIFT if len(levels) > 8 else B.RELAX_GRID)
    if layout == "superblock":
        d = (torch.rand(batch, o, i // 256, generator=gen) * 0.01).half()
        sc = torch.randint(0, 64, (batch, o, i // 16), generator=gen)
        eff = d.float().repeat_interleave(16, -1) * sc
        packed = refpack.pack_superblock(codes, d.numpy(), sc.numpy().astype(np.uint8))
    else:
        s = (torch.rand(batch, o, i // group, generator=gen) * 0.1).half()
        eff = s.float()
        pack = refpack.pack_base3 if layout == "base3" else refpack.pack_plain
        args = (codes, s.numpy()) if layout == "base3" else (codes, s.numpy(), len(levels), group)
        packed = pack(*args)
    w = eff.repeat_interleave(cfg.gs, -1) * torch.tensor(levels)[torch.from_numpy(codes).long()]
    return cfg, torch.from_numpy(np.ascontiguousarray(packed)), w


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("case", PACKED, ids=lambda c: f"{c[0]}-{len(c[1])}-{c[2]}-{c[3]}x{c[4]}x{c[5]}")
def test_packed_products(dev, case, dtype):
    """Identity rows read the weights themselves, bit for bit; random rows keep the bound of the sums; one
    token, a few, and enough for whole tiles."""
    print(f"packed {case} {dtype}", flush=True)
    layout, levels, group, batch, o, i = case
    gen = rng_of(o, i, len(levels))
    cfg, packed, w = packed_layer(*case, gen)
    lin = B.Linear(cfg, packed.to(dev))
    w = w.to(dtype)
    off = offsets_of([i] * batch, dev)
    y = torch.empty(batch * i, o, dtype=dtype, device=dev)
    lin.forward(torch.eye(i).repeat(batch, 1).to(dtype).to(dev), y, offsets=off)
    assert torch.equal(y.cpu().view(batch, i, o), w.transpose(1, 2))
    for counts in ([1] * batch, [3] * (batch - 1) + [0] if batch > 1 else [5],
                   [40] + [2] * (batch - 1), [290] + [17] * (batch - 1)):
        rows = sum(counts) + 1
        off = offsets_of(counts, dev)
        x = torch.randn(rows, i, generator=gen).to(dtype)
        y = torch.full((rows, o), 7.0, dtype=dtype, device=dev)
        lin.forward(x.to(dev), y, offsets=off)
        for e, (a, b) in enumerate(split(off)):
            we, xe = w[e].double(), x[a:b].double()
            assert_close(y[a:b], xe @ we.t(), xe.abs() @ we.abs().t(), i, dtype, str(counts))
        assert (y[rows - 1] == 7).all()
    lin.destroy()


def test_packed_codes_beyond_the_levels_are_the_last_one(dev):
    """Two bits hold four codes where there are three levels."""
    cfg = B.LayerConfig(16, 128, inputs.L3, 128)
    packed = torch.full((B.packed_size(cfg),), 255, dtype=torch.uint8)
    packed[-32:] = torch.full((16,), 0.5).half().view(torch.uint8)
    lin = B.Linear(cfg, packed.to(dev))
    x = torch.ones(1, 128, dtype=BF16, device=dev)
    y = torch.empty(1, 16, dtype=BF16, device=dev)
    lin.forward(x, y)
    assert (y == 64).all()


@pytest.mark.parametrize("counts", [[2048], [700, 0, 130, 20], [300, 300, 300, 300]])
@pytest.mark.parametrize("layout,levels,group", [("group", inputs.L8, 128), ("superblock", inputs.L8, 16),
                                                 ("base3", inputs.L3, 32), ("group", inputs.L4, 256)])
def test_packed_products_with_many_rows(dev, layout, levels, group, counts):
    """Whole tiles, against the dense product with the same weights, which has the same sums in another order."""
    gen, o, i, e = rng_of(group, len(counts)), 2048, 1280, len(counts)
    cfg, packed, w = packed_layer(layout, levels, group, e, o, i, gen)
    lin = B.Linear(cfg, packed.to(dev))
    rows, off = sum(counts), offsets_of(counts, dev)
    x = torch.randn(rows, i, generator=gen).to(BF16).to(dev)
    y = torch.empty(rows, o, dtype=BF16, device=dev)
    lin.forward(x, y, offsets=off)
    w = w.to(BF16).to(dev)
    for k, (a, b) in enumerate(split(off)):
        xe, we = x[a:b].double(), w[k].double()
        assert_close(y[a:b], (xe @ we.t()).cpu(), (xe.abs() @ we.abs().t()).cpu(), i, BF16, f"{layout} {k}")


@pytest.mark.parametrize("rows", [1, 40, 700])
def test_packed_products_from_any_address(dev, rows):
    """x and y that begin at an odd element, and calls on two streams at once."""
    gen, o, i = rng_of(rows, 6), 136, 640
    cfg, packed, w = packed_layer("group", inputs.L4, 64, 1, o, i, gen)
    lin = B.Linear(cfg, packed.to(dev))
    torch.cuda.synchronize()
    x = torch.randn(rows, i, generator=gen).to(BF16)
    xd = torch.zeros(rows * i + 3, dtype=BF16, device=dev)[3:].view(rows, i)
    xd.copy_(x)
    ys = [torch.zeros(rows * o + 1, dtype=BF16, device=dev)[1:].view(rows, o) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in ys]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, y in zip(streams, ys):
            lin.forward(xd, y, stream=s)
    torch.cuda.synchronize()
    w = w[0].to(BF16).double()
    assert_close(ys[0], x.double() @ w.t(), x.double().abs() @ w.abs().t(), i, BF16)
    assert torch.equal(ys[0], ys[1])


def test_packed_values_that_are_not_finite(dev):
    """A scale that is infinite or NaN reaches its own channel, a bad token its own row."""
    gen = rng_of(77)
    for rows in (3, 200):
        cfg, packed, _ = packed_layer("group", inputs.L4, 64, 1, 40, 320, gen)
        scales = packed[-2 * 40 * 5:].view(torch.float16)
        scales[7 * 5 + 4], scales[9 * 5] = float("inf"), float("nan")
        lin = B.Linear(cfg, packed.to(dev))
        x = torch.randn(rows, 320, generator=gen).to(BF16)
        x[1, 319] = float("nan")
        y = torch.empty(rows, 40, dtype=BF16, device=dev)
        lin.forward(x.to(dev), y)
        bad = torch.zeros(rows, 40, dtype=torch.bool)
        bad[1], bad[:, 7], bad[:, 9] = True, True, True
        assert torch.equal(~torch.isfinite(y.cpu()), bad)


@pytest.mark.parametrize("layout", ["group", "superblock", "base3"])
def test_from_tokens_to_the_packed_layer(dev, layout):
    """The operators as they are used: H of two experts from their ragged tokens (in two batches), steps,
    pack, the packed layer on the same tokens, and its error against the dense layer, which must be the hard
    loss that the library reports for H."""
    levels = inputs.L3 if layout == "base3" else inputs.L8
    e, o, i, counts = 2, 96, 256, [700, 420]
    W, _ = layer_inputs(o, i, batch=e, seed=4)
    gen = rng_of(11)
    x = torch.randn(sum(counts), i, generator=gen).to(BF16).to(dev)
    W = torch.from_numpy(W).to(BF16).to(dev)
    off = offsets_of(counts, dev)
    half = torch.tensor([0, 300, 300], device=dev), torch.tensor([300, 700, 1120], device=dev)
    h = torch.empty(e, i, i, device=dev)
    B.gram(x, h, offsets=half[0])
    B.gram(x, h, offsets=half[1], accumulate=True)
    for k, (a, b) in enumerate(split(off)):
        xe = x[a:b].cpu().double()
        assert_close(h[k], xe.t() @ xe, xe.abs().t() @ xe.abs(), b - a + 1, FP32, "H")
    cfg = B.LayerConfig(o, i, levels, 32, e, LAYOUTS[layout], B.PREC_FP32, seed=1)
    layer = B.Layer(cfg, W, h)
    for t in range(3):
        layer.step(B.StepParams(tau=1.0 - 0.3 * t, lr_scales=0.0 if layout == "superblock" else 5e-5))
    hard = torch.zeros(e, device=dev)
    codes = torch.empty(e, o, i, dtype=torch.uint8, device=dev)
    scales = torch.empty(e, o, i // cfg.gs, device=dev)
    layer.harden(codes=codes, scales=scales, hard_loss=hard)
    packed = torch.empty(B.packed_size(cfg), dtype=torch.uint8, device=dev)
    layer.pack(packed)
    layer.destroy()
    lin = B.Linear(cfg, packed)
    del packed
    y, yq = torch.empty(1120, o, dtype=BF16, device=dev), torch.empty(1120, o, dtype=BF16, device=dev)
    B.grouped_forward(x, W, y, offsets=off)
    lin.forward(x, yq, offsets=off)
    wq = scales.repeat_interleave(cfg.gs, -1) * torch.tensor(levels, device=dev)[codes.long()]
    wb = wq.to(BF16)
    yd = torch.empty_like(yq)
    B.grouped_forward(x, wb, yd, offsets=off)
    for k, (a, b) in enumerate(split(off)):
        xe, we = x[a:b].cpu().double(), wb[k].cpu().double()
        mag = xe.abs() @ we.abs().t()
        assert_close(yq[a:b], xe @ we.t(), mag, i, BF16, "packed")
        assert_close(yd[a:b], xe @ we.t(), mag, i, BF16, "dense")
        # tr((W - Wq) H (W - Wq)^T) = |X (W - Wq)^T|^2.  In 64 bits from the same W, codes and tokens the
        # two agree to H's fp32 rounding, (b - a) 2^-23 of each entry, and the loss's own 1e-5.
        r = W[k].cpu().double() - wq[k].cpu().double()
        err = ((xe @ r.t()) ** 2).sum().item()
        lim = (b - a) * 2.0 ** -23 * ((r.abs() @ (xe.abs().t() @ xe.abs())) * r.abs()).sum().item()
        assert abs(hard[k].item() - err) <= lim + 1e-5 * err


def test_linear_is_refused_while_a_stream_is_captured(dev):
    cfg, packed, _ = packed_layer("group", inputs.L4, 64, 1, 32, 128, rng_of(5))
    packed = packed.to(dev)
    ready = B.Linear(cfg, packed)
    x, y = torch.ones(2, 128, dtype=BF16, device=dev), torch.empty(2, 32, dtype=BF16, device=dev)
    ready.forward(x, y)
    want = y.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(B.GsqError, match="captured"):
            B.Linear(cfg, packed)
        ready.forward(x, y)
    for k in (1, 2, 4):                          # powers of two scale exactly
        x.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.float(), want.float() * k)
        y.zero_()


def test_no_rows(dev):
    """Batches without a row: outputs keep what they had, sums over no rows are zero."""
    x, y = torch.empty(0, 64, dtype=BF16, device=dev), torch.empty(0, 32, dtype=BF16, device=dev)
    w = torch.ones(2, 32, 64, dtype=BF16, device=dev)
    off = torch.zeros(3, dtype=torch.int64, device=dev)
    B.grouped_forward(x, w, y, offsets=off)
    B.grouped_input_grad(y, w, x, offsets=off)
    B.grouped_weight_grad(y, x, w, offsets=off)
    assert not w.any()
    h = torch.ones(2, 64, 64, device=dev)
    B.gram(x, h, offsets=off, accumulate=True)
    assert (h == 1).all()
    B.gram(x, h, offsets=off)
    assert not h.any()
    B.quantize_rows(x, torch.empty(0, 64, dtype=torch.int8, device=dev), torch.empty(0, device=dev))
