"""The low-rank adapters against 64-bit references.

* Small whole numbers (hidden below 2^16, sums below 2^24, scales powers of two) are exact on every way: the outputs
  must be the reference's, rounded once, bit for bit.
* Random values: a sum of K products in fp32 is off by at most K 2^-23 of the sum of magnitudes.  hidden enters the second
  product as two 16-bit parts: off by (eps / 2)^2 of it (bf16 2^-16, fp16 2^-22, and 2^-36 of the row's largest there),
  which makes (eps / 2)^2 + (2 rank + 4) 2^-23 of the sum of magnitudes; then the output's half step.
"""
import pytest

from oracle import pack as refpack
from paper_2604_18556_amd import binding as B

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


def whole(shape, gen, top=2):
    return torch.randint(-top, top + 1, shape, generator=gen).double()


def offsets_of(counts, first=0):
    return torch.tensor([first] + list(counts)).cumsum(0)


def segments(off, index, n):
    """(rows, adapter or -1) of each segment."""
    o = off.tolist()
    for k, (a, b) in enumerate(zip(o, o[1:])):
        e = k if index is None else index[k]
        yield slice(a, b), e if 0 <= e < n else -1


class Ref:
    """All results of one case in 64 bits, and the magnitudes that the roundings are relative to."""

    def __init__(self, x, dy, a, b, off, index, scales, base, dbase):
        n, r, q = a.shape[0], x.shape[0], a.shape[1]
        s = torch.ones(n, dtype=torch.float64) if scales is None else scales.double()
        self.h, self.dh = torch.full((r, q), 7.0).double(), torch.full((r, q), 7.0).double()
        self.y, self.dx = torch.full((r, b.shape[1]), 7.0).double(), torch.full((r, a.shape[2]), 7.0).double()
        self.ymag, self.dxmag, self.hmag, self.dhmag = (torch.zeros_like(t) for t in (self.y, self.dx, self.h, self.dh))
        self.da, self.db, self.damag, self.dbmag = (torch.zeros_like(t) for t in (a, b, a, b))
        for rows, e in segments(off, index, n):
            self.y[rows] = 0.0 if base is None else base[rows]
            self.dx[rows] = 0.0 if dbase is None else dbase[rows]
            self.h[rows], self.dh[rows] = 0.0, 0.0
            if e < 0:
                continue
            xr, dr = x[rows], dy[rows]
            self.h[rows], self.hmag[rows] = xr @ a[e].t(), xr.abs() @ a[e].abs().t()
            self.dh[rows], self.dhmag[rows] = s[e] * (dr @ b[e]), s[e].abs() * (dr.abs() @ b[e].abs())
            self.y[rows] += s[e] * (self.h[rows] @ b[e].t())
            self.dx[rows] += self.dh[rows] @ a[e]
            self.ymag[rows] = s[e].abs() * (self.hmag[rows] @ b[e].abs().t())
            self.dxmag[rows] = self.dhmag[rows] @ a[e].abs()
            self.da[e] += self.dh[rows].t() @ xr
            self.db[e] += s[e] * (dr.t() @ self.h[rows])
            self.damag[e] += self.dhmag[rows].t() @ xr.abs()
            self.dbmag[e] += s[e].abs() * (dr.abs().t() @ self.hmag[rows])


class Case:
    """Device tensors of one case; `shift`: elements before each array's first."""

    def __init__(self, dev, dtype, x, dy, a, b, off, index, scales, base, dbase, shift=0):
        def moved(t, of=dtype):
            m = torch.zeros(t.numel() + shift, dtype=of, device=dev)[shift:].view(t.shape)
            return m.copy_(t.to(of))

        r, q = x.shape[0], a.shape[1]
        self.x, self.dy, self.a, self.b = (moved(t) for t in (x, dy, a, b))
        self.base, self.dbase = (None if t is None else moved(t) for t in (base, dbase))
        self.where = {"offsets": None if off is None else off.to(dev),
                      "index": None if index is None else torch.tensor(index, dtype=torch.int32, device=dev),
                      "scales": None if scales is None else moved(scales, FP32)}
        self.h, self.dh = (moved(torch.full((r, q), 7.0), FP32) for _ in range(2))
        self.y, self.dx = moved(torch.full((r, b.shape[1]), 7.0)), moved(torch.full((r, a.shape[2]), 7.0))
        self.da, self.db = moved(torch.full(a.shape, 7.0), FP32), moved(torch.full(b.shape, 7.0), FP32)

    def rows(self):
        B.adapter_forward(self.x, self.a, self.b, self.h, self.y, base=self.base, **self.where)
        B.adapter_input_grad(self.dy, self.a, self.b, self.dh, self.dx, base=self.dbase, **self.where)

    def weights(self, da=None, db=None, accumulate=False):
        B.adapter_weight_grad(self.dy, self.x, self.h, self.dh, self.da if da is None else da,
                              self.db if db is None else db, accumulate=accumulate, **self.where)


# rows of each segment, adapter of each (None: its own), adapters, out, in, rank: one row; empty segments; one adapter in
# several; none; odd sizes; ranks around the instructions' 16 and 32; a long segment beside short ones
SHAPES = [([1], None, 1, 1, 1, 1), ([1], None, 1, 64, 128, 16), ([1] * 9, [3, -1, 0, 3, 1, 7, 2, -5, 0], 4, 136, 264, 16),
          ([3], None, 1, 40, 72, 5), ([17, 0, 5], None, 3, 100, 264, 8), ([64, 65, 1], [0, 0, 1], 2, 257, 130, 17),
          ([0], None, 1, 8, 8, 4), ([130, 3], None, 2, 77, 203, 32), ([40, 0, 7, 20], [1, 0, -1, 1], 3, 520, 712, 40),
          ([300, 2], None, 2, 272, 520, 64), ([33], None, 1, 1000, 96, 100), ([200, 9], [1, 0], 2, 264, 328, 128),
          ([20, 3], None, 2, 48, 2048, 512), ([2] * 70, [k % 5 for k in range(70)], 5, 24, 48, 16), ([5], None, 1, 4104, 24, 33),
          ([1100, 40], None, 2, 1032, 640, 24), ([7, 90], None, 2, 16, 3000, 72)]


def whole_case(dev, counts, index, n, o, i, q, dtype, shift=0, first=2, based=True):
    gen = rng_of(len(counts), o, i, q)
    rows = first + sum(counts) + 3
    off = offsets_of(counts, first)
    x, dy = whole((rows, i), gen), whole((rows, o), gen)
    a, b = whole((n, q, i), gen, 1), whole((n, o, q), gen, 1)
    scales = 2.0 ** torch.randint(-1, 2, (n,), generator=gen).double()
    base, dbase = (whole((rows, o), gen, 99), whole((rows, i), gen, 99)) if based else (None, None)
    return (Ref(x, dy, a, b, off, index, scales, base, dbase),
            Case(dev, dtype, x, dy, a, b, off, index, scales, base, dbase, shift))


def assert_exact(ref, c, dtype):
    c.rows()
    assert torch.equal(c.h.cpu(), ref.h.float()) and torch.equal(c.dh.cpu(), ref.dh.float())
    assert torch.equal(c.y.cpu(), ref.y.to(dtype))
    assert torch.equal(c.dx.cpu(), ref.dx.to(dtype))
    c.weights()
    assert torch.equal(c.da.cpu(), ref.da.float()) and torch.equal(c.db.cpu(), ref.db.float())


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,index,n,o,i,q", SHAPES, ids=lambda v: str(v) if isinstance(v, int) else "")
def test_adapters_of_whole_numbers_are_exact(dev, counts, index, n, o, i, q, dtype):
    """Forward and all gradients; rows before the first and behind the last segment stay as they were."""
    print(f"exact {counts[:4]} {n} {o}x{i} {q} {dtype}", flush=True)
    ref, c = whole_case(dev, counts, index, n, o, i, q, dtype)
    assert_exact(ref, c, dtype)
    c.weights(accumulate=True)
    assert torch.equal(c.da.cpu(), 2 * ref.da.float()) and torch.equal(c.db.cpu(), 2 * ref.db.float())
    da, db = torch.empty_like(c.a), torch.empty_like(c.b)
    c.weights(da, db)
    assert torch.equal(da.cpu(), ref.da.to(dtype)) and torch.equal(db.cpu(), ref.db.to(dtype))


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,index,n,o,i,q", [([1500, 30], [1, 0], 2, 12296, 1040, 24), ([900, 0, 800], None, 3, 1032, 11264, 48),
                                                  ([2000], None, 1, 9216, 9216, 200), ([3, 1700, 2], [0, -1, 1], 2, 10240, 2056, 64),
                                                  ([5, 3] * 150, [k * 7 % 201 - 1 for k in range(300)], 200, 136, 264, 16)])
def test_large_adapters_of_whole_numbers_are_exact(dev, counts, index, n, o, i, q, dtype):
    """As above, against 64-bit products on the GPU: sizes that no cache holds, and more segments and adapters than a
    wavefront has lanes.  Values up to 1 (few of them not 0), so that hidden and the sums stay exact."""
    print(f"large {counts[:4]} {n} {o}x{i} {q} {dtype}", flush=True)
    gen = torch.Generator(device=dev).manual_seed(o + i + q)
    rows, off = sum(counts), offsets_of(counts)

    def numbers(*shape):
        return (torch.randint(-1, 2, shape, generator=gen, device=dev) * torch.randint(0, 2, shape, generator=gen, device=dev)).double()

    x, dy, a, b = numbers(rows, i), numbers(rows, o), numbers(n, q, i), numbers(n, o, q)
    base, dbase = numbers(rows, o) * 9, numbers(rows, i) * 9
    c = Case(dev, dtype, x, dy, a, b, off, index, None, base, dbase)
    c.rows()
    c.weights()
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for r, e in segments(off, index, n):
        y, dx = base[r], dbase[r]
        h, dh = torch.zeros(2, r.stop - r.start, q, dtype=torch.float64, device=dev)
        if e >= 0:
            h, dh = x[r] @ a[e].t(), dy[r] @ b[e]
            y, dx = y + h @ b[e].t(), dx + dh @ a[e]
            da[e] += dh.t() @ x[r]
            db[e] += dy[r].t() @ h
        assert torch.equal(c.h[r], h.float()) and torch.equal(c.dh[r], dh.float())
        assert torch.equal(c.y[r], y.to(dtype)) and torch.equal(c.dx[r], dx.to(dtype))
    assert torch.equal(c.da, da.float()) and torch.equal(c.db, db.float())


@pytest.mark.parametrize("counts,o", [([1, 2], 8), ([40, 70], 8), ([40, 70], 72), ([130, 1], 1001), ([300, 5], 1096), ([1100, 900], 9224)])
@pytest.mark.parametrize("shift", [0, 1])
def test_rows_without_an_adapter_are_the_base_bit_by_bit(dev, counts, o, shift):
    """Also what is not finite there, whatever x holds; without a base zeros; in place nothing changes."""
    gen, r, q = rng_of(o), sum(counts) + 2, 16
    bits = torch.randint(-32768, 32768, (r, o), generator=gen).short()
    base = torch.zeros(r * o + shift, dtype=torch.int16, device=dev)[shift:].view(r, o).copy_(bits).view(BF16)
    x, a, b = torch.full((r, 24), float("nan"), dtype=BF16, device=dev), torch.ones(2, q, 24, dtype=BF16, device=dev), torch.ones(2, o, q, dtype=BF16, device=dev)
    where = {"offsets": offsets_of(counts).to(dev), "index": torch.full((2,), -1, dtype=torch.int32, device=dev)}
    mine = r - 2
    for given, want in ((base, bits), (None, torch.zeros_like(bits))):
        y, h = torch.full((r, o), 7.0, dtype=BF16, device=dev), torch.full((r, q), 7.0, device=dev)
        B.adapter_forward(x, a, b, h, y, base=given, **where)
        assert torch.equal(y[:mine].view(torch.int16).cpu(), want[:mine]) and not h[:mine].any()
        assert (y[mine:] == 7).all() and (h[mine:] == 7).all()
    B.adapter_forward(x, a, b, h, base, base=base, **where)
    assert torch.equal(base.view(torch.int16).cpu(), bits)


@pytest.mark.parametrize("shift", [1, 3, 4])
@pytest.mark.parametrize("q", [5, 16, 72])
def test_addresses_of_any_element_alignment(dev, shift, q):
    for o, i in ((72, 136), (33, 67)):
        ref, c = whole_case(dev, [5, 90, 1], [1, 0, 1], 2, o, i, q, BF16, shift)
        assert_exact(ref, c, BF16)


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_without_a_base_and_in_place(dev, dtype):
    args = (dev, [40, 3, 0, 70], [2, -1, 0, 1], 3, 264, 200, 24, dtype)
    ref, c = whole_case(*args, based=False)
    assert_exact(ref, c, dtype)
    assert not c.y[42:45].any() and not c.h[42:45].any()
    ref, c = whole_case(*args)
    live = slice(2, 115)
    c.y.copy_(c.base)
    c.dx.copy_(c.dbase)
    c.base, c.dbase = c.y, c.dx
    c.rows()
    assert torch.equal(c.y[live].cpu(), ref.y[live].to(dtype)) and torch.equal(c.dx[live].cpu(), ref.dx[live].to(dtype))


def test_one_segment_without_offsets_or_scales(dev):
    gen, r, o, i, q = rng_of(5), 37, 136, 72, 16
    x, dy, a, b = whole((r, i), gen), whole((r, o), gen), whole((3, q, i), gen, 1), whole((3, o, q), gen, 1)
    ref = Ref(x, dy, a, b, torch.tensor([0, r]), [2], None, None, None)
    c = Case(dev, BF16, x, dy, a, b, None, [2], None, None, None)
    assert_exact(ref, c, BF16)


def within(got, ref, mag, rel, dtype, small=0.0):
    half = 0.0 if dtype == FP32 else torch.finfo(dtype).eps / 2
    tiny = 0.0 if dtype == FP32 else torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    err = mag * rel + small
    bound = err + half * (ref.abs() + err) + ref.abs() * 2.0 ** -23 + tiny
    return ((got.double().cpu() - ref).abs() <= bound).all()


@pytest.mark.parametrize("size", [1.0, 1e4, 1e-5])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("counts,index,n,o,i,q", [([1] * 6, [0, 1, -1, 1, 0, 1], 2, 512, 1032, 16), ([200, 0, 33], None, 3, 264, 1000, 64),
                                                  ([9, 70], None, 2, 77, 203, 5), ([600], None, 1, 520, 768, 200)])
def test_adapters_of_random_values(dev, counts, index, n, o, i, q, dtype, size):
    """`size` is that of A: hidden beyond fp16's largest value, and below its smallest normal one."""
    gen, rows, off = rng_of(o, i, q), sum(counts), offsets_of(counts)
    x = torch.randn(rows, i, generator=gen).mul_(torch.randn(i, generator=gen).mul_(0.5).exp_()).to(dtype).double()
    dy = torch.randn(rows, o, generator=gen).to(dtype).double()
    a = (torch.randn(n, q, i, generator=gen) * (size * i ** -0.5)).to(dtype).double()
    b = (torch.randn(n, o, q, generator=gen) * (0.05 / max(size, 1.0))).to(dtype).double()
    scales = torch.rand(n, generator=gen).double().float() + 0.5
    base, dbase = (torch.randn(rows, k, generator=gen).to(dtype).double() for k in (o, i))
    ref = Ref(x, dy, a, b, off, index, scales, base, dbase)
    c = Case(dev, dtype, x, dy, a, b, off, index, scales, base, dbase)
    c.rows()
    c.weights()
    step = 2.0 ** -23
    split = (torch.finfo(dtype).eps / 2) ** 2 + (2.0 ** -36 * q if dtype == FP16 else 0)
    assert within(c.h, ref.h, ref.hmag, i * step, FP32) and within(c.dh, ref.dh, ref.dhmag, (o + 2) * step, FP32)
    wide = 2.0 ** -36 * ref.hmag.amax(-1, keepdim=True) * b.abs().sum(-1).amax() * 2
    assert within(c.y, ref.y, ref.ymag, split + (i + 2 * q + 4) * step, dtype, wide)
    wide = 2.0 ** -36 * ref.dhmag.amax(-1, keepdim=True) * a.abs().sum(1).amax() * 2
    assert within(c.dx, ref.dx, ref.dxmag, split + (o + 2 * q + 4) * step, dtype, wide)
    longest = max(counts) * len(counts)
    assert within(c.da, ref.da, ref.damag, (longest + o + 4) * step, FP32)
    assert within(c.db, ref.db, ref.dbmag, (longest + i + 4) * step, FP32)


def test_gradients_are_the_forwards_differences(dev):
    """f = <dy, y> is linear in x, A, B and base: with whole numbers its differences are exact."""
    gen, counts, index, n, o, i, q = rng_of(1), [6, 2, 11], [1, 0, 1], 2, 40, 56, 8
    rows, off = sum(counts), offsets_of(counts)
    x, dy, a, b = whole((rows, i), gen, 1), whole((rows, o), gen, 1), whole((n, q, i), gen, 1), whole((n, o, q), gen, 1)
    c = Case(dev, FP16, x, dy, a, b, off, index, None, None, None)
    c.rows()
    c.weights()

    def f():
        # whole numbers up to 2^11 are exact in fp16
        y, h = torch.empty_like(c.y), torch.empty_like(c.h)
        B.adapter_forward(c.x, c.a, c.b, h, y, **c.where)
        assert y.abs().max() <= 2048
        return (y.double() * c.dy.double()).sum().item()

    base = f()
    for t, grad, places in ((c.x, c.dx, ((0, 0), (7, 3), (18, 55))), (c.a, c.da, ((0, 0, 0), (1, 7, 55), (1, 2, 3))),
                            (c.b, c.db, ((0, 39, 7), (1, 0, 0), (1, 20, 5)))):
        for at in places:
            t[at] += 1
            assert f() - base == grad[at].item()
            t[at] -= 1


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("q", [5, 24])
def test_values_that_are_not_finite_stay_where_they_belong(dev, q, dtype):
    """A bad row of x, dy or base reaches its own row, a bad adapter its own rows."""
    gen, counts, n, o, i = rng_of(q), [20, 1, 70], 3, 72, 136
    rows, off = sum(counts), offsets_of(counts)
    x, dy, a, b = whole((rows, i), gen), whole((rows, o), gen), whole((n, q, i), gen, 1), whole((n, o, q), gen, 1)
    base = whole((rows, o), gen)
    a[1, q - 1, 3], b[1, 5, 0] = float("inf"), float("nan")
    x[19, i - 1], x[30, 0], dy[19, 0], base[50, 7] = float("nan"), float("inf"), float("inf"), float("nan")
    x[20] = 1.0
    ref = Ref(x, dy, a, b, off, None, None, base, None)
    c = Case(dev, dtype, x, dy, a, b, off, None, None, base, None)
    c.rows()
    c.weights()
    for got, want in ((c.y, ref.y), (c.dx, ref.dx)):
        got = got.cpu()
        bad = ~torch.isfinite(want)
        # a row that is not finite need not be so at the same places: infinities may meet as NaN
        row = bad.any(-1)
        assert torch.equal(~torch.isfinite(got).all(-1), row)
        assert torch.equal(got[~row], want[~row].to(dtype))
    assert torch.equal(~torch.isfinite(c.y.cpu()[50]), torch.arange(o) == 7)
    for got, want in ((c.da, ref.da), (c.db, ref.db)):
        assert torch.equal(torch.isfinite(got.cpu()), torch.isfinite(want))
        assert torch.equal(got.cpu()[2][torch.isfinite(want[2])], want[2][torch.isfinite(want[2])].float())


@pytest.mark.parametrize("rows,q", [(1, 8), (5, 200), (70, 8), (70, 40), (70, 200)])
def test_hidden_between_the_largest_of_16_bits_and_of_32(dev, rows, q):
    """hidden = +-2^127 (2 - 2^-9) is finite, but rounded to bf16 it would not be.  Its two parts are exact, and so are y and
    dx: +-255.75 before the base."""
    n = 24
    x = torch.zeros(rows, n, dtype=torch.float64)
    x[::2, :2], x[1::2, :2] = 1.0, -1.0
    a = torch.zeros(1, q, n, dtype=torch.float64)
    a[0, q - 1, 0], a[0, q - 1, 1] = 2.0 ** 127 * (2 - 2.0 ** -7), 1.5 * 2.0 ** 119
    b = torch.zeros(1, n, q, dtype=torch.float64)
    b[0, 3, q - 1], b[0, 5, q - 1] = 2.0 ** -120, -(2.0 ** -121)
    base = torch.full((rows, n), 7.0).double()
    base[::2, 3], base[1::2, 3] = -256.0, 256.0
    args = (torch.tensor([0, rows]), None, None, base, base)
    ref = Ref(x, x, a, b, *args)
    c = Case(dev, BF16, x, x, a, b, *args)
    B.adapter_forward(c.x, c.a, c.b, c.h, c.y, base=c.base, **c.where)
    assert torch.equal(c.h.cpu(), ref.h.float()) and c.h.abs().amax() == 2.0 ** 127 * (2 - 2.0 ** -9)
    assert torch.equal(c.y.cpu(), ref.y.to(BF16)) and (ref.y[:, 3].abs() == 0.25).all()
    # the other way round: B has the large values, A the small ones
    bt, at = a.transpose(1, 2).contiguous(), b.transpose(1, 2).contiguous()
    ref = Ref(x, x, at, bt, *args)
    c = Case(dev, BF16, x, x, at, bt, *args)
    B.adapter_input_grad(c.dy, c.a, c.b, c.dh, c.dx, base=c.dbase, **c.where)
    assert torch.equal(c.dh.cpu(), ref.dh.float()) and torch.equal(c.dx.cpu(), ref.dx.to(BF16))


def test_wrong_offsets_and_indexes_touch_nothing_outside(dev):
    gen, o, i, q, r = rng_of(8), 24, 40, 8, 20
    x, dy, a, b = whole((r, i), gen), whole((r, o), gen), whole((2, q, i), gen, 1), whole((2, o, q), gen, 1)
    for off, index in (([-5, 4, 3, 99], [0, 1, 0]), ([1 << 40, -(1 << 62), 1 << 62, 7], [0, 0, 1]),
                       ([0, 5, 10, 20], [2, -(1 << 31), (1 << 31) - 1])):
        c = Case(dev, BF16, x, dy, a, b, torch.tensor(off), index, None, None, None)
        pools = [torch.full((r + 2, w), 7.0, dtype=d, device=dev) for w, d in ((o, BF16), (i, BF16), (q, FP32), (q, FP32))]
        c.y, c.dx, c.h, c.dh = (p[1:-1] for p in pools)
        c.rows()
        c.h.fill_(1)
        c.dh.fill_(1)
        c.weights()
        for p in pools:
            assert (p[0] == 7).all() and (p[-1] == 7).all()
    assert not c.da.any() and not c.db.any() and not c.y.any()


def test_no_rows(dev):
    a, b = torch.ones(2, 4, 16, dtype=BF16, device=dev), torch.ones(2, 24, 4, dtype=BF16, device=dev)
    x, y, h = torch.empty(0, 16, dtype=BF16, device=dev), torch.empty(0, 24, dtype=BF16, device=dev), torch.empty(0, 4, device=dev)
    off = torch.zeros(3, dtype=torch.int64, device=dev)
    B.adapter_forward(x, a, b, h, y, offsets=off)
    B.adapter_input_grad(y, a, b, h, x, offsets=off)
    da, db = torch.ones(2, 4, 16, device=dev), torch.ones(2, 24, 4, device=dev)
    B.adapter_weight_grad(y, x, h, h, da, db, offsets=off, accumulate=True)
    assert (da == 1).all() and (db == 1).all()
    B.adapter_weight_grad(y, x, h, h, da, db, offsets=off)
    assert not da.any() and not db.any()


def test_offsets_beyond_32_bits(dev):
    """Rows whose elements lie past 2^31; only the last ones are used."""
    gen, i, o, q, rows = rng_of(3), 1024, 1032, 8, (1 << 21) + 40
    x, dy = torch.zeros(rows, i, dtype=BF16, device=dev), torch.zeros(rows, o, dtype=BF16, device=dev)
    tx, tdy, a, b = whole((5, i), gen), whole((5, o), gen), whole((1, q, i), gen, 1), whole((1, o, q), gen, 1)
    live = slice(rows - 6, rows - 1)
    x[live], dy[live] = tx.to(BF16).to(dev), tdy.to(BF16).to(dev)
    ref = Ref(tx, tdy, a, b, torch.tensor([0, 5]), None, None, None, None)
    ad, bd = a.to(BF16).to(dev), b.to(BF16).to(dev)
    off = torch.tensor([rows - 6, rows - 1], device=dev)
    h, dh = torch.full((rows, q), 7.0, device=dev), torch.full((rows, q), 7.0, device=dev)
    out = torch.full((rows, o), 7.0, dtype=BF16, device=dev)
    B.adapter_forward(x, ad, bd, h, out, offsets=off)
    assert torch.equal(out[live].cpu(), ref.y.to(BF16)) and (out[:rows - 6] == 7).all() and (out[rows - 1] == 7).all()
    out = out.view(-1)[:rows * i].view(rows, i).fill_(7)
    B.adapter_input_grad(dy, ad, bd, dh, out, offsets=off)
    assert torch.equal(out[live].cpu(), ref.dx.to(BF16)) and (out[:rows - 6] == 7).all() and (out[rows - 1] == 7).all()
    da, db = torch.empty(1, q, i, device=dev), torch.empty(1, o, q, device=dev)
    B.adapter_weight_grad(dy, x, h, dh, da, db, offsets=off)
    assert torch.equal(da.cpu(), ref.da.float()) and torch.equal(db.cpu(), ref.db.float())


def test_requests_beside_a_packed_layer(dev):
    """As they are used: a packed projection shared by all requests, its output the adapters' base in place; then the
    gradients beside that of the projection's dense copy.  Captured once and replayed for other rows, offsets and
    adapters with eager calls between, and on two streams at once."""
    gen, o, i, q, n, r, s = rng_of(12), 96, 256, 16, 3, 40, 6
    levels = (-1.5, -0.5, 0.5, 1.5)
    codes = torch.randint(0, 4, (1, o, i), generator=gen)
    sc = (torch.rand(1, o, i // 64, generator=gen) * 0.02).half()
    packed = torch.from_numpy(refpack.pack_plain(codes.numpy().astype("uint8"), sc.numpy(), 4, 64))
    lin = B.Linear(B.LayerConfig(o, i, levels, 64), packed.to(dev))
    wq = (sc.float().repeat_interleave(64, -1) * torch.tensor(levels)[codes]).to(BF16)
    a, b = (torch.randn(n, q, i, generator=gen) * 0.1).to(BF16), (torch.randn(n, o, q, generator=gen) * 0.1).to(BF16)
    scales = torch.tensor([2.0, 0.5, 1.0])
    ad, bd, sd, wd = a.to(dev), b.to(dev), scales.to(dev), wq.to(dev)
    x, dy = torch.zeros(r, i, dtype=BF16, device=dev), torch.zeros(r, o, dtype=BF16, device=dev)
    off, index = torch.zeros(s + 1, dtype=torch.int64, device=dev), torch.zeros(s, dtype=torch.int32, device=dev)
    where = {"offsets": off, "index": index, "scales": sd}

    def outputs():
        return {"y": torch.empty(r, o, dtype=BF16, device=dev), "h": torch.empty(r, q, device=dev),
                "dh": torch.empty(r, q, device=dev), "dx": torch.empty(r, i, dtype=BF16, device=dev),
                "da": torch.empty(n, q, i, device=dev), "db": torch.empty(n, o, q, device=dev)}

    def calls(t):
        lin.forward(x, t["y"])
        B.adapter_forward(x, ad, bd, t["h"], t["y"], base=t["y"], **where)
        B.grouped_input_grad(dy, wd, t["dx"])
        B.adapter_input_grad(dy, ad, bd, t["dh"], t["dx"], base=t["dx"], **where)
        B.adapter_weight_grad(dy, x, t["h"], t["dh"], t["da"], t["db"], **where)

    t = outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(t)
    half = torch.finfo(BF16).eps / 2
    for counts, ids in (([40, 0, 0, 0, 0, 0], [1, 0, 0, 0, 0, 0]), ([1, 2, 3, 4, 10, 20], [0, 1, 2, 2, -1, 0]),
                        ([0, 0, 20, 0, 20, 0], [0, 1, 2, 0, 1, 2])):
        xr, dyr = torch.randn(r, i, generator=gen).to(BF16), torch.randn(r, o, generator=gen).to(BF16)
        x.copy_(xr)
        dy.copy_(dyr)
        off.copy_(offsets_of(counts))
        index.copy_(torch.tensor(ids, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in t.items()}
        for v in t.values():
            v.fill_(3)
        calls(t)
        torch.cuda.synchronize()
        for k, v in t.items():
            assert torch.equal(got[k], v), k
        xd, dd, wq64 = xr.double(), dyr.double(), wq[0].double()
        ref = Ref(xd, dd, a.double(), b.double(), off.cpu(), ids, scales, xd @ wq64.t(), dd @ wq64)
        # the base is rounded to 16 bits, and the sum once more; sums in fp32 are far below
        mag = ref.ymag + xd.abs() @ wq64.abs().t()
        assert within(t["y"], ref.y, mag, half + (2 * i + 64) * 2.0 ** -23 + 2.0 ** -16, BF16)
        mag = ref.dxmag + dd.abs() @ wq64.abs()
        assert within(t["dx"], ref.dx, mag, half + (2 * o + 64) * 2.0 ** -23 + 2.0 ** -16, BF16)
        assert within(t["da"], ref.da, ref.damag, (r + o + 4) * 2.0 ** -23, FP32)
        assert within(t["db"], ref.db, ref.dbmag, (r + i + 4) * 2.0 ** -23, FP32)
    others, streams = [outputs() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for u, stream in zip(others, streams):
            with torch.cuda.stream(stream):
                calls(u)
    torch.cuda.synchronize()
    for u in others:
        for k, v in t.items():
            assert torch.equal(u[k], v), k


def test_rows_sorted_by_adapter(dev):
    """Rows that come in any order of adapters: group_rows' offsets and slots bring them together and back."""
    gen, r, o, i, q, n = rng_of(14), 50, 40, 72, 8, 4
    ids = torch.randint(-1, n, (r, 1), generator=gen, dtype=torch.int32)
    x, a, b = whole((r, i), gen), whole((n, q, i), gen, 1), whole((n, o, q), gen, 1)
    off, slots = torch.empty(n + 1, dtype=torch.int64, device=dev), torch.empty(r, 1, dtype=torch.int32, device=dev)
    B.group_rows(ids.to(dev), off, slots, torch.empty(r, dtype=torch.int32, device=dev))
    xs, ys = torch.zeros(r, i, dtype=BF16, device=dev), torch.zeros(r, o, dtype=BF16, device=dev)
    y = torch.empty(r, o, dtype=BF16, device=dev)
    B.dispatch_rows(x.to(BF16).to(dev), slots, xs)
    B.adapter_forward(xs, a.to(BF16).to(dev), b.to(BF16).to(dev), torch.empty(r, q, device=dev), ys, offsets=off)
    B.combine_rows(ys, slots, y)
    ref = torch.stack([b[e] @ (a[e] @ x[k]) if e >= 0 else torch.zeros(o).double() for k, e in enumerate(ids[:, 0])])
    assert torch.equal(y.cpu(), ref.to(BF16))
