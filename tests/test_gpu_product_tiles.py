"""The products' large tiles, each at sizes where the rules choose it (product_cases.py).

Inputs are small whole numbers, and the packed weights have powers of two as scales, so that every product and sum
is exact in fp32: the outputs must be the 64-bit reference's, rounded once, bit for bit.
"""
import numpy as np
import pytest

from oracle import pack as refpack
from paper_2604_18556_amd import binding as B

import product_cases as cases

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
DTYPES = pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
FIRST, BEHIND = 5, 9         # rows before the first group and behind the last


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load()
    return torch.device("cuda:0")


def generator(dev, *seed):
    return torch.Generator(device=dev).manual_seed(sum(17 ** k * v for k, v in enumerate(seed)))


def numbers(gen, *shape, top=1):
    return torch.randint(-top, top + 1, shape, generator=gen, device=gen.device, dtype=torch.int8)


def moved(t, shift):
    """A copy of t that begins `shift` elements past an aligned address."""
    m = torch.zeros(t.numel() + shift, dtype=t.dtype, device=t.device)[shift:].view(t.shape)
    return m.copy_(t)


def offsets_of(counts, dev):
    return torch.tensor([FIRST] + list(counts)).cumsum(0).to(dev)


def groups_of(counts):
    ends = np.cumsum([FIRST] + list(counts)).tolist()
    return list(zip(ends, ends[1:]))


@DTYPES
@pytest.mark.parametrize("case", cases.ROWS, ids=cases.label)
def test_rows(dev, case, dtype):
    kind, counts, o, i, shift, _ = case
    print(f"rows {case} {dtype}", flush=True)
    gen, e, rows = generator(dev, o, i, sum(counts)), len(counts), FIRST + sum(counts) + BEHIND
    ks, ns = (o, i) if kind == "input_grad" else (i, o)
    # sums of whole numbers stay below 2^11, which fp16 holds exactly, but are rounded in bf16
    a, w = numbers(gen, rows, ks, top=2), numbers(gen, e, o, i, top=2)
    out = torch.full((rows, ns), 7.0, dtype=dtype, device=dev)
    off = offsets_of(counts, dev)
    if kind == "int8":
        ones = torch.ones(max(rows, e * o), device=dev)
        B.grouped_forward_i8(moved(a, shift), ones[:rows], moved(w, shift), ones[:e * o].view(e, o), out, offsets=off)
    else:
        call = B.grouped_forward if kind == "forward" else B.grouped_input_grad
        call(moved(a.to(dtype), shift), moved(w.to(dtype), shift), out, offsets=off)
    for k, (first, end) in enumerate(groups_of(counts)):
        we = w[k].double() if kind == "input_grad" else w[k].double().t()
        assert torch.equal(out[first:end], (a[first:end].double() @ we).to(dtype)), k
    assert (out[:FIRST] == 7).all() and (out[rows - BEHIND:] == 7).all()


@DTYPES
@pytest.mark.parametrize("case", cases.SUMS, ids=cases.label)
def test_sums(dev, case, dtype):
    """dW in both types and H, and both added to what is there."""
    kind, counts, o, i, shift, _ = case
    print(f"sums {case} {dtype}", flush=True)
    gen, e, rows = generator(dev, o, i, sum(counts)), len(counts), FIRST + sum(counts) + BEHIND
    x, off = numbers(gen, rows, i), offsets_of(counts, dev)
    xd = moved(x.to(dtype), shift)
    if kind == "gram":
        y, yd, ends = x, xd, (FP32,)
    else:
        y, ends = numbers(gen, rows, o), (dtype, FP32)
        yd = moved(y.to(dtype), shift)

    def call(out, **how):
        if kind == "gram":
            B.gram(xd, out, offsets=off, **how)
        else:
            B.grouped_weight_grad(yd, xd, out, offsets=off, **how)

    for end in ends:
        out = torch.full((e, y.shape[1], i), 7.0, dtype=end, device=dev)
        call(out)
        refs = [y[a:b].double().t() @ x[a:b].double() for a, b in groups_of(counts)]
        for k, ref in enumerate(refs):
            assert torch.equal(out[k], ref.to(end)), k
    out.fill_(3.0)
    call(out, accumulate=True)
    for k, ref in enumerate(refs):
        assert torch.equal(out[k], (ref + 3).float()), k


def packed_layer(layout, levels, group, batch, o, i, gen):
    """Random codes, scales that are powers of two, their packed bytes (by the oracle), and the weights."""
    codes = torch.randint(0, len(levels), (batch, o, i), generator=gen, dtype=torch.uint8)
    c = codes.numpy()
    power = lambda lo, hi, *shape: 2.0 ** torch.randint(lo, hi + 1, shape, generator=gen).float()
    if layout == "superblock":
        d, sc = power(-4, -3, batch, o, i // 256), power(0, 3, batch, o, i // 16)
        eff = d.repeat_interleave(16, -1) * sc
        packed = refpack.pack_superblock(c, d.half().numpy(), sc.numpy().astype(np.uint8))
    else:
        eff = power(-4, -1, batch, o, i // group)
        s = eff.half().numpy()
        packed = refpack.pack_base3(c, s) if layout == "base3" else refpack.pack_plain(c, s, len(levels), group)
    w = torch.tensor(levels)[codes.int()]
    w.view(batch, o, i // group, group).mul_(eff[..., None])
    return torch.from_numpy(np.ascontiguousarray(packed)), w


@pytest.mark.parametrize("case", cases.PACKED, ids=cases.label)
def test_packed(dev, case):
    """One handle for rows of both types."""
    layout, levels, group, counts, o, i, shift, _ = case
    print(f"packed {case}", flush=True)
    e, rows = len(counts), FIRST + sum(counts) + BEHIND
    packed, w = packed_layer(layout, levels, group, e, o, i, generator("cpu", o, i, len(levels)))
    kept = {"group": B.LAYOUT_GROUP, "base3": B.LAYOUT_BASE3, "superblock": B.LAYOUT_SUPERBLOCK}[layout]
    lin = B.Linear(B.LayerConfig(o, i, levels, group, e, kept,
                                 relaxation=B.RELAX_SHIFT if len(levels) > 8 else B.RELAX_GRID), packed.to(dev))
    x, off, w = numbers(generator(dev, o, i, sum(counts)), rows, i, top=2), offsets_of(counts, dev), w.to(dev)
    for dtype in (BF16, FP16):
        y = torch.full((rows, o), 7.0, dtype=dtype, device=dev)
        lin.forward(moved(x.to(dtype), shift), y, offsets=off)
        for k, (a, b) in enumerate(groups_of(counts)):
            assert torch.equal(y[a:b], (x[a:b].double() @ w[k].double().t()).to(dtype)), (dtype, k)
        assert (y[:FIRST] == 7).all() and (y[rows - BEHIND:] == 7).all()
    lin.destroy()


def test_packed_rows_beyond_small_tiles(dev):
    """2^30 results of an x that begins at an odd element: as many 16 x 16 tiles would pass a launch."""
    rows, o, i = 1 << 16, 1 << 14, 2048
    levels = (-1.5, -0.5, 0.5, 1.5)
    cfg = B.LayerConfig(o, i, levels, 256)
    packed = torch.randint(0, 256, (B.packed_size(cfg),), generator=generator(dev, 3), device=dev, dtype=torch.uint8)
    packed[-2 * o * i // 256:] = torch.ones(o * i // 256, dtype=FP16, device=dev).view(torch.uint8)
    lin = B.Linear(cfg, packed)
    x = numbers(generator(dev, 4), rows, i).to(BF16)
    want, got = torch.empty(rows, o, dtype=BF16, device=dev), torch.empty(rows, o, dtype=BF16, device=dev)
    lin.forward(x, want)
    lin.forward(moved(x, 1), got)
    assert torch.equal(got, want)
    code = packed[:o * i // 4].view(o, i // 4, 1) >> torch.tensor([0, 2, 4, 6], dtype=torch.uint8, device=dev) & 3
    w = torch.tensor(levels, device=dev)[code.int()].view(o, i)
    for r in (0, 1, 777, rows - 2, rows - 1):
        assert torch.equal(got[r], (w.double() @ x[r].double()).to(BF16))
    lin.destroy()


def fields(data, width, count):
    """`count` little-endian fields of `width` bits in the bytes of the last dimension."""
    word = torch.zeros(data.shape[:-1], dtype=torch.int64, device=data.device)
    for k in range(data.shape[-1]):
        word |= data[..., k].long() << (8 * k)
    return word[..., None] >> torch.arange(count, device=data.device) * width & (1 << width) - 1


@pytest.mark.parametrize("layout,levels,group,i", [("group", L, g, i) for L, g, i in ((cases.L2, 64, 8192), (cases.L4, 16, 4096))]
                         + [("superblock", cases.L8, 16, 4096)])
def test_large_packed_layers_are_laid_out_whole(dev, layout, levels, group, i):
    """More codes, scales or sub-scales than threads lay out: the last layer's weights as much as the first's."""
    e, o = 5, 4096
    super_block = layout == "superblock"
    cfg = B.LayerConfig(o, i, levels, group, e, B.LAYOUT_SUPERBLOCK if super_block else B.LAYOUT_GROUP)
    assert e * o * i // 32 * (1 if len(levels) == 2 else 2) > 16384 * 256
    packed = torch.randint(0, 256, (B.packed_size(cfg),), generator=generator(dev, i, group), device=dev, dtype=torch.uint8)
    power = lambda n: (2.0 ** torch.randint(-4, 0, (n, 1), generator=generator(dev, 7), device=dev)).half().view(torch.uint8)
    if super_block:
        rec = packed.view(-1, 110)
        rec[:, :2] = power(rec.shape[0])
        rec = rec.view(e, -1, 110)
    else:
        width = 1 if len(levels) == 2 else 2
        codes, scales = packed[:e * o * i * width // 8].view(e, -1, width), packed[e * o * i * width // 8:]
        scales.copy_(power(e * o * i // group).view(-1))
        scales = scales.view(torch.float16).view(e, -1)
    lin = B.Linear(cfg, packed)
    x = numbers(generator(dev, 5), 2 * e, i).to(BF16)
    y = torch.empty(2 * e, o, dtype=BF16, device=dev)
    lin.forward(x, y, offsets=torch.arange(0, 2 * e + 1, 2, device=dev))
    for k in (0, e - 1):
        if super_block:
            s = rec[k, :, :2].contiguous().view(torch.float16).float() * fields(rec[k, :, 2:14].view(-1, 4, 3), 6, 4).view(-1, 16)
            c = fields(rec[k, :, 14:].view(-1, 32, 3), 3, 8)
        else:
            s, c = scales[k].float(), fields(codes[k], width, 8)
        w = torch.tensor(levels, device=dev)[c.view(-1, group)] * s.view(-1, 1)
        w = w.to(BF16).double().view(o, i)
        assert torch.equal(y[2 * k:2 * k + 2], (x[2 * k:2 * k + 2].double() @ w.t()).to(BF16)), k
    lin.destroy()
