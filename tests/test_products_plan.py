"""The rules that cut the products into tiles, compiled on their own with the host compiler: the plan of each
case that the GPU tests run to have a kernel tested."""
import os
import subprocess

import pytest

import product_cases as cases
from paper_2604_18556_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PLAN = r"""
#include "gsq_plan.h"
#include <cstdio>
#include <cstring>
int main() {
  char kind[32];
  long long r, g, o, i;
  int tight;
  while (std::scanf("%31s %lld %lld %lld %lld %d", kind, &r, &g, &o, &i, &tight) == 6) {
    const auto is = [&](const char* s) { return !std::strcmp(kind, s); };
    if (is("weight_grad") || is("gram")) {
      const gsq::SumsPlan p = gsq::plan_sums(r, g, is("gram") ? i : o, i, tight, is("gram"));
      std::printf("%s %d\n", p.split ? "split" : "ring", p.size);
      continue;
    }
    const int slabs = (int)gsq::tiles_of(is("input_grad") ? o : i, is("int8") ? 128 : 64);
    const gsq::RowsPlan p = is("packed") ? gsq::plan_packed(r, g, o, (int)gsq::tiles_of(i, 128), tight)
                                         : gsq::plan_rows(r, g, is("input_grad") ? i : o, slabs, tight,
                                                          is("input_grad"), is("int8"));
    std::printf("%s %dx%d\n", p.split ? "split" : "ring", p.height, p.width);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """(kind, rows, groups, O, I, tight) of many products to their plans."""
    folder = tmp_path_factory.mktemp("plan")
    src, exe = folder / "plan.cpp", folder / "plan"
    src.write_text(PLAN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2604_18556_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True, capture_output=True, text=True)

    def ask(products):
        text = "".join(" ".join(str(int(v) if isinstance(v, bool) else v) for v in p) + "\n" for p in products)
        return subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
    return ask


def test_plans_of_the_tested_cases(plans):
    listed = [(c[0], sum(c[1]), len(c[1]), c[2], c[3], cases.tight(c[0], *c[2:5])) for c in cases.ROWS + cases.SUMS]
    listed += [("packed", sum(c[3]), len(c[3]), c[4], c[5], c[6] == 0) for c in cases.PACKED]
    want = [c[-1] for c in cases.ROWS + cases.SUMS + cases.PACKED]
    got = plans(listed)
    wrong = [(p, g, w) for p, g, w in zip(listed, got, want) if g != w]
    assert len(got) == len(want) and not wrong


def test_every_large_tile_has_a_case():
    rows = {(c[0], c[-1]) for c in cases.ROWS}
    for kind in ("forward", "input_grad", "int8"):
        for plan in ("ring 256x256", "ring 128x256", "ring 64x256", "ring 128x128"):
            assert (kind, plan) in rows, (kind, plan)
    sums = {(c[0], c[-1], cases.tight(c[0], *c[2:5])) for c in cases.SUMS}
    for kind in ("weight_grad", "gram"):
        assert {(kind, "ring 256", True), (kind, "ring 128", True), (kind, "ring 128", False)} <= sums
    bits = {2: 1, 3: 2, 4: 2, 8: 3, 16: 4}
    packed = {(3 if c[0] == "superblock" else bits[len(c[1])], c[0] == "superblock" or c[2] == 16) for c in cases.PACKED}
    assert packed == {(b, fine) for b in (1, 2, 3, 4) for fine in (False, True)}
    for b in (2, 3, 4):
        assert {c[-1] for c in cases.PACKED if bits[len(c[1])] == b} >= {"ring 256x256", "ring 128x256", "ring 64x256"}
    odd = {(3 if c[0] == "superblock" else bits[len(c[1])], c[0] == "superblock" or c[2] == 16)
           for c in cases.PACKED if c[6] and c[-1] == "ring 128x256"}
    assert odd == packed


LIMITS = r"""
#include "gsq_plan.h"
#include <cstdio>
#include <random>
std::mt19937_64 gen(1);
int64_t draw(double bits) { return (int64_t)std::exp2(std::uniform_real_distribution<double>(0, bits)(gen)); }
int main() {
  long taken = 0, wrong = 0;
  const auto note = [&](const char* what, bool must, bool fits, int64_t r, int64_t g, int64_t o, int64_t i) {
    taken += must;
    if (must && !fits && ++wrong < 10)
      std::printf("%s rows %lld groups %lld O %lld I %lld\n", what, (long long)r, (long long)g, (long long)o, (long long)i);
  };
  for (int k = 0; k < 400000; ++k) {
    const int64_t r = draw(29.01), g = k & 1 ? 1 : draw(16), o = draw(21.01), i = draw(21.01);
    const bool tight = gen() & 1, flag = gen() & 1, bytes = gen() & 1;
    using namespace gsq;
    const auto rows_fit = [&](const RowsPlan& p, int waves) {
      return p.height && fits_launch(most_panels(r, g, p.height) * tiles_of(o, p.width), 64 * (p.split ? waves : 4));
    };
    const bool must = (r / 64 + std::min(r, g)) * tiles_of(o, 64) < (int64_t)1 << 23;
    const int slabs = (int)tiles_of(i, bytes ? 128 : 64), blocks = (int)tiles_of(i, 128);
    note("rows", must, rows_fit(plan_rows(r, g, o, slabs, tight, flag && !bytes, bytes), std::min(slabs, 8)), r, g, o, i);
    const RowsPlan p = plan_packed(r, g, o, blocks, tight);
    note("packed", must, rows_fit(p, std::min(blocks, p.height == 16 ? 16 : 8)), r, g, o, i);
    const SumsPlan s = plan_sums(r, g, flag ? i : o, i, tight, flag);
    note("sums", g * tiles_of(flag ? i : o, 64) * tiles_of(i, 64) < (int64_t)1 << 23,
         fits_launch(sum_tiles(g, flag ? i : o, i, flag, s.size), 64 * s.waves), r, g, o, i);
  }
  std::printf("%ld %ld\n", taken, wrong);
}
"""


def test_products_below_the_stated_limit_fit_a_launch(tmp_path):
    """The header's bound on the tiles, over sizes up to its limits: what is below it has a plan that one launch
    holds."""
    src, exe = tmp_path / "limits.cpp", tmp_path / "limits"
    src.write_text(LIMITS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2604_18556_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True, capture_output=True, text=True)
    *faults, last = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()
    taken, wrong = map(int, last.split())
    assert taken > 100000 and wrong == 0, faults


BLOCKS = r"""
#include "gsq_plan.h"
#include <cstdio>
#include <cstdlib>
int main(int argc, char** argv) {
  for (int k = 1; k < argc; ++k) {
    const unsigned b = gsq::unpack_blocks(std::atoll(argv[k]));
    std::printf("%u %d\n", b, b > 0 && gsq::fits_launch(b, 256));
  }
}
"""


def test_packed_layers_of_any_size_are_laid_out_by_one_launch(tmp_path):
    """Elements that gsq_linear_init lays out, from one channel to its largest layer: two for each 32 weights."""
    src, exe = tmp_path / "blocks.cpp", tmp_path / "blocks"
    src.write_text(BLOCKS)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_18556_amd", "csrc"), str(src), "-o",
                    str(exe)], check=True, capture_output=True, text=True)
    counts = [16, 64, 256, 257, 16384 * 256, 16384 * 256 + 1, 1 << 32, 1 << 40, 65535 * (1 << 21) * (1 << 21) // 16]
    out = subprocess.run([str(exe), *map(str, counts)], check=True, capture_output=True, text=True).stdout.split()
    blocks, fits = list(map(int, out[::2])), list(map(int, out[1::2]))
    assert blocks == [1, 1, 1, 2] + [16384] * 5 and all(fits)


KEPT = r"""
#include "gsq_plan.h"
#include <cstdio>
int main() {
  long long b, o, i;
  int bits, gs, super;
  while (std::scanf("%lld %lld %lld %d %d %d", &b, &o, &i, &bits, &gs, &super) == 6) {
    const gsq::KeptBytes k = gsq::kept_bytes(b, o, i, bits, gs, super);
    std::printf("%lld\n", (long long)(k.codes + k.scales + k.sub));
  }
}
"""


def test_kept_bytes_of_a_packed_layer_are_as_the_header_says(tmp_path):
    """Never more than a quarter above the packed size of the layer rounded up to whole units of 16 x 128."""
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libgsq.so not built (run __graft_entry__.build())")
    src, exe = tmp_path / "kept.cpp", tmp_path / "kept"
    src.write_text(KEPT)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_18556_amd", "csrc"), str(src), "-o",
                    str(exe)], check=True, capture_output=True, text=True)
    layers = []
    for batch, o, units in ((1, 1, 1), (1, 5, 3), (3, 16, 1), (2, 17, 32), (1, 4096, 16), (64, 2048, 28)):
        layers += [(B.LAYOUT_SUPERBLOCK, cases.L8, 3, 16, batch, o, 256 * units)]
        for gs in (16, 32, 64, 128, 256):
            layers += [(B.LAYOUT_BASE3, cases.L3, 2, gs, batch, o, gs * units)]
            layers += [(B.LAYOUT_GROUP, levels, bits, gs, batch, o, gs * units)
                       for levels, bits in ((cases.L2, 1), (cases.L4, 2), (cases.L8, 3), (cases.L16, 4))]
    text = "".join(f"{b} {o} {i} {bits} {256 if lay == B.LAYOUT_SUPERBLOCK else gs} {int(lay == B.LAYOUT_SUPERBLOCK)}\n"
                   for lay, _, bits, gs, b, o, i in layers)
    kept = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout.split()
    worst = 0
    for (lay, levels, bits, gs, b, o, i), bytes_ in zip(layers, map(int, kept), strict=True):
        whole = B.packed_size(B.LayerConfig(-(-o // 16) * 16, -(-i // 128) * 128, levels, gs, b, lay,
                                            relaxation=B.RELAX_SHIFT if bits == 4 else B.RELAX_GRID))
        assert whole <= bytes_ <= 1.25 * whole, (lay, bits, gs, b, o, i)
        worst = max(worst, bytes_ / B.packed_size(B.LayerConfig(o, i, levels, gs, b, lay, relaxation=B.RELAX_SHIFT)))
    assert worst > 8                               # the layer's own size is no bound
