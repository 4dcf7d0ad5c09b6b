"""What the products refuse, and in what words, before anything reaches the device."""
import ctypes
import os
import re
import subprocess
from types import SimpleNamespace

import pytest

from paper_2604_18556_amd import binding as B

torch = pytest.importorskip("torch")
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libgsq.so not built (run __graft_entry__.build())")
    return B.load()


def sizes(groups=2, out=8, inn=16, dtype=B.DT_BF16, rows=4):
    return B.CGrouped(groups, out, inn, dtype, rows)


BAD_SIZES = [dict(groups=0), dict(groups=65536), dict(out=0), dict(out=(1 << 21) + 1), dict(inn=0),
             dict(inn=(1 << 21) + 1), dict(dtype=B.DT_FP32), dict(dtype=9), dict(rows=-1),
             dict(rows=(1 << 29) + 1)]


@pytest.mark.parametrize("bad", BAD_SIZES)
def test_sizes_are_checked(lib, bad):
    g, a = ctypes.byref(sizes(**bad)), P(64)
    calls = [lambda: lib.gsq_grouped_forward(g, a, a, a, a, None),
             lambda: lib.gsq_grouped_input_grad(g, a, a, a, a, None),
             lambda: lib.gsq_grouped_weight_grad(g, a, a, a, a, B.DT_FP32, 0, None),
             lambda: lib.gsq_grouped_forward_i8(g, a, a, a, a, a, a, None)]
    if "out" not in bad:                       # the Gram matrix has no output features
        calls.append(lambda: lib.gsq_gram(g, a, a, a, 0, None))
    for call in calls:
        assert call() == B.GSQ_EINVAL
        assert lib.gsq_last_error()


def test_arrays_are_checked(lib):
    g, a, no, odd = ctypes.byref(sizes()), P(64), None, P(65)
    E = B.GSQ_EINVAL
    assert lib.gsq_grouped_forward(None, a, a, a, a, None) == E
    for bad in (no, odd):
        assert lib.gsq_grouped_forward(g, bad, a, a, a, None) == E
        assert lib.gsq_grouped_forward(g, a, bad, a, a, None) == E
        assert lib.gsq_grouped_forward(g, a, a, bad, a, None) == E      # two groups need offsets
        assert lib.gsq_grouped_forward(g, a, a, a, bad, None) == E
        assert lib.gsq_grouped_input_grad(g, bad, a, a, a, None) == E
        assert lib.gsq_grouped_input_grad(g, a, bad, a, a, None) == E
        assert lib.gsq_grouped_input_grad(g, a, a, a, bad, None) == E
        assert lib.gsq_grouped_weight_grad(g, bad, a, a, a, B.DT_BF16, 0, None) == E
        assert lib.gsq_grouped_weight_grad(g, a, bad, a, a, B.DT_BF16, 0, None) == E
        assert lib.gsq_grouped_weight_grad(g, a, a, a, bad, B.DT_BF16, 0, None) == E
        assert lib.gsq_gram(g, bad, a, a, 0, None) == E
        assert lib.gsq_gram(g, a, a, bad, 0, None) == E
        assert lib.gsq_grouped_forward_i8(g, a, bad, a, a, a, a, None) == E
        assert lib.gsq_grouped_forward_i8(g, a, a, a, bad, a, a, None) == E
        assert lib.gsq_grouped_forward_i8(g, a, a, a, a, a, bad, None) == E
        assert lib.gsq_quantize_rows(bad, B.DT_BF16, 1, 8, a, a, None) == E
        assert lib.gsq_quantize_rows(a, B.DT_BF16, 1, 8, a, bad, None) == E
    assert lib.gsq_gram(g, a, a, P(66), 0, None) == E                    # fp32 needs 4 bytes
    assert lib.gsq_grouped_weight_grad(g, a, a, a, P(66), B.DT_FP32, 0, None) == E
    assert lib.gsq_grouped_forward_i8(g, None, a, a, a, a, a, None) == E
    assert lib.gsq_quantize_rows(a, B.DT_BF16, 1, 8, None, a, None) == E


def test_weight_grad_types(lib):
    g, a = ctypes.byref(sizes()), P(64)
    assert lib.gsq_grouped_weight_grad(g, a, a, a, a, B.DT_FP16, 0, None) == B.GSQ_EINVAL
    assert lib.gsq_grouped_weight_grad(g, a, a, a, a, B.DT_BF16, 1, None) == B.GSQ_EINVAL
    assert b"FP32" in lib.gsq_last_error()


def test_integer_sums_stay_exact(lib):
    a = P(64)
    assert lib.gsq_grouped_forward_i8(ctypes.byref(sizes(inn=131072)), a, a, a, a, a, a, None) == B.GSQ_EINVAL
    assert b"131071" in lib.gsq_last_error()
    assert 128 * 128 * 131071 < 2 ** 31


def test_quantize_sizes(lib):
    a = P(64)
    for dtype, rows, cols in ((7, 1, 8), (0, -1, 8), (0, (1 << 23) + 1, 8), (0, 1, 0), (0, 1, (1 << 21) + 1)):
        assert lib.gsq_quantize_rows(a, dtype, rows, cols, a, a, None) == B.GSQ_EINVAL


def test_no_rows_need_no_arrays(lib):
    """A batch without a row is no error, whatever its row arrays' addresses are."""
    g, a = ctypes.byref(sizes(groups=1, rows=0)), P(64)
    assert lib.gsq_grouped_forward(g, None, a, None, None, None) == B.GSQ_OK
    assert lib.gsq_grouped_input_grad(g, None, a, None, None, None) == B.GSQ_OK
    assert lib.gsq_grouped_forward_i8(g, None, None, a, a, None, None, None) == B.GSQ_OK
    assert lib.gsq_quantize_rows(None, B.DT_BF16, 0, 8, None, None, None) == B.GSQ_OK


def test_products_of_more_tiles_than_a_launch_holds(lib):
    """The grid is checked before anything is enqueued."""
    g, a = ctypes.byref(sizes(groups=1, out=1 << 21, inn=64, rows=1 << 29)), P(64)
    for st in (lib.gsq_grouped_forward(g, a, a, None, a, None),
               lib.gsq_grouped_forward_i8(g, a, a, a, a, None, a, None),
               lib.gsq_grouped_weight_grad(ctypes.byref(sizes(groups=65535, out=1 << 21, inn=1 << 21)), a, a, a, a,
                                           B.DT_FP32, 0, None)):
        assert st == B.GSQ_EINVAL
        assert b"tiles" in lib.gsq_last_error()


def test_header_and_library_have_the_same_calls(lib):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "gsq_products.h")).read()
    assert set(re.findall(r"^gsq_status\s+(gsq_\w+)\s*\(", text, re.M)) == set(B.PRODUCT_EXPORTS)
    for name in B.PRODUCT_EXPORTS:
        assert getattr(lib, name) is not None


def test_header_is_plain_c(tmp_path):
    """The header compiles as C, and its struct is the binding's."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gsq_products.h"\n'
                   'int main(void) { printf("%zu %zu %d", sizeof(gsq_grouped), offsetof(gsq_grouped, rows), '
                   'GSQ_DT_FP16); return 0; }\n')
    r = subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I",
                        "/opt/rocm/include", str(src), "-o", str(tmp_path / "layout")], capture_output=True, text=True)
    if r.returncode:
        pytest.skip("cannot compile against hip_runtime_api.h: " + r.stderr[-300:])
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [ctypes.sizeof(B.CGrouped), B.CGrouped.rows.offset, B.DT_FP16]


def test_linear_refusals(lib):
    h = P()
    cfg = B.LayerConfig(8, 256, (-1.0, 0.0, 1.0))
    need = B.packed_size(cfg)
    c = cfg.to_c()
    E = B.GSQ_EINVAL
    assert lib.gsq_linear_init(None, P(64), need, None, ctypes.byref(h)) == E
    assert lib.gsq_linear_init(ctypes.byref(c), None, need, None, ctypes.byref(h)) == E
    assert lib.gsq_linear_init(ctypes.byref(c), P(64), need - 1, None, ctypes.byref(h)) == E
    assert lib.gsq_linear_init(ctypes.byref(c), P(64), need, None, None) == E
    bad = B.LayerConfig(8, 200, (-1.0, 0.0, 1.0)).to_c()
    assert lib.gsq_linear_init(ctypes.byref(bad), P(64), need, None, ctypes.byref(h)) == E
    for big in (B.LayerConfig((1 << 21) + 1, 16, (-1.0, 1.0), 16),
                B.LayerConfig(1, (1 << 21) + 16, (-1.0, 1.0), 16),
                B.LayerConfig(1, 16, (-1.0, 1.0), 16, batch=65536)):
        b = big.to_c()
        assert lib.gsq_linear_init(ctypes.byref(b), P(64), 1 << 40, None, ctypes.byref(h)) == E
    assert h.value is None
    assert lib.gsq_linear_forward(None, P(64), B.DT_BF16, 1, None, P(64), None) == E
    assert lib.gsq_linear_destroy(None) == B.GSQ_OK


def test_c_struct_layout():
    assert ctypes.sizeof(B.CGrouped) == 24 and B.CGrouped.rows.offset == 16


def test_binding_checks_tensors_before_the_library():
    """Host tensors, wrong shapes and wrong types raise before a pointer is passed on."""
    x, w, y = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(2, 4, 8, dtype=torch.bfloat16), \
        torch.zeros(3, 4, dtype=torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="device tensor"):
        B.grouped_forward(x, w, y, offsets=off)
    with pytest.raises(ValueError, match="need offsets"):
        B.grouped_forward(x, w, y)
    with pytest.raises(ValueError, match="shape"):
        B.grouped_forward(x[:, :4], w, y, offsets=off)
    with pytest.raises(ValueError, match="shape"):
        B.grouped_forward(x, w, y, offsets=off[:2])
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        B.grouped_forward(x.float(), w.float(), y.float(), offsets=off)
    with pytest.raises(ValueError, match="square"):
        B.gram(x, torch.zeros(4, 8))
    with pytest.raises(ValueError, match="rows x features"):
        B.gram(x[0], torch.zeros(8, 8))
    with pytest.raises(ValueError, match="groups x O x I"):
        B.grouped_input_grad(y, w[0, 0], x)
    with pytest.raises(ValueError, match="shape"):
        B.quantize_rows(x, torch.zeros(3, 7, dtype=torch.int8), torch.zeros(3))
    with pytest.raises(ValueError, match="device tensor"):
        B.Linear(B.LayerConfig(4, 16, (-1.0, 1.0), 16), torch.zeros(64, dtype=torch.uint8))


BIG = (1 << 32) + 8          # 8 in its low 32 bits


@pytest.mark.parametrize("call", [
    lambda t: B.grouped_forward(t(1, BIG), t(8, BIG), t(1, 8)),
    lambda t: B.grouped_forward(t(1, 8), t(BIG, 8), t(1, BIG)),
    lambda t: B.grouped_forward(t(1, 8), t(BIG, 8, 8), t(1, 8), offsets=t(BIG + 1, dtype=torch.int64)),
    lambda t: B.grouped_input_grad(t(1, BIG), t(BIG, 8), t(1, 8)),
    lambda t: B.grouped_weight_grad(t(1, 8), t(1, BIG), t(8, BIG)),
    lambda t: B.quantize_rows(t(1, BIG), t(1, BIG, dtype=torch.int8), t(1, dtype=torch.float32)),
    lambda t: B.grouped_forward_i8(t(1, BIG, dtype=torch.int8), t(1, dtype=torch.float32), t(8, BIG, dtype=torch.int8),
                                   t(8, dtype=torch.float32), t(1, 8))])
def test_sizes_beyond_32_bits_are_refused_not_cut(call):
    """A size whose low 32 bits are a fine size would be taken for that one."""
    with pytest.raises(ValueError, match="32 bits"):
        call(lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="meta"))


@pytest.mark.parametrize("name", ["out_features", "in_features", "batch", "group_size"])
def test_layers_beyond_32_bits_are_refused_not_cut(name):
    cfg = B.LayerConfig(8, 256, (-1.0, 1.0))
    setattr(cfg, name, (1 << 32) + getattr(cfg, name))
    with pytest.raises(ValueError, match=name):
        B.packed_size(cfg)


def test_streams_of_another_device_are_refused():
    """The tensors are checked to be on the current device: their kernel may not go to another one's stream."""
    assert B._raw_stream(SimpleNamespace(cuda_stream=64, device_index=1), 1) == 64
    with pytest.raises(ValueError, match="stream is on device 1"):
        B._raw_stream(SimpleNamespace(cuda_stream=64, device_index=1), 0)


@pytest.mark.parametrize("helper", ["lin_of", "tile_at", "swz", "load_rows", "wait_vm", "slab_barrier"])
def test_helpers_that_two_files_have_are_the_same(helper):
    """The contraction has its own copy of these, as its measured traffic is recorded for its exact source: a
    change to one belongs in both."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_18556_amd", "csrc")
    bodies = []
    for name in ("gsq_slab.hpp", "gsq_contract.hip"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, name)).read())
        body = re.search(r"(template <[^>]*>\s*)?__device__ __forceinline__ \w+ " + helper + r"\(.*?\}\n", text, re.S)
        assert body, (name, helper)
        bodies.append(" ".join(body[0].split()))
    assert bodies[0] == bodies[1]
