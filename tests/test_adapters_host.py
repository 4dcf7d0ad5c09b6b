"""What the adapters refuse, before anything reaches the device."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2604_18556_amd import binding as B

torch = pytest.importorskip("torch")
P = ctypes.c_void_p
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E = B.GSQ_EINVAL


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libgsq.so not built (run __graft_entry__.build())")
    return B.load()


def sizes(segments=2, adapters=2, rank=8, out=16, inn=24, dtype=B.DT_BF16, rows=4):
    return B.CAdapters(segments, adapters, rank, out, inn, dtype, rows)


def calls(lib, g):
    """The three calls, as functions of their arrays; the last takes the type of the gradients and accumulate."""
    return (lambda *v: lib.gsq_adapter_forward(g, *v, None), lambda *v: lib.gsq_adapter_input_grad(g, *v, None),
            lambda *v, dt=B.DT_FP32, add=0: lib.gsq_adapter_weight_grad(g, *v, dt, add, None))


@pytest.mark.parametrize("bad", [
    dict(segments=0), dict(segments=65536), dict(adapters=0), dict(adapters=65536), dict(rank=0), dict(rank=513),
    dict(out=0), dict(out=(1 << 21) + 1), dict(inn=0), dict(inn=(1 << 21) + 1), dict(dtype=B.DT_FP32), dict(dtype=9),
    dict(rows=-1), dict(rows=(1 << 29) + 1)])
def test_sizes_are_checked(lib, bad):
    a = P(64)
    for call in calls(lib, ctypes.byref(sizes(**bad))):
        assert call(*[a] * 9) == E and lib.gsq_last_error()


def test_arrays_are_checked(lib):
    a = P(64)
    forward, grad, weights = calls(lib, ctypes.byref(sizes()))
    # x, a, b, offsets, index, scales, base, hidden, y; dy, x, hidden, dhidden, offsets, index, scales, da, db
    for call, optional, words in ((forward, (4, 5, 6), (5, 7)), (grad, (4, 5, 6), (5, 7)), (weights, (5, 6), (2, 3, 6, 7, 8))):
        for k in range(9):
            args = [a] * 9
            if k not in optional:
                args[k] = None
                assert call(*args) == E, k
            args[k] = P(65)
            assert call(*args) == E, k
            if k in words or k == (3 if call is not weights else 4):
                args[k] = P(66)
                assert call(*args) == E, k
    assert weights(*[a] * 9, dt=B.DT_FP16) == E
    assert weights(*[a] * 9, dt=B.DT_BF16, add=1) == E and b"FP32" in lib.gsq_last_error()
    for call in calls(lib, None):
        assert call(*[a] * 9) == E
    g3 = ctypes.byref(sizes(segments=3))         # without an index, each segment has its own adapter
    assert lib.gsq_adapter_forward(g3, a, a, a, a, None, a, a, a, a, None) == E
    assert lib.gsq_adapter_weight_grad(g3, a, a, a, a, a, None, a, a, a, B.DT_FP32, 0, None) == E
    assert b"index" in lib.gsq_last_error()


def test_no_rows_need_no_arrays(lib):
    g, a = ctypes.byref(sizes(rows=0)), P(64)
    assert lib.gsq_adapter_forward(g, None, a, a, a, None, None, None, None, None, None) == B.GSQ_OK
    assert lib.gsq_adapter_input_grad(g, None, a, a, a, None, None, None, None, None, None) == B.GSQ_OK


def test_more_tiles_than_a_launch_holds(lib):
    a = P(64)
    g = ctypes.byref(sizes(segments=1, adapters=1, out=1 << 21, inn=1 << 21, rows=1 << 29))
    assert lib.gsq_adapter_forward(g, a, a, a, a, a, a, a, a, a, None) == E and b"tiles" in lib.gsq_last_error()
    assert lib.gsq_adapter_input_grad(g, a, a, a, a, a, a, a, a, a, None) == E
    g = ctypes.byref(sizes(adapters=65535, out=1 << 21, inn=1 << 21, rank=512))
    assert lib.gsq_adapter_weight_grad(g, a, a, a, a, a, a, a, a, a, B.DT_FP32, 0, None) == E
    assert b"tiles" in lib.gsq_last_error()


def test_header_and_library_have_the_same_calls(lib):
    text = open(os.path.join(ROOT, "include", "gsq_adapters.h")).read()
    assert set(re.findall(r"^gsq_status\s+(gsq_\w+)\s*\(", text, re.M)) == set(B.ADAPTER_EXPORTS)
    for name in B.ADAPTER_EXPORTS:
        assert getattr(lib, name) is not None


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gsq_adapters.h"\n'
                   'int main(void) { printf("%zu %zu %zu", sizeof(gsq_adapters), offsetof(gsq_adapters, dtype), '
                   'offsetof(gsq_adapters, rows)); return 0; }\n')
    r = subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                        "/opt/rocm/include", str(src), "-o", str(tmp_path / "layout")], capture_output=True, text=True)
    if r.returncode:
        pytest.skip("cannot compile against hip_runtime_api.h: " + r.stderr[-300:])
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [ctypes.sizeof(B.CAdapters), B.CAdapters.dtype.offset, B.CAdapters.rows.offset]


def test_binding_checks_tensors_before_the_library():
    bf = torch.bfloat16
    x, a, b = torch.zeros(3, 24, dtype=bf), torch.zeros(2, 8, 24, dtype=bf), torch.zeros(2, 16, 8, dtype=bf)
    h, y = torch.zeros(3, 8), torch.zeros(3, 16, dtype=bf)
    off = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="device tensor"):
        B.adapter_forward(x, a, b, h, y, offsets=off)
    with pytest.raises(ValueError, match="need an index"):
        B.adapter_forward(x, a, b, h, y)
    with pytest.raises(ValueError, match="b must have the shape"):
        B.adapter_forward(x, a, b[:, :, :4], h, y, offsets=off)
    with pytest.raises(ValueError, match="adapters x rank"):
        B.adapter_forward(x, a[0], b, h, y, offsets=off)
    with pytest.raises(ValueError, match="shape"):
        B.adapter_forward(x, a, b, h[:, :4], y, offsets=off)
    with pytest.raises(ValueError, match="shape"):
        B.adapter_forward(x, a, b, h, y, offsets=off, index=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="shape"):
        B.adapter_input_grad(y, a, b, h, y, offsets=off)
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        B.adapter_forward(x.float(), a, b, h, y, offsets=off)
    with pytest.raises(ValueError, match="device tensor"):
        B.adapter_weight_grad(y, x, h, h, a.float(), b.float(), offsets=off)
    big = (1 << 32) + 8
    meta = {"dtype": bf, "device": "meta"}
    with pytest.raises(ValueError, match="32 bits"):
        B.adapter_forward(torch.empty(1, big, **meta), torch.empty(1, 8, big, **meta), torch.empty(1, 8, 8, **meta), h, y)
