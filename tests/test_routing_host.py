"""What the routing refuses, before anything reaches the device, and the rule that orders ids."""
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


def routing(tokens=4, dtype=B.DT_BF16, **kw):
    base = dict(experts=16, top_k=4, groups=4, top_groups=2)
    base.update(kw)
    return B.Routing(**base).to_c(tokens, dtype)


def exchange(tokens=4, rows=8, copies=2, cols=16, dtype=B.DT_BF16):
    return B.CExchange(tokens, rows, copies, cols, dtype)


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(tokens=(1 << 25) + 1), dict(dtype=3), dict(dtype=-1), dict(experts=0), dict(experts=1025),
    dict(groups=0), dict(groups=3), dict(groups=65, experts=130), dict(top_groups=0), dict(top_groups=5), dict(top_k=0),
    dict(top_k=9), dict(experts=64, groups=1, top_groups=1, top_k=33), dict(score=2), dict(score=-1),
    dict(group_score=2), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_routing_sizes_are_checked(lib, bad):
    r, a = ctypes.byref(routing(**bad)), P(64)
    assert lib.gsq_route(r, a, a, a, a, None) == E and lib.gsq_last_error()
    assert lib.gsq_route_grad(r, a, a, a, a, None) == E and lib.gsq_last_error()


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(tokens=(1 << 29) + 1), dict(rows=-1), dict(rows=(1 << 29) + 1), dict(copies=0),
    dict(copies=1025), dict(cols=0), dict(cols=(1 << 21) + 1), dict(dtype=3)])
def test_exchange_sizes_are_checked(lib, bad):
    g, a = ctypes.byref(exchange(**bad)), P(64)
    assert lib.gsq_dispatch_rows(g, a, a, a, None) == E and lib.gsq_last_error()
    assert lib.gsq_combine_rows(g, a, a, a, a, None) == E and lib.gsq_last_error()
    assert lib.gsq_combine_rows_grad(g, a, a, a, a, a, a, None) == E and lib.gsq_last_error()


def test_order_sizes_are_checked(lib):
    a = P(64)
    for count, groups in ((-1, 4), ((1 << 30) + 1, 4), (4, 0), (4, 4097)):
        assert lib.gsq_group_rows(a, count, groups, a, a, a, None) == E and lib.gsq_last_error()


@pytest.mark.parametrize("bad", [None, P(65), P(66)], ids=["null", "odd", "half"])
def test_arrays_are_checked(lib, bad):
    a, r, g = P(64), ctypes.byref(routing(dtype=B.DT_FP32)), ctypes.byref(exchange(dtype=B.DT_FP32))

    def each(call, n, skip=()):
        for k in range(n):
            if k in skip and bad is None:
                continue
            args = [a] * n
            args[k] = bad
            assert call(*args) == E, k

    each(lambda *v: lib.gsq_route(r, *v, None), 4, skip=(1,))          # no bias is fine
    each(lambda *v: lib.gsq_route_grad(r, *v, None), 4)
    each(lambda ids, *v: lib.gsq_group_rows(ids, 4, 4, *v, None), 4)
    each(lambda *v: lib.gsq_dispatch_rows(g, *v, None), 3)
    each(lambda *v: lib.gsq_combine_rows(g, *v, None), 4, skip=(2,))   # nor are weights needed
    each(lambda *v: lib.gsq_combine_rows_grad(g, *v, None), 6)
    assert lib.gsq_route(None, a, a, a, a, None) == E
    assert lib.gsq_dispatch_rows(None, a, a, a, None) == E


def test_no_tokens_need_no_arrays(lib):
    r, g = ctypes.byref(routing(tokens=0)), ctypes.byref(exchange(tokens=0, rows=0))
    assert lib.gsq_route(r, None, None, None, None, None) == B.GSQ_OK
    assert lib.gsq_route_grad(r, None, None, None, None, None) == B.GSQ_OK
    assert lib.gsq_dispatch_rows(g, None, None, None, None) == B.GSQ_OK
    assert lib.gsq_combine_rows(g, None, None, None, None, None) == B.GSQ_OK
    assert lib.gsq_combine_rows_grad(g, None, None, None, None, None, None, None) == B.GSQ_OK


def test_header_and_library_have_the_same_calls(lib):
    text = open(os.path.join(ROOT, "include", "gsq_routing.h")).read()
    assert set(re.findall(r"^gsq_status\s+(gsq_\w+)\s*\(", text, re.M)) == set(B.ROUTING_EXPORTS)
    for name in B.ROUTING_EXPORTS:
        assert getattr(lib, name) is not None


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gsq_routing.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu %zu %d %d %d %d", sizeof(gsq_routing), '
                   'offsetof(gsq_routing, scale), offsetof(gsq_routing, dtype), sizeof(gsq_exchange), '
                   'offsetof(gsq_exchange, dtype), GSQ_SCORE_SOFTMAX, GSQ_SCORE_SIGMOID, GSQ_GROUP_MAX, '
                   'GSQ_GROUP_TOP2); return 0; }\n')
    r = subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                        "/opt/rocm/include", str(src), "-o", str(tmp_path / "layout")], capture_output=True, text=True)
    if r.returncode:
        pytest.skip("cannot compile against hip_runtime_api.h: " + r.stderr[-300:])
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [ctypes.sizeof(B.CRouting), B.CRouting.scale.offset, B.CRouting.dtype.offset,
                                     ctypes.sizeof(B.CExchange), B.CExchange.dtype.offset, B.SCORE_SOFTMAX,
                                     B.SCORE_SIGMOID, B.GROUP_MAX, B.GROUP_TOP2]


def test_binding_checks_tensors_before_the_library():
    r, i32 = B.Routing(8, 2), torch.int32
    logits, ids, w = torch.zeros(3, 8), torch.zeros(3, 2, dtype=i32), torch.zeros(3, 2)
    with pytest.raises(ValueError, match="device tensor"):
        B.route(r, logits, ids, w)
    with pytest.raises(ValueError, match="two dimensions"):
        B.route(r, logits[0], ids, w)
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        B.route(r, logits.double(), ids, w)
    with pytest.raises(ValueError, match="shape"):
        B.route(B.Routing(7, 2), logits, ids, w)
    with pytest.raises(ValueError, match="shape"):
        B.route(r, logits, ids, w, bias=torch.zeros(7))
    with pytest.raises(ValueError, match="shape"):
        B.route_grad(r, logits, ids, w, torch.zeros(3, 7))
    with pytest.raises(ValueError, match="shape"):
        B.group_rows(ids, torch.zeros(9, dtype=torch.int64), ids.view(-1), torch.zeros(6, dtype=i32))
    with pytest.raises(ValueError, match="device tensor"):
        B.group_rows(ids, torch.zeros(9, dtype=torch.int64), ids, torch.zeros(6, dtype=i32))
    x, rows = torch.zeros(3, 16), torch.zeros(6, 16)
    with pytest.raises(ValueError, match="shape"):
        B.dispatch_rows(x, ids[:2], rows)
    with pytest.raises(ValueError, match="shape"):
        B.combine_rows(rows[:, :8], ids, x)
    with pytest.raises(ValueError, match="device tensor"):
        B.combine_rows_grad(x, rows, ids, w, rows, w)


BIG = (1 << 32) + 8          # 8 in its low 32 bits


@pytest.mark.parametrize("call", [
    lambda t: B.route(B.Routing(BIG, 1), t(1, BIG), t(1, 1, dtype=torch.int32), t(1, 1)),
    lambda t: B.route(B.Routing(8, 1, score=1 << 32), t(1, 8), t(1, 1, dtype=torch.int32), t(1, 1)),
    lambda t: B.route(B.Routing(8, 1, group_score=1 << 32), t(1, 8), t(1, 1, dtype=torch.int32), t(1, 1)),
    lambda t: B.dispatch_rows(t(1, BIG), t(1, 1, dtype=torch.int32), t(1, BIG)),
    lambda t: B.combine_rows(t(1, 8), t(1, BIG, dtype=torch.int32), t(1, 8)),
    lambda t: B.group_rows(t(1, dtype=torch.int32), t(BIG + 1, dtype=torch.int64), t(1, dtype=torch.int32),
                           t(1, dtype=torch.int32))])
def test_sizes_beyond_32_bits_are_refused_not_cut(call, monkeypatch):
    monkeypatch.setattr(B, "_checked", lambda *a: 0)
    with pytest.raises(ValueError, match="32 bits"):
        call(lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta"))


def test_plan_of_the_order(tmp_path):
    """LDS, scratch and places for every size: the histograms fit 64 KB, the chunks cover the ids, and their counts fit
    the array that holds them."""
    src = tmp_path / "plan.cpp"
    src.write_text(r'''
#include <cstdio>
#include "gsq_plan.h"
int main() {
  using namespace gsq;
  for (int64_t n = 1; n <= ((int64_t)1 << 30); n += n < 300 ? 1 : n / 7 + 1)
    for (int g : {1, 2, 3, 64, 255, 256, 257, 1000, 2048, 3000, 4095, 4096}) {
      const OrderPlan p = plan_order(n, g);
      bool ok = p.waves >= 1 && 64 * p.waves <= p.threads && p.threads <= 1024 && p.chunks >= 1 && p.chunks <= 128;
      ok = ok && p.chunks * p.chunk >= n && (p.chunks - 1) * p.chunk < n;
      if (p.chunks == 1) ok = ok && (p.waves + 1) * g * 4 + 64 <= 65536 && n <= 16384;
      else ok = ok && p.waves * g * 4 <= 65536 && 2 * (g + (g < p.threads ? p.threads : 0)) * 4 + 64 <= 65536 && (int64_t)p.chunks * g <= n && p.threads <= 512;
      if (!ok) { std::printf("%lld %d\n", (long long)n, g); return 1; }
    }
  return 0;
}
''')
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_18556_amd", "csrc"), str(src), "-o",
                    str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_counts_of_the_order_fit_the_ids_places(tmp_path):
    """Less than a quarter of the places and one chunk's counts, whatever the last chunk holds."""
    src = tmp_path / "plan.cpp"
    src.write_text(r'''
#include <cstdio>
#include "gsq_plan.h"
int main() {
  using namespace gsq;
  double most = 0;
  for (int g : {1, 2, 3, 7, 64, 100, 255, 256, 257, 1000, 2047, 2048, 2049, 3000, 4095, 4096})
    for (int64_t n = 8193; n <= ((int64_t)1 << 30); n += n < 17000 ? 1 : n / 7 + 1) {
      const OrderPlan p = plan_order(n, g);
      if (p.chunks == 1) continue;
      const int64_t words = (int64_t)p.chunks * g;
      most = std::max(most, (double)words / n);
      if (4 * words >= n + 4 * g || words > n) { std::printf("%lld ids, %d groups: %lld\n", (long long)n, g, (long long)words); return 1; }
    }
  if (most < 0.49 || most > 0.51) { std::printf("%f\n", most); return 1; }
  return 0;
}
''')
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2604_18556_amd", "csrc"), str(src), "-o",
                    str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
