"""What the compiler is not told about the instructions that the kernels write out, checked in the object code of
the library as it was built: matrix instructions, copies to LDS and the waits between them and others.

Wait states are counted along straight code: one for each instruction, N + 1 for `s_nop N`.
"""
import os
import re
import struct
import subprocess

import pytest

from paper_2604_18556_amd import binding as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
KEEP = 40                    # instructions looked back


def code_objects(path):
    """The gfx950 code objects of the bundles in a built library."""
    data, at = open(path, "rb").read(), 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        entries, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(entries):
            offset, size, name = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + name].decode()
            p += 24 + name
            if target.endswith("gfx950"):
                yield data[at + offset:at + offset + size]
        at += 24


def registers(text):
    out = set()
    for kind, lo, hi, kind1, one in re.findall(r"\b([vas])\[(\d+):(\d+)\]|\b([vas])(\d+)\b", text):
        out |= {(kind, k) for k in range(int(lo), int(hi) + 1)} if kind else {(kind1, int(one))}
    return out


class Instruction:
    def __init__(self, text):
        self.text = text
        self.name, _, operands = text.partition(" ")
        first, _, rest = operands.partition(",")
        self.mfma = self.name.startswith("v_mfma")
        self.vector = self.name.startswith("v_") and not self.mfma
        self.states = int(first, 0) + 1 if self.name == "s_nop" else 1
        stores = self.name.startswith(("ds_write", "global_store", "global_load_lds", "scratch_store", "buffer_store"))
        self.writes = set() if stores else registers(first)
        self.reads = registers(operands if stores else rest)

    def before(self, recent, kind):
        """(wait states between, instruction) of the nearest ones before it."""
        states = 0
        for other in reversed(recent):
            if kind(other):
                yield states, other
            states += other.states


def instructions(lines):
    """Those of a kernel's disassembly; None stands where straight code ends."""
    for line in lines:
        one = line.split("//")[0].strip()
        yield Instruction(one)
        if one.startswith(("s_branch", "s_endpgm", "s_setpc")):
            yield None


def along(code):
    """Each instruction, and those right before it."""
    recent = []
    for i in code:
        if i is None:
            recent = []
            continue
        yield i, recent
        recent = (recent + [i])[-KEEP:]


def too_near(code, kind, touched, other, states):
    """Pairs of an instruction of a kind and an `other` one less than `states` before it that writes what it
    touches, and how many of the kind there are."""
    pairs, found = [], 0
    for i, recent in along(code):
        mine = touched(i) if kind(i) else set()
        if mine:
            found += 1
            pairs += [(o.text, i.text) for n, o in i.before(recent, other) if n < states and o.writes & mine]
    return pairs, found


def operands_written(code):
    """Two wait states between a vector instruction and the product that reads what it wrote: the compiler keeps
    them for its own products, but not for written-out ones."""
    return too_near(code, lambda i: i.mfma, lambda i: i.reads, lambda o: o.vector, 2)


def sums_touched(code):
    """18 wait states, enough for the longest product, before anything but a product touches an accumulator
    register that a product has written."""
    return too_near(code, lambda i: not i.mfma, lambda i: {r for r in i.reads | i.writes if r[0] == "a"},
                    lambda o: o.mfma, 18)


def bases_written(code):
    """Five wait states between a vector instruction and a copy whose uniform base it wrote."""
    return too_near(code, lambda i: i.name.startswith("global_load_lds"), lambda i: {r for r in i.reads if r[0] == "s"},
                    lambda o: o.vector, 5)


def test_mistakes_are_seen():
    def code(*lines):
        return list(instructions(lines))

    product = "v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]"
    assert operands_written(code("v_mov_b32_e32 v9, v1", "s_nop 0", product))[0]
    assert not operands_written(code("v_mov_b32_e32 v9, v1", "s_nop 1", product))[0]
    assert not operands_written(code("v_mov_b32_e32 v9, v1", "s_branch 8", product))[0]
    assert not operands_written(code("v_mov_b32_e32 v12, v4", product))[0]
    read = "v_accvgpr_read_b32 v0, a2"
    assert sums_touched(code(product, "s_nop 15", "s_nop 0", read))[0]
    assert not sums_touched(code(product, "s_nop 15", "s_nop 1", read))[0]
    assert sums_touched(code(product, "global_store_dwordx4 v[0:1], a[0:3], off"))[0]
    copy = "global_load_lds_dwordx4 v76, s[8:9]"
    assert bases_written(code("v_readfirstlane_b32 s9, v2", "s_mov_b32 m0, s22", "s_nop 0", copy))[0]
    assert not bases_written(code("v_readfirstlane_b32 s9, v2", "s_nop 2", "s_mov_b32 m0, s22", "s_nop 0", copy))[0]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its instructions} of those with matrix instructions."""
    if not (os.path.exists(B._LIB_PATH) and os.path.exists(OBJDUMP)):
        pytest.skip("libgsq.so or llvm-objdump is missing")
    out = {}
    for k, code in enumerate(code_objects(B._LIB_PATH)):
        path = tmp_path_factory.mktemp("code") / f"{k}.o"
        path.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            label = re.match(r"[0-9a-f]+ <(\S+)>:", part)
            if label and "v_mfma" in part:
                out[label[1]] = list(instructions(line for line in part.splitlines() if line.startswith("\t")))
    return out


@pytest.mark.parametrize("rule,least", [(operands_written, 20000), (sums_touched, 1000), (bases_written, 300)])
def test_wait_states(kernels, rule, least):
    found = 0
    for name, code in kernels.items():
        pairs, n = rule(code)
        found += n
        assert not pairs, (name, pairs[:3])
    assert found >= least


def test_copies_to_lds_have_m0_for_themselves(kernels):
    """A kernel with written-out copies writes M0 for each of them, right before it, and uses it for nothing else.
    (Whole tiles of the packed layer copy by the compiler's own instructions.)"""
    found = 0
    for name, code in kernels.items():
        if not re.search(r"k_(rows|sums)_(tile|split)|k_packed_shared", name):
            continue
        copies = [k for k, i in enumerate(code) if i and i.name.startswith("global_load_lds")]
        uses = [k for k, i in enumerate(code) if i and re.search(r"\bm0\b", i.text)]
        assert uses == [k - 2 for k in copies], name
        assert all(code[k - 2].text.startswith("s_mov_b32 m0,") and code[k - 1].text == "s_nop 0" for k in copies), name
        found += len(copies)
    assert found > 1000
