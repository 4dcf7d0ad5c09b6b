"""Copies to LDS that are still on their way when their place is written again, looked for in the object code of the
library as it was built: along every way through a kernel, jumps included."""
import os
import re
import subprocess

import pytest

from paper_2604_18556_amd import binding as B
from test_object_code import OBJDUMP, code_objects


def kernel_code(part):
    """(address, instruction, address it may jump to or None) of a kernel's disassembly, and its first address."""
    first, name = re.match(r"([0-9a-f]+) <(\S+)>:", part).groups()
    code = []
    for line in part.splitlines():
        m = re.match(r"\t(.*?)\s*// ([0-9A-F]+):(.*)", line)
        if m:
            jump = re.search(r"<%s(?:\+0x([0-9a-f]+))?>" % re.escape(name), m[3])
            code.append((int(m[2], 16), m[1].strip(), int(first, 16) + int(jump[1] or "0", 16) if jump else None))
    return code


def written_over(code):
    """Stores to LDS that some way reaches from a copy to LDS without a wait for all of the wavefront's loads, and how
    many of both there are."""
    index = {at: k for k, (at, _, _) in enumerate(code)}
    copies = [k for k, (_, text, _) in enumerate(code) if text.startswith("global_load_lds")]
    todo, seen, bad = [k + 1 for k in copies], set(), []
    while todo:
        k = todo.pop()
        if k in seen or k >= len(code):
            continue
        seen.add(k)
        _, text, jump = code[k]
        if text.startswith("s_waitcnt") and "vmcnt(0)" in text or text.startswith("s_endpgm"):
            continue
        if text.startswith("ds_write"):
            bad.append(text)
        if text.startswith(("s_branch", "s_cbranch")):
            todo.append(index[jump])
        assert not text.startswith(("s_setpc", "s_swappc", "s_call")), text
        if not text.startswith("s_branch"):
            todo.append(k + 1)
    return bad, len(copies), sum(text.startswith("ds_write") for _, text, _ in code)


def test_mistakes_are_seen():
    def code(*lines):
        text = "0000000000000100 <k>:\n" + "\n".join(
            f"\t{t} // {256 + 4 * k:012X}: 00000000" + (f" <k+0x{4 * to:x}>" if to is not None else "")
            for k, (t, to) in enumerate((line, None) if isinstance(line, str) else line for line in lines))
        return kernel_code(text)

    copy, wait, store = "global_load_lds_dwordx4 v76, s[8:9]", "s_waitcnt vmcnt(0)", "ds_write_b128 v1, v[2:5]"
    assert written_over(code(copy, "s_barrier", store, "s_endpgm"))[0]
    assert written_over(code(copy, wait, store, "s_endpgm")) == ([], 1, 1)
    assert written_over(code(copy, "s_waitcnt vmcnt(8) lgkmcnt(0)", store, "s_endpgm"))[0]
    assert not written_over(code(store, copy, "s_endpgm"))[0]
    # a wait that one way leaves out, and a loop back to the store
    assert written_over(code(copy, ("s_cbranch_scc1 1", 3), wait, store, "s_endpgm"))[0]
    assert written_over(code(store, copy, ("s_cbranch_scc1 65533", 0), "s_endpgm"))[0]
    assert not written_over(code(copy, ("s_branch 1", 3), store, wait, "s_endpgm"))[0]


def test_sums_of_adapters_wait_for_their_copies():
    """The wavefronts' sums of dA and dB are written where their slabs were copied to."""
    if not (os.path.exists(B._LIB_PATH) and os.path.exists(OBJDUMP)):
        pytest.skip("libgsq.so or llvm-objdump is missing")
    kernels = 0
    for co in code_objects(B._LIB_PATH):
        if b"k_adapter_weights" not in co:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "-"], check=True, capture_output=True, input=co).stdout.decode()
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            if not re.match(r"[0-9a-f]+ <\S*k_adapter_weights\S*>:", part):
                continue
            bad, copies, stores = written_over(kernel_code(part))
            assert not bad, (part.split("\n", 1)[0], bad)
            assert stores
            kernels += copies > 0
    assert kernels >= 8
