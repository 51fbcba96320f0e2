"""The compiled kernels wait long enough between a matrix instruction and the first use of its result.

A 32 x 32 x 16 product of fp16 takes 8 passes, one of 16 x 16 x 4 in fp64 16, and what reads or overwrites its result without being a matrix instruction may be issued 3 states behind those at the
earliest: the hardware does not wait by itself, the compiler puts instructions or s_nop between.  It has left them out behind a loop with a way out of its middle, and what was read then was an older value."""
import os
import re
import subprocess

import pytest

from paper_2502_00021_amd import build


def passes(name):
    return 16 if "f64" in name else 8


def registers(text):
    m = re.fullmatch(r"([va])\[(\d+):(\d+)\]", text)
    if m:
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.fullmatch(r"([va])(\d+)", text)
    return {(m[1], int(m[2]))} if m else set()


def too_soon(assembly):
    """(matrix instructions, uses of a result that come too soon), on every path behind each of them."""
    code, labels = [], {}
    for line in assembly.split("\n"):
        line = line.split(";")[0]
        m = re.match(r"(\S+):", line)
        if m:
            labels[m[1]] = len(code)
            continue
        m = re.match(r"\s+([a-z]\w+)\s*(.*)$", line)
        if m:
            code.append((m[1], [t.strip() for t in m[2].split(",")] if m[2] else []))
    products, found = 0, []
    for i, (name, operands) in enumerate(code):
        if not name.startswith("v_mfma"):
            continue
        products += 1
        result, paths, seen, enough = registers(operands[0]), [(i + 1, 0)], {}, passes(name) + 3
        while paths:
            at, states = paths.pop()
            while states < enough and at < len(code) and seen.get(at, enough) > states:
                seen[at] = states
                name, operands = code[at]
                if name == "s_endpgm":
                    break
                if name.startswith("v_mfma"):
                    states += passes(name)
                elif name == "s_nop":
                    states += int(operands[0], 0) + 1
                else:
                    if set().union(*map(registers, operands)) & result:
                        found.append((i, at, name, operands, states))
                        break
                    states += 1
                if name == "s_branch":
                    at = labels[operands[0]]
                    continue
                if name.startswith("s_cbranch"):
                    paths.append((labels[operands[0]], states))
                at += 1
    return products, found


def test_the_search_itself():
    straight = "\tv_mfma_f32_32x32x16_f16 v[0:15], v[20:23], v[24:27], v[0:15]\n"
    assert too_soon(straight + "\ts_nop 10\n\tv_add_f32_e32 v30, v3, v30\n\ts_endpgm\n") == (1, [])
    assert len(too_soon(straight + "\ts_nop 9\n\tv_add_f32_e32 v30, v3, v30\n\ts_endpgm\n")[1]) == 1
    twice = "\tv_mfma_f64_16x16x4_f64 v[0:7], v[20:21], v[24:25], v[0:7]\n\ts_nop 15\n\ts_nop {}\n\tv_add_f64 v[30:31], v[6:7], v[30:31]\n\ts_endpgm\n"
    assert too_soon(twice.format(2)) == (1, []) and len(too_soon(twice.format(1))[1]) == 1
    assert len(too_soon(straight + "\ts_nop 9\n\tv_add_f32_e32 v30, v16, v30\n\ts_endpgm\n")[1]) == 0
    loop = ("\ts_branch .L2\n.L1:\n" + straight + "\ts_cbranch_scc1 .L1\n\ts_cbranch_vccz .L3\n.L2:\n\ts_nop 15\n\ts_branch .L1\n.L3:\n{}\tglobal_store_dwordx4 v[40:41], v[4:7], off\n\ts_endpgm\n")
    assert len(too_soon(loop.format(""))[1]) == 1 and too_soon(loop.format("\ts_nop 8\n"))[1] == []


@pytest.mark.parametrize("source", ["orthogonalise.hip"])
def test_results_of_matrix_instructions(source, tmp_path):
    flags = [f for f in build.HIPFLAGS if f != "-shared"]
    out = tmp_path / "code.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-S", "--offload-device-only", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, os.path.join(build.CSRC, source), "-o", str(out)],
                   check=True, stderr=subprocess.DEVNULL)
    products, found = too_soon(out.read_text())
    assert products > 300 and not found, found[:5]
