"""Static checks of the clear track's generated gfx950 code (no GPU).

A 16 x 16 x 32 matrix instruction runs on while the next instructions issue, and a vector instruction that touches its result within
seven issue slots sees the old one: the compiler has to fill the slots (s_nop N counts N + 1), the hardware does not wait.  In one kernel
it did not where a sum had been moved behind a branch, and one value in four was wrong.  Every way through every kernel is walked here.
"""
import os
import re
import subprocess

import pytest

from paper_2601_18511_amd import build as hip_build

SLOTS = 7


@pytest.fixture(scope="module", params=("ppmv.hip", "ppkv.hip"))
def kernels(request, tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "out.s")
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    cmd = [hip_build.hipcc_path()] + flags + ["--cuda-device-only", "-S", "-o", out, os.path.join(hip_build.CSRC, request.param)]
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert proc.returncode == 0, proc.stdout
    text = open(out).read()
    return {m.group(1): m.group(2) for m in re.finditer(r"^(_Z\S+):.*?\n(.*?)^\.Lfunc_end", text, re.S | re.M)}


def _registers(operands):
    found = set()
    for m in re.finditer(r"\b([va])(\d+)\b|\b([va])\[(\d+):(\d+)\]", operands):
        if m.group(1):
            found.add((m.group(1), int(m.group(2))))
        else:
            found.update((m.group(3), r) for r in range(int(m.group(4)), int(m.group(5)) + 1))
    return found


def _program(body):
    """Instructions, and where each may go on."""
    code, labels = [], {}
    for line in body.split("\n"):
        line = line.split(";")[0].strip()
        label = re.match(r"(\.LBB\S+):", line)
        if label:
            labels[label.group(1)] = len(code)
        elif line and not line.startswith(".") and not line.endswith(":"):
            code.append(line)

    def after(i):
        op, _, operands = code[i].partition(" ")
        if op == "s_endpgm":
            return []
        if op == "s_branch":
            return [labels[operands.strip()]]
        return [labels[operands.strip()], i + 1] if op.startswith("s_cbranch") else [i + 1]

    return code, after


def _too_early(body):
    code, after = _program(body)
    for i, line in enumerate(code):
        if not line.startswith("v_mfma"):
            continue
        result = _registers(line.split(None, 1)[1].split(",")[0])
        seen, todo = {}, [(j, 0) for j in after(i)]
        while todo:
            j, slots = todo.pop()
            if j >= len(code) or slots >= SLOTS or seen.get(j, SLOTS) <= slots:
                continue
            seen[j] = slots
            op, _, operands = code[j].partition(" ")
            if op == "s_nop":
                slots += int(operands.split()[0])
            elif op.startswith("v_mfma"):
                if _registers(operands.split(",")[0]) >= result:
                    continue
            elif op.startswith(("v_", "ds_", "global_", "buffer_", "scratch_", "flat_")) and _registers(operands) & result:
                yield line, code[j], slots
                continue
            todo += [(k, slots + 1) for k in after(j)]


def _short_waits(body):
    """Written waits s_waitcnt vmcnt(N > 0) and, where that is below N, the fewest loads between one and a load to LDS in front of it.

    Such a wait is for the loads to LDS, with N later loads of weights left under way: were they fewer, it would end too early."""
    code, labels, written, inside = [], {}, [], False
    for line in body.split("\n"):
        inside = "#ASMSTART" in line or inside and "#ASMEND" not in line
        line = line.split(";")[0].strip()
        label = re.match(r"(\.LBB\S+):", line)
        if label:
            labels[label.group(1)] = len(code)
        elif line and not line.startswith(".") and not line.endswith(":"):
            code.append(line)
            written.append(inside)
    before = [[] for _ in code]
    for i, line in enumerate(code):
        op, _, operands = line.partition(" ")
        to = [] if op in ("s_endpgm", "s_branch") else [i + 1]
        to += [labels[operands.strip()]] if op == "s_branch" or op.startswith("s_cbranch") else []
        for j in to:
            if j < len(code):
                before[j].append(i)
    for i, line in enumerate(code):
        wait = re.match(r"s_waitcnt vmcnt\((\d+)\)", line)
        if not wait or not written[i] or int(wait.group(1)) == 0:
            continue
        left, seen, todo, least = int(wait.group(1)), {}, [(j, 0) for j in before[i]], None
        while todo:
            j, loads = todo.pop()
            if seen.get(j, left) <= loads:
                continue
            seen[j] = loads
            if re.match(r"(global|buffer)_load", code[j]):
                if re.search(r"\blds\b|_lds_", code[j]):
                    least = loads if least is None else min(least, loads)
                    continue
                loads += 1
            todo += [(k, loads) for k in before[j]]
        yield left, least


def test_the_check_of_waits_sees_what_it_should():
    dma, load = "buffer_load_dwordx4 v1, s[0:3], 0 offen lds\n", "global_load_dwordx4 v[2:5], v[6:7], off\n"
    wait = ";;#ASMSTART\ns_waitcnt vmcnt(2)\n;;#ASMEND\ns_endpgm\n"
    assert list(_short_waits(dma + load + load + wait)) == [(2, None)]
    assert list(_short_waits(dma + load + wait)) == [(2, 1)]
    assert list(_short_waits(dma + load + "s_cbranch_scc1 .LBB0_1\n" + load + ".LBB0_1:\n" + wait)) == [(2, 1)]


def test_waits_for_lds_leave_no_more_loads_than_follow(kernels):
    counted = 0
    for name, body in kernels.items():
        for left, least in _short_waits(body):
            counted += 1
            assert least is None, (name, left, least)
    assert counted > 100 or not any("many_tokens" in name for name in kernels)


def test_the_check_sees_what_it_should():
    mfma = "v_mfma_f32_16x16x32_f16 v[14:17], v[2:5], v[26:29], v[14:17]\n"
    assert list(_too_early(mfma + "s_cbranch_scc1 .LBB0_1\ns_nop 7\n.LBB0_1:\nv_fma_f32 v10, v34, v14, v10\ns_endpgm\n"))
    assert list(_too_early(mfma + "s_nop 5\nv_add_f32_e32 v1, v1, v17\ns_endpgm\n"))
    assert not list(_too_early(mfma + "s_nop 6\nv_add_f32_e32 v1, v1, v17\ns_endpgm\n"))
    assert not list(_too_early(mfma + "v_add_f32_e32 v1, v1, v18\ns_endpgm\n"))


def test_no_result_of_a_matrix_instruction_is_touched_too_early(kernels):
    counted = 0
    for name, body in kernels.items():
        counted += body.count("v_mfma")
        assert not list(_too_early(body)), name
    assert counted > 300


def test_no_packed_fp32(kernels):
    for name, body in kernels.items():
        assert not re.search(r"v_pk_(add|mul|fma)_f32", body), name
