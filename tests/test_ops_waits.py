"""The waits between attention's matrix products and the instructions that take their
registers, in the compiled kernels.

A vector or memory instruction may read or overwrite a matrix product's result only some
instructions' time after it (8 for bfloat16's product, 10 for float32's); the hardware does not
hold it back.  The compiler puts the waits, but was seen to miss one across the end of a block.
Here every path on from every product is followed."""
import os
import re
import subprocess

import pytest

from paper_2308_04623_amd import build

STATES = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}


def registers(text):
    out = set()
    for m in re.finditer(r"(?<![\w])v(?:(\d+)|\[(\d+):(\d+)\])", text):
        lo, hi = (m.group(1), m.group(1)) if m.group(1) else (m.group(2), m.group(3))
        out.update(range(int(lo), int(hi) + 1))
    return out


def functions(text):
    name, code = None, {}
    for line in text.split("\n"):
        start = re.match(r"(_Z\w+):", line)
        line = line.split(";")[0].strip()
        if start:
            name = start.group(1)
            code[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and line and (line.startswith(".LBB") or not line.startswith(".")):
            code[name].append(line)
    return code


def early(code):
    """(product, instruction, states between them) for all that come too early."""
    labels = {line[:-1]: i for i, line in enumerate(code) if line.startswith(".LBB")}

    def after(i):
        op, *args = code[i].split()
        if op == "s_endpgm":
            return []
        to = [labels[args[0]]] if op == "s_branch" or op.startswith("s_cbranch") else []
        return to if op == "s_branch" else to + [i + 1]

    for i, line in enumerate(code):
        if not line.startswith("v_mfma"):
            continue
        op, args = line.split(None, 1)
        result = registers(args.split(", ")[0])
        at, paths = {}, [(j, 0) for j in after(i)]
        while paths:
            j, states = paths.pop()
            if states >= STATES[op] or at.get(j, 99) <= states:
                continue
            at[j] = states
            other, *rest = code[j].split(None, 1)
            if other.startswith("v_mfma"):
                out, a, b, _ = rest[0].split(", ")
                if (registers(a) | registers(b)) & result:
                    yield line, code[j], states
                if registers(out) == result:  # (adds to it: the hardware waits)
                    continue
            elif re.match(r"v_|ds_|global_|flat_|buffer_", other) and registers(code[j]) & result:
                yield line, code[j], states
                continue
            if not other.endswith(":"):
                states += 1 + (int(rest[0]) if other == "s_nop" else 0)
            paths += [(k, states) for k in after(j)]


def test_the_search_finds_an_early_read():
    product = "v_mfma_f32_16x16x4_f32 v[4:7], v1, v2, v[4:7]"
    on_a_path = [product, "s_cbranch_scc1 .LBB0_2", ".LBB0_1:", "v_mov_b32_e32 v9, v10", "s_nop 7", ".LBB0_2:",
                 "v_max_f32_e32 v3, v5, v5", "s_endpgm"]
    assert [x[2] for x in early(on_a_path)] == [1]
    on_a_path.insert(6, "s_nop 8")
    assert not list(early(on_a_path))
    assert not list(early([product, product, "s_nop 9", "v_mov_b32_e32 v3, v4", "s_endpgm"]))


def test_results_are_taken_when_they_are_complete(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no compiler")
    out = str(tmp_path / "attn.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc, *flags, "-I", os.path.join(build.ROOT, "include"), "--cuda-device-only", "-S",
                    os.path.join(build.HERE, "csrc", "ops_attn.hip"), "-o", out], check=True, capture_output=True)
    kernels = functions(open(out).read())
    assert sum(line.startswith("v_mfma") for code in kernels.values() for line in code) > 1000
    for name, code in kernels.items():
        assert not list(early(code)), name
