"""Static checks on the code hipcc generates for the products on a base in 8-bit integers and for the kernels on rows of logits (CPU only:
cross-compilation).

The persistent product makes the same assumptions as the bf16 one (named AGPRs, hazards, M0: see test_kernel_isa.py), and its accumulators turn from whole
numbers into fp32 in place, by statements that name them too."""
import os
import re
import subprocess

import pytest

from test_kernel_isa import (CSRC, HIPCC, ROOT, _lds_writes_pending_at_a_barrier as pending_writes, test_all_agprs_allocated_and_nothing_spilled,
                             test_m0_is_written_and_consumed_inside_one_statement, test_main_loop_has_no_instruction_clumps,
                             test_no_kernel_takes_scratch_memory,
                             test_no_mfma_reads_a_register_a_vector_alu_instruction_has_just_written)

CHECKS = [test_all_agprs_allocated_and_nothing_spilled, test_m0_is_written_and_consumed_inside_one_statement,
          test_no_mfma_reads_a_register_a_vector_alu_instruction_has_just_written, test_main_loop_has_no_instruction_clumps]
SCRATCH = test_no_kernel_takes_scratch_memory
for _name in [n for n in globals() if n.startswith("test_")]:
    del globals()[_name]


def assembly(tmp, source):
    out = str(tmp / (source + ".s"))
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "--cuda-device-only",
           "-S", os.path.join(CSRC, source), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return open(out).read()


@pytest.fixture(scope="module")
def q8_kernels(tmp_path_factory):
    parts = re.split(r"^(_ZN5lobra25gemm_persistent_q8_kernel\w+):", assembly(tmp_path_factory.mktemp("isa"), "gemm_persistent_q8.hip"), flags=re.M)
    ks = []
    for i in range(1, len(parts), 2):
        body = parts[i + 1]
        end = body.index(".end_amdhsa_kernel")
        code = [l.split(";")[0].strip() for l in body[:body.rindex("s_endpgm", 0, end) + 8].split("\n")]
        ks.append((parts[i], [l for l in code if l and not l.startswith(".")], body[end:end + 3000]))
    assert len(ks) == 1, [k[0] for k in ks]
    return ks


@pytest.mark.parametrize("check", CHECKS, ids=lambda f: f.__name__)
def test_q8_kernel(q8_kernels, check):
    check(q8_kernels)


def test_only_the_named_statements_touch_agprs(q8_kernels):
    mfma = re.compile(r"(v_mfma_i32_16x16x64_i8|v_mfma_f32_16x16x32_bf16) (a\[\w+:\w+\]), v\[\d+:\d+\], v\[\d+:\d+\], (a\[\w+:\w+\]|0)$")
    rd, wr = re.compile(r"v_accvgpr_read_b32 v\d+, a\[(\w+)\]$"), re.compile(r"v_accvgpr_write_b32 a\[(\w+)\], v\d+$")
    for name, code, _ in q8_kernels:
        users = [l for l in code if re.search(r"\ba(\[|\d)", l)]
        bad = [l for l in users if not (mfma.match(l) or rd.match(l) or wr.match(l))]
        assert not bad, (name, bad[:5])
        for l in users:
            m = mfma.match(l)
            if m:
                assert m.group(3) in ("0", m.group(2)), l
        # every accumulator is turned into fp32 once, behind the last MFMA of whole numbers and the wait states it needs
        at = [i for i, l in enumerate(code) if wr.match(l)]
        assert len(at) == 256, len(at)
        first = min(i for i, l in enumerate(code) if rd.match(l))
        last = max(i for i in range(first) if code[i].startswith("v_mfma"))
        assert code[last:first].count("s_nop 15") == 2, code[last:first]


@pytest.mark.parametrize("source", ["gemm_persistent_q8.hip", "gemm_tile_q8.hip", "q8.hip", "q8_few.hip", "distill.hip", "beam.hip"])
def test_lds_writes_are_waited_for(tmp_path, source):
    parts = re.split(r"^(_ZN5lobra\w+):", assembly(tmp_path, source), flags=re.M)
    barriers = 0
    for name, body in zip(parts[1::2], parts[2::2]):
        if ".end_amdhsa_kernel" not in body:
            continue
        lines = [l.split(";")[0].strip() for l in body[:body.index(".end_amdhsa_kernel")].split("\n")]
        lines = [l for l in lines if l and (not l.startswith(".") or l.endswith(":"))]
        barriers += sum(l.startswith("s_barrier") for l in lines)
        assert not pending_writes(lines), (name, pending_writes(lines)[0])
    assert barriers >= 1, source


@pytest.mark.parametrize("source,least", [("gemm_persistent_q8.hip", 1), ("gemm_tile_q8.hip", 6), ("q8.hip", 5), ("q8_few.hip", 5), ("distill.hip", 20), ("beam.hip", 10)])
def test_no_scratch_memory(tmp_path, source, least):
    SCRATCH(tmp_path, source, least)
