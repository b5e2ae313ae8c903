"""Static checks on the code hipcc generates for the kernels of the steps around the LoRA linears (CPU only: cross-compilation).

The gated form of the persistent product makes the same assumptions as the product itself (named AGPRs, hazards, M0: see
test_kernel_isa.py); the ring of the few-token product waits for its copies by count, which scratch memory's loads would disturb.
"""
import os
import re
import subprocess

import pytest

from test_kernel_isa import (CSRC, HIPCC, ROOT, _lds_writes_pending_at_a_barrier as pending_writes, test_all_agprs_allocated_and_nothing_spilled,
                             test_m0_is_written_and_consumed_inside_one_statement,
                             test_main_loop_has_no_instruction_clumps, test_no_kernel_takes_scratch_memory,
                             test_no_mfma_reads_a_register_a_vector_alu_instruction_has_just_written, test_only_the_named_statements_touch_agprs)

GATED_CHECKS = [test_only_the_named_statements_touch_agprs, test_all_agprs_allocated_and_nothing_spilled,
                test_m0_is_written_and_consumed_inside_one_statement, test_no_mfma_reads_a_register_a_vector_alu_instruction_has_just_written,
                test_main_loop_has_no_instruction_clumps]
SCRATCH = test_no_kernel_takes_scratch_memory
# (imported for their bodies: they are collected where they stand)
for _name in [n for n in globals() if n.startswith("test_")]:
    del globals()[_name]


@pytest.fixture(scope="module")
def gated_kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("isa") / "gemm_persistent_gated.s")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "--cuda-device-only",
           "-S", os.path.join(CSRC, "gemm_persistent_gated.hip"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    parts = re.split(r"^(_ZN5lobra28gemm_persistent_gated_kernel\w+):", open(out).read(), flags=re.M)
    ks = []
    for i in range(1, len(parts), 2):
        body = parts[i + 1]
        end = body.index(".end_amdhsa_kernel")
        code = [l.split(";")[0].strip() for l in body[:body.rindex("s_endpgm", 0, end) + 8].split("\n")]
        ks.append((parts[i], [l for l in code if l and not l.startswith(".")], body[end:end + 3000]))
    assert len(ks) == 4, [k[0] for k in ks]      # two activations, with and without [g | u]
    return ks


@pytest.mark.parametrize("check", GATED_CHECKS, ids=lambda f: f.__name__)
def test_gated_kernels(gated_kernels, check):
    check(gated_kernels)


@pytest.mark.parametrize("source", ["gemm_persistent_gated.hip", "gated_skinny.hip", "logprob.hip", "grad_clip.hip", "block_norm.hip"])
def test_lds_writes_are_waited_for(tmp_path, source):
    out = str(tmp_path / "k.s")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "--cuda-device-only",
           "-S", os.path.join(CSRC, source), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    parts = re.split(r"^(_ZN5lobra\w+):", open(out).read(), flags=re.M)
    barriers = 0
    for name, body in zip(parts[1::2], parts[2::2]):
        if ".end_amdhsa_kernel" not in body:
            continue
        lines = [l.split(";")[0].strip() for l in body[:body.index(".end_amdhsa_kernel")].split("\n")]
        lines = [l for l in lines if l and (not l.startswith(".") or l.endswith(":"))]
        barriers += sum(l.startswith("s_barrier") for l in lines)
        assert not pending_writes(lines), (name, pending_writes(lines)[0])
    assert barriers >= 1, source


@pytest.mark.parametrize("source,least", [("gemm_persistent_gated.hip", 4), ("gated_skinny.hip", 6), ("logprob.hip", 16), ("grad_clip.hip", 3), ("gated.hip", 8)])
def test_no_scratch_memory(tmp_path, source, least):
    SCRATCH(tmp_path, source, least)


# Registers that do not fit and stand in scratch memory, bytes a lane at most.  The norms' backward kernels with sums over tokens hold a row, (one
# packet a lane) the next one, gains, the task's gate and three fp32 sums per element: more than the 128 registers that 16 waves a compute unit
# leave.  The four-block fp32 product of few tokens is at the 256 of two workgroups.  None of them waits for copies by count, which scratch
# memory's loads would disturb.  (element type, threads of a team, packets of a lane, sums)
NORM_BACKWARD = {("t", 64, 1, 1): 40, ("t", 256, 1, 1): 40, ("t", 512, 1, 1): 40, ("t", 1024, 2, 1): 360,
                 ("f", 1024, 2, 1): 120, ("f", 1024, 4, 1): 620, ("f", 1024, 4, 0): 180}


@pytest.mark.parametrize("source,kernels", [("block_norm.hip", 104), ("gated_few_f32.hip", 6)])
def test_scratch_memory_has_its_bounds(tmp_path, source, kernels):
    out = str(tmp_path / "k.s")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "--cuda-device-only",
           "-S", os.path.join(CSRC, source), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    parts = re.split(r"^\s*\.amdhsa_kernel (\w+)$", open(out).read(), flags=re.M)
    sizes = {name: int(re.search(r"; ScratchSize: (\d+)", body).group(1)) for name, body in zip(parts[1::2], parts[2::2])}
    assert len(sizes) == kernels, (source, len(sizes))
    for name, size in sizes.items():
        most = 72 if "gated_few_kernelILi4E" in name else 0
        m = re.search(r"block_norm_bwd_kernelI([ft])Lb[01]ELi(\d+)ELi(\d)ELb([01])ELb[01]E", name)
        if m:
            most = NORM_BACKWARD.get((m.group(1), int(m.group(2)), int(m.group(3)), int(m.group(4))), 0)
        assert size <= most, (name, size, most)


def test_lds_writes_of_the_fp32_product_of_few_tokens_are_waited_for(tmp_path):
    test_lds_writes_are_waited_for(tmp_path, "gated_few_f32.hip")
