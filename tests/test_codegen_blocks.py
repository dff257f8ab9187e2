"""Code-generation checks of the products over row groups (host only: hipcc emits the gfx950 assembly, nothing
runs).  No kernel spills to scratch memory, which would be in the loop that holds the accumulators, and the loop over
the stages of the tiles waits for its loads only where the waves meet."""
import os
import re
import subprocess

import pytest

from paper_2609_21483_amd import build as BLD


@pytest.mark.parametrize("source", ["ffn.hip", "int8.hip"])
def test_no_scratch_and_one_wait_per_stage(tmp_path, source):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    flags = [f for f in BLD.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = tmp_path / "out.s"
    subprocess.run([hipcc, *flags, "-S", "--cuda-device-only", os.path.join(BLD.CSRC, source), "-o", str(out)],
                   check=True, capture_output=True)
    asm = out.read_text()
    sizes = re.findall(r"; ScratchSize: (\d+)", asm)
    assert len(sizes) >= 10 and set(sizes) == {"0"}
    assert "v_pk_fma_f32" not in asm and "v_pk_mul_f32" not in asm and "v_pk_add_f32" not in asm
    # basic blocks that hold products and loads into LDS: a stage of the steady loop
    loops = 0
    for block in re.split(r"\n\.LBB\w+:", asm):
        products = len(re.findall(r"\bv_mfma", block))
        if products >= 16 and "global_load_lds_dwordx4" in block and "s_barrier" in block:
            loops += 1
            assert len(re.findall(r"s_waitcnt[^\n]*vmcnt", block)) <= 1, block[:400]
    assert loops >= 4
