"""Code-generation checks of the norm, the gate, the routing's losses and AdamW (host only: hipcc emits the gfx950
assembly, nothing runs).  No kernel spills to scratch memory or holds packed fp32 arithmetic, and the loop over strips of
dx has as many memory instructions as the wait for a strip's loads counts: those of one more strip and the stores of
two."""
import os
import re
import subprocess

import pytest

from paper_2609_21483_amd import build as BLD


def assembly(tmp_path, source):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    flags = [f for f in BLD.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = tmp_path / "out.s"
    subprocess.run([hipcc, *flags, "-S", "--cuda-device-only", os.path.join(BLD.CSRC, source), "-o", str(out)],
                   check=True, capture_output=True)
    return out.read_text()


@pytest.mark.parametrize("source,kernels", [("norm.hip", 13), ("router.hip", 20), ("adamw.hip", 2)])
def test_no_scratch_and_no_packed_fp32(tmp_path, source, kernels):
    asm = assembly(tmp_path, source)
    sizes = re.findall(r"; ScratchSize: (\d+)", asm)
    assert len(sizes) >= kernels and set(sizes) == {"0"}
    assert "v_pk_fma_f32" not in asm and "v_pk_mul_f32" not in asm and "v_pk_add_f32" not in asm
    if source != "router.hip":
        return
    for kc, broad in ((1, 0), (2, 0), (3, 0), (3, 1), (4, 0), (4, 1)):
        start = re.search(r"\n(_ZN\w*gate_grad_kernelILi%dELb%d\w*):" % (kc, broad), asm)
        body = asm[start.end():asm.index(".Lfunc_end", start.end())]
        # the strips' loop: from its wait for a strip behind which there are one more strip's loads and 8 stores, to its end
        loop = body[body.index(f"vmcnt({kc + 8})"):body.rindex("s_endpgm")]
        assert len(re.findall(r"\bv_mfma", loop)) == 8 * kc
        assert len(re.findall(r"global_load_lds_dwordx4", loop)) == kc
        assert len(re.findall(r"global_store", loop)) == 4
        assert len(re.findall(r"global_load(?!_lds)|buffer_|flat_", loop)) == 0
        assert "vmcnt" not in loop[6:]  # and no other wait
