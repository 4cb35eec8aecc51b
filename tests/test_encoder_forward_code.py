"""Generated code of the encoder attention's forward kernel.  It leaves its output by way of the LDS that held its ring of blocks, so a barrier of the workgroup has to stand between
the last reads of values, of either sweep, and those stores: without one, a wave that is done overwrites values that a slower one still reads."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{head_dim: instructions of its forward kernel}"""
    out = str(tmp_path_factory.mktemp("code") / "encoder_attn.s")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-S",
                    "--cuda-device-only", os.path.join(ROOT, "paper_2509_22622_amd", "csrc", "encoder_attn.hip"), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    return {d: [line.split()[0] for line in re.search(rf"^_ZN2ll25ll_encoder_forward_kernelILi{d}E[^\n]*:[^\n]*\n([\s\S]*?)^\.Lfunc_end", text, re.M).group(1).splitlines()
                if re.match(r"\t[a-z]", line)] for d in (64, 128)}


@pytest.mark.parametrize("d", [64, 128])
def test_a_barrier_stands_behind_each_sweep(kernels, d):
    code = kernels[d]
    reads = [i for i, op in enumerate(code) if op.startswith("ds_read_b64_tr")]
    writes = [i for i, op in enumerate(code) if op.startswith("ds_write_b128") and i > reads[-1]]
    assert len(writes) >= d // 16, "the output's pieces"
    sweeps = [a for a, b in zip(reads, reads[1:]) if b - a > 200] + [reads[-1]]               # the last read of each sweep: a loop's reads stand close together
    assert len(sweeps) == 2, sweeps
    for last, until in zip(sweeps, [reads[reads.index(sweeps[0]) + 1], writes[0]]):
        assert "s_barrier" in code[last:until], f"nothing between a read of values at instruction {last} and {until}"
