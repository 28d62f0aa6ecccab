"""The walk of test_codegen_hazards over the kernels of the calls on packed batches and of the head's gradient."""
import concurrent.futures
import os
import re
import subprocess

import pytest

from paper_2601_17261_amd import build as B
from test_codegen_hazards import barrier_faults, functions, wait_state_faults

SOURCES = ["glue_packed.hip", "glue_norm_rope.hip", "ce_few.hip", "ce_grad.hip", "ce_grad_f32.hip"]
PRODUCTS = "gemm_bf16_aligned.hip"


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")

    def one(src):
        out = os.path.join(str(d), src.replace(".hip", ".s"))
        subprocess.run([B.HIPCC] + B.FLAGS + ["-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            return f.read()
    files = [PRODUCTS] + SOURCES
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(files)) as ex:
        return dict(zip(files, ex.map(one, files)))


@pytest.fixture(scope="module")
def kernels(assembly):
    return {src: functions(text) for src, text in assembly.items()}


@pytest.mark.parametrize("src", SOURCES)
def test_lds_writes_are_complete_at_barriers(kernels, src):
    found = {name: barrier_faults(*f) for name, f in kernels[src].items()}
    assert found
    assert not any(found.values()), "\n".join("%s: %s" % (n, v[0]) for n, v in found.items() if v)


@pytest.mark.parametrize("src", SOURCES)
def test_matrix_instructions_are_the_compilers(kernels, src):
    """None is written out, so that the compiler keeps the distances to their results"""
    assert not any(ins.mfma and ins.in_asm for body, _ in kernels[src].values() for ins in body)
    assert not any(wait_state_faults(*f) for f in kernels[src].values())


def test_the_gradients_products_spill_nothing_into_their_loop(assembly, kernels):
    """gemm_bf16_gradient_kernel<OUT, RAGGED>: the fp32 sums (OUT = 3) spill addresses that the ends of tiles read, the others nothing"""
    found = re.findall(r"\.name:\s+\S*gemm_bf16_gradient_kernelILi(\d)ELb\d\S*$.*?\.vgpr_spill_count:\s+(\d+)", assembly[PRODUCTS], re.M | re.S)
    assert len(found) == 6
    for out, spilled in found:
        assert int(spilled) <= (43 if out == "3" else 0), (out, spilled)
    for name, (body, succ) in kernels[PRODUCTS].items():
        if "gemm_bf16_gradient_kernel" not in name:
            continue
        loops = [body[t:i + 1] for i, s in enumerate(succ) for t in s if t <= i]
        slices = min((l for l in loops if any(ins.mfma for ins in l)), key=len)
        assert sum(ins.mfma for ins in slices) == 128, name
        assert not [ins.text for ins in slices if ins.op.startswith("scratch")], name
