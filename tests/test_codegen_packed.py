"""The walk of test_codegen_hazards over the kernels of the calls on packed batches and of the head's gradient."""
import concurrent.futures
import os
import subprocess

import pytest

from paper_2601_17261_amd import build as B
from test_codegen_hazards import barrier_faults, functions, wait_state_faults

SOURCES = ["glue_packed.hip", "glue_norm_rope.hip", "ce_few.hip", "ce_grad.hip", "ce_grad_f32.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")

    def one(src):
        out = os.path.join(str(d), src.replace(".hip", ".s"))
        subprocess.run([B.HIPCC] + B.FLAGS + ["-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            return functions(f.read())
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(one, SOURCES)))


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
