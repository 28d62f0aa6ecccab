"""The walk of test_codegen_hazards for LDS writes at barriers, over the sources that neither it nor test_codegen_packed takes."""
import concurrent.futures
import os
import subprocess

import pytest

import test_codegen_hazards as hazards
import test_codegen_packed as packed
from paper_2601_17261_amd import build as B

# (the entry points have no kernels)
SOURCES = [s for s in B.SOURCES if s not in hazards.SOURCES + packed.SOURCES + ["agzo_api.hip"]]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")

    def one(src):
        out = os.path.join(str(d), src.replace(".hip", ".s"))
        subprocess.run([B.HIPCC] + B.FLAGS + ["-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            return hazards.functions(f.read())
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(one, SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_lds_writes_are_complete_at_barriers(kernels, src):
    found = {name: hazards.barrier_faults(*f) for name, f in kernels[src].items()}
    assert found
    assert not any(found.values()), "\n".join("%s: %s" % (n, v[0]) for n, v in found.items() if v)
