"""The walk of test_codegen_hazards over the kernels of a cache in pages and of verification, and what their loops over keys spill."""
import concurrent.futures
import os
import subprocess

import pytest

from paper_2601_17261_amd import build as B
from test_codegen_hazards import barrier_faults, functions, wait_state_faults

SOURCES = ["glue_cache.hip", "glue_paged.hip", "verify.hip"]


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
    assert not any(ins.mfma and ins.in_asm for body, _ in kernels[src].values() for ins in body)
    assert not any(wait_state_faults(*f) for f in kernels[src].values())


@pytest.mark.parametrize("src", SOURCES)
def test_no_access_goes_by_a_generic_address(kernels, src):
    """(a flat access waits for LDS too)"""
    assert not [ins.text for body, _ in kernels[src].values() for ins in body if ins.op.startswith("flat_")]


def test_the_loops_over_keys_reload_only_for_masked_tiles(kernels):
    """In the innermost loop with a tile's matrix instructions, which is that of the first of a kernel's two passes, a reload waits for the next tile's loads too: at most one, in the kernel
    of few rows and in the one of 256 where a mask is made, in the one of 128 before the loads"""
    found = 0
    for name, (body, succ) in kernels["glue_paged.hip"].items():
        if "join" in name:
            continue
        loops = [(t, i) for i, s in enumerate(succ) for t in s if t <= i]
        least = (32, 32) if "wide" in name else (16, 0)      # matrix instructions, exponentials
        tiles = [(t, i) for t, i in loops if sum(ins.mfma for ins in body[t:i + 1]) >= least[0] and sum(ins.op.startswith("v_exp") for ins in body[t:i + 1]) >= least[1]]
        t, i = min(tiles, key=lambda l: l[1] - l[0])
        found += 1
        assert sum(ins.op.startswith("scratch") for ins in body[t:i + 1]) <= 1, name
    assert found == 10


def test_loads_to_lds_that_are_written_out_have_their_wait_states(kernels):
    """five between a scalar register that a vector instruction writes and a load that reads it, one between m0 and a load to LDS: the compiler keeps them only where it knows of the load"""
    found = 0
    for name, (body, _) in kernels["glue_paged.hip"].items():
        for i, ins in enumerate(body):
            if ins.op.startswith("buffer_load") and ins.text.split()[-1] == "lds":
                found += 1
                assert ins.in_asm and "wide" in name
                assert body[i - 1].text.split()[:2] == ["s_nop", "4"] and body[i - 2].text.startswith("s_mov_b32 m0")
    assert found > 0
