"""Which phase a kernel waits for before it gives up its shared memory after a wait that ran out: the one that the last load into
each stage completes.  On the CPU, with the kernels' own arithmetic and a model of the barriers' phases."""
import ctypes as C
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_04652_b200", "csrc")


@pytest.fixture(scope="module")
def last_fill_parity(tmp_path_factory):
    out = tmp_path_factory.mktemp("ring")
    src, so = out / "ring.cpp", out / "ring.so"
    src.write_text('#include "csp_ring.cuh"\n'
                   'extern "C" int parity(uint32_t n, uint32_t stages, uint32_t s) { return csp::dev::last_fill_parity(n, stages, s); }\n')
    subprocess.check_call(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)])
    return C.CDLL(str(so)).parity


class Barrier:
    """One load per phase.  A parity wait ends when the phase in front of the current one has that parity."""

    def __init__(self):
        self.complete = 0

    def wait_ends(self, parity):
        return (self.complete - 1) % 2 == parity


@pytest.mark.parametrize("stages", [1, 2, 3, 4, 5, 7, 8])
def test_the_last_load_of_every_stage_is_waited_for(last_fill_parity, stages):
    for issued in range(0, 5 * stages + 2):
        for s in range(stages):
            mine = [i for i in range(issued) if i % stages == s]
            parity = last_fill_parity(issued, stages, s)
            if not mine:
                assert parity == -1
                continue
            bar = Barrier()
            bar.complete = len(mine) - 1                # all but the last one have landed
            assert not bar.wait_ends(parity), (issued, s)
            assert bar.wait_ends(parity ^ 1)            # what made a wait for either parity no wait at all
            bar.complete += 1
            assert bar.wait_ends(parity), (issued, s)


def test_counts_near_the_end_of_32_bits(last_fill_parity):
    top = 2 ** 32 - 1
    assert last_fill_parity(top, 4, 3) == ((top - 4) // 4) % 2
    assert last_fill_parity(top, 1, 0) == (top - 1) % 2


def test_no_kernel_waits_for_either_parity():
    """`neither parity is complete` is never true, so a loop on it ends at once."""
    either = re.compile(r"!\s*mbar_try_wait\(([^,;]+), 0\)\s*&&\s*!\s*mbar_try_wait\(\1, 1\)")
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            assert not either.search(f.read()), name


def test_every_kernel_that_fills_a_ring_drains_it():
    """After its last barrier, so that a wait that ran out behind the last load is seen too."""
    for name in ("csp_chunk.cu", "csp_chunk_few.cu", "csp_decode.cu", "csp_score.cu", "csp_score_persist.cu", "csp_score_tc.cu"):
        with open(os.path.join(CSRC, name)) as f:
            src = f.read()
        assert "mbar_expect_tx" in src and "drain_ring(" in src, name
