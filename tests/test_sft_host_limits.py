"""Arguments of the supervised fine-tuning calls at the ends of their range, and what they refuse before any launch (no GPU)."""
import ctypes as C
import subprocess
import sys

import pytest

FAKE = 0x10000   # a non-null, 256-byte aligned address that is never dereferenced on these paths
P = C.c_void_p


@pytest.fixture(scope="module")
def b():
    from paper_2403_17031_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("M", [1, 2, 3, 100, 9000])
def test_any_number_of_rows_may_be_asked_for_in_a_piece(b, M):
    """More than there are: one piece. (In a process of its own: a division by zero would end this one.)"""
    code = "from paper_2403_17031_b200 import binding as b; print(b.lmhead_xent_scratch_bytes(%d, 64, 1000, %%d))" % M
    most, whole = [subprocess.run([sys.executable, "-c", code % rows], capture_output=True, text=True) for rows in (2 ** 63 - 1, M)]
    assert whole.returncode == 0 and (most.returncode, most.stdout) == (0, whole.stdout)
