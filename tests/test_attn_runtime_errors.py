"""CPU-only: attention's kernels whose LDS the HIP runtime refuses are errors of the call.  The HIP runtime's functions are replaced in a process
of its own, so that nothing reaches a device."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUNTIME = r"""
#include <stdlib.h>
int hipFuncSetAttribute(const void *f, int attribute, int value) { (void)f; (void)attribute; (void)value; return atoi(getenv("PAC_TEST_ATTRIBUTE")); }
int hipLaunchKernel() { return 0; }
int hipGetLastError(void) { return 0; }
"""

# the few-row kernels of 128 values a head, and 16 wavefronts' results of 16 heads, take more LDS than a launch has by default
CALLS = r"""
import ctypes as C
from paper_2408_10746_amd import binding as pb
L, F = pb.lib(), [(1 << 30) * (k + 1) for k in range(16)]
a = pb.pac_attn(2, 2, 128, 1, 0.1)
m = lambda *at: [x for p in at for x in (p, 256)]
out = [L.pac_attn_forward(a, F[0], 1, 300, *m(*F[1:5]), F[5], None),
       L.pac_attn_backward(a, F[0], 1, 300, *m(*F[1:5]), F[5], *m(*F[6:10]), F[10], 1 << 29, None)]
c = pb.pac_kv4(F[0], 100, 16, 1, 128)
out.append(L.pac_kv4_attend(c, 16, 0.1, 1, F[1], 64, 64, F[2], F[3], 2048, F[4], 2048, F[5], 1 << 29, None))
print(*out)
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
@pytest.mark.parametrize("attribute,want", [(1, "7"), (0, "0")])
def test_refused_lds_is_an_error(tmp_path, attribute, want):
    src, so = tmp_path / "runtime.c", tmp_path / "runtime.so"
    src.write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, (str(so), os.environ.get("LD_PRELOAD")))), PAC_TEST_ATTRIBUTE=str(attribute), PYTHONPATH=ROOT)
    got = subprocess.run([sys.executable, "-c", CALLS], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=ROOT, timeout=120)
    assert got.returncode == 0, got.stdout
    assert got.stdout.split()[-3:] == [want] * 3, got.stdout
