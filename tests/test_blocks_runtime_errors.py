"""CPU-only: a kernel whose LDS the HIP runtime refuses is an error of the call.  The HIP runtime's functions are replaced in a process of
its own, so that nothing reaches a device."""
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

CALLS = r"""
from paper_2408_10746_amd import binding as pb
L, A = pb.lib(), 1 << 20
out = []
for M, K, N in ((4096, 4096, 4096), (64, 4096, 4096)):
    out.append(L.pac_mx4_linear(A, M, K, K, 2 * A, 3 * A, N, None, 0, 1 << 40, pb.PAC_BF16, N, None))
    out.append(L.pac_mx4_linear_x4(A, 5 * A, M, K, 2 * A, 3 * A, N, None, 0, 1 << 40, pb.PAC_BF16, N, None))
for M in (1, 4096):
    out.append(L.pac_mx4_linear_dx(A, M, 4096, 4096, 2 * A, 3 * A, 4096, 1 << 40, pb.PAC_BF16, 4096, None))
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
    assert got.stdout.split()[-6:] == [want] * 6, got.stdout
