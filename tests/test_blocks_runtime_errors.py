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


SHARED = r"""
import ctypes as C
from paper_2408_10746_amd import binding as pb
L, A, FAR = pb.lib(), 1 << 20, 1 << 40
OK, RANGE = pb.PAC_OK, pb.PAC_ERR_RANGE
M, K, N = 100, 512, 256                                   # rows of 1024 bytes of x, 512 of y in bf16
X, W, S, B = FAR, FAR + (1 << 30), FAR + (2 << 30), FAR + (3 << 30)
wb, sb = N * 256, N * 16

def lin(y, x=X, sx=K, sy=N, M=M, ydt=pb.PAC_BF16):
    return L.pac_mx4_linear(x, M, K, sx, W, S, N, B, 0, y, ydt, sy, None)
def lin4(y, x=X, xs=X + (1 << 20)):
    return L.pac_mx4_linear_x4(x, xs, M, K, W, S, N, B, 0, y, pb.PAC_BF16, N, None)
def linq(y, x=X, ws=A, xdt=pb.PAC_BF16):
    return L.pac_mx4_linear_qx(x, xdt, M, K, K, W, S, N, B, 0, y, pb.PAC_BF16, N, ws, M * 272, None)
def dx(out, dy=X):
    return L.pac_mx4_linear_dx(dy, M, N, N, W, S, K, out, pb.PAC_BF16, K, None)

def want(status, *got):
    assert all(g == status for g in got), (status, got)

# apart, and end to end
want(OK, lin(A), lin(X + M * K * 2), lin(X - M * N * 2), lin(W + wb), lin(W - M * N * 2), lin(B + 4 * N))
want(RANGE, lin(X), lin(X + M * K * 2 - 2), lin(X - M * N * 2 + 2), lin(W), lin(W + wb - 16), lin(S + sb - 8), lin(B + 4 * N - 4), lin(B - 2 * M * N + 16))
# side by side in one buffer: x's columns, then y's; fp32 beside bf16; one value into each other; rows of other distances
want(OK, lin(X + 2 * K, sx=K + N, sy=K + N), lin(X + 2 * K, sx=K + 2 * N, sy=K // 2 + N, ydt=pb.PAC_F32), lin(X + 1024, sx=1024, sy=2048, M=50))
want(RANGE, lin(X + 2 * K - 2, sx=K + N, sy=K + N), lin(X + 2 * K, sx=K + N - 8, sy=K + N - 8), lin(X + 2 * K, sx=K + 2 * N, sy=K + N), lin(X + 1024, sx=1024, sy=1024 + 512))
want(OK, lin4(A), lin4(X + M * 256), lin4(X + (1 << 20) + M * 16))
want(RANGE, lin4(X + M * 256 - 2), lin4(X + (1 << 20) + M * 16 - 2), lin4(W), lin4(S))
want(OK, linq(2 * A), linq(A + M * 272), linq(A - M * N * 2))
want(RANGE, linq(A), linq(A + M * 272 - 2), linq(2 * A, ws=X), linq(2 * A, ws=W), linq(2 * A, ws=X + 2 * M * K, xdt=pb.PAC_F32), linq(X))
want(OK, dx(A), dx(X + 2 * M * N))
want(RANGE, dx(X), dx(X + 2 * M * N - 2), dx(W + wb - 2), dx(S))
def conv(x, codes=W, scales=S, stride=K):
    one = L.pac_mx4_quantize(x, pb.PAC_BF16, N, K, stride, codes, scales, None)
    assert one == L.pac_mx4_dequantize(codes, scales, N, K, x, pb.PAC_BF16, stride, None)
    return one
want(OK, conv(X), conv(W + wb), conv(X, scales=W + wb))
want(RANGE, conv(W), conv(W + wb - 2), conv(S), conv(X, scales=W + wb - 8), conv(X, codes=X + 2 * N * K - 16))

d, rows = 64, 10
by = 4 * d * rows
P = [FAR + (k << 20) for k in range(6)]
b = pb.pac_block_norm(d, pb.PAC_F32, 0, d, 1e-5, *P)
x, o, dy, dn = (FAR + (32 + k << 20) for k in range(4))
def fwd(y=A, n=2 * A, x=x, o=o):
    return L.pac_block_norm_forward(C.byref(b), rows, x, o, y, n, None)
want(OK, fwd(), fwd(y=x), fwd(n=o), fwd(y=x, n=o), fwd(y=o, n=x), fwd(y=x + by), fwd(y=None), fwd(n=2 * A, y=2 * A), fwd(y=P[0] + 4 * d))
want(RANGE, fwd(y=x + 4 * d), fwd(n=o - 4 * d), fwd(y=A, n=A + 4 * d), fwd(y=P[0]), fwd(n=P[5] + 4 * d - 4), fwd(y=P[3]))
need = pb.pac_block_norm_workspace_bytes(b, rows)
G = [FAR + (64 + k << 20) for k in range(6)]
def bwd(dx=A, do=2 * A, g=G, ws=3 * A):
    return L.pac_block_norm_backward(C.byref(b), rows, x, o, dy, dn, dx, do, *g, ws, need, None)
want(OK, bwd(), bwd(dx=dy), bwd(do=dn), bwd(dx=dn, do=dy), bwd(dx=x, do=o), bwd(dx=None, do=None), bwd(g=[None] * 6, ws=None))
want(RANGE, bwd(dx=dy + 4 * d), bwd(do=dn + 4 * d), bwd(dx=A, do=A), bwd(dx=A, do=A + 4 * d), bwd(dx=P[2]), bwd(ws=x), bwd(ws=A), bwd(ws=G[0] - 16), bwd(ws=P[4]))
for k in range(6):
    for other in (P[k], P[(k + 1) % 6], x, dn, 2 * A, G[(k + 1) % 6]):
        want(RANGE, bwd(g=G[:k] + [other] + G[k + 1:]))
print("fine")
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
def test_results_that_share_memory_with_operands_are_refused(tmp_path):
    """Addresses alone, nothing is read: kernels are launched by nobody here."""
    src, so = tmp_path / "runtime.c", tmp_path / "runtime.so"
    src.write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, (str(so), os.environ.get("LD_PRELOAD")))), PAC_TEST_ATTRIBUTE="0", PYTHONPATH=ROOT)
    got = subprocess.run([sys.executable, "-c", SHARED], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=ROOT, timeout=120)
    assert got.returncode == 0 and got.stdout.split()[-1] == "fine", got.stdout
