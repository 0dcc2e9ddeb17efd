"""CPU-only: which kernels packed attention launches, by the grids that it asks for.  The HIP runtime's functions are replaced in a process of its own, so
that nothing reaches a device."""
import os
import shutil
import subprocess
import sys

import pytest

from attn_kernels import few, workgroups

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUNTIME = r"""
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
typedef struct { uint32_t x, y, z; } dim3;
int hipFuncSetAttribute(const void *f, int attribute, int value) { (void)f; (void)attribute; (void)value; return 0; }
int __hipPushCallConfiguration(dim3 blocks, dim3 threads, size_t lds, void *stream)
{
    (void)stream;
    printf("%u %u %zu ", blocks.x, threads.x, lds);
    return 1; /* goes no further */
}
int hipGetLastError(void) { return 0; }
"""

SIZES = [(heads, d, batch, rows, causal) for heads in (1, 2, 3, 5, 10, 12, 16, 20, 32, 40, 64, 128, 192) for d in (8, 32, 40, 64, 72, 96, 104, 128)
         for batch, rows in ((1, 19), (1, 127), (1, 128), (1, 700), (2, 300), (4, 511), (4, 512), (1, 1788), (3, 4096), (1, 8192), (16, 4096), (64, 3000))
         for causal in (False, True)]

CALLS = r"""
import ctypes as C, sys
from paper_2408_10746_amd import binding as pb
L, F = pb.lib(), [(1 << 40) * (k + 1) for k in range(12)]
libc = C.CDLL(None)
for line in sys.stdin:
    heads, d, batch, rows, causal = map(int, line.split())
    a, m = pb.pac_attn(heads, heads, d, causal, 0.1), lambda *at: [x for p in at for x in (p, heads * d)]
    assert L.pac_attn_forward(a, F[0], batch, rows, *m(*F[1:5]), F[5], None) == 0
    libc.puts(b"")
    assert L.pac_attn_backward(a, F[0], batch, rows, *m(*F[1:5]), F[5], *m(*F[6:10]), F[10], 1 << 40, None) == 0
    libc.puts(b"")
libc.fflush(None)
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
def test_the_rule_is_the_librarys(tmp_path):
    src, so = tmp_path / "runtime.c", tmp_path / "runtime.so"
    src.write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, (str(so), os.environ.get("LD_PRELOAD")))), PYTHONPATH=ROOT)
    calls = "".join(" ".join(str(int(x)) for x in s) + "\n" for s in SIZES)
    got = subprocess.run([sys.executable, "-c", CALLS], input=calls, env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, cwd=ROOT, timeout=120)
    assert got.returncode == 0, got.stderr
    launches = [[tuple(map(int, words[i:i + 3])) for i in range(0, len(words), 3)] for words in map(str.split, got.stdout.splitlines())]
    assert len(launches) == 2 * len(SIZES)
    for size, forward, backward in zip(SIZES, launches[::2], launches[1::2]):
        assert len(forward) == 1 and len(backward) in (2, 3), size
        for blocks, threads, lds in (forward[0], backward[0]):  # dq comes first; LDS asked for at the launch is the few rows' kernels'
            assert (blocks, threads, lds > 0) == (workgroups(*size), 256, few(*size)), size
    assert {few(*s) for s in SIZES} == {False, True}
