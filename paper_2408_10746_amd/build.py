"""Build libpac.so (the HIP kernels and the C ABI) in-tree for gfx950."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libpac.so")
OBJ_DIR = os.path.join(_HERE, "_build")
SOURCES = ["pac_api.hip", "pac_kernels.hip", "pac_gram.hip", "pac_gram32.hip", "pac_probe.hip", "pac_plan.hip", "pac_quant.hip", "pac_ladder.hip",
           "pac_mx4.hip", "pac_norm.hip", "pac_attn.hip", "pac_kv4.hip"]
HEADERS = ["pac_gemm.h", "pac_mma.h", "pac_internal.h", "pac_span.h", "pac_attn_tile.h", os.path.join("..", "..", "include", "pac.h"),
           os.path.join("..", "..", "include", "pac_plan.h"),
           os.path.join("..", "..", "include", "pac_quant.h"),
           os.path.join("..", "..", "include", "pac_tier.h"),
           os.path.join("..", "..", "include", "pac_ladder.h"),
           os.path.join("..", "..", "include", "pac_mx4.h"),
           os.path.join("..", "..", "include", "pac_norm.h"),
           os.path.join("..", "..", "include", "pac_attn.h"),
           os.path.join("..", "..", "include", "pac_kv4.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]
# Products of attention's backward pass are read by the vector units one by one: their matrix instructions write vector registers, not
# accumulation registers that would have to be copied (4001 + 6143 tokens there and back, when it was chosen, 2645 -> 2500 us)
SOURCE_FLAGS = {"pac_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def _sources():
    return [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]


def _object(src: str) -> str:
    return os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")


def _command(src: str):
    return [hipcc()] + HIPCC_FLAGS + SOURCE_FLAGS.get(src, [])


def _made_alike(src: str) -> bool:
    """Was the source's object made by the command that would make it now?"""
    try:
        with open(_object(src) + ".command") as f:
            return f.read() == "\n".join(_command(src))
    except FileNotFoundError:
        return False


def is_stale() -> bool:
    if not os.path.exists(LIB) or not all(os.path.exists(_object(s)) and _made_alike(s) for s in _sources()):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in [os.path.join(CSRC, f) for f in _sources() + HEADERS] + [_object(s) for s in _sources()])


def _compile_one(src: str, force: bool) -> str:
    obj = _object(src)
    path = os.path.join(CSRC, src)
    if not force and os.path.exists(obj) and _made_alike(src):
        t = os.path.getmtime(obj)
        if all(os.path.getmtime(os.path.join(CSRC, f)) <= t for f in [src] + HEADERS):
            return obj
    tmp = obj + ".tmp%d" % os.getpid()
    res = subprocess.run(_command(src) + ["-c", "-o", tmp, path],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed on %s:\n%s" % (src, res.stdout))
    with open(tmp + ".command", "w") as f:
        f.write("\n".join(_command(src)))
    if os.path.exists(obj + ".command"):
        os.remove(obj + ".command")  # at no time does it speak of another object
    os.replace(tmp, obj)
    os.replace(tmp + ".command", obj + ".command")
    return obj


def build_lib(force: bool = True) -> str:
    """Compile every HIP source (one hipcc process per file, side by side) and link libpac.so.
    force=False recompiles only the objects older than their source or a header, or made with other flags."""
    if not force and not is_stale():
        return LIB
    os.makedirs(OBJ_DIR, exist_ok=True)
    srcs = _sources()
    with ThreadPoolExecutor(max_workers=min(len(srcs), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(lambda s: _compile_one(s, force), srcs))
    tmp = LIB + ".tmp%d" % os.getpid()
    res = subprocess.run([hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs,
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc link failed:\n" + res.stdout)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build_lib("--incremental" not in sys.argv))
