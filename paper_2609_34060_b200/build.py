"""In-tree build of the CUDA library (libkvc.so) for sm_100a with nvcc.

``python -m paper_2609_34060_b200.build`` compiles every ``csrc/*.cu`` and links
them into ``paper_2609_34060_b200/libkvc.so``, and ``csrc/marshal.cpp`` into
``_marshal`` (the Python binding's argument blocks), whose file carries the interpreter's
tag as it is compiled against that one's headers.  The shared objects sit beside the sources
(they are git-ignored but travel with a snapshot of the tree).
"""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libkvc.so")
EXT_SUFFIX = sysconfig.get_config_var("EXT_SUFFIX")
MARSHAL = os.path.join(HERE, "_marshal" + EXT_SUFFIX)

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stamp(paths) -> str:
    h = hashlib.sha256()
    for p in sorted(paths):
        h.update(p.encode())
        with open(p, "rb") as f:
            h.update(f.read())
    h.update(" ".join(NVCC_FLAGS).encode())
    return h.hexdigest()


def _current(made: str, stamp_file: str, stamp: str) -> bool:
    return os.path.exists(made) and os.path.exists(stamp_file) and open(stamp_file).read() == stamp


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    srcs = sources()
    deps = srcs + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh", ".cpp"))]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "kvc.h"))
    stamp = _stamp(deps)
    stamp_file, marshal_stamp = os.path.join(OBJ, "stamp"), os.path.join(OBJ, "stamp" + EXT_SUFFIX)
    lib = force or not _current(LIB, stamp_file, stamp)
    marshal = lib or not _current(MARSHAL, marshal_stamp, stamp)     # another interpreter's may be there
    if not marshal:
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    nvcc = _nvcc()
    objs = []
    procs = []
    for s in srcs if lib else []:
        o = os.path.join(OBJ, os.path.basename(s)[:-3] + ".o")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if ptxas_info else []) + ["-c", s, "-o", o]
        if verbose:
            print(" ".join(cmd))
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(o)
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "marshal.cpp"), "-o", MARSHAL]
    procs.append((cmd[-3], subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for s, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose or ptxas_info:
            sys.stderr.write(out)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("compiler failed")
    with open(marshal_stamp, "w") as f:
        f.write(stamp)
    untagged = os.path.join(HERE, "_marshal.so")     # of a build that did not tell interpreters apart: any would import it
    if os.path.exists(untagged):
        os.remove(untagged)
    if lib:
        subprocess.check_call([nvcc, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"])
        with open(stamp_file, "w") as f:
            f.write(stamp)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, ptxas_info="--ptxas" in sys.argv))
