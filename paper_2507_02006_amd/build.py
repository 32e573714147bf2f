"""Builds libaires.so (gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libaires.so")
SOURCES = [os.path.join(HERE, "csrc", n) for n in
           ("aires.cpp", "train.cpp", "kernels.hip", "narrow.hip", "spmm.hip", "normalize.hip", "scratch.hip",
            "layernorm.hip", "adamw.hip", "xent.hip", "xent_few.hip")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # packed fp32 instructions are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def build(force: bool = True) -> str:
    if force or not os.path.exists(LIB):
        tmp = LIB + ".tmp%d" % os.getpid()
        with tempfile.TemporaryDirectory() as objs:
            # one compiler per source, all at once
            outs = [os.path.join(objs, os.path.basename(x) + ".o") for x in SOURCES]
            running = [subprocess.Popen([HIPCC, *FLAGS, "-c", "-o", o, x]) for x, o in zip(SOURCES, outs)]
            codes = [p.wait() for p in running]
            for x, rc in zip(SOURCES, codes):
                if rc:
                    raise subprocess.CalledProcessError(rc, "%s %s" % (HIPCC, x))
            subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp, *outs])
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
