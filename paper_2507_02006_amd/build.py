"""Builds libaires.so (gfx950, hipcc) and _calls.so (torch tensors, g++) in-tree."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libaires.so")
CALLS = os.path.join(HERE, "_calls.so")  # the training calls over torch tensors
SOURCES = [os.path.join(HERE, "csrc", n) for n in
           ("aires.cpp", "train.cpp", "layers.cpp", "kernels.hip", "narrow.hip", "spmm.hip", "normalize.hip", "scratch.hip",
            "layernorm.hip", "adamw.hip", "xent.hip", "xent_few.hip", "xent_rows.hip", "rmsnorm.hip",
            "quantize8.hip", "product8.hip", "logprobs.hip", "gradnorm.hip")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # packed fp32 instructions are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def _calls_command(out: str) -> list[str]:
    """g++ line of the module over torch tensors (host code only; it calls
    libaires.so, found next to it)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension as ext
    inc = [x for d in [*ext.include_paths(), sysconfig.get_paths()["include"]] for x in ("-isystem", d)]
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-DTORCH_EXTENSION_NAME=_calls",
            "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), *inc,
            os.path.join(HERE, "csrc", "calls.cpp"), "-o", out, "-L" + lib, "-ltorch_python", "-ltorch", "-ltorch_cpu",
            "-lc10"]


def build(force: bool = True) -> str:
    if force or not (os.path.exists(LIB) and os.path.exists(CALLS)):
        tmp, ctmp = LIB + ".tmp%d" % os.getpid(), CALLS + ".tmp%d" % os.getpid()
        with tempfile.TemporaryDirectory() as objs:
            # one compiler per source, all at once
            outs = [os.path.join(objs, os.path.basename(x) + ".o") for x in SOURCES]
            lines = [[HIPCC, *FLAGS, "-c", "-o", o, x] for x, o in zip(SOURCES, outs)]
            cobj = os.path.join(objs, "calls.o")
            whole = _calls_command(cobj)
            at = whole.index("-o") + 2
            lines.append([x for x in whole[:at] if x != "-shared"] + ["-c"])
            running = [subprocess.Popen(x) for x in lines]
            codes = [p.wait() for p in running]
            for x, rc in zip(lines, codes):
                if rc:
                    raise subprocess.CalledProcessError(rc, x)
            subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", "-Wl,-soname,libaires.so", "-o", tmp,
                                   *outs])
            subprocess.check_call(["g++", "-shared", "-o", ctmp, cobj, tmp, *whole[at:], "-Wl,-rpath,$ORIGIN"])
        os.replace(tmp, LIB)
        os.replace(ctmp, CALLS)
    return LIB


if __name__ == "__main__":
    print(build())
