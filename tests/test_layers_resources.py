"""Scratch memory of the layers' kernels, from the metadata that the compiler
writes into the library's code objects (no GPU needed)."""
import os
import re

import pytest

import paper_2507_02006_amd as pkg
from test_kernel_resources import code_objects, kernels

NAMES = "rms_|quantize|tiles8|join8|rows8|zero8|pack8|logp_|grad_norm|grad_squares|grad_scale"


def test_kernels_of_layers_stay_in_registers():
    lib = os.path.join(os.path.dirname(pkg.__file__), "libaires.so")
    if not os.path.exists(lib):
        pytest.skip("library not built")
    with open(lib, "rb") as f:
        found = {n: k for elf in code_objects(f.read()) for n, k in kernels(elf).items()}
    spilled, seen = {}, 0
    for n, k in found.items():
        m = re.search(r"_GLOBAL__N_1\d+(k_(?:%s)\w*?)(?=I|E|P|v)(\w*)" % NAMES, n)
        if m:
            seen += 1
            if k[".private_segment_fixed_size"]:
                spilled[m[1], tuple(int(x) for x in re.findall(r"L[ib](\d+)E", m[2]))] = k[".private_segment_fixed_size"]
    assert seen > 200
    # the widest rows of the norm's backward pass in mixed types (1024 threads have 128
    # registers each), and two registers of the largest tiles
    most = {("k_rms_backward", (0, 2, 3, 0)): 104, ("k_tiles8", (256, 256, 128, 64, 2, 0, 0)): 16}
    for key, size in spilled.items():
        assert size <= most.get(key, 0), (key, size)
