"""Scratch memory of the training kernels, from the metadata that the compiler
writes into the library's code objects (no GPU needed)."""
import os
import re

import pytest

import paper_2507_02006_amd as pkg
from test_kernel_resources import code_objects, kernels


def test_training_kernels_stay_in_registers_where_their_comments_say_so():
    lib = os.path.join(os.path.dirname(pkg.__file__), "libaires.so")
    if not os.path.exists(lib):
        pytest.skip("library not built")
    with open(lib, "rb") as f:
        found = {n: k for elf in code_objects(f.read()) for n, k in kernels(elf).items()}
    spilled, seen = {}, 0
    for n, k in found.items():
        m = re.search(r"_GLOBAL__N_1\d+(k_(?:ln_|adamw_|few|count|scores|rows|total|gradients|finish|zero|pack)\w*?)(?=I|E|P|v)(\w*)", n)
        if m:
            seen += 1
            if k[".private_segment_fixed_size"]:
                spilled[m[1], tuple(int(x) for x in re.findall(r"L[ib](\d+)E", m[2]))] = k[".private_segment_fixed_size"]
    assert seen > 200
    # the widest rows of the forward layer norm, dz in three planes, and (few.h) the most tiles
    most = {("k_ln_forward", (0, 8, 0)): 16, ("k_ln_forward", (0, 8, 1)): 16, ("k_scores", (1, 0, 256)): 64}
    for (name, args), size in spilled.items():
        if name == "k_few":
            kt, dt, waves, _, mode, kind = args
            assert kt * dt >= 8 and size <= 568, (args, size)
            assert mode in (1, 3) or size <= 16, (args, size)
            if args == (3, 4, 4, 2, 1, 0):
                assert size <= 104, size
        else:
            assert size <= most.get((name, args), 0), (name, args, size)
