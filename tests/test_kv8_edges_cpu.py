"""The paged 8-bit cache's host arithmetic and build at the edges, without a GPU."""
import ctypes as C
import os
import shutil
import subprocess
import textwrap

import numpy as np
import pytest

from oracle import kv8_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HDR = os.path.join(ROOT, "paper_2605_24011_b200", "csrc")


def _compiled(tmp_path, name, text, *more):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, out = tmp_path / (name + ".cpp"), tmp_path / name
    src.write_text(textwrap.dedent(text))
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", *more, "-I", HDR, str(src), "-o", str(out)], check=True)
    return str(out)


def test_up11_of_all_magnitudes(tmp_path):
    """The scale's rounding against the definition, subnormals among them."""
    lib = C.CDLL(_compiled(tmp_path, "up11.so", r"""
        #include "aq_kv8_runs.h"
        extern "C" uint32_t up11(uint32_t x) { return aq::kv8_up11(x); }
    """, "-shared", "-fPIC"))
    lib.up11.argtypes, lib.up11.restype = [C.c_uint32], C.c_uint32
    g = np.random.default_rng(1)
    edges = [x for e in range(0, 31) for x in (2 ** e - 1, 2 ** e, 2 ** e + 1) if x < 0x7F000000]
    # a block's need where its largest magnitude is 1.5 * 2^-125 and smaller
    halves = [int((np.float32(m) / np.float32(127)).view(np.uint32)) for m in (1.5 * 2.0 ** -125, 2.0 ** -133, 2.0 ** -126, 2.0 ** -119)]
    for x in edges + halves + [0, 0x7FFFFF, 0x800000, 0x7F000000] + [int(v) for v in g.integers(0, 0x7F000000, 3000)] + [int(v) for v in g.integers(0, 0x800000, 3000)]:
        got, want = lib.up11(x), O.up11(np.uint32(x).view(np.float32))
        assert got == int(want.view(np.uint32)), hex(x)
    assert lib.up11(0x7F800000) == 0x7F800000
