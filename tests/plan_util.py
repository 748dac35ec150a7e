"""The launches' arithmetic (csrc/hb_linear_plan.hpp, csrc/hb_append_plan.hpp) for tests, compiled for the host."""
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

import pytest

from paper_2309_04875_amd import build

SOURCE = r"""
#include "hb_append_plan.hpp"
#include "hb_linear_plan.hpp"
using namespace hb;
extern "C" {
int form(int flush, uint64_t rows, uint64_t outs) { return linear_form(flush, rows, outs); }
uint64_t row_tiles(int form, uint64_t rows) { return linear_row_tiles(kLinearForm[form], rows); }
uint64_t groups(int form, uint64_t outs) { return linear_groups(kLinearForm[form], outs); }
uint64_t launch_tiles(uint64_t groups, uint64_t threads) { return linear_launch_tiles(groups, threads); }
uint32_t pair(uint32_t block, uint32_t count) { return linear_pair(block, count); }
uint32_t append_blocks(uint64_t tokens, uint64_t groups) { return append_shape(tokens, groups).blocks; }
uint64_t append_tokens(uint64_t stored, uint64_t asked) { return append_launch_tokens(stored, asked); }
}
"""


@functools.lru_cache(maxsize=None)
def plan():
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    with tempfile.TemporaryDirectory() as where:
        source, library = os.path.join(where, "plan.cpp"), os.path.join(where, "plan.so")
        with open(source, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + build.CSRC, source, "-o", library], check=True)
        lib = ctypes.CDLL(library)
    u32, u64, i = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int
    for name, result, *args in (("form", i, i, u64, u64), ("row_tiles", u64, i, u64), ("groups", u64, i, u64), ("launch_tiles", u64, u64, u64), ("pair", u32, u32, u32),
                                ("append_blocks", u32, u64, u64), ("append_tokens", u64, u64, u64)):
        getattr(lib, name).restype, getattr(lib, name).argtypes = result, args
    return lib
