"""The cut of a group's rows into chunks, run on the CPU up to the most rows that a call may have."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

from paper_2604_15821_amd import build

MOST_ROWS = 2 ** 31 - 4097


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    compiler = shutil.which("g++") or shutil.which("c++") or shutil.which("clang++")
    if compiler is None:
        pytest.skip("no C++ compiler for the host")
    d = tmp_path_factory.mktemp("chunk_cut")
    src = d / "cut.cpp"
    src.write_text("#define __host__\n#define __device__\n"
                   f'#include "{os.path.join(build.CSRC, "chunk_cut.h")}"\n'
                   'extern "C" void cut(int rows, int most, int unit, int* out) {\n'
                   "  const janus::ChunkCut c = janus::chunk_cut(rows, most, unit);\n"
                   "  out[0] = c.each, out[1] = c.count;\n}\n")
    lib = d / "cut.so"
    subprocess.run([compiler, "-O2", "-fwrapv", "-std=c++17", "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    f = C.CDLL(str(lib)).cut

    def call(rows, most, unit=32):
        out = (C.c_int * 2)()
        f(rows, most, unit, out)
        return out[0], out[1]
    return call


def test_chunks_cover_every_group(cut):
    rng = random.Random(5)
    sizes = [0, 1, 31, 32, 33, 511, 512, 513, 16_223, 16_224, 16_225, 2 ** 30, 2 ** 31 - 131_073, 2 ** 31 - 131_072,
             2 ** 31 - 20_000, 2 ** 31 - 16_385, 2 ** 31 - 16_224, MOST_ROWS - 1, MOST_ROWS]
    sizes += [rng.randrange(MOST_ROWS) for _ in range(300)] + [MOST_ROWS - rng.randrange(200_000) for _ in range(300)]
    for most in (512, 544, 4096, 16_224, 16_384):
        for rows in sizes:
            each, count = cut(rows, most)
            if rows == 0:
                assert (each, count) == (0, 1)
                continue
            assert 0 < each <= most and each % 32 == 0, (rows, most)
            assert each * (count - 1) < rows <= each * count, (rows, most)
            assert count <= -(-rows // most), (rows, most)
