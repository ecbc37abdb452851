"""The cross entropy's copies of its operands read rows of 8 columns at a time up
to the next multiple of 64: the kernel's own load, compiled for the host, over
matrices that end where their memory ends."""
import os
import subprocess

import pytest

from paper_2411_12364_gb300 import build

PROGRAM = r"""
#include <sys/mman.h>
#include <unistd.h>
#include <cstdio>
#include <vector>
#include "um_planes.cuh"

template <typename T> int check(int R, int D, int ld) {
    const size_t page = (size_t)sysconf(_SC_PAGESIZE);
    const size_t bytes = ((size_t)(R - 1) * ld + D) * sizeof(T), room = (bytes + page - 1) / page * page;
    char *at = (char *)mmap(nullptr, room + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS,
                            -1, 0);
    if (at == MAP_FAILED || mprotect(at + room, page, PROT_NONE)) return 1;
    T *src = (T *)(at + room - bytes);
    for (size_t i = 0; i < bytes / sizeof(T); ++i) src[i] = T((float)(i % 251) + 1.f);
    const bool wide = D % 8 == 0 && (uintptr_t)src % 16 == 0 && ld * sizeof(T) % 16 == 0;
    int bad = 0;
    for (int r = 0; r < R; ++r)
        for (int c = 0; c < (D + 63) / 64 * 64; c += 8) {
            const um::Piece<T> p = um::read_piece(src + (size_t)r * ld, c, D, wide);
            T v[8];
            memcpy(v, &p, sizeof v);
            for (int k = 0; k < 8; ++k)
                bad += (float)v[k] != (c + k < D ? (float)(((size_t)r * ld + c + k) % 251) + 1.f : 0.f);
        }
    munmap(at, room + page);
    return bad;
}

int main() {
    int bad = 0;
    for (int D = 1; D <= 200; ++D)
        for (int R : {1, 2, 16})
            for (int gap : {0, 1, 8, 56}) bad += check<float>(R, D, D + gap) + check<__nv_bfloat16>(R, D, D + gap);
    printf(bad ? "wrong\n" : "done\n");
    return bad != 0;
}
"""


@pytest.mark.parametrize("optimise", ["-O0", "-O2"])
def test_nothing_past_a_row_is_read(tmp_path, optimise):
    source, program = tmp_path / "planes.cu", tmp_path / "planes"
    source.write_text(PROGRAM)
    subprocess.run([build.nvcc(), *build.ARCH, "-std=c++17", optimise, "-I", build.CSRC,
                    str(source), "-o", str(program)], check=True, capture_output=True)
    out = subprocess.run([str(program)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "done", (out.returncode, out.stdout)
