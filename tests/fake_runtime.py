"""The library's own host code against a runtime of two imaginary devices
(fake_cudart.cpp), for tests on a machine without a GPU.  ``run`` executes a
script in a process of its own, where the calls below and ``log()``, the
runtime calls made so far, are at hand."""
import glob
import os
import shutil
import subprocess
import sys

import pytest

from paper_2411_12364_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import ctypes as C
import sys
from paper_2411_12364_gb300 import binding as b
lib = b.load(sys.argv[1])
lib.fake_log.restype = C.c_char_p
FAKE = 1 << 20


def log():
    return lib.fake_log().decode().splitlines()


def attend(dtype=b.BF16, max_new=1, dim=128):
    c = b.KVCache(FAKE, FAKE, 64, 2, 16, dim, dtype)
    need = lib.ultramem_paged_attention_workspace(dtype, 4, 2, dim, max_new)
    return lib.ultramem_paged_attention(C.byref(c), FAKE, 4 * dim, 4, FAKE, FAKE, FAKE, 4, 1,
                                        max_new, max_new, 1.0, 2 * FAKE, None, 3 * FAKE, need, None)


def norm_args(dim=2048):
    return b.BlockNormArgs(FAKE, None, None, None, None, None, dim, dim, 64, dim, b.BF16, 0, 1, 1,
                           0, 1.0, 1.0, 1e-5)


def norm():
    a = norm_args()
    return lib.ultramem_block_norm(C.byref(a), 2 * FAKE, 3 * FAKE, 4 * FAKE, None)


def grad(dim=2048):
    a = norm_args(dim)
    need = lib.ultramem_block_norm_backward_workspace(64, dim)
    return lib.ultramem_block_norm_backward(
        C.byref(a), 2 * FAKE, 3 * FAKE, dim, 4 * FAKE, dim, 5 * FAKE, 6 * FAKE, None, 7 * FAKE,
        None, 8 * FAKE, None, 9 * FAKE, need, None)


CALLS = dict(decode=attend, chunk=lambda: attend(max_new=64), narrow=lambda: attend(dim=64),
             fp32=lambda: attend(dtype=b.F32, max_new=64), wide=lambda: attend(dim=256), norm=norm,
             grad=grad, wide_grad=lambda: grad(8192))
"""


@pytest.fixture(scope="module")
def fake_library(tmp_path_factory):
    compiler, toolkit = shutil.which("g++"), os.path.dirname(os.path.dirname(build.nvcc()))
    lib = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    objects = glob.glob(os.path.join(build.OBJDIR, "*.cu.o"))
    if len(objects) != len(build._sources()) or not build.up_to_date():
        build.build(force=True)
        objects = glob.glob(os.path.join(build.OBJDIR, "*.cu.o"))
    subprocess.run([compiler, "-std=c++17", "-fPIC", "-shared", "-I",
                    os.path.join(toolkit, "include"), "-Wl,--no-undefined", "-Wl,-Bsymbolic", "-o",
                    lib, os.path.join(ROOT, "tests", "fake_cudart.cpp"), *objects], check=True,
                   capture_output=True)
    return lib


def run(fake_library, body):
    """In a process of its own: what the library keeps starts empty."""
    out = subprocess.run([sys.executable, "-c", SCRIPT + body, fake_library], cwd=ROOT,
                         capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "done", out.stdout + out.stderr
