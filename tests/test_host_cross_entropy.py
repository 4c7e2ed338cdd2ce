"""The cross entropy's kernels compiled as host code (host_hip/), with a plain form of the matrix
instructions and of the loads that write LDS, on arrays that end before or begin behind a page
without access: an access past any array, the parts of the workspace among them, ends the program,
and results are compared with the definition. And its plans over a range of sizes."""
import os
import subprocess

import pytest

from tests import host_hip_build as host

pytestmark = pytest.mark.skipif(host.compiler() is None, reason="needs clang")

# GPU instructions and what stands for them on the host
FORMS = [
    ("return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;",
     "return host_hip::lds_at(p);"),
    ('asm volatile("s_mov_b32 m0, %0\\n\\ts_nop 0\\n\\tglobal_load_lds_dwordx4 %1, %2"\n'
     '                     : : "s"(to), "v"(offset[j]), "s"(from[j]) : "memory");',
     "host_hip::load_lds(to, from[j] + offset[j]);"),
    ('asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(decltype(steps)::n * S::kLoads)\n'
     '                     : "memory");', ";"),
    ('asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");', ";")]


@pytest.fixture(scope="module")
def xent(tmp_path_factory):
    folder = str(tmp_path_factory.mktemp("cross_entropy"))
    for name in ("vocab_gemm.h", "linear_cross_entropy.h"):
        with open(os.path.join(host.CSRC, name)) as f:
            text = f.read()
        if name == "vocab_gemm.h":
            for gpu, plain in FORMS:
                assert text.count(gpu) == 1, gpu
                text = text.replace(gpu, plain)
        with open(os.path.join(folder, name), "w") as f:
            f.write(host.as_host_code(text))
    out = os.path.join(folder, "cross_entropy")
    r = subprocess.run(
        [host.compiler(), "-x", "c++", "-std=c++20", "-O1", "-w", "-ffp-contract=off",
         "-I" + host.HOST_HIP, "-I" + folder, "-I" + host.CSRC,
         "-I" + os.path.join(host.ROOT, "include"),
         os.path.join(host.HOST_HIP, "cross_entropy.cpp"),
         os.path.join(host.CSRC, "linear_cross_entropy.cpp"), "-o", out],
        capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return out


def run(exe, *args):
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])


def test_no_rows(xent):
    run(xent, "empty")


def test_plans(xent):
    run(xent, "plans")


# (dtype, rows, words, width, apart, shift, tiles, piece, uneven). Tiles 0 to 4: 256 x 256, 128 x 128,
# 128 x 64, 64 x 64 and 16 x 128 (F64 has no first); -1: the plan's, split where it says so. Rows
# that go straight to LDS (whole steps of 128 bytes at whole vectors) and through registers.
@pytest.mark.parametrize("case", [
    (1, 1, 1, 1, 0, 0, -1, 0, 0), (2, 1, 9, 64, 0, 0, -1, 0, 0), (3, 3, 5, 7, 0, 0, -1, 0, 1),
    (0, 17, 70, 16, 0, 0, -1, 0, 1), (0, 65, 63, 33, 2, 1, -1, 0, 1), (1, 64, 64, 32, 0, 0, -1, 0, 0),
    (1, 70, 131, 45, 3, 1, -1, 0, 1), (2, 66, 129, 128, 64, 0, -1, 0, 1),
    (3, 130, 257, 100, 0, 1, -1, 0, 0), (2, 33, 300, 31, 1, 0, -1, 0, 1),
    # products split along their long axes
    (2, 5, 40, 1600, 0, 0, -1, 0, 1), (3, 20, 19, 1541, 1, 0, -1, 0, 0), (1, 3, 70, 520, 0, 0, -1, 0, 1),
    (0, 2, 9, 261, 0, 0, -1, 0, 0), (2, 700, 5, 20, 0, 0, -1, 0, 1), (1, 9, 900, 12, 0, 0, -1, 0, 1),
    # every tile
    (2, 257, 300, 64, 0, 0, 0, 0, 1), (1, 130, 270, 33, 0, 0, 0, 0, 0), (3, 100, 60, 70, 0, 1, 0, 0, 1),
    (2, 129, 140, 128, 0, 0, 1, 0, 0), (0, 70, 130, 17, 0, 0, 1, 0, 1), (1, 131, 70, 64, 0, 0, 2, 0, 1),
    (0, 150, 67, 32, 0, 0, 2, 0, 0), (2, 70, 130, 65, 0, 0, 3, 0, 1), (3, 63, 65, 256, 0, 0, 3, 0, 0),
    (2, 33, 130, 320, 0, 0, 4, 0, 1), (0, 16, 129, 20, 0, 0, 4, 0, 0), (1, 17, 260, 96, 0, 0, 4, 0, 1),
    # pieces of the vocabulary
    (2, 20, 700, 40, 0, 0, -1, 256, 1), (1, 33, 530, 32, 0, 0, -1, 256, 0),
    (0, 9, 300, 16, 0, 0, 1, 256, 1), (3, 17, 513, 64, 0, 0, 3, 256, 1)])
def test_cross_entropy(xent, case):
    run(xent, "run", *case)
