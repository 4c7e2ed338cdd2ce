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
