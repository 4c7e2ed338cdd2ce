"""Builds a kernel file of the library as a program for the host, with the header in
host_hip/ in HIP's place. The file itself is compiled; only what no host compiler takes is
rewritten: barriers for the compiler's register allocation go, and GPU instructions end the
program."""
import os
import re
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2509_02197_amd", "csrc")
HOST_HIP = os.path.join(HERE, "host_hip")


def compiler():
    for c in ("/opt/rocm/llvm/bin/clang++", "clang++"):
        if shutil.which(c):
            return c
    return None


def as_host_code(text):
    text = re.sub(r'asm volatile\("" : [^;]*;', ";", text)
    text = re.sub(r"__shared__ (alignas\([^()]*(?:\([^()]*\))?[^()]*\))", r"\1 __shared__", text)
    # GPU instructions: no case here reaches them
    return re.sub(r'asm volatile\(\s*"(?!")[^;]*;', "std::abort();", text)


def build(name, folder):
    """The program of host_hip/<name>.cpp, which includes csrc/<name>.hip."""
    with open(os.path.join(CSRC, name + ".hip")) as f:
        text = as_host_code(f.read())
    with open(os.path.join(folder, name + ".host.inc"), "w") as f:
        f.write(text)
    out = os.path.join(folder, name)
    r = subprocess.run([compiler(), "-x", "c++", "-std=c++20", "-O1", "-w", "-ffp-contract=off",
                        "-I" + HOST_HIP, "-I" + folder, "-I" + CSRC,
                        "-I" + os.path.join(ROOT, "include"),
                        os.path.join(HOST_HIP, name + ".cpp"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return out
