"""The token operators' kernels compiled as host code (host_hip/), on arrays that end before or
begin behind a page without access: an access past any array ends the program, and results are
compared with the definitions. Extents are those where segments, chunks, slabs and vectors end
unevenly."""
import subprocess

import pytest

from tests import host_hip_build as host

pytestmark = pytest.mark.skipif(host.compiler() is None, reason="needs clang")


def run(exe, *args):
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])


@pytest.fixture(scope="module")
def conv(tmp_path_factory):
    return host.build("causal_conv", str(tmp_path_factory.mktemp("causal_conv")))


# (dtype, weights' dtype, act, taps, batch, steps, channels, ragged)
@pytest.mark.parametrize("case", [
    (1, 1, 0, 4, 1, 1, 1, 0), (1, 1, 1, 4, 2, 100, 5, 1), (2, 1, 1, 4, 3, 67, 40, 1),
    (2, 2, 0, 1, 2, 33, 17, 0), (3, 1, 1, 2, 5, 9, 70, 1), (0, 0, 1, 8, 2, 71, 9, 1),
    (2, 1, 1, 8, 1, 130, 21, 0), (1, 1, 0, 3, 4, 35, 130, 1), (0, 0, 0, 5, 3, 0, 4, 0),
    (3, 3, 0, 6, 2, 3, 600, 0), (1, 1, 1, 7, 40, 5, 3, 1), (1, 1, 1, 4, 0, 5, 3, 0)])
def test_causal_conv(conv, case):
    run(conv, *case)


@pytest.fixture(scope="module")
def scan(tmp_path_factory):
    return host.build("selective_scan_f32", str(tmp_path_factory.mktemp("selective_scan")))


# (dtype, batch, steps, channels, states, groups, ragged, optional). Several segments from 256
# steps on.
@pytest.mark.parametrize("case", [
    (1, 1, 1, 1, 1, 1, 0, 1), (1, 2, 37, 5, 3, 1, 1, 1), (1, 2, 300, 40, 16, 1, 1, 0),
    (2, 1, 19, 70, 16, 2, 0, 1), (3, 3, 33, 6, 8, 3, 1, 1), (0, 2, 21, 9, 16, 1, 1, 1),
    (0, 1, 13, 40, 64, 1, 0, 1), (1, 1, 18, 33, 64, 1, 0, 1), (1, 2, 11, 10, 128, 2, 1, 1),
    (2, 1, 520, 3, 20, 1, 0, 1), (1, 3, 0, 4, 5, 1, 0, 1), (1, 1, 1000, 2, 5, 2, 0, 1),
    (0, 1, 400, 2, 33, 1, 0, 0), (1, 0, 5, 4, 3, 1, 0, 1), (3, 2, 48, 31, 7, 1, 1, 1)])
def test_selective_scan(scan, case):
    run(scan, *case)
