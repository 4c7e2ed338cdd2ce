"""Kernels compiled as host code (host_hip/), on arrays that end before or begin behind a page
without access: an access past any array ends the program, and results are compared with the
definitions. Extents are those where workgroups, spans, lanes and vectors end unevenly."""
import subprocess

import pytest

from tests import host_hip_build as host

pytestmark = pytest.mark.skipif(host.compiler() is None, reason="needs clang")


def program(name, tmp_path_factory):
    return host.build(name, str(tmp_path_factory.mktemp(name)))


@pytest.fixture(scope="module")
def recurrence(tmp_path_factory):
    return program("recurrence", tmp_path_factory)


def run(exe, *args):
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])


# (dtype, gate, batch, steps, channels, ragged). Rows of 16 and of 64 lanes, one span and many;
# 1030 and 600 steps of few channels: the last span reads the maps of those before it.
@pytest.mark.parametrize("case", [
    (1, 0, 1, 100, 5, 0), (1, 0, 1, 1030, 5, 0), (1, 1, 2, 1030, 40, 1), (0, 1, 1, 600, 5, 0),
    (0, 0, 2, 5000, 17, 1), (2, 1, 1, 4200, 20, 0), (3, 0, 1, 1500, 70, 0), (1, 0, 1, 5000, 64, 1),
    (2, 0, 3, 17000, 3, 1), (1, 1, 1, 70000, 1, 0), (3, 1, 5, 1, 9, 0), (2, 1, 2, 0, 4, 0),
    (0, 1, 1, 9000, 1, 0)])
def test_recurrence(recurrence, case):
    run(recurrence, *case)


@pytest.fixture(scope="module")
def layer_norm(tmp_path_factory):
    return program("layer_norm", tmp_path_factory)


# (dtype, weights' dtype, rows, n, elements between rows). Rows of 16 lanes up to those longer
# than a workgroup's registers, whole vectors and not.
@pytest.mark.parametrize("case", [
    (1, 1, 1, 1, 0), (1, 1, 5, 64, 0), (2, 1, 67, 100, 3), (2, 2, 9, 515, 0), (3, 3, 2, 2047, 1),
    (0, 0, 4, 2047, 0), (1, 1, 3, 9000, 0), (2, 1, 2, 20011, 0), (1, 1, 2, 40000, 0),
    (0, 0, 1, 9001, 0), (3, 1, 130, 8, 0), (2, 1, 700, 33, 0), (0, 0, 0, 30, 0),
    (1, 1, 1, 16390, 5), (2, 2, 2, 33000, 0)])
def test_layer_norm(layer_norm, case):
    run(layer_norm, *case)


@pytest.mark.parametrize("rows,n", [
    (1, (1 << 26) - 1), (1, 1 << 26), (3, (1 << 26) + 1), (1, (1 << 31) - (1 << 16) - 1),
    ((1 << 31) - (1 << 16) - 1, 1), (1 << 30, 5000), (5000, 1 << 30)])
def test_layer_norm_of_any_extent_fits_a_dispatch(layer_norm, rows, n):
    run(layer_norm, rows, n)
