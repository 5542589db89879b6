"""Which tiles the experts' products take at the sizes of the GPU tests that are meant for them (no
GPU needed: the rule is host code, compiled here)."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_experts_large_tiles as large
import test_gpu_mixture as mixture

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_1503_08294_amd", "csrc")


@pytest.fixture(scope="module")
def side(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    source = d / "rule.cpp"
    source.write_text('#include "experts_rule.h"\n'
                      'extern "C" int side(int f32, long pairs, int experts, int dim, int hidden, '
                      'int aligned) {\n'
                      '  return gsn::tile_side(f32, pairs, experts, dim, hidden, aligned);\n}\n')
    lib = str(d / "rule.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", str(source),
                    "-o", lib], check=True)
    f = ctypes.CDLL(lib).side
    f.argtypes = [ctypes.c_int, ctypes.c_long, *[ctypes.c_int] * 4]
    return lambda tokens, experts, k, dim, hidden, f32=False, aligned=True: f(
        f32, tokens * k, experts, dim, hidden, aligned)


def sizes(test):
    """The values of a test's parameters of sizes."""
    return next(m.args[1] for m in test.pytestmark if m.args[0].startswith("tokens"))


def test_large_tiles(side):
    for s in (*mixture.WIDE, *sizes(large.test_sums_of_few_stages)):
        assert side(*s) == 256, s
        assert side(*s, f32=True) == 64, s
    for rest in (1, 17, 40, 129):
        assert side(3 * (256 * 12 + rest), 3, 1, 520, 1304) == 256
    for dim, hidden in large.FAR:
        assert side(4300, 2, 2, dim, hidden) == 256
    assert side(3000, 4, 2, 1032, 1544) == 256  # batches in which nobody has an expert


def test_middle_tiles(side):
    for s in mixture.LOOSE:
        assert side(*s) == 128, s
    # aligned sizes, rows of x that begin anywhere
    assert side(3000, 4, 2, 520, 704, aligned=False) == 128
    assert side(3000, 4, 2, 515, 701) == 128


def test_small_tiles(side):
    for s in ((300, 3, 1, 136, 72), (20, 64, 2, 72, 40), (17_001, 4, 2, 7, 2000),
              (17_001, 4, 2, 2000, 7), (127, 1, 1, 4096, 4096), (0, 1, 1, 64, 64)):
        assert side(*s) == 64, s
