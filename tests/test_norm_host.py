"""Host arithmetic of the norms' launches."""
import ctypes
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2608_28726_gb300", "csrc")
SM, SYSTEM, SUMS = 228 * 1024, 1024, 512  # bytes of an SM; of each CTA: reserved, static


@pytest.fixture(scope="module")
def stages(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    tmp = tmp_path_factory.mktemp("norm")
    (tmp / "norm.cpp").write_text("""
#include "pr_norm_host.h"
extern "C" int stages(long long d, int esize, int wsize, int groups, int ctas, int k, int weights,
                      int least, long long* smem, int* row_bytes) {
  const prh::NormStages s = prh::norm_stages(d, esize, wsize, groups, ctas, k, weights, least);
  *smem = (long long)s.smem;
  *row_bytes = s.row_bytes;
  return s.fits ? s.stages : -1;
}
extern "C" int two_rows(long long n_rows, int num_sms, long long d, int esize, int wsize) {
  return prh::norm_two_rows(n_rows, num_sms, d, esize, wsize);
}
""")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-O1", "-shared", "-fPIC", "-I", CSRC,
                    str(tmp / "norm.cpp"), "-o", str(tmp / "norm.so")], check=True)
    lib = ctypes.CDLL(str(tmp / "norm.so"))
    lib.stages.argtypes = [ctypes.c_longlong] + [ctypes.c_int] * 7 + [
        ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(ctypes.c_int)]

    def call(*args):
        smem, row = ctypes.c_longlong(), ctypes.c_int()
        return lib.stages(*args, ctypes.byref(smem), ctypes.byref(row)), smem.value, row.value
    lib.two_rows.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    call.two_rows = lib.two_rows
    return call


@pytest.mark.parametrize("esize", [2, 4])
@pytest.mark.parametrize("wsize", [2, 4])
def test_as_many_ctas_fit_an_sm_as_the_grid_counts_on(stages, esize, wsize):
    """Every width of rows in shared memory, every kernel's groups of rows in a CTA, with one or two
    arrays of weights and one to three rows to a place."""
    fitted = 0
    for groups, words in ((8, (17, 128)), (4, (65, 128)), (2, (129, 512)), (1, (257, 4096))):
        step = 1 if groups > 1 else 7
        for d in range((words[0] - 1) * 16 // esize + 1, words[1] * 16 // esize + 1, step):
            for ctas in (1, 2, 3):
                for k in (1, 2, 3):
                    for weights in (1, 2):
                        n, smem, row = stages(d, esize, wsize, groups, ctas, k, weights, 1)
                        if n < 0:
                            continue
                        fitted += 1
                        assert ctas * (smem + SUMS + SYSTEM) <= SM, (d, groups, ctas, k, weights, n, smem)
                        # the 16-byte words that a row touches, wherever it begins
                        touched = max((off + d * esize + 15) // 16 * 16 for off in range(0, 16, esize))
                        assert 1 <= n <= 4 and row % 16 == 0 and row >= touched
                        # the weights, a barrier for each place, the places
                        assert smem >= weights * d * wsize + groups * n * (8 + k * row)
    assert fitted > 1000


def test_rows_that_are_not_staged_take_their_weights_alone(stages):
    for d in (1, 7, 8, 64, 128):
        assert stages(d, 2, 4, 0, 1, 2, 2, 1)[:2] == (0, 2 * 4 * ((d + 7) // 8 * 8))


def test_two_rows_share_an_sm_where_there_are_rows_and_places(stages):
    """As measured on 152 SMs: not for some hundred rows, nor for rows with fewer than three places."""
    for n_rows, d, esize, wsize, want in (
            (153, 5120, 2, 2, False), (304, 6144, 2, 2, False), (608, 4288, 2, 2, False),
            (1700, 4288, 2, 2, True), (8000, 5120, 2, 2, True), (8000, 5600, 2, 2, True),
            (8000, 2560, 4, 4, True), (1700, 6144, 2, 2, False), (8000, 6144, 2, 2, False),
            (8000, 2960, 4, 4, False)):
        assert bool(stages.two_rows(n_rows, 152, d, esize, wsize)) == want, (n_rows, d)


def test_no_kernel_is_compiled_that_no_width_takes():
    """bf16 rows of more than 2,048 words are read again instead."""
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    from paper_2608_28726_gb300 import build as prbuild
    names = subprocess.run([nm, "-C", "--defined-only", prbuild.build()], check=True, text=True,
                           capture_output=True).stdout
    rows = {w for w in names.splitlines() if "norm_rows<" in w}
    assert any("norm_rows<float, 512, 8, true, true>" in w for w in rows)
    assert not [w for w in rows if "norm_rows<__nv_bfloat16, 512, 8" in w]
