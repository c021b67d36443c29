"""Loads and stores of eight elements promise no more alignment than elements have (no GPU needed: the compiler says where one does)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_00404_amd", "csrc")
SOURCE = """
#include "elementwise.h"
template <typename T, bool PAST>
__device__ void all(T* p, int64_t n) {
    RawUnit<T> r;
    float v[8];
    load_whole<PAST>(p, r);
    load_raw<PAST>(p, n, r);
    load_back<PAST>(p, 8, 3, n, r);
    unpack(r, 3, v);
    load_row<true>(p + 1, v);
    load_part<T, true>(p + 1, n, v);
    store_row<true>(p + 2, v);
    store_part<T, true>(p + 2, n, v);
    store_unit<PAST>(p + 3, n, v);
}
__global__ void k(bf16_t* a, float* b, int64_t n) {
    all<bf16_t, false>(a, n);
    all<bf16_t, true>(a, n);
    all<float, false>(b, n);
    all<float, true>(b, n);
}
"""


def test_no_load_or_store_is_declared_more_aligned_than_it_is(tmp_path):
    if not shutil.which("hipcc"):
        pytest.skip("no compiler")
    src = tmp_path / "all.hip"
    src.write_text(SOURCE)
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-std=c++17", "-fsyntax-only", "-Werror=align-mismatch", "-I", CSRC, str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
