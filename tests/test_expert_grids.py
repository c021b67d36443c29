"""The largest launches of the mixture-of-experts calls: fewer than 2^32 threads along an axis of a grid, which is what HIP takes, and the next
larger size is refused as unsupported before anything is launched (no GPU needed: the library runs behind the stand-in for the runtime of
test_launches, and the addresses are never read)."""
import ctypes as C
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 1 << 30
UNSUPPORTED = -5
COUNT = "    if (++launches == failing) error = 1;\n"
NOTE = """
    unsigned long long gs[3] = {g.x, g.y, g.z}, bs[3] = {b.x, b.y, b.z};
    for (int i = 0; i < 3; ++i) if (gs[i] * bs[i] > widest) widest = gs[i] * bs[i];
"""


def _calls(metis):
    """name -> (a call for a size, the largest size it takes)"""
    L = metis.lib()
    keep = []

    def ref(x):
        keep.append(x)
        return C.byref(x)

    mat = lambda rows, cols, dtype=metis.BF16: ref(metis.Mat(FAKE, rows, cols, cols, dtype))
    mx8 = lambda rows, cols: ref(metis.Mx8(FAKE, FAKE, rows, cols))
    mx4 = lambda rows, cols: ref(metis.MxFp4(FAKE, FAKE, rows, cols))
    plan = lambda T, E, k: ref(metis.Plan(FAKE, FAKE, FAKE, T, E, k))
    router = ref(metis.Router(8, 1, 0, 1, 1, 1, 1.0))

    def product(S, E, N, K):
        return L.metis_experts_product(None, mat(S, K), mx4(E * N, K), plan(S, E, 1), 0, mat(S, N), FAKE, 1 << 60)

    def wgrad(T, K, N=1 << 18):
        return L.metis_experts_wgrad(None, mat(T, N), mat(T, K), plan(T, 1, 1), 0, mat(N, K), FAKE, 1 << 60)

    combine_grads = lambda T, D: L.metis_combine_grads(None, mat(T, D), mat(T, D), plan(T, 8, 1), FAKE, mat(T, D), FAKE)
    return {
        "route": (lambda T: L.metis_route(None, mat(T, 8), router, None, None, FAKE, FAKE), 16 * (2 ** 24 - 1)),
        "route gradients": (lambda T: L.metis_route_grads(None, mat(T, 8), router, FAKE, FAKE, mat(T, 8)), 16 * (2 ** 24 - 1)),
        "save": (lambda M: L.metis_quantize_mx8(None, mat(M, 64), mx8(M, 64)), 32 * (2 ** 24 - 1)),
        "restore": (lambda M: L.metis_dequantize_mx8(None, mx8(M, 64), mat(M, 64)), 32 * (2 ** 24 - 1)),
        "activation": (lambda M: L.metis_swiglu(None, mat(M, 64), mat(M, 32), mx8(M, 64)), 64 * (2 ** 24 - 1)),
        "activation, nothing saved": (lambda M: L.metis_swiglu(None, mat(M, 64), mat(M, 32), None), 64 * (2 ** 24 - 1)),
        "activation gradients": (lambda M: L.metis_swiglu_grads(None, mx8(M, 64), mat(M, 32), mat(M, 64), None), 64 * (2 ** 24 - 1)),
        "combine": (lambda T: L.metis_combine(None, mat(T, 64), plan(T, 8, 1), FAKE, mat(T, 64)), 32 * (2 ** 24 - 1)),
        "combine gradients, 64 threads": (lambda T: combine_grads(T, 64), 2 ** 26 - 1),
        "combine gradients, 128 threads": (lambda T: combine_grads(T, 1024), 2 ** 25 - 1),
        "combine gradients, 256 threads": (lambda T: combine_grads(T, 1032), 2 ** 24 - 1),
        "product, outputs": (lambda N: product(1, 1, N, 32), 128 * (2 ** 23 - 1)),
        "product, rows": (lambda S: product(S, 1, 32, 1 << 20), 2 ** 15 - 1),
        "product, weights' scales": (lambda N: product(16, 1, N, 32), 64 * (2 ** 24 - 3)),
        "weights transposed": (lambda n: L.metis_quantize_mx_t(None, mat(32, 8 * n), 1, mx4(8 * n, 32)), 2 ** 27 - 16),
        "weight gradient, few slots": (lambda n: wgrad(32, 8 * n), 2 ** 18 - 32),
        "weight gradient, no slots": (lambda n: wgrad(0, 8 * n), 2 ** 18 - 32),
    }


def _child(runtime):
    stub = C.CDLL(runtime, mode=C.RTLD_GLOBAL)
    sys.path.insert(0, ROOT)
    from paper_2509_00404_amd import metis
    widest = C.c_ulonglong.in_dll(stub, "widest")
    for name, (call, largest) in _calls(metis).items():
        widest.value = 0
        stub.fail_at(0)
        status = call(largest)
        assert status == 0 and stub.launch_count() > 0, (name, status)
        assert 2 ** 31 < widest.value < 2 ** 32, (name, widest.value)
        stub.fail_at(0)
        status = call(largest + 1)
        assert status == UNSUPPORTED and stub.launch_count() == 0, (name, status, stub.launch_count(), widest.value)


def test_launches_of_2_32_threads_are_refused(tmp_path):
    from paper_2509_00404_amd import metis
    from test_launches import RUNTIME
    if not os.path.exists(metis.LIB_PATH) or not shutil.which("gcc"):
        pytest.skip("library not built, or no C compiler")
    assert RUNTIME.count(COUNT) == 1
    src, runtime = tmp_path / "runtime.c", tmp_path / "runtime.so"
    src.write_text("unsigned long long widest;\n" + RUNTIME.replace(COUNT, NOTE + COUNT))
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(runtime), str(src)], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), str(runtime)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    _child(sys.argv[1])
