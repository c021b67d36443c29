"""Every kernel launch of the mixture-of-experts calls that fails is reported by the call that made it (no GPU needed: the library runs behind the
stand-in for the runtime of test_launches), and no kernel that keeps its accumulators in registers spills them."""
import ctypes as C
import os
import re
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 1 << 30                                   # an aligned address that is never read
LLVM = "/opt/rocm/llvm/bin/"


def _calls(metis):
    """name -> (a call of the library, the launches it makes)"""
    L = metis.lib()
    keep = []

    def ref(x):
        keep.append(x)
        return C.byref(x)

    def mat(rows, cols, dtype=metis.BF16):
        return ref(metis.Mat(FAKE, rows, cols, cols, dtype))

    def plan(T, E, k):
        return ref(metis.Plan(FAKE, FAKE, FAKE, T, E, k))

    def route(scores, grads=False):
        r = ref(metis.Router(256, 8, scores, 8, 4, 1, 1.0))
        if grads:
            return lambda: L.metis_route_grads(None, mat(1000, 256), r, FAKE, FAKE, mat(1000, 256, metis.F32))
        return lambda: L.metis_route(None, mat(1000, 256), r, FAKE, FAKE, FAKE, FAKE)

    def dispatch(T):
        return lambda: L.metis_dispatch(None, FAKE, plan(T, 64, 4), FAKE, 1 << 40)

    def product(T, E, k, N, K, gather, out):
        w = ref(metis.MxFp4(FAKE, FAKE, E * N, K))
        return lambda: L.metis_experts_product(None, mat(T if gather else T * k, K), w, plan(T, E, k), gather, mat(T * k, N, out), FAKE, 1 << 40)

    def wgrad(out, T=1000, g=metis.BF16):
        return lambda: L.metis_experts_wgrad(None, mat(4 * T, 512, g), mat(T, 1024), plan(T, 16, 4), 1, mat(16 * 512, 1024, out), FAKE, 1 << 40)

    mx8 = lambda rows, cols: ref(metis.Mx8(FAKE, FAKE, rows, cols))
    return {
        "route, softmax": (route(0), 1), "route, sigmoid": (route(1), 1), "route gradients": (route(0, True), 1),
        "plan, one workgroup": (dispatch(1000), 1), "plan, chunks": (dispatch(10000), 2),
        "product, one token": (product(1, 64, 4, 2048, 4096, 1, metis.BF16), 1),
        "product, few slots": (product(100, 64, 4, 2048, 4096, 0, metis.F32), 2),
        "product, many slots": (product(4000, 16, 4, 2048, 1056, 1, metis.BF16), 2),
        "product, contraction in parts, bf16": (product(256, 16, 4, 1024, 4096, 1, metis.BF16), 3),
        "product, contraction in parts, fp32": (product(256, 16, 4, 1024, 4096, 0, metis.F32), 3),
        "weight gradient, bf16": (wgrad(metis.BF16), 2), "weight gradient, fp32": (wgrad(metis.F32), 2),
        "weight gradient, operands of two types": (wgrad(metis.BF16, g=metis.F32), 3),
        "weight gradient, few slots, bf16": (wgrad(metis.BF16, 100), 2), "weight gradient, few slots, fp32": (wgrad(metis.F32, 100), 2),
        "weights transposed": (lambda: L.metis_quantize_mx_t(None, mat(4 * 512, 1024), 4, ref(metis.MxFp4(FAKE, FAKE, 4 * 1024, 512))), 1),
        "combine": (lambda: L.metis_combine(None, mat(400, 512), plan(100, 16, 4), FAKE, mat(100, 512, metis.F32)), 1),
        "combine gradients": (lambda: L.metis_combine_grads(None, mat(100, 512), mat(400, 512), plan(100, 16, 4), FAKE, mat(400, 512), FAKE), 1),
        "save": (lambda: L.metis_quantize_mx8(None, mat(100, 512), mx8(100, 512)), 1),
        "restore": (lambda: L.metis_dequantize_mx8(None, mx8(100, 512), mat(100, 512, metis.F32)), 1),
        "activation": (lambda: L.metis_swiglu(None, mat(100, 512), mat(100, 256), mx8(100, 512)), 1),
        "activation, nothing saved": (lambda: L.metis_swiglu(None, mat(100, 512), mat(100, 256), None), 1),
        "activation gradients": (lambda: L.metis_swiglu_grads(None, mx8(100, 512), mat(100, 256), mat(100, 512), mat(100, 256)), 1),
    }


def _child(runtime):
    stub = C.CDLL(runtime, mode=C.RTLD_GLOBAL)
    sys.path.insert(0, ROOT)
    from paper_2509_00404_amd import metis
    for name, (call, launches) in _calls(metis).items():
        stub.fail_at(0)
        assert call() == 0, name
        assert stub.launch_count() == launches, (name, stub.launch_count())
        for i in range(1, launches + 1):
            stub.fail_at(i)
            status = call()
            assert status == -4, f"{name}: launch {i} of {launches} failed, status {status}"


def test_failed_launches_are_reported(tmp_path):
    from paper_2509_00404_amd import metis
    from test_launches import RUNTIME
    if not os.path.exists(metis.LIB_PATH) or not shutil.which("gcc"):
        pytest.skip("library not built, or no C compiler")
    src, runtime = tmp_path / "runtime.c", tmp_path / "runtime.so"
    src.write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(runtime), str(src)], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), str(runtime)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_products_need_no_scratch(tmp_path):
    from paper_2509_00404_amd import metis
    if not os.path.exists(metis.LIB_PATH) or not os.path.exists(LLVM + "llvm-readelf"):
        pytest.skip("library not built, or no reader of code objects")
    lib = shutil.copy(metis.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([LLVM + "llvm-objdump", "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    scratch = {}
    for image in sorted(tmp_path.glob("lib.so.*gfx950")):
        notes = subprocess.run([LLVM + "llvm-readelf", "--notes", str(image)], check=True, capture_output=True, text=True).stdout
        for name, size in re.findall(r"\.name:\s+(\S*k_(?:experts|route|plan|quantize_mx_t|quantize_rows|swiglu|combine)\S*)\n.*?\.private_segment_fixed_size:\s*(\d+)",
                                     notes, re.S):
            scratch[name] = int(size)
    assert len(scratch) >= 30 and not any(scratch.values()), {k: v for k, v in scratch.items() if v}


if __name__ == "__main__":
    _child(sys.argv[1])
