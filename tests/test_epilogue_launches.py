"""What the calls around the products ask of the HIP runtime, without a GPU (the library runs behind the stand-in of test_launches; addresses are never
read): launches that fail are reported by the call that made them, the largest sizes stay below 2^32 threads along an axis of a grid, which is what HIP
takes, outputs over rows that are still read are refused, and a kernel's limit of dynamic LDS is never left below what a call needs, whichever threads call at once."""
import ctypes as C
import os
import shutil
import subprocess
import sys
import threading

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE, OTHER = 1 << 30, 1 << 60
COUNT = "    if (++launches == failing) error = 1;\n"
NOTE = """
    unsigned long long gs[3] = {g.x, g.y, g.z}, bs[3] = {b.x, b.y, b.z};
    for (int i = 0; i < 3; ++i) if (gs[i] * bs[i] > widest) widest = gs[i] * bs[i];
"""
# A limit above 64 KB is set by a call that lets others overtake it: it returns once another has set one, or after a second without.
SET = "int hipFuncSetAttribute(const void* f, int a, int v) { return 0; }\n"
LIMITS = """
#include <unistd.h>
static const void* fns[64];
static int limits[64], fn_count;
static volatile int turns, waiting, exceeded;
static int slot(const void* f) {
    for (int i = 0; i < fn_count; ++i) if (fns[i] == f) return i;
    fns[fn_count] = f;
    limits[fn_count] = 65536;
    return fn_count++;
}
int is_waiting(void) { return waiting; }
int exceeded_count(void) { return exceeded; }
int hipFuncSetAttribute(const void* f, int a, int v) {
    limits[slot(f)] = v;
    const int mine = ++turns;
    if (v > 65536) {
        waiting = 1;
        for (int i = 0; i < 100 && turns == mine; ++i) usleep(10000);
        usleep(20000);
        waiting = 0;
    }
    return 0;
}
"""
CHECK = "    if (l > (size_t)limits[slot(f)]) { ++exceeded; error = 1; }\n"


class _Calls:
    def __init__(self, metis):
        self.m, self.L, self.keep = metis, metis.lib(), []

    def ref(self, x):
        self.keep.append(x)
        return C.byref(x)

    def mat(self, rows, cols, dtype=0, at=FAKE):
        return self.ref(self.m.Mat(at, rows, cols, cols, dtype))

    def linear(self, T, N, K, dense=True, workspace=FAKE, out=0):
        x, q = (self.mat(T, K), None) if dense else (None, self.ref(self.m.MxFp4(FAKE, FAKE, T, K)))
        return self.L.metis_mxfp4_linear(None, x, q, self.ref(self.m.MxFp4(FAKE, FAKE, N, K)), None, self.mat(T, N, out, OTHER), workspace, 1 << 60 if workspace else 0)

    def layernorm(self, T, N):
        return self.L.metis_layernorm(None, self.mat(T, N), None, None, 1e-5, self.mat(T, N), FAKE)

    def layernorm_grads(self, T, N, at=OTHER):
        return self.L.metis_layernorm_grads(None, self.mat(T, N), self.mat(T, N), FAKE, None, None, self.mat(T, N, 0, at), FAKE, FAKE, FAKE, 1 << 60)

    def linear_grads(self, T, N):
        return self.L.metis_linear_grads(None, self.mat(T, N), self.mat(T, N), 2, None, self.mat(T, N), FAKE, FAKE, 1 << 60)

    def dropout(self, T, N):
        return self.L.metis_dropout(None, self.mat(T, N), self.ref(self.m.Mask(0.1, 1, None)), None, self.mat(T, N))


def _failed(stub, c):
    for name, call, launches in [
        ("one token", lambda: c.linear(1, 14336, 4096), 1), ("few rows", lambda: c.linear(24, 4096, 14336), 2),
        ("few rows, quantized", lambda: c.linear(24, 4096, 14336, False), 1), ("few tiles", lambda: c.linear(1111, 2057, 2080), 2),
        ("parts", lambda: c.linear(128, 4096, 14336), 3), ("parts, quantized, no workspace", lambda: c.linear(128, 4096, 14336, False, None), 1),
        ("many tiles", lambda: c.linear(4096, 4096, 1024, False), 1), ("streamed", lambda: c.linear(16384, 4096, 14336, False, None, 1), 1),
        ("layer norm", lambda: c.layernorm(16384, 4096), 1), ("layer norm, long rows", lambda: c.layernorm(4, 40000), 1),
        ("its gradients", lambda: c.layernorm_grads(16384, 4096), 2), ("its gradients, few rows", lambda: c.layernorm_grads(64, 4096), 1),
        ("its gradients, few rows in their place", lambda: c.layernorm_grads(64, 4096, FAKE), 2),
        ("its gradients, long rows", lambda: c.layernorm_grads(64, 40000), 3), ("the epilogue's gradient", lambda: c.linear_grads(16384, 14336), 2),
        ("the epilogue's gradient, few rows", lambda: c.linear_grads(64, 14336), 1), ("dropout", lambda: c.dropout(333, 1027), 1),
    ]:
        stub.fail_at(0)
        assert call() == 0, name
        assert stub.launch_count() == launches, (name, stub.launch_count())
        for i in range(1, launches + 1):
            stub.fail_at(i)
            status = call()
            assert status == -4, f"{name}: launch {i} of {launches} failed, status {status}"


def _workspaces(stub, c):
    """Rows quantized already: cut into parts, which are joined, from the very byte on that the query asks for."""
    L, quantized = c.L, c.L.metis_mxfp4_linear_quantized_workspace_bytes
    for T, N, K, cut in [(128, 4096, 14336, True), (128, 1024, 4096, True), (129, 777, 2080, True), (1111, 2057, 2080, False), (16384, 4096, 14336, False),
                         (64, 4096, 14336, False), (1, 14336, 4096, False), (300, 520, 512, False)]:
        need = quantized(T, N, K)
        assert (need > 0) == cut, (T, N, K)
        for at, size, launches in ((FAKE, need, 1 + cut), (FAKE, need - cut, 1), (None, 0, 1), (FAKE + 64, need, 1)):
            stub.fail_at(0)
            assert L.metis_mxfp4_linear(None, None, c.ref(c.m.MxFp4(FAKE, FAKE, T, K)), c.ref(c.m.MxFp4(FAKE, FAKE, N, K)), None, c.mat(T, N, 0, OTHER), at, size) == 0
            assert stub.launch_count() == launches, (T, N, K, size)
    assert quantized(0, 40, 64) == 0 and quantized(128, 1024, 4080) == 0 and quantized(1 << 28, 40, 64) == 0


def _largest(stub, c):
    widest = C.c_ulonglong.in_dll(stub, "widest")
    wide, tall = 1 << 28, (1 << 32) - 1
    for name, call in [
        ("layer norm, columns", lambda: c.layernorm(4, wide)), ("layer norm, rows", lambda: c.layernorm(tall, 8)),
        ("its gradients, 2^27 columns", lambda: c.layernorm_grads(4, wide // 2)), ("its gradients, columns", lambda: c.layernorm_grads(4, wide)),
        ("its gradients, many rows of them", lambda: c.layernorm_grads(5000, wide)), ("its gradients, rows", lambda: c.layernorm_grads(tall, 8)),
        ("its gradients, rows of one", lambda: c.layernorm_grads(tall, 1)),
        ("the epilogue's gradient, columns", lambda: c.linear_grads(4, wide)), ("the epilogue's gradient, rows", lambda: c.linear_grads(tall, 8)),
        ("dropout, columns", lambda: c.dropout(15, wide)), ("dropout, rows", lambda: c.dropout(tall // 256 * 256, 8)),
        ("no rows", lambda: c.layernorm_grads(0, wide)), ("product, outputs", lambda: c.linear(1, wide - 1, 32)), ("product, few rows", lambda: c.linear(64, wide - 1, 32)),
        ("product, long contraction", lambda: c.linear(64, 1, 1 << 26)),
    ]:
        widest.value = 0
        stub.fail_at(0)
        status = call()
        assert status == 0 and stub.launch_count() > 0, (name, status)
        assert widest.value < 2 ** 32, (name, widest.value)


def _in_place(stub, c):
    """Outputs over X: refused, with nothing launched, where X is quantized on the spot; any memory between its rows is free."""
    m, L, INVALID = c.m, c.L, -1

    def call(T=4, N=64, K=64, x=(FAKE, 64), y=(OTHER, 64), pre=None, dtype=0, out=0):
        e = c.ref(m.Epilogue(None, 0, C.pointer(m.Mat(pre[0], T, N, pre[1], out)) if pre else None, None, None))
        stub.fail_at(0)
        status = L.metis_mxfp4_linear(None, c.ref(m.Mat(x[0], T, K, x[1], dtype)), None, c.ref(m.MxFp4(OTHER, OTHER, N, K)), e,
                                      c.ref(m.Mat(y[0], T, N, y[1], out)), FAKE, 1 << 40)
        assert (status == 0) == (stub.launch_count() > 0)
        return status

    assert L.metis_mxfp4_linear_workspace_bytes(4, 64, 64) == 0 and L.metis_mxfp4_linear_workspace_bytes(16, 64, 64) == 0
    assert call() == 0 and call(y=(FAKE, 64)) == INVALID and call(pre=(FAKE, 64)) == INVALID and call(pre=(OTHER, 64)) == 0
    assert call(y=(FAKE + 3 * 128 + 126, 64)) == INVALID and call(y=(FAKE + 4 * 128, 64)) == 0          # the last element; right behind it
    assert call(y=(FAKE - 4 * 128 + 2, 64)) == INVALID and call(y=(FAKE - 4 * 128, 64)) == 0
    wide = (FAKE, 128)
    assert call(x=wide, y=(FAKE + 128, 128)) == 0 and call(x=wide, y=(FAKE + 126, 128)) == INVALID      # columns beside X's in one buffer
    assert call(x=wide, y=(FAKE + 128, 128), pre=(FAKE + 2, 128)) == INVALID
    assert call(T=3, x=(FAKE, 128), y=(FAKE + 128, 192)) == INVALID and call(T=2, x=(FAKE, 128), y=(FAKE + 128, 192)) == 0
    assert call(T=1, y=(FAKE + 64, 64), dtype=1, out=1) == INVALID and call(T=16, y=(FAKE, 64)) == INVALID and call(T=16, x=wide, y=(FAKE + 128, 128)) == 0
    assert L.metis_mxfp4_linear_workspace_bytes(17, 64, 64) > 0 and call(T=17, y=(FAKE, 64)) == 0 and call(T=17, pre=(FAKE, 64)) == 0


def _threads(stub, c):
    """64 rows quantized already: of one kernel instance, K = 4096 takes 8 waves and 73 728 bytes of LDS, 3584 seven and 64 512."""
    status = []
    large, small = (lambda: status.append(c.linear(64, 8192, 4096, False))), (lambda: status.append(c.linear(64, 8192, 3584, False)))
    threads = [threading.Thread(target=large), threading.Thread(target=small)]
    threads[0].start()
    while threads[0].is_alive() and not stub.is_waiting():
        pass
    assert stub.is_waiting()                             # the larger limit is set, and not noted yet
    threads[1].start()
    for t in threads:
        t.join()
    large()
    assert status == [0, 0, 0] and stub.exceeded_count() == 0, (status, stub.exceeded_count())


@pytest.mark.parametrize("check", ["failed", "workspaces", "largest", "in_place", "threads"])
def test_behind_a_stand_in_for_the_runtime(tmp_path, check):
    from paper_2509_00404_amd import metis
    from test_launches import RUNTIME
    if not os.path.exists(metis.LIB_PATH) or not shutil.which("gcc"):
        pytest.skip("library not built, or no C compiler")
    assert RUNTIME.count(COUNT) == 1 and RUNTIME.count(SET) == 1
    text = RUNTIME.replace(COUNT, NOTE + COUNT)
    text = "#include <stddef.h>\nunsigned long long widest;\n" + LIMITS + text.replace(SET, "").replace(COUNT, COUNT + CHECK)
    src, runtime = tmp_path / "runtime.c", tmp_path / "runtime.so"
    src.write_text(text)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(runtime), str(src)], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), check, str(runtime)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def _child(check, runtime):
    stub = C.CDLL(runtime, mode=C.RTLD_GLOBAL)
    sys.path.insert(0, ROOT)
    from paper_2509_00404_amd import metis
    {"failed": _failed, "workspaces": _workspaces, "largest": _largest, "in_place": _in_place, "threads": _threads}[check](stub, _Calls(metis))


if __name__ == "__main__":
    _child(*sys.argv[1:])
