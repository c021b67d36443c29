"""What the combination reads of a plan: the slots of the choices alone; its gradients need the end of the used slots too."""
import ctypes as C

import pytest
import torch

FAKE = 1 << 30
INVALID = -1


def test_gradients_refuse_a_plan_without_offsets():
    import os
    from paper_2509_00404_amd import metis
    if not os.path.exists(metis.LIB_PATH):
        pytest.skip("library not built")
    m, p = metis.Mat(FAKE, 8, 64, 64, 0), metis.Plan(None, None, FAKE, 4, 8, 2)
    y = metis.Mat(FAKE, 4, 64, 64, 0)
    assert metis.lib().metis_combine_grads(None, C.byref(y), C.byref(m), C.byref(p), FAKE, C.byref(m), FAKE) == INVALID


@pytest.mark.gpu
def test_combine_of_slots_alone():
    from paper_2509_00404_amd import metis
    T, k, D = 33, 3, 72
    g = torch.Generator(device="cuda").manual_seed(0)
    plan = metis.dispatch(torch.randint(0, 8, (T, k), generator=g, device="cuda", dtype=torch.int32), 8)
    rows, w = torch.randn((T * k, D), generator=g, device="cuda"), torch.rand((T, k), generator=g, device="cuda")
    want = metis.combine(rows, plan, torch.empty((T, D), device="cuda"), w)
    y = torch.full((T, D), float("nan"), device="cuda")
    bare = metis.Plan(None, None, plan.slot.data_ptr(), T, 8, k)
    status = metis.lib().metis_combine(metis._stream(), C.byref(metis._mat(rows)), C.byref(bare), w.data_ptr(), C.byref(metis._mat(y)))
    assert status == 0 and torch.equal(y, want)
