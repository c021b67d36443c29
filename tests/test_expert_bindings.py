"""What the Python bindings of the mixture-of-experts calls refuse before the library sees it."""
import pytest
import torch


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    return m


@pytest.mark.gpu
def test_dispatch_into_a_plan_of_other_experts(metis):
    """(its choices of the experts that the plan does not have would be left out without a word)"""
    idx = torch.arange(64, device="cuda", dtype=torch.int32).view(32, 2)
    with pytest.raises(AssertionError):
        metis.dispatch(idx, 64, plan=metis.ExpertPlan(32, 8, 2))
    plan = metis.ExpertPlan(32, 64, 2)
    assert metis.dispatch(idx, 64, plan=plan) is plan and plan.offsets.tolist() == list(range(65))


@pytest.mark.parametrize("name,codes", [("MxTensor", 32), ("Mx8Tensor", 64)])
def test_host_buffers(metis, name, codes):
    """(kernels would follow the host's addresses)"""
    with pytest.raises(AssertionError):
        getattr(metis, name)(4, 64, buffers=(torch.zeros((4, codes), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)))
