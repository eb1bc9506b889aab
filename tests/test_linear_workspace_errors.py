"""Sizes that only the backward pass refuses: the binding reports the size, not the pointers that its question leaves out."""
import pytest

from paper_2511_21016_amd import binding


def test_a_size_that_only_the_backward_pass_refuses():
    p = binding.make_linear_params(1 << 20, 1, 1, 16385, 16, 16, binding.GKA_BF16)
    assert binding.linear_forward_workspace_bytes(p) > 0 and binding.linear_backward_workspace_bytes(p) == 0
    plan = binding._LinearPlan(p)
    assert binding._workspace_bytes(plan, False) > 0
    with pytest.raises(binding.GkaError) as e:
        binding._workspace_bytes(plan, True)
    assert e.value.status == binding.GKA_ERR_SHAPE


@pytest.mark.parametrize("backward", [False, True])
def test_what_both_refuse(backward):
    plan = binding._LinearPlan(binding.make_linear_params(2, 3, 2, 16, 16, 16, binding.GKA_BF16))
    with pytest.raises(binding.GkaError) as e:
        binding._workspace_bytes(plan, backward)
    assert e.value.status == binding.GKA_ERR_SHAPE
