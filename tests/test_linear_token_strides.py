"""Rows of single tokens cut out of long tensors: of one token no stride to the next is used, however large it is, and only the walks
over whole sequences limit it. Launches go to a recorder in the HIP runtime's place."""
import pytest
import torch

from hip_recorder import record
from paper_2511_21016_amd import binding

LIMIT = 1 << 23


def test_strides_that_single_tokens_may_have():
    record(f"""
X = 0x10000000
far = (4 * {LIMIT}, {LIMIT}, 128)
strides = dict(q_stride=far, k_stride=far, v_stride=far, o_stride=far)
for T in (1, 2):
    p = binding.make_linear_params(2, 16, 16, T, 128, 128, binding.GKA_BF16, cache_tokens=8, **strides)
    walk = binding.GKA_OK if T == 1 else binding.GKA_ERR_UNSUPPORTED
    assert binding.linear_decode_raw(p, X, X, X, X, X, X, X) == binding.GKA_OK
    assert binding.linear_decode_shared_raw(p, X, X, X, X, X, X, X, X, X, X) == binding.GKA_OK
    assert binding.linear_forward_raw(p, X, X, X, X, X, workspace=X, workspace_bytes=1 << 40) == walk
    assert binding.linear_backward_raw(p, X, X, X, X, X, X, X, X, X, workspace=X, workspace_bytes=1 << 40) == walk
""")


@pytest.mark.parametrize("T", [4095, 4096, 1 << 20])
def test_a_token_of_a_long_tensor_through_the_binding(T):
    """The strides of q[:, t] [B, H, d], and of one token stored heads first, are ones that the library takes."""
    long = torch.empty(2, T, 16, 128, dtype=torch.bfloat16, device="meta")
    first = torch.empty(2, 16, T, 128, dtype=torch.bfloat16, device="meta").transpose(1, 2)
    for x in (long[:, 7], long[:, 7:8], first[:, 7], first[:, 7:8]):
        strides = binding._row_strides(x, "x")
        assert strides[0] == x.stride(0) and strides[2] == x.stride(-2)
        record(f"""
X = 0x10000000
p = binding.make_linear_params(2, 16, 16, 1, 128, 128, binding.GKA_BF16, cache_tokens=8, q_stride={strides}, k_stride={strides})
assert binding.linear_decode_raw(p, X, X, X, X, X, X, X) == binding.GKA_OK
assert binding.linear_decode_shared_raw(p, X, X, X, X, X, X, X, X, X, X) == binding.GKA_OK
assert binding.linear_forward_raw(p, X, X, X, X, X, workspace=X, workspace_bytes=1 << 40) == binding.GKA_OK
""")
