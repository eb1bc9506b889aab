"""Linear attention: launch plans that the other tests leave out, against the float64 oracle. Many segments, scanned and added up, of states in
one slice and in several; in the backward pass head dimensions of unequal padded widths, where the walk of dv reads the summaries of
dk's walk with rows and columns exchanged."""
import pytest
import torch

from linear_testutil import check_backward, check_forward, make, states
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu

DIMS = [(64, 128), (128, 64), (256, 144), (144, 256), (16, 256), (256, 16), (48, 80), (192, 48), (256, 256), (64, 64), (128, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_k,d_v", DIMS)
@pytest.mark.parametrize("walk_chunks", [0, 1, 3])
def test_backward(walk_chunks, d_k, d_v, dtype):
    H, H_kv = (4, 2) if d_k + d_v < 300 else (1, 1)
    q, k, v, gate, dy = make(1, 601, H, H_kv, d_k, d_v, dtype, seed=walk_chunks)
    S, dS = states(1, H_kv, d_v, d_k), states(1, H_kv, d_v, d_k, seed=6)
    got = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S, dS_final=dS, walk_chunks=walk_chunks)
    check_backward(got, q, k, v, gate, dy, S, dS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_k,d_v", DIMS)
@pytest.mark.parametrize("walk_chunks", [1, 3])
def test_forward(walk_chunks, d_k, d_v, dtype):
    H, H_kv = (4, 2) if d_k + d_v < 300 else (1, 1)
    q, k, v, gate, _ = make(1, 1201, H, H_kv, d_k, d_v, dtype, seed=walk_chunks)
    S = states(1, H_kv, d_v, d_k)
    o, S1 = binding.gka_linear_forward(q, k, v, gate, S_init=S, return_state=True, walk_chunks=walk_chunks)
    check_forward(o, S1, q, k, v, gate, S)


def test_in_place_through_the_scan():
    q, k, v, gate, _ = make(2, 300, 2, 1, 144, 256)
    S = states(2, 1, 256, 144)
    first = S.clone()
    o, S1 = binding.gka_linear_forward(q, k, v, gate, S_init=S, S_final=S, walk_chunks=1)
    assert S1 is S
    check_forward(o, S, q, k, v, gate, first)


def test_a_padded_batch_of_packed_sequences():
    """Sequences of several lengths in each row of a batch, the rest of the row without numbers; gradients of the tokens that count."""
    q, k, v, gate, dy = make(3, 200, 4, 2, 64, 128)
    used = [200, 130, 64]
    gate[:, [0, 40]] = 0.0
    rows = [x.clone() for x in (q, k, v)]
    grad = dy.clone()
    for b, n in enumerate(used):
        for x in (*rows, grad):
            x[b, n:] = float("nan")
        if n < 200:
            gate[b, n] = 0.0
    o = binding.gka_linear_forward(*rows, gate)
    got = binding.gka_linear_backward(*rows, gate, grad)
    for b, n in enumerate(used):
        alone = [x[b:b + 1, :n].contiguous() for x in (q, k, v, gate, dy)]
        check_forward(o[b:b + 1, :n], None, *alone[:4])
        for n_grad in ("dq", "dk", "dv", "dgate"):
            assert torch.isfinite(got[n_grad][b, :n]).all(), n_grad
        want = binding.gka_linear_backward(*alone)
        # the same sums in the same chunks, but for the reverse walk's empty ones: a step of bf16, 2^-7, where one is rounded otherwise
        for x in ("dq", "dk", "dv"):
            torch.testing.assert_close(got[x][b:b + 1, :n], want[x], rtol=2.0 ** -7, atol=1e-5)
