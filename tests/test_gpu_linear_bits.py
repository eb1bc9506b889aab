"""Linear attention, bf16 tensors: nothing between the inputs and an output's own rounding has fewer bits than float32.

The measure: the share of outputs that are not the float64 oracle's value rounded once. A value computed with a relative error e
rounds the other way where it lies within e of the middle between two bf16 numbers, which are 2^-8 to 2^-7 of it apart: at most
2 e / 2^-8 of the values. Sums of some hundred float32 roundings of random sign have e of about 2^-22, and some outputs cancel to a
few times below their terms: a share of about 2^-13. States or masked products of 16 bits (e = 2^-18 or more) would leave 2^-9 to 2^-10."""
import numpy as np
import pytest
import torch

from linear_testutil import host, make, states
from oracle import gka_linear_oracle as lin
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu

SHARE = 2.0 ** -12


def rounded_otherwise(got, want):
    return float((got.cpu() != torch.from_numpy(want).to(torch.bfloat16)).double().mean())


@pytest.mark.parametrize("d_k,d_v,H,H_kv", [(128, 128, 4, 4), (128, 128, 4, 2), (64, 64, 4, 4), (256, 128, 2, 2)])
@pytest.mark.parametrize("walk_chunks", [0, 1])
def test_forward(walk_chunks, d_k, d_v, H, H_kv):
    q, k, v, gate, _ = make(2, 200, H, H_kv, d_k, d_v)
    S = states(2, H_kv, d_v, d_k)
    o = binding.gka_linear_forward(q, k, v, gate, S_init=S, walk_chunks=walk_chunks)
    assert rounded_otherwise(o, lin.forward(*map(host, (q, k, v, gate, S)))[0]) <= SHARE
    # the states are as exact whether or not they are asked for
    again, _ = binding.gka_linear_forward(q, k, v, gate, S_init=S, walk_chunks=walk_chunks, return_state=True)
    assert torch.equal(o, again)


@pytest.mark.parametrize("d_k,d_v,H,H_kv", [(128, 128, 4, 4), (128, 128, 4, 2), (64, 128, 4, 2)])
def test_gradients(d_k, d_v, H, H_kv):
    q, k, v, gate, dy = make(2, 200, H, H_kv, d_k, d_v)
    S, dS = states(2, H_kv, d_v, d_k), states(2, H_kv, d_v, d_k, seed=6)
    got = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S, dS_final=dS)
    want = lin.backward(*map(host, (q, k, v, gate, dy, S, dS)))
    for n in ("dq", "dk", "dv"):
        assert rounded_otherwise(got[n], want[n]) <= SHARE, n


def test_wiped_states():
    """Decays of a chunk with gates of 0 at many tokens: far apart in their logarithms, and still differences of float32's precision."""
    q, k, v, gate, _ = make(2, 200, 4, 4, 128, 128)
    gate[:, 1::3] = 0.0
    o = binding.gka_linear_forward(q, k, v, gate)
    assert rounded_otherwise(o, lin.forward(*map(host, (q, k, v, gate)))[0]) <= SHARE


def test_shared_prefix():
    B, N, H, d = 64, 4, 8, 128
    q, k, v, gate, _ = make(B, 1, H, H, d, d)
    _, kc, vc, gc, _ = make(B, N, H, H, d, d, seed=1)
    S, n = states(2, H, d, d), torch.arange(B, device="cuda", dtype=torch.int32) % N
    one = lambda x: x[:, 0].contiguous()
    args = [host(x) for x in (S, one(q), one(k), one(v), one(gate), kc, vc, gc)]
    want = lin.decode_shared(*args, n.cpu().numpy(), np.zeros((B, H, d)))[0]
    o = binding.gka_linear_decode_shared(S, one(q), one(k), one(v), one(gate), kc, vc, gc, n)
    assert rounded_otherwise(o, want) <= SHARE
