"""Linear attention with a decay for each head, gradients: parity with the float64 oracle and with differences."""
import numpy as np
import pytest
import torch

from linear_testutil import check_backward, host, make, states
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu


def run(B, T, H, H_kv, d_k, d_v, dtype="bf16", per_head=False, init=0, final=False, walk_chunks=0, **kw):
    q, k, v, gate, dy = make(B, T, H, H_kv, d_k, d_v, dtype, per_head, **kw)
    S_init = states(init, H_kv, d_v, d_k) if init else None
    dS = states(B, H_kv, d_v, d_k, seed=6) if final else None
    got = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S_init, dS_final=dS, walk_chunks=walk_chunks)
    check_backward(got, q, k, v, gate, dy, S_init, dS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 32, 63, 65, 130])
def test_lengths(T, dtype):
    run(2, T, 2, 2, 64, 64, dtype, init=2, final=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_k,d_v", [(16, 16), (16, 256), (48, 80), (64, 128), (128, 64), (128, 128), (256, 144), (256, 256)])
def test_head_dimensions(d_k, d_v, dtype):
    run(1, 97, 2, 2, d_k, d_v, dtype, init=1, final=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv", [(3, 1), (6, 2), (8, 1)])
@pytest.mark.parametrize("per_head", [False, True])
def test_heads_that_share_keys_and_values(H, H_kv, per_head, dtype):
    run(2, 150, H, H_kv, 32, 64, dtype, per_head, final=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("walk_chunks", [1, 2, 3, 100])
@pytest.mark.parametrize("init,final", [(0, False), (1, True), (2, False)])
def test_segments_and_states(walk_chunks, init, final, dtype):
    run(2, 401, 4, 2, 128, 128, dtype, init=init, final=final, walk_chunks=walk_chunks)


@pytest.mark.parametrize("share", [2, 3, 6])
def test_sequences_that_share_an_initial_state(share):
    run(6, 70, 2, 1, 64, 64, init=6 // share)


@pytest.mark.parametrize("gate_mean", [0.0, 8.0])
def test_fast_and_slow_decays(gate_mean):
    run(1, 300, 2, 2, 64, 64, gate_mean=gate_mean, init=1, final=True)


def test_a_long_sequence():
    run(1, 3001, 2, 2, 64, 64, gate_mean=5.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_sequences_have_the_gradients_of_their_parts(dtype):
    """A gate of 0: nothing flows through it, its own gradient is written as 0, those before are of their sequence alone."""
    q, k, v, gate, dy = make(1, 200, 2, 2, 64, 64, dtype)
    starts = [0, 1, 64, 70, 199]
    gate[:, starts] = 0.0
    got = binding.gka_linear_backward(q, k, v, gate, dy, walk_chunks=1)
    for lo, hi in zip(starts, starts[1:] + [200]):
        part = [x[:, lo:hi].contiguous() for x in (q, k, v, gate, dy)]
        part[3][:, 0] = 0.5                        # (multiplies a zero state)
        alone = {n: got[n][:, lo:hi] for n in ("dq", "dk", "dv", "dgate")}
        assert (alone["dgate"][:, 0] == 0).all()
        check_backward(alone, *part)


def test_layouts():
    q, k, v, gate, dy = make(2, 130, 4, 2, 64, 96)
    want = binding.gka_linear_backward(q, k, v, gate, dy)
    turned = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, dy)]
    got = binding.gka_linear_backward(*turned[:3], gate, turned[3])
    for n in want:
        assert got[n].is_contiguous() and torch.equal(got[n], want[n]), n


def test_differences():
    """Directional differences of the forward kernel itself, float32."""
    q, k, v, gate, dy = make(1, 100, 2, 1, 32, 32, "f32")
    S_init, dS = states(1, 1, 32, 32), states(1, 1, 32, 32, seed=6)
    got = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S_init, dS_final=dS)

    def loss(q, k, v, gate, S_init):
        o, S = binding.gka_linear_forward(q, k, v, gate, S_init=S_init, return_state=True)
        return (o.double() * dy.double()).sum().item() + (S.double() * dS.double()).sum().item()

    x = [q, k, v, gate, S_init]
    for i, n in enumerate(("dq", "dk", "dv", "dgate", "dS_init")):
        e = torch.randn(x[i].shape, generator=torch.Generator("cuda").manual_seed(i), device="cuda")
        h = 2.0 ** -9 * (0.05 if n == "dgate" else 1.0)
        up, down = ([y + s * h * e if j == i else y for j, y in enumerate(x)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * h)
        want = (got[n].double() * e.double()).sum().item()
        # outputs are float32 numbers of the loss's terms: sqrt(terms) 2^-24 of their size over 2 h, and the curvature h^2 e^3
        noise = 2.0 ** -24 * 8 * float(dy.norm() * v.norm()) / (2 * h)
        assert abs(slope - want) <= noise + 1e-3 * float(got[n].norm()), (n, slope, want, noise)


def test_every_run_gives_the_same_bits_and_keeps_the_workspaces_end():
    q, k, v, gate, dy = make(2, 500, 4, 2, 64, 128)
    S = states(1, 2, 128, 64)
    ws = binding.linear_workspace(q, k, v, gate, backward=True)
    guarded = torch.full((ws.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    want = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S)
    for _ in range(2):
        got = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S, workspace=guarded[:ws.numel()])
        assert all(torch.equal(got[n], want[n]) for n in want) and (guarded[ws.numel():] == 255).all()
