"""Linear attention with a decay for each head, whole sequences: parity with the float64 oracle."""
import numpy as np
import pytest
import torch

from linear_testutil import check_forward, host, make, states
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu


def run(B, T, H, H_kv, d_k, d_v, dtype="bf16", per_head=False, init=0, walk_chunks=0, **kw):
    q, k, v, gate, _ = make(B, T, H, H_kv, d_k, d_v, dtype, per_head, **kw)
    S_init = states(init, H_kv, d_v, d_k) if init else None
    o, S = binding.gka_linear_forward(q, k, v, gate, S_init=S_init, return_state=True, walk_chunks=walk_chunks)
    check_forward(o, S, q, k, v, gate, S_init)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 200])
def test_lengths(T, dtype):
    run(2, T, 2, 2, 64, 64, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_k,d_v", [(16, 16), (16, 256), (48, 80), (64, 128), (80, 48), (128, 64), (128, 128), (144, 32), (208, 192),
                                     (256, 16), (256, 256)])
def test_head_dimensions(d_k, d_v, dtype):
    run(1, 97, 2, 2, d_k, d_v, dtype, init=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (3, 1), (6, 2), (8, 1), (5, 5)])
@pytest.mark.parametrize("per_head", [False, True])
def test_heads(H, H_kv, per_head, dtype):
    run(2, 150, H, H_kv, 32, 64, dtype, per_head)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("walk_chunks", [1, 2, 3, 5, 100])
@pytest.mark.parametrize("init", [0, 1, 2])
def test_segments(walk_chunks, init, dtype):
    run(2, 401, 4, 2, 128, 128, dtype, init=init, walk_chunks=walk_chunks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_k,d_v", [(256, 256), (64, 32), (32, 256)])
def test_segments_of_other_shapes(d_k, d_v, dtype):
    run(2, 300, 2, 1, d_k, d_v, dtype, init=1, walk_chunks=1)


@pytest.mark.parametrize("gate_mean", [-2.0, 0.0, 6.0, 12.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_fast_and_slow_decays(gate_mean, dtype):
    run(1, 300, 2, 2, 64, 64, dtype, gate_mean=gate_mean, init=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("walk_chunks", [0, 1])
def test_gates_of_zero_and_one(walk_chunks, dtype):
    """Packed sequences: wiped states, several times within a chunk and at its borders; and no decay at all."""
    q, k, v, gate, _ = make(2, 260, 2, 2, 64, 64, dtype)
    gate[0, [0, 1, 2, 63, 64, 65, 100, 128, 191, 259]] = 0.0
    gate[1] = 1.0
    S_init = states(2, 2, 64, 64)
    o, S = binding.gka_linear_forward(q, k, v, gate, S_init=S_init, return_state=True, walk_chunks=walk_chunks)
    check_forward(o, S, q, k, v, gate, S_init)
    gate[:] = 0.0
    o, S = binding.gka_linear_forward(q, k, v, gate, S_init=S_init, return_state=True, walk_chunks=walk_chunks)
    check_forward(o, S, q, k, v, gate, S_init)


def _strided(x, layout):
    B, T, h, d = x.shape
    if layout == "heads":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "wide":                           # a slice of wider rows
        y = torch.full((B, T, h + 2, d + 16), float("nan"), dtype=x.dtype, device=x.device)
        y[:, :, 1:-1, 8:-8] = x
        return y[:, :, 1:-1, 8:-8]
    if layout == "time":                           # token-major batch
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layouts", [("heads",) * 4, ("wide",) * 4, ("time",) * 4, ("packed", "heads", "wide", "time")])
@pytest.mark.parametrize("B,H,H_kv", [(2, 4, 2), (1, 1, 1)])
def test_layouts(B, H, H_kv, layouts, dtype):
    q, k, v, gate, _ = make(B, 130, H, H_kv, 64, 96, dtype)
    out = torch.full((B, 130, H, 96), float("nan"), dtype=q.dtype, device="cuda")
    q, k, v, out = (_strided(x, l) for x, l in zip((q, k, v, out), layouts))
    whole = out if out._base is None else out._base
    before = torch.isnan(whole).sum().item()
    o, S = binding.gka_linear_forward(q, k, v, gate, return_state=True, out=out, walk_chunks=1)
    assert o is out
    check_forward(o, S, q, k, v, gate)
    assert before - torch.isnan(whole).sum().item() == out.numel()      # (nothing beside the output's rows was written)


def test_final_states_in_the_buffer_of_the_initial_ones():
    for walk_chunks in (0, 1):
        q, k, v, gate, _ = make(2, 200, 2, 2, 64, 128)
        S = states(2, 2, 128, 64)
        first = S.clone()
        o, S1 = binding.gka_linear_forward(q, k, v, gate, S_init=S, S_final=S, walk_chunks=walk_chunks)
        assert S1 is S
        check_forward(o, S, q, k, v, gate, first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_sequence(dtype):
    """Many chunks and segments; decays close to 1, so that early tokens matter to the end."""
    run(1, 5003, 2, 1, 32, 64, dtype, per_head=True, init=1)


def test_every_run_gives_the_same_bits():
    q, k, v, gate, _ = make(2, 700, 4, 2, 128, 128)
    o, S = binding.gka_linear_forward(q, k, v, gate, return_state=True)
    for _ in range(3):
        o2, S2 = binding.gka_linear_forward(q, k, v, gate, return_state=True)
        assert torch.equal(o, o2) and torch.equal(S, S2)


def test_workspace_contents_do_not_matter_and_its_end_is_kept():
    q, k, v, gate, _ = make(1, 900, 2, 2, 64, 64)
    want = binding.gka_linear_forward(q, k, v, gate)
    ws = binding.linear_workspace(q, k, v, gate)
    guarded = torch.full((ws.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    got = binding.gka_linear_forward(q, k, v, gate, workspace=guarded[:ws.numel()])
    assert torch.equal(want, got) and (guarded[ws.numel():] == 255).all()


def test_against_the_layer_without_its_solve():
    """alpha = 0 takes the layer's own readout to U_t q_t."""
    q, k, v, gate, _ = make(2, 300, 2, 2, 128, 128)
    lam, zero = torch.ones_like(gate), torch.zeros_like(gate)
    layer, st = binding.gka_forward(q, k, v, gate, lam, 2, alpha=zero, return_state=True)
    o, S = binding.gka_linear_forward(q, k, v, gate, return_state=True)
    # both outputs are bf16; the layer rounds its masked products to bf16 as well (2^-8 of terms that are below |v| 2 or so)
    assert (layer.float() - o.float()).abs().max().item() <= 2.0 ** -6 * host(o).max()
    assert (st["U_final"] - S).abs().max().item() <= 2.0 ** -8 * S.abs().max().item()
