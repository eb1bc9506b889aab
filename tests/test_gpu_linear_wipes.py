"""Linear attention, packed sequences: a gate of 0 is a border that nothing crosses, infinities and NaN of the sequence on its other side
included. What lies on this side keeps its bits: it is compared with a run that has ordinary numbers there."""
import pytest
import torch

from linear_testutil import make, states
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), float("-inf")]


def spoil(x, lo, hi):
    """x with infinities and NaN in all rows of tokens lo .. hi - 1."""
    x = x.clone()
    part = x[:, lo:hi]
    part.copy_(torch.tensor(BAD, device=x.device).to(x.dtype)[torch.arange(part.numel(), device=x.device) % 3].view(part.shape))
    return x


def bad_states(S):
    return torch.tensor(BAD, device=S.device)[torch.arange(S.numel(), device=S.device) % 3].view(S.shape)


def same(a, b):
    assert torch.isfinite(b).all()
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_k,d_v,H,H_kv", [(64, 64, 2, 2), (128, 128, 4, 2), (128, 128, 2, 2), (256, 256, 2, 1), (64, 256, 2, 2)])
@pytest.mark.parametrize("walk_chunks", [0, 1, 2])
@pytest.mark.parametrize("border", [1, 5, 31, 32, 63, 64, 65, 117, 128, 149])
def test_tokens_behind_a_border(border, walk_chunks, d_k, d_v, H, H_kv, dtype):
    q, k, v, gate, _ = make(2, 150, H, H_kv, d_k, d_v, dtype, seed=border)
    gate[:, border] = 0.0
    S = states(2, H_kv, d_v, d_k)
    run = lambda q, k, v, S: binding.gka_linear_forward(q, k, v, gate, S_init=S, return_state=True, walk_chunks=walk_chunks)
    want, S_want = run(q, k, v, S)
    bad = [spoil(x, 0, border) for x in (q, k, v)]
    for x in ((bad[0], k, v, S), (q, bad[1], v, S), (q, k, bad[2], S), (q, k, v, bad_states(S)), (*bad, bad_states(S))):
        o, S1 = run(*x)
        same(o[:, border:], want[:, border:])
        same(S1, S_want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("walk_chunks", [0, 1])
def test_a_sequence_between_two(walk_chunks, dtype):
    """Borders in one chunk, in neighbouring ones, next to each other; only the sequences in between are whole."""
    q, k, v, gate, _ = make(1, 400, 4, 2, 128, 128, dtype)
    starts = [0, 3, 4, 20, 50, 64, 100, 190, 260, 321, 400]
    gate[:, starts[:-1]] = 0.0
    want, S_want = binding.gka_linear_forward(q, k, v, gate, return_state=True, walk_chunks=walk_chunks)
    for odd in (0, 1):
        x = [q, k, v]
        for lo, hi in list(zip(starts, starts[1:]))[odd::2]:
            x = [spoil(t, lo, hi) for t in x]
        o, S = binding.gka_linear_forward(*x, gate, return_state=True, walk_chunks=walk_chunks)
        for lo, hi in list(zip(starts, starts[1:]))[1 - odd::2]:
            same(o[:, lo:hi], want[:, lo:hi])
        if odd == 0:
            same(S, S_want)
        else:
            assert not torch.isfinite(S).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv,d_k,d_v", [(2, 2, 64, 64), (4, 2, 128, 128), (2, 2, 128, 128), (4, 2, 64, 128)])
@pytest.mark.parametrize("walk_chunks", [0, 1])
@pytest.mark.parametrize("border", [1, 33, 63, 64, 65, 120, 149])
def test_gradients_on_both_sides_of_a_border(border, walk_chunks, H, H_kv, d_k, d_v, dtype):
    q, k, v, gate, dy = make(2, 150, H, H_kv, d_k, d_v, dtype, seed=border)
    gate[:, border] = 0.0
    if border > 1:
        gate[:, border // 2] = 1e-6                # (a gate whose gradient comes from the states)
    S, dS = states(2, H_kv, d_v, d_k), states(2, H_kv, d_v, d_k, seed=6)
    grads = lambda q, k, v, dy, S, dS: binding.gka_linear_backward(q, k, v, gate, dy, S_init=S, dS_final=dS, walk_chunks=walk_chunks)
    want = grads(q, k, v, dy, S, dS)
    before = grads(*(spoil(x, 0, border) for x in (q, k, v, dy)), bad_states(S), dS)
    behind = grads(*(spoil(x, border, 150) for x in (q, k, v, dy)), S, bad_states(dS))
    for n in ("dq", "dk", "dv", "dgate"):
        same(before[n][:, border:], want[n][:, border:])
        same(behind[n][:, :border], want[n][:, :border])
    same(behind["dS_init"], want["dS_init"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_gradient_at_initial_states_behind_a_first_gate_of_zero(dtype):
    q, k, v, gate, dy = make(2, 70, 2, 2, 64, 64, dtype)
    gate[:, 0] = 0.0
    got = binding.gka_linear_backward(q, k, v, gate, spoil(dy, 0, 70), S_init=states(2, 2, 64, 64))
    assert (got["dS_init"] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv", [(2, 2), (8, 2)])
def test_decode(H, H_kv, dtype):
    q, k, v, gate, _ = make(2, 5, H, H_kv, 64, 96, dtype)
    gate[:, 2] = 0.0
    S = states(2, H_kv, 96, 64)
    clean, S_clean = [], []
    for x in ((q, k, v, S), (*(spoil(t, 0, 2) for t in (q, k, v)), bad_states(S))):
        S_out = torch.empty_like(S)
        clean.append(binding.gka_linear_decode(x[3], *x[:3], gate, S_out=S_out))
        S_clean.append(S_out)
    same(clean[1][:, 2:], clean[0][:, 2:])
    same(S_clean[1], S_clean[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv", [(2, 2), (8, 2)])
@pytest.mark.parametrize("border", [0, 1, 40, 63, 64, 70, 128, 150])
def test_shared_prefix(border, H, H_kv, dtype):
    B, N, d = 4, 160, 64
    q, k, v, gate, _ = make(B, 1, H, H_kv, d, d, dtype)
    _, kc, vc, gc, _ = make(B, N, H, H_kv, d, d, dtype, seed=1)
    gc[:, border] = 0.0
    gc[:, border // 2] = 0.0
    S = states(1, H_kv, d, d)
    one = lambda x: x[:, 0].contiguous()
    n = torch.full((B,), 150, dtype=torch.int32, device="cuda")
    if border == 150:
        gate[:] = 0.0                              # (the new token's own)
    run = lambda S, kc, vc: binding.gka_linear_decode_shared(S, one(q), one(k), one(v), one(gate), kc.clone(), vc.clone(), gc.clone(), n)
    same(run(bad_states(S), spoil(kc, 0, border), spoil(vc, 0, border)), run(S, kc, vc))


def test_a_gate_of_zero_for_a_head():
    """Every token by itself."""
    q, k, v, _, dy = make(1, 130, 2, 2, 64, 64, "f32")
    gate = torch.tensor([0.0, 0.9], device="cuda")
    want = binding.gka_linear_forward(q, k, v, gate)
    x = [spoil(t, 60, 61) for t in (q, k, v)]
    o = binding.gka_linear_forward(*x, gate)
    same(torch.cat([o[:, :60, 0], o[:, 61:, 0]], 1), torch.cat([want[:, :60, 0], want[:, 61:, 0]], 1))
