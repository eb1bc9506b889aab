"""Linear attention: infinities and NaN in a token's rows reach what depends on the token and nothing else. What does not depend on it
keeps its bits: it is compared with a run that has ordinary numbers there (rows that a padded batch leaves unwritten)."""
import pytest
import torch

from linear_testutil import make, states
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), float("-inf")]


def spoil(x, t0):
    """x with infinities and NaN in all rows from token t0 on."""
    x = x.clone()
    tail = x[:, t0:]
    tail.copy_(torch.tensor(BAD, device=x.device).to(x.dtype)[torch.arange(tail.numel(), device=x.device) % 3].view(tail.shape))
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,H_kv", [(64, 2, 2), (128, 4, 2), (128, 2, 2), (256, 2, 1)])
@pytest.mark.parametrize("walk_chunks", [0, 1])
@pytest.mark.parametrize("t0", [1, 5, 20, 37, 64, 117])
def test_tokens_before_keep_their_outputs(t0, walk_chunks, d, H, H_kv, dtype):
    q, k, v, gate, _ = make(2, 150, H, H_kv, d, d, dtype, seed=t0)
    S = states(2, H_kv, d, d)
    want = binding.gka_linear_forward(q, k, v, gate, S_init=S, walk_chunks=walk_chunks)
    for which in ((0,), (1,), (2,), (3,), (0, 1, 2, 3)):
        x = [spoil(t, t0) if i in which else t for i, t in enumerate((q, k, v, gate))]
        o = binding.gka_linear_forward(*x, S_init=S, walk_chunks=walk_chunks)
        assert torch.equal(o[:, :t0], want[:, :t0]), which
        if which != (3,):                          # (what gates outside 0 .. 1 do to their own tokens is not defined)
            assert not torch.isfinite(o[:, t0:]).all(-1).any(), which


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("walk_chunks", [0, 1])
@pytest.mark.parametrize("bad", BAD)
def test_one_feature_of_one_token(bad, walk_chunks, dtype):
    T, d = 150, 128
    q, k, v, gate, _ = make(2, T, 4, 2, d, d, dtype)
    want, S_want = binding.gka_linear_forward(q, k, v, gate, return_state=True, walk_chunks=walk_chunks)
    for t, f in ((0, 0), (17, 5), (40, 127), (63, 64), (149, 30)):
        x = v.clone()
        x[1, t, 1, f] = bad
        o, S = binding.gka_linear_forward(q, k, x, gate, return_state=True, walk_chunks=walk_chunks)
        spoilt = torch.zeros_like(o, dtype=torch.bool)
        spoilt[1, t:, 2:, f] = True                # (kv head 1: query heads 2 and 3)
        assert torch.equal(o[~spoilt], want[~spoilt]) and not torch.isfinite(o[spoilt]).any(), (t, f)
        spoilt = torch.zeros_like(S, dtype=torch.bool)
        spoilt[1, 1, f] = True
        assert torch.equal(S[~spoilt], S_want[~spoilt]) and not torch.isfinite(S[spoilt]).any(), (t, f)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,H_kv", [(64, 2, 2), (128, 4, 2), (128, 2, 2)])
@pytest.mark.parametrize("walk_chunks", [0, 1])
@pytest.mark.parametrize("t0", [5, 37, 64, 117])
def test_gradients(t0, walk_chunks, d, H, H_kv, dtype):
    q, k, v, gate, dy = make(2, 150, H, H_kv, d, d, dtype, seed=t0)
    S, dS = states(2, H_kv, d, d), states(2, H_kv, d, d, seed=6)
    grads = lambda q, k, v, dy: binding.gka_linear_backward(q, k, v, gate, dy, S_init=S, dS_final=dS, walk_chunks=walk_chunks)
    want = grads(q, k, v, dy)
    # dq of a token depends on the keys and values up to it
    for x in ((q, spoil(k, t0), v, dy), (q, k, spoil(v, t0), dy)):
        assert torch.equal(grads(*x)["dq"][:, :t0], want["dq"][:, :t0])
    # dk and dv on the queries and gradients from it on
    front = lambda x: spoil(x.flip(1), 150 - t0).flip(1).contiguous()
    for x in ((front(q), k, v, dy), (q, k, v, front(dy))):
        got = grads(*x)
        assert torch.equal(got["dk"][:, t0:], want["dk"][:, t0:]) and torch.equal(got["dv"][:, t0:], want["dv"][:, t0:])


def test_a_padded_batch_with_gates_of_zero_is_cut_off():
    """Tokens of other sequences behind a gate of 0 in one row of the batch: nothing of later ones reaches earlier ones."""
    q, k, v, gate, _ = make(1, 200, 2, 2, 64, 64)
    gate[:, 90] = 0.0
    want = binding.gka_linear_forward(q, k, v, gate)
    o = binding.gka_linear_forward(spoil(q, 90), spoil(k, 90), spoil(v, 90), gate)
    assert torch.equal(o[:, :90], want[:, :90])
