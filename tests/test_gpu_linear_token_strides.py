"""Linear attention on tokens cut out of long tensors, rows more than 2^23 elements from batch to batch and token to token: to the
bits of packed rows."""
import pytest
import torch

from linear_testutil import make, states
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu


def far(x, tokens, heads_first):
    """[B, T, h, d] as a slice of T tokens of a tensor of `tokens`."""
    B, T, h, d = x.shape
    whole = torch.empty((B, h, tokens, d) if heads_first else (B, tokens, h, d), dtype=x.dtype, device=x.device)
    whole = whole.transpose(1, 2) if heads_first else whole
    part = whole[:, tokens // 2:tokens // 2 + T]
    part.copy_(x)
    return part


@pytest.mark.parametrize("heads_first", [False, True])
def test_one_token(heads_first):
    q, k, v, gate, dy = make(2, 1, 16, 8, 128, 128)
    S = states(2, 8, 128, 128)
    x = [far(t, 8192, heads_first) for t in (q, k, v)]
    one = lambda t: t[:, 0]
    a, b = S.clone(), S.clone()
    want = binding.gka_linear_decode(a, q, k, v, gate)
    assert torch.equal(binding.gka_linear_decode(b, *map(one, x), one(gate).contiguous()), one(want)) and torch.equal(a, b)
    assert torch.equal(binding.gka_linear_decode(S.clone(), *x, gate), want)
    out = far(torch.zeros_like(want), 8192, heads_first)
    assert torch.equal(binding.gka_linear_forward(*x, gate, S_init=S, out=out), binding.gka_linear_forward(q, k, v, gate, S_init=S))
    grads = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S)
    got = binding.gka_linear_backward(*x, gate, far(dy, 8192, heads_first), S_init=S)
    assert all(torch.equal(got[n], grads[n]) for n in grads)
    caches = lambda: [torch.zeros(2, 4, 8, 128, dtype=q.dtype, device="cuda"), torch.zeros(2, 4, 8, 128, dtype=q.dtype, device="cuda"),
                      torch.ones(2, 4, 8, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")]
    shared = lambda *t: binding.gka_linear_decode_shared(S, *t, one(gate).contiguous(), *caches())
    assert torch.equal(shared(*map(one, x)), shared(*(one(t).contiguous() for t in (q, k, v))))


def test_tokens_far_apart():
    """decode: tokens 2^23 elements from each other."""
    q, k, v, gate, _ = make(1, 3, 2, 2, 64, 64)
    S = states(1, 2, 64, 64)
    wide = torch.zeros(1, 3, 1 << 23, dtype=q.dtype, device="cuda")
    wide[..., :128] = q.flatten(2)
    rows = wide[..., :128].unflatten(-1, (2, 64))
    assert rows.stride(1) == 1 << 23
    assert torch.equal(binding.gka_linear_decode(S.clone(), rows, k, v, gate), binding.gka_linear_decode(S.clone(), q, k, v, gate))
