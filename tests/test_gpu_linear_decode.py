"""Linear attention with a decay for each head, single tokens: stored states and shared prefixes."""
import numpy as np
import pytest
import torch

from linear_testutil import absolute, check, check_forward, host, make, states
from oracle import gka_linear_oracle as lin
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,H_kv,d_k,d_v", [(1, 1, 1, 1, 128, 128), (3, 1, 4, 2, 16, 16), (2, 5, 6, 2, 48, 80), (1, 2, 8, 1, 256, 256),
                                                (5, 1, 3, 3, 80, 16), (2, 13, 2, 2, 64, 144), (40, 1, 32, 32, 64, 64),
                                                (300, 2, 8, 8, 16, 96)])
@pytest.mark.parametrize("per_head", [False, True])
def test_decode(B, T, H, H_kv, d_k, d_v, per_head, dtype):
    q, k, v, gate, _ = make(B, T, H, H_kv, d_k, d_v, dtype, per_head)
    S = states(B, H_kv, d_v, d_k)
    S_out = torch.full_like(S, float("nan"))
    o = binding.gka_linear_decode(S, q, k, v, gate, S_out=S_out)
    check_forward(o, S_out, q, k, v, gate, S)
    # in place, to the same bits
    here = S.clone()
    assert torch.equal(binding.gka_linear_decode(here, q, k, v, gate), o) and torch.equal(here, S_out)


def test_decode_one_token_without_a_token_dimension():
    q, k, v, gate, _ = make(2, 3, 4, 2, 64, 64)
    S = states(2, 2, 64, 64)
    a, b = S.clone(), S.clone()
    many = binding.gka_linear_decode(a, q, k, v, gate)
    for t in range(3):
        one = binding.gka_linear_decode(b, q[:, t], k[:, t], v[:, t], gate[:, t].contiguous())
        assert torch.equal(one, many[:, t])
    assert torch.equal(a, b)


def test_decode_from_shared_states():
    q, k, v, gate, _ = make(6, 2, 2, 2, 64, 64)
    S = states(2, 2, 64, 64)
    S_out = torch.empty(6, 2, 64, 64, device="cuda")
    o = binding.gka_linear_decode(S, q, k, v, gate, S_out=S_out)
    check_forward(o, S_out, q, k, v, gate, S)


def test_decode_gate_of_zero():
    q, k, v, gate, _ = make(2, 3, 2, 2, 64, 64)
    gate[:, 1] = 0.0
    S = states(2, 2, 64, 64)
    S_out = torch.empty_like(S)
    check_forward(binding.gka_linear_decode(S, q, k, v, gate, S_out=S_out), S_out, q, k, v, gate, S)


def shared_inputs(P, F, N, H, H_kv, d_k, d_v, dtype, per_head, lengths, seed=0):
    B = P * F
    q, k, v, gate, _ = make(B, 1, H, H_kv, d_k, d_v, dtype, per_head, seed=seed)
    _, kc, vc, gc, _ = make(B, N, H, H_kv, d_k, d_v, dtype, per_head, seed=seed + 1)
    r = np.random.default_rng(seed + 2)
    lengths = torch.tensor(r.integers(0, N, B) if lengths is None else lengths, dtype=torch.int32, device="cuda")
    one = lambda x: x[:, 0].contiguous()
    return (states(P, H_kv, d_v, d_k), one(q), one(k), one(v), gate if per_head else one(gate), kc, vc, None if per_head else gc,
            lengths)


def check_shared(args, out):
    S, q, k, v, gate, kc, vc, gc, lengths = args
    d_k, d_v, N = q.shape[-1], v.shape[-1], kc.shape[1]
    n = lengths.cpu().numpy()
    before = out.clone()
    h = [host(x) for x in (S, q, k, v, gate, kc, vc, gc)]
    want = lin.decode_shared(*h, n, host(out))
    mag = lin.decode_shared(*map(absolute, h), n, np.zeros(out.shape))
    got = binding.gka_linear_decode_shared(S, q, k, v, gate, kc, vc, gc, lengths, out=out)
    assert got is out
    active = (n >= 0) & (n < N)
    check("o", out[torch.tensor(active)], want[0][active], mag[0][active], d_k, d_v, N)
    assert torch.equal(out[torch.tensor(~active)], before[torch.tensor(~active)])
    for x, ref in zip((kc, vc, gc), want[1:]):
        assert x is None or np.array_equal(host(x), ref)       # (bits: rows are copied or left alone)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,F,N,H,H_kv,d_k,d_v", [(1, 1, 1, 1, 1, 128, 128), (1, 4, 32, 2, 2, 128, 128), (2, 3, 65, 6, 2, 64, 64),
                                                  (1, 7, 200, 8, 1, 48, 80), (2, 37, 9, 5, 1, 16, 256), (3, 2, 130, 2, 2, 256, 16),
                                                  (1, 33, 40, 9, 3, 256, 256), (5, 1, 64, 2, 1, 80, 144)])
@pytest.mark.parametrize("per_head", [False, True])
def test_shared(P, F, N, H, H_kv, d_k, d_v, per_head, dtype):
    args = shared_inputs(P, F, N, H, H_kv, d_k, d_v, dtype, per_head, None)
    check_shared(args, torch.zeros(P * F, H, d_v, dtype=args[1].dtype, device="cuda"))


def test_shared_in_bulk():
    """So many sequences that a workgroup takes many columns."""
    args = shared_inputs(2, 300, 20, 8, 4, 64, 64, "bf16", False, None)
    check_shared(args, torch.zeros(600, 8, 64, dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_in_bulk_of_one_query_head_with_idle_rows(dtype):
    lengths = np.random.default_rng(4).integers(-3, 24, 2200)
    args = shared_inputs(2, 1100, 20, 4, 4, 64, 64, dtype, False, lengths)
    check_shared(args, torch.full((2200, 4, 64), 3.0, dtype=args[1].dtype, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_idle_rows_full_caches_and_borders(dtype):
    args = shared_inputs(2, 6, 129, 4, 2, 64, 64, dtype, False, [-1, 0, 1, 62, 63, 64, 65, 127, 128, 129, 2 ** 31 - 1, -2 ** 31])
    check_shared(args, torch.full((12, 4, 64), 3.0, dtype=args[1].dtype, device="cuda"))


def test_shared_rows_behind_the_length_are_not_read():
    args = list(shared_inputs(1, 4, 100, 2, 2, 64, 64, "bf16", False, [0, 10, 64, 99]))
    kc, vc, gc, lengths = args[5:]
    clean = [x.clone() for x in (kc, vc, gc)]
    want = binding.gka_linear_decode_shared(*args[:5], *clean, lengths)
    for b, n in enumerate(lengths.tolist()):
        for x in (kc, vc, gc):
            x[b, n:] = float("nan")
    assert torch.equal(binding.gka_linear_decode_shared(*args[:5], kc, vc, gc, lengths), want)


def test_shared_gates_of_zero():
    args = shared_inputs(1, 3, 80, 2, 2, 64, 64, "bf16", False, [5, 70, 79])
    args[7][:, [3, 66]] = 0.0
    check_shared(args, torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"))


def test_shared_cache_of_more_than_2_to_the_31_elements():
    N, H_kv, d = 1 << 18, 32, 256
    kc = torch.zeros(2, N, H_kv, d, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    gc = torch.ones(2, N, H_kv, device="cuda")
    S, q, k, v, gate, k8, v8, g8, _ = shared_inputs(1, 2, 8, 32, H_kv, d, d, "bf16", False, None)
    lengths = torch.tensor([7, 3], dtype=torch.int32, device="cuda")
    kc[:, :8], vc[:, :8], gc[:, :8] = k8, v8, g8
    want = binding.gka_linear_decode_shared(S, q, k, v, gate, k8, v8, g8, lengths)
    assert torch.equal(binding.gka_linear_decode_shared(S, q, k, v, gate, kc, vc, gc, lengths), want)
    assert torch.equal(kc[:, :8], k8) and torch.equal(vc[:, :8], v8)
    # the far end of one sequence's cache: all but the last rows hold nothing
    kc[1, N - 8:], vc[1, N - 8:], gc[1, N - 8:] = k8[1], v8[1], g8[1]
    kc[1, :8], vc[1, :8], gc[1, :8] = 0, 0, 1
    far = binding.gka_linear_decode_shared(S, q, k, v, gate, kc, vc, gc, torch.tensor([7, N - 8 + 3], dtype=torch.int32, device="cuda"))
    assert torch.equal(far[0], want[0]) and (far[1].float() - want[1].float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
