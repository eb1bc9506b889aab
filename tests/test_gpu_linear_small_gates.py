"""Linear attention, the gradient of gates close to 0: <dS_t, S_{t-1}>, of the size of the states whatever the gate is.

Bounds. In a chunk that holds a gate below 1/16 (64 tokens, float32 tensors 32) the gradients are sums of products that carry no
division: off by at most n 2^-24 of their magnitudes' sum (the oracle on the inputs' magnitudes), n = d_k + d_v + T + 64 as in
linear_testutil. Elsewhere they are a sum over the tokens from t on, each as exact as a float32 output, over a gate of 1/16 at least."""
import numpy as np
import pytest
import torch

from linear_testutil import absolute, host, make, near, states
from oracle import gka_linear_oracle as lin
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu

SMALL = 1 / 16
WIPED = 3.8e-44


def check_dgate(got, q, k, v, gate, dy, S_init=None, dS_final=None, norm=2e-5):
    args = [host(x) for x in (q, k, v, gate, dy, S_init, dS_final)]
    T, d_k, d_v = q.shape[1], q.shape[-1], v.shape[-1]
    ref, mag = lin.backward(*args), lin.backward(*map(absolute, args))
    tokens = np.broadcast_to(args[3], (q.shape[0], T, k.shape[2]))
    # the derivatives of single tokens also where there is one gate for a head
    if gate.dim() == 1:
        ref_t = lin.backward(*args[:3], tokens, *args[4:])["dgate"]
        mag_t = lin.backward(*map(absolute, args[:3]), tokens, *map(absolute, args[4:]))["dgate"]
    else:
        ref_t, mag_t = ref["dgate"], mag["dgate"]
    C = 64 if q.dtype == torch.bfloat16 else 32
    padded = np.pad(tokens, ((0, 0), (0, -T % C), (0, 0)), constant_values=1.0)
    small = ((padded > WIPED) & (padded < SMALL)).reshape(q.shape[0], -1, C, k.shape[2]).any(2).repeat(C, 1)[:, :T]
    n = d_k + d_v + T + 64
    x = (np.abs(args[0]) * mag["dq"]).sum(-1).reshape(*q.shape[:2], k.shape[2], -1).sum(-1) + (np.abs(args[1]) * mag["dk"]).sum(-1)
    total = np.flip(np.cumsum(np.flip(x, 1), 1), 1)
    if dS_final is not None:
        S_abs = lin.forward(*map(absolute, (args[0], args[1], args[2], args[3], args[5])))[1]
        total = total + (S_abs * np.abs(args[6])).sum((-1, -2))[:, None]
    bound = n * 2.0 ** -24 * np.where(small, mag_t, total / np.maximum(tokens, SMALL)) + 2.0 ** -24 * np.abs(ref_t)
    out = host(got["dgate"])
    wiped = tokens <= WIPED
    if gate.dim() == 1:
        assert (np.abs(out - np.where(wiped, 0, ref_t).sum((0, 1))) <= bound.sum((0, 1)) + 2.0 ** -24 * np.abs(out)).all()
        return
    assert (out[wiped] == 0).all()
    over = np.where(wiped, 0, np.abs(out - ref_t) - bound)
    assert over.max() <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))
    near("dgate", torch.from_numpy(np.where(wiped, 0, out)), np.where(wiped, 0, ref_t), norm)


def run(B, T, H, H_kv, d_k, d_v, dtype, gates, init=0, final=False, walk_chunks=0, **kw):
    """gates: {token: value}, of the last head; or a function of the gates"""
    q, k, v, gate, dy = make(B, T, H, H_kv, d_k, d_v, dtype, **kw)
    if callable(gates):
        gate = gates(gate)
    else:
        for t, g in gates.items():
            gate[:, t, -1] = g
    S = states(init, H_kv, d_v, d_k) if init else None
    dS = states(B, H_kv, d_v, d_k, seed=6) if final else None
    got = binding.gka_linear_backward(q, k, v, gate, dy, S_init=S, dS_final=dS, walk_chunks=walk_chunks)
    check_dgate(got, q, k, v, gate, dy, S, dS)


VALUES = [0.06, 1e-2, 1e-4, 1e-8, 1e-20, 1e-36, 1e-42]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [0, 1, 31, 32, 63, 64, 100, 199])
def test_one_small_gate(t, dtype):
    for i, g in enumerate(VALUES):
        run(1, 200, 2, 2, 64, 64, dtype, {t: g}, init=i % 2, final=i % 3 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("walk_chunks", [0, 1, 2, 3])
@pytest.mark.parametrize("H,H_kv,d_k,d_v", [(2, 2, 128, 128), (4, 2, 64, 128), (3, 1, 128, 64), (2, 2, 256, 144), (2, 1, 48, 80), (1, 1, 16, 256),
                                            (2, 2, 144, 16)])
def test_shapes_and_segments(H, H_kv, d_k, d_v, walk_chunks, dtype):
    run(2, 333, H, H_kv, d_k, d_v, dtype, {0: 1e-6, 70: 1e-3, 71: 1e-9, 190: 1e-20, 191: 0.0, 195: 2e-2, 320: 1e-5, 332: 1e-7}, init=1,
        final=True, walk_chunks=walk_chunks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 65, 128])
def test_lengths(T, dtype):
    for init, final in ((0, False), (1, False), (0, True), (2, True)):
        run(2, T, 2, 1, 32, 48, dtype, {T - 1: 1e-5, T // 2: 1e-12, 0: 1e-3}, init=init, final=final)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate_mean", [-20.0, -6.0, -3.0, -1.0])
def test_many_small_gates(gate_mean, dtype):
    run(2, 300, 4, 2, 64, 64, dtype, {}, init=2, final=True, gate_mean=gate_mean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_gates_between_wiping_ones(dtype):
    def gates(gate):
        gate[:, [0, 5, 63, 64, 65, 130, 199]] = 0.0
        gate[:, [1, 4, 6, 62, 66, 129, 131, 198]] = 1e-10
        return gate
    run(2, 200, 2, 2, 64, 64, dtype, gates, init=1, final=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_gate_for_a_head(dtype):
    run(2, 300, 8, 4, 64, 64, dtype, lambda _: torch.tensor([1e-30, 1e-3, 0.9, 0.0], device="cuda"), init=1, final=True, per_head=True)


def test_tensors_with_strides():
    q, k, v, gate, dy = make(2, 130, 4, 2, 64, 96)
    gate[:, 40::50] = 1e-9
    want = binding.gka_linear_backward(q, k, v, gate, dy)
    turned = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, dy)]
    assert torch.equal(binding.gka_linear_backward(*turned[:3], gate, turned[3])["dgate"], want["dgate"])
    check_dgate(want, q, k, v, gate, dy)


@pytest.mark.parametrize("per_head", [False, True])
def test_more_tokens_than_one_part_of_the_sum(per_head):
    if per_head:
        run(1, 4500, 2, 2, 16, 16, "f32", lambda _: torch.tensor([0.95, 1e-2], device="cuda"), per_head=True)
    else:
        run(1, 4500, 2, 2, 16, 16, "f32", {3: 1e-6, 4095: 1e-4, 4096: 1e-9, 4400: 1e-20}, final=True)


def test_more_chunks_than_workgroups():
    """Chunks with small gates here and there among many states."""
    def gates(gate):
        gate[3::7, 40] = 1e-7
        gate[::5, 99] = 1e-3
        return gate
    run(300, 100, 4, 4, 16, 16, "bf16", gates)


def test_what_wiping_gates_cut_off_stays_out():
    """Infinities and NaN in the rows of another packed sequence: behind it, the gradients of its own gates keep their bits."""
    q, k, v, gate, dy = make(1, 60, 2, 2, 64, 64)
    gate[:, [0, 30]] = 0.0
    gate[:, [10, 40]] = 1e-8
    want = binding.gka_linear_backward(q, k, v, gate, dy)["dgate"]
    bad = dy.clone()
    bad[:, 30:] = float("nan")
    got = binding.gka_linear_backward(q, k, v, gate, bad)["dgate"]
    assert torch.equal(got[:, :30], want[:, :30])


@pytest.mark.parametrize("g", [1e-8, 1e-30])
def test_differences(g):
    """The loss is linear in one gate: a large step has no curvature."""
    q, k, v, gate, dy = make(1, 100, 2, 1, 32, 32, "f32")
    S, dS = states(1, 1, 32, 32), states(1, 1, 32, 32, seed=6)
    for t in (0, 40, 99):
        x = gate.clone()
        x[:, t] = g
        got = binding.gka_linear_backward(q, k, v, x, dy, S_init=S, dS_final=dS)["dgate"][0, t, 0].item()

        def loss(value):
            x[:, t] = value
            o, S1 = binding.gka_linear_forward(q, k, v, x, S_init=S, return_state=True)
            return (o.double() * dy.double()).sum().item() + (S1.double() * dS.double()).sum().item()

        # outputs of float32: sqrt(terms) 2^-24 of their size, over the step
        noise = 2.0 ** -24 * 8 * float(dy.norm() * v.norm()) / 0.5
        assert abs((loss(0.5 + g) - loss(g)) / 0.5 - got) <= noise, (t, got)


def test_every_run_gives_the_same_bits_in_any_workspace_and_in_a_graph():
    q, k, v, gate, dy = make(2, 500, 4, 2, 64, 128)
    gate[:, 100::130] = 1e-9
    want = binding.gka_linear_backward(q, k, v, gate, dy)["dgate"]
    n = binding.linear_workspace(q, k, v, gate, backward=True).numel()
    for fill in (255, 0):
        ws = torch.full((n + 4096,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(binding.gka_linear_backward(q, k, v, gate, dy, workspace=ws[:n])["dgate"], want) and (ws[n:] == fill).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.gka_linear_backward(q, k, v, gate, dy, workspace=ws[:n])["dgate"]
    for i in range(3):
        gate[:, 50] = (0.9, 1e-5, 0.5)[i]          # (chunks come and go)
        want = binding.gka_linear_backward(q, k, v, gate, dy)["dgate"]
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
