"""Linear attention as a program uses it: a prompt, tokens on its states, samples behind a shared prefix, folding their caches
into states; calls on other streams and in HIP graphs; a training step."""
import numpy as np
import pytest
import torch

from linear_testutil import check, check_backward, host, make, absolute, slack
from oracle import gka_linear_oracle as lin
from paper_2511_21016_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_samples_fold_and_tokens(dtype):
    """One prompt, four samples of it of up to 12 tokens in a suffix cache, their states from the cache, three more tokens on those."""
    H, H_kv, d_k, d_v, F, N = 4, 2, 64, 96, 4, 12
    q, k, v, gate, _ = make(1, 150, H, H_kv, d_k, d_v, dtype)
    sq, sk, sv, sg, _ = make(F, N + 3, H, H_kv, d_k, d_v, dtype, seed=1)
    _, S = binding.gka_linear_forward(q, k, v, gate, return_state=True)
    kc = torch.zeros(F, N, H_kv, d_k, dtype=q.dtype, device="cuda")
    vc = torch.zeros(F, N, H_kv, d_v, dtype=q.dtype, device="cuda")
    gc = torch.ones(F, N, H_kv, device="cuda")
    used = torch.tensor([12, 1, 7, 12])            # (the second and third stop early)
    lengths = torch.zeros(F, dtype=torch.int32, device="cuda")
    outs = []
    for t in range(N):
        now = torch.where(t < used.cuda(), lengths, -1)
        outs.append(binding.gka_linear_decode_shared(S, sq[:, t], sk[:, t], sv[:, t], sg[:, t].contiguous(), kc, vc, gc, now,
                                                     out=torch.zeros(F, H, d_v, dtype=q.dtype, device="cuda")))
        lengths += 1
    own = torch.empty(F, H_kv, d_v, d_k, device="cuda")
    binding.gka_linear_forward(torch.zeros_like(sq[:, :N]), kc, vc, gc, S_init=S, S_final=own)
    more = binding.gka_linear_decode(own, sq[:, N:], sk[:, N:], sv[:, N:], sg[:, N:].contiguous())
    for b in range(F):
        n = int(used[b])
        whole = [np.concatenate([host(x)[:1], host(y)[b:b + 1, :n], host(y)[b:b + 1, N:]], 1)
                 for x, y in ((q, sq), (k, sk), (v, sv), (gate, sg))]
        ref, mag = lin.forward(*whole), lin.forward(*map(absolute, whole))
        T = 150 + n + 3
        for t in range(n):
            check("sample", outs[t][b], ref[0][0, 150 + t], mag[0][0, 150 + t], d_k, d_v, T)
        assert all((outs[t][b] == 0).all() for t in range(n, N))
        check("tokens", more[b], ref[0][0, 150 + n:], mag[0][0, 150 + n:], d_k, d_v, T)
        check("state", own[b], ref[1][0], mag[1][0], d_k, d_v, T)


class _Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, gate):
        ctx.save_for_backward(q, k, v, gate)
        return binding.gka_linear_forward(q, k, v, gate)

    @staticmethod
    def backward(ctx, dy):
        g = binding.gka_linear_backward(*ctx.saved_tensors, dy.contiguous())
        return g["dq"], g["dk"], g["dv"], g["dgate"]


def test_training_step_through_autograd():
    q, k, v, gate, dy = make(2, 130, 4, 2, 64, 64)
    leaves = [x.requires_grad_() for x in (q, k, v, gate)]
    _Layer.apply(*leaves).backward(dy)
    check_backward({n: x.grad for n, x in zip(("dq", "dk", "dv", "dgate"), leaves)}, *(x.detach() for x in leaves), dy)


def test_other_streams():
    """Two calls at once on two streams, with a workspace each."""
    a, b = make(2, 700, 4, 2, 64, 128), make(2, 700, 4, 2, 64, 128, seed=7)
    want = [(binding.gka_linear_forward(*x[:4]), binding.gka_linear_backward(*x)) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, x in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append((binding.gka_linear_forward(*x[:4]), binding.gka_linear_backward(*x)))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w[0], g[0]) and all(torch.equal(w[1][n], g[1][n]) for n in w[1])


def test_graph_of_all_calls():
    """Captured once, replayed with new inputs and eager work in between: every replay gives the eager result. Two graphs with a
    workspace each."""
    H, H_kv, d, F = 4, 2, 64, 4
    q, k, v, gate, dy = make(1, 500, H, H_kv, d, d)
    tq, tk, tv, tg, _ = (x[:, 0].contiguous() for x in make(F, 1, H, H_kv, d, d, seed=1))
    kc, vc = (torch.zeros(F, 8, H_kv, d, dtype=q.dtype, device="cuda") for _ in range(2))
    gc = torch.ones(F, 8, H_kv, device="cuda")
    lengths = torch.zeros(F, dtype=torch.int32, device="cuda")
    o = torch.empty_like(q)
    S = torch.zeros(1, H_kv, d, d, device="cuda")
    S4 = torch.zeros(F, H_kv, d, d, device="cuda")
    so, to = (torch.zeros(F, H, d, dtype=q.dtype, device="cuda") for _ in range(2))

    def step(ws, wsb):
        binding.gka_linear_forward(q, k, v, gate, S_final=S, out=o, workspace=ws)
        g = binding.gka_linear_backward(q, k, v, gate, dy, workspace=wsb)
        binding.gka_linear_decode_shared(S, tq, tk, tv, tg, kc, vc, gc, lengths, out=so)
        binding.gka_linear_decode(S, tq, tk, tv, tg, S_out=S4, out=to)
        lengths.add_(1)
        return [o, S, so, to, S4, kc, vc, *g.values()]

    spaces = [(binding.linear_workspace(q, k, v, gate), binding.linear_workspace(q, k, v, gate, backward=True)) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*spaces[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for ws in spaces[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step(*ws)
        graphs.append((graph, outs))
    for i in range(4):
        q.copy_(make(1, 500, H, H_kv, d, d, seed=10 + i)[0])
        dy.mul_(0.5)
        lengths.fill_(i)
        kc0, vc0, gc0 = kc.clone(), vc.clone(), gc.clone()
        eager = [x.clone() for x in step(*spaces[2])]
        torch.cuda.synchronize()
        for graph, outs in graphs:
            lengths.fill_(i)
            for x, y in zip((kc, vc, gc), (kc0, vc0, gc0)):
                x.copy_(y)
            for x in (o, S, so, to, S4):
                x.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, eager):
                assert torch.equal(a, b)
