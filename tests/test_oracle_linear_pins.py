"""Pins of the linear-attention oracle: explicit double sums, reductions to simpler cases, finite differences."""
import numpy as np
import pytest

from oracle import gka_linear_oracle as lin


def _inputs(B=2, T=5, H=4, H_kv=2, d_k=3, d_v=2, per_head=False, seed=0):
    r = np.random.default_rng(seed)
    gate = r.uniform(0.3, 1.0, H_kv) if per_head else r.uniform(0.3, 1.0, (B, T, H_kv))
    return (r.standard_normal((B, T, H, d_k)), r.standard_normal((B, T, H_kv, d_k)), r.standard_normal((B, T, H_kv, d_v)), gate)


def _double_sum(q, k, v, gate, S0=None):
    B, T, H, _ = q.shape
    H_kv = k.shape[2]
    y = np.zeros((B, T, H, v.shape[-1]))
    for b in range(B):
        for h in range(H):
            m = h // (H // H_kv)
            g = np.full(T, gate[m]) if gate.ndim == 1 else gate[b, :, m]
            for t in range(T):
                for s in range(t + 1):
                    y[b, t, h] += np.prod(g[s + 1:t + 1]) * (k[b, s, m] @ q[b, t, h]) * v[b, s, m]
                if S0 is not None:
                    y[b, t, h] += np.prod(g[:t + 1]) * S0[b // (B // S0.shape[0]), m] @ q[b, t, h]
    return y


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_forward_is_the_double_sum(per_head, shared):
    q, k, v, gate = _inputs(per_head=per_head)
    S0 = np.random.default_rng(1).standard_normal((1 if shared else 2, 2, 2, 3))
    np.testing.assert_allclose(lin.forward(q, k, v, gate)[0], _double_sum(q, k, v, gate), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(lin.forward(q, k, v, gate, S0)[0], _double_sum(q, k, v, gate, S0), rtol=1e-12, atol=1e-12)


def test_final_state_continues_the_sequence():
    q, k, v, gate = _inputs(T=7)
    whole, S = lin.forward(q, k, v, gate)
    first, S1 = lin.forward(q[:, :3], k[:, :3], v[:, :3], gate[:, :3])
    rest, S2 = lin.forward(q[:, 3:], k[:, 3:], v[:, 3:], gate[:, 3:], S1)
    np.testing.assert_allclose(np.concatenate([first, rest], 1), whole, rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(S2, S, rtol=1e-12, atol=1e-13)


def test_a_gate_of_zero_starts_anew():
    q, k, v, gate = _inputs(T=6)
    gate[:, 4] = 0.0
    np.testing.assert_allclose(lin.forward(q, k, v, gate)[0][:, 4:], lin.forward(q[:, 4:], k[:, 4:], v[:, 4:], gate[:, 4:])[0],
                               rtol=1e-12)


@pytest.mark.parametrize("per_head", [False, True])
def test_gradients_are_the_differences(per_head):
    q, k, v, gate = _inputs(per_head=per_head)
    r = np.random.default_rng(2)
    S0, dy, dS = r.standard_normal((1, 2, 2, 3)), r.standard_normal((2, 5, 4, 2)), r.standard_normal((2, 2, 2, 3))
    got = lin.backward(q, k, v, gate, dy, S0, dS)

    def loss(*x):
        y, S = lin.forward(*x)
        return (y * dy).sum() + (S * dS).sum()

    x = [q, k, v, gate, S0]
    for i, name in enumerate(("dq", "dk", "dv", "dgate", "dS_init")):
        want = np.empty_like(x[i])
        for at in np.ndindex(x[i].shape):
            e = np.zeros_like(x[i])
            e[at] = 1e-5
            want[at] = (loss(*x[:i], x[i] + e, *x[i + 1:]) - loss(*x[:i], x[i] - e, *x[i + 1:])) / 2e-5
        # (the loss is a polynomial of degree T + 2 with values of order 10: differences hold to h^2 + 1e-16 / h, about 1e-9)
        np.testing.assert_allclose(got[name], want, rtol=1e-6, atol=1e-6, err_msg=name)


def test_decay_gradient_from_the_products_of_the_others():
    """dgamma_t gamma_t = <dS_final, S_T> + sum_{s >= t} (q_s . dq_s - k_s . dk_s): what the library sums up."""
    q, k, v, gate = _inputs(T=9)
    r = np.random.default_rng(3)
    S0, dy, dS = r.standard_normal((2, 2, 2, 3)), r.standard_normal((2, 9, 4, 2)), r.standard_normal((2, 2, 2, 3))
    got = lin.backward(q, k, v, gate, dy, S0, dS)
    S = lin.forward(q, k, v, gate, S0)[1]
    x = (q * got["dq"]).sum(-1).reshape(2, 9, 2, 2).sum(-1) - (k * got["dk"]).sum(-1)
    total = np.flip(np.cumsum(np.flip(x, 1), 1), 1) + (S * dS).sum((-1, -2))[:, None]
    np.testing.assert_allclose(got["dgate"] * gate, total, rtol=1e-10, atol=1e-10)


@pytest.mark.parametrize("per_head", [False, True])
def test_shared_decode_is_the_whole_sequence(per_head):
    q, k, v, gate = _inputs(B=4, T=6, per_head=per_head)
    S0 = np.random.default_rng(4).standard_normal((2, 2, 2, 3))
    y, _ = lin.forward(q, k, v, gate, S0)
    N = 6
    kc, vc = np.zeros((4, N, 2, 3)), np.zeros((4, N, 2, 2))
    gc = None if per_head else np.ones((4, N, 2))
    for t in range(6):
        lengths = np.array([t, t, t, -1])
        o, kc, vc, gc = lin.decode_shared(S0, q[:, t], k[:, t], v[:, t], gate if per_head else gate[:, t], kc, vc, gc, lengths,
                                          np.full((4, 4, 2), 7.0))
        np.testing.assert_allclose(o[:3], y[:3, t], rtol=1e-11, atol=1e-12)
        assert (o[3] == 7.0).all() and (kc[3] == 0).all()
