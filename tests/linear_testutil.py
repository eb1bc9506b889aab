"""Inputs, bounds and comparisons of the linear-attention tests.

Bounds. `absolute` is the oracle's result on the inputs' magnitudes: the sum of |term| over everything that is summed up for an
output. A float32 chain of n roundings is off by at most n 2^-24 of it; a term passes through a dot product over the
features, sums over the tokens behind it and some 64 roundings of its decay (exp2 of a difference of log2 sums), weights and pieces:
n = d_k + d_v + T + 64. A bf16 output adds half a step, 2^-8 |y|, and two-piece operands 2^-16 of the sum: two pieces of 8 bits, rounded.
"""
import numpy as np
import torch

from oracle import gka_linear_oracle as lin

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(B, T, H, H_kv, d_k, d_v, dtype="bf16", per_head=False, gate_mean=3.0, seed=0, device="cuda"):
    """q, k, v, gate, dy on the device; q and k normalised."""
    r = np.random.default_rng(seed)

    def rows(*shape, unit=False):
        x = r.standard_normal(shape)
        x = x / np.linalg.norm(x, axis=-1, keepdims=True) if unit else x
        return torch.tensor(x, dtype=torch.float32).to(DTYPES[dtype]).to(device)

    gate = 1 - 2.0 ** (-3 - 6 * r.random(H_kv)) if per_head else 1 / (1 + np.exp(-(r.standard_normal((B, T, H_kv)) + gate_mean)))
    return (rows(B, T, H, d_k, unit=True), rows(B, T, H_kv, d_k, unit=True), rows(B, T, H_kv, d_v),
            torch.tensor(gate, dtype=torch.float32, device=device), rows(B, T, H, d_v))


def states(n, H_kv, d_v, d_k, seed=5, device="cuda"):
    return torch.tensor(np.random.default_rng(seed).standard_normal((n, H_kv, d_v, d_k)) * 3 / np.sqrt(d_k), dtype=torch.float32,
                        device=device)


def host(x):
    return None if x is None else x.detach().float().cpu().numpy().astype(np.float64)


def absolute(x):
    return None if x is None else np.abs(x)


def slack(d_k, d_v, T, dtype):
    """(relative to the output, relative to the sum of magnitudes) that an output of this type may be off by."""
    n = d_k + d_v + T + 64
    return (2.0 ** -8, 2.0 ** -16 + n * 2.0 ** -24) if dtype == torch.bfloat16 else (0.0, n * 2.0 ** -24)


def check(name, got, want, magnitude, d_k, d_v, T):
    assert got.dtype in (torch.float32, torch.bfloat16)
    rel, total = slack(d_k, d_v, T, got.dtype)
    got = host(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    over = np.abs(got - want) - (rel * np.abs(want) + total * magnitude + 1e-30)
    assert np.isfinite(got).all() and over.max() <= 0, (name, float(over.max()), np.unravel_index(over.argmax(), over.shape))


def near(name, got, want, bound):
    """Relative distance in the 2-norm."""
    off = float(np.linalg.norm(host(got) - want) / max(np.linalg.norm(want), 1e-300))
    assert off <= bound, (name, off)


def check_forward(got, S, q, k, v, gate, S_init=None):
    args = [host(x) for x in (q, k, v, gate, S_init)]
    d_k, (T, d_v) = q.shape[-1], (q.shape[1], v.shape[-1])
    y, S_ref = lin.forward(*args)
    y_abs, S_abs = lin.forward(*map(absolute, args))
    check("o", got, y, y_abs, d_k, d_v, T)
    if S is not None:
        check("S_final", S, S_ref, S_abs, d_k, d_v, T)
        # three pieces of 8 bits hold a float32: roundings of random sign, sqrt(T) 2^-24 at most on average
        near("S_final", S, S_ref, 2.0 ** -24 * max(4.0, np.sqrt(T)))


def check_backward(got, q, k, v, gate, dy, S_init=None, dS_final=None):
    args = [host(x) for x in (q, k, v, gate, dy, S_init, dS_final)]
    d_k, (T, d_v) = q.shape[-1], (q.shape[1], v.shape[-1])
    ref, mag = lin.backward(*args), lin.backward(*map(absolute, args))
    n = d_k + d_v + T + 64
    for name in ("dq", "dk", "dv", *(["dS_init"] if S_init is not None else [])):
        check(name, got[name], ref[name], mag[name], d_k, d_v, T)
    # dgate: the sums q . dq and k . dk over the tokens from t on, each term as exact as a float32 output, divided by the gate
    group = q.shape[2] // k.shape[2]
    a = (args[0], args[1])
    x = (np.abs(a[0]) * mag["dq"]).sum(-1).reshape(*q.shape[:2], k.shape[2], group).sum(-1) + (np.abs(a[1]) * mag["dk"]).sum(-1)
    total = np.flip(np.cumsum(np.flip(x, 1), 1), 1)
    if dS_final is not None:
        S_abs = lin.forward(*map(absolute, (args[0], args[1], args[2], args[3], args[5])))[1]
        total = total + (S_abs * np.abs(args[6])).sum((-1, -2))[:, None]
    bound = total * n * 2.0 ** -24 / args[3]
    if gate.dim() == 1:
        bound = bound.sum((0, 1))
    over = np.abs(host(got["dgate"]) - ref["dgate"]) - bound - 2.0 ** -24 * np.abs(ref["dgate"])
    assert over.max() <= 0, ("dgate", float(over.max()))
    near("dgate", got["dgate"], ref["dgate"], 2e-5)
    return ref
