"""Oracle of linear attention with a decay for each head, in float64, token by token from the definition:

    S_t = gamma_t S_{t-1} + v_t k_t^T,    y_{g,t} = S_t q_{g,t}        (S [d_v, d_k], g: the query heads that share S)

and its gradients by the recurrence's own chain rule. Nothing here is chunked; nothing is shared with the library.

Shapes: q [B,T,H,d_k], k [B,T,H_kv,d_k], v [B,T,H_kv,d_v], gate [B,T,H_kv] or [H_kv], states [B,H_kv,d_v,d_k] (initial ones
also [B/F,..]: each shared by F consecutive sequences).
"""
import numpy as np


def _f64(*xs):
    return [None if x is None else np.asarray(x, dtype=np.float64) for x in xs]


def _gates(gate, B, T, H_kv):
    return np.broadcast_to(gate, (B, T, H_kv)) if gate.ndim == 1 else gate


def _start(S_init, B, H_kv, d_v, d_k):
    if S_init is None:
        return np.zeros((B, H_kv, d_v, d_k))
    return np.repeat(S_init, B // S_init.shape[0], axis=0)


def forward(q, k, v, gate, S_init=None):
    """y [B,T,H,d_v] and the states after the last token."""
    q, k, v, gate, S_init = _f64(q, k, v, gate, S_init)
    B, T, H, d_k = q.shape
    H_kv, d_v = v.shape[2:]
    g = _gates(gate, B, T, H_kv)
    S = _start(S_init, B, H_kv, d_v, d_k)
    y = np.empty((B, T, H, d_v))
    for t in range(T):
        S = g[:, t, :, None, None] * S + v[:, t, :, :, None] * k[:, t, :, None, :]
        y[:, t] = np.einsum("bhij,bhgj->bhgi", S, q[:, t].reshape(B, H_kv, H // H_kv, d_k)).reshape(B, H, d_v)
    return y, S


def backward(q, k, v, gate, dy, S_init=None, dS_final=None):
    """dict of dq, dk, dv, dgate (like gate) and dS_init (like S_init; [B,..] without one) for the loss
    sum(y * dy) + sum(S_T * dS_final). dgate is the derivative itself, also at gates of 0."""
    q, k, v, gate, dy, S_init, dS_final = _f64(q, k, v, gate, dy, S_init, dS_final)
    B, T, H, d_k = q.shape
    H_kv, d_v = v.shape[2:]
    g = _gates(gate, B, T, H_kv)
    S = [_start(S_init, B, H_kv, d_v, d_k)]
    for t in range(T):
        S.append(g[:, t, :, None, None] * S[-1] + v[:, t, :, :, None] * k[:, t, :, None, :])
    dq, dk, dv, dgate = np.empty_like(q), np.empty_like(k), np.empty_like(v), np.empty((B, T, H_kv))
    R = np.zeros_like(S[0]) if dS_final is None else dS_final.copy()      # dL/dS_t
    for t in reversed(range(T)):
        qt, dyt = q[:, t].reshape(B, H_kv, -1, d_k), dy[:, t].reshape(B, H_kv, -1, d_v)
        R = R + np.einsum("bhgi,bhgj->bhij", dyt, qt)
        dq[:, t] = np.einsum("bhij,bhgi->bhgj", S[t + 1], dyt).reshape(B, H, d_k)
        dv[:, t] = np.einsum("bhij,bhj->bhi", R, k[:, t])
        dk[:, t] = np.einsum("bhij,bhi->bhj", R, v[:, t])
        dgate[:, t] = (R * S[t]).sum((-1, -2))
        R = g[:, t, :, None, None] * R
    if S_init is not None:
        R = R.reshape(S_init.shape[0], -1, *R.shape[1:]).sum(1)
    return {"dq": dq, "dk": dk, "dv": dv, "dgate": dgate.sum((0, 1)) if gate.ndim == 1 else dgate, "dS_init": R}


def decode_shared(S_prefix, q, k, v, gate, k_cache, v_cache, gate_cache, lengths, out):
    """(o, k_cache, v_cache, gate_cache) after one token of each sequence; `out`: what o holds of sequences that take no part."""
    S_prefix, q, k, v, gate, k_cache, v_cache, gate_cache, out = _f64(S_prefix, q, k, v, gate, k_cache, v_cache, gate_cache, out)
    B, N = k_cache.shape[:2]
    S0 = _start(S_prefix, B, *S_prefix.shape[1:])
    k_cache, v_cache, out = k_cache.copy(), v_cache.copy(), out.copy()
    gate_cache = None if gate_cache is None else gate_cache.copy()
    for b in range(B):
        n = int(lengths[b])
        if not 0 <= n < N:
            continue
        k_cache[b, n], v_cache[b, n] = k[b], v[b]
        if gate_cache is not None:
            gate_cache[b, n] = gate[b]
        S = S0[b]
        for j in range(n + 1):
            g = gate if gate_cache is None else gate_cache[b, j]
            S = g[:, None, None] * S + v_cache[b, j][:, :, None] * k_cache[b, j][:, None, :]
        out[b] = np.einsum("hij,hgj->hgi", S, q[b].reshape(S.shape[0], -1, S.shape[2])).reshape(out[b].shape)
    return out, k_cache, v_cache, gate_cache
