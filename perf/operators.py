"""Linear attention with a decay for each head, as a list of measurable cases.

The operators (float32 states S [d_v, d_k] of each sequence and key/value head; a query head reads the state of its group)
  forward    S_t = gamma_t S_{t-1} + v_t k_t^T, y_t = S_t q_t over whole sequences
  backward   its gradients at q, k, v, the decays and the initial state
  decode     one token, or a few, on stored states
  shared     one token of each of many sequences that continue a common prefix: the prefix is one state, the tokens
             behind it lie in a cache of keys, values and decays for each sequence

Inputs follow the synthetic workloads of this package (`synth.py`): L2-normalised q and k, v ~ N(0, 1), decays
sigmoid(N(m, 1)) per token and head, or one for each head between 1 - 2^-3 and 1 - 2^-9.

With `own` false `run` computes the plain form: chunk-wise products and sums in float32, decays in float64.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_CHUNK = 64

# Values that a case leaves out.
_DEFAULTS = {
    "dtype": "bf16",        # of q, k, v, y
    "per_head": False,      # one decay for each head instead of one per token and head
    "gate_mean": 3.0,       # m of the decays per token
    "packed": False,        # forward: several sequences one behind the other, a decay of 0 at the first token of each
    "layout": "packed",     # "fused": q, k, v are slices of one projection's output rows; "heads": stored [B, H, T, d]
    "init": False,          # continues from given states
    "F": 1,                 # consecutive sequences that share an initial state / a prefix
    "state": False,         # forward: the final states are asked for; backward: gradients at the states, too
    "N": 0,                 # shared: tokens that a suffix cache has room for
    "idle": False,          # shared: a padded batch, some of its rows hold no sequence
}


def listed():
    return [
        # --- prompts and the forward half of training
        # a short prompt of one sequence: the smallest call, where launches and latency count
        {"name": "forward_short_prompt", "kind": "forward", "B": 1, "H": 8, "Hkv": 8, "T": 77, "dk": 128, "dv": 128,
         "state": True},
        # the forward half of a training step of a 4K-context layer
        {"name": "forward_4k", "kind": "forward", "B": 4, "H": 16, "Hkv": 16, "T": 4096, "dk": 128, "dv": 128},
        # a long prompt, four query heads to a state, one decay for each head; the states go to the decode cache
        {"name": "forward_32k_grouped", "kind": "forward", "B": 1, "H": 32, "Hkv": 8, "T": 32768, "dk": 128, "dv": 128,
         "per_head": True, "state": True},
        # float32 tensors, narrow keys, an odd length, continued from states that two sequences share
        {"name": "forward_f32", "kind": "forward", "B": 4, "H": 4, "Hkv": 4, "T": 1001, "dk": 64, "dv": 128, "dtype": "f32",
         "gate_mean": 2.0, "init": True, "F": 2, "state": True},
        # --- training: the gradients
        # of the 4K-context layer
        {"name": "backward_4k", "kind": "backward", "B": 4, "H": 16, "Hkv": 16, "T": 4096, "dk": 128, "dv": 128},
        # of a grouped layer with one decay for each head, on a part of a longer sequence: states in, gradients at them out
        {"name": "backward_grouped", "kind": "backward", "B": 2, "H": 12, "Hkv": 4, "T": 1337, "dk": 64, "dv": 128,
         "per_head": True, "layout": "fused", "init": True, "state": True},
        # float32 tensors at a small size: numerics work, unit-test-like calls
        {"name": "backward_f32_small", "kind": "backward", "B": 1, "H": 2, "Hkv": 2, "T": 256, "dk": 64, "dv": 64,
         "dtype": "f32", "gate_mean": 2.0},
        # --- decoding
        # one interactive sequence
        {"name": "decode_1_sequence", "kind": "decode", "B": 1, "H": 16, "Hkv": 16, "T": 1, "dk": 128, "dv": 128},
        # a full serving batch: 256 sequences of a layer with 32 states each
        {"name": "decode_256_sequences", "kind": "decode", "B": 256, "H": 32, "Hkv": 32, "T": 1, "dk": 128, "dv": 128},
        # speculative decoding: four tokens per call, grouped heads
        {"name": "decode_4_tokens", "kind": "decode", "B": 48, "H": 32, "Hkv": 8, "T": 4, "dk": 128, "dv": 128,
         "per_head": True},
        # --- decoding behind a shared prefix
        # four samples of one prompt, short suffixes
        {"name": "shared_4_samples", "kind": "shared", "B": 4, "H": 16, "Hkv": 16, "dk": 128, "dv": 128, "F": 4, "N": 32},
        # sampling in bulk: 64 samples of each of four prompts, suffixes of up to 128 tokens, some rows of the batch idle
        {"name": "shared_256_samples", "kind": "shared", "B": 256, "H": 32, "Hkv": 32, "dk": 128, "dv": 128, "F": 64,
         "N": 128, "idle": True},
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _head_dims(rng):
    """Mostly the usual widths, now and then any multiple of 16 up to 256, and keys narrower than values."""
    roll = rng.random()
    if roll < 0.45:
        return 128, 128
    if roll < 0.6:
        return 64, 64
    if roll < 0.7:
        return 64, 128
    return 16 * rng.randint(1, 16), 16 * rng.randint(1, 16)


def draw(rng):
    kind = rng.choice(["forward", "forward", "backward", "decode", "shared"])
    dk, dv = _head_dims(rng)
    hkv = rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 32])
    group = rng.choice([1, 1, 1, 2, 3, 4, 8]) if hkv <= 8 else rng.choice([1, 1, 2])
    case = {"kind": kind, "H": hkv * group, "Hkv": hkv, "dk": dk, "dv": dv,
            "dtype": "bf16" if rng.random() < 0.75 else "f32", "per_head": rng.random() < 0.4}
    if not case["per_head"]:
        case["gate_mean"] = rng.choice([1.0, 2.0, 3.0, 4.0, 5.0])
    row = (dk + dv) * (group + 1) * hkv * (2 if case["dtype"] == "bf16" else 4)   # bytes of a token's rows
    if kind in ("forward", "backward"):
        longest = (1 << 29 if kind == "forward" else 1 << 28) // row
        case["B"] = _log_int(rng, 1, 32)
        case["T"] = _log_int(rng, 1, max(1, min(32768, longest // case["B"])))
        case["layout"] = rng.choice(["packed", "packed", "fused", "heads"])
        case["init"] = rng.random() < 0.4
        case["state"] = rng.random() < 0.5
        case["packed"] = kind == "forward" and not case["per_head"] and rng.random() < 0.2
    else:
        most = (1 << 29) // (4 * dk * dv * hkv)
        case["B"] = _log_int(rng, 1, max(1, min(256, most)))
        if kind == "decode":
            case["T"] = rng.choice([1, 1, 1, 1, 2, 3, 4, 5, 8, 13])
            case["init"] = True
        else:
            case["N"] = _log_int(rng, 1, max(1, min(256, (1 << 29) // (case["B"] * row))))
            case["idle"] = rng.random() < 0.3
    shares = [f for f in (2, 3, 4, 8, 16, 64) if case["B"] % f == 0]
    if shares and (kind == "shared" or (case.get("init") and rng.random() < 0.4)):
        case["F"] = rng.choice(shares)
    if kind == "shared" and rng.random() < 0.3:
        case["F"] = case["B"]
    return case


def _generator(seed):
    return torch.Generator("cuda").manual_seed(int(seed))


def _rows(case, gen):
    """q, k [..., d_k] and v [..., d_v] of B sequences of T tokens in the case's layout."""
    B, T, H, Hkv, dk, dv = (case[n] for n in ("B", "T", "H", "Hkv", "dk", "dv"))
    dtype = _DTYPES[case["dtype"]]

    def unit(*shape):
        return torch.nn.functional.normalize(torch.randn(*shape, generator=gen, device="cuda"), dim=-1).to(dtype)

    if case["layout"] == "fused":
        # one row per token: all queries, all keys, all values
        row = torch.empty(B, T, H * dk + Hkv * (dk + dv), dtype=dtype, device="cuda")
        q, k, v = (x.unflatten(-1, (-1, d)) for x, d in zip(row.split([H * dk, Hkv * dk, Hkv * dv], -1), (dk, dk, dv)))
    elif case["layout"] == "heads":
        q, k, v = (torch.empty(B, h, T, d, dtype=dtype, device="cuda").transpose(1, 2)
                   for h, d in ((H, dk), (Hkv, dk), (Hkv, dv)))
    else:
        q, k, v = (torch.empty(B, T, h, d, dtype=dtype, device="cuda") for h, d in ((H, dk), (Hkv, dk), (Hkv, dv)))
    q.copy_(unit(B, T, H, dk))
    k.copy_(unit(B, T, Hkv, dk))
    v.copy_(torch.randn(B, T, Hkv, dv, generator=gen, device="cuda"))
    return q, k, v


def _decays(case, gen, shape):
    if case["per_head"]:
        return 1 - torch.exp2(-3 - 6 * torch.rand(case["Hkv"], generator=gen, device="cuda"))
    return torch.sigmoid(torch.randn(*shape, generator=gen, device="cuda") + case["gate_mean"])


def _states(case, gen, n):
    """States as a prefix of normalised keys leaves them: elements of size 1 / sqrt(d_k) times a few."""
    return torch.randn(n, case["Hkv"], case["dv"], case["dk"], generator=gen, device="cuda") * (3 / math.sqrt(case["dk"]))


def prepare(case, seed):
    case = {**_DEFAULTS, **case}
    gen = _generator(seed)
    B, H, Hkv, dk, dv = (case[n] for n in ("B", "H", "Hkv", "dk", "dv"))
    dtype = _DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] in ("forward", "backward"):
        T = case["T"]
        st["q"], st["k"], st["v"] = _rows(case, gen)
        st["gate"] = _decays(case, gen, (B, T, Hkv))
        if case["packed"]:
            first = torch.rand(B, T, generator=gen, device="cuda") < 4 / T
            st["gate"][first] = 0.0
        st["S_init"] = _states(case, gen, B // case["F"]) if case["init"] else None
        if case["kind"] == "forward":
            st["out"] = torch.empty(B, T, H, dv, dtype=dtype, device="cuda")
        else:
            st["dy"] = torch.randn(B, T, H, dv, generator=gen, device="cuda").to(dtype)
            st["dS_final"] = _states(case, gen, B) if case["state"] else None
    elif case["kind"] == "decode":
        st["q"], st["k"], st["v"] = _rows(case, gen)
        st["gate"] = _decays(case, gen, (B, case["T"], Hkv))
        st["S"] = _states(case, gen, B // case["F"])
        # the states after the tokens have buffers of their own: the program may still go back to those before them
        st["S_out"] = torch.empty(B, Hkv, dv, dk, device="cuda")
        st["out"] = torch.empty(B, case["T"], H, dv, dtype=dtype, device="cuda")
    else:
        N = case["N"]
        st["S"] = _states(case, gen, B // case["F"])
        # the caches: the tokens behind the prefix, rows that no token has filled yet hold k = v = 0 and a decay of 1
        _, st["k_cache"], st["v_cache"] = _rows({**case, "T": N, "H": 1}, gen)
        lengths = torch.randint(0, N, (B,), generator=gen, device="cuda", dtype=torch.int32)
        if case["idle"]:
            lengths[torch.rand(B, generator=gen, device="cuda") < 0.1] = -1
        st["lengths"] = lengths
        free = torch.arange(N, device="cuda") >= lengths[:, None]
        st["k_cache"][free] = 0
        st["v_cache"][free] = 0
        if case["per_head"]:
            st["gate_cache"] = None
        else:
            st["gate_cache"] = _decays(case, gen, (B, N, Hkv))
            st["gate_cache"][free] = 1.0
        q, k, v = _rows({**case, "T": 1}, gen)
        st["q"], st["k"], st["v"] = q[:, 0], k[:, 0], v[:, 0]
        st["gate"] = _decays(case, gen, (B, Hkv))
        st["out"] = torch.zeros(B, H, dv, dtype=dtype, device="cuda")
    return st


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _log_decay(gate, B, T, Hkv):
    """log gamma [B, Hkv, T] in float64, with the library's floor at -100."""
    g = gate.double()
    g = g.expand(B, T, Hkv) if g.dim() == 1 else g
    return torch.log(g).clamp(min=-100.0).transpose(1, 2)


def _chunks(x, heads):
    """[B, T, h, d] -> float32 [B, heads, h / heads, chunks, C, d], zeros behind the last token."""
    B, T, h, d = x.shape
    x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, -T % _CHUNK))
    return x.reshape(B, -1, _CHUNK, heads, h // heads, d).permute(0, 3, 4, 1, 2, 5).contiguous()


def _rows_of(x, T):
    """The inverse of _chunks, without the padding."""
    B, heads, group, n, c, d = x.shape
    return x.permute(0, 3, 4, 1, 2, 5).reshape(B, n * c, heads * group, d)[:, :T]


def _chunk_decays(gate, B, T, Hkv):
    """Within chunks: zeta [B, Hkv, 1, n, C], M[t, s], weights zeta_C / zeta_s; E [B, Hkv, n]: log decay up to a chunk's end."""
    log = torch.nn.functional.pad(_log_decay(gate, B, T, Hkv), (0, -T % _CHUNK)).unflatten(-1, (-1, _CHUNK))
    G = log.cumsum(-1)
    M = torch.exp(G[..., :, None] - G[..., None, :]).tril().float().unsqueeze(2)
    return G.exp().float().unsqueeze(2), M, torch.exp(G[..., -1:] - G).float().unsqueeze(2), G[..., -1].cumsum(-1)


def _chunk_states(delta, E, S0):
    """States [B, Hkv, n + 1, a, b] before each chunk and after the last, from what each chunk adds (delta)."""
    B, Hkv, n, a, b = delta.shape
    before = torch.nn.functional.pad(E, (1, 0))                  # log decay before chunk 0, .., after the last
    decay = torch.exp((before[..., :, None] - E[..., None, :]).clamp(max=0.0)).tril(-1).float()
    S = torch.matmul(decay, delta.reshape(B, Hkv, n, a * b))
    if S0 is not None:
        S = S + before.exp().float()[..., None] * S0.reshape(B, Hkv, 1, a * b)
    return S.reshape(B, Hkv, n + 1, a, b)


def _shared_rows(S, B):
    return None if S is None else S.repeat_interleave(B // S.shape[0], 0)


def _plain_forward(q, k, v, gate, S0):
    B, T, H, _ = q.shape
    Hkv = k.shape[2]
    zeta, M, w, E = _chunk_decays(gate, B, T, Hkv)
    qc, kc, vc = _chunks(q, Hkv), _chunks(k, Hkv), _chunks(v, Hkv)
    delta = torch.matmul((vc * w[..., None]).transpose(-1, -2).contiguous(), kc)[:, :, 0]
    S = _chunk_states(delta, E, _shared_rows(S0, B))
    y = zeta[..., None] * torch.matmul(qc, S[:, :, None, :-1].transpose(-1, -2).contiguous())
    y = y + torch.matmul(torch.matmul(qc, kc.transpose(-1, -2).contiguous()) * M, vc)
    return _rows_of(y, T).to(q.dtype), S[:, :, -1].contiguous()


def _plain_backward(q, k, v, gate, dy, S0, dS_final):
    B, T, H, _ = q.shape
    Hkv = k.shape[2]
    zeta, M, w, E = _chunk_decays(gate, B, T, Hkv)
    qc, kc, vc, dyc = _chunks(q, Hkv), _chunks(k, Hkv), _chunks(v, Hkv), _chunks(dy, Hkv)
    turn = lambda x: x.transpose(-1, -2).contiguous()  # noqa: E731
    S = _chunk_states(torch.matmul(turn(vc * w[..., None]), kc)[:, :, 0], E, _shared_rows(S0, B))
    # the gradients' states: from the last chunk to the first
    back = torch.matmul(turn(dyc * zeta[..., None]), qc).sum(2)
    n = back.shape[2]
    total = E[..., -1:]
    E_back = total - torch.nn.functional.pad(E, (1, 0))[..., :-1].flip(-1)   # log decay from a chunk's start to the end
    R = _chunk_states(back.flip(2), E_back, dS_final).flip(2)                # after the last chunk: R[n], .. before chunk 0: R[0]
    R_end = R[:, :, None, 1:]
    dq = zeta[..., None] * torch.matmul(dyc, S[:, :, None, :-1]) + torch.matmul(torch.matmul(dyc, turn(vc)) * M, kc)
    Mt = turn(M)
    dv = w[..., None] * torch.matmul(kc, turn(R_end)) + (torch.matmul(turn(torch.matmul(qc, turn(kc))) * Mt, dyc)).sum(2, keepdim=True)
    dk = w[..., None] * torch.matmul(vc, R_end) + (torch.matmul(turn(torch.matmul(dyc, turn(vc))) * Mt, qc)).sum(2, keepdim=True)
    # d loss / d log gamma_t: what the tokens from t on read of the states before t
    per_token = (qc.double() * dq.double()).sum(-1).sum(2) - (kc.double() * dk.double()).sum(-1)[:, :, 0]
    dlog = per_token.flatten(-2)[..., :T].flip(-1).cumsum(-1).flip(-1)
    if dS_final is not None:
        dlog = dlog + (S[:, :, n].double() * dS_final.double()).sum((-1, -2))[..., None]
    if gate.dim() == 1:
        dgate = (dlog.sum((0, 2)) / gate.double()).float()
    else:
        dgate = (dlog.transpose(1, 2) / gate.double()).float()
    out = {"dq": _rows_of(dq, T).to(q.dtype), "dk": _rows_of(dk, T).to(q.dtype), "dv": _rows_of(dv, T).to(q.dtype), "dgate": dgate}
    if S0 is not None:
        out["dS_init"] = R[:, :, 0].unflatten(0, (S0.shape[0], -1)).sum(1)
    return out


def _plain_decode(q, k, v, gate, S0):
    """T tokens as one block."""
    B, T, H, _ = q.shape
    Hkv = k.shape[2]
    G = _log_decay(gate, B, T, Hkv).cumsum(-1)
    M = torch.exp(G[..., :, None] - G[..., None, :]).tril().float()[:, :, None]
    head = lambda x: x.float().unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1, 4).contiguous()  # noqa: E731
    qh, kh, vh = head(q), head(k), head(v)
    S = _shared_rows(S0, B)
    y = G.exp().float()[:, :, None, :, None] * torch.matmul(qh, S[:, :, None].transpose(-1, -2).contiguous())
    y = y + torch.matmul(torch.matmul(qh, kh.transpose(-1, -2).contiguous()) * M, vh)
    w = torch.exp(G[..., -1:] - G).float()[..., None]
    S1 = G[..., -1].exp().float()[..., None, None] * S + torch.matmul((vh[:, :, 0] * w).transpose(-1, -2).contiguous(), kh[:, :, 0])
    return y.permute(0, 3, 1, 2, 4).flatten(2, 3).to(q.dtype), S1


def _plain_shared(st):
    """The new token goes into the caches, then all of a sequence's suffix is read."""
    q, k, v, gate, lengths = st["q"], st["k"], st["v"], st["gate"], st["lengths"].long()
    B, H, dk = q.shape
    N, Hkv = st["k_cache"].shape[1:3]
    here = torch.arange(N, device=q.device)[None] == lengths[:, None]             # (no row of an idle sequence)
    st["k_cache"].copy_(torch.where(here[..., None, None], k[:, None], st["k_cache"]))
    st["v_cache"].copy_(torch.where(here[..., None, None], v[:, None], st["v_cache"]))
    if st["gate_cache"] is None:
        log = _log_decay(gate, B, N, Hkv)
    else:
        st["gate_cache"].copy_(torch.where(here[..., None], gate[:, None], st["gate_cache"]))
        log = _log_decay(st["gate_cache"], B, N, Hkv)
    log = torch.where(torch.arange(N, device=q.device) <= lengths[:, None, None], log, 0.0)
    G = log.cumsum(-1)
    weight = torch.exp(G[..., -1:] - G) * (torch.arange(N, device=q.device) <= lengths[:, None, None])
    qh = q.float().unflatten(1, (Hkv, -1))                                         # [B, Hkv, G, dk]
    kh, vh = (x.float().transpose(1, 2).contiguous() for x in (st["k_cache"], st["v_cache"]))
    S = _shared_rows(st["S"], B)
    y = G[..., -1].exp().float()[..., None, None] * torch.matmul(qh, S.transpose(-1, -2).contiguous())
    y = y + torch.matmul(torch.matmul(qh, kh.transpose(-1, -2).contiguous()) * weight.float()[:, :, None], vh)
    active = (lengths >= 0) & (lengths < N)
    st["out"].copy_(torch.where(active[:, None, None], y.flatten(1, 2).to(q.dtype), st["out"]))
    return st["out"]


def _caches(st):
    return {n: st[n] for n in ("k_cache", "v_cache", "gate_cache") if st[n] is not None}


def run(st):
    case = st["case"]
    if own:
        from paper_2511_21016_amd import binding
        if case["kind"] == "forward":
            if "workspace" not in st:              # a program keeps it for all calls of these sizes
                st["workspace"] = binding.linear_workspace(st["q"], st["k"], st["v"], st["gate"])
            return binding.gka_linear_forward(st["q"], st["k"], st["v"], st["gate"], S_init=st["S_init"],
                                              return_state=case["state"], workspace=st["workspace"], out=st["out"])
        if case["kind"] == "backward":
            if "workspace" not in st:
                st["workspace"] = binding.linear_workspace(st["q"], st["k"], st["v"], st["gate"], backward=True)
            return binding.gka_linear_backward(st["q"], st["k"], st["v"], st["gate"], st["dy"], S_init=st["S_init"],
                                               dS_final=st["dS_final"], workspace=st["workspace"])
        if case["kind"] == "decode":
            y = binding.gka_linear_decode(st["S"], st["q"], st["k"], st["v"], st["gate"], S_out=st["S_out"], out=st["out"])
            return y, st["S_out"]
        y = binding.gka_linear_decode_shared(st["S"], st["q"], st["k"], st["v"], st["gate"], st["k_cache"], st["v_cache"],
                                             st["gate_cache"], st["lengths"], out=st["out"])
        return {"y": y, **_caches(st)}
    if case["kind"] == "forward":
        y, S = _plain_forward(st["q"], st["k"], st["v"], st["gate"], st["S_init"])
        return (y, S) if case["state"] else y
    if case["kind"] == "backward":
        return _plain_backward(st["q"], st["k"], st["v"], st["gate"], st["dy"], st["S_init"], st["dS_final"])
    if case["kind"] == "decode":
        return _plain_decode(st["q"], st["k"], st["v"], st["gate"], st["S"])
    return {"y": _plain_shared(st), **_caches(st)}


def work(case):
    case = {**_DEFAULTS, **case}
    B, H, Hkv, dk, dv = (case[n] for n in ("B", "H", "Hkv", "dk", "dv"))
    size = 2 if case["dtype"] == "bf16" else 4
    state = 4 * Hkv * dk * dv                     # bytes of a sequence's states
    product = 2 * dk * dv                         # flops of a state's product with a vector, or of an update
    if case["kind"] == "shared":
        N = case["N"]
        used = B * (N + 1) / 2 * (0.9 if case["idle"] else 1.0)      # cached tokens, the new one among them, on average
        cache = Hkv * ((dk + dv) * size + (0 if case["per_head"] else 4))
        rows = B * size * (H * (dk + dv) + Hkv * (dk + dv))
        return {"bytes": int(B // case["F"] * state + used * cache + rows),
                "flops": int(B * H * product + used * H * 2 * (dk + dv))}
    T = case["T"]
    gates = 4 * Hkv * (1 if case["per_head"] else B * T)
    rows = B * T * size
    if case["kind"] == "decode":
        return {"bytes": rows * (H + Hkv) * (dk + dv) + gates + B // case["F"] * state + B * state,
                "flops": B * T * product * (H + Hkv)}
    init = B // case["F"] * state if case["init"] else 0
    if case["kind"] == "forward":
        return {"bytes": rows * (H + Hkv) * (dk + dv) + gates + init + (B * state if case["state"] else 0),
                "flops": B * T * product * (H + Hkv)}
    # q, k, v, dy in, dq, dk, dv out; readouts of S for dq, of dS for dk and dv, updates of both
    return {"bytes": rows * (H * (2 * dk + dv) + 2 * Hkv * (dk + dv)) + 2 * gates + 2 * init + (B * state if case["state"] else 0),
            "flops": B * T * product * (2 * H + 3 * Hkv)}


# ---- the definitions in 64 bits: the recurrences token by token ------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    case = st["case"]
    with torch.no_grad():
        if case["kind"] == "shared":
            return _exact_shared(st)
        B, T, H, Hkv = case["B"], case["T"], case["H"], case["Hkv"]
        q, k, v = (st[n].double().transpose(0, 1) for n in ("q", "k", "v"))           # [T, B, h, d]
        gate = st["gate"].double()
        gate = gate.expand(T, B, Hkv) if case["per_head"] else gate.transpose(0, 1)
        S = st["S"] if case["kind"] == "decode" else st["S_init"]
        if S is None:
            S = torch.zeros(B, Hkv, case["dv"], case["dk"], dtype=torch.float64, device="cuda")
        else:
            S = S.double().repeat_interleave(case["F"], 0)
        if case["kind"] == "backward":
            return _exact_backward(st, q, k, v, gate, S)
        y = torch.empty(T, B, Hkv, H // Hkv, case["dv"], dtype=torch.float64, device="cuda")
        for t in range(T):
            S = gate[t][..., None, None] * S + v[t][..., :, None] * k[t][..., None, :]
            y[t] = (S[:, :, None] * q[t].unflatten(1, (Hkv, -1))[..., None, :]).sum(-1)
        y = y.flatten(2, 3).transpose(0, 1)
        return (y, S) if case["kind"] == "decode" or case["state"] else y


def _exact_backward(st, q, k, v, gate, S):
    case = st["case"]
    T, Hkv, B = case["T"], case["Hkv"], case["B"]
    dy = st["dy"].double().transpose(0, 1)
    group = lambda x: x.unflatten(1, (Hkv, -1))  # noqa: E731  [B, Hkv, G, d]
    span = max(1, math.isqrt(T))
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dgate = torch.empty(T, B, Hkv, dtype=torch.float64, device="cuda")
    marks = []
    for t in range(T):                            # the state before every span-th token
        if t % span == 0:
            marks.append(S)
        S = gate[t][..., None, None] * S + v[t][..., :, None] * k[t][..., None, :]
    R = torch.zeros_like(S) if st["dS_final"] is None else st["dS_final"].double()
    for m in reversed(range(len(marks))):
        lo, hi = m * span, min(T, (m + 1) * span)
        before = [marks[m]]
        for t in range(lo, hi):
            before.append(gate[t][..., None, None] * before[-1] + v[t][..., :, None] * k[t][..., None, :])
        for t in reversed(range(lo, hi)):
            R = R + (group(dy[t])[..., :, None] * group(q[t])[..., None, :]).sum(2)
            dq[t] = (before[t + 1 - lo][:, :, None] * group(dy[t])[..., :, None]).sum(-2).flatten(1, 2)
            dv[t] = (R * k[t][..., None, :]).sum(-1)
            dk[t] = (R * v[t][..., :, None]).sum(-2)
            dgate[t] = (R * before[t - lo]).sum((-1, -2))
            R = gate[t][..., None, None] * R
    out = {"dq": dq.transpose(0, 1), "dk": dk.transpose(0, 1), "dv": dv.transpose(0, 1)}
    out["dgate"] = dgate.sum((0, 1)) if case["per_head"] else dgate.transpose(0, 1)
    if st["S_init"] is not None:
        out["dS_init"] = R.unflatten(0, (-1, case["F"])).sum(1)
    return out


def _exact_shared(st):
    case = st["case"]
    Hkv, N = case["Hkv"], case["N"]
    lengths = st["lengths"].long()
    S = st["S"].double().repeat_interleave(case["F"], 0)
    out = {"y": None, **_caches(st)}
    for name, new in (("k_cache", "k"), ("v_cache", "v"), ("gate_cache", "gate")):
        if name in out:
            cache = out[name].clone()
            for b, n in enumerate(lengths.tolist()):
                if 0 <= n < N:
                    cache[b, n] = st[new][b]
            out[name] = cache
    for j in range(N):
        there = (j <= lengths)[:, None, None, None]
        g = st["gate"] if case["per_head"] else out["gate_cache"][:, j]
        g = g.double().expand(case["B"], Hkv)[..., None, None]
        S1 = g * S + out["v_cache"][:, j].double()[..., :, None] * out["k_cache"][:, j].double()[..., None, :]
        S = torch.where(there, S1, S)
    y = (S[:, :, None] * st["q"].double().unflatten(1, (Hkv, -1))[..., None, :]).sum(-1).flatten(1, 2)
    active = (lengths >= 0) & (lengths < N)
    out["y"] = torch.where(active[:, None, None], y, st["out"].double())
    for name in _caches(st):
        out[name] = out[name].double()
    return out
