"""CPU-side checks of the linear-attention entry points: bad arguments are refused on the host before any launch, by the library
and by the binding; launch plans stay within grids, LDS and workspaces."""
import pytest
import torch

from hip_recorder import record
from paper_2511_21016_amd import binding

X = 0x10000000


def _p(**kw):
    base = dict(B=4, H=4, H_kv=2, T=100, d_k=64, d_v=64, io_dtype=binding.GKA_BF16, cache_tokens=8)
    base.update(kw)
    return binding.make_linear_params(**base)


def _forward(p, **kw):
    a = dict(q=X, k=X, v=X, gate=X, o=X, S_init=None, S_final=None, workspace=X, workspace_bytes=1 << 40)
    a.update(kw)
    return binding.linear_forward_raw(p, *(a[n] for n in ("q", "k", "v", "gate", "o", "S_init", "S_final", "workspace", "workspace_bytes")))


def _backward(p, **kw):
    a = dict(q=X, k=X, v=X, gate=X, dy=X, dq=X, dk=X, dv=X, dgate=X, S_init=None, dS_final=None, dS_init=None, workspace=X,
             workspace_bytes=1 << 40)
    a.update(kw)
    return binding.linear_backward_raw(p, *a.values())


def _decode(p, **kw):
    a = dict(S_in=X, S_out=X, q=X, k=X, v=X, gate=X, o=X)
    a.update(kw)
    return binding.linear_decode_raw(p, *a.values())


def _shared(p, **kw):
    a = dict(S=X, q=X, k=X, v=X, gate=X, k_cache=X, v_cache=X, gate_cache=X, lengths=X, o=X)
    a.update(kw)
    return binding.linear_decode_shared_raw(p, *a.values())


CALLS = (_forward, _backward, _decode, _shared)

SHAPE = [dict(B=0), dict(B=-1), dict(H=0), dict(H_kv=0), dict(H=3), dict(H_kv=8), dict(d_k=0), dict(d_v=-16), dict(share=3),
         dict(share=-1), dict(share=8), dict(walk_chunks=-1), dict(B=1 << 24, H=4), dict(q_stride=(64, 0, 64)),
         dict(k_stride=(64, -64, 64)), dict(v_stride=(6400, 100, 64)), dict(o_stride=(25600, 256, 60)), dict(q_stride=(25600, 256, 32))]
UNSUPPORTED = [dict(d_k=8), dict(d_k=65), dict(d_v=24), dict(d_k=272), dict(d_v=512), dict(io_dtype=2), dict(io_dtype=-1),
               dict(gate_per_head=2), dict(gate_per_head=-1)]


@pytest.mark.parametrize("call", CALLS)
def test_parameters_are_refused(call):
    for bad in SHAPE:
        assert call(_p(**bad)) == binding.GKA_ERR_SHAPE, bad
    for bad in UNSUPPORTED:
        assert call(_p(**bad)) == binding.GKA_ERR_UNSUPPORTED, bad
    assert call(None) == binding.GKA_ERR_NULL
    if call is _shared:
        assert call(_p(cache_tokens=0)) == binding.GKA_ERR_SHAPE
    else:
        assert call(_p(T=0)) == binding.GKA_ERR_SHAPE


def test_queries_of_bad_parameters_are_zero():
    for bad in SHAPE + UNSUPPORTED + [dict(T=0), dict(T=-5)]:
        assert binding.linear_forward_workspace_bytes(_p(**bad)) == 0, bad
        assert binding.linear_backward_workspace_bytes(_p(**bad)) == 0, bad
    assert binding.linear_forward_workspace_bytes(None) == 0


def test_pointers_and_workspaces_are_refused():
    for call, needed in ((_forward, ("q", "k", "v", "gate", "o")), (_backward, ("q", "k", "v", "gate", "dy", "dq", "dk", "dv", "dgate")),
                         (_decode, ("S_in", "S_out", "q", "k", "v", "gate", "o")),
                         (_shared, ("S", "q", "k", "v", "gate", "k_cache", "v_cache", "gate_cache", "lengths", "o"))):
        for n in needed:
            assert call(_p(), **{n: None}) == binding.GKA_ERR_NULL, (call, n)
            if n not in ("gate", "dgate", "gate_cache", "lengths"):
                assert call(_p(), **{n: X + 8}) == binding.GKA_ERR_SHAPE, (call, n)
    assert _forward(_p(), S_init=X + 4) == _forward(_p(), S_final=X + 4) == binding.GKA_ERR_SHAPE
    assert _forward(_p(share=2), S_init=X, S_final=X) == _decode(_p(share=2)) == binding.GKA_ERR_SHAPE
    for call, query in ((_forward, binding.linear_forward_workspace_bytes), (_backward, binding.linear_backward_workspace_bytes)):
        p = _p(T=1000, walk_chunks=2)
        need = query(p)
        assert need > 0 and need % 256 == 0
        for ws in (dict(workspace=None), dict(workspace=X + 128), dict(workspace_bytes=need - 1)):
            assert call(p, **ws) == binding.GKA_ERR_WORKSPACE, (call, ws)


def test_library_host_code_under_asan_ubsan():
    from paper_2511_21016_amd import build
    import test_sanitizers
    lib = build.build_host_sanitized()
    test_sanitizers.run_pytest_under(build.sanitizer_runtime(), ["tests/test_linear_abi.py::test_parameters_are_refused",
                                                                 "tests/test_linear_abi.py::test_queries_of_bad_parameters_are_zero",
                                                                 "tests/test_linear_abi.py::test_pointers_and_workspaces_are_refused"],
                                     {"GKA_LIBRARY": lib})


# ---- the binding's own checks (nothing can be launched: the library's entry points are replaced)


@pytest.fixture
def no_launch(monkeypatch):
    binding.load_library()
    calls = []
    for name in ("linear_forward_raw", "linear_backward_raw", "linear_decode_raw", "linear_decode_shared_raw"):
        monkeypatch.setattr(binding, name, lambda *a, _name=name, **kw: calls.append(_name) or binding.GKA_OK)
    return calls


def _tensors(device="cpu", B=2, T=3, H=4, H_kv=2, d_k=64, d_v=32, dtype=torch.bfloat16):
    rows = lambda h, d: torch.zeros(B, T, h, d, dtype=dtype, device=device)
    return rows(H, d_k), rows(H_kv, d_k), rows(H_kv, d_v), torch.ones(B, T, H_kv, device=device)


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_tensors_off_the_gpu_are_refused(no_launch, device):
    q, k, v, gate = _tensors(device)
    S = torch.zeros(2, 2, 32, 64, device=device)
    one = lambda x: x[:, 0]
    for call in (lambda: binding.gka_linear_forward(q, k, v, gate), lambda: binding.gka_linear_backward(q, k, v, gate, q),
                 lambda: binding.gka_linear_decode(S, q, k, v, gate), lambda: binding.linear_workspace(q, k, v, gate),
                 lambda: binding.gka_linear_decode_shared(S, one(q), one(k), one(v), one(gate), k, v, gate,
                                                          torch.zeros(2, dtype=torch.int32, device=device))):
        with pytest.raises(ValueError):
            call()
    assert no_launch == []


@pytest.fixture
def pretend_gpu(monkeypatch, no_launch):
    """CPU tensors pass for ones on device 0."""
    monkeypatch.setattr(binding, "_stream_of", lambda t: 0)

    monkeypatch.setattr(binding, "_on_device", lambda index, call, *args: call(*args))
    return no_launch


def test_shapes_types_and_strides_are_refused(pretend_gpu):
    q, k, v, gate = _tensors()
    S = torch.zeros(2, 2, 32, 64)
    o = torch.zeros(2, 3, 4, 32, dtype=torch.bfloat16)
    forward = lambda q=q, k=k, v=v, gate=gate, **kw: binding.gka_linear_forward(q, k, v, gate, **kw)
    assert forward(S_init=S, out=o) is o and pretend_gpu == ["linear_forward_raw"]
    pretend_gpu.clear()
    cases = [dict(k=k[:, :2]), dict(k=k[..., :32]), dict(v=v[:1]), dict(v=v[:, :, :1]), dict(gate=gate[..., :1]), dict(gate=gate[0, 0, :1]),
             dict(gate=gate.bfloat16()), dict(gate=gate.transpose(0, 1)), dict(q=q[0]), dict(q=q.transpose(-1, -2)),
             dict(out=o[..., :16]), dict(out=o.float()), dict(S_init=S[0]), dict(S_init=S.transpose(-1, -2)), dict(S_init=S.bfloat16()),
             dict(S_init=torch.zeros(3, 2, 32, 64)), dict(S_final=S[:1]), dict(S_init=S.repeat(1, 1, 2, 1)[:, :, ::2])]
    for bad in cases:
        with pytest.raises((ValueError, TypeError)):
            forward(**bad)
    with pytest.raises(TypeError):
        forward(q=q.half(), k=k.half(), v=v.half())
    with pytest.raises(TypeError):
        forward(k=k.float())
    for bad in (o[:, :2], o.float(), v):
        with pytest.raises((ValueError, TypeError)):
            binding.gka_linear_backward(q, k, v, gate, bad)
    with pytest.raises(ValueError):
        binding.gka_linear_backward(q, k, v, gate, o, dS_final=S[:1])
    with pytest.raises(ValueError):
        binding.gka_linear_decode(S[:1], q, k, v, gate)            # shared states cannot be updated in place
    with pytest.raises(ValueError):
        binding.gka_linear_decode(S, q[:, 0], k, v, gate)
    kc, vc, gc, n = torch.zeros(2, 8, 2, 64, dtype=q.dtype), torch.zeros(2, 8, 2, 32, dtype=q.dtype), torch.ones(2, 8, 2), torch.zeros(2, dtype=torch.int32)
    shared = lambda gate=gate[:, 0].contiguous(), kc=kc, vc=vc, gc=gc, n=n: binding.gka_linear_decode_shared(
        S[:1], q[:, 0], k[:, 0], v[:, 0], gate, kc, vc, gc, n)
    shared()
    assert pretend_gpu == ["linear_decode_shared_raw"]
    for bad in (dict(kc=kc[:1]), dict(kc=kc[0]), dict(vc=vc[:, :4]), dict(vc=kc), dict(kc=kc.float()), dict(gc=None), dict(gc=gc[..., :1]),
                dict(gate=torch.ones(2)), dict(n=n.long()), dict(n=n[:1]), dict(kc=kc.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises((ValueError, TypeError)):
            shared(**bad)
    assert pretend_gpu == ["linear_decode_shared_raw"]


def test_strides_that_the_binding_hands_over():
    rows = binding._row_strides
    x = torch.zeros(2, 3, 4, 64)
    assert rows(x, "x") == (0, 0, 0)
    assert rows(x.transpose(1, 2).contiguous().transpose(1, 2), "x") == (3 * 4 * 64, 64, 3 * 64)
    assert rows(torch.zeros(2, 3, 6, 80)[:, :, 1:5, 16:], "x") == (3 * 6 * 80, 6 * 80, 80)
    # dimensions of size 1 get the strides of packed rows, whatever torch says
    assert rows(torch.zeros(1, 3, 1, 80)[..., :64].as_strided((1, 3, 1, 64), (7, 80, 3, 1)), "x") == (3 * 80, 80, 64)
    # (one token: its stride is not used)
    assert rows(torch.zeros(5, 2, 4, 64)[:, 0], "x")[::2] == (2 * 4 * 64, 64)
    with pytest.raises(ValueError):
        rows(x.transpose(-1, -2), "x")


# ---- launch plans, with a recorder in the HIP runtime's place


SIZES = [(1, 1, 1, 1, 16, 16), (1, 8, 8, 77, 128, 128), (4, 16, 16, 4096, 128, 128), (1, 32, 8, 32768, 128, 128), (2, 6, 2, 1000, 256, 80),
         (3, 4, 1, 500, 48, 256), (64, 32, 32, 200, 64, 64)]


@pytest.mark.parametrize("dtype", ["GKA_BF16", "GKA_F32"])
def test_grids_and_limits(dtype):
    calls = record(f"""
X = 0x10000000
for device in (0, 1):
    set_device(device)
    for B, H, H_kv, T, d_k, d_v in {SIZES}:
        for walk in (0, 1, 7):
            p = binding.make_linear_params(B, H, H_kv, T, d_k, d_v, binding.{dtype}, cache_tokens=64, walk_chunks=walk)
            ws = dict(workspace=X, workspace_bytes=binding.linear_forward_workspace_bytes(p))
            assert binding.linear_forward_raw(p, X, X, X, X, X, X, X, **ws) == 0
            ws["workspace_bytes"] = binding.linear_backward_workspace_bytes(p)
            assert binding.linear_backward_raw(p, X, X, X, X, X, X, X, X, X, X, X, 2 * X, **ws) == 0
            assert binding.linear_decode_raw(p, X, X, X, X, X, X, X) == 0
            assert binding.linear_decode_shared_raw(p, X, X, X, X, X, X, X, X, X, X) == 0
""")
    raised, launches = {}, [c for c in calls if c["kind"] == "launch"]
    half = len(launches) // 2
    seen = 0
    for c in calls:
        if c["kind"] == "attribute":
            raised[c["mangled"], c["device"]] = c["value"]
        elif c["kind"] == "launch":
            device, seen = int(seen >= half), seen + 1
            assert 0 < c["grid"] <= 0x7fffffff and c["block"] <= 1024 and c["lds"] <= 160 << 10
            if c["lds"] > 64 << 10:
                assert raised.get((c["mangled"], device), 0) >= c["lds"], (c["kernel"], device)
    for name in ("linear_walk_kernel", "linear_scan_kernel", "linear_gate_kernel", "linear_decode_kernel", "linear_shared_kernel"):
        assert any(name in c["mangled"] for c in launches), name


def test_sizes_beyond_the_limits_are_refused():
    longest = 0x7fffe000
    for call in CALLS:
        size = "cache_tokens" if call is _shared else "T"
        for bad in (dict(B=1 << 20), dict(B=1 << 20, H=128, H_kv=1), {size: longest + 1}, {size: 0x7fffffff}):
            assert call(_p(**bad)) == binding.GKA_ERR_SHAPE, (call, bad)
        p = _p()
        p.reserved = 1
        assert call(p) == binding.GKA_ERR_UNSUPPORTED
    for states in (dict(S_init=2 * X, dS_init=2 * X), dict(dS_final=2 * X, dS_init=2 * X)):
        assert _backward(_p(), **states) == binding.GKA_ERR_SHAPE


HUGE = [((1 << 21) - 1, 1, 1, 1, 16, 16), (1 << 20, 1, 1, 1, 256, 256), (1 << 20, 1, 1, 5000, 16, 256), (1 << 16, 64, 16, 1, 32, 16),
        (1, 1, 1, 0x7fffe000, 16, 16), (2, 1, 1, 0x7fffe000, 256, 256), (1 << 15, 1, 1, 100000, 64, 64)]


def test_launches_of_huge_sizes_fit_the_grid():
    calls = record(f"""
X = 0x10000000
for B, H, H_kv, T, d_k, d_v in {HUGE}:
    for walk in (0, 1):
        p = binding.make_linear_params(B, H, H_kv, T, d_k, d_v, binding.GKA_BF16, cache_tokens=64, walk_chunks=walk)
        ws = dict(workspace=X, workspace_bytes=1 << 60)
        allowed = (binding.GKA_OK, binding.GKA_ERR_SHAPE)
        assert binding.linear_forward_raw(p, X, X, X, X, X, X, X, **ws) in allowed
        assert binding.linear_backward_raw(p, X, X, X, X, X, X, X, X, X, X, X, 2 * X, **ws) in allowed
        assert binding.linear_decode_raw(p, X, X, X, X, X, X, X) == 0
        assert binding.linear_decode_shared_raw(p, X, X, X, X, X, X, X, X, X, X) == 0
""")
    launches = [c for c in calls if c["kind"] == "launch"]
    assert launches
    for c in launches:
        assert 0 < c["grid"] and c["grid"] * c["block"] < 1 << 32, c


def test_states_in_place_go_through_the_scan():
    """With several segments the last one may end before another has started: the old states are then read by the scan alone."""
    source = """
X = 0x10000000
p = binding.make_linear_params(2, 2, 2, 200, 64, 64, binding.GKA_BF16, walk_chunks=1)
assert binding.linear_forward_raw(p, X, X, X, X, X, 2 * X, {final}, workspace=X, workspace_bytes=1 << 40) == 0
"""
    scans = lambda final: sum("linear_scan_kernel" in c["mangled"] for c in record(source.format(final=final)) if c["kind"] == "launch")
    assert scans("2 * X") == 1 and scans("3 * X") == 0
