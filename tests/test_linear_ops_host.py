"""The linear layer's operators and dropout without a GPU: the oracle's own pins (published numbers, differences), and every refusal of the C ABI and
of the binding, which come before anything is launched."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import linear_ops as lo

FAKE, NULL = 0x1000, 0          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def sol():
    from paper_2003_10688_amd import sol as s

    if not os.path.exists(s.LIB_PATH):
        from paper_2003_10688_amd import build

        build.build(verbose=False)
    s.lib()
    return s


def test_philox_known_answers():
    """The generator's published test vectors (10 rounds)."""
    got = lo.philox4x32(np.array([[0, 0, 0, 0]]), (0, 0))[0]
    assert [int(v) for v in got] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    got = lo.philox4x32(np.array([[f, f, f, f]]), (f, f))[0]
    assert [int(v) for v in got] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    got = lo.philox4x32(np.array([[0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344]]), (0xA4093822, 0x299F31D0))[0]
    assert [int(v) for v in got] == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_kept_share_and_independence(p):
    """Shares of 2^20 elements within five standard deviations; other calls, steps and seeds give other masks."""
    a = lo.dropout_kept(1024, 1024, p, 7)
    sd = np.sqrt(p * (1 - p) / a.size)
    assert abs(a.mean() - (1 - p)) <= 5 * sd + 2.0**-17
    for other in (lo.dropout_kept(1024, 1024, p, 7, call=1), lo.dropout_kept(1024, 1024, p, 7, step=1), lo.dropout_kept(1024, 1024, p, 7 + (1 << 32))):
        same = (a == other).mean()                       # of two independent masks: p^2 + (1 - p)^2
        q = p * p + (1 - p) ** 2
        assert abs(same - q) <= 5 * np.sqrt(q * (1 - q) / a.size) + 2.0**-16


@pytest.mark.parametrize("name", lo.ACTS)
def test_slopes_are_differences(name):
    z = np.linspace(-6, 6, 241) + 0.0125                 # not at ReLU's corner
    h = 1e-5
    assert np.allclose(lo.slope(name, z), (lo.act(name, z + h) - lo.act(name, z - h)) / (2 * h), atol=1e-9)


@pytest.mark.parametrize("name", lo.ACTS)
def test_oracle_gradients_are_differences(name):
    rng = np.random.default_rng(3)
    x, w, b, r, g = rng.standard_normal((5, 7)), rng.standard_normal((11, 7)), rng.standard_normal(11), rng.standard_normal((5, 11)), rng.standard_normal((5, 11))
    drop = (0.3, 1234567890123, 5, 2)
    loss = lambda x_, w_, b_: float((lo.linear_fused(x_, w_, b_, name, drop, r)[0] * g).sum())  # noqa: E731
    z = lo.linear_fused(x, w, b, name, drop, r)[1]
    for t, grad, at in ((x, 0, 0), (w, 1, 1), (b, 2, 2)):
        want = lo.linear_fused_bwd(g, x, w, z, name, drop)[grad]
        for idx in list(np.ndindex(t.shape))[::5]:
            h = 1e-6
            up, down = t.copy(), t.copy()
            up[idx] += h
            down[idx] -= h
            args = lambda v: [v if i == at else a for i, a in enumerate((x, w, b))]  # noqa: E731
            assert abs((loss(*args(up)) - loss(*args(down))) / (2 * h) - want[idx]) <= 1e-6


def desc(sol, m=4, i=16, o=8, dtype=0, act=0, ldx=0, ldy=0, ldr=0):
    return sol.LinearDesc(m, i, o, dtype, act, ldx, ldy, ldr)


def forward(sol, ld, x=FAKE, w=FAKE, bias=NULL, drop=None, res=NULL, y=FAKE + 0x1000, pre=NULL, ws=NULL, nbytes=0):
    return sol.lib().sol_linear_fused(ld, x, w if w != FAKE else 0x9000, bias, drop, res, y, pre, ws, nbytes, NULL)


def backward(sol, ld, dy=FAKE, x=0x3000, w=0x9000, pre=0x5000, drop=None, dx=0x6000, dw=0x7000, dw_dt=0, db=0x8000, ws=0xA000, nbytes=1 << 40):
    return sol.lib().sol_linear_backward(ld, dy, x, w, pre, drop, dx, dw, dw_dt, db, ws, nbytes, NULL)


def test_forward_refusals(sol):
    L = sol.lib()
    assert forward(sol, None) == 1 and b"descriptor" in L.sol_last_error()
    assert forward(sol, desc(sol), x=NULL) == 1 and forward(sol, desc(sol), y=NULL) == 1
    assert L.sol_linear_fused(desc(sol), FAKE, NULL, NULL, None, NULL, 0x2000, NULL, NULL, 0, NULL) == 1
    for bad in (dict(m=-1), dict(i=0), dict(o=0), dict(act=5), dict(act=-1), dict(ldx=15), dict(ldy=7), dict(ldr=7), dict(ldx=-16)):
        assert forward(sol, desc(sol, **bad)) == 2, bad
    assert forward(sol, desc(sol, dtype=2)) == 3
    for bad in (dict(i=(1 << 20) + 1), dict(o=(1 << 20) + 1), dict(i=1 << 16, o=1 << 16), dict(ldx=(1 << 21) + 1), dict(m=1 << 20, ldx=1 << 11), dict(m=1 << 28)):
        assert forward(sol, desc(sol, **bad)) == 6, bad
    for bad in (dict(x=FAKE + 4), dict(w=0x9008), dict(bias=FAKE + 4), dict(res=FAKE + 2), dict(y=FAKE + 8), dict(pre=FAKE + 1)):
        assert forward(sol, desc(sol), **bad) == 4, bad
    assert forward(sol, desc(sol), y=FAKE) == 6                              # y on x
    assert forward(sol, desc(sol), pre=FAKE + 0x1000) == 6                   # z on y
    assert forward(sol, desc(sol, ldr=16), res=FAKE + 0x1000) == 6           # y on the residual, another pitch
    odd = desc(sol, i=17)
    need = L.sol_linear_fused_workspace_bytes(odd)
    assert need >= 4 * 17 * 4
    assert forward(sol, odd) == 5 and forward(sol, odd, ws=0xB000, nbytes=need - 1) == 5
    assert forward(sol, odd, ws=NULL, nbytes=need) == 1 and forward(sol, odd, ws=0xB004, nbytes=need) == 4
    assert L.sol_linear_fused_workspace_bytes(desc(sol)) == 0 and L.sol_linear_fused_workspace_bytes(desc(sol, m=-1)) == 0
    assert forward(sol, desc(sol, m=0), x=NULL, y=NULL) == 0                 # nothing to do


def test_backward_refusals(sol):
    L = sol.lib()
    assert backward(sol, None) == 1 and backward(sol, desc(sol), dy=NULL) == 1
    assert backward(sol, desc(sol), x=NULL) == 1 and backward(sol, desc(sol), w=NULL) == 1
    assert backward(sol, desc(sol, act=2), pre=NULL) == 1
    assert backward(sol, desc(sol), dw_dt=1) == 3                            # a bf16 gradient of fp32 weights
    assert backward(sol, desc(sol, act=9)) == 2 and backward(sol, desc(sol, ldy=3)) == 2
    for bad in (dict(dy=FAKE + 4), dict(x=0x3002), dict(w=0x9004), dict(pre=0x5004), dict(dx=0x6008), dict(dw=0x7004), dict(db=0x8004), dict(ws=0xA008)):
        assert backward(sol, desc(sol), **bad) == 4, bad
    for bad in (dict(dx=FAKE), dict(dw=0x9000), dict(dx=0x5000), dict(dx=0x3000), dict(dw=0x6000), dict(db=0x7000)):
        assert backward(sol, desc(sol), **bad) == 6, bad
    need = L.sol_linear_backward_workspace_bytes(desc(sol, act=2))
    assert need >= 4 * 8 * 4 and backward(sol, desc(sol, act=2), nbytes=need - 1) == 5
    assert backward(sol, desc(sol, act=2), ws=NULL, nbytes=need) == 1


def test_dropout_refusals(sol):
    L = sol.lib()
    ok = sol.Dropout(0.5, 1)
    call = lambda rows=4, cols=8, dt=0, x=FAKE, d=ok, res=NULL, y=FAKE: L.sol_dropout(rows, cols, dt, x, d, res, y, NULL)  # noqa: E731
    assert call(rows=-1) == 2 and call(cols=0) == 2 and call(dt=3) == 3 and call(rows=1 << 20, cols=1 << 12) == 6
    assert call(d=None) == 1 and call(x=NULL) == 1 and call(y=NULL) == 1
    assert call(x=FAKE + 4) == 4 and call(res=FAKE + 2) == 4 and call(y=FAKE + 8) == 4
    for p in (-0.1, 1.5, float("nan"), float("inf")):
        assert call(d=sol.Dropout(p, 1)) == 2, p
        assert forward(sol, desc(sol), drop=sol.Dropout(p, 1)) == 2 and backward(sol, desc(sol), drop=sol.Dropout(p, 1)) == 2
    bad = sol.Dropout(0.5, 1)
    bad.step = 0x1002
    assert call(d=bad) == 4
    assert call(rows=0, x=NULL, y=NULL) == 0


def test_other_calls_refuse_the_new_activations(sol):
    xd, cd = sol.TensorDesc(1, 8, 8, 16, sol.F32), sol.ConvDesc(8, 16, 3, 3, 1, 1, 1, 1)
    for act in (sol.ACT_GELU, sol.ACT_GELU_TANH, sol.ACT_SILU):
        assert sol.lib().sol_conv2d_fused(xd, FAKE, cd, FAKE, NULL, NULL, NULL, act, None, FAKE, NULL, NULL, NULL) == 2
        assert sol.lib().sol_linear(4, 16, 8, 0, C.c_void_p(FAKE), C.c_void_p(FAKE), C.c_void_p(0), act, C.c_void_p(FAKE), C.c_void_p(0)) == 2


@pytest.mark.parametrize("kind", ["conv", "dw", "linear"])
def test_networks_refuse_the_new_activations(sol, kind):
    layer = {"kind": "linear", "out": 5} if kind == "linear" else {"kind": "conv", "cout": 8, "kh": 1, "kw": 1, "sh": 1, "sw": 1, "ph": 0, "pw": 0, "bn": False, "dw": kind == "dw"}
    for act, want in ((sol.ACT_NONE, 0), (sol.ACT_RELU, 0), (sol.ACT_GELU, 6), (sol.ACT_GELU_TANH, 6), (sol.ACT_SILU, 6), (-1, 6)):      # 6: SOL_ERR_UNSUPPORTED
        arr = sol.make_layer_array([layer])
        arr[0].act = act
        h = C.c_void_p(0)
        st = sol.lib().sol_network_create(arr, 1, C.byref(sol.TensorDesc(2, 1, 1, 8, sol.BF16)), 0, C.byref(h))
        assert st == want, (act, sol.lib().sol_last_error())
        if st == 0:
            sol.lib().sol_network_destroy(h)


def test_binding_refuses_what_is_not_on_the_gpu(sol):
    import torch

    x, w = torch.zeros(4, 32), torch.zeros(8, 32)
    with pytest.raises(ValueError):
        sol.sol_linear_fused(x, w, 8)
    with pytest.raises(ValueError):
        sol.sol_linear_backward(torch.zeros(4, 8), x, w)
    with pytest.raises(ValueError):
        sol.sol_dropout(x, sol.Dropout(0.5, 1))
    with pytest.raises(ValueError):
        sol.Dropout(0.5, 1, step=torch.zeros(1, dtype=torch.int32))


def test_scratch_and_results_come_from_the_stream_that_the_call_runs_on(sol, monkeypatch):
    """Memory from the current stream could be handed out there again while the kernels on another stream still use it."""
    import contextlib

    import torch

    log, side = [], object()

    class Operand(torch.Tensor):
        def new_empty(self, *a, **k):
            log.append("alloc")
            return torch.empty(4)

        def record_stream(self, s):
            log.append(s)

    @contextlib.contextmanager
    def stream(s):
        assert s is side
        log.append("enter")
        yield
        log.append("leave")

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: "current")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: log.append(s))
    x = torch.zeros(4).as_subclass(Operand)
    sol._scratch(None, 4, x, side)
    assert log == ["enter", "alloc", "leave"]                  # freed behind the call, for that stream alone
    log.clear()
    sol._result(x, (4,), torch.float32, side)
    assert log == ["enter", "alloc", "leave", "current"]       # freed by the caller, behind the uses on its stream
    log.clear()
    sol._scratch(None, 4, x, None), sol._result(x, (4,), torch.float32, None)
    assert log == ["alloc", "alloc"]


@pytest.mark.parametrize("dtype,i,per_row", [(1, 1, 8), (1, 2, 8), (1, 3, 8), (0, 1, 4)])
def test_rows_whose_copy_passes_32_bits(sol, dtype, i, per_row):
    """x of few features has fewer than 2^31 elements where its copy to aligned rows has more groups of eight than 32 bits count, with a step of the grid beyond the last."""
    L = sol.lib()
    most = ((1 << 32) - (1 << 21)) // per_row
    for m, want in ((1 << 24, 5), (most, 5), (most + 1, 6), (1 << 29, 5 if per_row == 4 else 6), ((1 << 31) // i - 1, 6)):       # 5: the workspace is too small, 6: refused
        ld = desc(sol, m=m, i=i, o=1, dtype=dtype)
        assert forward(sol, ld, ws=0xB000, nbytes=1) == want and backward(sol, ld, nbytes=1) == want, m
        bytes_ = (L.sol_linear_fused_workspace_bytes(ld), L.sol_linear_backward_workspace_bytes(ld))
        assert bytes_[0] == (m * per_row * 8 * (2 if dtype else 4) if want == 5 else 0) and (bytes_[1] > bytes_[0] or want == 6), m
    ld = desc(sol, m=(1 << 28) - 1, i=8, o=1, dtype=dtype)                  # rows that are not copied
    assert L.sol_linear_fused_workspace_bytes(ld) == 0 and backward(sol, ld, nbytes=1) == 5


def test_a_stream_of_another_device_is_refused(sol, monkeypatch):
    """Kernels on the current device's tensors cannot be launched on it."""
    import torch
    from types import SimpleNamespace

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 500 + device, raising=False)
    x = SimpleNamespace(get_device=lambda: 1, device="cuda:1")
    mine, current, other = (SimpleNamespace(device_index=d, cuda_stream=h) for d, h in ((1, 77), (1, 501), (0, 78)))
    assert sol._on_current(x, None, None) == (501, None) and sol._on_current(x, None, current) == (501, None) and sol._on_current(x, None, mine) == (77, mine)
    with pytest.raises(ValueError, match="stream of cuda:0"):
        sol._on_current(x, None, other)


def test_sizes_that_a_c_int_does_not_hold_are_refused(sol):
    """2^32 + 8 rows are not 8 rows."""
    import torch

    for shape, stride in (((2**32 + 8, 1), (1, 1)), ((2**31, 1), (1, 1)), ((8, 16), (2**32 + 64, 1)), ((1, 2**32 + 64), (1, 1))):
        t = torch.empty_strided(shape, stride, device="meta")
        with pytest.raises(sol.SolError) as e:
            sol._rows(t, shape[1], "x", t)
        assert e.value.status == 6
    t = torch.empty_strided((1, 16), (2**32 + 64, 1), device="meta")      # the pitch of a single row does not matter
    assert sol._rows(t, 16, "x", t)[1] == 16
