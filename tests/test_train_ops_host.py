"""Layer norm, embedding and gradient clipping without a GPU: the oracle's gradients against differences, and the refusals of the C entry points and of the binding."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import train_ops as to

NULL, FAKE = 0, 0x1000          # FAKE is never dereferenced: validation fails first


@pytest.fixture(scope="module")
def sol():
    from paper_2003_10688_amd import sol as s

    if not os.path.exists(s.LIB_PATH):
        from paper_2003_10688_amd import build

        build.build(verbose=False)
    s.lib()
    return s


def test_oracle_gradients_are_differences():
    rng = np.random.default_rng(3)
    x, gamma, beta, g, res = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    loss = lambda x_, gm, bt: float((to.layer_norm(x_, gm, bt)[0] * g).sum() + (x_ * res).sum())  # noqa: E731
    _, mean, rstd = to.layer_norm(x, gamma, beta)
    grads = to.layer_norm_bwd(g, x, mean, rstd, gamma, res)
    for at, t in enumerate((x, gamma, beta)):
        for idx in np.ndindex(t.shape):
            up, down = t.copy(), t.copy()
            up[idx] += 1e-6
            down[idx] -= 1e-6
            args = lambda v: [v if i == at else a for i, a in enumerate((x, gamma, beta))]  # noqa: E731
            assert abs((loss(*args(up)) - loss(*args(down))) / 2e-6 - grads[at][idx]) <= 1e-6
    tokens, table = np.array([2, 0, -1, 2, 9, 3]), rng.standard_normal((4, 5))
    g = rng.standard_normal((6, 5))
    g[[2, 4]] = 0                                              # padding, and a token outside the table: rows that do not depend on it
    loss = lambda t: float((np.nan_to_num(to.embedding(tokens, t, 1.5)) * g).sum())  # noqa: E731
    want = to.embedding_bwd(g, tokens, 4, 1.5)
    for idx in np.ndindex(table.shape):
        up, down = table.copy(), table.copy()
        up[idx] += 1e-6
        down[idx] -= 1e-6
        assert abs((loss(up) - loss(down)) / 2e-6 - want[idx]) <= 1e-6


def norm_desc(sol, rows=4, cols=16, dtype=0, ldx=0, ldy=0, eps=1e-5):
    return sol.LayerNormDesc(rows, cols, dtype, ldx, ldy, eps)


def norm(sol, nd, x=FAKE, gamma=0x2000, beta=0x3000, y=0x4000, mean=0x5000, rstd=0x6000):
    return sol.lib().sol_layer_norm(nd, x, gamma, beta, y, mean, rstd, NULL)


def norm_backward(sol, nd, dy=FAKE, x=0x2000, gamma=0x3000, mean=0x4000, rstd=0x5000, res=0x6000, dx=0x7000, dgamma=0x8000, dbeta=0x9000, ws=0xA000, nbytes=1 << 40):
    return sol.lib().sol_layer_norm_backward(nd, dy, x, gamma, mean, rstd, res, dx, dgamma, dbeta, ws, nbytes, NULL)


def test_layer_norm_refusals(sol):
    L = sol.lib()
    assert norm(sol, None) == 1 and b"descriptor" in L.sol_last_error()
    assert norm(sol, norm_desc(sol), x=NULL) == 1 and norm(sol, norm_desc(sol), y=NULL) == 1
    for bad in (dict(rows=-1), dict(cols=0), dict(ldx=15), dict(ldy=-16), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40)):
        assert norm(sol, norm_desc(sol, **bad)) == 2, bad
    assert norm(sol, norm_desc(sol, dtype=2)) == 3
    for bad in (dict(cols=(1 << 20) + 1), dict(ldx=(1 << 21) + 1), dict(ldy=(1 << 21) + 1)):
        assert norm(sol, norm_desc(sol, **bad)) == 6, bad
    for bad in (dict(x=FAKE + 4), dict(gamma=0x2004), dict(beta=0x3008), dict(y=0x4002), dict(mean=0x5004), dict(rstd=0x6004)):
        assert norm(sol, norm_desc(sol), **bad) == 4, bad
    for bad in (dict(y=0x2000), dict(y=0x3000), dict(mean=FAKE), dict(rstd=0x2000), dict(mean=0x4000), dict(rstd=0x5000)):
        assert norm(sol, norm_desc(sol), **bad) == 6, bad
    assert norm(sol, norm_desc(sol, ldx=32), y=FAKE) == 6                   # y in the place of x, another pitch
    assert norm(sol, norm_desc(sol, rows=0), x=NULL, y=NULL) == 0           # nothing to do


def test_layer_norm_backward_refusals(sol):
    L = sol.lib()
    assert norm_backward(sol, None) == 1
    for bad in (dict(dy=NULL), dict(x=NULL), dict(mean=NULL), dict(rstd=NULL)):
        assert norm_backward(sol, norm_desc(sol), **bad) == 1, bad
    assert norm_backward(sol, norm_desc(sol, ldy=3)) == 2 and norm_backward(sol, norm_desc(sol, dtype=-1)) == 3
    assert norm_backward(sol, norm_desc(sol, ldy=1 << 22)) == 6
    for bad in (dict(dy=FAKE + 4), dict(x=0x2002), dict(gamma=0x3004), dict(mean=0x4004), dict(rstd=0x5008), dict(res=0x6008), dict(dx=0x7004), dict(dgamma=0x8004), dict(dbeta=0x9004)):
        assert norm_backward(sol, norm_desc(sol), **bad) == 4, bad
    for bad in (dict(dx=FAKE), dict(dx=0x2000), dict(dgamma=0x3000), dict(dbeta=0x5000), dict(dgamma=0x6000), dict(dgamma=0x7000), dict(dbeta=0x8000)):
        assert norm_backward(sol, norm_desc(sol), **bad) == 6, bad
    big = norm_desc(sol, rows=100000, cols=1000)
    need = L.sol_layer_norm_backward_workspace_bytes(big)
    assert need >= 2 * 1000 * 4
    assert norm_backward(sol, big, nbytes=need - 1) == 5 and norm_backward(sol, big, ws=NULL, nbytes=need) == 1 and norm_backward(sol, big, ws=0xA004, nbytes=need) == 4
    assert L.sol_layer_norm_backward_workspace_bytes(norm_desc(sol, rows=-1)) == 0
    assert norm_backward(sol, norm_desc(sol, rows=0), dgamma=NULL, dbeta=NULL) == 0


def embed_desc(sol, tokens=6, vocab=10, cols=16, dtype=0, bits=32, ldt=0, ldy=0, scale=1.0, pad=-1):
    return sol.EmbeddingDesc(tokens, vocab, cols, dtype, bits, ldt, ldy, scale, pad)


def embed(sol, ed, tokens=FAKE, table=0x2000, y=0x3000):
    return sol.lib().sol_embedding(ed, tokens, table, y, NULL)


def embed_backward(sol, ed, tokens=FAKE, dy=0x2000, dtable=0x3000, dt=0, acc=0, ws=0x4000, nbytes=1 << 40):
    return sol.lib().sol_embedding_backward(ed, tokens, dy, dtable, dt, acc, ws, nbytes, NULL)


def test_embedding_refusals(sol):
    L = sol.lib()
    for call in (embed, embed_backward):
        assert call(sol, None) == 1 and call(sol, embed_desc(sol), tokens=NULL) == 1
        for bad in (dict(tokens=-1), dict(vocab=0), dict(cols=0), dict(ldt=15), dict(ldy=-1), dict(scale=float("nan")), dict(scale=float("inf"))):
            assert call(sol, embed_desc(sol, **bad)) == 2, bad
        for bad in (dict(dtype=2), dict(bits=16), dict(bits=0)):
            assert call(sol, embed_desc(sol, **bad)) == 3, bad
        for bad in (dict(cols=(1 << 20) + 1), dict(ldt=(1 << 21) + 1), dict(vocab=(1 << 24) + 1), dict(tokens=(1 << 30) + 1)):
            assert call(sol, embed_desc(sol, **bad)) == 6, bad
        assert call(sol, embed_desc(sol), tokens=FAKE + 2) == 4 and call(sol, embed_desc(sol, bits=64), tokens=FAKE + 4) == 4
    assert embed(sol, embed_desc(sol), table=NULL) == 1 and embed(sol, embed_desc(sol), y=NULL) == 1
    assert embed(sol, embed_desc(sol), table=0x2004) == 4 and embed(sol, embed_desc(sol), y=0x3004) == 4
    assert embed(sol, embed_desc(sol), y=0x2000) == 6 and embed(sol, embed_desc(sol), y=FAKE) == 6
    assert embed(sol, embed_desc(sol, tokens=0), tokens=NULL, table=NULL, y=NULL) == 0
    assert embed_backward(sol, embed_desc(sol), dy=NULL) == 1 and embed_backward(sol, embed_desc(sol), dtable=NULL) == 1
    assert embed_backward(sol, embed_desc(sol, tokens=0), dtable=NULL) == 1                 # zeros have to go somewhere
    assert embed_backward(sol, embed_desc(sol), dt=1) == 3                                  # a bf16 gradient of an fp32 table
    assert embed_backward(sol, embed_desc(sol), dy=0x2004) == 4 and embed_backward(sol, embed_desc(sol), dtable=0x3008) == 4
    assert embed_backward(sol, embed_desc(sol), dtable=0x2000) == 6 and embed_backward(sol, embed_desc(sol), dtable=FAKE) == 6
    big = embed_desc(sol, tokens=100000)
    need = L.sol_embedding_backward_workspace_bytes(big)
    assert need > 100000 * 4
    assert embed_backward(sol, big, nbytes=need - 1) == 5 and embed_backward(sol, big, ws=NULL, nbytes=need) == 1 and embed_backward(sol, big, ws=0x4008, nbytes=need) == 4
    assert L.sol_embedding_backward_workspace_bytes(embed_desc(sol, tokens=-1)) == 0


def grads(sol, *entries):
    return (sol.Grad * len(entries))(*[sol.Grad(*e) for e in entries]) if entries else None


def test_grad_refusals(sol):
    L = sol.lib()
    clip = lambda arr, n=None, m=1.0, norm=0x100, ws=0x200, nbytes=1 << 30: L.sol_grad_clip(arr, len(arr) if n is None else n, m, norm, ws, nbytes, NULL)  # noqa: E731
    ok = grads(sol, (0x1000, 0x2000, 100, 0), (0x3000, 0x3000, 7, 1))
    assert clip(ok, n=-1) == 2 and L.sol_grad_clip(None, 1, 1.0, 0x100, 0x200, 1 << 30, NULL) == 1
    assert L.sol_grad_norm(None, 1, 0x100, 0x200, 1 << 30, NULL) == 1 and L.sol_grad_norm(ok, -1, 0x100, 0x200, 1 << 30, NULL) == 2
    for m in (0.0, -1.0, float("nan")):
        assert clip(ok, m=m) == 2
    assert clip(ok, norm=NULL) == 1 and clip(ok, norm=0x102) == 4
    need = L.sol_grad_workspace_bytes(ok, 2)
    assert need >= 16 and clip(ok, nbytes=need - 1) == 5 and clip(ok, ws=NULL) == 1 and clip(ok, ws=0x208) == 4
    assert L.sol_grad_norm(ok, 2, 0x100, 0x200, need - 1, NULL) == 5
    for e, want in (((NULL, 0x2000, 4, 0), 1), ((0x1000, NULL, 4, 0), 1), ((0x1002, 0x2000, 4, 0), 4), ((0x1000, 0x2002, 4, 0), 4), ((0x1001, 0x2000, 4, 1), 4), ((0x1000, 0x2000, 4, 2), 3),
                    ((0x1000, 0x2000, 1 << 40, 0), 6)):
        assert clip(grads(sol, e)) == want, e
    assert clip(grads(sol, (0x1000, 0x2000, 1 << 39, 0), (1 << 50, 1 << 51, 1 << 39, 1))) == 6          # together
    assert clip(grads(sol, *[(0x1000, 0x1000, 0, 0)] * 32769)) == 6
    # memory that two entries share: the same tensor twice, an output on another gradient, overlapping ends, an output that starts inside its own gradient
    for entries in (((0x1000, 0x1000, 4, 0), (0x1000, 0x1000, 4, 0)), ((0x1000, 0x2000, 4, 0), (0x2000, 0x3000, 4, 0)), ((0x1000, 0x5000, 8, 0), (0x3000, 0x5010, 8, 0)),
                    ((0x1000, 0x1004, 8, 0),), ((0x1000, 0x1000, 8, 1), (0x100e, 0x100e, 8, 1)),
                    tuple((0x10000 + 0x100 * i, 0x10000 + 0x100 * i, 4, 0) for i in range(400)) + ((0x10100, 0x90000, 1, 0),)):
        assert clip(grads(sol, *entries)) == 6, entries
    assert L.sol_grad_workspace_bytes(grads(sol, (0x1000, 0, 5, 9)), 1) == 0


def test_clip_refuses_a_norm_inside_the_gradients(sol):
    """The norm is written while gradients are scaled: it may not be a part of one, nor of what is written for it.  Behind the last element and in front of the first there is room."""
    L = sol.lib()
    clip = lambda arr, norm: L.sol_grad_clip(arr, len(arr), 1.0, norm, NULL, 0, NULL)  # noqa: E731  no workspace: 5 where everything else is right
    for many in (1, 300):
        arr = grads(sol, *[(0x10000 + 0x100 * i, 0x80000 + 0x100 * i, 4, 0) for i in range(many)])
        last = 0x100 * (many - 1)
        for at in (0x10000, 0x1000c, 0x80000, 0x8000c, 0x10000 + last, 0x8000c + last):
            assert clip(arr, at) == 6, hex(at)
        for at in (0xfffc, 0x10010, 0x7fffc, 0x80010, 0x10010 + last, 0x80010 + last):
            assert clip(arr, at) == 5, hex(at)
    half = grads(sol, (0x10002, 0x10002, 3, 1))         # bf16: the norm's 4 bytes reach over its first element, or begin on its last
    assert clip(half, 0x10000) == 6 and clip(half, 0x10004) == 6 and clip(half, 0x10008) == 5


def test_binding_refuses_what_is_not_on_the_gpu(sol):
    import torch

    x, v = torch.zeros(4, 32), torch.zeros(32)
    for f in (lambda: sol.sol_layer_norm(x, v, v), lambda: sol.sol_layer_norm_backward(x, x, torch.zeros(4), torch.zeros(4), v),
              lambda: sol.sol_embedding(torch.zeros(3, dtype=torch.int64), x), lambda: sol.sol_embedding_backward(x, torch.zeros(4, dtype=torch.int64), 9),
              lambda: sol.sol_grad_norm([x]), lambda: sol.sol_grad_clip([x], 1.0), lambda: sol.sol_grad_norm([])):
        with pytest.raises(ValueError):
            f()


def test_networks_clip_only_when_they_train(sol):
    layers = sol.make_layer_array([{"kind": "linear", "out": 8}])
    for flags, want in ((0, 6), (sol.NET_TRAINING, 5)):                      # not created for training; no parameter buffer bound
        h = C.c_void_p(0)
        assert sol.lib().sol_network_create(layers, 1, C.byref(sol.TensorDesc(2, 1, 1, 8, sol.F32)), flags, C.byref(h)) == 0
        assert sol.lib().sol_network_clip_gradients(h, 1.0, 0x100, 0x200, 1 << 20, NULL) == want
        assert (sol.lib().sol_network_clip_workspace_bytes(h) > 0) == bool(flags)
        sol.lib().sol_network_destroy(h)
    assert sol.lib().sol_network_clip_gradients(None, 1.0, 0x100, 0x200, 1 << 20, NULL) == 1 and sol.lib().sol_network_clip_workspace_bytes(None) == 0


class Recorder:
    """The library, but for the calls that would launch kernels: those are noted down with their arguments and return 0."""

    def __init__(self, real, names):
        self.real, self.names, self.calls = real, names, []

    def __getattr__(self, name):
        if name in self.names:
            return lambda *args: self.calls.append((name, args)) or 0
        return getattr(self.real, name)


@pytest.fixture
def host_network(sol, monkeypatch):
    """A training network in host memory, whose device calls are noted down only, and which may make no tensor once it is there."""
    import torch

    rec = Recorder(sol.lib(), ("sol_network_clip_gradients", "sol_network_backward"))
    monkeypatch.setattr(sol, "lib", lambda: rec)
    monkeypatch.setattr(sol, "_addr", lambda t: 0 if t is None else t.data_ptr() if isinstance(t, torch.Tensor) else int(t))
    net = sol.Network([{"kind": "linear", "out": 8}], (2, 8, 1, 1), sol.F32, device="cpu", flags=sol.NET_TRAINING)

    def none(*args, **kw):
        raise AssertionError("a tensor made by the call belongs to the current stream, not to the call's")

    for name in ("zeros", "empty"):
        monkeypatch.setattr(torch, name, none)
    return net, rec


class OtherStream:
    cuda_stream = 0x77


def test_network_clipping_makes_nothing_on_the_current_stream(sol, host_network):
    """Its norm and its scratch, which the call's stream writes, are there before the first call."""
    net, rec = host_network
    norm = net.clip_gradients(0.5, stream=OtherStream)
    (name, args), = rec.calls
    assert name == "sol_network_clip_gradients" and args[1] == 0.5 and args[2] == norm.data_ptr() and args[5] == 0x77
    need = rec.sol_network_clip_workspace_bytes(net._h)
    assert need > 0 and args[4] >= need and args[3] == net.clip_space.data_ptr()
    net.clip_gradients(0.25, stream=OtherStream)
    assert rec.calls[1][1][2:] == args[2:]


def test_network_backward_makes_nothing_on_the_current_stream(sol, host_network):
    """Likewise the loss."""
    import ctypes

    net, rec = host_network
    x, labels = ctypes.addressof(ctypes.create_string_buffer(64)), 0x40
    loss = net.backward(x, labels, stream=OtherStream)
    (name, args), = rec.calls
    assert name == "sol_network_backward" and args[1:4] == (x, labels, loss.data_ptr()) and args[-1] == 0x77 and loss.data_ptr() == net.loss.data_ptr()


def test_clip_refuses_a_workspace_inside_what_it_reads_or_writes(sol):
    """The partial sums lie there while gradients are read and results and the norm written.  Only the bytes that are needed count; each call here is refused, so that nothing is launched."""
    L = sol.lib()
    for many in (1, 300):
        arr = grads(sol, *[(0x100000 + 0x100 * i, 0x800000 + 0x100 * i, 4, 0) for i in range(many)])
        need, last = L.sol_grad_workspace_bytes(arr, many), 0x100 * (many - 1)
        assert need == 8 * many
        for call in (lambda ws, norm, n=need: L.sol_grad_norm(arr, many, norm, ws, n, NULL), lambda ws, norm, n=need: L.sol_grad_clip(arr, many, 1.0, norm, ws, n, NULL)):
            for ws in (0x100000, 0x100000 + last, 0x100000 - need + 16 & ~15):
                assert call(ws, 0x40) == 6 and b"workspace" in L.sol_last_error(), hex(ws)
            ws = 0x4000000
            for norm in (ws, ws + need - 4):
                assert call(ws, norm) == 6 and b"workspace" in L.sol_last_error()
                assert call(ws, norm, 1 << 20) == 6
        for ws in (0x800000, 0x800000 + last):                    # where clipping writes
            assert L.sol_grad_clip(arr, many, 1.0, 0x40, ws, need, NULL) == 6 and b"workspace" in L.sol_last_error()
    half = grads(sol, (0x10010, 0x20010, 3, 1))
    assert L.sol_grad_norm(half, 1, 0x40, 0x10010, 8, NULL) == 6 and L.sol_grad_clip(half, 1, 1.0, 0x40, 0x20010, 8, NULL) == 6
