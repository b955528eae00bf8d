"""The linear layer with its epilogue, its backward pass, and dropout, through the public entry points against the 64-bit oracle.

Two kinds of checks.  Whole numbers: inputs are small integers and dropout's factor is 2 (p = 1/2), so that every product and every sum below 2^24 is exact
in fp32 whatever its order, and the outputs have to be EQUAL (for bf16 after one rounding of the exact value); this catches a single product
too many or too few.  Real numbers: tolerances are counted in roundings (`half` = half a step of the output type, U = 2^-24 for a sum's additions).
"""
import numpy as np
import pytest
import torch

from oracle import linear_ops as lo

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0**-24, "bf16": 2.0**-8}      # half a step, relative
U = 2.0**-24
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
DROP = (0.5, 0x123456789ABCDEF, 3, 41)          # p, seed, call, step


@pytest.fixture(scope="module")
def sol():
    from paper_2003_10688_amd import sol as s

    s.lib()
    return s


def dev(a, dt="f32", pitch=0, fill=float("nan")):
    """Device tensor of a 2-d array; pitch: so many more columns per row, which hold `fill`."""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to("cuda:0", TDT[dt])
    if not pitch:
        return t
    wide = torch.full((a.shape[0], a.shape[1] + pitch), fill, dtype=TDT[dt], device="cuda:0")
    wide[:, :a.shape[1]] = t
    return wide[:, :a.shape[1]]


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def pack(w, dt):
    block = 64 if dt == "bf16" else 32
    p = torch.zeros((w.shape[0], -(-w.shape[1] // block) * block), dtype=TDT[dt], device="cuda:0")
    p[:, :w.shape[1]] = dev(w, dt)
    return p


def grid(a, dt):
    """Values that dt holds exactly."""
    return a if dt == "f32" and a.dtype == np.float32 else host(torch.from_numpy(np.asarray(a, np.float32)).to(TDT[dt]))


def dropper(sol, drop):
    if drop is None:
        return None
    p, seed, call, step = drop
    return sol.Dropout(p, seed, call, torch.tensor([step], dtype=torch.int32, device="cuda:0"))


def act_id(sol, name):
    return {n: i for i, n in enumerate(lo.ACTS)}[name]


SHAPES = [
    # rows, in, out                    what it reaches
    (1, 1, 1),
    (1, 8, 8), (3, 5, 7),
    (2, 64, 64), (16, 100, 33),
    (17, 2048, 1000),                  # a classifier
    (65, 72, 130), (64, 96, 513),      # tiles of 64 with remainders
    (129, 250, 65), (200, 1531, 257),  # odd rows
    (33, 4096, 40),                    # a long reduction, few tiles
    (777, 33, 1030),                   # tiles of 128 and more
    (2050, 40, 1700),
    (2600, 72, 5130),                  # the largest tiles, with remainders
    (5121, 136, 2570),
    (1, 2048, 10), (16, 2056, 33), (32, 1032, 520), (65, 2088, 72), (128, 2048, 4100), (9, 4096, 8200), (64, 1031, 515),    # weights streamed past few rows, with remainders of all three
    (5121, 200, 3300), (5121, 3300, 150), (150, 3300, 5121), (264, 2056, 8200),     # more of them than the GPU has compute units, in each of the three products
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_whole_numbers(sol, dt, rows, n_in, n_out):
    """Forward and backward, equal to the last bit: every product and sum is a whole number below 2^24."""
    rng = np.random.default_rng([rows, n_in, n_out])
    ints = lambda *s: rng.integers(-2, 3, s).astype(np.float32)  # noqa: E731
    x, w, b, r, g = ints(rows, n_in), ints(n_out, n_in), ints(n_out), ints(rows, n_out), ints(rows, n_out)
    pitch = (rows * 7 + n_in) % 3 * 8 + (5 if rows % 2 else 0)
    xd, wd = dev(x, dt, pitch), pack(w, dt)
    for act, drop, res in (("none", None, None), ("relu", DROP, r), ("relu", None, None), ("none", DROP, r)):
        y, z = sol.sol_linear_fused(xd, wd, n_out, bias=dev(b[None])[0], act=act_id(sol, act), drop=dropper(sol, drop),
                                    residual=dev(res, dt, pitch) if res is not None else None, want_preact=True)
        want, wz = lo.linear_fused(x, w, b, act, drop, res)
        assert np.array_equal(host(z), grid(wz, dt)) and np.array_equal(host(y), grid(want, dt))
        zq = grid(wz, dt)
        dx, dw, db = sol.sol_linear_backward(dev(g, dt, pitch), xd, wd, preact=z, act=act_id(sol, act), drop=dropper(sol, drop))
        wdx, wdw, wdb, _ = lo.linear_fused_bwd(g, x, w, zq, act, drop)
        assert np.array_equal(host(dx), grid(wdx, dt)) and np.array_equal(host(dw), grid(wdw, dt)) and np.array_equal(host(db), wdb)
        if dt == "bf16":
            _, dw32, _ = sol.sol_linear_backward(dev(g, dt), xd, wd, preact=z, act=act_id(sol, act), drop=dropper(sol, drop), need_dx=False, need_db=False, dw_dtype=torch.float32)
            assert np.array_equal(host(dw32), wdw)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 3, 33, 200, 300])
def test_every_element_of_a_row_counts(sol, dt, rows):
    """Ones times ones: the sum is the number of elements, for lengths that end anywhere in a 16-byte piece and in a stage."""
    for n_in in (*range(1, 18), *range(509, 530), 1531, 2045, 2049):
        x = dev(np.ones((rows, n_in), np.float32), dt)
        y, _ = sol.sol_linear_fused(x, pack(np.ones((40, n_in), np.float32), dt), 40)
        assert np.array_equal(host(y), grid(np.full((rows, 40), float(n_in)), dt)), n_in


# ---- the tile kernels, one product at a time, on reductions longer than their rings: whole numbers against torch's fp32 product of the same whole numbers
KINDS = ("forward", "dx", "dw")


def ints_on_gpu(gen, rows, cols, dt, gap=0):
    """Whole numbers -2 .. 2 in rows that `gap` columns of NaN lie between."""
    t = torch.full((rows, cols + gap), float("nan"), dtype=TDT[dt], device="cuda:0")[:, :cols]
    return t.copy_(torch.randint(-2, 3, (rows, cols), generator=gen, device="cuda:0", dtype=torch.int8))


def packed_on_gpu(w):
    block = 64 if w.dtype == torch.bfloat16 else 32
    p = torch.zeros((w.shape[0], -(-w.shape[1] // block) * block), dtype=w.dtype, device="cuda:0")
    p[:, :w.shape[1]] = w
    return p


def check_product(sol, kind, dt, n, c, k, tiles, plain):
    """A product of n rows and c columns over k has to run on a tile in `tiles` (0: streamed weights) and be right to the last bit.  plain: no activation and no dropout, so that the backward products read dy itself
    where its rows are aligned."""
    gen = torch.Generator(device="cuda:0").manual_seed(n * 31 + c * 7 + k)
    ints = lambda rows, cols, gap=0: ints_on_gpu(gen, rows, cols, dt, gap)  # noqa: E731
    act, d = (sol.ACT_NONE, None) if plain else (sol.ACT_RELU, sol.Dropout(0.5, 7, 3))
    if kind == "forward":
        x, w, b, r = ints(n, k, 8), ints(c, k), torch.randint(-2, 3, (c,), generator=gen, device="cuda:0").float(), ints(n, c, 5)
        y, z = sol.sol_linear_fused(x, packed_on_gpu(w), c, bias=b, act=act, drop=d, residual=r, want_preact=True)
        assert sol.sol_debug_linear_tile(0) in tiles
        wz = x.float() @ w.float().t() + b
        v = wz if plain else sol.sol_dropout(wz.clamp(min=0), d)
        assert torch.equal(z, wz.to(TDT[dt])) and torch.equal(y, (v + r.float()).to(TDT[dt]))
        return
    m, n_in, n_out = (n, c, k) if kind == "dx" else (k, c, n)
    x, w, g = ints(m, n_in, 8), ints(n_out, n_in), ints(m, n_out, 8)
    z = None if plain else ints(m, n_out)
    dx, dw, _ = sol.sol_linear_backward(g, x, packed_on_gpu(w), preact=z, act=act, drop=d, need_dx=kind == "dx", need_dw=kind == "dw", need_db=False)
    assert sol.sol_debug_linear_tile(KINDS.index(kind)) in tiles
    dz = g.float() if plain else sol.sol_dropout(g.float().contiguous(), d) * (z > 0)
    if kind == "dx":
        assert torch.equal(dx, (dz @ w.float()).to(TDT[dt]))
    else:
        assert torch.equal(dw, (dz.t() @ x.float()).to(TDT[dt]))


# stages of 64 products and the length of the last: the ring of the 256-tile kernel has ten units, four a stage, and repeats after five stages
HUGE = [(1, 40), (2, 56), (3, 8), (4, 64), (4, 8), (5, 24), (5, 64), (6, 40), (7, 13), (8, 61), (9, 56), (10, 8), (11, 64), (11, 48), (12, 1), (13, 31), (16, 16), (21, 40)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("stages,last", HUGE)
def test_largest_tiles_over_every_turn_of_their_ring(sol, kind, stages, last):
    """Rows and columns end inside a tile, the reduction inside a 16-byte piece (odd: rows are copied), inside a stage or on its end."""
    k = (stages - 1) * 64 + last
    check_product(sol, kind, "bf16", 3904, 4000, k, (256,), True)
    check_product(sol, kind, "bf16", 3900, 4001, k, (256,), False)


RINGS = [       # type, rows, columns, the tile
    ("bf16", 950, 1000, 64),        # up to 256 tiles: a ring of five stages forward, three backward
    ("bf16", 500, 900, 64),         # the same, with streamed weights for the longest reductions forward
    ("bf16", 1100, 1304, 64),       # more
    ("bf16", 2000, 1992, 128),      # up to 256: a ring of four
    ("bf16", 2900, 2801, 128),      # more: rings of two
    ("f32", 500, 900, 64),
    ("f32", 2000, 1990, 128),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dt,n,c,tile", RINGS)
def test_smaller_tiles_over_every_turn_of_their_rings(sol, kind, dt, n, c, tile):
    stage = 64 if dt == "bf16" else 32
    for stages, last in ((8, 8), (9, 16), (10, stage), (11, 12), (12, 31), (13, 5), (17, 24), (30, 8)):
        k = (stages - 1) * stage + last
        check_product(sol, kind, dt, n, c, k, (tile, 0) if n == 500 and kind == "forward" else (tile,), stages % 2 == 0)


def close(got, want, tol, what):
    bad = np.abs(got - want) - tol
    assert np.all(np.isfinite(got)) and bad.max() <= 0, f"{what}: off by {np.abs(got - want).flat[bad.argmax()]:.3g}, {tol.flat[bad.argmax()]:.3g} allowed, at {np.unravel_index(bad.argmax(), bad.shape)}"


# Roundings of an activation in fp32 (exp2 and the reciprocal: 1 ulp each; the tail's fit 1.5e-7; about ten operations): relative to |z| and slope's size
ACT_ERR = 3e-6


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", lo.ACTS)
@pytest.mark.parametrize("rows,n_in,n_out,p", [(5, 40, 24, 0.1), (130, 777, 201, 0.25), (300, 512, 1100, 0.0), (2600, 64, 5130, 0.1)])
def test_real_numbers(sol, dt, act, rows, n_in, n_out, p):
    rng = np.random.default_rng([rows, n_in, n_out, len(act)])
    x, w = grid(rng.standard_normal((rows, n_in)), dt), grid(rng.standard_normal((n_out, n_in)) * (2 / np.sqrt(n_in)), dt)
    b, r, g = rng.standard_normal(n_out).astype(np.float32), grid(rng.standard_normal((rows, n_out)), dt), grid(rng.standard_normal((rows, n_out)), dt)
    drop = (p, 99 + (7 << 40), 1, 0) if p else None
    y, z = sol.sol_linear_fused(dev(x, dt), pack(w, dt), n_out, bias=dev(b[None])[0], act=act_id(sol, act), drop=dropper(sol, drop), residual=dev(r, dt), want_preact=True)
    want, wz = lo.linear_fused(x, w, b, act, drop, r)
    half, scale = HALF[dt], 1 / (1 - p) * 1.001
    # a sum of n products: at most n + 1 additions, each off by U of the partial sum, which is at most the sum of magnitudes
    zerr = (n_in + 2) * U * (np.abs(x) @ np.abs(w).T + np.abs(b))
    close(host(z), wz, half * np.abs(wz) * 1.01 + zerr, "z")
    # |act'| <= 1.13; then dropout's factor, the residual's addition and the output's rounding
    close(host(y), want, half * np.abs(want) * 1.01 + scale * (1.13 * zerr + ACT_ERR * np.abs(wz)) + 4 * U * (np.abs(want) + np.abs(r)), "y")

    zq = host(z)
    dx, dw, db = sol.sol_linear_backward(dev(g, dt), dev(x, dt), pack(w, dt), preact=z, act=act_id(sol, act), drop=dropper(sol, drop))
    wdx, wdw, wdb, wdz = lo.linear_fused_bwd(g, x, w, zq, act, drop)
    gz = lo.dropout(np.abs(g), *drop) if drop else np.abs(g)
    edz = ACT_ERR * 2 * gz                                    # of dz before it is rounded: slopes are at most 1.13
    rdz = half * np.abs(wdz) * 1.01 + edz if dt == "bf16" else edz      # bf16: as the products take it
    close(host(dx), wdx, half * np.abs(wdx) * 1.01 + rdz @ np.abs(w) + (n_out + 2) * U * (np.abs(wdz) @ np.abs(w)), "dx")
    close(host(dw), wdw, half * np.abs(wdw) * 1.01 + rdz.T @ np.abs(x) + (rows + 20) * U * (np.abs(wdz).T @ np.abs(x)), "dW")
    close(host(db), wdb, edz.sum(0) + (rows + 20) * U * np.abs(wdz).sum(0), "db")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,p", [(1, 1, 0.5), (1, 2048, 0.1), (3, 7, 0.25), (64, 2048, 0.5), (129, 1001, 0.1), (5, 13, 1.0), (5, 13, 0.0), (1000, 257, 0.999)])
def test_dropout(sol, dt, rows, cols, p):
    rng = np.random.default_rng([rows, cols])
    x, r = grid(rng.standard_normal((rows, cols)), dt), grid(rng.standard_normal((rows, cols)), dt)
    drop = (p, 2**63 + 12345, 2**32 - 1, -2)                  # the step word's bits are what counts
    t = (p, 2**63 + 12345, 2**32 - 1, 2**32 - 2)
    for res in (None, r):
        want = lo.dropout(x, *t) + (0 if res is None else res)
        got = host(sol.sol_dropout(dev(x, dt), dropper(sol, drop), residual=None if res is None else dev(res, dt)))
        # the factor and the product round once each, the sum and the output once each
        close(got, want, HALF[dt] * np.abs(want) * 1.01 + 4 * U * (np.abs(lo.dropout(x, *t)) + np.abs(want)), "y")
        if res is None:
            assert np.array_equal(got == 0, (want == 0))
    a = dev(x, dt)
    b = a.clone()
    want = sol.sol_dropout(a, dropper(sol, drop), residual=dev(r, dt))
    assert torch.equal(sol.sol_dropout(b, dropper(sol, drop), residual=dev(r, dt), out=b), want) and torch.equal(b, want)   # in place


def test_dropout_masks_agree(sol):
    """The product's epilogue, its backward pass and the pass on its own drop the same elements, whatever the pitches."""
    rows, n_in, n_out = 77, 64, 203
    x, w = torch.ones((rows, n_in), device="cuda:0", dtype=torch.bfloat16), pack(np.ones((n_out, n_in)), "bf16")
    d = dropper(sol, (0.3, 5, 9, 1))
    y, _ = sol.sol_linear_fused(x, w, n_out, drop=d, out=torch.empty((rows, n_out + 5), device="cuda:0", dtype=torch.bfloat16)[:, :n_out])
    alone = sol.sol_dropout(torch.ones((rows, n_out), device="cuda:0"), d)
    assert torch.equal(y != 0, alone != 0)
    _, dw, db = sol.sol_linear_backward(torch.ones((rows, n_out), device="cuda:0", dtype=torch.bfloat16), x, w, drop=d, need_dx=False, dw_dtype=torch.float32)
    kept = (alone != 0).float().sum(0)
    scale = 65536 / (65536 - round(0.3 * 65536))
    # dz = the factor, rounded to bf16, in every kept place
    assert torch.equal(dw[:, 0], kept * float(torch.tensor(scale).to(torch.bfloat16))) and torch.allclose(db, kept * scale, rtol=77 * U)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 72, 24), (70, 40, 90), (70, 41, 90), (300, 200, 700)])
def test_what_lies_between_rows(sol, dt, rows, n_in, n_out):
    """Gaps of NaN beside x, dy and the residual do not reach a result, and the gaps of y stay as they were."""
    rng = np.random.default_rng(rows)
    x, w, r = rng.integers(-2, 3, (rows, n_in)), rng.integers(-2, 3, (n_out, n_in)), rng.integers(-2, 3, (rows, n_out))
    for pitch in (3, 8, 64):
        out = torch.full((rows, n_out + pitch), 7.0, dtype=TDT[dt], device="cuda:0")
        sol.sol_linear_fused(dev(x, dt, pitch), pack(w, dt), n_out, residual=dev(r, dt, pitch), out=out[:, :n_out])
        assert np.array_equal(host(out[:, :n_out]), grid(lo.linear_fused(x, w, residual=r)[0], dt)) and torch.all(out[:, n_out:] == 7)
        dx, dw, db = sol.sol_linear_backward(dev(r, dt, pitch), dev(x, dt, pitch), pack(w, dt))
        want = lo.linear_fused_bwd(r, x, w, None)
        assert np.array_equal(host(dx), grid(want[0], dt)) and np.array_equal(host(dw), grid(want[1], dt)) and np.array_equal(host(db), want[2])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n_in,n_out", [(9, 40, 30), (140, 72, 200)])
def test_rows_that_are_not_finite(sol, dt, rows, n_in, n_out):
    """An infinity or a NaN in one row of x stays in that row of y and dx; dropped places are 0 even there; activations take their limits."""
    rng = np.random.default_rng(2)
    x, w = rng.integers(1, 3, (rows, n_in)).astype(np.float32), rng.integers(1, 3, (n_out, n_in)).astype(np.float32)
    x[2, 3], x[4, 0], x[5, n_in - 1] = np.inf, np.nan, -np.inf
    for act in lo.ACTS:
        y, z = sol.sol_linear_fused(dev(x, dt), pack(w, dt), n_out, act=act_id(sol, act), want_preact=True)
        y, z = host(y), host(z)
        fine = np.delete(np.arange(rows), [2, 4, 5])
        assert np.all(np.isfinite(y[fine])) and np.all(z[2] == np.inf) and np.all(z[5] == -np.inf) and np.all(np.isnan(z[4]))
        assert np.all(y[2] == np.inf) and (np.all(y[4] == 0) if act == "relu" else np.all(np.isnan(y[4])))
        assert np.all(y[5] == -np.inf) if act == "none" else np.all(np.abs(y[5]) < 1e-30)
        g = np.ones((rows, n_out), np.float32)
        zt = dev(np.where(np.isnan(z), 0, z), dt)
        dx, _, db = sol.sol_linear_backward(dev(g, dt), dev(np.where(np.isfinite(x), x, 0), dt), pack(w, dt), preact=zt, act=act_id(sol, act))
        assert np.all(np.isfinite(host(dx))) and np.all(np.isfinite(host(db)))          # slopes of infinite z are 0 and 1
        assert np.all(host(dx)[5] == (host(dx)[0] if act == "none" else 0))
    d = dropper(sol, DROP)
    y, _ = sol.sol_linear_fused(dev(x, dt), pack(w, dt), n_out, drop=d)
    kept = lo.dropout_kept(rows, n_out, *DROP)
    assert np.all(host(y)[~kept] == 0) and np.all(np.isnan(host(y)[4][kept[4]]))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_equal_rows_equal_bits_and_repeats(sol, dt):
    """A call repeated gives the same bits, for every output."""
    rng = np.random.default_rng(8)
    x, w, g = dev(rng.standard_normal((333, 520)), dt), pack(rng.standard_normal((410, 520)), dt), dev(rng.standard_normal((333, 410)), dt)
    d = dropper(sol, (0.1, 3, 0, 0))
    first = None
    for _ in range(3):
        y, z = sol.sol_linear_fused(x, w, 410, act=sol.ACT_GELU, drop=d, want_preact=True)
        got = (y, z) + sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_GELU, drop=d)
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


@pytest.mark.parametrize("dt,rows,n_in,n_out", [("bf16", 1, 2048, 1000), ("bf16", 16, 4096, 520), ("bf16", 77, 2056, 300), ("f32", 130, 1100, 90), ("f32", 20, 2000, 1000),
                                                ("bf16", 500, 700, 900), ("bf16", 2000, 1000, 1992), ("bf16", 2900, 700, 2801), ("bf16", 3900, 500, 4001), ("f32", 500, 333, 900),
                                                ("f32", 2000, 500, 1990)])
def test_equal_rows_give_equal_bits(sol, dt, rows, n_in, n_out):
    """Copies of one row: every row of y, z and dx has the bits of the first, wherever in a tile it lies."""
    rng = np.random.default_rng([rows, n_in])
    same = lambda n: dev(rng.standard_normal((1, n)), dt).expand(rows, n).contiguous()  # noqa: E731
    x, w, g = same(n_in), pack(rng.standard_normal((n_out, n_in)) / np.sqrt(n_in), dt), same(n_out)
    y, z = sol.sol_linear_fused(x, w, n_out, act=sol.ACT_SILU, residual=g, want_preact=True)
    dx, _, _ = sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_SILU, need_dw=False)
    for t in (y, z, dx):
        assert torch.equal(t, t[:1].expand_as(t).contiguous())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 128, 2048), (512, 256, 512), (40, 2048, 1000), (2600, 72, 5130)])
def test_what_bits_do_not_depend_on(sol, dt, rows, n_in, n_out):
    """Neither the outputs without a product (z, db) nor where anything lies in memory changes the order of a sum; asking for dx or dW alone may."""
    rng = np.random.default_rng([rows, n_out])
    x, w, g = dev(rng.standard_normal((rows, n_in)), dt), pack(rng.standard_normal((n_out, n_in)) / np.sqrt(n_in), dt), dev(rng.standard_normal((rows, n_out)), dt)
    y, z = sol.sol_linear_fused(x, w, n_out, act=sol.ACT_SILU, want_preact=True)
    bw = lambda x_=x, w_=w, g_=g, **kw: sol.sol_linear_backward(g_, x_, w_, preact=z, act=sol.ACT_SILU, **kw)  # noqa: E731
    want, one = bw(), (bw(need_dw=False)[0], bw(need_dx=False)[1])
    keep, room = [], torch.empty(1 << 27, dtype=torch.uint8, device="cuda:0")
    for i in range(3):
        x2, w2, g2 = x.clone(), w.clone(), g.clone()
        keep.append((x2, w2, g2))
        assert torch.equal(sol.sol_linear_fused(x2, w2, n_out, act=sol.ACT_SILU)[0], y)
        assert all(torch.equal(a, b) for a, b in zip(bw(x2, w2, g2, workspace=room[i * 4096:]), want))
        got = bw(x2, w2, g2, need_db=False)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(bw(need_dw=False, need_db=False)[0], one[0]) and torch.equal(bw(need_dx=False, need_db=False)[1], one[1]) and torch.equal(bw(need_dx=False, need_dw=False)[2], want[2])


def block_forward(sol, x, w1, b1, w2, b2, hidden, d1, d2):
    """A feed-forward block with a residual: x + dropout(W2 dropout(gelu(W1 x + b1)) + b2)."""
    h, z = sol.sol_linear_fused(x, w1, hidden, bias=b1, act=sol.ACT_GELU, drop=d1, want_preact=True)
    y, _ = sol.sol_linear_fused(h, w2, x.shape[1], bias=b2, drop=d2, residual=x)
    return y, h, z


def block_backward(sol, g, x, h, z, w1, w2, d1, d2):
    dh, dw2, db2 = sol.sol_linear_backward(g, h, w2, drop=d2)
    dx, dw1, db1 = sol.sol_linear_backward(dh, x, w1, preact=z, act=sol.ACT_GELU, drop=d1)
    return dx + g, dw1, db1, dw2, db2


def block_inputs(dt, rows, width, hidden, seed=1):
    rng = np.random.default_rng(seed)
    a = {"x": rng.standard_normal((rows, width)), "w1": rng.standard_normal((hidden, width)) / np.sqrt(width), "w2": rng.standard_normal((width, hidden)) / np.sqrt(hidden),
         "g": rng.standard_normal((rows, width))}
    a = {k: grid(v, dt) for k, v in a.items()}
    a["b1"], a["b2"] = rng.standard_normal(hidden).astype(np.float32), rng.standard_normal(width).astype(np.float32)
    return a


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width,hidden", [(50, 96, 384), (257, 200, 801)])
def test_block_against_the_oracle(sol, dt, rows, width, hidden):
    """The operators as they are used together.  Each step adds its own roundings; relative 2-norms: bf16 rounds h, y, dh, dz and the outputs (five times
    2^-8 / sqrt(3) at most, added up), fp32 sums of up to 801 products."""
    a = block_inputs(dt, rows, width, hidden)
    s1, s2 = (0.1, 77, 0, 6), (0.2, 77, 1, 6)
    h, z = lo.linear_fused(a["x"], a["w1"], a["b1"], "gelu", s1)
    y, _ = lo.linear_fused(h, a["w2"], a["b2"], "none", s2, a["x"])
    dh, dw2, db2, _ = lo.linear_fused_bwd(a["g"], h, a["w2"], None, "none", s2)
    dx, dw1, db1, _ = lo.linear_fused_bwd(dh, a["x"], a["w1"], z, "gelu", s1)
    x, w1, w2, g = dev(a["x"], dt), pack(a["w1"], dt), pack(a["w2"], dt), dev(a["g"], dt)
    d1, d2 = dropper(sol, s1), dropper(sol, s2)
    gy, gh, gz = block_forward(sol, x, w1, dev(a["b1"][None])[0], w2, dev(a["b2"][None])[0], hidden, d1, d2)
    got = (gy,) + block_backward(sol, g, x, gh, gz, w1, w2, d1, d2)
    tol = 5 * HALF["bf16"] / np.sqrt(3) if dt == "bf16" else 1e-5
    for name, v, want in zip(("y", "dx", "dw1", "db1", "dw2", "db2"), got, (y, dx + a["g"], dw1, db1, dw2, db2)):
        assert np.linalg.norm(host(v) - want) <= tol * np.linalg.norm(want), name


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_gradients_are_differences(sol, act):
    """Directional derivatives in fp32 by central differences of the kernels' own forward pass."""
    rng = np.random.default_rng(4)
    rows, n_in, n_out = 40, 36, 52
    x, w, b, g = rng.standard_normal((rows, n_in)), rng.standard_normal((n_out, n_in)) / 6, rng.standard_normal(n_out), rng.standard_normal((rows, n_out))
    d, act = dropper(sol, (0.25, 11, 0, 0)), act_id(sol, act)
    out = lambda x_, w_, b_: host(sol.sol_linear_fused(dev(x_), pack(w_, "f32"), n_out, bias=dev(b_[None])[0], act=act, drop=d)[0])  # noqa: E731
    z = sol.sol_linear_fused(dev(x), pack(w, "f32"), n_out, bias=dev(b[None])[0], act=act, want_preact=True)[1]
    grads = [host(t) for t in sol.sol_linear_backward(dev(g), dev(x), pack(w, "f32"), preact=z, act=act, drop=d)]
    for i, t in enumerate((x, w, b)):
        u = rng.standard_normal(t.shape)
        h = 2.0**-7
        up, down = [x, w, b], [x, w, b]
        up[i], down[i] = t + h * u, t - h * u
        slope = float(((out(*up) - out(*down)) * g).sum()) / (2 * h)
        want = float((grads[i] * u).sum())
        # h^2 / 6 of a third derivative of order one along a step of unit size per element, and fp32 roundings over 2h
        assert abs(slope - want) <= 1e-3 * np.linalg.norm(grads[i]) * np.linalg.norm(u), (i, slope, want)


def test_another_stream_and_caller_workspace(sol):
    rng = np.random.default_rng(6)
    x, w, g = dev(rng.standard_normal((100, 77)), "bf16"), pack(rng.standard_normal((90, 77)), "bf16"), dev(rng.standard_normal((100, 90)), "bf16")
    d = dropper(sol, (0.1, 3, 0, 0))
    y, z = sol.sol_linear_fused(x, w, 90, act=sol.ACT_SILU, drop=d, want_preact=True)
    want = (y, z) + sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_SILU, drop=d) + (sol.sol_dropout(g, d),)
    torch.cuda.synchronize()
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    st = torch.cuda.Stream()
    y, z2 = sol.sol_linear_fused(x, w, 90, act=sol.ACT_SILU, drop=d, want_preact=True, workspace=ws, stream=st)
    got = (y, z2) + sol.sol_linear_backward(g, x, w, preact=z2, act=sol.ACT_SILU, drop=d, workspace=ws, stream=st) + (sol.sol_dropout(g, d, stream=st),)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with pytest.raises(sol.SolError) as e:
        sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_SILU, workspace=ws[:1024])
    assert e.value.status == 5


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_calls_on_other_streams_without_a_workspace(sol, dt):
    """Two streams that have work in front of the calls, each with a forward and a backward pass of its own, while the current stream frees and allocates tensors of the sizes that
    the calls take: neither stream's scratch or results are the other's or the current stream's, nor what the current stream still reads."""
    rng = np.random.default_rng(21)
    rows, n_in, n_out = 700, 333, 520                             # dz, a copy of x, column sums and parts are scratch
    data = [(dev(rng.standard_normal((rows, n_in)), dt), pack(rng.standard_normal((n_out, n_in)) / 18, dt), dev(rng.standard_normal((rows, n_out)), dt)) for _ in range(2)]
    d = sol.Dropout(0.1, 8)

    def run(k, **kw):
        x, w, g = data[k]
        y, z = sol.sol_linear_fused(x, w, n_out, act=sol.ACT_GELU, drop=d, want_preact=True, **kw)
        return (y, z) + sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_GELU, drop=d, **kw) + (sol.sol_dropout(g, d, **kw),)

    want = [run(0), run(1)]
    big = torch.randn((4096, 4096), device="cuda:0")

    def wait_a_while():                                           # milliseconds of the current stream
        for _ in range(4):
            big @ big

    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        read = torch.randn((rows, n_out), device="cuda:0").to(TDT[dt])
        copy = read.clone()
        torch.cuda.synchronize()
        for st in streams:
            with torch.cuda.stream(st):
                wait_a_while()
        wait_a_while()
        late = read + 0                                           # the current stream reads it behind that, but its memory is free at once
        del read
        got = [run(k, stream=streams[k]) for k in range(2)]
        sizes = (rows * n_out, rows * n_out // 2, n_out * n_in, n_out * n_in // 2, rows * 512, rows * 192, rows * n_in, n_out, 1 << 20, 1 << 22)
        junk = [torch.full((n,), float("nan"), device="cuda:0") for n in sizes for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(late, copy)
        assert all(torch.equal(a, b) for k in range(2) for a, b in zip(got[k], want[k]))
        del junk, got, late


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_captured_and_replayed(sol, dt):
    """A captured training step of the block; the step word changes between the replays, and so do the masks."""
    a = block_inputs(dt, 130, 72, 288, seed=5)
    x, w1, w2, g = dev(a["x"], dt), pack(a["w1"], dt), pack(a["w2"], dt), dev(a["g"], dt)
    b1, b2 = dev(a["b1"][None])[0], dev(a["b2"][None])[0]
    step = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    d1, d2 = sol.Dropout(0.1, 5, 0, step), sol.Dropout(0.2, 5, 1, step)

    def run():
        y, h, z = block_forward(sol, x, w1, b1, w2, b2, 288, d1, d2)
        return (y,) + block_backward(sol, g, x, h, z, w1, w2, d1, d2)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    last = None
    for i in (0, 3, 3, 9):
        step.fill_(i)
        want = [t.clone() for t in run()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, out)), i
        assert last is None or torch.equal(last[1], want[0]) == (last[0] == i)
        last = (i, want[0])


def test_captured_on_a_second_stream(sol):
    """Two branches of one graph, the second on a stream given to the calls, both with scratch of their own; replayed with other work between."""
    rng = np.random.default_rng(31)
    data = [(dev(rng.standard_normal((260, 333)), "bf16"), pack(rng.standard_normal((520, 333)) / 18, "bf16"), dev(rng.standard_normal((260, 520)), "bf16")) for _ in range(2)]
    step = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    d = sol.Dropout(0.1, 8, 0, step)

    def run(k, **kw):
        x, w, g = data[k]
        y, z = sol.sol_linear_fused(x, w, 520, act=sol.ACT_GELU, drop=d, want_preact=True, **kw)
        return (y, z) + sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_GELU, drop=d, **kw) + (sol.sol_dropout(g, d, **kw),)

    run(0), run(1)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = [run(0), run(1, stream=side)]
        torch.cuda.current_stream().wait_stream(side)
    for i in (0, 2, 2, 7):
        step.fill_(i)
        want = [[t.clone() for t in run(k)] for k in range(2)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for k in range(2) for a, b in zip(out[k], want[k])), i


def test_no_rows(sol):
    x = torch.empty((0, 24), device="cuda:0")
    w = pack(np.ones((16, 24)), "f32")
    y, z = sol.sol_linear_fused(x, w, 16, want_preact=True)
    assert y.shape == (0, 16) and z.shape == (0, 16)
    dx, dw, db = sol.sol_linear_backward(torch.empty((0, 16), device="cuda:0"), x, w)
    assert dx.shape == (0, 24) and not dw.any() and not db.any()
    assert sol.sol_dropout(torch.empty((0, 16), device="cuda:0"), sol.Dropout(0.5, 1)).shape == (0, 16)


def test_expanded_rows_are_refused(sol):
    """Rows that lie on each other have no pitch."""
    x, w, row = torch.zeros((4, 32), device="cuda:0"), pack(np.ones((8, 32)), "f32"), torch.zeros((1, 8), device="cuda:0")
    bad = [lambda: sol.sol_linear_fused(x[:1].expand(4, 32), w, 8), lambda: sol.sol_linear_fused(x, w, 8, residual=row.expand(4, 8)), lambda: sol.sol_linear_fused(x, w, 8, out=row.expand(4, 8)),
           lambda: sol.sol_linear_backward(row.expand(4, 8), x, w), lambda: sol.sol_linear_fused(x.as_strided((4, 32), (16, 1)), w, 8)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was not refused")


@pytest.mark.parametrize("dt,pitch", [("bf16", 30000), ("f32", 30000), ("bf16", 30002)])
def test_rows_that_span_more_than_4_gb(sol, dt, pitch):
    """Views of one wide tensor (4.2 and 8.4 GB) give the bits that dense tensors give; 30002: x and dy are copied to aligned rows."""
    rows, n_in, n_out = 70000, 72, 264
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda:0").to(TDT[dt])  # noqa: E731
    wide = torch.full((rows, pitch), float("nan"), dtype=TDT[dt], device="cuda:0")
    x, g, r, out = (wide[:, at:at + n] for at, n in ((0, n_in), (1024, n_out), (4096, n_out), (8192, n_out)))
    for t in (x, g, r):
        t.copy_(rnd(rows, t.shape[1]))
    w, d = rnd(n_out, 128 if dt == "bf16" else 96), sol.Dropout(0.25, 77, 2)
    w[:, n_in:] = 0
    for act in (sol.ACT_NONE, sol.ACT_SILU):
        y, z = sol.sol_linear_fused(x, w, n_out, act=act, drop=d, residual=r, want_preact=True, out=out)
        yd, zd = sol.sol_linear_fused(x.contiguous(), w, n_out, act=act, drop=d, residual=r.contiguous(), want_preact=True)
        assert torch.equal(y, yd) and torch.equal(z, zd)
        drop = None if act == sol.ACT_NONE else d                # without either, dy itself is what the products read
        got = sol.sol_linear_backward(g, x, w, preact=z, act=act, drop=drop, need_db=act != sol.ACT_NONE)
        want = sol.sol_linear_backward(g.contiguous(), x.contiguous(), w, preact=z, act=act, drop=drop, need_db=act != sol.ACT_NONE)
        assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(got, want))
    assert torch.isnan(wide[:, n_in:1024]).all() and torch.isnan(wide[:, 8192 + n_out:]).all()


def test_as_many_rows_as_are_copied(sol):
    """The largest copy of x that is not refused (68.7 GB): every row of y, and dW, whose copy runs beside dz.  Whole numbers, so equal to the last bit."""
    rows = (1 << 29) - (1 << 18)
    if torch.cuda.mem_get_info()[0] < 170e9:
        pytest.skip("needs 170 GB of free memory")
    gen = torch.Generator(device="cuda:0").manual_seed(9)
    x = torch.empty((rows, 3), dtype=torch.bfloat16, device="cuda:0")
    for part in x.split(1 << 26):
        part.copy_(torch.randint(-1, 2, part.shape, generator=gen, device="cuda:0", dtype=torch.int8))
    w = pack(np.array([[1, 2, -3]]), "bf16")
    y, _ = sol.sol_linear_fused(x, w, 1)
    assert all(torch.equal(b[:, 0], a[:, 0] + 2 * a[:, 1] - 3 * a[:, 2]) for a, b in zip(x.split(1 << 26), y.split(1 << 26)))
    g = torch.randint(-1, 2, (rows, 1), generator=gen, device="cuda:0", dtype=torch.int8).bfloat16()      # independent of x: sums of some ten thousand, exact in any order
    _, dw, _ = sol.sol_linear_backward(g, x, w, need_dx=False, need_db=False, dw_dtype=torch.float32)
    assert torch.equal(dw[0].double(), sum((b.double() * a.double()).sum(0) for a, b in zip(x.split(1 << 26), g.split(1 << 26))))
    del x, y, g, dw
    torch.cuda.empty_cache()


def test_large_tiles_at_the_end_of_32_bit_offsets(sol):
    """dW over rows whose last lies 4.28 GB behind the first: whole numbers, so equal to the last bit to that of dense rows."""
    rows, n, pitch = 21400, 4096, 100000
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    ints = lambda: torch.randint(-1, 2, (rows, n), generator=gen, device="cuda:0").bfloat16()  # noqa: E731
    x = torch.full((rows, pitch), float("nan"), dtype=torch.bfloat16, device="cuda:0")[:, :n]
    x.copy_(ints())
    g, w = ints(), torch.zeros((n, n), dtype=torch.bfloat16, device="cuda:0")
    kw = dict(need_dx=False, need_db=False, dw_dtype=torch.float32)
    _, dw, _ = sol.sol_linear_backward(g, x, w, **kw)
    assert torch.equal(dw, sol.sol_linear_backward(g, x.contiguous(), w, **kw)[1])
    want = g[:, :64].float().t() @ x[:, :64].float()
    assert torch.equal(dw[:64, :64], want)


def test_two_streams_at_once_and_graphs_that_share_a_workspace(sol):
    """Layers of two sizes: run on two streams together, with a workspace each; captured into two graphs with one workspace, replayed in turn."""
    rng = np.random.default_rng(12)
    layers = []
    for rows, n_in, n_out in ((300, 130, 700), (41, 900, 260)):
        layers.append([dev(rng.standard_normal((rows, n_in)), "bf16", 3), pack(rng.standard_normal((n_out, n_in)) / 30, "bf16"), dev(rng.standard_normal((rows, n_out)), "bf16"), n_out])
    d = sol.Dropout(0.1, 4, 1)

    def run(k, **kw):
        x, w, g, n_out = layers[k]
        y, z = sol.sol_linear_fused(x, w, n_out, act=sol.ACT_GELU, drop=d, want_preact=True, **kw)
        return (y, z) + sol.sol_linear_backward(g, x, w, preact=z, act=sol.ACT_GELU, drop=d, **kw)

    want = [run(0), run(1)]
    torch.cuda.synchronize()
    spaces = [torch.empty(1 << 22, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    kept = [[] for _ in range(2)]
    for _ in range(4):
        for k in range(2):
            with torch.cuda.stream(streams[k]):                  # the results belong to the stream that writes them
                kept[k].append(run(k, workspace=spaces[k]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in range(2) for got in kept[k] for a, b in zip(got, want[k]))

    graphs, outs = [], []
    for k in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            outs.append(run(k, workspace=spaces[0]))
    for i in range(3):
        layers[i % 2][0].mul_(-1)
        want = [[t.clone() for t in run(k)] for k in range(2)]
        for k in (0, 1):
            graphs[k].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for k in range(2) for a, b in zip(outs[k], want[k])), i


def test_sizes_that_a_c_int_does_not_hold_are_refused(sol):
    """2^32 + 8 rows, whose low 32 bits are 8."""
    x = torch.empty((2**32 + 8, 1), dtype=torch.bfloat16, device="cuda:0")
    w = pack(np.ones((1, 1)), "bf16")
    for f in (lambda: sol.sol_dropout(x, sol.Dropout(0.5, 1), out=x), lambda: sol.sol_dropout(x.view(8, -1), sol.Dropout(0.5, 1), out=x.view(8, -1)),
              lambda: sol.sol_linear_fused(x, w, 1, out=x), lambda: sol.sol_linear_backward(x, x, w)):
        with pytest.raises(sol.SolError) as e:
            f()
        assert e.value.status == 6
    del x
    torch.cuda.empty_cache()


def test_refusals_of_the_binding(sol):
    x, w = torch.zeros((4, 32), device="cuda:0"), pack(np.ones((8, 32)), "f32")
    bad = [lambda: sol.sol_linear_fused(x.t(), w, 8), lambda: sol.sol_linear_fused(x.double(), w, 8), lambda: sol.sol_linear_fused(x, w[:7], 8),
           lambda: sol.sol_linear_fused(x, w, 8, bias=torch.zeros(7, device="cuda:0")), lambda: sol.sol_linear_fused(x, w, 8, bias=torch.zeros(8, device="cuda:0", dtype=torch.bfloat16)),
           lambda: sol.sol_linear_fused(x, w, 8, residual=torch.zeros((3, 8), device="cuda:0")), lambda: sol.sol_linear_fused(x, w, 8, out=torch.zeros((4, 8), device="cuda:0", dtype=torch.bfloat16)),
           lambda: sol.sol_linear_backward(torch.zeros((5, 8), device="cuda:0"), x, w), lambda: sol.sol_linear_backward(torch.zeros((4, 8), device="cuda:0"), x, w, dw_dtype=torch.float16),
           lambda: sol.sol_linear_backward(torch.zeros((4, 8), device="cuda:0"), x, w, preact=torch.zeros((4, 9), device="cuda:0")),
           lambda: sol.sol_dropout(x.t(), sol.Dropout(0.5, 1)), lambda: sol.sol_dropout(x, sol.Dropout(0.5, 1), residual=torch.zeros(4, device="cuda:0")),
           lambda: sol.sol_dropout(x.half(), sol.Dropout(0.5, 1))]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was not refused")
    with pytest.raises(sol.SolError) as e:
        sol.sol_linear_backward(torch.zeros((4, 8), device="cuda:0"), x, w, act=sol.ACT_GELU)     # no preact
    assert e.value.status == 1
