"""The root-mean-square norm and the gated layer against their plain statements in 64 bits (gated_plain.py)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import gated_plain as plain  # noqa: E402
import ops_plain  # noqa: E402
import paper_2105_13336_amd as P  # noqa: E402
from ops_plain import CAP, FLOOR, ROUND, U  # noqa: E402

T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TYPES = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def ops():
    h = P.tensile_ops_create()
    yield h
    h.close()


def say(msg):
    print(msg, flush=True)


def host(t):
    return t.detach().cpu().double().numpy()


def up(a, dtype="f32", odd=False):
    """a on the GPU in the given type; odd: rows at odd places, NaN between, before and behind them."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).to(T[dtype])
    if not odd:
        return t.cuda()
    rows, cols = t.shape
    buf = torch.full((1 + rows * (cols + 3) + 8,), float("nan"), dtype=T[dtype], device="cuda")
    v = buf[1:].as_strided((rows, cols), (cols + 3, 1))
    v.copy_(t)
    return v


def room(rows, cols, dtype, odd=False):
    return up(np.full((rows, cols), 7.0), dtype, odd)


def untouched(t):
    """Whether what lies between the rows of an odd tensor is still NaN."""
    rows, cols = t.shape
    return rows < 2 or bool(t.as_strided((rows - 1, 3), (cols + 3, 1), t.storage_offset() + cols).isnan().all())


def ckpt(rows, cols, odd=False):
    if not odd:
        return P.Checkpoint.empty(rows, cols)
    groups = (cols + 31) // 32
    q = torch.full((3 + rows * (cols + 5) + 8,), 99, dtype=torch.int8, device="cuda")
    s = torch.full((3 + rows * (groups + 2) + 8,), 99, dtype=torch.uint8, device="cuda")
    return P.Checkpoint(q[3:].as_strided((rows, cols), (cols + 5, 1)), s[3:].as_strided((rows, groups), (groups + 2, 1)))


def ckpt_untouched(c):
    rows, cols = c.q.shape
    groups = c.scale.shape[1]
    if rows < 2:
        return True
    return bool((c.q.as_strided((rows - 1, 5), (cols + 5, 1), c.q.storage_offset() + cols) == 99).all()) and \
        bool((c.scale.as_strided((rows - 1, 2), (groups + 2, 1), c.scale.storage_offset() + groups) == 99).all())


def filled(values, cap=248, odd=False):
    """A checkpoint of the values (64 bits), made on the host; -> (checkpoint, what it holds)"""
    q, code = ops_plain.pack(values, cap)
    c = ckpt(*values.shape, odd)
    c.q.copy_(torch.from_numpy(q))
    c.scale.copy_(torch.from_numpy(code))
    return c, ops_plain.unpack(q, code)


def near(got, want, bound, label):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, label
    bad = ~(np.abs(got - want) <= bound)
    bad &= ~(np.isnan(got) & np.isnan(want))
    if bad.any():
        k = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {bad.sum()} of {bad.size} off, first at {k}: {got[k]} for {want[k]}, bound {np.broadcast_to(bound, want.shape)[k]}")


def holds(c, want, e, dtype, label):
    """The checkpoint holds what is within e of want: its scales are those of such values, and so are its values, to half a scale."""
    code = c.scale.cpu().numpy().astype(np.int64)
    cols = want.shape[1]
    a, spread = np.abs(ops_plain.groups_of(want)).max(axis=2), np.abs(ops_plain.groups_of(e)).max(axis=2)
    assert (code >= ops_plain.code_of(np.maximum(a - spread, 0), CAP[dtype])).all() and (code <= ops_plain.code_of(a + spread, CAP[dtype])).all(), label + " codes"
    value = ops_plain.unpack(c.q.cpu().numpy(), code.astype(np.uint8))
    near(value, want, 0.5 * np.repeat(np.exp2(code - 127.0), 32, axis=1)[:, :cols] + e, label)


def activations(rng, rows, cols):
    return rng.standard_normal((rows, cols)) * np.where(rng.random(cols) < 0.05, 6.0, 1.0)


# ------------------------------------------------------------------ root-mean-square norm

COLS = [1, 2, 8, 33, 64, 100, 128, 129, 500, 512, 513, 768, 1024, 1025, 2048, 2049, 4096, 4100, 8192, 8199, 16384, 16385, 40_003]
PAIRS = [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]


def check_norm(ops, dtype, param, rows, cols, residual=True, total=True, keep=True, eps=1e-6, odd=False, x=None):
    rng = np.random.default_rng(rows * 31 + cols)
    xd = up(activations(rng, rows, cols) + 0.3 if x is None else x, dtype, odd)
    rd = up(activations(rng, rows, cols), dtype, odd) if residual else None
    gamma = up(1 + 0.2 * rng.standard_normal(cols), param)
    y, rstd = room(rows, cols, dtype, odd), torch.empty(rows, device="cuda")
    tot = room(rows, cols, dtype, odd) if total else None
    c = ckpt(rows, cols, odd) if keep else None
    P.tensile_rms_norm(ops, xd, gamma, y, eps=eps, residual=rd, total=tot, xhat=c, rstd=rstd)
    s = host(xd) + (host(rd) if residual else 0)
    y0, xh0, rstd0 = plain.rms_norm(s, host(gamma), eps)
    label = f"{dtype}/{param} {rows}x{cols}"
    # s is rounded (2 units of a square), a square passes through at most 8 * 2 additions in a lane (8 * 5 in a row above 16384), 6 across lanes and 16
    # across wavefronts, then a division, a sum, a root and a reciprocal: half of it in the reciprocal of the root
    unit = ((72 if cols > 16_384 else 48) / 2 + 4) * U
    near(rstd, rstd0, unit * rstd0, label + " rstd")
    e = (unit + 2 * U) * np.abs(xh0) + (U * np.abs(s) * rstd0[:, None] if residual else 0)
    near(y, y0, ROUND[dtype] * np.abs(y0) + FLOOR[dtype] + (1.01 * e + 2 * U * np.abs(xh0)) * np.abs(host(gamma)), label + " y")
    if total:
        near(tot, s, 1.01 * (ROUND[dtype] + U) * np.abs(s) + FLOOR[dtype], label + " total")
    if keep:
        holds(c, xh0, e, dtype, label + " xhat")
    if odd:
        assert untouched(y) and (tot is None or untouched(tot)) and (c is None or ckpt_untouched(c)), label


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,param", PAIRS)
def test_rms_norm(ops, dtype, param, cols):
    say(f"rms norm {dtype} {cols}")
    for rows in (1, 5, 70):
        check_norm(ops, dtype, param, rows, cols)


@pytest.mark.parametrize("dtype,param", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
def test_rms_norm_parts_and_places(ops, dtype, param):
    check_norm(ops, dtype, param, 9, 768, residual=False, total=False, keep=False)
    check_norm(ops, dtype, param, 9, 100, residual=False, total=False)
    check_norm(ops, dtype, param, 9, 768, total=False, keep=False)
    check_norm(ops, dtype, param, 6, 16_500, residual=False)
    for cols in (7, 100, 768, 1500, 5000, 9001, 17_001):
        check_norm(ops, dtype, param, 11, cols, odd=True)


def test_rms_norm_of_many_rows(ops):
    """More rows than teams: every team goes on to further rows."""
    for cols in (16, 128, 300, 768, 2000, 3000, 6000, 12_000):
        check_norm(ops, "bf16", "f32", 40_000 if cols <= 128 else 4_007, cols)
    check_norm(ops, "f32", "f32", 1500, 17_000)


def test_rms_norm_of_zero_small_and_non_finite_rows(ops):
    cols = 776
    x = np.random.default_rng(1).standard_normal((6, cols))
    x[1] = 0.0
    x[2, 700] = np.nan
    x[3, 5] = np.inf
    x[5] *= 1e-12
    xd, g = up(x, "bf16"), torch.full((cols,), 2.0, device="cuda")
    y, c, rstd = torch.empty_like(xd), P.Checkpoint.empty(6, cols), torch.empty(6, device="cuda")
    P.tensile_rms_norm(ops, xd, g, y, xhat=c, rstd=rstd)
    back = torch.empty_like(xd)
    P.tensile_ckpt_unpack(ops, c, back)
    assert not bool(y[1].any()) and not bool(back[1].any()) and abs(float(rstd[1]) * 1e-3 - 1) < 1e-6
    # a NaN spoils its row; an infinity leaves the row's other values at 0 = finite * (1/inf), and is itself inf * 0
    assert bool(y[2].isnan().all()) and bool(back[2].isnan().all())
    assert bool(y[3, 5].isnan()) and not bool(y[3, 6:].any()) and float(rstd[3]) == 0.0
    assert bool(back[3, :32].isnan().all()) and not bool(back[3, 32:].any())
    assert bool(y[[0, 4, 5]].isfinite().all()) and bool(back[[0, 4, 5]].isfinite().all())
    check_norm(ops, "f32", "f32", 4, 300, x=np.random.default_rng(2).standard_normal((4, 300)) * 1e-12, residual=False, eps=1e-30)
    # eps = 0 on a row of zeros: 0 * inf, as the formula has it, also in the last, partial group; the smallest eps above 0: zeros
    P.tensile_rms_norm(ops, xd, g, y, eps=0.0, xhat=c, rstd=rstd)
    P.tensile_ckpt_unpack(ops, c, back)
    assert bool(y[1].isnan().all()) and bool(back[1].isnan().all()) and bool(y[0].isfinite().all())
    P.tensile_rms_norm(ops, xd, g, y, eps=1e-60)
    assert not bool(y[1].any())


def check_norm_backward(ops, dtype, param, rows, cols, residual=True, params=True, odd=False, in_place=""):
    rng = np.random.default_rng(rows * 17 + cols)
    dy = up(rng.standard_normal((rows, cols)) * 0.1, dtype, odd)
    dr = up(rng.standard_normal((rows, cols)) * 0.1, dtype, odd) if residual else None
    c, xh = filled(activations(rng, rows, cols), CAP[dtype], odd)
    rstd = up(np.exp(rng.standard_normal(rows)))
    gamma = up(1 + 0.2 * rng.standard_normal(cols), param)
    dy0, dr0, g0, rstd0 = host(dy), host(dr) if residual else 0, host(gamma), host(rstd)
    dx = dy if in_place == "dy" else dr if in_place == "dr" else room(rows, cols, dtype, odd)
    dg = torch.full((cols,), 5.0, dtype=T[param], device="cuda") if params else None
    P.tensile_rms_norm_backward(ops, dy, c, rstd, gamma, dx, dg, dresidual=dr)
    want, dg0 = plain.rms_norm_backward(dy0, xh, rstd0, g0)
    t = np.abs(dy0 * g0)
    # the mean: chains of at most 8 * 2 additions in a lane (8 * 5 in a long row), 6 across lanes, 16 across wavefronts
    size = rstd0[:, None] * (t + np.abs(xh) * (t * np.abs(xh)).mean(axis=1, keepdims=True))
    label = f"{dtype}/{param} {rows}x{cols}"
    near(dx, want + dr0, (ROUND[dtype] + U) * np.abs(want + dr0) + FLOOR[dtype] + 80 * U * size + 2 * U * np.abs(dr0), label + " dx")
    if params:
        # rows of a team in turn, teams of a workgroup, partial sums in 32 strands
        length = rows / min(rows, 256) + 16 + 64 + 8
        near(dg, dg0, (ROUND[param] + U) * np.abs(dg0) + FLOOR[param] + length * U * np.abs(dy0 * xh).sum(axis=0), label + " dgamma")
    if odd:
        assert untouched(dx)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,param", PAIRS)
def test_rms_norm_backward(ops, dtype, param, cols):
    say(f"rms norm backward {dtype} {cols}")
    for rows in (1, 5, 70):
        check_norm_backward(ops, dtype, param, rows, cols)


@pytest.mark.parametrize("dtype,param", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
def test_rms_norm_backward_parts_and_places(ops, dtype, param):
    for cols in (7, 100, 768, 1500, 5000, 17_001):
        check_norm_backward(ops, dtype, param, 11, cols, odd=True)
        check_norm_backward(ops, dtype, param, 11, cols, residual=False, params=False)
        check_norm_backward(ops, dtype, param, 300, cols, in_place="dy")
        check_norm_backward(ops, dtype, param, 300, cols, in_place="dr")


def test_rms_norm_backward_of_many_rows(ops):
    for cols in (16, 128, 300, 768, 2000, 3000, 8000):
        check_norm_backward(ops, "bf16", "f32", 40_000 if cols <= 128 else 4_007, cols)


@pytest.mark.parametrize("cols", [64, 512, 800, 4096, 20_000])
def test_rms_norm_backward_against_differences(ops, cols):
    """Rows whose normalised form is held exactly (0, 2 and -2): the gradient is that of the norm itself."""
    rng = np.random.default_rng(cols)
    rows = 4
    xh = np.zeros((rows, cols))
    for r in range(rows):
        xh[r, rng.permutation(cols)[:cols // 4]] = rng.choice([-2.0, 2.0], cols // 4)
    sigma, gamma, dy = np.exp(rng.standard_normal((rows, 1))), 1 + 0.3 * rng.standard_normal(cols), rng.standard_normal((rows, cols))
    s = sigma * xh
    c, held = filled(xh)
    assert np.array_equal(held, xh)
    dx, dg = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda")
    P.tensile_rms_norm_backward(ops, up(dy), c, up(1 / sigma[:, 0]), up(gamma), dx, dg)
    loss = lambda s, g: (dy * plain.rms_norm(s, g, 0.0)[0]).sum()
    step = 1e-5
    for _ in range(4):
        d, e = rng.standard_normal((rows, cols)), rng.standard_normal(cols)
        for got, ds, dgm in ((np.vdot(host(dx), d), d, 0), (np.vdot(host(dg), e), 0, e)):
            diff = (loss(s + step * ds, gamma + step * dgm) - loss(s - step * ds, gamma - step * dgm)) / (2 * step)
            # the differences (step^2, and 2^-52 / step of the loss's magnitude), and 32 bits in each product
            assert abs(got - diff) <= 1e-6 * np.abs(dy).sum() * 4, (cols, got, diff)


def test_rms_norm_in_place_and_without_rows(ops):
    rng = np.random.default_rng(8)
    for cols in (100, 768, 5000, 16_500):
        x, r = up(rng.standard_normal((30, cols)), "bf16"), up(rng.standard_normal((30, cols)), "bf16")
        g = torch.ones(cols, device="cuda")
        y, t = torch.empty_like(x), torch.empty_like(x)
        P.tensile_rms_norm(ops, x, g, y, residual=r, total=t)
        for yi, ti in ((0, 1), (1, 0)):
            both = [x.clone(), r.clone()]
            P.tensile_rms_norm(ops, both[0], g, both[yi], residual=both[1], total=both[ti])
            assert torch.equal(both[yi], y) and torch.equal(both[ti], t)
    none, c, dg = torch.empty(0, 40, device="cuda"), P.Checkpoint.empty(0, 40), torch.full((40,), 7.0, device="cuda")
    P.tensile_rms_norm(ops, none, dg, none, xhat=c, rstd=torch.empty(0, device="cuda"))
    P.tensile_rms_norm_backward(ops, none, c, torch.empty(0, device="cuda"), dg.clone(), none, dg)
    assert not bool(dg.any())


# ------------------------------------------------------------------ the gated layer

SIZES = [(1, 1, 1), (1, 8, 1), (2, 3, 5), (3, 17, 33), (5, 64, 32), (33, 100, 31), (31, 33, 65), (32, 784, 512), (64, 128, 64), (100, 200, 96),
         (129, 257, 130), (300, 96, 700), (257, 1000, 300), (1, 4096, 100), (2, 4097, 70), (8, 31, 1000), (40, 3000, 64), (70, 16, 16)]


def check_gated(ops, dtype, M, K, F, act="silu", bias=None, keep=True, odd=False):
    say(f"gated {dtype} {M}x{K}x{F} {act}")
    rng = np.random.default_rng(M * 7 + K * 3 + F)
    x = up(activations(rng, M, K), dtype, odd)
    wg, wu = (up(rng.standard_normal((F, K)) * K ** -0.5, dtype, odd) for _ in range(2))
    bg, bu = (up(rng.standard_normal(F), bias) for _ in range(2)) if bias else (None, None)
    h = room(M, F, dtype, odd)
    cg, cu = (ckpt(M, F, odd) if keep else None for _ in range(2))
    P.tensile_gated_linear(ops, x, wg, wu, h, b_gate=bg, b_up=bu, act=act, gate=cg, up=cu)
    b0, b1 = (host(bg), host(bu)) if bias else (0.0, 0.0)
    x0, wg0, wu0 = host(x), host(wg), host(wu)
    h0, g0, u0 = plain.gated(x0, wg0, wu0, b0, b1, act)
    n = plain.chain(K, dtype, 64)
    eg, eu = (n * U * (np.abs(x0) @ np.abs(w).T + np.abs(b)) for w, b in ((wg0, b0), (wu0, b1)))
    value = np.abs(plain.activation(g0, act)[0])
    ev = 1.13 * eg + plain.activation_error(g0, act, dtype)[0]
    label = f"{dtype} {M}x{K}x{F} {act}"
    near(h, h0, (ROUND[dtype] + 2 * U) * np.abs(h0) + FLOOR[dtype] + 1.01 * (ev * (np.abs(u0) + eu) + value * eu), label + " h")
    if dtype == "f32" and K >= 16:
        # roundings of a sum's partial sums are independent: n of them, each of up to the whole sum's size, give sqrt(n) units (a factor of 4 is
        # a chance of less than 1e-4), in g and in u, beside those of the activation
        got = host(h)
        assert np.linalg.norm(got - h0) <= 4 * U * (2 * np.sqrt(n) + 16) * np.linalg.norm(np.maximum(np.abs(g0), 1) * np.maximum(np.abs(u0), 1)), label
    if keep:
        holds(cg, g0, eg, dtype, label + " gate")
        holds(cu, u0, eu, dtype, label + " up")
    if odd:
        assert untouched(h) and (not keep or (ckpt_untouched(cg) and ckpt_untouched(cu))), label


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gated(ops, dtype, M, K, F):
    check_gated(ops, dtype, M, K, F)
    check_gated(ops, dtype, M, K, F, act="gelu", bias=dtype, keep=False)
    check_gated(ops, dtype, M, K, F, act="gelu_tanh", bias="f32", odd=True)


@pytest.mark.parametrize("dtype,K", [("bf16", 72), ("bf16", 133), ("f16", 264), ("f32", 100)])
def test_gated_of_many_tokens(ops, dtype, K):
    """Enough large tiles for the whole card, with ragged edges, and with whole ones."""
    check_gated(ops, dtype, 2_100, K, 3_901, odd=True)
    check_gated(ops, dtype, 2_304, K, 3_712, act="gelu", bias="f32")


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_of_few_tokens_and_long_sums(ops, dtype):
    for M in (1, 2, 7, 16, 17, 32, 33, 64, 65):
        check_gated(ops, dtype, M, 2_050, 160, keep=M != 7)
    check_gated(ops, dtype, 1, 9_000, 40, odd=True)
    check_gated(ops, dtype, 16, 20_000, 33)


def test_gated_keeps_what_is_lost_to_itself(ops):
    """A NaN or infinity in a token spoils its row, one in a weight its feature (and the feature's group in the checkpoint)."""
    for dtype, M, K, F in (("bf16", 150, 200, 100), ("f32", 20, 64, 100), ("f16", 2_200, 64, 4_000)):
        rng = np.random.default_rng(5)
        x, wg, wu = rng.standard_normal((M, K)), rng.standard_normal((F, K)), rng.standard_normal((F, K))
        x[3, 7], x[M - 1, K - 1], wg[40, 0], wu[F - 1, K - 1] = np.nan, np.inf, np.inf, np.nan
        h, cg, cu = room(M, F, dtype), ckpt(M, F), ckpt(M, F)
        P.tensile_gated_linear(ops, up(x, dtype), up(wg, dtype), up(wu, dtype), h, gate=cg, up=cu)
        lost = ~np.isfinite(host(h))
        rows, cols = np.isin(np.arange(M), (3, M - 1)), np.isin(np.arange(F), (40, F - 1))
        # (-inf through the activation is NaN, +inf infinite: nothing finite comes of either, but for 0 of a large negative gate)
        assert not lost[~rows][:, ~cols].any() and lost[3].all() and lost[~rows][:, F - 1].all() and lost[~rows][:, 40].all()
        code = cg.scale.cpu().numpy()
        assert (code[3] == 255).all() and (code[~rows][:, 1] == 255).all() and (code[~rows][:, 0] < 255).all()
        assert (cu.scale.cpu().numpy()[~rows][:, -1] == 255).all() and (cu.scale.cpu().numpy()[~rows][:, 0] < 255).all()


def check_gated_backward(ops, dtype, M, K, F, act="silu", keep=True, odd=False, in_place=False, product=True):
    say(f"gated backward {dtype} {M}x{K}x{F} {act}")
    rng = np.random.default_rng(M * 5 + K * 3 + F)
    dh = up(rng.standard_normal((M, F)) * 0.1, dtype, odd)
    (cg, g), (cu, u) = (filled(activations(rng, M, F) * 1.5, CAP[dtype], odd) for _ in range(2))
    wg, wu = (up(rng.standard_normal((F, K)) * F ** -0.5, dtype, odd) if product else None for _ in range(2))
    dx = room(M, K, dtype, odd) if product else None
    dh0 = host(dh)
    dgate = dh if in_place else room(M, F, dtype, odd)
    dup = room(M, F, dtype, odd)
    c = (cu if in_place else ckpt(M, F, odd)) if keep else None
    P.tensile_gated_linear_backward(ops, dh, cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=dx, act=act, h_ckpt=c)
    dg0, du0, h0 = plain.gated_grad(dh0, g, u, act)
    ev, es = plain.activation_error(g, act, dtype)
    label = f"{dtype} {M}x{K}x{F} {act}"
    near(dgate, dg0, (ROUND[dtype] + 3 * U) * np.abs(dg0) + FLOOR[dtype] + es * np.abs(dh0 * u), label + " dgate")
    near(dup, du0, (ROUND[dtype] + 3 * U) * np.abs(du0) + FLOOR[dtype] + ev * np.abs(dh0), label + " dup")
    if product:
        a, b, wg0, wu0 = host(dgate), host(dup), host(wg), host(wu)
        size = np.abs(a) @ np.abs(wg0) + np.abs(b) @ np.abs(wu0)
        want = a @ wg0 + b @ wu0
        n = plain.chain(2 * F, dtype, 64)
        near(dx, want, (ROUND[dtype] + U) * np.abs(want) + FLOOR[dtype] + n * U * size, label + " dx")
        if dtype == "f32" and F >= 16:
            # (as above)
            assert np.linalg.norm(host(dx) - want) <= 4 * U * (np.sqrt(n) + 2) * np.linalg.norm(np.sqrt((a * a) @ (wg0 * wg0) + (b * b) @ (wu0 * wu0))), label
    if keep:
        holds(c, h0, ev * np.abs(u) + 2 * U * np.abs(h0), dtype, label + " h")
    if odd:
        assert untouched(dgate) and untouched(dup) and (not product or untouched(dx)) and (c is None or ckpt_untouched(c)), label


@pytest.mark.parametrize("M,K,F", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gated_backward(ops, dtype, M, K, F):
    check_gated_backward(ops, dtype, M, K, F)
    check_gated_backward(ops, dtype, M, K, F, act="gelu", keep=False, in_place=True)
    check_gated_backward(ops, dtype, M, K, F, act="gelu_tanh", odd=True)
    check_gated_backward(ops, dtype, M, K, F, act="gelu", in_place=True, product=False)


@pytest.mark.parametrize("dtype,F", [("bf16", 40), ("f16", 75), ("f32", 30)])
def test_gated_backward_of_many_tokens(ops, dtype, F):
    check_gated_backward(ops, dtype, 4_100, 3_999, F, odd=True)
    check_gated_backward(ops, dtype, 4_096, 4_096, F)
    check_gated_backward(ops, dtype, 8_190, 767, F)    # (tiles of 192 columns)
    check_gated_backward(ops, dtype, 8_192, 768, F, act="gelu")
    check_gated_backward(ops, dtype, 2_049, 2_100, F)  # (... of 128)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_with_split_sums(ops, dtype):
    """Few tiles and long sums, of which the last step is a part of one, or there is none."""
    for M, K, F in ((40, 1_700, 100), (64, 2_048, 64), (200, 3_001, 130), (3, 8_200, 33), (32, 9_001, 64), (20, 1_700, 40)):
        check_gated(ops, dtype, M, K, F, act="gelu", bias="f32")
        check_gated_backward(ops, dtype, M, F, K, act="gelu")
        check_gated_backward(ops, dtype, M, F, K, odd=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_backward_of_few_tokens_and_long_sums(ops, dtype):
    for M in (1, 2, 16, 33, 65):
        check_gated_backward(ops, dtype, M, 200, 2_050, keep=M != 16)
    check_gated_backward(ops, dtype, 3, 40, 20_000, odd=True)


@pytest.mark.parametrize("act", plain.ACTS)
def test_gated_backward_against_differences(ops, act):
    """Of the layer itself, through its own forward pass's statement, at projections that the checkpoints hold exactly."""
    rng = np.random.default_rng(2)
    M, K, F = 6, 40, 96
    x = rng.integers(-4, 5, (M, K)).astype(float)
    wg, wu = (rng.integers(-1, 2, (F, K)) * (rng.random((F, K)) < 0.2) / 4.0 for _ in range(2))
    _, g, u = plain.gated(x, wg, wu, 0.0, 0.0, act)
    (cg, held_g), (cu, held_u) = filled(g), filled(u)
    assert np.array_equal(held_g, g) and np.array_equal(held_u, u)
    dh = rng.standard_normal((M, F))
    dgate, dup, dx = torch.empty(M, F, device="cuda"), torch.empty(M, F, device="cuda"), torch.empty(M, K, device="cuda")
    P.tensile_gated_linear_backward(ops, up(dh), cg, cu, dgate, dup, w_gate=up(wg), w_up=up(wu), dx=dx, act=act)
    dwg, dwu, zero = torch.empty(F, K, device="cuda"), torch.empty(F, K, device="cuda"), None
    cx, held_x = filled(x)
    assert np.array_equal(held_x, x)
    P.tensile_linear_grad(ops, dgate, cx, dwg, dbias=zero)
    P.tensile_linear_grad(ops, dup, cx, dwu)
    loss = lambda x, wg, wu: (dh * plain.gated(x, wg, wu, 0.0, 0.0, act)[0]).sum()
    step = 1e-5
    for got, which in ((dx, 0), (dwg, 1), (dwu, 2)):
        args = [x, wg, wu]
        d = rng.standard_normal(args[which].shape)
        plus, minus = list(args), list(args)
        plus[which], minus[which] = args[which] + step * d, args[which] - step * d
        diff = (loss(*plus) - loss(*minus)) / (2 * step)
        size = np.abs(dh).sum() * (1 + np.abs(u).max()) * np.abs(d).sum() / d.size ** 0.5
        assert abs(np.vdot(host(got), d) - diff) <= 2e-6 * size, (act, which)


def test_activations_of_extremes(ops):
    """Gates far out: the activation is 0 or the gate itself, its slope 0 or 1, and nothing is NaN."""
    g = np.array([[0.0, 100, -100, 1e30, -1e30, 3e37, -3e37, 1e-30]])
    for act in plain.ACTS:
        for k in range(8):
            c, held = filled(np.repeat(g[:, k:k + 1], 4, axis=1))
            one, _ = filled(np.ones((1, 4)))
            dgate, dup, ch = torch.empty(1, 4, device="cuda"), torch.empty(1, 4, device="cuda"), ckpt(1, 4)
            P.tensile_gated_linear_backward(ops, torch.ones(1, 4, device="cuda"), c, one, dgate, dup, act=act, h_ckpt=ch)
            v = held[0, 0]
            if abs(v) > 50:
                assert bool((dgate == float(v > 0)).all()) and np.array_equal(host(dup), np.maximum(held, 0)), (act, v)
            else:
                near(dgate, np.full((1, 4), 0.5), 1e-6, act)
                near(dup, held / 2, 1e-6 * np.abs(held), act)
            x, w, eye = up([[held[0, 0]]]), up([[1.0]]), up([[1 / held[0, 0]]]) if v else up([[0.0]])
            h = torch.empty(1, 1, device="cuda")
            P.tensile_gated_linear(ops, x, w, eye, h, act=act)       # act(v) * 1
            want = plain.activation(held[:, :1], act)[0] * (host(x) * host(eye))
            near(h, want, 8 * U * np.abs(want) + 1e-30, act)


def test_gated_without_rows(ops):
    x, w = torch.empty(0, 40, device="cuda"), torch.ones(24, 40, device="cuda")
    h, c = torch.empty(0, 24, device="cuda"), P.Checkpoint.empty(0, 24)
    P.tensile_gated_linear(ops, x, w, w, h, gate=c, up=c)
    P.tensile_gated_linear_backward(ops, h, c, c, h, torch.empty(0, 24, device="cuda"), w_gate=w, w_up=w, dx=x)


# ------------------------------------------------------------------ together

def block(ops, o, p, x, dy, c, stream=None):
    """A gated block y = x + gated(norm(x)) Wd^T up to h, and back from dh."""
    P.tensile_rms_norm(ops, x, p["g"], o["n"], xhat=c["n"], rstd=o["rstd"], stream=stream)
    P.tensile_gated_linear(ops, o["n"], p["wg"], p["wu"], o["h"], act="silu", gate=c["g"], up=c["u"], stream=stream)
    P.tensile_gated_linear_backward(ops, dy, c["g"], c["u"], o["both"][:, :p["wg"].shape[0]], o["both"][:, p["wg"].shape[0]:], w_gate=p["wg"], w_up=p["wu"],
                                    dx=o["dn"], h_ckpt=c["h"], stream=stream)
    P.tensile_linear_grad(ops, o["both"], c["n"], o["dw"], gamma=p["g"], beta=p["zero"], stream=stream)
    P.tensile_linear_grad(ops, dy, c["h"], o["dd"], stream=stream)
    P.tensile_rms_norm_backward(ops, o["dn"], c["n"], o["rstd"], p["g"], o["dx"], o["dg"], dresidual=o["dn"], stream=stream)


def setting(M, K, F, seed=0):
    torch.manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda")
    p = {"g": 1 + 0.1 * r(K), "zero": torch.zeros(K, device="cuda"), "wg": (r(F, K) * K ** -0.5).bfloat16(), "wu": (r(F, K) * K ** -0.5).bfloat16()}
    return p, r(M, K).bfloat16(), (0.1 * r(M, F)).bfloat16()


def outputs(M, K, F):
    e = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")
    f = torch.float32
    return {"n": e(M, K), "rstd": e(M, dtype=f), "h": e(M, F), "both": e(M, 2 * F), "dn": e(M, K), "dw": e(2 * F, K, dtype=f), "dd": e(F, F, dtype=f),
            "dx": e(M, K), "dg": e(K, dtype=f)}


def kept(M, K, F):
    return {"n": P.Checkpoint.empty(M, K), "g": P.Checkpoint.empty(M, F), "u": P.Checkpoint.empty(M, F), "h": P.Checkpoint.empty(M, F)}


def test_a_block_against_autograd(ops):
    """The whole block's gradients against autograd in 32 bits: each tensor between is rounded to bf16 (2^-9 rms relative or less), each checkpoint
    to half a scale (1 % rms of a group): a few per cent together, where a wrong formula is off by all of it."""
    M, K, F = 500, 200, 520
    p, x, dy = setting(M, K, F)
    o = outputs(M, K, F)
    block(ops, o, p, x, dy, kept(M, K, F))
    xr = x.float().cpu().requires_grad_()
    g, wg, wu = (p[n].float().cpu().requires_grad_() for n in ("g", "wg", "wu"))
    n = xr * torch.rsqrt(xr.square().mean(1, keepdim=True) + 1e-6) * g
    n.retain_grad()
    h = torch.nn.functional.silu(n @ wg.t()) * (n @ wu.t())
    h.backward(dy.float().cpu())
    assert float((o["h"].float().cpu() - h.detach()).norm() / h.detach().norm()) < 0.01
    far = lambda a, b: float((a.float().cpu() - b).norm() / b.norm())
    assert far(o["dw"][:F], wg.grad) < 0.05 and far(o["dw"][F:], wu.grad) < 0.05 and far(o["dg"], g.grad) < 0.05
    assert far(o["dx"], xr.grad + n.grad) < 0.05 and far(o["dn"], n.grad) < 0.05
    assert far(o["dd"], dy.float().cpu().t() @ h.detach()) < 0.05


@pytest.mark.parametrize("M,K,F", [(3, 200, 640), (600, 256, 640), (2_100, 64, 4_000)])
def test_captured_and_replayed(ops, M, K, F):
    """A graph of the whole block, with eager work between the replays and new inputs for each."""
    p, x, dy = setting(M, K, F)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fixed, c = outputs(M, K, F), kept(M, K, F)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        block(ops, fixed, p, x, dy, c, side)
    for seed in range(1, 5):
        _, x1, dy1 = setting(M, K, F, seed)
        x.copy_(x1)
        dy.copy_(dy1)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in fixed.items()}
        eager = outputs(M, K, F)
        block(ops, eager, p, x, dy, kept(M, K, F))
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(got[n], eager[n]), (seed, n)


def test_two_graphs_and_eager_calls_side_by_side(ops):
    """Graphs of one handle captured on one stream, launched on two, beside eager calls on a third: each has scratch memory of its own."""
    M, K, F = 100, 2_048, 1_024                        # (split sums, forward and backward)
    p, x, dy = setting(M, K, F)
    want = outputs(M, K, F)
    block(ops, want, p, x, dy, kept(M, K, F))
    torch.cuda.synchronize()
    side, runs = torch.cuda.Stream(), []
    for _ in range(2):
        o, c, graph = outputs(M, K, F), kept(M, K, F), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for _ in range(10):
                block(ops, o, p, x, dy, c, side)
        runs.append((o, graph, torch.cuda.Stream(), c))                # (the graph writes to the checkpoints: they have to live)
    eager, c = outputs(M, K, F), kept(M, K, F)
    for _ in range(3):
        for _, graph, stream, _ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        for _ in range(10):
            block(ops, eager, p, x, dy, c)
        torch.cuda.synchronize()
        for o in (runs[0][0], runs[1][0], eager):
            assert all(torch.equal(o[n], want[n]) for n in want)


def test_threads_and_streams_share_a_handle(ops):
    import threading
    jobs = []
    for k, (M, K, F) in enumerate(((100, 2_048, 1_024), (7, 500, 200), (300, 300, 300))):
        p, x, dy = setting(M, K, F, k)
        want = outputs(M, K, F)
        block(ops, want, p, x, dy, kept(M, K, F))
        jobs.append((p, x, dy, want, outputs(M, K, F), kept(M, K, F), torch.cuda.Stream()))
    torch.cuda.synchronize()

    def work(p, x, dy, _, got, c, stream):
        for _ in range(20):
            block(ops, got, p, x, dy, c, stream)
    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for j in jobs:
        assert all(torch.equal(j[3][n], j[4][n]) for n in j[3])


def test_rows_too_far_apart_for_32_bits(ops):
    """Rows 2^23 bytes and more apart."""
    rng = np.random.default_rng(3)
    M, K, F, ld = 5, 40, 33, (1 << 22) + 8
    far = lambda a, dtype: torch.empty(a.shape[0] * ld, dtype=T[dtype], device="cuda").as_strided(a.shape, (ld, 1)).copy_(torch.from_numpy(a))
    x0, wg0, wu0 = rng.standard_normal((M, K)), rng.standard_normal((F, K)), rng.standard_normal((F, K))
    for dtype in ("bf16", "f32"):
        x, wg, wu = far(x0, dtype), far(wg0, dtype), far(wu0, dtype)
        h, want = room(M, F, dtype), room(M, F, dtype)
        P.tensile_gated_linear(ops, x, wg, wu, h)
        P.tensile_gated_linear(ops, x.contiguous(), wg.contiguous(), wu.contiguous(), want)
        # the same products in another order
        near(h, host(want), 4 * ROUND[dtype] * np.abs(host(want)) + 100 * U * 40, dtype)
        (cg, _), (cu, _) = filled(host(want), CAP[dtype]), filled(host(want), CAP[dtype])
        dx, dx0 = room(M, K, dtype), room(M, K, dtype)
        dg, du = room(M, F, dtype), room(M, F, dtype)
        P.tensile_gated_linear_backward(ops, h, cg, cu, dg, du, w_gate=wg, w_up=wu, dx=dx)
        P.tensile_gated_linear_backward(ops, h, cg, cu, dg, du, w_gate=wg.contiguous(), w_up=wu.contiguous(), dx=dx0)
        size = np.abs(host(dg)) @ np.abs(wg0) + np.abs(host(du)) @ np.abs(wu0)
        near(dx, host(dx0), 4 * ROUND[dtype] * np.abs(host(dx0)) + 100 * U * size, dtype)


@pytest.mark.parametrize("M,wide", [(40, 70), (256, 32_768), (130, 49_152)])
def test_tiles_of_rows_too_far_apart_for_32_bits(ops, M, wide):
    """The same with more tokens: few tiles, whose sums are split, and more than the card has places for."""
    rng = np.random.default_rng(M)
    short = 1_600 if wide < 100 else 40
    far = lambda a, ld: torch.empty(a.shape[0] * ld, dtype=torch.bfloat16, device="cuda").as_strided(a.shape, (ld, 1)).copy_(a)
    x, wg, wu = (up(rng.standard_normal(s) * short ** -0.5, "bf16") for s in ((M, short), (wide, short), (wide, short)))
    h, want = room(M, wide, "bf16"), room(M, wide, "bf16")
    P.tensile_gated_linear(ops, far(x, (1 << 22) + 8), wg, wu, h)
    P.tensile_gated_linear(ops, x, wg, wu, want)
    # the same products in another order: to a rounding of each and the sums' own
    off = (h.double() - want.double()).abs()
    assert bool((off <= 4 * ROUND["bf16"] * want.double().abs() + 100 * U * short).all())
    dgate, dup, dx, dx0 = room(M, short, "bf16"), far(room(M, short, "bf16"), (1 << 22) + 8), room(M, wide, "bf16"), room(M, wide, "bf16")
    g, _ = filled(rng.standard_normal((M, short)))
    wg, wu = wg.t().contiguous(), wu.t().contiguous()
    P.tensile_gated_linear_backward(ops, x, g, g, dgate, dup, w_gate=wg, w_up=wu, dx=dx)
    P.tensile_gated_linear_backward(ops, x, g, g, dgate, dup.contiguous(), w_gate=wg, w_up=wu, dx=dx0)
    size = dgate.double().abs() @ wg.double().abs() + dup.double().abs() @ wu.double().abs()
    assert bool(((dx.double() - dx0.double()).abs() <= 4 * ROUND["bf16"] * dx0.double().abs() + 100 * U * size).all())


def test_gated_backward_keeps_a_lost_group_to_itself(ops):
    """A NaN group of gate or up spoils its own columns of dgate and dup (up: of dgate), its row of dx, and nothing else - also at the end of a row."""
    M, K, F = 70, 50, 72
    rng = np.random.default_rng(3)
    g, u = rng.standard_normal((M, F)), rng.standard_normal((M, F))
    g[4, 70], u[9, 3] = np.inf, np.nan
    (cg, _), (cu, _) = filled(g), filled(u)
    w = torch.ones(F, K, device="cuda")
    dgate, dup, dx, c = room(M, F, "f32"), room(M, F, "f32"), room(M, K, "f32"), ckpt(M, F)
    P.tensile_gated_linear_backward(ops, torch.ones(M, F, device="cuda"), cg, cu, dgate, dup, w_gate=w, w_up=w, dx=dx, h_ckpt=c)
    where = lambda *cells: np.array([[any(r == a and b <= k < e for a, b, e in cells) for k in range(F)] for r in range(M)])
    assert np.array_equal(np.isnan(host(dgate)), where((4, 64, 72), (9, 0, 32)))
    assert np.array_equal(np.isnan(host(dup)), where((4, 64, 72)))
    assert np.array_equal(np.isnan(host(dx)).any(1), np.isin(np.arange(M), (4, 9))) and bool(dx[[4, 9]].isnan().all())
    code = c.scale.cpu().numpy()
    assert code[4].tolist()[2] == 255 and code[9].tolist()[0] == 255 and (code == 255).sum() == 2


def test_refused_allocation_is_an_error_and_the_next_call_works(tuning):
    h = P.tensile_ops_create()
    p, x, dy = setting(100, 2_048, 1_024)
    o, c = outputs(100, 2_048, 1_024), kept(100, 2_048, 1_024)
    tuning("alloc_fail", 1)
    with pytest.raises(P.TensileError) as e:
        P.tensile_gated_linear(h, x, p["wg"], p["wu"], o["h"])
    assert e.value.code == P.binding.TENSILE_E_NOMEM
    block(h, o, p, x, dy, c)
    torch.cuda.synchronize()
    assert bool(o["dx"].isfinite().all())
    h.close()


def test_refusals(ops):
    f = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")
    x, g, c, rstd = f(4, 64), f(64, dtype=torch.float32), P.Checkpoint.empty(4, 64), f(4, dtype=torch.float32)

    def refused(call, word, code=P.binding.TENSILE_E_INVAL):
        with pytest.raises(P.TensileError) as e:
            call()
        assert e.value.code == code and word in str(e.value), str(e.value)

    norm, norm_b = P.tensile_rms_norm, P.tensile_rms_norm_backward
    refused(lambda: norm(ops, x.cpu(), g, x), "x")
    refused(lambda: norm(ops, None, g, x), "x")
    refused(lambda: norm(ops, x, None, x), "gamma")
    refused(lambda: norm(ops, x, g, None), "NULL")
    refused(lambda: norm(ops, x, g, f(4, 64, dtype=torch.float16)), "y")
    refused(lambda: norm(ops, x, g, x, eps=-1.0), "eps")
    refused(lambda: norm(ops, x, g, x, eps=float("nan")), "eps")
    refused(lambda: norm(ops, x, g, x, eps=1e39), "eps")
    refused(lambda: norm(ops, x, g[:63], x), "gamma")
    refused(lambda: norm(ops, x, g.half(), x), "param_type")
    refused(lambda: norm(ops, x, g, x, residual=x.clone(), total=x), "total")
    refused(lambda: norm(ops, x, g, x, residual=f(4, 63)), "residual")
    refused(lambda: norm(ops, x, g, x, xhat=P.Checkpoint.empty(4, 63)), "xhat")
    refused(lambda: norm(ops, x, g, x, rstd=f(3, dtype=torch.float32)), "rstd")
    refused(lambda: norm_b(ops, x, c, None, g, x), "rstd")
    refused(lambda: norm_b(ops, x, None, rstd, g, x), "NULL")
    refused(lambda: norm_b(ops, x, P.Checkpoint.empty(4, 65), rstd, g, x), "xhat")
    refused(lambda: norm_b(ops, x, c, rstd, g, x, dgamma=g[:60]), "dgamma")
    gated, back = P.tensile_gated_linear, P.tensile_gated_linear_backward
    w, h, ch = f(32, 64), f(4, 32), P.Checkpoint.empty(4, 32)
    refused(lambda: gated(ops, None, w, w, h), "x")
    refused(lambda: gated(ops, x, None, w, h), "w_gate")
    refused(lambda: gated(ops, x, w, None, h), "w_up")
    refused(lambda: gated(ops, x, w, f(31, 64), h), "w_up")
    refused(lambda: gated(ops, x, f(32, 63), f(32, 63), h), "w_gate")
    refused(lambda: gated(ops, x, w.half(), w.half(), h), "w_gate")
    refused(lambda: gated(ops, x, f(0, 64), f(0, 64), f(4, 1)), "w_gate")
    refused(lambda: gated(ops, x, w.t().contiguous().t(), w, h), "contiguous")
    refused(lambda: gated(ops, x, w, w, f(4, 33)), "h")
    refused(lambda: gated(ops, x, w, w, f(4, 32, dtype=torch.float32)), "h")
    refused(lambda: gated(ops, x, w, w, h, b_gate=f(32)), "b_gate")
    refused(lambda: gated(ops, x, w, w, h, b_up=f(32)), "b_up")
    refused(lambda: gated(ops, x, w, w, h, b_gate=f(32).half(), b_up=f(32).half()), "param_type")
    refused(lambda: gated(ops, x, w, w, h, act="relu"), "relu")
    refused(lambda: gated(ops, x, w, w, h, gate=P.Checkpoint.empty(4, 31)), "gate")
    refused(lambda: gated(ops, x, w, w, h, up=P.Checkpoint.empty(3, 32)), "up")
    refused(lambda: gated(ops, x, w, w, h, gate=ch, up=ch), "up is gate")
    refused(lambda: back(ops, None, ch, ch, h, h), "dh")
    refused(lambda: back(ops, h, None, ch, h, f(4, 32)), "gate")
    refused(lambda: back(ops, h, ch, P.Checkpoint.empty(4, 31), h, f(4, 32)), "up")
    refused(lambda: back(ops, h, ch, ch, h, h), "dup")
    refused(lambda: back(ops, h, ch, ch, f(4, 33), h), "dgate")
    refused(lambda: back(ops, h, ch, ch, h, f(4, 32), w_gate=w, w_up=w), "dx")
    refused(lambda: back(ops, h, ch, ch, h, f(4, 32), dx=x), "dx")
    refused(lambda: back(ops, h, ch, ch, h, f(4, 32), w_gate=f(31, 64), w_up=f(31, 64), dx=x), "w_gate")
    refused(lambda: back(ops, h, ch, ch, h, f(4, 32), w_gate=w, w_up=w, dx=f(4, 63)), "dx")
    refused(lambda: back(ops, h, ch, ch, h, f(4, 32), act="tanh"), "tanh")
    closed = P.tensile_ops_create()
    closed.close()
    refused(lambda: gated(closed, x, w, w, h), "freed")


def test_results_in_the_place_of_what_is_read(ops):
    """h over x, or dx over dgate or dup, of one size: other workgroups still read those, so the calls are refused; dx over dh is no such case."""
    M, n = 70, 96
    rng = np.random.default_rng(8)
    x, wg, wu = up(rng.standard_normal((M, n)), "bf16"), up(rng.standard_normal((n, n)) / 8, "bf16"), up(rng.standard_normal((n, n)) / 8, "bf16")
    x0 = x.clone()
    for h, word in ((x, "h is x"), (wg[:M], "h is x or a weight"), (wu[:M], "h is x or a weight")):
        with pytest.raises(P.TensileError) as e:
            P.tensile_gated_linear(ops, x, wg, wu, h)
        assert e.value.code == P.binding.TENSILE_E_INVAL and word in str(e.value)
    h, cg, cu = torch.empty_like(x), ckpt(M, n), ckpt(M, n)
    P.tensile_gated_linear(ops, x, wg, wu, h, gate=cg, up=cu)
    dh = up(rng.standard_normal((M, n)), "bf16")
    dgate, dup, dx = (torch.empty_like(x) for _ in range(3))
    P.tensile_gated_linear_backward(ops, dh, cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=dx)
    for into in (dgate, dup, wg[:M], wu[:M]):
        with pytest.raises(P.TensileError) as e:
            P.tensile_gated_linear_backward(ops, dh, cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=into)
        assert e.value.code == P.binding.TENSILE_E_INVAL and "dx is dgate" in str(e.value)
    with pytest.raises(P.TensileError):
        P.tensile_gated_linear_backward(ops, dh, cg, cu, dh, dup, w_gate=wg, w_up=wu, dx=dh)
    P.tensile_gated_linear_backward(ops, dh, cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=dh)
    assert torch.equal(x, x0) and torch.equal(dh, dx)


@pytest.mark.parametrize("dtype", TYPES)
def test_more_tiles_than_a_launch_takes(ops, dtype):
    """Over 2,048 tiles in a direction are several launches: of 32 and of 64 features, of 64 columns backward, and of 128 tokens."""
    check_gated(ops, dtype, 2, 24, 70_001, act="gelu", bias="f32", odd=True)
    check_gated(ops, dtype, 40, 16, 140_003, bias="f32", odd=True)
    check_gated_backward(ops, dtype, 3, 140_003, 24, odd=True)
    check_gated_backward(ops, dtype, 33, 270_000, 16)
    check_gated(ops, dtype, 270_001, 8, 9, act="gelu_tanh", bias=dtype, odd=True)
    check_gated_backward(ops, dtype, 270_001, 8, 9, odd=True)


def test_offsets_beyond_32_bits(ops):
    """1,050,000 tokens of 2,056 columns: elements and bytes, of matrices and of checkpoints, beyond 2^31.  First, last and middle rows against 64 bits."""
    M, n, dtype = 1_050_000, 2_056, "bf16"
    rng = np.random.default_rng(9)
    torch.manual_seed(9)
    x = torch.randn(M, n, device="cuda", dtype=torch.bfloat16)
    gamma = up(1 + 0.2 * rng.standard_normal(n))
    wg, wu = (up(rng.standard_normal((n, n)) * n ** -0.5, dtype) for _ in range(2))
    y, h, xhat, cg, cu, ch, rstd = torch.empty_like(x), torch.empty_like(x), ckpt(M, n), ckpt(M, n), ckpt(M, n), ckpt(M, n), torch.empty(M, device="cuda")
    P.tensile_rms_norm(ops, x, gamma, y, xhat=xhat, rstd=rstd)
    P.tensile_gated_linear(ops, y, wg, wu, h, gate=cg, up=cu)
    dgate, dup, dx, ds, dgamma = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma)
    P.tensile_gated_linear_backward(ops, x, cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=dx, h_ckpt=ch)
    P.tensile_rms_norm_backward(ops, dx, xhat, rstd, gamma, ds, dgamma, dresidual=x)
    wg0, wu0, gamma0 = host(wg), host(wu), host(gamma)
    chain, chain2 = plain.chain(n, dtype, 64), plain.chain(2 * n, dtype, 64)
    for first in (0, 1_044_400, M - 40):         # (row 1,044,496 is where 2^31 elements end)
        at = slice(first, first + 100)
        part = lambda c: P.Checkpoint(c.q[at], c.scale[at])
        held = lambda c: ops_plain.unpack(c.q[at].cpu().numpy(), c.scale[at].cpu().numpy())
        y0, xh0, rstd0 = plain.rms_norm(host(x[at]), gamma0, 1e-6)
        unit = (48 / 2 + 4) * U
        near(y[at], y0, ROUND[dtype] * np.abs(y0) + (1.01 * unit + 4 * U) * np.abs(xh0 * gamma0), "y")
        holds(part(xhat), xh0, (unit + 2 * U) * np.abs(xh0), dtype, "xhat")
        h0, g0, u0 = plain.gated(host(y[at]), wg0, wu0, 0.0, 0.0, "silu")
        eg, eu = (chain * U * (np.abs(host(y[at])) @ np.abs(w).T) for w in (wg0, wu0))
        holds(part(cg), g0, eg, dtype, "gate")
        holds(part(cu), u0, eu, dtype, "up")
        value, error = np.abs(plain.activation(g0, "silu")[0]), 1.13 * eg + plain.activation_error(g0, "silu", dtype)[0]
        near(h[at], h0, (ROUND[dtype] + 2 * U) * np.abs(h0) + FLOOR[dtype] + 1.01 * (error * (np.abs(u0) + eu) + value * eu), "h")
        g, u, d = held(cg), held(cu), host(x[at])
        dg0, du0, again = plain.gated_grad(d, g, u, "silu")
        ev, es = plain.activation_error(g, "silu", dtype)
        near(dgate[at], dg0, (ROUND[dtype] + 3 * U) * np.abs(dg0) + FLOOR[dtype] + es * np.abs(d * u), "dgate")
        near(dup[at], du0, (ROUND[dtype] + 3 * U) * np.abs(du0) + FLOOR[dtype] + ev * np.abs(d), "dup")
        holds(part(ch), again, ev * np.abs(u) + 2 * U * np.abs(again), dtype, "h in 8 bits")
        a, b = host(dgate[at]), host(dup[at])
        want = a @ wg0 + b @ wu0
        near(dx[at], want, (ROUND[dtype] + U) * np.abs(want) + FLOOR[dtype] + chain2 * U * (np.abs(a) @ np.abs(wg0) + np.abs(b) @ np.abs(wu0)), "dx")
        xh, t = held(xhat), np.abs(host(dx[at]) * gamma0)
        r0 = host(rstd[at])
        want = plain.rms_norm_backward(host(dx[at]), xh, r0, gamma0)[0]
        size = r0[:, None] * (t + np.abs(xh) * (t * np.abs(xh)).mean(axis=1, keepdims=True))
        near(ds[at], want + d, (ROUND[dtype] + U) * np.abs(want + d) + FLOOR[dtype] + 80 * U * size + 2 * U * np.abs(d), "ds")
    assert bool(dgamma.isfinite().all())
