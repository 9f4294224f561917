"""The operators on 8-bit checkpoints of activations against their plain statements in 64 bits (ops_plain.py)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import ops_plain as plain  # noqa: E402
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


def up(a, dtype="f32", ld=None, skew=0):
    """a on the GPU in the given type; ld: distance of the rows; skew: elements between an aligned address and the first."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).to(T[dtype])
    if t.dim() != 2 or (ld is None and skew == 0):
        return t.cuda()
    rows, cols = t.shape
    ld = cols if ld is None else ld
    buf = torch.full((skew + rows * ld + 8,), 77.0, dtype=T[dtype], device="cuda")
    v = buf[skew:].as_strided((rows, cols), (ld, 1))
    v.copy_(t)
    return v


def room(rows, cols, dtype, ld=None, skew=0):
    return up(np.zeros((rows, cols)), dtype, ld, skew)


def ckpt(rows, cols, ld_q=None, ld_s=None, skew=0):
    """An empty checkpoint; with distances given, one whose rows lie at odd places between sentinels."""
    if ld_q is None:
        return P.Checkpoint.empty(rows, cols)
    groups = (cols + 31) // 32
    q = torch.full((skew + rows * ld_q + 8,), 99, dtype=torch.int8, device="cuda")
    s = torch.full((skew + rows * ld_s + 8,), 99, dtype=torch.uint8, device="cuda")
    return P.Checkpoint(q[skew:].as_strided((rows, cols), (ld_q, 1)), s[skew:].as_strided((rows, groups), (ld_s, 1)))


def filled(values, cap=248, **kw):
    """A checkpoint of the values (64 bits), made on the host; -> (checkpoint, what it holds)"""
    q, code = plain.pack(values, cap)
    c = ckpt(*values.shape, **kw)
    c.q.copy_(torch.from_numpy(q))
    c.scale.copy_(torch.from_numpy(code))
    return c, plain.unpack(q, code)


def near(got, want, bound, label):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, label
    bad = ~(np.abs(got - want) <= bound)
    bad &= ~(np.isnan(got) & np.isnan(want))
    if bad.any():
        k = np.argwhere(bad)[0]
        raise AssertionError(f"{label}: {bad.sum()} of {bad.size} off, first at {tuple(k)}: {got[tuple(k)]} for {want[tuple(k)]}")


def activations(rng, rows, cols):
    return rng.standard_normal((rows, cols)) * np.where(rng.random(cols) < 0.05, 6.0, 1.0)


# ------------------------------------------------------------------ checkpoints

SHAPES = [(1, 1), (1, 7), (3, 8), (2, 31), (5, 32), (4, 33), (7, 64), (3, 100), (2, 255), (33, 256), (1, 4097), (300, 40), (2000, 96)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_pack_and_unpack(ops, dtype, rows, cols):
    rng = np.random.default_rng(rows * 7919 + cols)
    x = activations(rng, rows, cols) * np.exp2(rng.integers(-12, 9, (rows, 1)))
    for kw_x, kw_c in (({}, {}), ({"ld": cols + 5, "skew": 3}, {"ld_q": cols + 3, "ld_s": (cols + 31) // 32 + 1, "skew": 1})):
        xd = up(x, dtype, **kw_x)
        c = ckpt(rows, cols, **kw_c)
        P.tensile_ckpt_pack(ops, xd, c)
        q, code = plain.pack(host(xd), CAP[dtype])
        assert np.array_equal(c.scale.cpu().numpy(), code) and np.array_equal(c.q.cpu().numpy(), q)
        for out in TYPES:
            y = room(rows, cols, out, **kw_x)
            P.tensile_ckpt_unpack(ops, c, y)
            want = plain.unpack(q, code)
            near(y, want, FLOOR[out] if out == "f16" else 0.0, f"unpack to {out}")
        if kw_c:                                       # nothing is written between the rows
            flat = torch.as_strided(c.q, (rows * (cols + 3),), (1,))
            assert bool((flat.view(rows, cols + 3)[:, cols:] == 99).all())
            flat = torch.as_strided(c.scale, (rows * ((cols + 31) // 32 + 1),), (1,))
            assert bool((flat.view(rows, -1)[:, (cols + 31) // 32:] == 99).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_at_the_ends_of_the_range(ops, dtype):
    """Zeros, the smallest and largest numbers, quotients that round to 127 and to 128, ties, infinities and NaN."""
    info = torch.finfo(T[dtype])
    rows = [np.zeros(32), np.r_[np.full(16, info.tiny), np.full(16, -info.tiny)], np.full(32, info.max), np.full(32, -info.max),
            np.r_[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, np.zeros(26)], np.r_[127.25, 1.0, np.zeros(30)], np.r_[127.5, 1.0, 3.0, np.zeros(29)],
            np.r_[127.75, 1.0, np.zeros(30)], np.r_[128.0, 1.0, np.zeros(30)], np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), -np.inf],
            np.r_[np.ones(5), np.nan, np.ones(26)], np.r_[info.max, info.tiny, np.zeros(30)], np.full(32, info.smallest_normal * 3)]
    x = np.tile(np.stack(rows), (1, 3))
    x[:, 32:64] = np.linspace(-1, 1, 32)               # a harmless group in between
    xd = up(x, dtype)
    c = ckpt(*x.shape)
    P.tensile_ckpt_pack(ops, xd, c)
    q, code = plain.pack(host(xd), CAP[dtype])
    assert np.array_equal(c.scale.cpu().numpy(), code) and np.array_equal(c.q.cpu().numpy(), q)
    y = room(*x.shape, dtype)
    P.tensile_ckpt_unpack(ops, c, y)
    got = host(y)
    assert np.array_equal(np.isnan(got), np.repeat(code == 255, 32, axis=1))
    assert np.isfinite(got[~np.isnan(got)]).all()


def test_codes_by_hand(ops):
    """Every code: 0 is a scale of zero, 255 NaN, the others powers of two."""
    q = torch.tensor([[-127, -1, 0, 1, 2, 64, 127]], dtype=torch.int8, device="cuda").repeat(256, 1)
    c = P.Checkpoint(q, torch.arange(256, dtype=torch.uint8, device="cuda")[:, None])
    y = torch.empty(256, 7, device="cuda")
    P.tensile_ckpt_unpack(ops, c, y)
    want = plain.unpack(q.cpu().numpy(), np.arange(256, dtype=np.uint8)[:, None]).astype(np.float32)
    assert np.array_equal(y.cpu().numpy()[1:249], want[1:249]) and np.array_equal(y.cpu().numpy()[0], np.zeros(7))
    assert np.isnan(y.cpu().numpy()[255]).all()


def test_no_rows(ops):
    x, c = torch.empty(0, 40, device="cuda"), P.Checkpoint.empty(0, 40)
    g = torch.ones(40, device="cuda")
    dg, db, dw, bias = (torch.full(s, 7.0, device="cuda") for s in ((40,), (40,), (40, 40), (40,)))
    P.tensile_ckpt_pack(ops, x, c)
    P.tensile_ckpt_unpack(ops, c, x)
    P.tensile_layer_norm(ops, x, g, g, x, xhat=c, rstd=torch.empty(0, device="cuda"))
    P.tensile_gelu(ops, x, x, ckpt=c)
    P.tensile_gelu_backward(ops, x, c, x)
    P.tensile_layer_norm_backward(ops, x, c, torch.empty(0, device="cuda"), g, x, dg, db)
    P.tensile_linear_grad(ops, x, c, dw, dbias=bias, gamma=g, beta=g)
    for t in (dg, db, dw, bias):
        assert not bool(t.any())


# ------------------------------------------------------------------ layer norm

NORM_COLS = [1, 2, 8, 33, 64, 100, 128, 129, 500, 512, 513, 768, 1024, 1025, 2048, 2049, 4096, 4100, 8192, 8199, 16384, 16385, 40_003]


def check_norm(ops, dtype, param, rows, cols, residual=True, total=True, keep=True, eps=1e-5, skew=0, seed=0, x=None):
    rng = np.random.default_rng(seed + rows * 31 + cols)
    layout = {"ld": cols + 3, "skew": 1} if skew else {}
    xd = up(activations(rng, rows, cols) + 0.5 if x is None else x, dtype, **layout)
    rd = up(activations(rng, rows, cols), dtype, **layout) if residual else None
    gamma, beta = up(1 + 0.2 * rng.standard_normal(cols), param), up(0.2 * rng.standard_normal(cols), param)
    y, rstd = room(rows, cols, dtype, **layout), torch.empty(rows, device="cuda")
    tot = room(rows, cols, dtype, **layout) if total else None
    c = ckpt(rows, cols, **({"ld_q": cols + 5, "ld_s": (cols + 31) // 32 + 2, "skew": 3} if skew else {})) if keep else None
    P.tensile_layer_norm(ops, xd, gamma, beta, y, eps=eps, residual=rd, total=tot, xhat=c, rstd=rstd)
    s = host(xd) + (host(rd) if residual else 0)
    y0, xh0, rstd0 = plain.layer_norm(s, host(gamma), host(beta), eps)
    label = f"{dtype}/{param} {rows}x{cols}"
    # the mean is off by no more than c * U * max|s|, c the length of its chain of additions (at most 8 * 16 + 22) and
    # the rounding of s itself; the variance by twice that relative to sigma, and its own sum
    c_sum = 64 if cols <= 16_384 else 160
    e = c_sum * U * (np.abs(s).max(axis=1) * rstd0 + 2)
    e = e[:, None] * (1 + np.abs(xh0))
    near(rstd, rstd0, (c_sum * U * (np.abs(s).max(axis=1) * rstd0 + 2)) * rstd0, label + " rstd")
    near(y, y0, ROUND[dtype] * np.abs(y0) + FLOOR[dtype] + 1.01 * e * np.abs(host(gamma)) + 4 * U * (np.abs(y0) + np.abs(host(beta))), label + " y")
    if total:
        near(tot, s, 1.01 * (ROUND[dtype] + U) * np.abs(s) + FLOOR[dtype], label + " total")
    if keep:
        code = c.scale.cpu().numpy().astype(np.int64)
        a, spread = np.abs(plain.groups_of(xh0)).max(axis=2), np.abs(plain.groups_of(e)).max(axis=2)
        assert (code >= plain.code_of(np.maximum(a - spread, 0), CAP[dtype])).all() and (code <= plain.code_of(a + spread, CAP[dtype])).all(), label + " codes"
        value = plain.unpack(c.q.cpu().numpy(), code.astype(np.uint8))
        near(value, xh0, 0.5 * np.repeat(np.exp2(code - 127.0), 32, axis=1)[:, :cols] + e, label + " xhat")


@pytest.mark.parametrize("cols", NORM_COLS)
@pytest.mark.parametrize("dtype,param", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_layer_norm(ops, dtype, param, cols):
    say(f"layer norm {dtype} {cols}")
    for rows in (1, 5, 70):
        check_norm(ops, dtype, param, rows, cols)


@pytest.mark.parametrize("dtype,param", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
def test_layer_norm_without_the_optional_parts(ops, dtype, param):
    check_norm(ops, dtype, param, 9, 768, residual=False, total=False, keep=False)
    check_norm(ops, dtype, param, 9, 100, residual=False, total=False, keep=True)
    check_norm(ops, dtype, param, 9, 768, residual=True, total=False, keep=False)
    check_norm(ops, dtype, param, 6, 16_500, residual=False, total=True, keep=True)


@pytest.mark.parametrize("cols", [7, 100, 768, 1500, 5000, 9001, 17_001])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_at_odd_places(ops, dtype, cols):
    check_norm(ops, dtype, "f32", 11, cols, skew=1)


def test_layer_norm_of_many_rows(ops):
    """More rows than teams: every team goes on to further rows."""
    for cols in (16, 128, 300, 768, 2000, 3000):
        check_norm(ops, "bf16", "f32", 40_000 if cols <= 128 else 6_007, cols)


def test_layer_norm_of_a_large_mean(ops):
    """Centred before squaring: no cancellation where the mean is a thousand times the deviation."""
    rng = np.random.default_rng(5)
    for cols in (100, 768, 3000, 20_000):
        check_norm(ops, "f32", "f32", 8, cols, residual=False, total=False, x=1000 + rng.standard_normal((8, cols)))


def test_layer_norm_of_constant_and_of_non_finite_rows(ops):
    cols = 776
    x = np.random.default_rng(1).standard_normal((5, cols))
    x[1] = 3.0
    x[2, 700] = np.nan
    x[3, 5] = np.inf
    xd, g, b = up(x, "bf16"), torch.full((cols,), 2.0, device="cuda"), torch.full((cols,), 0.25, device="cuda")
    y, c, rstd = torch.empty_like(xd), P.Checkpoint.empty(5, cols), torch.empty(5, device="cuda")
    P.tensile_layer_norm(ops, xd, g, b, y, xhat=c, rstd=rstd)
    back = torch.empty_like(xd)
    P.tensile_ckpt_unpack(ops, c, back)
    assert bool((y[1] == 0.25).all()) and not bool(back[1].any()) and abs(float(rstd[1]) * 1e-5 ** 0.5 - 1) < 1e-6
    assert bool(y[2:4].isnan().all()) and bool(back[2:4].isnan().all())
    assert bool(y[[0, 4]].isfinite().all()) and bool(back[[0, 4]].isfinite().all())
    # eps = 0 on a constant row: 0 * inf, as the formula has it, also in the last, partial group
    P.tensile_layer_norm(ops, xd, g, b, y, eps=0.0, xhat=c, rstd=rstd)
    P.tensile_ckpt_unpack(ops, c, back)
    assert bool(y[1].isnan().all()) and bool(back[1].isnan().all()) and bool(y[0].isfinite().all())


def check_norm_backward(ops, dtype, param, rows, cols, residual=True, params=True, skew=0, in_place="", values=None):
    rng = np.random.default_rng(rows * 17 + cols)
    layout = {"ld": cols + 3, "skew": 1} if skew else {}
    dy = up(rng.standard_normal((rows, cols)) * 0.1, dtype, **layout)
    dr = up(rng.standard_normal((rows, cols)) * 0.1, dtype, **layout) if residual else None
    c, xh = filled(activations(rng, rows, cols) if values is None else values, CAP[dtype],
                   **({"ld_q": cols + 5, "ld_s": (cols + 31) // 32 + 2, "skew": 3} if skew else {}))
    rstd = up(np.exp(rng.standard_normal(rows)))
    gamma = up(1 + 0.2 * rng.standard_normal(cols), param)
    dy0, dr0, g0, rstd0 = host(dy), host(dr) if residual else 0, host(gamma), host(rstd)
    dx = dy if in_place == "dy" else dr if in_place == "dr" else room(rows, cols, dtype, **layout)
    dg, db = (torch.full((cols,), 5.0, dtype=T[param], device="cuda") for _ in range(2)) if params else (None, None)
    P.tensile_layer_norm_backward(ops, dy, c, rstd, gamma, dx, dg, db, dresidual=dr)
    want, dg0, db0 = plain.layer_norm_backward(dy0, xh, rstd0, g0)
    h = np.abs(dy0 * g0)
    # the two means: chains of at most 8 * 2 additions in a lane (8 * 5 in a long row), 6 across lanes, 16 across wavefronts
    size = rstd0[:, None] * (h + h.mean(axis=1, keepdims=True) + np.abs(xh) * (h * np.abs(xh)).mean(axis=1, keepdims=True))
    label = f"{dtype}/{param} {rows}x{cols}"
    near(dx, want + dr0, (ROUND[dtype] + U) * np.abs(want + dr0) + FLOOR[dtype] + 80 * U * size + 2 * U * np.abs(dr0), label + " dx")
    if params:
        # rows of a team in turn, teams of a workgroup, partial sums in 32 strands
        chain = rows / min(rows, 256) + 16 + 64 + 8
        near(dg, dg0, (ROUND[param] + U) * np.abs(dg0) + FLOOR[param] + chain * U * (np.abs(dy0 * xh)).sum(axis=0), label + " dgamma")
        near(db, db0, (ROUND[param] + U) * np.abs(db0) + FLOOR[param] + chain * U * np.abs(dy0).sum(axis=0), label + " dbeta")


@pytest.mark.parametrize("cols", NORM_COLS)
@pytest.mark.parametrize("dtype,param", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_layer_norm_backward(ops, dtype, param, cols):
    say(f"layer norm backward {dtype} {cols}")
    for rows in (1, 5, 70):
        check_norm_backward(ops, dtype, param, rows, cols)


@pytest.mark.parametrize("dtype,param", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
def test_layer_norm_backward_parts_and_places(ops, dtype, param):
    for cols in (7, 100, 768, 1500, 5000, 17_001):
        check_norm_backward(ops, dtype, param, 11, cols, skew=1)
        check_norm_backward(ops, dtype, param, 11, cols, residual=False, params=False)
        check_norm_backward(ops, dtype, param, 300, cols, in_place="dy")
        check_norm_backward(ops, dtype, param, 300, cols, in_place="dr")


def test_layer_norm_backward_of_many_rows(ops):
    for cols in (16, 128, 300, 768, 2000, 3000, 8000):
        check_norm_backward(ops, "bf16", "f32", 40_000 if cols <= 128 else 4_007, cols)


def test_layer_norm_backward_keeps_a_lost_row_to_itself(ops):
    """A NaN group spoils its own row and its own columns' dgamma, nothing else - also at the end of a row."""
    rows, cols = 9, 40
    v = np.random.default_rng(3).standard_normal((rows, cols))
    v[4, 35] = np.inf
    c, _ = filled(v)
    dy, g = torch.ones(rows, cols, device="cuda"), torch.ones(cols, device="cuda")
    dx, dg, db = torch.empty_like(dy), torch.empty_like(g), torch.empty_like(g)
    P.tensile_layer_norm_backward(ops, dy, c, torch.ones(rows, device="cuda"), g, dx, dg, db)
    lost = dx.isnan().any(1).cpu().numpy()
    assert lost.tolist() == [k == 4 for k in range(rows)]
    assert dg.isnan().cpu().numpy().tolist() == [k >= 32 for k in range(cols)] and bool((db == rows).all())


@pytest.mark.parametrize("cols", [64, 512, 800, 4096, 20_000])
def test_layer_norm_backward_against_differences(ops, cols):
    """Rows whose normalised form is held exactly (0, 2 and -2): the gradient is that of the norm itself."""
    rng = np.random.default_rng(cols)
    rows = 4
    xh = np.zeros((rows, cols))
    for r in range(rows):
        at = rng.permutation(cols)[:cols // 4]
        xh[r, at[::2]], xh[r, at[1::2]] = 2.0, -2.0
    sigma, gamma, beta = np.exp(rng.standard_normal((rows, 1))), 1 + 0.3 * rng.standard_normal(cols), rng.standard_normal(cols)
    s = sigma * xh + 0.3
    dy = rng.standard_normal((rows, cols))
    c, held = filled(xh)
    assert np.array_equal(held, xh)
    dx, dg, db = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    P.tensile_layer_norm_backward(ops, up(dy), c, up(1 / sigma[:, 0]), up(gamma), dx, dg, db)
    loss = lambda s, g, b: (dy * plain.layer_norm(s, g, b, 0.0)[0]).sum()
    step = 1e-5
    for _ in range(4):
        d, dgm, dbt = rng.standard_normal((rows, cols)), rng.standard_normal(cols), rng.standard_normal(cols)
        for got, dirs in ((np.vdot(host(dx), d), (d, 0, 0)), (np.vdot(host(dg), dgm), (0, dgm, 0)), (np.vdot(host(db), dbt), (0, 0, dbt))):
            diff = (loss(s + step * dirs[0], gamma + step * dirs[1], beta + step * dirs[2])
                    - loss(s - step * dirs[0], gamma - step * dirs[1], beta - step * dirs[2])) / (2 * step)
            # error of the differences (step^2, and 2^-52 / step of the loss's magnitude), of 32 bits in each product
            size = np.abs(dy).sum() * 4
            assert abs(got - diff) <= 1e-6 * size, (cols, got, diff)


def test_layer_norm_in_place(ops):
    rng = np.random.default_rng(8)
    for cols in (100, 768, 5000, 16_500):
        x, r = up(rng.standard_normal((30, cols)), "bf16"), up(rng.standard_normal((30, cols)), "bf16")
        g, b = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
        y, t = torch.empty_like(x), torch.empty_like(x)
        P.tensile_layer_norm(ops, x, g, b, y, residual=r, total=t)
        for yi, ti in ((0, 1), (1, 0)):
            both = [x.clone(), r.clone()]
            P.tensile_layer_norm(ops, both[0], g, b, both[yi], residual=both[1], total=both[ti])
            assert torch.equal(both[yi], y) and torch.equal(both[ti], t)


# ------------------------------------------------------------------ gelu

@pytest.mark.parametrize("tanh", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 33), (5, 100), (64, 768), (7, 4099)])
def test_gelu(ops, dtype, tanh, rows, cols):
    rng = np.random.default_rng(rows + cols)
    x = activations(rng, rows, cols) * 2
    x.reshape(-1)[::5] *= 1e-3
    if cols > 40:
        x[0, :8] = [0, -0.0, 30, -30, 100, -100, 5.5, -5.5]
    for kw, kc in (({}, {}), ({"ld": cols + 3, "skew": 1}, {"ld_q": cols + 5, "ld_s": (cols + 31) // 32 + 2, "skew": 3})):
        xd, y, c = up(x, dtype, **kw), room(rows, cols, dtype, **kw), ckpt(rows, cols, **kc)
        P.tensile_gelu(ops, xd, y, ckpt=c, tanh=tanh)
        x0 = host(xd)
        want, _ = plain.gelu(x0, tanh)
        # the distribution function to 7.5e-8 (or a reciprocal's and an exponential's few units), times x
        near(y, want, (ROUND[dtype] + 2 * U) * np.abs(want) + FLOOR[dtype] + 5e-7 * np.abs(x0), "gelu")
        q, code = plain.pack(x0, CAP[dtype])
        assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.scale.cpu().numpy(), code)
        alone = room(rows, cols, dtype, **kw)
        P.tensile_gelu(ops, xd, alone, tanh=tanh)
        assert torch.equal(alone, y)

        xh = plain.unpack(q, code)
        dy, dx, yc = up(rng.standard_normal((rows, cols)), dtype, **kw), room(rows, cols, dtype, **kw), ckpt(rows, cols, **kc)
        P.tensile_gelu_backward(ops, dy, c, dx, y_ckpt=yc, tanh=tanh)
        y0, slope = plain.gelu(xh, tanh)
        want = host(dy) * slope
        near(dx, want, (ROUND[dtype] + 2 * U) * np.abs(want) + FLOOR[dtype] + 1e-6 * (1 + np.abs(xh)) * np.abs(host(dy)), "gelu backward")
        got_code = yc.scale.cpu().numpy().astype(np.int64)
        value, e = plain.unpack(yc.q.cpu().numpy(), got_code.astype(np.uint8)), 5e-7 * np.abs(xh) + 2 * U * np.abs(y0)
        near(value, y0, 0.5 * np.repeat(np.exp2(got_code - 127.0), 32, axis=1)[:, :cols] + e, "checkpoint of gelu")
        a = np.abs(plain.groups_of(y0)).max(axis=2)
        spread = np.abs(plain.groups_of(e)).max(axis=2)
        assert (got_code >= plain.code_of(np.maximum(a - spread, 0), CAP[dtype])).all() and (got_code <= plain.code_of(a + spread, CAP[dtype])).all()
        # in place
        P.tensile_gelu(ops, xd, xd, tanh=tanh)
        assert torch.equal(xd, y)
        P.tensile_gelu_backward(ops, dy, c, dy, y_ckpt=c, tanh=tanh)
        assert torch.equal(dy, dx) and torch.equal(c.q, yc.q) and torch.equal(c.scale, yc.scale)


@pytest.mark.parametrize("tanh", [False, True])
def test_gelu_backward_against_differences(ops, tanh):
    rng = np.random.default_rng(2)
    c, x = filled(rng.standard_normal((20, 96)) * 3)
    dy = rng.standard_normal(x.shape)
    dx = torch.empty(x.shape, device="cuda")
    P.tensile_gelu_backward(ops, up(dy), c, dx, tanh=tanh)
    h = 1e-5
    diff = dy * (plain.gelu(x + h, tanh)[0] - plain.gelu(x - h, tanh)[0]) / (2 * h)
    # the differences: h^2 and 2^-52 |x| / h; 32 bits as in test_gelu
    near(dx, diff, np.abs(dy) * (1e-9 + 1e-10 * (1 + np.abs(x)) + 2e-6 * (1 + np.abs(x))), "differences")


@pytest.mark.parametrize("tanh", [False, True])
def test_gelu_of_extremes(ops, tanh):
    x = torch.tensor([[1e30, -1e30, 3e38, -3e38, 1e-30, -1e-30, float("nan"), float("inf"), 0.0]], dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    P.tensile_gelu(ops, x, y, tanh=tanh)
    assert torch.equal(y[0, [0, 2, 7, 8]], x[0, [0, 2, 7, 8]]) and not bool(y[0, [1, 3]].any()) and bool(y[0, 6].isnan())
    c, _ = filled(host(x[:, :4]))
    dx = torch.empty(1, 4, device="cuda")
    P.tensile_gelu_backward(ops, torch.ones(1, 4, device="cuda"), c, dx, tanh=tanh)
    held = plain.unpack(c.q.cpu().numpy(), c.scale.cpu().numpy())
    assert np.array_equal(dx.cpu().numpy(), np.where(held == 0, 0.5, (held > 0).astype(float)).astype(np.float32))


# ------------------------------------------------------------------ weight gradient

def check_grad(ops, dtype, grad, M, N, K, affine=None, bias=True, skew=0, seed=0, cap=248):
    rng = np.random.default_rng(seed + M + 3 * N + 5 * K)
    dy = up(rng.standard_normal((M, N)), dtype, **({"ld": N + 3, "skew": 1} if skew else {}))
    c, x = filled(activations(rng, M, K), cap, **({"ld_q": K + 5, "ld_s": (K + 31) // 32 + 2, "skew": 3} if skew else {}))
    gamma, beta = (up(1 + 0.3 * rng.standard_normal(K), affine), up(0.3 * rng.standard_normal(K), affine)) if affine else (None, None)
    dw = room(N, K, grad, **({"ld": K + 2, "skew": 1} if skew else {}))
    db = torch.full((N,), 3.0, dtype=T[grad], device="cuda") if bias else None
    P.tensile_linear_grad(ops, dy, c, dw, dbias=db, gamma=gamma, beta=beta)
    dy0 = host(dy)
    product, db0 = plain.linear_grad(dy0, x)
    want = product * host(gamma) + db0[:, None] * host(beta) if affine else product
    # chains: 16 products to an instruction, an instruction after the other, then the parts
    chain = M / 16 + 24 + 64
    size = np.abs(dy0).T @ np.abs(x)
    size_b = np.abs(dy0).sum(axis=0)
    e = chain * U * size
    if affine:
        e = e * np.abs(host(gamma)) + chain * U * size_b[:, None] * np.abs(host(beta)) + 4 * U * np.abs(want)
    label = f"{dtype}->{grad} {M}x{N}x{K}"
    near(dw, want, (ROUND[grad] + U) * np.abs(want) + FLOOR[grad] + e, label + " dw")
    if bias:
        near(db, db0, (ROUND[grad] + U) * np.abs(db0) + FLOOR[grad] + chain * U * size_b, label + " dbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 5, 40), (2, 8, 32), (17, 10, 256), (32, 512, 784), (63, 129, 130), (64, 128, 128),
                                   (65, 127, 129), (100, 300, 33), (1000, 10, 17), (255, 256, 256), (513, 100, 500)])
def test_linear_grad(ops, dtype, M, N, K):
    say(f"linear grad {dtype} {M}x{N}x{K}")
    check_grad(ops, dtype, "f32", M, N, K)
    check_grad(ops, dtype, dtype, M, N, K, affine="f32", bias=False)
    check_grad(ops, dtype, "f32", M, N, K, affine=dtype, skew=1)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_grad_with_the_rows_split(ops, dtype):
    """Few tiles and many rows: the sum is cut into parts, the last of them shorter or of a single row."""
    for M, N, K in ((4096, 128, 128), (4097, 130, 96), (12_289, 10, 40), (2049, 300, 257)):
        say(f"linear grad split {dtype} {M}x{N}x{K}")
        check_grad(ops, dtype, "f32", M, N, K, affine="f32")
        check_grad(ops, dtype, dtype, M, N, K)


def test_linear_grad_of_larger_tiles(ops):
    for M, N, K in ((300, 1024, 1100), (1024, 2048, 2304), (96, 4096, 4200)):
        say(f"linear grad large {M}x{N}x{K}")
        check_grad(ops, "bf16", "bf16", M, N, K)
        check_grad(ops, "bf16", "f32", M, N, K, affine="f32")


def test_linear_grad_of_larger_tiles_at_odd_places(ops):
    """Rows that start at any element, that end inside a load, and rows of the product that are split."""
    for M, N, K in ((131, 2049, 2307), (2100, 2050, 2305), (33, 2056, 2320), (31, 2049, 2304), (544, 2048, 2304), (577, 2044, 2290)):
        say(f"linear grad large, odd places {M}x{N}x{K}")
        check_grad(ops, "bf16", "f32", M, N, K, affine="f32", skew=1)
        check_grad(ops, "bf16", "bf16", M, N, K, affine="bf16")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_linear_grad_of_wider_tiles(ops, dtype):
    """Gradients in several pieces: tiles of twice the checkpoint's columns, whole and ragged, with and without parts."""
    for M, N, K in ((64, 2048, 2304), (97, 2050, 2001), (1, 2048, 2047), (2100, 500, 1001), (4352, 128, 2048)):
        say(f"linear grad wider {dtype} {M}x{N}x{K}")
        check_grad(ops, dtype, "f32", M, N, K, affine="f32")
        check_grad(ops, dtype, dtype, M, N, K, skew=1)


def test_linear_grad_of_larger_tiles_keeps_non_finite_values_apart(ops):
    M, N, K = 70, 2050, 2300
    rng = np.random.default_rng(16)
    dy, v = rng.standard_normal((M, N)), rng.standard_normal((M, K))
    dy[69, 3], dy[0, 2049] = np.inf, np.nan
    v[69, 2290] = np.nan                               # its group: columns 2272 .. 2299
    c, _ = filled(v)
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    P.tensile_linear_grad(ops, up(dy, "bf16"), c, dw, dbias=db)
    want = np.zeros((N, K), dtype=bool)
    want[3], want[2049], want[:, 2272:] = True, True, True
    assert np.array_equal(~np.isfinite(dw.cpu().numpy()), want)
    assert np.array_equal(np.isinf(db.cpu().numpy()), np.arange(N) == 3) and np.array_equal(np.isnan(db.cpu().numpy()), np.arange(N) == 2049)


def test_linear_grad_keeps_every_bit_of_the_gradient(ops):
    """One row: each element is one product of the gradient's 24 (or 11) bits with the checkpoint's 7."""
    rng = np.random.default_rng(4)
    for dtype in TYPES:
        dy = up(rng.standard_normal((1, 200)) * np.exp2(rng.integers(-8, 8, (1, 200))), dtype)
        c, x = filled(rng.standard_normal((1, 96)))
        dw = torch.empty(200, 96, device="cuda")
        P.tensile_linear_grad(ops, dy, c, dw)
        near(dw, host(dy).T @ x, 2 * U * np.abs(host(dy).T @ x), dtype)


def test_linear_grad_of_non_finite_values(ops):
    """An infinity or a NaN reaches the elements that it belongs to, and no others; rows that do not exist bring none in."""
    M, N, K = 70, 140, 140
    rng = np.random.default_rng(6)
    dy, v = rng.standard_normal((M, N)), rng.standard_normal((M, K))
    dy[69, 3], dy[0, 130] = np.inf, np.nan
    v[33, 50] = np.nan                                 # its group: columns 32 .. 63
    for dtype in TYPES:
        c, x = filled(v)
        dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
        P.tensile_linear_grad(ops, up(dy, dtype), c, dw, dbias=db)
        got = ~np.isfinite(dw.cpu().numpy())
        want = np.zeros((N, K), dtype=bool)
        want[3], want[130], want[:, 32:64] = True, True, True
        assert np.array_equal(got, want), dtype
        assert np.array_equal(np.isinf(db.cpu().numpy()), np.arange(N) == 3) and np.array_equal(np.isnan(db.cpu().numpy()), np.arange(N) == 130)


def test_linear_grad_against_differences(ops):
    """loss = sum dy * (X W^T + bias), X the norm's output: linear in W and bias, so the difference is exact."""
    rng = np.random.default_rng(9)
    M, N, K = 50, 30, 70
    c, xh = filled(rng.standard_normal((M, K)))
    dy, gamma, beta, W, b = (rng.standard_normal(s) for s in ((M, N), (K,), (K,), (N, K), (N,)))
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    P.tensile_linear_grad(ops, up(dy), c, dw, dbias=db, gamma=up(gamma), beta=up(beta))
    loss = lambda W, b: (dy * ((xh * gamma + beta) @ W.T + b)).sum()
    for _ in range(4):
        dW, dB = rng.standard_normal((N, K)), rng.standard_normal(N)
        got = np.vdot(host(dw), dW) + np.vdot(host(db), dB)
        diff = (loss(W + dW, b + dB) - loss(W - dW, b - dB)) / 2
        size = (np.abs(dy).T @ np.abs(xh * gamma + beta) * np.abs(dW)).sum() + (np.abs(dy).sum(axis=0) * np.abs(dB)).sum()
        assert abs(got - diff) <= 64 * U * size


# ------------------------------------------------------------------ calls

def test_views_of_three_dimensions(ops):
    x = torch.randn(2, 5, 64, device="cuda").to(torch.bfloat16)
    y, c = torch.empty_like(x), P.Checkpoint.empty(10, 64)
    P.tensile_gelu(ops, x, y, ckpt=c)
    flat = torch.empty(10, 64, dtype=torch.bfloat16, device="cuda")
    P.tensile_gelu(ops, x.view(10, 64), flat)
    assert torch.equal(flat, y.view(10, 64))


def test_offsets_beyond_32_bits(ops):
    """Rows 2^31 elements apart, and more than 2^32 elements in one matrix."""
    big = torch.empty(2 ** 32 + 4096, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((3, 72), (2 ** 31, 1))
    x.copy_(torch.randn(3, 72, device="cuda"))
    c, c2 = P.Checkpoint.empty(3, 72), P.Checkpoint.empty(3, 72)
    P.tensile_ckpt_pack(ops, x, c)
    P.tensile_ckpt_pack(ops, x.contiguous(), c2)
    assert torch.equal(c.q, c2.q) and torch.equal(c.scale, c2.scale)
    g = torch.ones(72, device="cuda")
    y, near_y = big.as_strided((3, 72), (2 ** 31, 1), 1024), torch.empty(3, 72, dtype=torch.bfloat16, device="cuda")
    P.tensile_layer_norm(ops, x, g, g, y)
    P.tensile_layer_norm(ops, x.contiguous(), g, g, near_y)
    assert torch.equal(y, near_y)
    dw, dw2 = torch.empty(72, 72, device="cuda"), torch.empty(72, 72, device="cuda")
    P.tensile_linear_grad(ops, x, c, dw)
    P.tensile_linear_grad(ops, x.contiguous(), c, dw2)
    assert torch.equal(dw, dw2)
    rows = 2 ** 27 + 2
    flat = big[: rows * 32].view(rows, 32)
    flat[:2].copy_(torch.randn(2, 32, device="cuda"))
    flat[2 ** 27:].copy_(torch.randn(2, 32, device="cuda"))
    whole = P.Checkpoint(torch.empty(rows, 32, dtype=torch.int8, device="cuda"), torch.empty(rows, 1, dtype=torch.uint8, device="cuda"))
    P.tensile_ckpt_pack(ops, flat, whole)
    for part in (slice(0, 2), slice(2 ** 27, rows)):
        c = P.Checkpoint.empty(2, 32)
        P.tensile_ckpt_pack(ops, flat[part], c)
        assert torch.equal(whole.q[part], c.q) and torch.equal(whole.scale[part], c.scale)


def test_same_bits_again_and_on_another_stream(ops):
    rng = np.random.default_rng(12)
    dy, dz = up(rng.standard_normal((3000, 768)), "bf16"), up(rng.standard_normal((3000, 300)), "bf16")
    c, _ = filled(rng.standard_normal((3000, 768)))
    g, rstd = torch.ones(768, device="cuda"), torch.ones(3000, device="cuda")
    results = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side, None, side):
        out = [torch.empty_like(dy), torch.empty(768, device="cuda"), torch.empty(768, device="cuda"), torch.empty(300, 768, device="cuda")]
        side.wait_stream(torch.cuda.current_stream())
        P.tensile_layer_norm_backward(ops, dy, c, rstd, g, out[0], out[1], out[2], stream=stream)
        P.tensile_linear_grad(ops, dz, c, out[3], stream=stream)
        torch.cuda.synchronize()
        results.append(out)
    for out in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out, results[0]))


def test_captured_and_replayed(ops):
    """A graph of the whole set, with eager work between the replays and new inputs for each."""
    M, N, K = 2048, 256, 768
    x, dz = torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    g, b = torch.rand(K, device="cuda"), torch.rand(K, device="cuda")
    c, ga, gc = P.Checkpoint.empty(M, K), P.Checkpoint.empty(M, K), P.Checkpoint.empty(M, K)

    def outputs():
        return {n: torch.empty(s, dtype=t, device="cuda") for n, s, t in
                (("y", (M, K), x.dtype), ("rstd", (M,), torch.float32), ("a", (M, K), x.dtype), ("da", (M, K), x.dtype), ("dx", (M, K), x.dtype),
                 ("dg", (K,), torch.float32), ("db", (K,), torch.float32), ("dw", (N, K), torch.float32), ("bias", (N,), torch.float32))}

    def work(o, stream):
        P.tensile_layer_norm(ops, x, g, b, o["y"], xhat=c, rstd=o["rstd"], stream=stream)
        P.tensile_gelu(ops, o["y"], o["a"], ckpt=ga, stream=stream)
        P.tensile_gelu_backward(ops, o["a"], ga, o["da"], y_ckpt=gc, stream=stream)
        P.tensile_linear_grad(ops, dz, gc, o["dw"], stream=stream)
        P.tensile_linear_grad(ops, dz, c, o["dw"], dbias=o["bias"], gamma=g, beta=b, stream=stream)
        P.tensile_layer_norm_backward(ops, o["da"], c, o["rstd"], g, o["dx"], o["dg"], o["db"], stream=stream)

    def refill(seed):
        torch.manual_seed(seed)
        x.copy_(torch.randn(M, K, device="cuda"))
        dz.copy_(torch.randn(M, N, device="cuda"))

    refill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(outputs(), side)                          # the scratch of this stream
    torch.cuda.synchronize()
    fixed = outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work(fixed, side)
    for seed in range(1, 5):
        refill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in fixed.items()}
        eager = outputs()
        work(eager, None)
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(got[n], eager[n]), (seed, n)


def test_threads_share_a_handle(ops):
    import threading
    rng = np.random.default_rng(21)
    jobs = []
    for k, cols in enumerate((300, 768, 1500, 2500)):
        dy = up(rng.standard_normal((1200, cols)), "bf16")
        c, _ = filled(rng.standard_normal((1200, cols)))
        g, rstd = torch.ones(cols, device="cuda"), torch.ones(1200, device="cuda")
        want = [torch.empty_like(dy), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
        P.tensile_layer_norm_backward(ops, dy, c, rstd, g, *want)
        jobs.append((dy, c, rstd, g, want, [torch.empty_like(t) for t in want], torch.cuda.Stream()))
    torch.cuda.synchronize()

    def work(job):
        dy, c, rstd, g, _, got, stream = job
        for _ in range(20):
            P.tensile_layer_norm_backward(ops, dy, c, rstd, g, *got, stream=stream)
    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for j in jobs:
        assert all(torch.equal(a, b) for a, b in zip(j[4], j[5]))


def test_refused_allocation_is_an_error_and_the_next_call_works(tuning):
    h = P.tensile_ops_create()
    dy, g, rstd = torch.ones(100, 64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(100, device="cuda")
    c, _ = filled(np.ones((100, 64)))
    out = [torch.empty_like(dy), torch.empty_like(g), torch.empty_like(g)]
    tuning("alloc_fail", 1)
    with pytest.raises(P.TensileError) as e:
        P.tensile_layer_norm_backward(h, dy, c, rstd, g, *out)
    assert e.value.code == P.binding.TENSILE_E_NOMEM
    P.tensile_layer_norm_backward(h, dy, c, rstd, g, *out)
    torch.cuda.synchronize()
    assert bool((out[2] == 100).all())
    h.close()


def test_refusals(ops):
    f = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")
    x, g, c = f(4, 64), f(64, dtype=torch.float32), P.Checkpoint.empty(4, 64)
    rstd = f(4, dtype=torch.float32)

    def refused(call, word):
        with pytest.raises(P.TensileError) as e:
            call()
        assert e.value.code == P.binding.TENSILE_E_INVAL and word in str(e.value), str(e.value)

    refused(lambda: P.tensile_ckpt_pack(ops, x.cpu(), c), "x")
    refused(lambda: P.tensile_ckpt_pack(ops, x.double(), c), "x")
    refused(lambda: P.tensile_ckpt_pack(ops, x.t(), c), "contiguous")
    refused(lambda: P.tensile_ckpt_pack(ops, f(5, 64), c), "shape")
    refused(lambda: P.tensile_ckpt_pack(ops, f(4, 63), c), "shape")
    refused(lambda: P.tensile_ckpt_pack(ops, f(1, 64).expand(4, 64), c), "overlap")
    refused(lambda: P.tensile_ckpt_pack(ops, x, None), "NULL")
    refused(lambda: P.Checkpoint(c.q, c.scale[:, :1]), "belong")
    refused(lambda: P.Checkpoint(c.q.float(), c.scale), "int8")
    refused(lambda: P.tensile_layer_norm(ops, x, g, g, f(4, 64, dtype=torch.float16)), "y")
    refused(lambda: P.tensile_layer_norm(ops, x, g, g, x, eps=-1.0), "eps")
    refused(lambda: P.tensile_layer_norm(ops, x, g, g, x, eps=float("nan")), "eps")
    refused(lambda: P.tensile_layer_norm(ops, x, g[:63], g, x), "gamma")
    refused(lambda: P.tensile_layer_norm(ops, x, g.half(), g.half(), x), "param_type")
    refused(lambda: P.tensile_layer_norm(ops, x, g, g.bfloat16(), x), "beta")
    refused(lambda: P.tensile_layer_norm(ops, x, g, g, x, residual=x.clone(), total=x), "total")
    refused(lambda: P.tensile_layer_norm(ops, x, g, g, x, residual=f(4, 63)), "residual")
    refused(lambda: P.tensile_layer_norm_backward(ops, x, c, None, g, x), "rstd")
    refused(lambda: P.tensile_layer_norm_backward(ops, x, c, rstd, g, x, dgamma=g), "dgamma")
    refused(lambda: P.tensile_layer_norm_backward(ops, x, P.Checkpoint.empty(4, 65), rstd, g, x), "xhat")
    refused(lambda: P.tensile_gelu(ops, x, f(4, 64, dtype=torch.float32)), "y")
    refused(lambda: P.tensile_gelu_backward(ops, x, c, f(3, 64)), "dx")
    refused(lambda: P.tensile_linear_grad(ops, f(4, 10), c, f(64, 10)), "dw")
    refused(lambda: P.tensile_linear_grad(ops, f(4, 10), c, f(10, 64, dtype=torch.float16)), "dw")
    refused(lambda: P.tensile_linear_grad(ops, f(4, 10), c, f(10, 64), gamma=g), "gamma")
    refused(lambda: P.tensile_linear_grad(ops, f(5, 10), c, f(10, 64)), "c")
    h = P.tensile_ops_create()
    h.close()
    refused(lambda: P.tensile_gelu(h, x, x), "freed")
