"""The gated layer's kernels at sizes that reach each of them (test_gated_kernels.py asserts which sizes do), against 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import gated_plain as plain  # noqa: E402
import gated_sizes  # noqa: E402
import paper_2105_13336_amd as P  # noqa: E402
from ops_plain import CAP, FLOOR, ROUND, U  # noqa: E402
from test_gpu_gated import T, TYPES, check_gated, check_gated_backward, filled, host, near, room, say, up  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    h = P.tensile_ops_create()
    yield h
    h.close()


# ------------------------------------------------------------------ every kernel, with its loop in its steady state

@pytest.mark.parametrize("kernel,dtype,M,K,F", gated_sizes.cases(gated_sizes.FORWARD))
def test_forward(ops, kernel, dtype, M, K, F):
    """Every activation, with and without biases, checkpoints, gaps between rows."""
    check_gated(ops, dtype, M, K, F, act="gelu_tanh", bias="f32", odd=True)
    check_gated(ops, dtype, M, K, F, act="silu", keep=False)
    if M * F < 1_000_000 or (M, F) == (2_040, 3_901):
        check_gated(ops, dtype, M, K, F, act="gelu", bias=dtype)


@pytest.mark.parametrize("kernel,dtype,M,K,F", gated_sizes.cases(gated_sizes.BACKWARD))
def test_backward(ops, kernel, dtype, M, K, F):
    check_gated_backward(ops, dtype, M, K, F, act="gelu_tanh", odd=True)
    if M * K < 10_000_000:
        check_gated_backward(ops, dtype, M, K, F, act="silu", keep=False)


# ------------------------------------------------------------------ numbers at the ends of their ranges

LEAST = 1.1e-36                                         # SiLU at -87.3, from where on it may be 0, is 1.02e-36


@pytest.mark.parametrize("dtype", TYPES)
def test_silu_to_its_stated_accuracy(ops, dtype):
    """act(g)*u of one product each, g = u = x*1, from -120 to 120, by tiles and up to 32 tokens; its derivative from a checkpoint."""
    x = up(np.concatenate([np.linspace(-120, 120, 60_001), np.linspace(-90, -86, 4_001), np.linspace(-1, 1, 2_001) * 1e-3])[:, None], dtype)
    one = up([[1.0]], dtype)
    x0 = host(x)
    within = U * (8 + 2 * np.abs(x0))
    value = plain.activation(x0, "silu")[0]
    want = value * x0                                   # (one product more, rounded to 32 bits and then to the type)
    bound = np.where(x0 >= -87.3, (within + U) * np.abs(want), LEAST * np.abs(x0)) + ROUND[dtype] * np.abs(want) * 1.001 + FLOOR[dtype]
    h = torch.empty_like(x)
    P.tensile_gated_linear(ops, x, one, one, h)
    near(h, want, bound, "tiles")
    ends = torch.cat([x[:8], x[30_000:30_008], x[60_001:60_017]])
    few = torch.empty_like(ends)
    P.tensile_gated_linear(ops, ends, one, one, few)
    assert torch.equal(few, torch.cat([h[:8], h[30_000:30_008], h[60_001:60_017]]))
    c, g = filled(np.concatenate([np.arange(-127, 128) * 2.0 ** k for k in (-12, -7, -3, -1, 0)])[:, None])
    unit, _ = filled(np.ones(g.shape))
    dh = torch.ones(g.shape, dtype=T[dtype], device="cuda")
    dgate, dup = torch.empty_like(dh), torch.empty_like(dh)
    P.tensile_gated_linear_backward(ops, dh, c, unit, dgate, dup)
    value, slope = plain.activation(g, "silu")
    within = np.where(g >= -87.3, U * (8 + 2 * np.abs(g)), 0)
    near(dup, value, (ROUND[dtype] + within) * 1.001 * np.abs(value) + np.where(g >= -87.3, 0, LEAST) + FLOOR[dtype], "value")
    near(dgate, slope, ROUND[dtype] * 1.001 * np.abs(slope) + within * (1 + np.abs(g)) + np.where(g >= -87.3, 0, LEAST) + FLOOR[dtype], "slope")


@pytest.mark.parametrize("M", [20, 300, 2_100])
def test_f16_below_its_normal_numbers(ops, M):
    """Inputs, and gradients between the two steps of the backward pass, below 2^-14: the products take them as they are."""
    K, F = 200, 3_901 if M > 2_000 else 300
    rng = np.random.default_rng(M)
    x = up(rng.standard_normal((M, K)) * 2e-6, "f16")
    wg, wu = (up(rng.standard_normal((F, K)) * 1e3, "f16") for _ in range(2))
    h = torch.empty(M, F, dtype=torch.float16, device="cuda")
    cg, cu = P.Checkpoint.empty(M, F), P.Checkpoint.empty(M, F)
    P.tensile_gated_linear(ops, x, wg, wu, h, gate=cg, up=cu)
    x0, wg0, wu0 = host(x), host(wg), host(wu)
    assert (np.abs(x0) < 2.0 ** -14).all() and (x0 != 0).mean() > 0.9
    h0, g0, u0 = plain.gated(x0, wg0, wu0, 0.0, 0.0, "silu")
    n = plain.chain(K, "f16")
    eg, eu = (n * U * (np.abs(x0) @ np.abs(w).T) for w in (wg0, wu0))
    value, ev = np.abs(plain.activation(g0, "silu")[0]), 1.13 * eg + plain.activation_error(g0, "silu", "f16")[0]
    near(h, h0, (ROUND["f16"] + 2 * U) * np.abs(h0) + FLOOR["f16"] + 1.01 * (ev * (np.abs(u0) + eu) + value * eu), "h")
    dh = up(rng.standard_normal((M, F)) * 2e-6, "f16")
    dgate, dup, dx = torch.empty_like(h), torch.empty_like(h), torch.empty_like(x)
    P.tensile_gated_linear_backward(ops, dh, cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=dx)
    a, b = host(dgate), host(dup)
    assert (np.abs(a) < 2.0 ** -14).all() and (a != 0).mean() > 0.1 and (b != 0).mean() > 0.1
    want, size = a @ wg0 + b @ wu0, np.abs(a) @ np.abs(wg0) + np.abs(b) @ np.abs(wu0)
    near(dx, want, (ROUND["f16"] + U) * np.abs(want) + FLOOR["f16"] + plain.chain(2 * F, "f16", 64) * U * size, "dx")
    assert np.abs(want).max() > 2.0 ** -14              # (they are not taken as zeros)


def test_f16_beyond_its_largest_number(ops):
    """A dgate beyond 65,504 is infinite, and so is its row of dx, whatever the other terms of the sum are; other rows are not."""
    M, K, F = 40, 24, 64
    (c, g), (u, _) = filled(np.full((M, F), 4.0)), filled(np.full((M, F), 4.0))
    dh = torch.ones(M, F, dtype=torch.float16, device="cuda")
    dh[7, 5] = 6e4
    w, v = torch.full((F, K), 2.0 ** -10, dtype=torch.float16, device="cuda"), torch.zeros(F, K, dtype=torch.float16, device="cuda")
    dgate, dup, dx = torch.empty_like(dh), torch.empty_like(dh), torch.empty(M, K, dtype=torch.float16, device="cuda")
    P.tensile_gated_linear_backward(ops, dh, c, u, dgate, dup, w_gate=w, w_up=v, dx=dx)
    where = torch.zeros_like(dgate, dtype=torch.bool)
    where[7, 5] = True
    assert torch.equal(dgate.isinf(), where) and torch.equal(dup.isinf(), where)
    assert bool((~dx[7].isfinite()).all()) and bool(dx[torch.arange(M) != 7].isfinite().all())


# ------------------------------------------------------------------ rows far apart

def apart(a, ld, dtype):
    """a with its rows ld elements apart"""
    buf = torch.empty(((a.shape[0] - 1) * ld + a.shape[1],), dtype=T[dtype], device="cuda")
    return buf.as_strided(a.shape, (ld, 1)).copy_(a)


def check_apart(ops, dtype, M, K, F, ld_tokens=None, ld_weights=None):
    """x, dgate and dup, or the weights, with their rows so far apart, against 64 bits."""
    say(f"{dtype} {M}x{K}x{F}, rows {ld_tokens}, {ld_weights} apart")
    rng = np.random.default_rng(M + K + F)
    far = lambda t, ld: apart(t, ld, dtype) if ld else t
    x = far(up(rng.standard_normal((M, K)), dtype), ld_tokens)
    wg, wu = (far(up(rng.standard_normal((F, K)) * K ** -0.5, dtype), ld_weights) for _ in range(2))
    h = room(M, F, dtype)
    P.tensile_gated_linear(ops, x, wg, wu, h)
    x0, wg0, wu0 = host(x), host(wg), host(wu)
    h0, g0, u0 = plain.gated(x0, wg0, wu0, 0.0, 0.0, "silu")
    n = plain.chain(K, dtype, 64)
    eg, eu = (n * U * (np.abs(x0) @ np.abs(w).T) for w in (wg0, wu0))
    value, ev = np.abs(plain.activation(g0, "silu")[0]), 1.13 * eg + plain.activation_error(g0, "silu", dtype)[0]
    near(h, h0, (ROUND[dtype] + 2 * U) * np.abs(h0) + FLOOR[dtype] + 1.01 * (ev * (np.abs(u0) + eu) + value * eu), "h")
    del x, h
    (cg, _), (cu, _) = (filled(rng.standard_normal((M, F)), CAP[dtype]) for _ in range(2))
    dgate, dup, dx = far(room(M, F, dtype), ld_tokens), far(room(M, F, dtype), ld_tokens), room(M, K, dtype)
    P.tensile_gated_linear_backward(ops, up(rng.standard_normal((M, F)), dtype), cg, cu, dgate, dup, w_gate=wg, w_up=wu, dx=dx)
    a, b = host(dgate), host(dup)
    want = a @ wg0 + b @ wu0
    size = np.abs(a) @ np.abs(wg0) + np.abs(b) @ np.abs(wu0)
    near(dx, want, (ROUND[dtype] + U) * np.abs(want) + FLOOR[dtype] + plain.chain(2 * F, dtype, 64) * U * size, "dx")


SPAN = 1 << 31                                          # bytes from the first row to the last


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_far_apart_up_to_32(ops, dtype):
    """The last tokens of sequences: 16 MiB apart, whose offsets fit 32 bits, and too far."""
    size = 4 if dtype == "f32" else 2
    check_apart(ops, dtype, 24, 520, 200, ld_tokens=(16 << 20) // size)
    check_apart(ops, dtype, 32, 333, 100, ld_tokens=(64 << 20) // size)
    check_apart(ops, dtype, 5, 520, 200, ld_tokens=SPAN // 4 // size + 8)
    check_apart(ops, dtype, 32, 333, 700, ld_tokens=SPAN // 31 // size + 8)


@pytest.mark.parametrize("dtype", TYPES)
def test_weights_far_apart_up_to_32_tokens(ops, dtype):
    size, step = (4, 32) if dtype == "f32" else (2, 64)
    check_apart(ops, dtype, 7, 130, 100, ld_weights=(16 << 20) // size)
    check_apart(ops, dtype, 20, 130, 65, ld_weights=SPAN // (step - 1) // size + 8)
    check_apart(ops, dtype, 20, 130, 33, ld_weights=SPAN // 31 // size + 8)


@pytest.mark.parametrize("dtype", TYPES)
def test_tiles_of_rows_far_apart(ops, dtype):
    """Up to 16 MiB apart, and too far: 128 tokens (few, with sums split and whole, and many), 64 features, a step's rows of the weights."""
    size = 4 if dtype == "f32" else 2
    check_apart(ops, dtype, 100, 520, 200, ld_tokens=(16 << 20) // size)
    check_apart(ops, dtype, 130, 130, 2_000, ld_tokens=SPAN // 127 // size + 8)
    check_apart(ops, dtype, 40, 1_700, 90, ld_tokens=SPAN // 39 // size + 8)
    check_apart(ops, dtype, 256, 40, 9_000, ld_tokens=SPAN // 127 // size + 8)
    check_apart(ops, dtype, 200, 300, 150, ld_weights=SPAN // (31 if dtype == "f32" else 63) // size + 8)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_tiles_of_rows_far_apart_are_small_ones(ops, dtype):
    check_apart(ops, dtype, 2_040, 200, 3_901, ld_tokens=(9 << 20) // 2)
    check_apart(ops, dtype, 2_040, 200, 3_901, ld_tokens=(8 << 20) // 2)
