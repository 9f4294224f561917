"""The operators on 8-bit checkpoints at the edges of what their entry points allow, against plain statements or the ordinary form of the
same call."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import ops_plain as plain  # noqa: E402
import paper_2105_13336_amd as P  # noqa: E402
from test_gpu_ops import check_grad, filled, host, near, say, up  # noqa: E402

TYPES = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def ops():
    h = P.tensile_ops_create()
    yield h
    h.close()


# ------------------------------------------------------------------ weight gradient

def spread(c, ld_q=None, ld_s=None):
    """The same checkpoint with its rows further apart (what lies between them is never written)."""
    def far(t, ld):
        if ld is None:
            return t
        v = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (ld, 1))
        v.copy_(t)
        return v
    return P.Checkpoint(far(c.q, ld_q), far(c.scale, ld_s))


# 31 rows of a step: from 2^32 / 31 = 138,547,333 bytes between rows a row's offset needs more than 32 bits
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,far", [(3, dict(ld_s=2 ** 31)), (3, dict(ld_q=2 ** 31)), (40, dict(ld_s=2 ** 27 + 2 ** 23)), (40, dict(ld_q=2 ** 26 - 1, ld_s=2 ** 26)),
                                   (170, dict(ld_s=2 ** 27 + 2 ** 23)), (200, dict(ld_q=2 ** 20, ld_s=2 ** 26 - 1))])
def test_linear_grad_of_far_apart_rows(ops, dtype, M, far):
    """Pitches of the bytes and of the scales on both sides of what 32-bit offsets reach."""
    say(f"linear grad {dtype} {M} rows {far}")
    rng = np.random.default_rng(M)
    c, x = filled(rng.standard_normal((M, 72)) * np.exp2(rng.integers(-9, 9, (M, 1))))
    dy = up(rng.standard_normal((M, 72)), dtype)
    dw = torch.empty(72, 72, device="cuda")
    wide = spread(c, **far)
    P.tensile_linear_grad(ops, dy, wide, dw)
    want, size = host(dy).T @ x, np.abs(host(dy)).T @ np.abs(x)
    near(dw, want, (M / 16 + 90) * 2.0 ** -24 * size, "dw")
    del wide
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(65, 1, 1), (33, 1, 64), (96, 6, 2000), (300, 7, 15), (1000, 3, 300), (2049, 200, 9), (4097, 5, 130), (20_000, 2, 700)])
def test_linear_grad_of_few_columns(ops, dtype, M, N, K):
    """Fewer columns than a load takes (a classifier of two classes, a regression's one output): many steps, a ragged last one, up to 8 parts and more."""
    say(f"linear grad of few columns {dtype} {M}x{N}x{K}")
    check_grad(ops, dtype, "f32", M, N, K)
    check_grad(ops, dtype, dtype, M, N, K, affine="f32", bias=False)
    check_grad(ops, dtype, "f32", M, N, K, affine=dtype, skew=1)


@pytest.mark.parametrize("M,N,K", [(70, 140, 140), (33, 5, 40), (64, 2048, 2304), (4100, 130, 200)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_grad_of_every_nan(ops, dtype, M, N, K):
    """A NaN is one whatever its bits: the quiet one, and those whose only bits are the lowest or the highest below the quiet one's."""
    say(f"linear grad of NaN {dtype} {M}x{N}x{K}")
    bits, int_type = {"f32": ((0x7fc00000, 0x7f800001, 0x7fbfffff, -0x7fffff), torch.int32), "bf16": ((0x7fc0, 0x7f81, 0x7fbf, -0x7f), torch.int16),
                      "f16": ((0x7e00, 0x7c01, 0x7dff, -0x3ff), torch.int16)}[dtype]
    dy = up(np.ones((M, N)), dtype)
    for k, b in enumerate(bits):
        dy.view(int_type)[M - 1 - 7 * k, k] = b
    assert int(dy.isnan().sum()) == 4
    c, _ = filled(np.ones((M, K)))
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    for affine in ({}, dict(gamma=torch.ones(K, device="cuda"), beta=torch.ones(K, device="cuda"))):
        P.tensile_linear_grad(ops, dy, c, dw, dbias=db, **affine)
        assert bool(dw[:4].isnan().all()) and bool(db[:4].isnan().all())
        assert bool((dw[4:] == (2.0 if affine else 1.0) * M).all()) and bool((db[4:] == M).all())


# ------------------------------------------------------------------ layer norm

def test_layer_norm_with_an_eps_at_the_ends_of_its_range(ops):
    x = torch.stack([torch.ones(64, device="cuda"), torch.arange(64, device="cuda") * 1.0])
    g, b, y, rstd = torch.ones(64, device="cuda"), torch.full((64,), 0.25, device="cuda"), torch.empty_like(x), torch.empty(2, device="cuda")
    for eps in (1e39, 1e300, float("inf"), -1e-60):
        with pytest.raises(P.TensileError) as e:
            P.tensile_layer_norm(ops, x, g, b, y, eps=eps, rstd=rstd)
        assert e.value.code == P.binding.TENSILE_E_INVAL and "eps" in str(e.value)
    for eps in (1e-50, 1e-42, 1e-30):                 # a constant row: (x - mean) * rstd = 0 for any eps above 0
        P.tensile_layer_norm(ops, x, g, b, y, eps=eps, rstd=rstd)
        assert bool((y[0] == 0.25).all()) and bool(rstd.isfinite().all())
        near(y[1:], plain.layer_norm(host(x)[1:], 1.0, 0.25, eps)[0], 64 * 2.0 ** -24 * 4, "y")
    P.tensile_layer_norm(ops, x, g, b, y, eps=3e38, rstd=rstd)
    near(rstd, np.full(2, 3e38 ** -0.5), 4 * 2.0 ** -24 * 3e38 ** -0.5, "rstd")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [2 ** 25 - 24, 2 ** 25 + 40, 2 ** 26 + 40])
def test_layer_norm_backward_of_the_longest_rows(ops, dtype, cols):
    """Two launches' worth of parameter gradients and more.  Of two rows dbeta is one sum and dgamma one product and one sum, exact to their roundings."""
    say(f"layer norm backward {dtype} 2x{cols}")
    gen = torch.Generator(device="cuda").manual_seed(cols)
    dy = torch.randn(2, cols, generator=gen, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    c, xh = P.Checkpoint.empty(2, cols), torch.randn(2, cols, generator=gen, device="cuda")
    P.tensile_ckpt_pack(ops, xh, c)
    P.tensile_ckpt_unpack(ops, c, xh)
    g, rstd, dx = torch.ones(cols, device="cuda"), torch.ones(2, device="cuda"), torch.empty_like(dy)
    dg, db = torch.full_like(g, 7.0), torch.full_like(g, 7.0)
    P.tensile_layer_norm_backward(ops, dy, c, rstd, g, dx, dg, db)
    dy = dy.double()
    xh = xh.double()
    u = 2.0 ** -24
    assert bool(((db.double() - dy.sum(0)).abs() <= u * dy.sum(0).abs() * 1.01).all())
    assert bool(((dg.double() - (dy * xh).sum(0)).abs() <= 3 * u * (dy * xh).abs().sum(0)).all())
    want = dy - dy.mean(1, keepdim=True) - xh * (dy * xh).mean(1, keepdim=True)
    # the two means: chains of cols / 1024 / 8 additions in a thread, 8 in a chunk, 6 across lanes, 16 across wavefronts
    means = (cols / 8192 + 30) * u * (dy.abs().mean(1, keepdim=True) + xh.abs() * (dy * xh).abs().mean(1, keepdim=True))
    rounding = plain.ROUND[dtype] + 4 * u
    assert bool(((dx.double() - want).abs() <= rounding * want.abs() + means + 4 * u * (dy.abs() + xh.abs())).all())


# ------------------------------------------------------------------ gelu

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tanh", [False, True])
def test_gelu_of_infinities(ops, dtype, tanh):
    """x*Phi(x): inf at inf, NaN (a product with 0) at -inf; what is around them is finite and their group is lost."""
    for cols in (5, 64, 100):
        x = np.ones((3, cols))
        x[0, 1], x[1, 2], x[2, 3] = np.inf, -np.inf, np.nan
        xd = up(x, dtype)
        y, c = torch.empty_like(xd), P.Checkpoint.empty(3, cols)
        P.tensile_gelu(ops, xd, y, ckpt=c, tanh=tanh)
        got = host(y)
        assert got[0, 1] == np.inf and np.isnan(got[1, 2]) and np.isnan(got[2, 3])
        assert np.isfinite(got).sum() == got.size - 3
        assert np.array_equal(c.scale.cpu().numpy() == 255, np.arange((cols + 31) // 32)[None, :] == np.zeros((3, 1)))


def from_tails(x, tanh):
    """gelu in 64 bits from the tail 1 - P(|x|) of the form's distribution function P (1 + tanh and 1 + erf cancel where x is far below 0, in 64 bits too);
    -> value, derivative, the tail, exp(-x^2/2) or P, |2u| or 0"""
    from scipy.special import erfc
    a = np.abs(x)
    if tanh:
        k = np.sqrt(2 / np.pi)
        u2 = 2 * k * (a + 0.044715 * a ** 3)
        tail, e = 1 / (1 + np.exp(np.minimum(u2, 700))), 1 / (1 + np.exp(-u2))
        density = tail * e * 2 * k * (1 + 3 * 0.044715 * x * x)
    else:
        u2, tail, e = 0 * a, 0.5 * erfc(a / np.sqrt(2)), np.exp(-0.5 * a * a)
        density = e / np.sqrt(2 * np.pi)
    y, slope = np.maximum(x, 0) - a * tail, np.where(x < 0, tail, 1 - tail) + x * density
    for got, want in zip((y, slope), plain.gelu(x, tanh)):
        assert np.abs(got - want).max() < 1e-13
    return y, slope, tail, e, u2


@pytest.mark.parametrize("tanh", [False, True])
def test_gelu_to_32_bits(ops, tanh):
    """Errors counted in roundings, U = 2^-24 each; an exponential and a reciprocal are within 2.

    erf form: v has 5 (two products, a sum, a reciprocal), v*Q'(v) and its sum move R by at most 0.4 and 0.5 of that, so R is within 5 U absolutely,
    and R >= 0.35/(1 + |x|): 15 U (1 + |x|) relatively; exp(-x^2/2): three roundings of an exponent of x^2/2 and 2: 1.5 x^2 + 2; a product.
    tanh form: four roundings of the exponent |2u| and 2 of the exponential, three of t, a product.
    The derivative is 1 or 0 plus a product of the same numbers: e*(x/sqrt(2 pi) -+ R) or tail*(x*t*w -+ 1), w = d(2u)/dx, of 2 roundings more."""
    rng = np.random.default_rng(77)
    x = np.concatenate([np.linspace(-16, 16, 4096 - 7), [0.0, -0.0, 1e-20, -1e-20, 1e-3, -1e-3, 12.9], rng.standard_normal(4096), rng.standard_normal(4096) * 1e-2]).reshape(96, 128)
    xd = up(x)
    x = host(xd)
    y = torch.empty_like(xd)
    P.tensile_gelu(ops, xd, y, tanh=tanh)
    u, least = 2.0 ** -24, 1e-36                      # (a result below the normal numbers is 0: |x| * 2^-126)
    y0, _, tail, e, u2 = from_tails(x, tanh)
    a = np.abs(x)
    relative = (4 * u2 + 9) if tanh else 15 * (1 + a) + 1.5 * a * a + 4
    near(y, y0, 2 * u * np.abs(y0) + u * relative * a * tail + least, "gelu")

    c, v = filled(x)
    dy = torch.ones(x.shape, dtype=torch.float32, device="cuda")
    dx, yc = torch.empty_like(dy), P.Checkpoint.empty(*x.shape)
    P.tensile_gelu_backward(ops, dy, c, dx, y_ckpt=yc, tanh=tanh)
    _, slope, tail, e, u2 = from_tails(v, tanh)
    a = np.abs(v)
    if tanh:
        rest = a * e * (1.5957691216057308 + 0.21406444881780076 * v * v)                         # |x|*t*w; e is t here
        off = tail * ((4 * u2 + 8) * (rest + 1) + 8 * rest + 1)
    else:
        off = e * ((1.5 * a * a + 2) * (a * 0.3989422804014327 + 0.5) + 6 + a)
    near(dx, slope, 2 * u * np.abs(slope) + u * off + least, "derivative")


# ------------------------------------------------------------------ scratch memory

class PerThread:
    """hipStreamPerThread: the same value in every host thread, a queue of its own in each."""
    cuda_stream = 2


class Split:
    """A weight gradient whose rows are split, and a norm's backward pass: both leave partial sums in scratch memory."""

    def __init__(self, seed, M=4096, N=192, K=320):
        rng = np.random.default_rng(seed)
        self.dz, self.dy = up(rng.standard_normal((M, N)), "bf16"), up(rng.standard_normal((M, K)), "bf16")
        self.c, _ = filled(rng.standard_normal((M, K)))
        self.g, self.rstd = torch.ones(K, device="cuda"), torch.ones(M, device="cuda")
        self.out = [torch.empty(N, K, device="cuda"), torch.empty_like(self.dy), torch.empty_like(self.g), torch.empty_like(self.g)]

    def run(self, ops, stream=None):
        P.tensile_linear_grad(ops, self.dz, self.c, self.out[0], stream=stream)
        P.tensile_layer_norm_backward(ops, self.dy, self.c, self.rstd, self.g, *self.out[1:], stream=stream)

    def take(self):
        torch.cuda.synchronize()
        got = [t.clone() for t in self.out]
        for t in self.out:
            t.fill_(7.0)
        torch.cuda.synchronize()
        return got


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def in_thread(f):
    import threading
    result = []

    def run():
        try:
            result.append(f())
        except P.TensileError as e:
            result.append(e)
    t = threading.Thread(target=run)
    t.start()
    t.join()
    return result[0]


def test_the_per_thread_stream_has_scratch_for_each_thread(tuning):
    """A second thread's queue is another one: its call asks for memory of its own (refused here), not for the first thread's."""
    h, work = P.tensile_ops_create(), Split(1)
    work.run(h)
    want = work.take()
    work.run(h, PerThread)
    assert same(work.take(), want)
    tuning("alloc_fail", 1)
    refused = in_thread(lambda: work.run(h, PerThread))
    assert isinstance(refused, P.TensileError) and refused.code == P.binding.TENSILE_E_NOMEM
    work.run(h, PerThread)                             # this thread has its own already
    assert same(work.take(), want)
    assert in_thread(lambda: work.run(h, PerThread)) is None
    assert same(work.take(), want)
    h.close()


def test_threads_on_the_per_thread_stream(ops):
    import threading
    jobs = [Split(10 + k) for k in range(4)]
    want = []
    for j in jobs:
        j.run(ops)
        want.append(j.take())
    def many(j):
        for _ in range(20):
            j.run(ops, PerThread)
    threads = [threading.Thread(target=many, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for j, w in zip(jobs, want):
        assert same(j.take(), w)


def captured(ops, works, stream):
    """A graph of the works, one after the other, captured on the stream."""
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for w in works:
            w.run(ops, stream)
    return graph


def test_a_capture_has_scratch_of_its_own(tuning):
    """The calls of a capture ask for memory (refused here, once), whatever the stream had before; so do those of the next capture."""
    h, work, stream = P.tensile_ops_create(), Split(2), torch.cuda.Stream()
    work.run(h)
    want = work.take()
    work.run(h, stream)
    assert same(work.take(), want)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            tuning("alloc_fail", 1)
            try:
                work.run(h, stream)
                refused = 0
            except P.TensileError as e:
                refused = e.code
            tuning("alloc_fail", 0)
            work.run(h, stream)
        assert refused == P.binding.TENSILE_E_NOMEM
        graphs.append(graph)
    for graph in graphs * 3:
        graph.replay()
        assert same(work.take(), want)
        work.run(h, stream)
        assert same(work.take(), want)
    del graphs, graph
    h.close()


def test_a_capture_needs_no_earlier_call():
    h, work, stream = P.tensile_ops_create(), Split(3), torch.cuda.Stream()
    graph = captured(h, [work], stream)
    for _ in range(3):
        graph.replay()
        got = work.take()
        work.run(h)
        assert same(got, work.take())
    del graph
    h.close()


def test_graphs_of_one_stream_side_by_side_with_its_eager_calls(ops):
    """Two graphs captured on one stream, replayed on two others, while that stream and the current one run the same calls."""
    works = [Split(20 + k) for k in range(4)]
    want = []
    for w in works:
        w.run(ops)
        want.append(w.take())
    first, others = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    graphs = [captured(ops, [w], first) for w in works[:2]]
    for _ in range(20):
        torch.cuda.synchronize()
        for _ in range(4):
            for graph, s in zip(graphs, others):
                with torch.cuda.stream(s):
                    graph.replay()
            works[2].run(ops, first)
            works[3].run(ops)
        for w, t in zip(works, want):
            assert same(w.take(), t)


def test_a_capture_over_two_streams(ops):
    """Branches of one graph may run side by side: each has its own."""
    a, b = Split(30), Split(31)
    want = []
    for w in (a, b):
        w.run(ops)
        want.append(w.take())
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        a.run(ops, main)
        b.run(ops, side)
        main.wait_stream(side)
    for _ in range(10):
        graph.replay()
        assert same(a.take(), want[0])
        graph.replay()
        assert same(b.take(), want[1])


# ------------------------------------------------------------------ what a call is given

def test_a_checkpoint_that_is_moved(ops):
    """Its tensors may be replaced or be given other memory; none of the old is read.  (`held` keeps the old memory where it is.)"""
    c, v = filled(np.full((4, 70), 1.0))
    other, w = filled(np.full((4, 70), 1.5))
    held = c.q.view(4, 70), c.scale.view(4, 3)
    y = torch.empty(4, 70, device="cuda")

    def value():
        y.fill_(9.0)
        P.tensile_ckpt_unpack(ops, c, y)
        return host(y)

    assert np.array_equal(value(), v)
    c.q, c.scale = other.q, other.scale                # replaced
    assert np.array_equal(value(), w)
    c.q, c.scale = held
    assert np.array_equal(value(), v)
    c.q.set_(other.q)                                  # the same tensors in another place
    c.scale.set_(other.scale)
    assert np.array_equal(value(), w)
    kept = c.q.cpu(), c.scale.cpu()
    c.q, c.scale = kept                                # off the GPU: refused there ...
    with pytest.raises(P.TensileError) as e:
        P.tensile_ckpt_unpack(ops, c, y)
    assert e.value.code == P.binding.TENSILE_E_INVAL and "CUDA" in str(e.value)
    c.q, c.scale = (t.cuda() for t in kept)            # ... and back
    assert np.array_equal(value(), w) and c.shape == (4, 70)
    c.q = c.q[:2]                                      # half of it: the scales do not belong
    with pytest.raises(P.TensileError) as e:
        P.tensile_ckpt_unpack(ops, c, y[:2])
    assert "belong" in str(e.value)
    c.scale = c.scale[:2]
    P.tensile_ckpt_unpack(ops, c, y[:2])
    assert c.nbytes == 2 * (70 + 3)


def test_a_checkpoint_without_memory_is_refused(ops):
    c, y = P.Checkpoint(torch.ones(4, 64, dtype=torch.int8, device="cuda"), torch.ones(4, 2, dtype=torch.uint8, device="cuda")), torch.empty(4, 64, device="cuda")
    P.tensile_ckpt_unpack(ops, c, y)
    torch.cuda.synchronize()
    c.q.untyped_storage().resize_(0)
    with pytest.raises(P.TensileError) as e:
        P.tensile_ckpt_unpack(ops, c, y)
    assert e.value.code == P.binding.TENSILE_E_INVAL and "NULL" in str(e.value)


def every_call(ops, x, c, v, rstd, dw, db, stream=None):
    """One call of each entry point; x, dw: matrices, v: the norm's parameters, c: a checkpoint like x."""
    return {"ckpt_pack": lambda: P.tensile_ckpt_pack(ops, x, c, stream=stream),
            "ckpt_unpack": lambda: P.tensile_ckpt_unpack(ops, c, x, stream=stream),
            "layer_norm": lambda: P.tensile_layer_norm(ops, x, v, v, x, xhat=c, rstd=rstd, stream=stream),
            "layer_norm_backward": lambda: P.tensile_layer_norm_backward(ops, x, c, rstd, v, x, stream=stream),
            "gelu": lambda: P.tensile_gelu(ops, x, x, ckpt=c, stream=stream),
            "gelu_backward": lambda: P.tensile_gelu_backward(ops, x, c, x, stream=stream),
            "linear_grad": lambda: P.tensile_linear_grad(ops, x, c, dw, dbias=db, gamma=v, beta=v, stream=stream)}


def test_tensors_and_streams_of_another_device_are_refused(ops):
    """A kernel would follow their addresses on the handle's device.  (With a handle that says that it belongs to the next device: nothing gets as
    far as the library.)"""
    x, v, dw = torch.zeros(4, 64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, 64, device="cuda")
    c, rstd, db = P.Checkpoint.empty(4, 64), torch.zeros(4, device="cuda"), torch.zeros(64, device="cuda")
    elsewhere = P.OpsHandle(ops.ptr, ops.device + 1)
    try:
        for name, call in every_call(elsewhere, x, c, v, rstd, dw, db).items():
            with pytest.raises(P.TensileError) as e:
                call()
            assert e.value.code == P.binding.TENSILE_E_INVAL and "device" in str(e.value), name
        for check in (lambda: P.binding._mat(elsewhere.device, x, "x"), lambda: P.binding._vec(elsewhere.device, v, v.dtype, 64, "v"),
                      lambda: P.binding._ck(elsewhere.device, c), lambda: P.binding._stream_ptr(torch.cuda.Stream(), elsewhere)):
            with pytest.raises(P.TensileError) as e:
                check()
            assert "device" in str(e.value)
    finally:
        elsewhere._ptr = 0                             # (it is not this handle's to free)
    for name, call in every_call(ops, x, c, v, rstd, dw, db, stream=torch.cuda.Stream()).items():
        call()
    torch.cuda.synchronize()


def test_arguments_that_are_missing(ops):
    """None where a call needs a tensor is this library's error, like any other wrong argument."""
    x, v, dw = torch.zeros(4, 64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, 64, device="cuda")
    c, rstd = P.Checkpoint.empty(4, 64), torch.zeros(4, device="cuda")
    calls = {P.tensile_ckpt_pack: (x, c), P.tensile_ckpt_unpack: (c, x), P.tensile_layer_norm: (x, v, v, x), P.tensile_layer_norm_backward: (x, c, rstd, v, x),
             P.tensile_gelu: (x, x), P.tensile_gelu_backward: (x, c, x), P.tensile_linear_grad: (x, c, dw)}
    for call, args in calls.items():
        call(ops, *args)
        for k in range(len(args)):
            with pytest.raises(P.TensileError) as e:
                call(ops, *args[:k], None, *args[k + 1:])
            assert e.value.code == P.binding.TENSILE_E_INVAL, (call.__name__, k)
    for given in (dict(gamma=v), dict(beta=v)):
        with pytest.raises(P.TensileError):
            P.tensile_linear_grad(ops, x, c, dw, **given)
