"""Calls of the operators that are refused, without a GPU (host_calls.py): results that overlap what else a call reads or writes."""
import random

import pytest

from host_calls import BF16, F16, F32, SIZE, Host, ckpt, mat, ptr

G = 1 << 34                                             # places that are far from each other
INVAL = -1
SILU = 0


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    h = Host(tmp_path_factory.mktemp("host"))
    yield h
    h.close()


def allowed(reply):
    assert reply.code == 0 and reply.launches, reply


def refused(reply, message):
    assert reply.code == INVAL and reply.error == message and not reply.launches, reply


def place(k, rows, cols, **more):
    return ckpt(k * G, k * G + G // 2, rows, cols, **more)


# ------------------------------------------------------------------ gated layer

def gated(host, M=40, K=48, F=48, x=None, wg=None, wu=None, h=None, gate=None, up=None, type=BF16):
    return host("gated_linear", x or mat(1 * G, M, K, type=type), wg or mat(2 * G, F, K, type=type), wu or mat(3 * G, F, K, type=type), None, None, F32, SILU,
                h or mat(4 * G, M, F, type=type), gate, up)


def back(host, M=40, K=48, F=64, dh=None, gate=None, up=None, dgate=None, dup=None, h_c=None, wg=None, wu=None, dx=None, product=True):
    ws = (wg or mat(6 * G, F, K), wu or mat(7 * G, F, K), dx or mat(8 * G, M, K)) if product else (None, None, None)
    return host("gated_linear_backward", dh or mat(1 * G, M, F), gate or place(2, M, F), up or place(3, M, F), SILU, dgate or mat(4 * G, M, F),
                dup or mat(5 * G, M, F), h_c, *ws)


def test_a_gradient_in_the_place_of_dh_has_its_rows(host):
    M, F = 40, 64
    allowed(back(host, dgate=mat(G, M, F)))
    allowed(back(host, dup=mat(G, M, F)))
    allowed(back(host, dh=mat(G, M, F, 2 * F), dgate=mat(G, M, F, 2 * F), dup=mat(G + 2 * F, M, F, 2 * F)))
    # dh is contiguous, dgate the first half of a wider matrix that begins there: its row 1 is dh's row 2
    refused(back(host, dgate=mat(G, M, F, 2 * F)), "gated_linear_backward: dgate overlaps dh")
    refused(back(host, dup=mat(G, M, F, 2 * F)), "gated_linear_backward: dup overlaps dh")
    refused(back(host, dup=mat(G + 2 * F, M, F, 2 * F)), "gated_linear_backward: dup overlaps dh")         # (... the second half)
    refused(back(host, dh=mat(G, M, F, 2 * F), dgate=mat(G, M, F)), "gated_linear_backward: dgate overlaps dh")
    allowed(back(host, M=1, dh=mat(G, 1, F), dgate=mat(G, 1, F, 2 * F)))                                   # (one row)
    refused(back(host, dx=mat(G, M, 48)), "gated_linear_backward: dx overlaps dh")
    allowed(back(host, K=F, wg=mat(6 * G, F, F), wu=mat(7 * G, F, F), dx=mat(G, M, F)))
    refused(back(host, K=F, wg=mat(6 * G, F, F), wu=mat(7 * G, F, F), dx=mat(G, M, F, F + 8)), "gated_linear_backward: dx overlaps dh")
    refused(back(host, dx=mat(4 * G + 2, M, 48)), "gated_linear_backward: dgate overlaps dx")
    refused(back(host, dx=mat(5 * G + 2 * F, M, 48, 100)), "gated_linear_backward: dup overlaps dx")
    refused(back(host, dx=mat(7 * G + 6, M, 48)), "gated_linear_backward: dx overlaps w_up")


def test_a_checkpoint_in_the_place_of_another_is_all_of_it(host):
    M, F = 40, 64
    for product in (True, False):
        allowed(back(host, h_c=place(2, M, F), product=product))
        allowed(back(host, h_c=place(3, M, F), product=product))
        allowed(back(host, up=place(2, M, F), h_c=place(2, M, F), product=product))
        allowed(back(host, gate=place(2, M, F, ld_q=80, ld_scale=5), h_c=place(2, M, F, ld_q=80, ld_scale=5), product=product))
        refused(back(host, h_c=place(2, M, F, ld_q=80), product=product), "gated_linear_backward: h_c overlaps gate")
        refused(back(host, h_c=place(3, M, F, ld_scale=5), product=product), "gated_linear_backward: h_c overlaps up")
        refused(back(host, h_c=ckpt(2 * G, 9 * G, M, F), product=product), "gated_linear_backward: h_c overlaps gate")
        refused(back(host, h_c=ckpt(9 * G, 3 * G + G // 2, M, F), product=product), "gated_linear_backward: h_c.scale overlaps up.scale")
        refused(back(host, h_c=ckpt(2 * G, 3 * G + G // 2, M, F), product=product), "gated_linear_backward: h_c overlaps gate")
        refused(back(host, h_c=ckpt(4 * G, 9 * G, M, F), product=product), "gated_linear_backward: dgate overlaps h_c")


def test_h_and_its_checkpoints_lie_by_themselves(host):
    M, F = 40, 48
    allowed(gated(host))
    allowed(gated(host, gate=place(5, M, F), up=place(6, M, F)))
    refused(gated(host, h=mat(G, M, F)), "gated_linear: h is x or a weight matrix")
    refused(gated(host, h=mat(G + 2, M, F)), "gated_linear: h overlaps x")
    refused(gated(host, h=mat(G + 8, M, F, 200)), "gated_linear: h overlaps x")
    refused(gated(host, h=mat(3 * G - 64, M, F)), "gated_linear: h overlaps w_up")
    refused(gated(host, gate=ckpt(4 * G, 9 * G, M, F)), "gated_linear: h overlaps gate")
    refused(gated(host, up=ckpt(9 * G, 2 * G + 7, M, F)), "gated_linear: up.scale overlaps w_gate")
    refused(gated(host, gate=ckpt(5 * G, 5 * G + 40, M, F)), "gated_linear: gate overlaps gate.scale")
    refused(gated(host, gate=place(5, M, F), up=ckpt(5 * G + 8, 9 * G, M, F)), "gated_linear: gate overlaps up")
    # the two halves of a matrix's columns, and rows that take turns with those of x
    allowed(gated(host, x=mat(G, M, 48, 96), h=mat(G + 96, M, F, 96)))
    allowed(gated(host, x=mat(G, M, 48, 100), h=mat(G + 98, M, F, 100)))
    refused(gated(host, x=mat(G, M, 48, 96), h=mat(G + 94, M, F, 96)), "gated_linear: h overlaps x")
    refused(gated(host, x=mat(G, M, 48, 96), h=mat(G + 98, M, F, 96)), "gated_linear: h overlaps x")
    allowed(gated(host, x=mat(G, M, 48, 96), h=mat(G + 96 + 192 * (M - 1), M, F, 96)))
    allowed(gated(host, M=1, x=mat(G, 1, 48), h=mat(G + 96, 1, F)))


def test_overlaps_are_those_of_the_bytes(host):
    """Random places, against the sets of bytes."""
    rng = random.Random(4)
    met = 0
    for _ in range(600):
        M, K, F, type = rng.randint(1, 6), rng.randint(1, 5), rng.randint(1, 5), rng.choice([BF16, F32])
        size = SIZE[type]
        ld_x = rng.choice([K, K + rng.randint(0, 12), 12])
        ld_h = rng.choice([F, F + rng.randint(0, 12), 12, max(ld_x, F)])
        at = G + size * rng.randint(-30, 60)
        row = lambda begin, ld, n: {b for r in range(M) for b in range(begin + r * ld * size, begin + (r * ld + n) * size)}
        meets = bool(row(G, ld_x, K) & row(at, ld_h, F))
        reply = gated(host, M, K, F, x=mat(G, M, K, ld_x, type), h=mat(at, M, F, ld_h, type), type=type)
        assert (reply.code == INVAL) == meets and bool(reply.launches) != meets, (M, K, F, ld_x, ld_h, at - G, reply)
        if meets:
            assert reply.error in ("gated_linear: h overlaps x", "gated_linear: h is x or a weight matrix")
        met += meets
    assert 100 < met < 500


# ------------------------------------------------------------------ norms

def norm(host, name="rms_norm", M=40, K=48, x=None, residual=None, y=None, total=None, xhat=None):
    params = [ptr(9 * G)] if name == "rms_norm" else [ptr(9 * G), ptr(10 * G)]
    return host(name, x or mat(1 * G, M, K), residual, *params, F32, 1e-6, y or mat(3 * G, M, K), total, xhat, ptr(8 * G))


def norm_back(host, name="rms_norm_backward", M=40, K=48, dy=None, xhat=None, dresidual=None, dx=None):
    params = [ptr(10 * G)] if name == "rms_norm_backward" else [ptr(10 * G), ptr(11 * G)]
    return host(name, dy or mat(1 * G, M, K), xhat or place(2, M, K), ptr(8 * G), ptr(9 * G), F32, dresidual, dx or mat(4 * G, M, K), *params)


@pytest.mark.parametrize("name", ["rms_norm", "layer_norm"])
def test_a_norm_in_place_has_its_inputs_rows(host, name):
    M, K = 40, 48
    call = lambda **a: norm(host, name, **a)
    r = mat(2 * G, M, K, 60)
    allowed(call(residual=r, total=mat(4 * G, M, K), xhat=place(5, M, K)))
    allowed(call(y=mat(G, M, K)))
    allowed(call(residual=r, y=r, total=mat(G, M, K)))
    allowed(call(residual=mat(G, M, K), y=mat(G, M, K)))
    allowed(call(M=1, y=mat(G, 1, K, 100)))
    allowed(call(x=mat(G, M, K, 96), y=mat(G + 96, M, K, 96)))
    refused(call(y=mat(G, M, K, 56)), f"{name}: y overlaps x")
    refused(call(x=mat(G, M, K, 56), y=mat(G, M, K)), f"{name}: y overlaps x")
    refused(call(residual=r, y=mat(2 * G, M, K)), f"{name}: y overlaps residual")
    refused(call(residual=r, total=mat(2 * G, M, K)), f"{name}: total overlaps residual")
    refused(call(total=mat(G, M, K, 64)), f"{name}: total overlaps x")
    refused(call(total=mat(3 * G, M, K, 64)), f"{name}: total is y")
    refused(call(total=mat(3 * G + 8, M, K, 64)), f"{name}: y overlaps total")
    refused(call(y=mat(G + 2, M, K)), f"{name}: y overlaps x")
    refused(call(xhat=ckpt(G, 6 * G, M, K)), f"{name}: xhat overlaps x")
    refused(call(xhat=ckpt(6 * G, 3 * G + 5, M, K)), f"{name}: y overlaps xhat.scale")
    refused(call(xhat=ckpt(6 * G, 6 * G + 47, M, K)), f"{name}: xhat overlaps xhat.scale")


@pytest.mark.parametrize("name", ["rms_norm_backward", "layer_norm_backward"])
def test_a_norms_gradient_in_place_has_its_rows(host, name):
    M, K = 40, 48
    call = lambda **a: norm_back(host, name, **a)
    d = mat(3 * G, M, K, 60)
    allowed(call(dresidual=d))
    allowed(call(dx=mat(G, M, K)))
    allowed(call(dresidual=d, dx=d))
    allowed(call(dresidual=mat(G, M, K), dx=mat(G, M, K)))
    allowed(call(M=1, dx=mat(G, 1, K, 100)))
    refused(call(dx=mat(G, M, K, 56)), f"{name}: dx overlaps dy")
    refused(call(dresidual=d, dx=mat(3 * G, M, K)), f"{name}: dx overlaps dresidual")
    refused(call(dresidual=mat(G, M, K), dy=mat(5 * G, M, K), dx=mat(G + 4, M, K)), f"{name}: dx overlaps dresidual")
    refused(call(dx=mat(2 * G - 2, M, K)), f"{name}: dx overlaps xhat")
    refused(call(dx=mat(2 * G + G // 2 + 2, M, K)), f"{name}: dx overlaps xhat.scale")


# ------------------------------------------------------------------ elementwise calls and the weight gradient

def test_elementwise_calls_in_place_have_their_inputs_rows(host):
    M, K = 40, 48
    x, c = mat(G, M, K), place(2, M, K)
    gelu = lambda **a: host("gelu", a.get("x", x), a.get("y", mat(3 * G, M, K)), a.get("c"), 0)
    allowed(gelu(c=c))
    allowed(gelu(y=x))
    allowed(gelu(x=mat(G, M, K, 96), y=mat(G + 96, M, K, 96)))
    refused(gelu(y=mat(G, M, K, 56)), "gelu: y overlaps x")
    refused(gelu(y=mat(G + 2, M, K)), "gelu: y overlaps x")
    refused(gelu(c=ckpt(G + 1, 9 * G, M, K)), "gelu: c overlaps x")
    refused(gelu(c=ckpt(9 * G, 3 * G + 1, M, K)), "gelu: c.scale overlaps y")
    refused(gelu(c=ckpt(9 * G, 9 * G + 1, M, K)), "gelu: c overlaps c.scale")
    back = lambda **a: host("gelu_backward", a.get("dy", x), a.get("c", c), a.get("dx", mat(3 * G, M, K)), a.get("y_c"), 0)
    allowed(back(y_c=place(4, M, K)))
    allowed(back(y_c=c, dx=x))
    refused(back(dx=mat(G, M, K, 56)), "gelu_backward: dx overlaps dy")
    refused(back(y_c=place(2, M, K, ld_q=64)), "gelu_backward: y_c overlaps c")
    refused(back(y_c=place(2, M, K, ld_scale=4)), "gelu_backward: y_c overlaps c")
    refused(back(y_c=ckpt(2 * G, 9 * G, M, K)), "gelu_backward: y_c overlaps c")
    refused(back(y_c=ckpt(9 * G, 2 * G + G // 2, M, K)), "gelu_backward: y_c.scale overlaps c.scale")
    refused(back(y_c=ckpt(9 * G, 3 * G, M, K)), "gelu_backward: y_c.scale overlaps dx")
    allowed(host("ckpt_pack", x, c))
    refused(host("ckpt_pack", x, ckpt(G, 9 * G, M, K)), "ckpt_pack: c overlaps x")
    refused(host("ckpt_pack", x, ckpt(9 * G, G + 2 * M * K - 1, M, K)), "ckpt_pack: c.scale overlaps x")
    allowed(host("ckpt_pack", x, ckpt(9 * G, G + 2 * M * K, M, K)))
    allowed(host("ckpt_unpack", c, x))
    refused(host("ckpt_unpack", ckpt(G, 9 * G, M, K), x), "ckpt_unpack: y overlaps c")


def test_a_weight_gradient_lies_by_itself(host):
    M, N, K = 40, 24, 48
    grad = lambda dw: host("linear_grad", mat(G, M, N), place(2, M, K), None, None, F32, dw, None)
    allowed(grad(mat(3 * G, N, K)))
    refused(grad(mat(G, N, K)), "linear_grad: dw overlaps dy")
    refused(grad(mat(2 * G + 4, N, K)), "linear_grad: dw overlaps c")
    refused(grad(mat(2 * G + G // 2, N, K, type=F32)), "linear_grad: dw overlaps c.scale")


# ------------------------------------------------------------------ every argument by its name, and the reason

def test_norm_refusals_name_the_argument(host):
    M, K = 4, 64
    x, g, y = mat(G, M, K), ptr(9 * G), mat(3 * G, M, K)
    full = dict(x=x, residual=None, gamma=g, param=F32, eps=1e-6, y=y, total=None, xhat=None, rstd=ptr(8 * G))

    def call(**a):
        a = {**full, **a}
        return host("rms_norm", a["x"], a["residual"], a["gamma"], a["param"], a["eps"], a["y"], a["total"], a["xhat"], a["rstd"])
    allowed(call())
    for args, message in [(dict(x=None), "x is NULL"), (dict(y=None), "y is NULL"), (dict(gamma=None), "gamma is NULL"),
                          (dict(x=mat(0, M, K)), "x has no data (NULL)"), (dict(x=mat(G, M, K, type=7)), "x has an unknown type"),
                          (dict(x=mat(G + 1, M, K)), "x is not aligned to its elements"), (dict(x=mat(G, M, K, K - 1)), "x has rows that overlap (ld < cols)"),
                          (dict(x=mat(G, M, 0, 1)), "x needs rows >= 0 and cols >= 1"), (dict(x=mat(G, -1, K)), "x needs rows >= 0 and cols >= 1"),
                          (dict(y=mat(3 * G, M, K, type=F16)), "y differs in shape or type"), (dict(y=mat(3 * G, M, K - 1)), "y differs in shape or type"),
                          (dict(y=mat(3 * G + 1, M, K)), "y is not aligned to its elements"), (dict(residual=mat(2 * G, M + 1, K)), "residual differs in shape or type"),
                          (dict(total=mat(2 * G, M, K, type=F32)), "total differs in shape or type"), (dict(total=y), "total is y"),
                          (dict(xhat=place(2, M, K - 1)), "xhat differs in shape"), (dict(xhat=ckpt(2 * G, 0, M, K)), "xhat has no data (NULL)"),
                          (dict(xhat=place(2, M, K, ld_scale=1)), "xhat has rows that overlap (ld < cols)"),
                          (dict(param=F16), "param_type is neither TENSILE_F32 nor the activations' type"), (dict(gamma=ptr(9 * G + 2)), "gamma is not aligned to its elements"),
                          (dict(eps=-1.0), "eps is negative or not a finite 32-bit number"), (dict(eps=1e39), "eps is negative or not a finite 32-bit number")]:
        refused(call(**args), "rms_norm: " + message)

    full_b = dict(dy=x, xhat=place(2, M, K), rstd=ptr(8 * G), gamma=g, param=F32, dresidual=None, dx=y, dgamma=ptr(7 * G))

    def back_call(**a):
        a = {**full_b, **a}
        return host("rms_norm_backward", a["dy"], a["xhat"], a["rstd"], a["gamma"], a["param"], a["dresidual"], a["dx"], a["dgamma"])
    allowed(back_call())
    allowed(back_call(dgamma=None))
    for args, message in [(dict(dy=None), "dy is NULL"), (dict(xhat=None), "xhat is NULL"), (dict(rstd=None), "rstd is NULL"), (dict(gamma=None), "gamma is NULL"),
                          (dict(dx=None), "dx is NULL"), (dict(xhat=place(2, M, K + 1)), "xhat differs in shape"), (dict(dx=mat(3 * G, M, K + 1)), "dx differs in shape or type"),
                          (dict(dresidual=mat(4 * G, M, K, type=F32)), "dresidual differs in shape or type"), (dict(dgamma=ptr(7 * G + 2)), "dgamma is not aligned to its elements"),
                          (dict(param=7), "param_type is neither TENSILE_F32 nor the activations' type")]:
        refused(back_call(**args), "rms_norm_backward: " + message)


def test_gated_refusals_name_the_argument(host):
    M, K, F = 4, 64, 32
    x, w, v, h = mat(G, M, K), mat(2 * G, F, K), mat(3 * G, F, K), mat(4 * G, M, F)
    full = dict(x=x, wg=w, wu=v, bg=None, bu=None, param=F32, act=SILU, h=h, gate=None, up=None)

    def call(**a):
        a = {**full, **a}
        return host("gated_linear", *[a[n] for n in ("x", "wg", "wu", "bg", "bu", "param", "act", "h", "gate", "up")])
    allowed(call())
    allowed(call(bg=ptr(5 * G), bu=ptr(6 * G), gate=place(7, M, F), up=place(8, M, F)))
    allowed(call(wu=w))                                                 # (weights may be one matrix: they are only read)
    size = "is not (rows of x) x (rows of w_gate), or not of x's type"
    for args, message in [(dict(x=None), "x is NULL"), (dict(wg=None), "w_gate is NULL"), (dict(wu=None), "w_up is NULL"), (dict(h=None), "h is NULL"),
                          (dict(wu=mat(3 * G, F - 1, K)), "w_up differs in shape or type"), (dict(wg=mat(2 * G, F, K - 1), wu=mat(3 * G, F, K - 1)), "w_gate has not the columns of x"),
                          (dict(wg=mat(2 * G, F, K, type=F16), wu=mat(3 * G, F, K, type=F16)), "w_gate is not of x's type"),
                          (dict(wg=mat(2 * G, 0, K), wu=mat(3 * G, 0, K)), "w_gate has no rows"), (dict(h=mat(4 * G, M, F + 1)), "h " + size),
                          (dict(h=mat(4 * G, M + 1, F)), "h " + size), (dict(h=mat(4 * G, M, F, type=F32)), "h " + size), (dict(h=mat(4 * G + 1, M, F)), "h is not aligned to its elements"),
                          (dict(h=mat(G, M, F)), "h is x or a weight matrix"), (dict(h=mat(3 * G, M, F)), "h is x or a weight matrix"),
                          (dict(bg=ptr(5 * G)), "b_gate, b_up are given one without the other"), (dict(bu=ptr(5 * G)), "b_gate, b_up are given one without the other"),
                          (dict(bg=ptr(5 * G), bu=ptr(6 * G), param=F16), "param_type is neither TENSILE_F32 nor the activations' type"),
                          (dict(bg=ptr(5 * G + 2), bu=ptr(6 * G)), "b_gate is not aligned to its elements"), (dict(bg=ptr(5 * G), bu=ptr(6 * G + 1)), "b_up is not aligned to its elements"),
                          (dict(act=3), "activation is not one of TENSILE_SILU, TENSILE_GELU, TENSILE_GELU_TANH"),
                          (dict(act=-1), "activation is not one of TENSILE_SILU, TENSILE_GELU, TENSILE_GELU_TANH"),
                          (dict(gate=place(7, M, F - 1)), "gate differs in shape"), (dict(up=place(7, M - 1, F)), "up differs in shape"),
                          (dict(gate=place(7, M, F), up=place(7, M, F)), "up is gate")]:
        refused(call(**args), "gated_linear: " + message)

    dh, gate, up, dgate, dup = h, place(5, M, F), place(6, M, F), mat(7 * G, M, F), mat(8 * G, M, F)
    full_b = dict(dh=dh, gate=gate, up=up, act=SILU, dgate=dgate, dup=dup, h_c=None, wg=w, wu=v, dx=mat(9 * G, M, K))

    def back_call(**a):
        a = {**full_b, **a}
        return host("gated_linear_backward", *[a[n] for n in ("dh", "gate", "up", "act", "dgate", "dup", "h_c", "wg", "wu", "dx")])
    allowed(back_call())
    allowed(back_call(wg=None, wu=None, dx=None))
    together, like_w = "w_gate, w_up, dx are given one without the others", "w_gate has not a row for each column of dh, or is not of dh's type"
    for args, message in [(dict(dh=None), "dh is NULL"), (dict(gate=None), "gate is NULL"), (dict(up=None), "up is NULL"), (dict(dgate=None), "dgate is NULL"), (dict(dup=None), "dup is NULL"),
                          (dict(gate=place(5, M, F + 1)), "gate differs in shape"), (dict(up=place(6, M + 1, F)), "up differs in shape"), (dict(h_c=place(1, M, F - 1)), "h_c differs in shape"),
                          (dict(dgate=mat(7 * G, M, F + 1)), "dgate differs in shape or type"), (dict(dup=mat(8 * G, M, F, type=F16)), "dup differs in shape or type"),
                          (dict(dup=dgate), "dup is dgate"), (dict(act=5), "activation is not one of TENSILE_SILU, TENSILE_GELU, TENSILE_GELU_TANH"),
                          (dict(dx=None), together), (dict(wg=None), together), (dict(wu=None), together), (dict(wg=None, wu=None), together), (dict(wu=None, dx=None), together),
                          (dict(wg=mat(2 * G, F - 1, K), wu=mat(3 * G, F - 1, K)), like_w), (dict(wg=mat(2 * G, F, K, type=F32), wu=mat(3 * G, F, K, type=F32)), like_w),
                          (dict(wu=mat(3 * G, F, K + 1)), "w_up differs in shape or type"),
                          (dict(dx=mat(9 * G, M, K - 1)), "dx is not (rows of dh) x (columns of w_gate), or not of dh's type"),
                          (dict(dx=mat(9 * G, M, K, type=F16)), "dx is not (rows of dh) x (columns of w_gate), or not of dh's type"),
                          (dict(dx=mat(7 * G, M, K)), "dx is dgate, dup or a weight matrix"), (dict(dx=mat(3 * G, M, K)), "dx is dgate, dup or a weight matrix")]:
        refused(back_call(**args), "gated_linear_backward: " + message)
