"""Timed cases of the operators of a gated feed-forward network with its activations kept in 8 bits: the root-mean-square norm
with the residual's addition, and the gated layer behind it (two projections, an activation and a product), each with
its backward pass.

    xhat = s/sqrt(mean(s^2) + eps), s = x + residual;   y = xhat*gamma
    g = x Wg^T + bg;  u = x Wu^T + bu;   h = act(g)*u

Kept are xhat, g and u as checkpoints: signed bytes of which 32 consecutive values of a row share a power-of-two scale.  What
is held that way is returned as the values it stands for.  Sizes are those of the networks in ``workloads.models`` (an
encoder of width 768 with 16 x 512 tokens, a perceptron on 784 features, batch 32) and generic ones around them; a gated layer
has 8/3 of its input's features, up to the next multiple of 64.

``run`` computes an operator from elementary torch operations in 32 bits, or, where ``own`` is true, through this
package; ``exact`` states it once more in 64 bits.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GROUP = 32
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases

def _case(op, M, K, N=0, dtype="bf16", residual=False, total=False, ckpt=True, param="f32", act="silu", bias=False):
    """M tokens (rows), K features in, N of the gated layer.  residual: a second input (or an incoming gradient) is added; total: the
    sum is an output as well; ckpt: the call leaves checkpoints; param: the type of the norm's weights and of biases."""
    return {"op": op, "M": M, "K": K, "N": N, "dtype": dtype, "residual": residual, "total": total, "ckpt": ckpt, "param": param,
            "act": act, "bias": bias}


def listed():
    return [
        # one token answered: nothing is kept; what a call costs
        dict(_case("rms_norm", 1, 4_096, residual=True, total=True, ckpt=False, param="bf16"), name="rms norm 1x4096"),
        # a norm between two blocks, 16 sequences of 512 tokens: the sum goes on beside it
        dict(_case("rms_norm", 8_192, 768, residual=True, total=True), name="rms norm 8192x768"),
        # ... and its backward pass, where the residual path's gradient joins
        dict(_case("rms_norm_backward", 8_192, 768, residual=True), name="rms norm backward 8192x768"),
        # a wide network, an odd number of tokens
        dict(_case("rms_norm_backward", 16_381, 8_192, residual=True, param="bf16"), name="rms norm backward 16381x8192"),
        # one token answered by a wide layer: the weights are read once
        dict(_case("gated", 1, 4_096, 10_944, ckpt=False), name="gated 1x4096x10944"),
        # two dozen sequences answered at once, in half precision
        dict(_case("gated", 24, 4_096, 10_944, dtype="f16", ckpt=False), name="gated f16 24x4096x10944"),
        # the perceptron's first layer as a gated one, batch 32
        dict(_case("gated", 32, 784, 512, dtype="f32", act="gelu", bias=True), name="gated f32 32x784x512"),
        # training: the encoder's width
        dict(_case("gated", 8_192, 768, 2_048), name="gated 8192x768x2048"),
        # training: a wide layer, 16 sequences
        dict(_case("gated", 8_192, 4_096, 10_944, act="gelu_tanh"), name="gated 8192x4096x10944"),
        # backward passes: a short, odd batch in half precision
        dict(_case("gated_backward", 301, 1_000, 1_500, dtype="f16", act="gelu"), name="gated backward f16 301x1000x1500"),
        # ... the encoder's width
        dict(_case("gated_backward", 8_192, 768, 2_048), name="gated backward 8192x768x2048"),
        # ... a wide layer
        dict(_case("gated_backward", 8_192, 4_096, 10_944, act="gelu_tanh"), name="gated backward 8192x4096x10944"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rms_norm", "rms_norm_backward", "gated", "gated", "gated_backward", "gated_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    N = 0
    if op in ("gated", "gated_backward"):
        # (products in 32 bits take a multiple of the time)
        K, N = _log(rng, 16, 4_096), _log(rng, 16, 10_944)
        M = _log(rng, 1, 8_192 if dtype != "f32" else max(1, min(8_192, int(3e10 / (K * N)))))
    else:
        K = _log(rng, 16, 16_384)
        M = _log(rng, 1, min(65_536, (67e6 if dtype == "f32" else 134e6) / K))
    if rng.random() < 0.4:                             # ragged sizes are common, but so are even ones
        K, N, M = [max(1, v // 64 * 64) if v >= 64 else v for v in (K, N, M)]
    c = _case(op, M, K, N, dtype)
    c["residual"] = op in ("rms_norm", "rms_norm_backward") and rng.random() < 0.6
    c["total"] = op == "rms_norm" and c["residual"] and rng.random() < 0.6
    c["ckpt"] = op == "rms_norm_backward" or rng.random() < 0.7
    c["param"] = rng.choice(["f32", dtype])
    c["act"] = rng.choice(["silu", "silu", "gelu", "gelu_tanh"])
    c["bias"] = op == "gated" and rng.random() < 0.4
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _activations(gen, M, K):
    """Tokens of differing size, some features a few times larger than the others."""
    feature = torch.where(torch.rand(K, generator=gen, device="cuda") < 0.01, 6.0, 1.0)
    return _normal(gen, M, K) * feature * (0.5 + torch.rand(M, 1, generator=gen, device="cuda"))


def _gradients(gen, M, K, scale=1e-2):
    return _normal(gen, M, K) * (scale * (0.25 + torch.rand(M, 1, generator=gen, device="cuda")))


def _empty_checkpoint(M, K):
    return (torch.empty(M, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda")[:, :K],
            torch.empty(M, (K + GROUP - 1) // GROUP, dtype=torch.uint8, device="cuda"))


def _packed(v, dtype):
    """The bytes and scale codes of a checkpoint of v, in the buffers a program would hold them in."""
    q, code = _empty_checkpoint(*v.shape)
    _, byte, c = _quantised(v, dtype)
    q.copy_(byte)
    code.copy_(c)
    return q, code


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, M, K, N, T = case["op"], case["M"], case["K"], case["N"], TYPES[case["dtype"]]
    P = TYPES[case["param"]]
    s = dict(case)
    out = lambda *shape, dtype=T: torch.empty(*shape, dtype=dtype, device="cuda")
    weights = lambda n, k: (_normal(gen, n, k) * k ** -0.5).to(T)
    if op == "rms_norm":
        s["x"] = _activations(gen, M, K).to(T)
        s["r"] = _activations(gen, M, K).to(T) if case["residual"] else None
        s["gamma"] = (1 + 0.1 * _normal(gen, K)).to(P)
        s["y"], s["rstd"] = out(M, K), out(M, dtype=torch.float32)
        s["total_out"] = out(M, K) if case["total"] else None
        if case["ckpt"]:
            s["q"], s["code"] = _empty_checkpoint(M, K)
            s["value"] = out(M, K, dtype=torch.bfloat16)
    elif op == "rms_norm_backward":
        s["dy"] = _gradients(gen, M, K).to(T)
        s["dr"] = _gradients(gen, M, K).to(T) if case["residual"] else None
        x = _activations(gen, M, K)
        s["rstd"] = (x.square().mean(1) + EPS).rsqrt()
        s["q"], s["code"] = _packed(x * s["rstd"][:, None], T)
        s["gamma"] = (1 + 0.1 * _normal(gen, K)).to(P)
        s["dx"], s["dgamma"] = out(M, K), out(K, dtype=P)
    elif op == "gated":
        s["x"] = _activations(gen, M, K).to(T)
        s["wg"], s["wu"] = weights(N, K), weights(N, K)
        s["bg"], s["bu"] = [(0.1 * _normal(gen, N)).to(P) for _ in range(2)] if case["bias"] else (None, None)
        s["h"] = out(M, N)
        if case["ckpt"]:
            for name in ("g", "u"):
                s["q" + name], s["code" + name] = _empty_checkpoint(M, N)
                s["value" + name] = out(M, N, dtype=torch.bfloat16)
    else:
        s["dh"] = _gradients(gen, M, N).to(T)
        for name in ("g", "u"):
            s["q" + name], s["code" + name] = _packed(_activations(gen, M, N), T)
            s["w" + name] = weights(N, K)
            s["d" + name] = out(M, N)
        s["dx"] = out(M, K)
        if case["ckpt"]:
            s["q"], s["code"] = _empty_checkpoint(M, N)
            s["value"] = out(M, N, dtype=torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _quantised(v, dtype):
    """(values, bytes, codes) of a checkpoint of v (32 bits): the scale is the smallest power of two that leaves the
    largest of the group's quotients below 127.5, within the powers whose products are normal numbers and finite."""
    M, K = v.shape
    g = torch.nn.functional.pad(v, (0, -K % GROUP)).view(M, -1, GROUP)
    bits = g.abs().amax(2).view(torch.int32)
    code = (((bits + 0x10000) >> 23) - 6).clamp(1, 136 if dtype == torch.float16 else 248)
    code = torch.where(bits >= 0x7F800000, 255, code)
    scale = ((254 - code.clamp(max=253)) << 23).view(torch.float32)          # 2^(127 - code)
    q = (g * scale[:, :, None]).round().clamp(-127, 127).nan_to_num(0.0)
    value = _values(q.view(M, -1)[:, :K], code, K)
    return value, q.view(M, -1)[:, :K], code


def _values(q, code, K):
    scale = torch.where(code == 255, math.nan, (code.int() << 23).view(torch.float32))
    return q.float() * scale.repeat_interleave(GROUP, 1)[:, :K]


def _act(x, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return x * p, p * (1 + x * (1 - p))
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (x + 0.044715 * x * x * x))
        return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)
    p = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
    return x * p, p + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _plain(s):
    op, T = s["op"], TYPES[s["dtype"]]
    f = lambda name: None if s.get(name) is None else s[name].float()
    if op == "rms_norm":
        v = f("x") if s["r"] is None else f("x") + f("r")
        rstd = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
        xhat = v * rstd
        out = {"y": (xhat * f("gamma")).to(T), "rstd": rstd[:, 0]}
        if s["total"]:
            out["total"] = v.to(T)
        if s["ckpt"]:
            out["xhat"] = _quantised(xhat, T)[0].to(torch.bfloat16)
        return out
    if op == "rms_norm_backward":
        dy, xhat = f("dy"), _values(s["q"], s["code"], s["K"])
        g = dy * f("gamma")
        dx = s["rstd"][:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dr"] is not None:
            dx = dx + f("dr")
        return {"dx": dx.to(T), "dgamma": (dy * xhat).sum(0).to(TYPES[s["param"]])}
    if op == "gated":
        x = f("x")
        g, u = x @ f("wg").t(), x @ f("wu").t()
        if s["bias"]:
            g, u = g + f("bg"), u + f("bu")
        out = {"h": (_act(g, s["act"])[0] * u).to(T)}
        if s["ckpt"]:
            out["g"], out["u"] = (_quantised(v, T)[0].to(torch.bfloat16) for v in (g, u))
        return out
    g, u = (_values(s["q" + n], s["code" + n], s["N"]) for n in ("g", "u"))
    dh = f("dh")
    a, slope = _act(g, s["act"])
    dg, du = dh * u * slope, dh * a
    out = {"dg": dg.to(T), "du": du.to(T), "dx": (dg @ f("wg") + du @ f("wu")).to(T)}
    if s["ckpt"]:
        out["h"] = _quantised(a * u, T)[0].to(torch.bfloat16)
    return out


# ------------------------------------------------------------------------------------------------ the package's operators

@functools.lru_cache(maxsize=1)
def _package():
    import paper_2105_13336_amd as P
    return P, P.tensile_ops_create()


def _own(s):
    P, ops = _package()
    op = s["op"]
    if op == "rms_norm":
        c = P.Checkpoint(s["q"], s["code"]) if s["ckpt"] else None
        P.tensile_rms_norm(ops, s["x"], s["gamma"], s["y"], eps=EPS, residual=s["r"], total=s["total_out"], xhat=c, rstd=s["rstd"])
        out = {"y": s["y"], "rstd": s["rstd"]}
        if s["total"]:
            out["total"] = s["total_out"]
        if c is not None:
            P.tensile_ckpt_unpack(ops, c, s["value"])
            out["xhat"] = s["value"]
        return out
    if op == "rms_norm_backward":
        P.tensile_rms_norm_backward(ops, s["dy"], P.Checkpoint(s["q"], s["code"]), s["rstd"], s["gamma"], s["dx"], s["dgamma"],
                                    dresidual=s["dr"])
        return {"dx": s["dx"], "dgamma": s["dgamma"]}
    if op == "gated":
        g, u = (P.Checkpoint(s["q" + n], s["code" + n]) if s["ckpt"] else None for n in ("g", "u"))
        P.tensile_gated_linear(ops, s["x"], s["wg"], s["wu"], s["h"], b_gate=s["bg"], b_up=s["bu"], act=s["act"], gate=g, up=u)
        out = {"h": s["h"]}
        if s["ckpt"]:
            for n, c in (("g", g), ("u", u)):
                P.tensile_ckpt_unpack(ops, c, s["value" + n])
                out[n] = s["value" + n]
        return out
    g, u = (P.Checkpoint(s["q" + n], s["code" + n]) for n in ("g", "u"))
    c = P.Checkpoint(s["q"], s["code"]) if s["ckpt"] else None
    P.tensile_gated_linear_backward(ops, s["dh"], g, u, s["dg"], s["du"], w_gate=s["wg"], w_up=s["wu"], dx=s["dx"], act=s["act"], h_ckpt=c)
    out = {"dg": s["dg"], "du": s["du"], "dx": s["dx"]}
    if c is not None:
        P.tensile_ckpt_unpack(ops, c, s["value"])
        out["h"] = s["value"]
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ what it takes, and what is right

def work(case):
    """Each input read once, each output written once; a checkpoint that is made is written, what is restored from it too."""
    op, M, K, N, b, p = case["op"], case["M"], case["K"], case["N"], BYTES[case["dtype"]], BYTES[case["param"]]
    held = lambda rows, cols: rows * cols + rows * ((cols + GROUP - 1) // GROUP)
    kept = lambda rows, cols: held(rows, cols) + 2 * rows * cols if case["ckpt"] else 0
    if op == "rms_norm":
        return {"bytes": b * M * K * (2 + case["residual"] + case["total"]) + 4 * M + K * p + kept(M, K), "flops": 5 * M * K}
    if op == "rms_norm_backward":
        return {"bytes": b * M * K * (2 + case["residual"]) + held(M, K) + 4 * M + 2 * K * p, "flops": 9 * M * K}
    if op == "gated":
        return {"bytes": b * (M * K + 2 * N * K + M * N) + 2 * N * p * case["bias"] + 2 * kept(M, N), "flops": 4 * M * N * K + 12 * M * N}
    return {"bytes": b * (3 * M * N + 2 * N * K + M * K) + 2 * held(M, N) + kept(M, N), "flops": 4 * M * N * K + 20 * M * N}


def exact(case, seed):
    """In 64 bits, from the definitions, checkpoints among them: what they hold of values known to 64 bits."""
    s = prepare(case, seed)
    op, K, N = s["op"], s["K"], s["N"]
    d = lambda name: s[name].double()

    def held(q, code, cols):                           # q * 2^(code - 127)
        power = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), code.int() - 127)
        return q.double() * power[:, torch.arange(cols, device="cuda") // GROUP]

    def in_8_bits(v):                                  # multiples of a group's scale, a power of two; at most 127 of them
        rows, cols = v.shape
        groups = torch.zeros(rows, (cols + GROUP - 1) // GROUP * GROUP, dtype=v.dtype, device=v.device)
        groups[:, :cols] = v
        groups = groups.view(rows, -1, GROUP)
        mantissa, power = torch.frexp(groups.abs().max(2).values)          # 1/2 <= mantissa < 1
        power = power - 7 + (mantissa >= 127.5 / 128).int()
        power = torch.where(mantissa == 0, -126, power.clamp(-126, 9 if s["dtype"] == "f16" else 121))
        unit = torch.ldexp(torch.ones_like(mantissa), power)[:, :, None]
        return ((groups / unit).round().clamp(-127, 127) * unit).view(rows, -1)[:, :cols]

    def activation(x):                                 # value and derivative
        if s["act"] == "gelu":
            cdf = 0.5 * torch.erfc(-x / math.sqrt(2))
            return x * cdf, cdf + x * torch.exp(-x ** 2 / 2) / math.sqrt(2 * math.pi)
        # both others are x times a logistic function of z
        k, a = math.sqrt(2 / math.pi), 0.044715
        z, dz = (x, 1.0) if s["act"] == "silu" else (2 * k * (x + a * x ** 3), 2 * k * (1 + 3 * a * x ** 2))
        l = torch.sigmoid(z)
        return x * l, l + x * l * torch.sigmoid(-z) * dz

    if op == "rms_norm":
        v = d("x") if s["r"] is None else d("r") + d("x")
        rstd = (v.pow(2).sum(1) / K + EPS) ** -0.5
        out = {"y": v * d("gamma") * rstd[:, None], "rstd": rstd}
        if s["total"]:
            out["total"] = v
        if s["ckpt"]:
            out["xhat"] = in_8_bits(rstd[:, None] * v)
        return out
    if op == "rms_norm_backward":
        dy, xhat = d("dy"), held(s["q"], s["code"], K)
        dot = torch.sum(dy * d("gamma") * xhat, dim=1, keepdim=True) / K
        dx = (d("gamma") * dy - dot * xhat) * d("rstd")[:, None]
        return {"dx": dx if s["dr"] is None else d("dr") + dx, "dgamma": (xhat * dy).sum(0)}
    if op == "gated":
        both = torch.nn.functional.linear(d("x"), torch.cat([s["wg"], s["wu"]]).double())
        if s["bias"]:
            both = both + torch.cat([s["bg"], s["bu"]]).double()
        out = {"h": activation(both[:, :N])[0] * both[:, N:]}
        if s["ckpt"]:
            out["g"], out["u"] = in_8_bits(both[:, :N]), in_8_bits(both[:, N:])
        return out
    g, u = held(s["qg"], s["codeg"], N), held(s["qu"], s["codeu"], N)
    a, slope = activation(g)
    dg, du = slope * u * d("dh"), a * d("dh")
    out = {"dg": dg, "du": du, "dx": torch.cat([dg, du], 1) @ torch.cat([s["wg"], s["wu"]]).double()}
    if s["ckpt"]:
        out["h"] = in_8_bits(u * a)
    return out
