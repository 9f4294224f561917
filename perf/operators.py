"""Timed cases of the operators that keep saved activations in 8 bits: the checkpoints themselves, layer norm and GELU
with their backward passes from them, and the weight gradient of a linear layer that reads one.

A checkpoint holds a matrix of activations as signed bytes; 32 consecutive values of a row share a power-of-two scale.
What is held that way is returned as the values it stands for.  Sizes are those of the networks in ``workloads.models``
(a perceptron 784-512-256-10, an encoder of width 768 with 16 x 512 tokens, feature maps of convolutions) and
generic ones around them.

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
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ the cases

def _case(op, M, K, N=0, dtype="bf16", residual=False, total=False, ckpt=True, affine=False, param="f32", grad="f32", tanh=False,
          relu=False):
    """M tokens (rows), K features of the activation, N outputs of the linear layer.  residual: a second input (or an incoming
    gradient) is added; total: the sum is an output as well; ckpt: the call leaves a checkpoint; affine: the linear
    layer's input is a layer norm's output whose normalised form is what was kept; param, grad: types of the norm's
    parameters and of the weight gradient; relu: activations of which about half are zero."""
    return {"op": op, "M": M, "K": K, "N": N, "dtype": dtype, "residual": residual, "total": total, "ckpt": ckpt, "affine": affine,
            "param": param, "grad": grad, "tanh": tanh, "relu": relu}


def listed():
    return [
        # a feature map of a convolution network (64 x 256 channels of 56 x 56), packed before it leaves the GPU and restored
        dict(_case("checkpoint", 16_384, 3_136, dtype="f32", relu=True), name="checkpoint f32 16384x3136"),
        # short, odd rows in half precision
        dict(_case("checkpoint", 777, 1_001, dtype="f16"), name="checkpoint f16 777x1001"),
        # one token answered: nothing is kept; what a call costs
        dict(_case("layer_norm", 1, 768, residual=True, ckpt=False, param="bf16"), name="layer norm 1x768"),
        # the encoder's norm after a residual sum, 16 sequences of 512 tokens
        dict(_case("layer_norm", 8_192, 768, residual=True), name="layer norm 8192x768"),
        # ... and its backward pass
        dict(_case("layer_norm_backward", 8_192, 768), name="layer norm backward 8192x768"),
        # a wide network that norms before each block: the residual path's gradient joins; an odd number of tokens
        dict(_case("layer_norm_backward", 16_381, 8_192, residual=True, param="bf16"), name="layer norm backward 16381x8192"),
        # the encoder's activation, forward: the checkpoint replaces the 16-bit copy
        dict(_case("gelu", 8_192, 3_072), name="gelu 8192x3072"),
        # the last, short batch of a small network in 32 bits
        dict(_case("gelu_backward", 37, 1_000, dtype="f32", tanh=True, ckpt=False), name="gelu backward f32 37x1000"),
        # a wide feed-forward block, backward: the gradient, and what the next weight gradient reads
        dict(_case("gelu_backward", 16_384, 16_384, tanh=True), name="gelu backward 16384x16384"),
        # the perceptron's first layer, batch 32
        dict(_case("weight_grad", 32, 784, 512, dtype="f32"), name="weight grad f32 32x512x784"),
        # the encoder's first feed-forward layer, its input kept in normalised form
        dict(_case("weight_grad", 8_192, 768, 3_072, affine=True), name="weight grad 8192x3072x768"),
        # a wide layer, long batch
        dict(_case("weight_grad", 16_384, 8_192, 8_192, grad="bf16"), name="weight grad 16384x8192x8192"),
    ]


OPS = ["checkpoint", "layer_norm", "layer_norm_backward", "gelu", "gelu_backward", "weight_grad"]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(OPS)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    N = 0
    if op == "weight_grad":
        K, N = _log(rng, 16, 8_192), _log(rng, 8, 8_192)
        # (each of the three pieces of a 32-bit gradient is a product of its own)
        M = _log(rng, 1, 16_384 if dtype == "bf16" else 6_000)
    else:
        K = _log(rng, 16, 16_384)
        M = _log(rng, 1, min(65_536, (134e6 if dtype == "f32" else 268e6) / K))
    if rng.random() < 0.4:                             # ragged sizes are common, but so are even ones
        K, N, M = [max(1, v // 64 * 64) if v >= 64 else v for v in (K, N, M)]
    c = _case(op, M, K, N, dtype)
    c["residual"] = op in ("layer_norm", "layer_norm_backward") and rng.random() < 0.5
    c["total"] = op == "layer_norm" and c["residual"] and rng.random() < 0.5
    c["ckpt"] = op in ("checkpoint", "weight_grad", "layer_norm_backward") or rng.random() < 0.7
    c["affine"] = op == "weight_grad" and rng.random() < 0.5
    c["param"] = rng.choice(["f32", dtype])
    c["grad"] = rng.choice(["f32", dtype])
    c["tanh"] = op in ("gelu", "gelu_backward") and rng.random() < 0.5
    c["relu"] = op == "checkpoint" and rng.random() < 0.5
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
    M, K = v.shape
    q, code = _empty_checkpoint(M, K)
    value, byte, c = _quantised(v, dtype)
    q.copy_(byte)
    code.copy_(c)
    return q, code


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, M, K, N, T = case["op"], case["M"], case["K"], case["N"], TYPES[case["dtype"]]
    P = TYPES[case["param"]]
    s = dict(case)
    out = lambda *shape, dtype=T: torch.empty(*shape, dtype=dtype, device="cuda")
    if op == "checkpoint":
        x = _activations(gen, M, K)
        s["x"] = (x.relu_() if case["relu"] else x).to(T)
        s["y"] = out(M, K)
        s["q"], s["code"] = _empty_checkpoint(M, K)
    elif op == "layer_norm":
        s["x"] = _activations(gen, M, K).to(T)
        s["r"] = _activations(gen, M, K).to(T) if case["residual"] else None
        s["gamma"], s["beta"] = (1 + 0.1 * _normal(gen, K)).to(P), (0.1 * _normal(gen, K)).to(P)
        s["y"], s["rstd"] = out(M, K), out(M, dtype=torch.float32)
        s["total_out"] = out(M, K) if case["total"] else None
        if case["ckpt"]:
            s["q"], s["code"] = _empty_checkpoint(M, K)
            s["value"] = out(M, K, dtype=torch.bfloat16)
    elif op == "layer_norm_backward":
        s["dy"] = _gradients(gen, M, K).to(T)
        s["dr"] = _gradients(gen, M, K).to(T) if case["residual"] else None
        x = _activations(gen, M, K)
        x = x - x.mean(1, keepdim=True)
        s["rstd"] = (x.square().mean(1) + EPS).rsqrt()
        s["q"], s["code"] = _packed(x * s["rstd"][:, None], T)
        s["gamma"] = (1 + 0.1 * _normal(gen, K)).to(P)
        s["dx"], s["dgamma"], s["dbeta"] = out(M, K), out(K, dtype=P), out(K, dtype=P)
    elif op == "gelu":
        s["x"] = _activations(gen, M, K).to(T)
        s["y"] = out(M, K)
        if case["ckpt"]:
            s["q"], s["code"] = _empty_checkpoint(M, K)
            s["value"] = out(M, K, dtype=torch.bfloat16)
    elif op == "gelu_backward":
        s["dy"] = _gradients(gen, M, K).to(T)
        s["q"], s["code"] = _packed(_activations(gen, M, K).to(T).float(), T)
        s["dx"] = out(M, K)
        if case["ckpt"]:
            s["yq"], s["ycode"] = _empty_checkpoint(M, K)
            s["value"] = out(M, K, dtype=torch.bfloat16)
    elif op == "weight_grad":
        s["dy"] = _gradients(gen, M, N).to(T)
        s["q"], s["code"] = _packed(_activations(gen, M, K).to(T).float(), T)
        s["gamma"], s["beta"] = ((1 + 0.1 * _normal(gen, K)).to(P), (0.1 * _normal(gen, K)).to(P)) if case["affine"] else (None, None)
        s["dw"], s["db"] = out(N, K, dtype=TYPES[case["grad"]]), out(N, dtype=TYPES[case["grad"]])
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _grouped(v):
    M, K = v.shape
    return torch.nn.functional.pad(v, (0, -K % GROUP)).view(M, -1, GROUP)


def _quantised(v, dtype):
    """(values, bytes, codes) of a checkpoint of v (32 bits): the scale is the smallest power of two that leaves the
    largest of the group's quotients below 127.5, within the powers whose products are normal numbers and finite."""
    M, K = v.shape
    g = _grouped(v)
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


def _phi(x, tanh):
    """Phi(x) and its derivative; in the tanh form what stands for them."""
    if tanh:
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (x + 0.044715 * x * x * x))
        return 0.5 * (1 + t), 0.5 * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))), torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _plain(s):
    op, K, T = s["op"], s["K"], TYPES[s["dtype"]]
    f = lambda name: None if s.get(name) is None else s[name].float()
    if op == "checkpoint":
        return {"restored": _quantised(f("x"), T)[0].to(T)}
    if op == "layer_norm":
        v = f("x") if s["r"] is None else f("x") + f("r")
        d = v - v.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        xhat = d * rstd
        out = {"y": (xhat * f("gamma") + f("beta")).to(T), "rstd": rstd[:, 0]}
        if s["total"]:
            out["total"] = v.to(T)
        if s["ckpt"]:
            out["xhat"] = _quantised(xhat, T)[0].to(torch.bfloat16)
        return out
    if op == "layer_norm_backward":
        dy, xhat = f("dy"), _values(s["q"], s["code"], K)
        g = dy * f("gamma")
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dr"] is not None:
            dx = dx + f("dr")
        P = TYPES[s["param"]]
        return {"dx": dx.to(T), "dgamma": (dy * xhat).sum(0).to(P), "dbeta": dy.sum(0).to(P)}
    if op == "gelu":
        x = f("x")
        out = {"y": (x * _phi(x, s["tanh"])[0]).to(T)}
        if s["ckpt"]:
            out["x"] = _quantised(x, T)[0].to(torch.bfloat16)
        return out
    if op == "gelu_backward":
        x = _values(s["q"], s["code"], K)
        p, dp = _phi(x, s["tanh"])
        out = {"dx": (f("dy") * (p + x * dp)).to(T)}
        if s["ckpt"]:
            out["y"] = _quantised(x * p, T)[0].to(torch.bfloat16)
        return out
    dy, x = f("dy"), _values(s["q"], s["code"], K)
    if s["affine"]:
        x = x * f("gamma") + f("beta")
    G = TYPES[s["grad"]]
    return {"dw": (dy.t() @ x).to(G), "db": dy.sum(0).to(G)}


# ------------------------------------------------------------------------------------------------ the package's operators

@functools.lru_cache(maxsize=1)
def _package():
    import paper_2105_13336_amd as P
    return P, P.tensile_ops_create()


def _own(s):
    P, ops = _package()
    op = s["op"]
    if op == "checkpoint":
        c = P.Checkpoint(s["q"], s["code"])
        P.tensile_ckpt_pack(ops, s["x"], c)
        P.tensile_ckpt_unpack(ops, c, s["y"])
        return {"restored": s["y"]}
    if op == "layer_norm":
        c = P.Checkpoint(s["q"], s["code"]) if s["ckpt"] else None
        P.tensile_layer_norm(ops, s["x"], s["gamma"], s["beta"], s["y"], eps=EPS, residual=s["r"], total=s["total_out"], xhat=c,
                             rstd=s["rstd"])
        out = {"y": s["y"], "rstd": s["rstd"]}
        if s["total"]:
            out["total"] = s["total_out"]
        if c is not None:
            P.tensile_ckpt_unpack(ops, c, s["value"])
            out["xhat"] = s["value"]
        return out
    if op == "layer_norm_backward":
        P.tensile_layer_norm_backward(ops, s["dy"], P.Checkpoint(s["q"], s["code"]), s["rstd"], s["gamma"], s["dx"], s["dgamma"],
                                      s["dbeta"], dresidual=s["dr"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if op == "gelu":
        c = P.Checkpoint(s["q"], s["code"]) if s["ckpt"] else None
        P.tensile_gelu(ops, s["x"], s["y"], ckpt=c, tanh=s["tanh"])
        out = {"y": s["y"]}
        if c is not None:
            P.tensile_ckpt_unpack(ops, c, s["value"])
            out["x"] = s["value"]
        return out
    if op == "gelu_backward":
        c = P.Checkpoint(s["yq"], s["ycode"]) if s["ckpt"] else None
        P.tensile_gelu_backward(ops, s["dy"], P.Checkpoint(s["q"], s["code"]), s["dx"], y_ckpt=c, tanh=s["tanh"])
        out = {"dx": s["dx"]}
        if c is not None:
            P.tensile_ckpt_unpack(ops, c, s["value"])
            out["y"] = s["value"]
        return out
    P.tensile_linear_grad(ops, s["dy"], P.Checkpoint(s["q"], s["code"]), s["dw"], dbias=s["db"], gamma=s["gamma"], beta=s["beta"])
    return {"dw": s["dw"], "db": s["db"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ what it takes, and what is right

def work(case):
    """Each input read once, each output written once; a checkpoint that is made is written, what is restored from it too."""
    op, M, K, N, b = case["op"], case["M"], case["K"], case["N"], BYTES[case["dtype"]]
    n = M * K
    held = n + M * ((K + GROUP - 1) // GROUP)
    kept = held + 2 * n if case["ckpt"] else 0
    if op == "checkpoint":
        return {"bytes": 2 * b * n + held, "flops": 4 * n}
    if op == "layer_norm":
        return {"bytes": b * n * (2 + case["residual"] + case["total"]) + 4 * M + 2 * K * BYTES[case["param"]] + kept, "flops": 9 * n}
    if op == "layer_norm_backward":
        return {"bytes": b * n * (2 + case["residual"]) + held + 4 * M + 3 * K * BYTES[case["param"]], "flops": 14 * n}
    if op == "gelu":
        return {"bytes": 2 * b * n + kept, "flops": 12 * n}
    if op == "gelu_backward":
        return {"bytes": 2 * b * n + held + kept, "flops": 20 * n}
    return {"bytes": b * M * N + held + (N * K + N) * BYTES[case["grad"]], "flops": 2 * M * N * K}


def exact(case, seed):
    """In 64 bits, from the definitions.  A checkpoint's values are held against the numbers it stands for."""
    s = prepare(case, seed)
    op, M, K = s["op"], s["M"], s["K"]
    d = lambda name: None if s.get(name) is None else s[name].double()

    def held(q, code):                                 # q * 2^(code - 127)
        power = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), code.int() - 127)
        return q.double() * power[:, torch.arange(K, device="cuda") // GROUP]

    def gelu(x):                                       # value and derivative
        if s["tanh"]:
            k, a = math.sqrt(2 / math.pi), 0.044715
            u = k * (x + a * x ** 3)
            t = 1 - 2 / (torch.exp(2 * u) + 1)
            return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * a * x ** 2)
        cdf = 0.5 * torch.erfc(-x / math.sqrt(2))
        return x * cdf, cdf + x * torch.exp(-x ** 2 / 2) / math.sqrt(2 * math.pi)

    if op == "checkpoint":
        return {"restored": d("x")}
    if op == "layer_norm":
        v = d("x") + (d("r") if s["r"] is not None else 0)
        var, mu = torch.var_mean(v, dim=1, correction=0, keepdim=True)
        xhat = (v - mu) / (var + EPS).sqrt()
        out = {"y": d("beta") + d("gamma") * xhat, "rstd": (var[:, 0] + EPS) ** -0.5}
        if s["total"]:
            out["total"] = v
        if s["ckpt"]:
            out["xhat"] = xhat
        return out
    if op == "layer_norm_backward":
        dy, xhat = d("dy"), held(s["q"], s["code"])
        h = d("gamma") * dy
        dx = d("rstd")[:, None] * (h - (h.sum(1) / K)[:, None] - xhat * ((h * xhat).sum(1) / K)[:, None])
        return {"dx": dx if s["dr"] is None else dx + d("dr"), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}
    if op == "gelu":
        out = {"y": gelu(d("x"))[0]}
        if s["ckpt"]:
            out["x"] = d("x")
        return out
    if op == "gelu_backward":
        y, slope = gelu(held(s["q"], s["code"]))
        out = {"dx": slope * d("dy")}
        if s["ckpt"]:
            out["y"] = y
        return out
    x = held(s["q"], s["code"])
    if s["affine"]:
        x = d("gamma") * x + d("beta")
    return {"dw": torch.matmul(d("dy").t().contiguous(), x), "db": d("dy").sum(0)}
