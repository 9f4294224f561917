"""A stack of feed-forward blocks trained with its saved activations in 8 bits, and what that does to the iteration's memory plan.

    u = h W1^T + b1;  a = gelu(u);  v = a W2^T + b2;  h' = norm(v + h)          (h of the first block: norm(x))

Forward keeps of every norm the normalised rows (8 bits) and of every GELU its input (8 bits): one tensor of each width.  Backward
reads them as they are: the norm's backward pass, the GELU's (which makes the checkpoint of `a` that W2's gradient needs), and
the weight gradients - that of W1 from the checkpoint of the norm in front of it.  The products with the weights are torch's.

With --gated the blocks are gated ones, with a root-mean-square norm in front of each and the residual path beside it:

    n = norm(s);  a = silu(n Wg^T) * (n Wu^T);  s' = s + a W2^T                 (and a last norm behind them)

of which the norm's rows and both projections are kept in 8 bits; Wg and Wu are the halves of one matrix, W1, and have one gradient.

Every operator of the iteration is recorded with the tensors that it reads and makes, their sizes and its time: the tensor
access sequence for which the planner then decides what has to leave the GPU.  The same iteration with 16-bit activations
(kept: the norm's sum and output, the projections and a) is recorded next to it.

    python examples/feed_forward.py [--layers 12 --tokens 8192 --hidden 768 --ffn 3072] [--gated]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np  # noqa: E402
import torch  # noqa: E402

import paper_2105_13336_amd as P  # noqa: E402
from workloads.tas import TAS, Trace, even_grid, merge_traces  # noqa: E402

LINK_BYTES_PER_US = 64_000          # 64 GB/s host link
EPS = 1e-5


class Recorder:
    """Runs operators one by one and writes down what a tensor access sequence holds of them."""

    def __init__(self) -> None:
        self.trace, self.ids, self.events = Trace(), {}, []

    def op(self, reads, outs, run):
        """run() -> what it makes, in the order of the names `outs`"""
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        made = run()
        end.record()
        made = made if isinstance(made, tuple) else (made,)
        self.events.append((begin, end))
        new = self.trace.op(reads=[self.ids[n] for n in reads], outs=[(n, t.nbytes) for n, t in zip(outs, made)])
        self.ids.update(zip(outs, new))
        return made if len(made) > 1 else made[0]

    def sequence(self) -> TAS:
        torch.cuda.synchronize()
        T = 2 * self.trace.n_ops
        steps = even_grid(self.trace.n_ops, T)
        ns = np.ones(T, dtype=np.int64)
        ns[steps] = [max(1, int(b.elapsed_time(e) * 1e6)) for b, e in self.events]
        return merge_traces(T, [self.trace], [steps], ns, 0, LINK_BYTES_PER_US)


class FeedForward:
    """Parameters (bf16 weights and biases, f32 norms) and one training iteration, with activations kept in 8 or in 16 bits."""

    def __init__(self, layers: int, hidden: int, ffn: int, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda n, k: (torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5).bfloat16()
        z = lambda n: torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        self.layers, self.hidden, self.ffn, self.ops = layers, hidden, ffn, P.tensile_ops_create()
        self.p = {}
        for l in range(layers):
            self.p |= {f"w1.{l}": w(ffn, hidden), f"b1.{l}": z(ffn), f"w2.{l}": w(hidden, ffn), f"b2.{l}": z(hidden)}
        for l in range(layers + 1):
            self.p |= {f"g.{l}": torch.ones(hidden, device="cuda"), f"b.{l}": torch.zeros(hidden, device="cuda")}

    def iteration(self, x: torch.Tensor, target: torch.Tensor, rec: Recorder | None = None, kept_bits: int = 8):
        """-> (loss, gradients by name).  loss = mean over the tokens of |h - target|^2 / 2, summed over the features."""
        rec, p, ops = rec or Recorder(), self.p, self.ops
        run = self._in_8_bits if kept_bits == 8 else self._in_16_bits
        rec.op([], list(p) + ["x", "target"], lambda: (*p.values(), x, target))
        return run(rec, p, ops, x, target)

    def _in_8_bits(self, rec, p, ops, x, target):
        M, L = x.shape[0], self.layers
        new = lambda n, dtype=x.dtype: torch.empty(M, n, dtype=dtype, device="cuda")
        like = lambda n: torch.empty_like(p[n])

        def norm(l, v, h):
            y, c, rstd = new(self.hidden), P.Checkpoint.empty(M, self.hidden), torch.empty(M, device="cuda")
            P.tensile_layer_norm(ops, v, p[f"g.{l}"], p[f"b.{l}"], y, eps=EPS, residual=h, xhat=c, rstd=rstd)
            return y, c, rstd

        def gelu(u):
            a, c = torch.empty_like(u), P.Checkpoint.empty(M, self.ffn)
            P.tensile_gelu(ops, u, a, ckpt=c)
            return a, c

        def norm_backward(l, dh):
            dx, dg, db = torch.empty_like(dh), like(f"g.{l}"), like(f"b.{l}")
            P.tensile_layer_norm_backward(ops, dh, xhat[l], rstd[l], p[f"g.{l}"], dx, dg, db)
            return dx, dg, db

        def gelu_backward(da, c):
            du, ca = torch.empty_like(da), P.Checkpoint.empty(M, self.ffn)
            P.tensile_gelu_backward(ops, da, c, du, y_ckpt=ca)
            return du, ca

        def weight(l, which, dy, c, gamma=None, beta=None):
            dw, db = like(f"w{which}.{l}"), like(f"b{which}.{l}")
            P.tensile_linear_grad(ops, dy, c, dw, dbias=db, gamma=gamma, beta=beta)
            return dw, db

        xhat, rstd, kept_u = {}, {}, {}
        h, xhat[0], rstd[0] = rec.op(["x", "g.0", "b.0"], ["h.0", "xhat.0", "rstd.0"], lambda: norm(0, x, None))
        for l in range(L):
            u = rec.op([f"h.{l}", f"w1.{l}", f"b1.{l}"], [f"u.{l}"], lambda: torch.addmm(p[f"b1.{l}"], h, p[f"w1.{l}"].t()))
            a, kept_u[l] = rec.op([f"u.{l}"], [f"a.{l}", f"u8.{l}"], lambda: gelu(u))
            v = rec.op([f"a.{l}", f"w2.{l}", f"b2.{l}"], [f"v.{l}"], lambda: torch.addmm(p[f"b2.{l}"], a, p[f"w2.{l}"].t()))
            h, xhat[l + 1], rstd[l + 1] = rec.op([f"v.{l}", f"h.{l}", f"g.{l + 1}", f"b.{l + 1}"], [f"h.{l + 1}", f"xhat.{l + 1}", f"rstd.{l + 1}"],
                                                 lambda: norm(l + 1, v, h))
            del u, a, v
        loss, dh = self._loss(rec, h, target)
        grads = {}
        for l in reversed(range(L)):
            ds, grads[f"g.{l + 1}"], grads[f"b.{l + 1}"] = rec.op([f"dh.{l + 1}", f"xhat.{l + 1}", f"rstd.{l + 1}", f"g.{l + 1}"],
                                                                  [f"ds.{l}", f"dg.{l + 1}", f"db.{l + 1}"], lambda: norm_backward(l + 1, dh))
            da = rec.op([f"ds.{l}", f"w2.{l}"], [f"da.{l}"], lambda: ds @ p[f"w2.{l}"])
            du, a8 = rec.op([f"da.{l}", f"u8.{l}"], [f"du.{l}", f"a8.{l}"], lambda: gelu_backward(da, kept_u.pop(l)))
            grads[f"w2.{l}"], grads[f"b2.{l}"] = rec.op([f"ds.{l}", f"a8.{l}"], [f"dw2.{l}", f"db2.{l}"], lambda: weight(l, 2, ds, a8))
            grads[f"w1.{l}"], grads[f"b1.{l}"] = rec.op([f"du.{l}", f"xhat.{l}", f"g.{l}", f"b.{l}"], [f"dw1.{l}", f"db1.{l}"],
                                                        lambda: weight(l, 1, du, xhat[l], p[f"g.{l}"], p[f"b.{l}"]))
            dh = rec.op([f"ds.{l}", f"du.{l}", f"w1.{l}"], [f"dh.{l}"], lambda: torch.addmm(ds, du, p[f"w1.{l}"]))
            del da, du, a8, ds
        _, grads["g.0"], grads["b.0"] = rec.op(["dh.0", "xhat.0", "rstd.0", "g.0"], ["dx", "dg.0", "db.0"], lambda: norm_backward(0, dh))
        return loss, grads

    def _in_16_bits(self, rec, p, ops, x, target):
        """The same with torch's operators, what backward needs kept as it is."""
        F, L, D = torch.nn.functional, self.layers, self.hidden
        back = torch.ops.aten.native_layer_norm_backward
        s, h, stat, kept_u, kept_a = {}, {}, {}, {}, {}

        def norm(l, v, r):
            total = v if r is None else v + r
            y, mean, rstd = torch.native_layer_norm(total.float(), (D,), p[f"g.{l}"], p[f"b.{l}"], EPS)
            return (y.to(x.dtype), mean, rstd) if r is None else (y.to(x.dtype), mean, rstd, total)

        def norm_backward(l, dh):
            dx, dg, db = back(dh.float(), s[l].float(), (D,), *stat[l], p[f"g.{l}"], p[f"b.{l}"], (True, True, True))
            return dx.to(x.dtype), dg, db

        s[0] = x
        h[0], *stat[0] = rec.op(["x", "g.0", "b.0"], ["h.0", "mean.0", "rstd.0"], lambda: norm(0, x, None))
        for l in range(L):
            kept_u[l] = rec.op([f"h.{l}", f"w1.{l}", f"b1.{l}"], [f"u.{l}"], lambda: torch.addmm(p[f"b1.{l}"], h[l], p[f"w1.{l}"].t()))
            kept_a[l] = rec.op([f"u.{l}"], [f"a.{l}"], lambda: F.gelu(kept_u[l]))
            v = rec.op([f"a.{l}", f"w2.{l}", f"b2.{l}"], [f"v.{l}"], lambda: torch.addmm(p[f"b2.{l}"], kept_a[l], p[f"w2.{l}"].t()))
            h[l + 1], m, r, s[l + 1] = rec.op([f"v.{l}", f"h.{l}", f"g.{l + 1}", f"b.{l + 1}"],
                                              [f"h.{l + 1}", f"mean.{l + 1}", f"rstd.{l + 1}", f"s.{l + 1}"], lambda: norm(l + 1, v, h[l]))
            stat[l + 1] = [m, r]
        loss, dh = self._loss(rec, h[L], target)
        grads = {}
        for l in reversed(range(L)):
            n = l + 1
            ds, grads[f"g.{n}"], grads[f"b.{n}"] = rec.op([f"dh.{n}", f"s.{n}", f"mean.{n}", f"rstd.{n}", f"g.{n}"], [f"ds.{l}", f"dg.{n}", f"db.{n}"],
                                                          lambda: norm_backward(n, dh))
            da = rec.op([f"ds.{l}", f"w2.{l}"], [f"da.{l}"], lambda: ds @ p[f"w2.{l}"])
            grads[f"w2.{l}"], grads[f"b2.{l}"] = rec.op([f"ds.{l}", f"a.{l}"], [f"dw2.{l}", f"db2.{l}"], lambda: (ds.t() @ kept_a[l], ds.sum(0)))
            du = rec.op([f"da.{l}", f"u.{l}"], [f"du.{l}"], lambda: torch.ops.aten.gelu_backward(da, kept_u[l]))
            grads[f"w1.{l}"], grads[f"b1.{l}"] = rec.op([f"du.{l}", f"h.{l}"], [f"dw1.{l}", f"db1.{l}"], lambda: (du.t() @ h[l], du.sum(0)))
            dh = rec.op([f"ds.{l}", f"du.{l}", f"w1.{l}"], [f"dh.{l}"], lambda: torch.addmm(ds, du, p[f"w1.{l}"]))
        _, grads["g.0"], grads["b.0"] = rec.op(["dh.0", "x", "mean.0", "rstd.0", "g.0"], ["dx", "dg.0", "db.0"], lambda: norm_backward(0, dh))
        return loss, grads

    def _loss(self, rec, h, target):
        def run():
            d = h.float() - target.float()
            return 0.5 * d.square().sum(1).mean(), (d / d.shape[0]).to(h.dtype)
        return rec.op([f"h.{self.layers}", "target"], ["loss", f"dh.{self.layers}"], run)

    def update(self, grads, rate: float) -> None:
        for n, g in grads.items():
            self.p[n].sub_((rate * g.float()).to(self.p[n].dtype))


class GatedFeedForward(FeedForward):
    """The same of gated blocks: W1 [2 * ffn, hidden] is Wg above Wu."""

    def __init__(self, layers: int, hidden: int, ffn: int, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda n, k: (torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5).bfloat16()
        self.layers, self.hidden, self.ffn, self.ops = layers, hidden, ffn, P.tensile_ops_create()
        self.no_beta = torch.zeros(hidden, device="cuda")
        self.p = {}
        for l in range(layers):
            self.p |= {f"w1.{l}": w(2 * ffn, hidden), f"w2.{l}": w(hidden, ffn)}
        for l in range(layers + 1):
            self.p[f"g.{l}"] = torch.ones(hidden, device="cuda")

    def _in_8_bits(self, rec, p, ops, x, target):
        M, L, F = x.shape[0], self.layers, self.ffn
        new = lambda n, dtype=x.dtype: torch.empty(M, n, dtype=dtype, device="cuda")
        like = lambda n: torch.empty_like(p[n])

        def norm(l, v, s):
            n, t, c, rstd = new(self.hidden), new(self.hidden), P.Checkpoint.empty(M, self.hidden), torch.empty(M, device="cuda")
            P.tensile_rms_norm(ops, v, p[f"g.{l}"], n, eps=EPS, residual=s, total=None if s is None else t, xhat=c, rstd=rstd)
            return (n, c, rstd) if s is None else (n, c, rstd, t)

        def gated(l, n):
            a, g, u = new(F), P.Checkpoint.empty(M, F), P.Checkpoint.empty(M, F)
            P.tensile_gated_linear(ops, n, p[f"w1.{l}"][:F], p[f"w1.{l}"][F:], a, gate=g, up=u)
            return a, g, u

        def gated_backward(l, da, g, u):
            d, dn, a8 = new(2 * F), new(self.hidden), P.Checkpoint.empty(M, F)
            P.tensile_gated_linear_backward(ops, da, g, u, d[:, :F], d[:, F:], w_gate=p[f"w1.{l}"][:F], w_up=p[f"w1.{l}"][F:], dx=dn, h_ckpt=a8)
            return d, dn, a8

        def norm_backward(l, dn, ds):
            dx, dg = torch.empty_like(dn), like(f"g.{l}")
            P.tensile_rms_norm_backward(ops, dn, xhat[l], rstd[l], p[f"g.{l}"], dx, dg, dresidual=ds)
            return dx, dg

        def weight(name, dy, c, gamma=None):
            dw = like(name)
            P.tensile_linear_grad(ops, dy, c, dw, gamma=gamma, beta=None if gamma is None else self.no_beta)
            return dw

        xhat, rstd, g8, u8 = {}, {}, {}, {}
        s = x
        n, xhat[0], rstd[0] = rec.op(["x", "g.0"], ["n.0", "xhat.0", "rstd.0"], lambda: norm(0, x, None))
        for l in range(L):
            a, g8[l], u8[l] = rec.op([f"n.{l}", f"w1.{l}"], [f"a.{l}", f"g8.{l}", f"u8.{l}"], lambda: gated(l, n))
            v = rec.op([f"a.{l}", f"w2.{l}"], [f"v.{l}"], lambda: a @ p[f"w2.{l}"].t())
            n, xhat[l + 1], rstd[l + 1], s = rec.op([f"v.{l}", f"s.{l}" if l else "x", f"g.{l + 1}"], [f"n.{l + 1}", f"xhat.{l + 1}", f"rstd.{l + 1}", f"s.{l + 1}"],
                                                    lambda: norm(l + 1, v, s))
            del a, v
        rec.ids[f"h.{L}"] = rec.ids[f"n.{L}"]
        loss, dh = self._loss(rec, n, target)
        grads = {}
        ds, grads[f"g.{L}"] = rec.op([f"dh.{L}", f"xhat.{L}", f"rstd.{L}", f"g.{L}"], [f"ds.{L}", f"dg.{L}"], lambda: norm_backward(L, dh, None))
        for l in reversed(range(L)):
            da = rec.op([f"ds.{l + 1}", f"w2.{l}"], [f"da.{l}"], lambda: ds @ p[f"w2.{l}"])
            d, dn, a8 = rec.op([f"da.{l}", f"g8.{l}", f"u8.{l}", f"w1.{l}"], [f"d.{l}", f"dn.{l}", f"a8.{l}"], lambda: gated_backward(l, da, g8.pop(l), u8.pop(l)))
            grads[f"w2.{l}"] = rec.op([f"ds.{l + 1}", f"a8.{l}"], [f"dw2.{l}"], lambda: weight(f"w2.{l}", ds, a8))
            grads[f"w1.{l}"] = rec.op([f"d.{l}", f"xhat.{l}", f"g.{l}"], [f"dw1.{l}"], lambda: weight(f"w1.{l}", d, xhat[l], p[f"g.{l}"]))
            ds, grads[f"g.{l}"] = rec.op([f"dn.{l}", f"ds.{l + 1}", f"xhat.{l}", f"rstd.{l}", f"g.{l}"], [f"ds.{l}", f"dg.{l}"], lambda: norm_backward(l, dn, ds))
            del da, d, dn, a8
        return loss, grads

    def _in_16_bits(self, rec, p, ops, x, target):
        """The same with torch's operators, what backward needs kept as it is."""
        L, F = self.layers, self.ffn
        s, n, rstd, both, a = {0: x}, {}, {}, {}, {}

        def norm(l, v, r):
            total = v if r is None else v + r
            rs = torch.rsqrt(total.float().square().mean(1, keepdim=True) + EPS)
            y = (total * rs * p[f"g.{l}"]).to(x.dtype)
            return (y, rs) if r is None else (y, rs, total)

        def norm_backward(l, dn, ds):
            xhat, t = s[l].float() * rstd[l], dn.float() * p[f"g.{l}"]
            dx = rstd[l] * (t - xhat * (t * xhat).mean(1, keepdim=True))
            return (dx if ds is None else dx + ds).to(x.dtype), (dn * xhat).sum(0)

        def gated_backward(l, da):
            g, u = both[l][:, :F], both[l][:, F:]
            d = torch.cat([torch.ops.aten.silu_backward(da * u, g), da * torch.nn.functional.silu(g)], 1)
            return d, d @ p[f"w1.{l}"]

        n[0], rstd[0] = rec.op(["x", "g.0"], ["n.0", "rstd.0"], lambda: norm(0, x, None))
        for l in range(L):
            both[l] = rec.op([f"n.{l}", f"w1.{l}"], [f"both.{l}"], lambda: n[l] @ p[f"w1.{l}"].t())
            a[l] = rec.op([f"both.{l}"], [f"a.{l}"], lambda: torch.nn.functional.silu(both[l][:, :F]) * both[l][:, F:])
            v = rec.op([f"a.{l}", f"w2.{l}"], [f"v.{l}"], lambda: a[l] @ p[f"w2.{l}"].t())
            n[l + 1], rstd[l + 1], s[l + 1] = rec.op([f"v.{l}", f"s.{l}" if l else "x", f"g.{l + 1}"], [f"n.{l + 1}", f"rstd.{l + 1}", f"s.{l + 1}"],
                                                     lambda: norm(l + 1, v, s[l]))
        rec.ids[f"h.{L}"] = rec.ids[f"n.{L}"]
        loss, dh = self._loss(rec, n[L], target)
        grads = {}
        ds, grads[f"g.{L}"] = rec.op([f"dh.{L}", f"s.{L}" if L else "x", f"rstd.{L}", f"g.{L}"], [f"ds.{L}", f"dg.{L}"], lambda: norm_backward(L, dh, None))
        for l in reversed(range(L)):
            da = rec.op([f"ds.{l + 1}", f"w2.{l}"], [f"da.{l}"], lambda: ds @ p[f"w2.{l}"])
            grads[f"w2.{l}"] = rec.op([f"ds.{l + 1}", f"a.{l}"], [f"dw2.{l}"], lambda: ds.t() @ a[l])
            d, dn = rec.op([f"da.{l}", f"both.{l}", f"w1.{l}"], [f"d.{l}", f"dn.{l}"], lambda: gated_backward(l, da))
            grads[f"w1.{l}"] = rec.op([f"d.{l}", f"n.{l}"], [f"dw1.{l}"], lambda: d.t() @ n[l])
            ds, grads[f"g.{l}"] = rec.op([f"dn.{l}", f"ds.{l + 1}", f"s.{l}" if l else "x", f"rstd.{l}", f"g.{l}"], [f"ds.{l}", f"dg.{l}"],
                                         lambda: norm_backward(l, dn, ds))
        return loss, grads


def plan(tas: TAS, budget: int) -> dict:
    """The planner's swaps for the recorded iteration, until it fits the budget or nothing more can be done."""
    h = P.tas_load(tas)
    before, _ = P.tensile_tas_info(h)
    out = P.tensile_greedy_plan(h, budget, stop_at_budget=True, capacity=4096)
    h.close()
    swapped = int(tas.size_bytes[out["iv_tensor"]].sum()) if len(out["iv_tensor"]) else 0
    return {"peak": before, "planned": out["final_peak"], "swaps": len(out["iv_tensor"]), "swapped_bytes": swapped}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 12), ("tokens", 8192), ("hidden", 768), ("ffn", 3072), ("steps", 5)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--gated", action="store_true")
    args = ap.parse_args()
    model = (GatedFeedForward if args.gated else FeedForward)(args.layers, args.hidden, args.ffn)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, target = (torch.randn(args.tokens, args.hidden, generator=gen, device="cuda").bfloat16() for _ in range(2))
    grads, sequences = {}, {}
    for bits in (16, 8):
        for _ in range(2):                             # (the second one is recorded: nothing is loaded or allocated anew)
            rec = Recorder()
            loss, grads[bits] = model.iteration(x, target, rec, bits)
            sequences[bits] = rec.sequence()
        print(f"{bits:2d} bits: loss {float(loss):.4f}, operators {sequences[bits].step_ns.sum() / 1e6:.2f} ms", flush=True)
    off = {n: float((grads[8][n].float() - grads[16][n].float()).norm() / grads[16][n].float().norm()) for n in grads[8]}
    print(f"gradients: relative difference of the two, median {np.median(list(off.values())):.4f}, largest {max(off.values()):.4f}", flush=True)
    peaks = {b: plan(sequences[b], 0) for b in (16, 8)}
    budget = int(0.75 * peaks[8]["peak"])
    for bits in (16, 8):
        r = plan(sequences[bits], budget)
        print(f"{bits:2d} bits: peak {r['peak'] / 2 ** 20:.0f} MiB; for {budget / 2 ** 20:.0f} MiB: {r['swaps']} swaps of {r['swapped_bytes'] / 2 ** 20:.0f} MiB -> "
              f"{r['planned'] / 2 ** 20:.0f} MiB; as far as it goes {peaks[bits]['planned'] / 2 ** 20:.0f} MiB", flush=True)
    for k in range(args.steps):
        loss, g = model.iteration(x, target)
        model.update(g, 2.0 / args.hidden)             # (the loss is a sum over the features)
        print(f"step {k}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
