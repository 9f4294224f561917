"""A stack of feed-forward blocks trained with its saved activations in 8 bits, and what that does to the iteration's memory plan.

    u = h W1^T + b1;  a = gelu(u);  v = a W2^T + b2;  h' = norm(v + h)          (h of the first block: norm(x))

Forward keeps of every norm the normalised rows (8 bits) and of every GELU its input (8 bits): one tensor of each width.  Backward
reads them as they are: the norm's backward pass, the GELU's (which makes the checkpoint of `a` that W2's gradient needs), and
the weight gradients - that of W1 from the checkpoint of the norm in front of it.  The products with the weights are torch's.

Every operator of the iteration is recorded with the tensors that it reads and makes, their sizes and its time: the tensor
access sequence for which the planner then decides what has to leave the GPU.  The same iteration with 16-bit activations
(kept: the norm's sum and output, u and a) is recorded next to it.

    python examples/feed_forward.py [--layers 12 --tokens 8192 --hidden 768 --ffn 3072]
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
    args = ap.parse_args()
    model = FeedForward(args.layers, args.hidden, args.ffn)
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
