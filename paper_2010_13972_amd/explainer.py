"""An explainer network: SHAP values of a tree ensemble, approximately, at a fixed cost.

``gts.shap`` is exact, and its cost grows with the ensemble.  An ``Explainer`` learns to
give the same values: every training step draws rows, computes their exact values with
``gts.shap`` and fits a residual network to them with the operators of ``nn``.  Asked
for rows it then runs the network alone.  That pays for many rows of a large ensemble:
10 000 rows of the deep workload take it 0.24 ms and gts.shap 2.2, of the small covtype_med
0.25 and 0.31.  A single row is faster exact (17 to 44 us) than from the network's graph (60).

    x -> W_in, silu -> u                                     u: the residual stream
    per block:  gate = h W_g^T,  f = gelu(h W_1^T) W_2^T     h: the normed stream
                u, h = norm_residual(u, f, gate, scale)
    h -> W_out -> the values of every output, in units of their spread

Weights are float32; the products take bfloat16 copies that the optimizer's step
writes.  The bias column is the ensemble's own.  In float16, whose numbers end at 6e-8 and
65504, the backward pass runs on scaled gradients: those of the mean over 4096 rows of 784
values are below the least number otherwise.  The optimizer takes the scale off again, in
32 bits; gradients that overflow change nothing but the scale, which is halved.

    python -m paper_2010_13972_amd.explainer --workload covtype_med --steps 400
"""
from __future__ import annotations

import argparse
import time

import torch

from . import gts, nn

# In float16, the gradient of a value starts at this times its error: sums over some 1e5
# rows stay finite, and errors down to 1e-3 of the values' spread keep all their bits.
_SCALE = 0.125
_BLOCK = ("w_g", "b_g", "w_1", "b_1", "w_2", "b_2", "w_post", "w_pre", "scale")


class Explainer:
    """A network for the values of ``model`` (a gts.DeviceModel): ``width`` of the stream,
    ``blocks`` residual blocks of 4 width; dtype of the products; state_bits of AdamW."""

    def __init__(self, model: gts.DeviceModel, X, width: int = 512, blocks: int = 2,
                 dtype=torch.bfloat16, state_bits: int = 32, seed: int = 0):
        self.model, self.blocks, self.dtype = model, blocks, dtype
        self.shape = (model.num_groups, model.num_features)
        self.X = X
        phi = gts.shap(model, X[:1024])
        self.bias = phi[0, :, -1].float()
        values = phi[..., :-1].float()
        self.spread = float(values.std(correction=min(1, values.numel() - 1))) or 1.0
        # a feature that never varied keeps its unit: rows explained later may have other values
        same = (X == X[0]).all(0)
        self.mean = torch.where(same, X[0], X.mean(0))
        self.dev = torch.where(same, 1.0, X.std(0, correction=min(1, X.shape[0] - 1)).clamp_min(1e-6))
        g = torch.Generator(device=X.device).manual_seed(seed)
        m, outs = model.num_features, model.num_groups * model.num_features

        def weight(o, i, gain=1.0):
            return torch.randn(o, i, generator=g, device=X.device) * (gain * i ** -0.5)

        def vector(n, v):
            return torch.full((n,), v, device=X.device)

        self.names = ["w_in", "b_in"]
        tensors = [weight(width, m), vector(width, 0.0)]
        for b in range(blocks):
            self.names += [f"{n}.{b}" for n in _BLOCK]
            tensors += [weight(width, width), vector(width, 0.0), weight(4 * width, width),
                        vector(4 * width, 0.0), weight(width, 4 * width), vector(width, 0.0),
                        vector(width, 1.0), vector(width, 1.0), vector(width, 0.5)]
        self.names += ["w_out", "b_out"]
        tensors += [weight(outs, width, 0.1), vector(outs, 0.0)]
        self.master = tensors
        # the products' own copies; in float32, the weights themselves
        self.copies = None if dtype == torch.float32 else [t.to(dtype) for t in tensors]
        self.weights = dict(zip(self.names, tensors if self.copies is None else self.copies))
        self.state = nn.adamw_state(tensors, state_bits)
        self.step_number = 0
        self.loss_scale = torch.full((), _SCALE, device=X.device) if dtype == torch.float16 else None

    def _inputs(self, X):
        return ((X - self.mean) / self.dev).to(self.dtype)

    def forward(self, X, keep: bool = False):
        """(values in units of the spread, what backward needs if ``keep``)."""
        w, x = self.weights, self._inputs(X)
        u = nn.linear(x, w["w_in"], w["b_in"], act="silu", save_pre=keep)
        u, pre_in = u if keep else (u, None)
        h, kept = u, []
        for b in range(self.blocks):
            gate = nn.linear(h, w[f"w_g.{b}"], w[f"b_g.{b}"])
            z = nn.linear(h, w[f"w_1.{b}"], w[f"b_1.{b}"], act="gelu", save_pre=keep)
            z, pre = z if keep else (z, None)
            f = nn.linear(z, w[f"w_2.{b}"], w[f"b_2.{b}"])
            u, h_next = nn.norm_residual(u, f, w[f"w_post.{b}"], w[f"w_pre.{b}"], gate=gate,
                                         scale=w[f"scale.{b}"])
            if keep:
                kept.append((h, gate, z, pre, f, u))
            h = h_next
        return nn.linear(h, w["w_out"], w["b_out"]), (x, pre_in, kept, h)

    def backward(self, dy, kept):
        """The gradients of all weights, by name, for the gradient dy of forward's values."""
        w, g = self.weights, {}
        x, pre_in, blocks, h = kept
        dh, g["w_out"], g["b_out"] = nn.linear_backward(dy, h, w["w_out"])
        du = None
        for b in reversed(range(self.blocks)):
            h, gate, z, pre, f, u = blocks[b]
            n = nn.norm_residual_backward(du, dh, u, f, w[f"w_post.{b}"], w[f"w_pre.{b}"], gate=gate,
                                          scale=w[f"scale.{b}"])
            g[f"w_post.{b}"], g[f"w_pre.{b}"] = n["dw_post"], n["dw_pre"]
            g[f"scale.{b}"], du = n["dscale"], n["dx"]
            dz, g[f"w_2.{b}"], g[f"b_2.{b}"] = nn.linear_backward(n["df"], z, w[f"w_2.{b}"])
            dh, g[f"w_1.{b}"], g[f"b_1.{b}"] = nn.linear_backward(dz, h, w[f"w_1.{b}"], pre=pre,
                                                                  act="gelu")
            dg, g[f"w_g.{b}"], g[f"b_g.{b}"] = nn.linear_backward(n["dgate"], h, w[f"w_g.{b}"])
            dh = dh + dg   # rounded to the type, as every gradient on the way is
        if du is not None:   # the first block reads the stream itself
            dh = dh + du
        _, g["w_in"], g["b_in"] = nn.linear_backward(dh, x, w["w_in"], pre=pre_in, act="silu",
                                                     dx=False)
        return g

    def targets(self, X):
        """The exact values of X, without the bias, in units of their spread."""
        phi = gts.shap(self.model, X)[..., :-1]
        return phi.reshape(X.shape[0], -1).float() / self.spread

    def train_step(self, X, lr: float, max_norm: float = 1.0):
        """One step on the rows X; the mean square error before it, a device scalar."""
        want = self.targets(X)
        y, kept = self.forward(X, keep=True)
        off = y.float() - want
        mean = 2.0 / off.numel()
        dy = off * (mean if self.loss_scale is None else self.loss_scale)
        g = self.backward(dy.to(self.dtype), kept)
        grads = [g[n] for n in self.names]
        clip = nn.grad_clip(grads, max_norm)
        if self.loss_scale is not None:
            clip = self._unscale(clip, mean, max_norm)
        self.step_number += 1
        s = self.state
        nn.adamw_step(self.master, grads, s.m, s.v, m_scale=s.m_scale, v_scale=s.v_scale,
                      copies=self.copies, clip=clip, step=self.step_number, lr=lr,
                      weight_decay=0.01)
        return off.square().mean()

    def _unscale(self, clip, mean: float, max_norm: float):
        """grad_clip's result for the gradients as they are, from that of the scaled ones: the
        factor takes the scale off too.  Moves the scale: half after an overflow, then back
        by a thousandth a step."""
        s = self.loss_scale
        undo = mean / s
        norm = clip[0] * undo
        there = torch.isfinite(norm)
        factor = torch.where(there, (max_norm / (norm + 1e-6)).clamp(max=1.0) * undo, float("nan"))
        s.copy_(torch.where(there, s * 1.001, s * 0.5).clamp(2.0 ** -20, _SCALE))
        return torch.stack([norm, factor])

    def fit(self, steps: int, rows: int = 4096, lr: float = 1e-3, seed: int = 0, report=None):
        """Trains on `steps` batches of rows drawn from X.  report(step, loss): every 50th."""
        g = torch.Generator(device=self.X.device).manual_seed(seed)
        loss = None
        for i in range(steps):
            at = torch.randint(0, self.X.shape[0], (rows,), generator=g, device=self.X.device)
            warm = min(1.0, (i + 1) / 20) * (1.0 - 0.9 * i / max(1, steps))
            loss = self.train_step(self.X[at], lr * warm)
            if report is not None and (i % 50 == 0 or i + 1 == steps):
                report(i, float(loss))
        return loss

    def explain(self, X):
        """The network's values for X: [rows, G, M+1], float32, as gts.shap lays them out."""
        G, M = self.shape
        y, _ = self.forward(X)
        out = torch.empty(X.shape[0], G, M + 1, device=X.device)
        torch.mul(y.view(-1, G, M), self.spread, out=out[..., :M])
        out[..., M] = self.bias
        return out

    def server(self, rows: int):
        """A function that explains batches of exactly `rows` rows, as ``explain`` does, by
        replaying a HIP graph of its launches: a few rows take the device less time than the
        host needs to enqueue them.  The result is overwritten by the next call.  The graph
        reads the network's weights where they are, so it follows further training; the
        function keeps them, also where the network itself is dropped."""
        X = torch.zeros(rows, self.shape[1], device=self.X.device)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.explain(X)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = self.explain(X)

        def explain(batch):
            if batch.shape != X.shape:
                raise ValueError(f"the batch must have shape {tuple(X.shape)}")
            X.copy_(batch)
            graph.replay()
            return out
        # the graph holds addresses alone: its inputs live as long as the function
        explain.reads = (*self.weights.values(), self.mean, self.dev, self.bias)
        return explain


def explained(exact, got) -> float:
    """The share of the exact values' variance that `got` explains."""
    exact, got = exact[..., :-1].double(), got[..., :-1].double()
    return float(1 - (exact - got).square().sum() / (exact - exact.mean(0)).square().sum())


def _time(f, times: int = 50) -> float:
    f()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(times):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / times * 1e6


def main(argv=None):
    from . import synth

    p = argparse.ArgumentParser(description=__doc__.split("\n", 1)[0])
    p.add_argument("--workload", default="covtype_med", help="one of synth's workloads")
    p.add_argument("--steps", type=int, default=400)
    p.add_argument("--rows", type=int, default=4096, help="rows of a training step")
    p.add_argument("--width", type=int, default=512)
    p.add_argument("--blocks", type=int, default=2)
    p.add_argument("--lr", type=float, default=1e-3)
    p.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    p.add_argument("--dtype", default="bf16", choices=("bf16", "f16", "f32"))
    a = p.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[a.dtype]
    w = synth.workload(a.workload)
    X, held = torch.from_numpy(synth.sweep_rows(a.workload, 32768)).cuda(), torch.from_numpy(w.X).cuda()
    model = gts.prepare(w.ensemble, "f32")
    net = Explainer(model, X, a.width, a.blocks, dtype, a.state_bits)
    net.fit(a.steps, a.rows, a.lr,
            report=lambda i, loss: print(f"step {i}: mean square error {loss:.4f}", flush=True))
    exact = gts.shap(model, held)
    print(f"held-out rows: {explained(exact, net.explain(held)):.4f} of the variance explained")
    for rows in (1, held.shape[0]):
        serve = net.server(rows)
        print(f"{rows} rows: network {_time(lambda: net.explain(held[:rows])):.0f} us, as a graph "
              f"{_time(lambda: serve(held[:rows])):.0f} us, exact "
              f"{_time(lambda: gts.shap(model, held[:rows])):.0f} us", flush=True)


if __name__ == "__main__":
    main()
