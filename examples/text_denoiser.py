"""A small text-conditioned denoiser on the solver's batch, and the gradient of a loss on its eps.

One block of a diffusion denoiser with random weights: the latent in 2x2 patches as tokens, layer norm, cross attention to
the trajectory's text states, layer norm, eps. The rows of a batch are (trajectory, timestep) pairs; all rows of a trajectory
attend to one set of keys and values, picked by the miss list. It runs in the host-driven loop (``step`` / ``submit_eps``)
and, with the miss count on the device and every buffer its own, inside the captured loop of ``Solver.generate``.
``gradients`` is what guidance or the fitting of a prompt needs: d loss / d latents and d loss / d text states.

    python examples/text_denoiser.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_36522_gb300 import layers  # noqa: E402
from paper_2609_36522_gb300.solver import Solver  # noqa: E402


class TextDenoiser:
    """eps = sqrt(1 - a_t) x + 0.05 net(x, text): near the eps of standard normal data, so that sampling converges."""

    def __init__(self, latent_shape, alphas, rows, states, lengths=None, width=128, heads=4, kv_heads=2, dim=40,
                 dtype=torch.bfloat16, seed=0):
        c, h, w = latent_shape
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, m):
            return (torch.randn(n, m, generator=g, device="cuda") * n ** -0.5).to(dtype)

        self.shape, self.patch, self.tokens = latent_shape, 4 * c, h * w // 4
        self.heads, self.kv_heads, self.dim, self.width = heads, kv_heads, dim, width
        self.embed, self.unembed = weight(self.patch, width), weight(width, self.patch)
        self.wq, self.wo = weight(width, heads * dim), weight(heads * dim, width)
        self.wkv = weight(states.shape[2], 2 * kv_heads * dim)
        self.norms = [(1 + 0.1 * torch.randn(width, generator=g, device="cuda")).to(dtype) for _ in range(2)]
        self.shifts = [(0.1 * torch.randn(width, generator=g, device="cuda")).to(dtype) for _ in range(2)]
        self.sigma = torch.sqrt(1 - torch.tensor(alphas, dtype=torch.float32, device="cuda"))
        self.lengths = lengths
        self.set_text(states)
        # buffers for the captured loop, which allocates nothing
        n, t = rows, self.tokens
        self.buf = {k: torch.empty(n, t, m, dtype=dtype, device="cuda") for k, m in
                    (("p", self.patch), ("x", width), ("h", width), ("q", heads * dim), ("o", heads * dim), ("y", width),
                     ("e", self.patch))}
        self.eps = torch.empty(n, c * h * w, dtype=torch.float32, device="cuda")
        q = self.buf["q"].view(n, t, heads, dim)
        self.workspace = torch.empty(max(1, layers.cross_attention_workspace_bytes(q, self.k)), dtype=torch.uint8, device="cuda")

    def set_text(self, states):
        """states: [trajectories][length][features]; keys and values are made once per prompt, not per row."""
        self.states = states
        kv = (states @ self.wkv).view(*states.shape[:2], 2, self.kv_heads, self.dim)
        self.k, self.v = kv[:, :, 0], kv[:, :, 1]

    def patches(self, x):
        c, h, w = self.shape
        return x.view(-1, c, h // 2, 2, w // 2, 2).permute(0, 2, 4, 1, 3, 5)

    def __call__(self, x, miss_bt, count=None):
        """eps of rows x [n][D] with pairs miss_bt [n][2]; count: the device's miss count, the rows past it are stale."""
        n, b = x.shape[0], {k: t[:x.shape[0]] for k, t in self.buf.items()}
        c, h, w = self.shape
        b["p"].view(n, h // 2, w // 2, c, 2, 2).copy_(self.patches(x))
        torch.matmul(b["p"], self.embed, out=b["x"])
        layers.layer_norm(b["x"], self.norms[0], self.shifts[0], out=b["h"], count=count)
        torch.matmul(b["h"], self.wq, out=b["q"])
        heads = (n, self.tokens, self.heads, self.dim)
        layers.cross_attention(b["q"].view(heads), self.k, self.v, source=miss_bt[:, 0], lengths=self.lengths, count=count,
                               out=b["o"].view(heads), workspace=self.workspace)
        torch.matmul(b["o"], self.wo, out=b["y"])
        b["y"].add_(b["x"])
        layers.layer_norm(b["y"], self.norms[1], self.shifts[1], out=b["h"], count=count)
        torch.matmul(b["h"], self.unembed, out=b["e"])
        eps = self.eps[:n]
        net = b["e"].view(n, h // 2, w // 2, c, 2, 2).permute(0, 3, 1, 4, 2, 5)
        torch.mul(x, self.sigma[miss_bt[:, 1].long().clamp_(0, len(self.sigma) - 1), None], out=eps)
        eps.view(n, c, h // 2, 2, w // 2, 2).add_(net, alpha=0.05)
        return eps

    def gradients(self, x, miss_bt, deps):
        """(d loss / d x, d loss / d text states) for deps = d loss / d eps: the backward pass of the block."""
        n, (c, h, w) = x.shape[0], self.shape
        heads = (n, self.tokens, self.heads, self.dim)
        kw = {"source": miss_bt[:, 0], "lengths": self.lengths}
        e = self.patches(x).reshape(n, self.tokens, self.patch).to(self.embed.dtype) @ self.embed
        h1, *st1 = layers.layer_norm(e, self.norms[0], self.shifts[0], stats=True)
        q = (h1 @ self.wq).view(heads)
        o, lse = layers.cross_attention(q, self.k, self.v, stats=True, **kw)
        y = o.view(n, self.tokens, -1) @ self.wo + e
        _, *st2 = layers.layer_norm(y, self.norms[1], self.shifts[1], stats=True)
        dh = 0.05 * self.patches(deps).reshape(n, self.tokens, self.patch).to(self.embed.dtype) @ self.unembed.t()
        dy, _, _ = layers.layer_norm_backward(dh, y, *st2, self.norms[1], weight_grad=False, bias_grad=False)
        dq, dk, dv = layers.cross_attention_backward((dy @ self.wo.t()).view(heads), q, self.k, self.v, o, lse, **kw)
        de, _, _ = layers.layer_norm_backward(dq.view(n, self.tokens, -1) @ self.wq.t(), e, *st1, self.norms[0],
                                              weight_grad=False, bias_grad=False)
        dx = ((de + dy) @ self.embed.t()).float().view(n, h // 2, w // 2, c, 2, 2).permute(0, 3, 1, 4, 2, 5).reshape(n, -1)
        dx = dx + deps * self.sigma[miss_bt[:, 1].long(), None]
        return dx, torch.stack((dk, dv), 2).flatten(2) @ self.wkv.t()


def in_captured_loop(solver, net):
    """The denoiser for ``Solver.generate``: addresses in, the same eps buffer out."""
    rows = solver.batch * solver.window

    def at(ptr, dtype, cols):
        first = (ptr - solver.workspace.data_ptr()) // 4
        return solver.workspace.view(dtype)[first:first + rows * cols].view(rows, cols)

    return lambda bx, mb, nm: net(at(bx, torch.float32, solver.D), at(mb, torch.int32, 2), count=nm)


def main(T=50, window=25, batch=4, shape=(4, 32, 32)):
    torch.manual_seed(0)
    alphas = [0.02 + 0.98 * (i / T) ** 1.5 for i in range(T + 1)]
    states = torch.randn(batch, 77, 64, device="cuda").to(torch.bfloat16)
    lengths = torch.tensor([77 - 20 * b for b in range(batch)], dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        solver = Solver(T, window, shape, alphas, 1e-3, 0.05, batch=batch, stream=stream)
        net = TextDenoiser(shape, alphas, batch * solver.window, states, lengths)
        x0 = torch.randn(batch, solver.D, device="cuda")
        solver.init(x0)
        while (plan := solver.step()) is not None:
            if plan.n_miss:
                last = plan.batch_x.clone(), plan.miss_bt.clone()
                net(plan.batch_x, plan.miss_bt)
            solver.submit_eps(net.eps)
        stepped, evaluations = solver.result(), solver.nfe()
        generated = solver.generate(x0, in_captured_loop(solver, net))
        dx, dstates = net.gradients(*last, torch.ones_like(last[0]))
        layers.check()
    apart = float((generated - stepped).abs().max() / stepped.abs().max())
    print(f"{evaluations} evaluations; generate against step by step: {apart:.2e}; gradients {float(dx.norm()):.4g}, "
          f"{float(dstates.float().norm()):.4g}")
    return stepped, generated, dx, dstates


if __name__ == "__main__":
    main()
