"""The layers together on the solver's batch: examples/text_denoiser.py."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_36522_gb300 import build as pa_build
    pa_build.build()


def test_stepped_and_captured_generations_agree():
    """The host-driven loop computes the rows that are there, the captured loop all rows with the count on the device. The
    library's matrix products may round differently for another number of rows: 16-bit values in between, 2^-8 of
    a net's part of 0.05 in eps each, summed over at most T steps with weights below 1."""
    import torch
    import text_denoiser
    stepped, generated, dx, dstates = text_denoiser.main()
    assert torch.isfinite(stepped).all() and torch.isfinite(dx).all() and torch.isfinite(dstates).all()
    assert (generated - stepped).abs().max() <= 50 * 0.05 * 2.0 ** -8 * stepped.abs().max()


def test_gradients_match_autograd_in_64_bits():
    import torch
    import torch.nn.functional as F
    import text_denoiser
    torch.manual_seed(1)
    shape, n = (4, 16, 24), 7
    alphas = [0.05 * i + 0.02 for i in range(11)]
    states = torch.randn(3, 19, 32, device="cuda").to(torch.bfloat16)
    lengths = torch.tensor([19, 0, 8], dtype=torch.int32, device="cuda")
    net = text_denoiser.TextDenoiser(shape, alphas, n, states, lengths, width=64, heads=4, kv_heads=2, dim=24)
    x = torch.randn(n, 4 * 16 * 24, device="cuda")
    miss = torch.tensor([[b, i] for i, b in enumerate((0, 0, 0, 1, 2, 2, 2))], dtype=torch.int32, device="cuda")
    deps = torch.randn_like(x)
    eps = net(x, miss).clone()
    dx, dstates = net.gradients(x, miss, deps)
    xd, sd = x.double().requires_grad_(), states.double().requires_grad_()
    d = lambda t: t.double()  # noqa: E731
    e = net.patches(xd).reshape(n, net.tokens, net.patch) @ d(net.embed)
    h = F.layer_norm(e, (64,), d(net.norms[0]), d(net.shifts[0]))
    q = (h @ d(net.wq)).view(n, net.tokens, 4, 24)
    kv = (sd @ d(net.wkv)).view(3, 19, 2, 2, 24)
    src = miss[:, 0].long()
    k, v = (kv[:, :, i][src].repeat_interleave(2, 2) for i in (0, 1))
    s = torch.einsum("nqhd,nkhd->nhqk", q, k) * 24 ** -0.5
    there = (torch.arange(19, device="cuda")[None] < lengths[:, None])[src][:, None, None]
    p = torch.where(there, torch.softmax(s.masked_fill(~there, -1e30), -1), 0.0)
    y = torch.einsum("nhqk,nkhd->nqhd", p, v).reshape(n, net.tokens, -1) @ d(net.wo) + e
    out = F.layer_norm(y, (64,), d(net.norms[1]), d(net.shifts[1])) @ d(net.unembed)
    c, hh, w = shape
    out = out.view(n, hh // 2, w // 2, c, 2, 2).permute(0, 3, 1, 4, 2, 5).reshape(n, -1)
    want = xd * d(net.sigma)[miss[:, 1].long(), None] + 0.05 * out
    want.backward(d(deps))
    # a chain of about ten roundings to bfloat16, each 2^-8 of its value at most
    assert (eps - want).norm() <= 10 * 2.0 ** -8 * 0.05 * out.norm()
    net_part = xd.grad - d(deps) * d(net.sigma)[miss[:, 1].long(), None]
    assert (dx - xd.grad).norm() <= 10 * 2.0 ** -8 * net_part.norm()
    assert (dstates.double() - sd.grad).norm() <= 10 * 2.0 ** -8 * sd.grad.norm()
    assert not dstates[1].any()
