"""Layer norm and cross attention, forward and backward, against their
definitions in 64 bits.

Every tolerance is a bound on what rounding does, element by element, from u
(half a unit of the tensors' type: 2^-24, 2^-11, 2^-8) and the arithmetic in 32
bits. Layer norm: the output is rounded once, u |y|; sums of n terms are made
of at most 64 roundings in a row, so mean and variance are off by 64 2^-24 of
the row's largest magnitude. Attention: scores are off by e = (D + 8) 2^-24
scale sum |q||k|, so a probability by 2 e of itself (and 2^-21 for the
exponential); probabilities and their gradients enter the second product rounded
to 16 bits, u of each term (float16: at least 2^-24), and the result is rounded
once more (float16: by 2^-25 at least, half of its smallest number). The backward pass also sees out rounded in dout . out.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half of torch.finfo(type).eps
E32 = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_36522_gb300 import build as pa_build
    pa_build.build()


def _torch():
    import torch
    return torch, {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _near(got, want, tol, what):
    torch, _ = _torch()
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25
    got = got.double()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - tol
    assert (over <= 0).all(), (what, float(over.max()), float((got - want).abs().max()))


# ---- layer norm ----------------------------------------------------------------

def _norm_inputs(rows, cols, dtype, seed=0, offset=0.7):
    torch, dts = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = (n(rows, cols) * (0.5 + n(rows, 1).abs()) + offset * n(1, cols)).to(dts[dtype])
    return x, (1 + 0.2 * n(cols)).to(dts[dtype]), (0.2 * n(cols)).to(dts[dtype]), (0.1 * n(rows, cols)).to(dts[dtype])


def _norm_ref(x, w, b, dy, eps):
    """-> dict of (value, tolerance) in 64 bits."""
    torch, _ = _torch()
    u = {torch.float32: U["fp32"], torch.float16: U["fp16"], torch.bfloat16: U["bf16"]}[x.dtype]
    x, dy = x.double(), dy.double()
    one = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device)
    w, b = one if w is None else w.double(), 0 * one if b is None else b.double()
    mean = x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    xh = (x - mean) * r
    e = 64 * E32 * (1 + x.abs().amax(-1, keepdim=True) * r)  # of an xhat, and of r relative to itself
    y = xh * w + b
    g = dy * w
    s1, s2 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    dx = r * (g - s1 - xh * s2)
    big = g.abs().amax(-1, keepdim=True) * (1 + xh.abs().amax(-1, keepdim=True)) ** 2
    n = x.shape[0]
    return {"y": (y, u * y.abs() + 2 * e * w.abs() * (1 + xh.abs())),
            "mean": (mean[..., 0], (e / r)[..., 0]), "rstd": (r[..., 0], (e * r * (1 + xh.abs().amax(-1, keepdim=True)))[..., 0]),
            "dx": (dx, u * dx.abs() + 4 * e * r * big),
            "dw": ((dy * xh).sum(0), u * (dy * xh).sum(0).abs() + (2 * e * dy.abs() * (1 + xh.abs())).sum(0)
                   + E32 * n * (dy * xh).abs().sum(0)),
            "db": (dy.sum(0), u * dy.sum(0).abs() + E32 * n * dy.abs().sum(0))}


def _norm_check(x, w, b, dy, eps=1e-5, **kw):
    from paper_2609_36522_gb300 import layers
    ref = _norm_ref(x, w, b, dy, eps)
    y, mean, rstd = layers.layer_norm(x, w, b, eps=eps, stats=True)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db)):
        _near(got, *ref[name], name)
    again = layers.layer_norm_backward(dy, x, mean, rstd, w)
    assert all((p == q).all() for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (2, 16), (17, 24), (33, 40), (5, 64), (9, 65), (300, 320), (8, 333),
                                       (700, 640), (40, 1000), (7, 1032), (6, 1111), (50, 1280), (4, 2056), (5, 4104),
                                       (3, 8192), (3, 8193), (2, 9000), (2, 30000)])
def test_norm_matches_definition(rows, cols, dtype):
    _norm_check(*_norm_inputs(rows, cols, dtype))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_norm_many_rows(dtype):
    _norm_check(*_norm_inputs(20011, 72, dtype))


@pytest.mark.parametrize("dtype,rows,cols", [("fp32", 60001, 72), ("bf16", 80003, 72), ("fp16", 20005, 320), ("bf16", 30001, 128),
                                             ("fp32", 9001, 1000)])
def test_norm_rows_through_rings_and_sums_of_their_own(dtype, rows, cols):
    """As many rows as the kernels for many rows ask for, a last stage that is not full; also not one behind the
    other, over themselves, with a device count that ends inside a stage."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    x, w, b, dy = _norm_inputs(rows, cols, dtype)
    _norm_check(x, w, b, dy)
    y, mean, rstd = layers.layer_norm(x, w, b, stats=True)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w)
    wide = torch.zeros(rows, cols + 8, dtype=x.dtype, device="cuda")
    wide[:, :cols] = x
    _near(layers.layer_norm(wide[:, :cols], w, b), *_norm_ref(x, w, b, dy, 1e-5)["y"], "y")
    over = x.clone()
    assert (layers.layer_norm(over, w, b, out=over) == y).all()
    over = dy.clone()
    again = layers.layer_norm_backward(over, x, mean, rstd, w, dx=over)
    assert (over == dx).all() and (again[1] == dw).all() and (again[2] == db).all()
    n = rows - 37
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    layers.layer_norm(x, w, b, out=out, count=count)
    assert (out[:n] == y[:n]).all() and (out[n:] == 7.0).all()
    dx2, dw2, db2 = layers.layer_norm_backward(dy, x, mean, rstd, w, dx=torch.full_like(x, 7.0), count=count)
    assert (dx2[:n] == dx[:n]).all() and (dx2[n:] == 7.0).all()
    ref = _norm_ref(x[:n], w, b, dy[:n], 1e-5)
    _near(dw2, *ref["dw"], "dw")
    _near(db2, *ref["db"], "db")


@pytest.mark.parametrize("dtype,rows,cols", [("fp16", 90001, 64), ("fp16", 5003, 640), ("bf16", 5001, 1024), ("fp32", 30001, 256),
                                             ("fp32", 5000, 500), ("fp32", 1301, 585), ("fp16", 2003, 257), ("bf16", 1300, 1111),
                                             ("fp32", 700, 3010), ("bf16", 611, 4099), ("fp16", 320, 8189), ("fp32", 320, 8190)])
def test_norm_many_rows_of_both_directions(dtype, rows, cols):
    """Both directions through rings of rows, on 16-byte boundaries and not; strided, over themselves, with a device
    count, the last row at its tensor's end and beyond it NaN."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    x, w, b, dy = _norm_inputs(rows, cols, dtype)
    _norm_check(x, w, b, dy)
    _norm_check(x, None, b, dy)
    ref = _norm_ref(x, w, b, dy, 1e-5)
    y, mean, rstd = layers.layer_norm(x, w, b, stats=True)
    dx, dw, db = layers.layer_norm_backward(dy, x, mean, rstd, w)
    wide, dwide = (torch.full((rows, cols + 8), math.nan, dtype=x.dtype, device="cuda") for _ in range(2))
    wide[:, :cols] = x
    dwide[:, :cols] = dy
    _near(layers.layer_norm(wide[:, :cols], w, b), *ref["y"], "y")
    got = layers.layer_norm_backward(dwide[:, :cols], wide[:, :cols], mean, rstd, w, dx=dwide[:, :cols])
    for name, g in zip(("dx", "dw", "db"), got):
        _near(g, *ref[name], name)
    assert torch.isnan(dwide[:, cols:]).all()
    over = x.clone()
    assert (layers.layer_norm(over, w, b, out=over) == y).all()
    over = x.clone()
    again = layers.layer_norm_backward(dy, over, mean, rstd, w, dx=over)
    assert (over == dx).all() and (again[1] == dw).all() and (again[2] == db).all()
    only, none, _ = layers.layer_norm_backward(dy, x, mean, rstd, w, weight_grad=False, bias_grad=False)
    assert none is None
    _near(only, *ref["dx"], "dx")
    n = rows - 37
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    layers.layer_norm(x, w, b, out=out, count=count)
    assert (out[:n] == y[:n]).all() and (out[n:] == 7.0).all()
    dx2, dw2, db2 = layers.layer_norm_backward(dy, x, mean, rstd, w, dx=torch.full_like(x, 7.0), count=count)
    assert (dx2[:n] == dx[:n]).all() and (dx2[n:] == 7.0).all()
    ref = _norm_ref(x[:n], w, b, dy[:n], 1e-5)
    _near(dw2, *ref["dw"], "dw")
    _near(db2, *ref["db"], "db")


def test_norm_without_weights_and_single_gradients():
    from paper_2609_36522_gb300 import layers
    x, w, b, dy = _norm_inputs(21, 96, "bf16")
    _norm_check(x, None, None, dy)
    _norm_check(x, w, None, dy)
    _norm_check(x, None, b, dy)
    y, mean, rstd = layers.layer_norm(x, w, b, stats=True)
    full = layers.layer_norm_backward(dy, x, mean, rstd, w)
    part = layers.layer_norm_backward(dy, x, mean, rstd, w, weight_grad=False)
    assert part[1] is None and (part[2] == full[2]).all() and (part[0] == full[0]).all()
    none = layers.layer_norm_backward(dy, x, mean, rstd, w, weight_grad=False, bias_grad=False)
    assert none[1:] == (None, None) and (none[0] == full[0]).all()


def test_norm_large_offset_and_constant_rows():
    """A mean far above the spread (the variance is the two-pass one), a row of
    one value (variance 0), eps alone under the root."""
    torch, _ = _torch()
    x, w, b, dy = _norm_inputs(12, 200, "fp32", offset=0.0)
    x[:6] += 1000.0
    x[6] = 3.25
    _norm_check(x, w, b, dy)


@pytest.mark.parametrize("dtype,cols", [("bf16", 48), ("fp32", 30), ("fp16", 31)])
def test_norm_strided_offset_and_in_place(dtype, cols):
    """Rows inside wider ones, rows off the 16-byte boundaries, y over x, dx over dy."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    wide, _, _, dwide = _norm_inputs(26, cols + 9, dtype)
    _, w, b, _ = _norm_inputs(1, cols, dtype)
    for first in (0, 1, 8):
        x, dy = wide[:, first:first + cols], dwide[:, first:first + cols]
        _norm_check(x, w, b, dy)
    x, dy = wide[:, :cols], dwide[:, 1:1 + cols]
    y, mean, rstd = layers.layer_norm(x, w, b, stats=True)
    x3 = wide.clone().view(2, 13, -1)[..., :cols]  # three axes at one row distance
    y3, m3, r3 = layers.layer_norm(x3, w, b, stats=True)
    assert (y3.reshape(26, cols) == y).all() and (m3.reshape(-1) == mean).all()
    dx, _, _ = layers.layer_norm_backward(dy, x, mean, rstd, w)
    over = dwide.clone()
    layers.layer_norm_backward(over[:, 1:1 + cols], x, mean, rstd, w, dx=over[:, 1:1 + cols])
    assert (over[:, 1:1 + cols] == dx).all() and (over[:, :1] == dwide[:, :1]).all()
    assert (over[:, 1 + cols:] == dwide[:, 1 + cols:]).all()
    xc = wide.clone()
    layers.layer_norm(xc[:, :cols], w, b, out=xc[:, :cols])
    assert (xc[:, :cols] == y).all() and (xc[:, cols:] == wide[:, cols:]).all()


@pytest.mark.parametrize("n", [0, 1, 3, 5, 9, -2])
def test_norm_device_count(n):
    """Only the first `count` items: the rest of y and dx stays, the sums leave it out."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    x, w, b, dy = (t if t.dim() == 1 else t.view(5, 7, 40) for t in _norm_inputs(35, 40, "bf16"))
    k = min(max(n, 0), 5)
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    y, mean, rstd = layers.layer_norm(x, w, b, out=out, stats=True, count=count)
    yf, mf, rf = layers.layer_norm(x, w, b, stats=True)
    assert (y[:k] == yf[:k]).all() and (y[k:] == 7.0).all()
    dx = torch.full_like(x, 7.0)
    dx, dw, db = layers.layer_norm_backward(dy, x, mf, rf, w, dx=dx, count=count)
    assert (dx[k:] == 7.0).all()
    if k:
        ref = _norm_ref(x[:k].reshape(-1, 40), w, b, dy[:k].reshape(-1, 40), 1e-5)
        _near(dx[:k].reshape(-1, 40), *ref["dx"], "dx")
        _near(dw, *ref["dw"], "dw")
        _near(db, *ref["db"], "db")
    else:
        assert not dw.any() and not db.any()


def test_norm_no_rows():
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    x = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(40, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = layers.layer_norm(x, w, None, stats=True)
    dx, dw, db = layers.layer_norm_backward(x, x, mean, rstd, w)
    assert y.shape == x.shape and dx.shape == x.shape and not dw.any() and not db.any()


def test_norm_gradient_against_differences():
    """<dx, e> against (L(x + h e) - L(x - h e)) / 2h of the definition, L = <dy, y>."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    x, w, b, dy = _norm_inputs(9, 56, "fp32")
    y, mean, rstd = layers.layer_norm(x, w, b, stats=True)
    got = layers.layer_norm_backward(dy, x, mean, rstd, w)
    ref = _norm_ref(x, w, b, dy, 1e-5)

    def loss(xd, wd, bd):
        v, m = torch.var_mean(xd, -1, correction=0, keepdim=True)
        return ((xd - m) / torch.sqrt(v + 1e-5) * wd + bd).mul(dy.double()).sum()

    at = [x.double(), w.double(), b.double()]
    g = torch.Generator(device="cuda").manual_seed(3)
    for i, name in enumerate(("dx", "dw", "db")):
        e = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        hi, lo = ([t + s * h * e if k == i else t for k, t in enumerate(at)] for s in (1, -1))
        diff = (loss(*hi) - loss(*lo)) / (2 * h)
        tol = (ref[name][1] * e.abs()).sum() + 1e-7 * (ref[name][0] * e).abs().sum()
        assert (diff - (got[i].double() * e).sum()).abs() <= tol, name


# ---- cross attention -----------------------------------------------------------

def _attn_inputs(N, G, Q, K, H, J, D, dtype, seed=0, keep="all", sources=None):
    torch, dts = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = dts[dtype]
    first = n(1, 1, J, 1, D)
    q = (n(N, Q, J, H // J, D) + 0.5 * first).view(N, Q, H, D).to(dt)
    kv = n(G, K, 2, J, D)
    kv[:, :1, :1] += 1.5 * first.view(1, 1, 1, J, D)
    kv = kv.to(dt)
    kw = {}
    src = [i * G // max(N, 1) for i in range(N)] if sources is None else sources
    kw["source"] = torch.tensor([[s, 7] for s in src], dtype=torch.int32, device="cuda").view(N, 2)[:, 0]
    if keep in ("lengths", "both"):
        kw["lengths"] = torch.randint(0, K + 1, (G,), generator=g, device="cuda", dtype=torch.int32)
        if G > 1:
            kw["lengths"][0] = 0
        kw["lengths"][-1] = K
    if keep in ("mask", "both"):
        kw["mask"] = torch.rand(G, K, generator=g, device="cuda") < 0.7
        if G > 2:
            kw["mask"][1] = False
    # what does not count may hold anything
    kept = _kept(kv[:, :, 0], **{k: kw.get(k) for k in ("lengths", "mask")})
    kv[~kept] = torch.where(torch.rand(kv[~kept].shape, generator=g, device="cuda") < 0.5, float("nan"), float("inf")).to(dt)
    return q, kv[:, :, 0], kv[:, :, 1], (0.1 * n(N, Q, H, D)).to(dt), kw


def _kept(k, lengths=None, mask=None):
    torch, _ = _torch()
    kept = torch.ones(k.shape[:2], dtype=torch.bool, device=k.device)
    if lengths is not None:
        kept &= torch.arange(k.shape[1], device=k.device)[None] < lengths[:, None]
    if mask is not None:
        kept &= mask != 0
    return kept


def _attn_ref(q, k, v, do, source, scale, lengths=None, mask=None):
    """-> dict of (value, tolerance) in 64 bits, one row of one head after another source."""
    torch, _ = _torch()
    u = {torch.float16: U["fp16"], torch.bfloat16: U["bf16"]}[q.dtype]
    low = 2.0 ** -24 if q.dtype == torch.float16 else 0.0
    N, Q, H, D = q.shape
    G, K, J, _ = k.shape
    R = H // J
    f64 = dict(dtype=torch.float64, device=q.device)
    kept = _kept(k, lengths, mask)
    out, tout = torch.zeros(N, Q, H, D, **f64), torch.zeros(N, Q, H, D, **f64)
    lse, tlse = torch.full((N, Q, H), -math.inf, **f64), torch.zeros(N, Q, H, **f64)
    dq, tdq = torch.zeros_like(out), torch.zeros_like(out)
    dk, tdk, dv, tdv = (torch.zeros(G, K, J, D, **f64) for _ in range(4))
    for n, g in enumerate(source.tolist()):
        at = kept[g].nonzero()[:, 0]
        if not 0 <= g < G or at.numel() == 0:
            continue
        for h in range(H):
            j = h // R
            qq, dd = q[n, :, h].double(), do[n, :, h].double()
            kk, vv = k[g, at, j].double(), v[g, at, j].double()
            s = scale * qq @ kk.T
            p = torch.softmax(s, -1)
            o = p @ vv
            es = (D + 8) * E32 * scale * qq.abs() @ kk.abs().T
            e = 2 * es.amax(-1, keepdim=True) + 2.0 ** -21  # of a probability, relative
            out[n, :, h], lse[n, :, h] = o, torch.logsumexp(s, -1)
            tout[n, :, h] = (u + 2 * e) * (p @ vv.abs()) + low * vv.abs().sum(0) + u * o.abs()
            tlse[n, :, h] = e[:, 0] + 4 * E32 * lse[n, :, h].abs()
            dp = dd @ vv.T
            ds = p * (dp - (dd * o).sum(-1, keepdim=True))
            # of a value of ds: its own rounding, its probability's error, and those of dp and delta
            off = (u + 2 * e) * ds.abs() + low + p * (
                (dd.abs() * (2 * tout[n, :, h])).sum(-1, keepdim=True) + (D + 8) * E32 * dd.abs() @ vv.abs().T)
            dq[n, :, h] = scale * ds @ kk
            tdq[n, :, h] = scale * off @ kk.abs() + u * dq[n, :, h].abs()
            dk[g, at, j] += scale * ds.T @ qq
            tdk[g, at, j] += scale * off.T @ qq.abs()
            dv[g, at, j] += p.T @ dd
            tdv[g, at, j] += ((u + 2 * e) * p + low).T @ dd.abs()
    tdk += u * dk.abs() + 2.0 ** -18 * tdk / u  # sums over many rows in 32 bits
    tdv += u * dv.abs() + 2.0 ** -18 * tdv / u
    return {"out": (out, tout), "lse": (lse, tlse), "dq": (dq, tdq), "dk": (dk, tdk), "dv": (dv, tdv)}


def _lse_near(got, want, tol):
    torch, _ = _torch()
    none = torch.isinf(want)
    assert (got[none] == -math.inf).all()
    _near(got[~none], want[~none], tol[~none], "lse")


def _attn_check(q, k, v, do, kw, scale=None):
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    ref = _attn_ref(q, k, v, do, scale=q.shape[3] ** -0.5 if scale is None else scale, **kw)
    out, lse = layers.cross_attention(q, k, v, scale=scale, stats=True, **kw)
    _near(out, *ref["out"], "out")
    _lse_near(lse, *ref["lse"])
    assert (layers.cross_attention(q, k, v, scale=scale, **kw) == out).all()
    grads = layers.cross_attention_backward(do, q, k, v, out, lse, scale=scale, **kw)
    for name, got in zip(("dq", "dk", "dv"), grads):
        _near(got, *ref[name], name)
    again = layers.cross_attention_backward(do, q, k, v, out, lse, scale=scale, **kw)
    assert all((a == b).all() for a, b in zip(grads, again))
    layers.check()
    return out, lse, grads


# items, sources, tokens, keys, heads, key heads, head size
SHAPES = [
    (1, 1, 1, 1, 1, 1, 8), (1, 1, 1, 5, 2, 1, 16), (3, 3, 1, 300, 4, 4, 64), (2, 2, 1, 1030, 8, 2, 128),
    (4, 2, 33, 19, 4, 2, 24), (6, 3, 64, 77, 8, 8, 40), (5, 1, 130, 77, 2, 2, 80), (2, 2, 128, 128, 2, 2, 64),
    (3, 2, 127, 129, 2, 1, 64), (2, 1, 257, 255, 3, 3, 128), (4, 4, 20, 16, 5, 5, 160), (2, 1, 140, 200, 2, 1, 256),
    (1, 1, 700, 500, 2, 2, 72), (2, 2, 65, 333, 6, 2, 104), (7, 5, 9, 231, 2, 2, 120), (1, 1, 4, 2100, 3, 1, 96),
    (2, 1, 300, 1, 2, 2, 48), (9, 2, 50, 64, 4, 1, 8), (2, 2, 200, 600, 1, 1, 192), (3, 3, 2, 40, 7, 7, 208),
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_attention_matches_definition(shape, dtype):
    q, k, v, do, kw = _attn_inputs(*shape, dtype)
    _attn_check(q, k, v, do, kw)


@pytest.mark.parametrize("keep", ["lengths", "mask", "both"])
@pytest.mark.parametrize("shape", [(6, 3, 33, 19, 4, 2, 24), (5, 4, 140, 77, 2, 2, 40), (4, 3, 1, 700, 4, 1, 64),
                                   (3, 3, 150, 300, 4, 2, 128), (4, 4, 70, 260, 2, 2, 160)],
                         ids=lambda s: "x".join(map(str, s)))
def test_attention_keys_that_do_not_count(shape, keep):
    """Lengths of zero, masks that leave nothing, infinities and NaN in what does not count."""
    q, k, v, do, kw = _attn_inputs(*shape, "bf16", keep=keep)
    out, lse, (dq, dk, dv) = _attn_check(q, k, v, do, kw)
    kept = _kept(k, kw.get("lengths"), kw.get("mask"))
    assert not dk[~kept].any() and not dv[~kept].any()
    for n, g in enumerate(kw["source"].tolist()):
        if not kept[g].any():
            assert not out[n].any() and not dq[n].any()


# tensors of a megabyte and more go by bulk copies: whole tiles, tiles of several heads, last tiles, heads off the
# block widths, groups of heads that no tile holds whole
LARGE = [
    (10, 2, 515, 77, 4, 4, 40), (6, 3, 600, 300, 4, 2, 64), (4, 2, 700, 500, 3, 3, 128), (6, 2, 1024, 64, 3, 1, 80),
    (40, 4, 64, 100, 4, 4, 80), (30, 2, 1000, 90, 2, 2, 24), (4, 2, 520, 260, 8, 1, 160), (3, 1, 400, 333, 4, 2, 256),
    (70, 1, 1024, 31, 1, 1, 8), (8, 8, 130, 2000, 4, 4, 96), (20, 2, 1024, 150, 2, 2, 16), (5, 2, 600, 140, 2, 2, 208),
]


@pytest.mark.parametrize("keep", ["all", "lengths", "mask"])
@pytest.mark.parametrize("shape", LARGE, ids=lambda s: "x".join(map(str, s)))
def test_attention_by_bulk_copies(shape, keep):
    q, k, v, do, kw = _attn_inputs(*shape, "bf16" if shape[0] % 4 else "fp16", keep=keep)
    _attn_check(q, k, v, do, kw)


def test_attention_sources_in_any_order_and_unused():
    """Items not sorted by source, a source without items (its gradients are zero), default sources."""
    q, k, v, do, kw = _attn_inputs(7, 5, 21, 30, 2, 2, 40, "bf16", sources=[3, 0, 3, 1, 0, 4, 3])
    _, _, (_, dk, dv) = _attn_check(q, k, v, do, kw)
    assert not dk[2].any() and not dv[2].any()
    from paper_2609_36522_gb300 import layers
    a = layers.cross_attention(q[:5], k, v, source=None)
    import torch
    b = layers.cross_attention(q[:5], k, v, source=torch.arange(5, dtype=torch.int32, device="cuda"))
    assert (a == b).all()


@pytest.mark.parametrize("shape", [(4, 2, 1, 200, 2, 2, 64), (4, 2, 150, 200, 2, 2, 64)])
def test_attention_bad_source_is_reported(shape):
    from paper_2609_36522_gb300 import abi, layers
    q, k, v, do, kw = _attn_inputs(*shape, "bf16", sources=[0, 2, -1, 1])
    out, lse = layers.cross_attention(q, k, v, stats=True, **kw)
    with pytest.raises(abi.PaError) as e:
        layers.check()
    assert e.value.status == abi.PA_ERR_DEVICE
    layers.check()  # cleared
    assert not out[1].any() and not out[2].any() and out[0].any() and out[3].any()
    dq, dk, dv = layers.cross_attention_backward(do, q, k, v, out, lse, **kw)
    with pytest.raises(abi.PaError):
        layers.check()
    assert not dq[1].any() and not dq[2].any()
    good = [0, 3]
    ref = _attn_ref(q[good], k, v, do[good], kw["source"][good], 64 ** -0.5)
    _near(dk, *ref["dk"], "dk")
    _near(dv, *ref["dv"], "dv")


@pytest.mark.parametrize("n", [0, 1, 3, 4, 99, -1])
@pytest.mark.parametrize("shape", [(4, 2, 1, 300, 2, 2, 64), (4, 2, 150, 77, 2, 2, 40), (4, 2, 150, 300, 4, 2, 64)])
def test_attention_device_count(shape, n):
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    q, k, v, do, kw = _attn_inputs(*shape, "fp16")
    c = min(max(n, 0), 4)
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    layers.cross_attention(q, k, v, out=out, count=count, **kw)
    full, lse = layers.cross_attention(q, k, v, stats=True, **kw)
    assert (out[c:] == 7.0).all()
    ref = _attn_ref(q[:c], k, v, do[:c], kw["source"][:c], shape[6] ** -0.5)
    _near(out[:c], *ref["out"], "out")
    dq = torch.full_like(q, 7.0)
    _, dk, dv = layers.cross_attention_backward(do, q, k, v, full, lse, dq=dq, count=count, **kw)
    assert (dq[c:] == 7.0).all()
    _near(dq[:c], *ref["dq"], "dq")
    _near(dk, *ref["dk"], "dk")
    _near(dv, *ref["dv"], "dv")


def test_attention_strides():
    """Every tensor a view: heads before tokens, rows inside wider ones, gradients into a fused buffer."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    N, G, Q, K, H, J, D = 3, 2, 141, 150, 4, 2, 40
    q, k, v, do, kw = _attn_inputs(N, G, Q, K, H, J, D, "bf16")
    out, lse, grads = _attn_check(q, k, v, do, kw)

    def moved(t):  # heads outermost, a row of 64
        w = torch.full((t.shape[2], t.shape[0], t.shape[1], 64), float("nan"), dtype=t.dtype, device="cuda")
        m = w[..., 8:8 + D].permute(1, 2, 0, 3)
        m.copy_(t)
        return m

    qm, km, vm, dm, om = (moved(t) for t in (q, k, v, do, out))
    om.fill_(0)
    _, lm = layers.cross_attention(qm, km, vm, out=om, stats=True, **kw)
    assert (om == out).all() and (lm == lse).all()
    fused = torch.full((G, K, 2, J, D), 5.0, dtype=q.dtype, device="cuda")
    dq = moved(torch.zeros_like(q))
    layers.cross_attention_backward(dm, qm, km, vm, om, lm, dq=dq, dk=fused[:, :, 0], dv=fused[:, :, 1], **kw)
    assert (dq == grads[0]).all() and (fused[:, :, 0] == grads[1]).all() and (fused[:, :, 1] == grads[2]).all()


@pytest.mark.parametrize("tokens", [1, 140])
def test_attention_offsets_beyond_32_bits(tokens):
    """Keys and values spread over more than 2^32 bytes and 2^31 elements."""
    torch, _ = _torch()
    q, k, v, do, kw = _attn_inputs(1, 1, tokens, 290, 1, 1, 64, "bf16")
    step = (1 << 31) // 256
    buf = torch.empty(290 * step, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (1, 290, 2, 1, 64), (290 * step, step, 64, 64, 1))
    far[:, :, 0].copy_(k)
    far[:, :, 1].copy_(v)
    _attn_check(q, far[:, :, 0], far[:, :, 1], do, kw)


@pytest.mark.parametrize("tokens", [1, 130])
def test_attention_large_scores(tokens):
    """Scores far apart (one key takes all), large magnitudes, later keys above earlier ones by far."""
    torch, _ = _torch()
    q, k, v, do, kw = _attn_inputs(2, 1, tokens, 400, 2, 2, 64, "bf16")
    k = (k.float() * torch.linspace(0.1, 12.0, 400, device="cuda")[None, :, None, None]).to(k.dtype)
    _attn_check(q, k, v, do, kw)
    _attn_check(q, k, v, do, kw, scale=0.01)


def test_attention_empty_sizes():
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    q, k, v, do, kw = _attn_inputs(3, 2, 5, 12, 2, 2, 16, "fp16")
    out, lse = layers.cross_attention(q, k[:, :0], v[:, :0], stats=True, **kw)  # no keys
    assert not out.any() and (lse == -math.inf).all()
    dq, dk, dv = layers.cross_attention_backward(do, q, k[:, :0], v[:, :0], out, lse, **kw)
    assert not dq.any() and dk.numel() == 0
    e, src = q[:0], kw["source"][:0]
    out, lse = layers.cross_attention(e, k, v, stats=True, source=src)  # no items
    dq, dk, dv = layers.cross_attention_backward(e, e, k, v, out, lse, source=src)
    assert out.shape == e.shape and not dk.any() and not dv.any()
    t = q[:, :0]
    out, lse = layers.cross_attention(t, k, v, stats=True, **kw)  # no tokens
    dq, dk, dv = layers.cross_attention_backward(t, t, k, v, out, lse, **kw)
    assert not dk.any() and not dv.any()


def test_attention_gradient_against_differences():
    """<grad, e> against (L(x + h e) - L(x - h e)) / 2h of the definition, L = <dout, out>."""
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    q, k, v, do, kw = _attn_inputs(4, 2, 11, 23, 4, 2, 24, "fp16")
    k, v = k.contiguous(), v.contiguous()
    out, lse = layers.cross_attention(q, k, v, stats=True, **kw)
    got = layers.cross_attention_backward(do, q, k, v, out, lse, **kw)
    ref = _attn_ref(q, k, v, do, scale=24 ** -0.5, **kw)
    src = kw["source"].long()

    def loss(q, k, v):
        k, v = (t[src].repeat_interleave(2, 2) for t in (k, v))
        p = torch.softmax(torch.einsum("nqhd,nkhd->nhqk", q, k) * 24 ** -0.5, -1)
        return (torch.einsum("nhqk,nkhd->nqhd", p, v) * do.double()).sum()

    at = [t.double() for t in (q, k, v)]
    g = torch.Generator(device="cuda").manual_seed(3)
    for i, name in enumerate(("dq", "dk", "dv")):
        e = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        hi, lo = ([t + s * h * e if m == i else t for m, t in enumerate(at)] for s in (1, -1))
        diff = (loss(*hi) - loss(*lo)) / (2 * h)
        tol = (ref[name][1] * e.abs()).sum() + 1e-7 * (ref[name][0] * e).abs().sum()
        assert (diff - (got[i].double() * e).sum()).abs() <= tol, name


@pytest.mark.parametrize("tokens", [1, 200])
def test_layers_on_another_stream_and_in_a_graph(tokens):
    from paper_2609_36522_gb300 import layers
    torch, _ = _torch()
    q, k, v, do, kw = _attn_inputs(4, 2, tokens, 300, 4, 2, 64, "bf16", keep="mask")
    want, lse = layers.cross_attention(q, k, v, stats=True, **kw)
    wgrads = layers.cross_attention_backward(do, q, k, v, want, lse, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = layers.cross_attention(q, k, v, stream=side, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert (out == want).all()
    qs, out, ls = q.clone(), torch.zeros_like(q), torch.zeros_like(lse)
    count = torch.tensor([4], dtype=torch.int32, device="cuda")
    ws = torch.empty(max(1, layers.cross_attention_workspace_bytes(q, k, mask=True)), dtype=torch.uint8, device="cuda")
    wb = torch.empty(max(1, layers.cross_attention_workspace_bytes(q, k, mask=True, backward=True)), dtype=torch.uint8,
                     device="cuda")
    grads = [torch.zeros_like(t) for t in (q, k.contiguous(), v.contiguous())]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layers.cross_attention(qs, k, v, out=out, lse=ls, count=count, workspace=ws, **kw)
        layers.cross_attention_backward(do, qs, k, v, out, ls, dq=grads[0], dk=grads[1], dv=grads[2], count=count,
                                        workspace=wb, **kw)
    graph.replay()
    assert (out == want).all() and all((a == b).all() for a, b in zip(grads, wgrads))
    qs.copy_(q.flip(0))
    graph.replay()
    want2, lse2 = layers.cross_attention(qs, k, v, stats=True, **kw)
    assert (out == want2).all() and (ls == lse2).all()


# ---- refusals --------------------------------------------------------------------

def test_refusals():
    from paper_2609_36522_gb300 import abi, layers
    torch, _ = _torch()
    x, w, b, dy = _norm_inputs(6, 32, "bf16")
    y, mean, rstd = layers.layer_norm(x, w, b, stats=True)
    for call in (lambda: layers.layer_norm(x.cpu()), lambda: layers.layer_norm(x.double()),
                 lambda: layers.layer_norm(x, w.float()), lambda: layers.layer_norm(x, w[:16]),
                 lambda: layers.layer_norm(x.t()), lambda: layers.layer_norm(x, out=y[:3]),
                 lambda: layers.layer_norm(x, mean=mean.half()),
                 lambda: layers.layer_norm(torch.as_strided(x, (2, 2, 32), (96, 32, 1))),
                 lambda: layers.layer_norm_backward(dy[:3], x, mean, rstd, w),
                 lambda: layers.layer_norm_backward(dy, x, mean[:3], rstd, w),
                 lambda: layers.layer_norm(x, count=torch.tensor([1], device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: layers.layer_norm(x, eps=-1.0), abi.PA_ERR_ARG),
                         (lambda: layers.layer_norm(x, eps=float("nan")), abi.PA_ERR_ARG),
                         (lambda: layers.layer_norm(x[:1].expand(6, 32)), abi.PA_ERR_ARG),
                         (lambda: layers.layer_norm_backward(dy, x, mean, rstd, w, workspace=torch.empty(
                             16, dtype=torch.uint8, device="cuda")), abi.PA_ERR_WORKSPACE)):
        with pytest.raises(abi.PaError) as e:
            call()
        assert e.value.status == status
    q, k, v, do, kw = _attn_inputs(3, 2, 5, 12, 4, 2, 16, "bf16")
    out, lse = layers.cross_attention(q, k, v, stats=True, **kw)
    src = kw["source"]
    for call in (lambda: layers.cross_attention(q.float(), k.float(), v.float(), **kw),
                 lambda: layers.cross_attention(q, k.half(), v, **kw), lambda: layers.cross_attention(q, k, v[:, :5], **kw),
                 lambda: layers.cross_attention(q[0], k, v, **kw), lambda: layers.cross_attention(q, k, v, source=src.long()),
                 lambda: layers.cross_attention(q, k, v, source=src[:2]),
                 lambda: layers.cross_attention(q, k, v, lengths=src[:1], source=src),
                 lambda: layers.cross_attention(q, k, v, mask=torch.ones(2, 5, dtype=torch.bool, device="cuda"), source=src),
                 lambda: layers.cross_attention(q, k, v, out=out[:2], **kw),
                 lambda: layers.cross_attention_backward(do, q, k, v, out, lse[:2], **kw),
                 lambda: layers.cross_attention_backward(do[:2], q, k, v, out, lse, **kw)):
        with pytest.raises(ValueError):
            call()
    many = torch.zeros(3, 5, 4, 264, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: layers.cross_attention(q, k, v), lambda: layers.cross_attention(q[..., :12], k[..., :12], v[..., :12], **kw),
                 lambda: layers.cross_attention(q[:, :, :3], k, v, **kw), lambda: layers.cross_attention(many, many, many),
                 lambda: layers.cross_attention(q, k, v, scale=0.0, **kw), lambda: layers.cross_attention(q, k, v, scale=-1.0, **kw),
                 lambda: layers.cross_attention(q, k, v, scale=float("inf"), **kw),
                 lambda: layers.cross_attention(many[..., 4:20], k, v, **kw)):
        with pytest.raises(abi.PaError) as e:
            call()
        assert e.value.status == abi.PA_ERR_ARG
    mask = torch.ones(2, 12, dtype=torch.bool, device="cuda")
    with pytest.raises(abi.PaError) as e:
        layers.cross_attention(q, k, v, mask=mask, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"), **kw)
    assert e.value.status == abi.PA_ERR_WORKSPACE


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("shape", [(3, 2, 65, 2, 2, 2, 64), (5, 3, 33, 19, 4, 2, 24), (4, 1, 300, 77, 4, 4, 40),
                                   (1, 1, 257, 300, 4, 2, 128), (2, 2, 70, 130, 2, 2, 208)])
def test_attention_gradients_are_as_near_as_their_rounding(shape, dtype):
    """Probabilities and their gradients enter the second products with 16 bits and more, so nearly all of a gradient's
    error is that of its last rounding: the norm of the error is at most 1.25 of that of the exact gradient, rounded."""
    from paper_2609_36522_gb300 import layers
    q, k, v, do, kw = _attn_inputs(*shape, dtype)
    ref = _attn_ref(q, k, v, do, scale=shape[6] ** -0.5, **kw)
    out, lse = layers.cross_attention(q, k, v, stats=True, **kw)
    got = layers.cross_attention_backward(do, q, k, v, out, lse, **kw)
    for name, g in zip(("dq", "dk", "dv"), got):
        want = ref[name][0]
        rounding = float((want.to(g.dtype).double() - want).norm())
        assert float((g.double() - want).norm()) <= 1.25 * rounding, name


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_attention_gradients_of_a_single_key(dtype):
    """One key has all of the weight: its score does not matter, so dq and dk are 0 but for the rounding of dout . v,
    which both differences are made of: within 4 2^-24 of it for dq, and for dk (products the other way round) within the
    (D + 8) 2^-24 sum |dout||v| that a sum of D terms may be off by in each of the two. Scores are large, so that lse is off by
    more than that."""
    from paper_2609_36522_gb300 import layers
    q, k, v, do, kw = _attn_inputs(3, 2, 200, 1, 4, 2, 64, dtype)
    q = q * 8
    scale = 0.5
    out, lse = layers.cross_attention(q, k, v, scale=scale, stats=True, **kw)
    dq, dk, dv = layers.cross_attention_backward(do, q, k, v, out, lse, scale=scale, **kw)
    src = kw["source"].long()
    kd, vd = (t.double()[src][:, :, :, None].expand(-1, -1, -1, 2, -1).flatten(2, 3) for t in (k, v))  # [items][1][heads][D]
    dot = (do.double() * vd).sum(-1, keepdim=True).abs()
    most = (do.double() * vd).abs().sum(-1, keepdim=True)
    assert float(lse.abs().max()) > 30
    _near(dq, 0 * q.double(), 1.01 * 4 * E32 * scale * (dot + 72 * E32 * most) * kd.abs() + 2.0 ** -130, "dq")
    tol = 0 * k.double()
    each = (2 * 72 + 4) * E32 * scale * most * q.double().abs()
    tol.index_add_(0, src, each.sum(1, keepdim=True).view(3, 1, 2, 2, 64).sum(3))
    _near(dk, 0 * k.double(), 1.01 * tol + 2.0 ** -130, "dk")
