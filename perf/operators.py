"""Layer norm and cross attention, forward and backward, as cases that can be timed and compared.

They are the conditioning part of a text-conditioned denoiser on the batch that the solver hands over: ``items`` rows of
the batch, each a latent of ``tokens`` tokens; a row's trajectory (first column of the miss list) says whose encoder
states it attends to, so many rows share one set of keys and values. A ``grad`` case is the forward pass with the
statistics that the backward pass needs, then the backward pass.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


# ---- the cases ---------------------------------------------------------------

def _norm(rows, cols, dtype, grad, name=None):
    c = {"kind": "norm", "rows": rows, "cols": cols, "dtype": dtype, "grad": grad}
    return dict(c, name=name) if name else c


def _attn(items, sources, tokens, keys, heads, kv_heads, dim, dtype, grad, keep="all", name=None):
    """keep: which keys count. "all"; "lengths": a length per source, the first source's may be zero; "mask": single
    keys dropped as well."""
    c = {"kind": "attn", "items": items, "sources": sources, "tokens": tokens, "keys": keys, "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "grad": grad, "keep": keep}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one conditioning vector per row of an eight-row window: launches and latency are all there is
        _norm(8, 320, "bf16", False, "norm 8 rows"),
        # the whole window of 100 timesteps of a 64x64 latent, width 320
        _norm(409600, 320, "bf16", False, "norm window"),
        # 32 rows of 64x64 tokens, width 640, with gradients (guidance through the denoiser)
        _norm(131072, 640, "fp16", True, "norm grad"),
        # an odd width in 32 bits: rows off the 16-byte boundaries
        _norm(5003, 1111, "fp32", True, "norm grad odd fp32"),
        # a whole window of one trajectory: 100 rows share one prompt of 77 tokens
        _attn(100, 1, 4096, 77, 8, 8, 40, "bf16", False, "all", "attn window"),
        # eight trajectories of 32x32 tokens with prompts of different lengths, one of them empty, with gradients
        _attn(64, 8, 1024, 77, 8, 8, 80, "bf16", True, "lengths", "attn batched grad"),
        # gradients of 32 rows of a 64x64 latent that share two prompts
        _attn(32, 2, 4096, 77, 8, 8, 40, "fp16", True, "all", "attn window grad"),
        # single tokens, each with encoder states of its own (a pooled query per request): reads of K and V
        _attn(64, 64, 1, 4096, 16, 4, 64, "bf16", False, "lengths", "attn one token"),
        # long encoder states (another latent as the context): two products on the tensor cores
        _attn(2, 2, 4096, 2048, 16, 16, 128, "fp16", False, "all", "attn long"),
        # the same with shared heads, dropped keys and gradients
        _attn(2, 1, 2048, 2000, 16, 4, 128, "bf16", True, "mask", "attn long grad"),
        # everything small and odd
        _attn(5, 3, 33, 19, 4, 2, 24, "bf16", True, "mask", "attn small grad"),
        # 128x128 latents against three prompt chunks
        _attn(4, 2, 16384, 231, 5, 5, 64, "fp16", False, "lengths", "attn 128x128"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("norm", "attn")}
    while True:
        grad = rng.random() < 0.5
        if rng.random() < 0.35:
            cols = _log(rng, 16, 8192)
            if rng.random() < 0.7:
                cols = max(8, cols // 8 * 8)
            case = _norm(_log(rng, 1, 400000), cols, rng.choice(["bf16", "fp16", "fp32"]), grad)
        else:
            shared = rng.choice([1, 1, 2, 4, 8])
            kv_heads = rng.choice([1, 2, 4, 5, 8, 16]) if shared == 1 else rng.choice([1, 2, 4])
            items = _log(rng, 1, 100)
            case = _attn(items, min(items, _log(rng, 1, 16)), _log(rng, 1, 4096), _log(rng, 1, 4096), shared * kv_heads,
                         kv_heads, 8 * _log(rng, 1, 20), rng.choice(["bf16", "fp16"]), grad,
                         rng.choice(["all", "lengths", "mask"]))
        if _cost(case) <= most[case["kind"]]:
            return case


def _cost(case):
    """What a drawn case may not have more of than the largest listed one: values of the norm, or attention scores."""
    if case["kind"] == "norm":
        return case["rows"] * case["cols"] * (1 + case["grad"])
    scores = case["items"] * case["heads"] * case["tokens"] * case["keys"]
    rows = case["items"] * case["tokens"] * case["heads"] * case["dim"] * 2
    states = case["sources"] * case["keys"] * case["kv_heads"] * case["dim"] * 2
    return (scores + rows + states) * (1 + case["grad"])


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "norm":
        n, c = case["rows"] * case["cols"], case["cols"]
        if case["grad"]:  # x, dy; y, dx; weight, bias and their gradients
            return {"bytes": 4 * n * e + 4 * c * e, "flops": 20 * n}
        return {"bytes": 2 * n * e + 2 * c * e, "flops": 8 * n}
    part = {"all": 1.0, "lengths": 0.65, "mask": 0.65 * 0.8}[case["keep"]]  # of the keys, on average
    rows = case["items"] * case["tokens"] * case["heads"]
    states = case["sources"] * case["keys"] * case["kv_heads"] * case["dim"]
    if case["grad"]:  # q, dout; out, dq; k, v; dk, dv
        return {"bytes": (4 * rows * case["dim"] + 2 * states * part + 2 * states) * e,
                "flops": 14 * rows * case["keys"] * part * case["dim"]}
    return {"bytes": (2 * rows * case["dim"] + 2 * states * part) * e,
            "flops": 4 * rows * case["keys"] * part * case["dim"]}


# ---- inputs ------------------------------------------------------------------

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    if case["kind"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # activations: rows of different scale, some channels with an offset
        x = normal(rows, cols) * (0.5 + normal(rows, 1).abs()) + 0.7 * normal(1, cols)
        s = {"case": case, "x": x.to(dt), "weight": (1 + 0.2 * normal(cols)).to(dt), "bias": (0.2 * normal(cols)).to(dt)}
        if case["grad"]:
            s["dy"] = (0.1 * normal(rows, cols)).to(dt)
        return s
    rng = random.Random(seed)
    N, G, Q, K, H, J, D = (case[k] for k in ("items", "sources", "tokens", "keys", "heads", "kv_heads", "dim"))
    # the first token of a prompt draws much of the attention
    first = normal(1, 1, J, 1, D)
    q = (normal(N, Q, J, H // J, D) + 0.5 * first).view(N, Q, H, D).to(dt)
    kv = normal(G, K, 2, J, D)
    kv[:, :1, :1] += 1.5 * first.view(1, 1, 1, J, D)
    kv = kv.to(dt)
    # the miss list: trajectory-major pairs (trajectory, timestep); every trajectory has a row where there are enough
    own_rows = sorted(list(range(min(N, G))) + [rng.randrange(G) for _ in range(max(0, N - G))])
    miss = torch.tensor([[b, n] for n, b in enumerate(own_rows)], dtype=torch.int32, device=dev)
    s = {"case": case, "q": q, "k": kv[:, :, 0], "v": kv[:, :, 1], "miss": miss, "lengths": None, "mask": None,
         "scale": 1.0 / math.sqrt(D)}
    if case["keep"] != "all":
        lengths = [max(1, int(K * rng.uniform(0.3, 1.0))) for _ in range(G)]
        if G > 2:
            lengths[rng.randrange(G)] = 0  # an empty prompt
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
        if case["keep"] == "mask":
            s["mask"] = torch.rand(G, K, generator=g, device=dev) < 0.8
        # past a prompt's end lies what the buffer held before
        past = torch.arange(K, device=dev)[None, :] >= s["lengths"][:, None]
        kv.masked_fill_(past[:, :, None, None, None], float("inf"))
    if case["grad"]:
        s["dout"] = (0.1 * normal(N, Q, H, D)).to(dt)
    return s


# ---- one pass ----------------------------------------------------------------

def run(s):
    if s["case"]["kind"] == "norm":
        return (_own_norm if own else _plain_norm)(s)
    return (_own_attn if own else _plain_attn)(s)


def _own_norm(s):
    from paper_2609_36522_gb300 import layers
    if not s["case"]["grad"]:
        return {"y": layers.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)}
    y, mean, rstd = layers.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, stats=True)
    dx, dw, db = layers.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["weight"])
    return {"y": y, "dx": dx, "dweight": dw, "dbias": db}


def _own_attn(s):
    from paper_2609_36522_gb300 import layers
    kw = {"scale": s["scale"], "source": s["miss"][:, 0], "lengths": s["lengths"], "mask": s["mask"]}
    if not s["case"]["grad"]:
        return {"out": layers.cross_attention(s["q"], s["k"], s["v"], **kw)}
    out, lse = layers.cross_attention(s["q"], s["k"], s["v"], stats=True, **kw)
    dq, dk, dv = layers.cross_attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, **kw)
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}


def _plain_norm(s):
    x, w, b, dt = s["x"].float(), s["weight"].float(), s["bias"].float(), s["x"].dtype
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = (xc.square().mean(1, keepdim=True) + EPS).rsqrt()
    xh = xc * rstd
    y = (xh * w + b).to(dt)
    if not s["case"]["grad"]:
        return {"y": y}
    dy = s["dy"].float()
    gr = dy * w
    dx = rstd * (gr - gr.mean(1, keepdim=True) - xh * (gr * xh).mean(1, keepdim=True))
    return {"y": y, "dx": dx.to(dt), "dweight": (dy * xh).sum(0).to(dt), "dbias": dy.sum(0).to(dt)}


def _kept(s):
    """[sources][keys]: the keys that count."""
    G, K = s["case"]["sources"], s["case"]["keys"]
    kept = torch.ones(G, K, dtype=torch.bool, device=s["q"].device)
    if s["lengths"] is not None:
        kept &= torch.arange(K, device=kept.device)[None, :] < s["lengths"][:, None]
    if s["mask"] is not None:
        kept &= s["mask"]
    return kept


def _plain_attn(s):
    c, dt, scale = s["case"], s["q"].dtype, s["scale"]
    N, G, Q, K, H, J, D = (c[k] for k in ("items", "sources", "tokens", "keys", "heads", "kv_heads", "dim"))
    R = H // J
    kept = _kept(s)
    src = s["miss"][:, 0].long()
    zero = torch.zeros((), device=kept.device)
    k = torch.where(kept[:, :, None, None], s["k"].float(), zero)[src].permute(0, 2, 1, 3)      # [N][J][K][D]
    v = torch.where(kept[:, :, None, None], s["v"].float(), zero)[src].permute(0, 2, 1, 3)
    there = kept[src][:, None, None, :]                                                       # [N][1][1][K]

    def rows(x):  # [N][J][R * Q][D]: the heads that share keys, one after another
        return x.float().view(N, Q, J, R, D).permute(0, 2, 3, 1, 4).reshape(N, J, R * Q, D)

    def back(x):
        return x.view(N, J, R, Q, D).permute(0, 3, 1, 2, 4).reshape(N, Q, H, D).to(dt)

    q = rows(s["q"])
    p = torch.where(there, torch.matmul(q, k.transpose(2, 3)) * scale, torch.full_like(zero, -math.inf))
    top = p.amax(3, keepdim=True)
    p = torch.exp(p - torch.where(torch.isinf(top), zero, top))
    p = p / p.sum(3, keepdim=True).clamp_min(1e-30)
    o = torch.matmul(p, v)
    if not c["grad"]:
        return {"out": back(o)}
    do = rows(s["dout"])
    ds = p * (torch.matmul(do, v.transpose(2, 3)) - (do * o).sum(3, keepdim=True))
    of = (torch.arange(G, device=src.device)[:, None] == src[None, :]).float()                # [G][N]

    def states(x):  # the sum over the rows of each source
        return torch.matmul(of, x.reshape(N, J * K * D)).view(G, J, K, D).permute(0, 2, 1, 3).to(dt)

    return {"out": back(o), "dq": back(torch.matmul(ds, k) * scale), "dk": states(torch.matmul(ds.transpose(2, 3), q) * scale),
            "dv": states(torch.matmul(p.transpose(2, 3), do))}


# ---- the definition in 64 bits -----------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
        n = x.shape[1]
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        sd = torch.sqrt(var + EPS)
        xh = (x - mean) / sd
        y = torch.addcmul(b, xh, w)
        if not case["grad"]:
            return {"y": y}
        dy = s["dy"].double()
        a1 = (dy @ w) / n                                   # mean of dy w
        a2 = ((dy * xh) @ w) / n                            # mean of dy w xhat
        dx = (dy * w - a1[:, None] - xh * a2[:, None]) / sd
        return {"y": y, "dx": dx, "dweight": torch.einsum("rc,rc->c", dy, xh), "dbias": torch.einsum("rc->c", dy)}
    kept, J = _kept(s), case["kv_heads"]
    N, Q, H, D = s["q"].shape
    R = H // J
    out = torch.zeros(N, Q, H, D, dtype=torch.float64, device=s["q"].device)
    dq = torch.zeros_like(out) if case["grad"] else None
    dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device=s["q"].device) for _ in range(2))
    sources = s["miss"][:, 0].tolist()
    for g in sorted(set(sources)):
        at = kept[g].nonzero()[:, 0]
        if at.numel() == 0:
            continue
        items = torch.tensor([n for n, b in enumerate(sources) if b == g], device=at.device)
        for j in range(J):
            kj, vj = s["k"][g, at, j].double(), s["v"][g, at, j].double()
            dkj, dvj = torch.zeros_like(kj), torch.zeros_like(vj)
            for some in items.split(max(1, (1 << 27) // (Q * R * at.numel()))):
                qj = s["q"][some][:, :, j * R:(j + 1) * R].double()
                p = torch.softmax(torch.einsum("nqrd,kd->nqrk", qj, kj) * s["scale"], dim=-1)
                o = torch.einsum("nqrk,kd->nqrd", p, vj)
                out[some, :, j * R:(j + 1) * R] = o
                if case["grad"]:
                    do = s["dout"][some][:, :, j * R:(j + 1) * R].double()
                    dp = torch.einsum("nqrd,kd->nqrk", do, vj)
                    ds = p * (dp - (dp * p).sum(-1, keepdim=True)) * s["scale"]
                    dq[some, :, j * R:(j + 1) * R] = torch.einsum("nqrk,kd->nqrd", ds, kj)
                    dkj += torch.einsum("nqrk,nqrd->kd", ds, qj)
                    dvj += torch.einsum("nqrk,nqrd->kd", p, do)
            dk[g, at, j] += dkj
            dv[g, at, j] += dvj
    if not case["grad"]:
        return {"out": out}
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}
