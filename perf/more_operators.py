"""Measured cases of the 8-bit operators and of the tokens' log probabilities.

A model whose matrices are used in 8-bit integers scores tokens and learns from
the scores.  Six kinds of pass:

* ``norm``        the residual's addition and the root-mean-square norm, into
                  8-bit rows with a scale each, into the inputs' type, or both;
* ``norm_grad``   the gradients of its input and of its weight;
* ``linear``      activations times 8-bit weights (the weights' codes are kept,
                  as a server keeps them);
* ``train``       a layer's forward and backward: activations, weights and output
                  gradients quantised along both axes, three products;
* ``score``       log probabilities of given tokens, the rows' entropies and the
                  most likely alternatives;
* ``score_grad``  the gradient of the logits from those of the log probabilities
                  and entropies.

The sizes are those of the GPT-2-1.5B shard (hidden 1600, FFN 6400, vocabulary
50257), the BERT-Large one (1024, 4096, 30522), and odd ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
DEV = "cuda"
EPS = 1e-5


def listed():
    return [
        # one token's hidden state on its way into an 8-bit layer (decode)
        dict(name="norm-token", kind="norm", rows=1, cols=1600, dtype="bf16", weight="f32",
             residual=True, form="q", pad=0),
        # 8 sequences of 1024 between two layers, for a product in 8 bits and for the backward pass
        dict(name="norm-batch", kind="norm", rows=8192, cols=1600, dtype="bf16", weight="f32",
             residual=True, form="both", pad=0),
        # long odd rows out of a wider buffer
        dict(name="norm-odd", kind="norm", rows=2047, cols=6401, dtype="f16", weight="f16",
             residual=False, form="both", pad=7),
        # the backward pass of 8 sequences of 1024, with the residual stream's own gradient
        dict(name="norm-grad-batch", kind="norm_grad", rows=8192, cols=1600, dtype="bf16",
             weight="f32", residual=True, pad=0),
        # the same of a binary32 model of odd width, few rows, no residual
        dict(name="norm-grad-odd", kind="norm_grad", rows=301, cols=4095, dtype="f32",
             weight="f32", residual=False, pad=1),
        # one token through the FFN's first matrix
        dict(name="linear-token", kind="linear", m=1, n=6400, k=1600, dtype="bf16", out="bf16"),
        # a batch of 8 sequences of 1024 through the FFN's first matrix
        dict(name="linear-ffn", kind="linear", m=8192, n=6400, k=1600, dtype="bf16", out="bf16"),
        # a training step of BERT-Large's FFN matrix over an odd number of tokens
        dict(name="train-bert-ffn", kind="train", t=2047, n=4096, k=1024),
        # the same of GPT-2's, over 8 sequences of 1024
        dict(name="train-gpt2-ffn", kind="train", t=8192, n=6400, k=1600),
        # a decode step of three sequences: the sampled tokens' scores and five alternatives
        dict(name="score-few", kind="score", rows=3, vocab=50257, top=5, dtype="f32", masked=0,
             pad=0, tau=1.0),
        # scores of four sequences of 1024, the vocabulary padded to a multiple of 64 and masked
        dict(name="score-batch", kind="score", rows=4096, vocab=50304, top=20, dtype="bf16",
             masked=47, pad=0, tau=1.0),
        # the policy's gradient over four sequences of 1024
        dict(name="score-grad-batch", kind="score_grad", rows=4096, vocab=50257, dtype="bf16",
             masked=0, pad=47, tau=1.0),
    ]


MOST_MNK = 8192 * 6400 * 1600
MOST_LOGITS = 4096 * 50257
MOST_HIDDEN = 8192 * 1600


def _spread(rng, lo, hi):
    """A size between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "linear", "linear", "train", "score", "score",
                       "score_grad"])
    if kind in ("norm", "norm_grad"):
        rows = _spread(rng, 1, 16384)
        dtype = rng.choice(sorted(DTYPES))
        got = dict(kind=kind, rows=rows, cols=_spread(rng, 1, min(16384, MOST_HIDDEN // rows)),
                   dtype=dtype, weight=rng.choice(["f32", dtype]), residual=rng.random() < 0.5,
                   pad=rng.choice([0, 0, 3, 16]))
        if kind == "norm":
            got["form"] = rng.choice(["q", "out", "both"])
        return got
    if kind == "linear":
        m = _spread(rng, 1, 64) if rng.random() < 0.5 else _spread(rng, 65, 8192)
        k = _spread(rng, 32, 6400)
        n = _spread(rng, 16, max(16, min(50257, MOST_MNK // (m * k), MOST_LOGITS // m)))
        return dict(kind=kind, m=m, n=n, k=k, dtype=rng.choice(["bf16", "f16", "f32"]),
                    out=rng.choice(["bf16", "f16", "f32"]))
    if kind == "train":
        return dict(kind=kind, t=_spread(rng, 1, 8192), n=_spread(rng, 32, 6400),
                    k=_spread(rng, 32, 1600))
    rows = _spread(rng, 1, 4096)
    vocab = _spread(rng, 1000, min(131072, MOST_LOGITS // rows))
    got = dict(kind=kind, rows=rows, vocab=vocab, dtype=rng.choice(sorted(DTYPES)),
               masked=rng.choice([0, 0, 47, 300]), pad=rng.choice([0, 0, 5, 64]),
               tau=rng.choice([0.7, 1.0, 1.5]))
    if kind == "score":
        got["top"] = rng.choice([0, _spread(rng, 1, 256), _spread(rng, 1, 256)])
    return got


def work(case):
    c, kind = case, case["kind"]
    if kind == "norm":
        n, e, form = c["rows"] * c["cols"], SIZE[c["dtype"]], c["form"]
        # x and the residual read, their sum written; the output; codes written and read back
        each = e + (2 * e if c["residual"] else 0) + (0 if form == "q" else e)
        each += 0 if form == "out" else 1 + 1 + 2
        return {"bytes": n * each + c["cols"] * SIZE[c["weight"]] + 12 * c["rows"], "flops": 0}
    if kind == "norm_grad":
        n, e = c["rows"] * c["cols"], SIZE[c["dtype"]]
        return {"bytes": n * e * (4 if c["residual"] else 3) + 4 * c["rows"] +
                c["cols"] * (SIZE[c["weight"]] + 4), "flops": 0}
    if kind == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": m * k * SIZE[c["dtype"]] + n * k + 4 * n + m * n * SIZE[c["out"]],
                "flops": 2.0 * m * n * k}
    if kind == "train":
        t, n, k = c["t"], c["n"], c["k"]
        return {"bytes": 2 * t * k + 4 * n * k + 2 * t * n + 2 * t * n + 2 * t * k + 4 * n * k,
                "flops": 6.0 * t * n * k}
    z = c["rows"] * c["vocab"] * SIZE[c["dtype"]]
    if kind == "score":
        return {"bytes": z + c["rows"] * (8 * c["top"] + 20), "flops": 0}
    return {"bytes": 2 * z + c["rows"] * 24, "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _matrix(g, rows, cols, dtype, pad=0, sigma=1.0):
    """Normal values, a few columns of them twenty times the size (as hidden
    states have) and 1% outliers, as the first `cols` columns of a wider buffer."""
    x = torch.randn((rows, cols + pad), generator=g, device=DEV) * sigma
    x = x * torch.where(torch.rand(cols + pad, generator=g, device=DEV) < 0.002, 20.0, 1.0)
    x = torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.01, 4 * x, x)
    return x.to(DTYPES[dtype])[:, :cols]


def _empty(rows, cols, dtype, pad=0):
    return torch.empty((rows, cols + pad), dtype=DTYPES[dtype], device=DEV)[:, :cols]


def _wide(cols):
    """Bytes of a row of codes."""
    return -(-cols // 128) * 128


def _buffers(rows, cols):
    """Room for the codes and scales of a rows x cols matrix."""
    return (torch.empty(rows * _wide(cols), dtype=torch.int8, device=DEV),
            torch.empty(rows, device=DEV))


def _held(g, rows, cols):
    """Weights as they are held: codes (zero beyond cols) and the rows' scales."""
    codes = torch.randn((rows, _wide(cols)), generator=g, device=DEV).mul(40).round()
    codes = codes.clamp(-127, 127).to(torch.int8)
    codes[:, cols:] = 0
    scales = 0.0005 * (0.5 + torch.rand(rows, generator=g, device=DEV))
    return codes.view(-1), scales


def _logits(g, c):
    """Logits of a language model: a wide bulk and a few likely columns; the last
    `masked` of them are no tokens."""
    rows, vocab = c["rows"], c["vocab"]
    z = torch.randn((rows, vocab + c["pad"]), generator=g, device=DEV) * 2.0
    z += 6.0 * (torch.rand(z.shape, generator=g, device=DEV) < 0.002)
    z = z.to(DTYPES[c["dtype"]])[:, :vocab]
    z[:, vocab - c["masked"]:] = -math.inf
    return z


def _tokens(g, z, masked):
    """Half of them the likeliest, the others anything; some positions have none."""
    rows, vocab = z.shape
    tokens = torch.randint(0, vocab - masked, (rows,), generator=g, device=DEV)
    tokens = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.5, z.argmax(1), tokens)
    tokens[torch.rand(rows, generator=g, device=DEV) < 0.05] = -1
    return tokens.int()


def prepare(case, seed):
    c, kind = case, case["kind"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=c, kind=kind)
    if kind in ("norm", "norm_grad"):
        r, n, dtype, pad = c["rows"], c["cols"], c["dtype"], c["pad"]
        s["weight"] = (1.0 + 0.2 * torch.randn(n, generator=g, device=DEV)).to(DTYPES[c["weight"]])
        if kind == "norm":
            s["x"] = _matrix(g, r, n, dtype, pad)
            s["residual"] = _matrix(g, r, n, dtype, pad, sigma=3.0) if c["residual"] else None
            s["h"] = _empty(r, n, dtype, pad) if c["residual"] else None
            s["rstd"] = torch.empty(r, device=DEV)
            if c["form"] != "q":
                s["out"] = _empty(r, n, dtype, pad)
            if c["form"] != "out":
                s["q"] = _buffers(r, n)
                s["values"] = torch.empty((r, n), dtype=torch.bfloat16, device=DEV)
        else:
            s["h"] = _matrix(g, r, n, dtype, pad, sigma=3.0)
            s["rstd"] = (s["h"].double().square().mean(1) + EPS).rsqrt().float()
            s["dy"] = _matrix(g, r, n, dtype, pad, sigma=1e-3)
            s["dh"] = _matrix(g, r, n, dtype, pad, sigma=1e-3) if c["residual"] else None
            s["dx"] = _empty(r, n, dtype, pad)
            s["dw"] = torch.empty(n, device=DEV)
            s["work"] = torch.empty((64 + r // 16, n), device=DEV)
    elif kind == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        s["x"] = _matrix(g, m, k, c["dtype"])
        s["w"] = _held(g, n, k)
        s["xq"] = _buffers(m, k)
        s["y"] = torch.empty((m, n), dtype=DTYPES[c["out"]], device=DEV)
    elif kind == "train":
        t, n, k = c["t"], c["n"], c["k"]
        s["x"] = _matrix(g, t, k, "bf16")
        s["w"] = _matrix(g, n, k, "f32", sigma=0.02)
        s["dy"] = _matrix(g, t, n, "bf16", sigma=1e-3)
        for name, (a, b) in {"xq": (t, k), "xt": (k, t), "wq": (n, k), "wt": (k, n),
                             "gq": (t, n), "gt": (n, t)}.items():
            s[name] = _buffers(a, b)
        # the column maxima of the blocks of rows: at most one for 16 rows
        s["work"] = torch.empty(max(r * n for r, n in ((t // 16 + 1, max(n, k)), (n // 16 + 1, k))),
                                device=DEV)
        s["y"] = torch.empty((t, n), dtype=torch.bfloat16, device=DEV)
        s["dx"] = torch.empty((t, k), dtype=torch.bfloat16, device=DEV)
        s["dw"] = torch.empty((n, k), device=DEV)
    else:
        r = c["rows"]
        s["z"] = z = _logits(g, c)
        s["tokens"] = _tokens(g, z, c["masked"])
        if kind == "score":
            s["logp"] = torch.empty(r, device=DEV)
            s["stats"] = torch.empty((r, 3), device=DEV)
            if c["top"]:
                s["values"] = torch.empty((r, c["top"]), device=DEV)
                s["columns"] = torch.empty((r, c["top"]), dtype=torch.int32, device=DEV)
        else:
            s["stats"] = torch.cat([_stats64(z[i:i + 512], c["tau"])
                                    for i in range(0, r, 512)]).float()
            # advantages and a small bonus for entropy; the padding positions count for nothing
            counts = (s["tokens"] >= 0).float()
            s["dlogp"] = torch.randn(r, generator=g, device=DEV) * counts
            s["dentropy"] = -0.01 * counts
            s["dz"] = torch.empty((r, c["vocab"] + c["pad"]), dtype=z.dtype,
                                  device=DEV)[:, :c["vocab"]]
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2202_06009_amd as zo
    c, kind = s["case"], s["kind"]
    if kind == "norm":
        q = zo.I8(c["rows"], c["cols"], *s["q"]) if "q" in s else None
        zo.zo_rms_norm(s["x"], s["weight"], residual=s["residual"], h=s["h"], out=s.get("out"),
                       q=q, rstd=s["rstd"], eps=EPS)
        got = {"rstd": s["rstd"]}
        if s["h"] is not None:
            got["h"] = s["h"]
        if "out" in s:
            got["out"] = s["out"]
        if q is not None:
            zo.zo_i8_dequantize(q, s["values"])
            got["values"] = s["values"]
        return got
    if kind == "norm_grad":
        zo.zo_rms_norm_grad(s["dy"], s["h"], s["weight"], s["rstd"], s["dx"], s["dw"],
                            dh=s["dh"], work=s["work"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if kind == "linear":
        zo.zo_i8_linear(s["x"], zo.I8(c["n"], c["k"], *s["w"]), s["y"],
                        zo.I8(c["m"], c["k"], *s["xq"]))
        return {"y": s["y"]}
    if kind == "train":
        t, n, k = c["t"], c["n"], c["k"]
        xq, xt = zo.I8(t, k, *s["xq"]), zo.I8(k, t, *s["xt"])
        wq, wt = zo.I8(n, k, *s["wq"]), zo.I8(k, n, *s["wt"])
        gq, gt = zo.I8(t, n, *s["gq"]), zo.I8(n, t, *s["gt"])
        zo.zo_i8_quantize(s["x"], xq, xt, s["work"])
        zo.zo_i8_quantize(s["w"], wq, wt, s["work"])
        zo.zo_i8_product(xq, wq, s["y"])
        zo.zo_i8_quantize(s["dy"], gq, gt, s["work"])
        zo.zo_i8_product(gq, wt, s["dx"])
        zo.zo_i8_product(gt, xt, s["dw"])
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}
    if kind == "score":
        zo.zo_token_logprobs(s["z"], s["tokens"], s["logp"], s["stats"], s.get("values"),
                             s.get("columns"), tau=c["tau"])
        got = {"logp": s["logp"], "stats": s["stats"]}
        if c["top"]:
            got.update(values=s["values"], columns=s["columns"])
        return got
    zo.zo_token_logprobs_grad(s["z"], s["stats"], s["dz"], tokens=s["tokens"], dlogp=s["dlogp"],
                              dentropy=s["dentropy"], tau=c["tau"])
    return {"dz": s["dz"]}


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _rounded(x):
    """The codes of x (32 bits) along the last axis, as 32-bit numbers, and the rows'
    scales.  The quotients in 64 bits: next to a border 32 would take the other code."""
    most = x.abs().amax(-1, keepdim=True)
    scale = (most.double() / 127).float()
    codes = torch.where(scale > 0, x.double() / scale.double(), 0.0).round().clamp(-127, 127)
    return codes.float(), scale


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float()
    if c["residual"]:
        x = x + s["residual"].float()
    h = x.to(DTYPES[c["dtype"]])
    x, w = h.float(), s["weight"].float()
    rstd = 1.0 / (x.square().mean(1) + EPS).sqrt()
    got = {"rstd": rstd}
    if c["residual"]:
        got["h"] = h
    if "out" in s:
        got["out"] = (x * rstd[:, None] * w).to(h.dtype)
    if "q" in s:
        codes, scale = _rounded(x * w)
        got["values"] = (codes * (scale * rstd[:, None])).bfloat16()
    return got


def _plain_norm_grad(s):
    h, dy, rstd = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
    g, n = dy * s["weight"].float(), h * rstd
    dx = rstd * (g - n * (g * n).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["h"].dtype), "dw": (dy * n).sum(0)}


def _held_codes(held, cols):
    return held[0].view(held[1].shape[0], -1)[:, :cols].float(), held[1]


def _plain_score(s):
    c = s["case"]
    z, tau = s["z"].float(), c["tau"]
    vocab = c["vocab"]
    most = z.amax(1, keepdim=True)
    d = (z - most) / tau
    e = d.exp()
    total = e.sum(1)
    log_total = total.log()
    entropy = log_total - torch.where(e > 0, e * d, 0.0).sum(1) / total
    has = s["tokens"] >= 0
    logp = d.gather(1, s["tokens"].clamp(min=0).long()[:, None])[:, 0] - log_total
    got = {"logp": torch.where(has, logp, 0.0),
           "stats": torch.stack([most[:, 0], log_total, entropy], 1)}
    if c["top"]:
        bits = (z + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        # one whole number for value and column, so that of equal values the lowest column is first
        key = (order << 32) + (0xFFFFFFFF - torch.arange(vocab, device=DEV))
        at = 0xFFFFFFFF - (torch.topk(key, c["top"], dim=1).values & 0xFFFFFFFF)
        got.update(values=d.gather(1, at) - log_total[:, None], columns=at.int())
    return got


def _plain_score_grad(s):
    tau = s["case"]["tau"]
    most, log_total, entropy = s["stats"].unbind(1)
    logp = (s["z"].float() - most[:, None]) / tau - log_total[:, None]
    p = logp.exp()
    dz = -s["dlogp"][:, None] * p
    dz -= s["dentropy"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), 0.0)
    at = s["tokens"].clamp(min=0).long()[:, None]
    dz.scatter_add_(1, at, torch.where(s["tokens"] >= 0, s["dlogp"], 0.0)[:, None])
    return {"dz": (dz / tau).to(s["z"].dtype)}


def run(state):
    if own:
        return _run_own(state)
    s = state
    c, kind = s["case"], s["kind"]
    if kind == "norm":
        return _plain_norm(s)
    if kind == "norm_grad":
        return _plain_norm_grad(s)
    if kind == "linear":
        x, sx = _rounded(s["x"].float())
        w, sw = _held_codes(s["w"], c["k"])
        return {"y": ((x @ w.t()) * sx * sw).to(DTYPES[c["out"]])}
    if kind == "train":
        x, w, dy = s["x"].float(), s["w"], s["dy"].float()
        (xq, sx), (wq, sw), (gq, sg) = _rounded(x), _rounded(w), _rounded(dy)
        xt, sxt = _rounded(x.t().contiguous())
        wt, swt = _rounded(w.t().contiguous())
        gt, sgt = _rounded(dy.t().contiguous())
        return {"y": ((xq @ wq.t()) * sx * sw.t()).bfloat16(),
                "dx": ((gq @ wt.t()) * sg * swt.t()).bfloat16(),
                "dw": (gt @ xt.t()) * sgt * sxt.t()}
    if kind == "score":
        return _plain_score(s)
    return _plain_score_grad(s)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _grid64(x):
    """x (64 bits) as its 8-bit form along the last axis holds it: whole multiples,
    half to even, of the largest magnitude's 127th part, which is kept in 32 bits."""
    step = (x.abs().amax(-1, keepdim=True) / 127).float().double()
    return torch.nan_to_num(x / step, nan=0.0).round() * step


def _stats64(z, tau):
    z = z.double()
    most = z.max(1).values
    logp = torch.log_softmax(z / tau, 1)
    entropy = -torch.special.xlogy(logp.exp(), logp.exp()).sum(1)
    return torch.stack([most, torch.logsumexp(z / tau, 1) - most / tau, entropy], 1)


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind == "norm":
        h = s["x"].double()
        got = {}
        if c["residual"]:
            # the sum is kept in the inputs' type; of two 16-bit numbers it is exact in 64 bits
            h = (h + s["residual"].double()).to(s["x"].dtype)
            got["h"], h = h, h.double()
        w = s["weight"].double()
        rms = torch.sqrt((h * h).sum(1, keepdim=True) / c["cols"] + EPS)
        got["rstd"] = 1.0 / rms[:, 0]
        if "out" in s:
            got["out"] = h / rms * w
        if "q" in s:
            got["values"] = _grid64((h * w).float().double()) / rms
        return got
    if kind == "norm_grad":
        h, dy, w = s["h"].double(), s["dy"].double(), s["weight"].double()
        rstd = s["rstd"].double()[:, None]
        dot = (dy * w * h).sum(1, keepdim=True)
        dx = rstd * dy * w - rstd ** 3 * h * dot / c["cols"]
        if s["dh"] is not None:
            dx = dx + s["dh"].double()
        return {"dx": dx, "dw": torch.einsum("rc,rc->c", dy * rstd, h)}
    if kind == "linear":
        w = s["w"][0].view(c["n"], -1)[:, :c["k"]].double() * s["w"][1].double()[:, None]
        return {"y": _grid64(s["x"].double()) @ w.t()}
    if kind == "train":
        x, w, dy = s["x"].double(), s["w"].double(), s["dy"].double()
        return {"y": _grid64(x) @ _grid64(w).t(),
                "dx": _grid64(dy) @ _grid64(w.t()).t(),
                "dw": _grid64(dy.t()) @ _grid64(x.t()).t()}
    if kind == "score":
        return _score64(s)
    return _score_grad64(s)


def _score64(s):
    """Block by block of rows."""
    c, parts = s["case"], []
    for r0 in range(0, c["rows"], 512):
        z, tokens = s["z"][r0:r0 + 512].double(), s["tokens"][r0:r0 + 512].long()
        logp = torch.log_softmax(z / c["tau"], 1)
        picked = torch.zeros(len(z), dtype=torch.float64, device=DEV)
        has = (tokens >= 0).nonzero()[:, 0]
        picked[has] = logp[has, tokens[has]]
        part = {"logp": picked, "stats": _stats64(z, c["tau"])}
        if c["top"]:
            at = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :c["top"]]
            part.update(values=logp.gather(1, at), columns=at.int())
        parts.append(part)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _score_grad64(s):
    """From the logits alone: the given statistics are theirs, rounded."""
    c, tau = s["case"], s["case"]["tau"]
    dz = torch.zeros(s["z"].shape, dtype=torch.float64, device=DEV)
    for r0 in range(0, c["rows"], 512):
        z, tokens = s["z"][r0:r0 + 512].double(), s["tokens"][r0:r0 + 512].long()
        a = s["dlogp"][r0:r0 + 512].double()[:, None]
        b = s["dentropy"][r0:r0 + 512].double()[:, None]
        p = torch.softmax(z / tau, 1)
        plogp = torch.special.xlogy(p, p)
        part = -a * p - b * (plogp - p * plogp.sum(1, keepdim=True))
        has = (tokens >= 0).nonzero()[:, 0]
        part[has, tokens[has]] += a[has, 0]
        dz[r0:r0 + 512] = part / tau
    return {"dz": dz}
