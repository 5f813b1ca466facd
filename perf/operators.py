"""The 4-bit and distillation operators' measured cases.

A student whose weights are used in microscaled 4-bit floating point learns
from a teacher's top logits.  Five kinds of pass:

* ``quantize``  a matrix to 4 bits with a scale for each 32 values along its
                rows, its columns or both, and the values read back;
* ``linear``    activations times 4-bit weights (the weights' codes are kept,
                as a server keeps them);
* ``train``     a layer's forward and backward: activations, weights and
                output gradients quantised along both axes, three products;
* ``top``       the k largest logits of each row, their columns and the
                row's log-sum-exp (what a teacher hands over);
* ``distill``   the distillation loss and the gradient of the student's logits.

The sizes are those of the GPT-2-1.5B shard (hidden 1600, FFN 6400, vocabulary
50257), the BERT-Large one (1024, 4096, 30522), and odd ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
DEV = "cuda"


def listed():
    return [
        # one token's hidden state on its way into a 4-bit layer
        dict(name="quantize-token", kind="quantize", rows=1, cols=1600, dtype="bf16", form="rows",
             pad=0),
        # a GPT-2 FFN weight of the f32 shard, for the forward and the backward products
        dict(name="quantize-ffn-weight", kind="quantize", rows=6400, cols=1600, dtype="f32",
             form="both", pad=0),
        # activations of an odd batch with odd rows, out of a wider buffer
        dict(name="quantize-odd", kind="quantize", rows=8191, cols=4097, dtype="f16", form="both",
             pad=7),
        # one token through the FFN's first matrix
        dict(name="linear-token", kind="linear", m=1, n=6400, k=1600, dtype="bf16", out="bf16"),
        # a decode step of a few sequences through the vocabulary head
        dict(name="linear-head-few", kind="linear", m=11, n=50257, k=1600, dtype="bf16",
             out="f32"),
        # a batch of 8 sequences of 1024 through the FFN's first matrix
        dict(name="linear-ffn", kind="linear", m=8192, n=6400, k=1600, dtype="bf16", out="bf16"),
        # a training step of BERT-Large's FFN matrix over an odd number of tokens
        dict(name="train-bert-ffn", kind="train", t=2047, n=4096, k=1024),
        # the same of GPT-2's, over 8 sequences of 1024
        dict(name="train-gpt2-ffn", kind="train", t=8192, n=6400, k=1600),
        # a teacher's answers for three positions
        dict(name="top-few", kind="top", rows=3, vocab=50257, top=8, dtype="f32", pad=0, tau=1.0),
        # a teacher's answers for four sequences of 1024
        dict(name="top-batch", kind="top", rows=4096, vocab=50257, top=64, dtype="bf16", pad=47,
             tau=2.0),
        # the loss of a handful of BERT positions
        dict(name="distill-few", kind="distill", rows=5, vocab=30522, top=16, dtype="f32", pad=0,
             tau=1.0, tail=True, labels=False),
        # the loss of four sequences of 1024, mixed with the labels' cross entropy
        dict(name="distill-batch", kind="distill", rows=4096, vocab=50257, top=64, dtype="bf16",
             pad=47, tau=2.0, tail=True, labels=True),
    ]


MOST_MNK = 8192 * 6400 * 1600
MOST_LOGITS = 4096 * 50257


def _spread(rng, lo, hi):
    """A size between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "train", "top", "distill"])
    if kind == "quantize":
        rows = _spread(rng, 1, 16384)
        return dict(kind=kind, rows=rows, cols=_spread(rng, 1, min(8192, 33554432 // rows)),
                    dtype=rng.choice(sorted(DTYPES)), form=rng.choice(["rows", "cols", "both"]),
                    pad=rng.choice([0, 0, 3, 16]))
    if kind == "linear":
        m = _spread(rng, 1, 32) if rng.random() < 0.5 else _spread(rng, 33, 8192)
        k = _spread(rng, 32, 6400)
        n = _spread(rng, 16, max(16, min(50257, MOST_MNK // (m * k), MOST_LOGITS // m)))
        return dict(kind=kind, m=m, n=n, k=k, dtype=rng.choice(["bf16", "f16", "f32"]),
                    out=rng.choice(["bf16", "f16", "f32"]))
    if kind == "train":
        t, n, k = _spread(rng, 1, 8192), _spread(rng, 32, 6400), _spread(rng, 32, 1600)
        return dict(kind=kind, t=t, n=n, k=k)
    rows = _spread(rng, 1, 4096)
    vocab = _spread(rng, 1000, min(131072, MOST_LOGITS // rows))
    got = dict(kind=kind, rows=rows, vocab=vocab, top=_spread(rng, 1, 256),
               dtype=rng.choice(sorted(DTYPES)), pad=rng.choice([0, 0, 5, 64]),
               tau=rng.choice([1.0, 1.5, 2.0]))
    if kind == "distill":
        got.update(tail=rng.random() < 0.5, labels=rng.random() < 0.5)
    return got


def work(case):
    c, kind = case, case["kind"]
    held = 17.0 / 32.0     # bytes of a value held in 4 bits with its share of the scale
    if kind == "quantize":
        n = c["rows"] * c["cols"]
        forms = 2 if c["form"] == "both" else 1
        # read, codes written, and read back to 16-bit values
        return {"bytes": n * SIZE[c["dtype"]] + forms * n * (2 * held + 2), "flops": 0}
    if kind == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": m * k * SIZE[c["dtype"]] + n * k * held + m * n * SIZE[c["out"]],
                "flops": 2.0 * m * n * k}
    if kind == "train":
        t, n, k = c["t"], c["n"], c["k"]
        return {"bytes": 2 * t * k + 4 * n * k + 2 * t * n + 2 * t * n + 2 * t * k + 4 * n * k,
                "flops": 6.0 * t * n * k}
    z = c["rows"] * c["vocab"] * SIZE[c["dtype"]]
    if kind == "top":
        return {"bytes": z + c["rows"] * (8 * c["top"] + 4), "flops": 0}
    return {"bytes": 2 * z + c["rows"] * (8 * c["top"] + 16), "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _matrix(g, rows, cols, dtype, pad=0, sigma=1.0):
    """Normal values with 1% outliers of ten times the size, as the first
    `cols` columns of a buffer of cols + pad."""
    x = torch.randn((rows, cols + pad), generator=g, device=DEV) * sigma
    x = torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.01, 10 * x, x)
    return x.to(DTYPES[dtype])[:, :cols]


def _padded(rows, cols):
    return -(-rows // 64) * 64, -(-cols // 128) * 128


def _held(g, rows, cols):
    """Weights as they are held: random codes and scale exponents near 2^-6 in
    the order of the framework's matrices (codes by 16 rows of 128 columns,
    scales by 64), zero beyond cols."""
    rp, cp = _padded(rows, cols)
    codes = torch.randint(0, 256, (rp, cp // 2), generator=g, device=DEV, dtype=torch.uint8)
    codes[rows:] = 0
    at = torch.arange(cp // 2, device=DEV) * 2
    codes[:, at >= cols] = 0
    if cols % 2:
        codes[:, cols // 2] &= 15
    scales = torch.randint(118, 124, (rp, cp // 32), generator=g, device=DEV, dtype=torch.uint8)
    scales[rows:] = 0
    scales[:, torch.arange(cp // 32, device=DEV) * 32 >= cols] = 0
    kt = cp // 128
    codes = codes.view(rp // 16, 16, kt, 4, 16).permute(0, 2, 3, 1, 4).reshape(-1)
    scales = scales.view(rp // 64, 4, 16, kt, 4).permute(0, 3, 4, 2, 1).reshape(-1)
    return codes, scales


def _logits(g, rows, vocab, dtype, pad):
    """Logits of a language model: a wide bulk and a few likely columns."""
    z = torch.randn((rows, vocab + pad), generator=g, device=DEV) * 2.0
    z += 6.0 * (torch.rand(z.shape, generator=g, device=DEV) < 0.002)
    return z.to(DTYPES[dtype])[:, :vocab]


def prepare(case, seed):
    c, kind = case, case["kind"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=c, kind=kind)
    if kind == "quantize":
        r, n = c["rows"], c["cols"]
        s["x"] = _matrix(g, r, n, c["dtype"], c["pad"])
        for name, (a, b) in {"rows": (r, n), "cols": (n, r)}.items():
            if c["form"] in (name, "both"):
                s[name] = _buffers(a, b)
                s[name + "_values"] = torch.empty((a, b), dtype=torch.bfloat16, device=DEV)
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
        s["y"] = torch.empty((t, n), dtype=torch.bfloat16, device=DEV)
        s["dx"] = torch.empty((t, k), dtype=torch.bfloat16, device=DEV)
        s["dw"] = torch.empty((n, k), device=DEV)
    elif kind == "top":
        s["z"] = _logits(g, c["rows"], c["vocab"], c["dtype"], c["pad"])
        s["values"] = torch.empty((c["rows"], c["top"]), device=DEV)
        s["columns"] = torch.empty((c["rows"], c["top"]), dtype=torch.int32, device=DEV)
        s["lse"] = torch.empty(c["rows"], device=DEV)
    else:
        r, v, k = c["rows"], c["vocab"], c["top"]
        z = _logits(g, r, v, c["dtype"], c["pad"])
        u = z.float() + 1.5 * torch.randn((r, v), generator=g, device=DEV)   # the teacher's
        s["values"], at = torch.topk(u, k, dim=1)
        s["lse"] = torch.logsumexp(u / c["tau"], 1)
        # some rows keep fewer than k slots, some positions are padding
        keep = torch.randint(1, k + 1, (r, 1), generator=g, device=DEV)
        keep = torch.where(torch.rand((r, 1), generator=g, device=DEV) < 0.75, k, keep)
        s["columns"] = torch.where(torch.arange(k, device=DEV)[None] < keep, at, -1).int()
        s["weight"] = (torch.rand(r, generator=g, device=DEV) < 0.95).float()
        s["weight"][0] = 1.0
        s["labels"] = torch.randint(0, v, (r,), generator=g, device=DEV, dtype=torch.int32)
        s["labels"][torch.rand(r, generator=g, device=DEV) < 0.1] = -1
        s["z"] = z
        s["loss"] = torch.empty(r, device=DEV)
        s["dz"] = torch.empty((r, v + c["pad"]), dtype=z.dtype, device=DEV)[:, :v]
    return s


def _buffers(rows, cols):
    """Room for the codes and scales of a rows x cols matrix."""
    rp, cp = _padded(rows, cols)
    return (torch.empty(rp * cp // 2, dtype=torch.uint8, device=DEV),
            torch.empty(rp * cp // 32, dtype=torch.uint8, device=DEV))


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2202_06009_amd as zo
    c, kind = s["case"], s["kind"]
    if kind == "quantize":
        r, n = c["rows"], c["cols"]
        q = zo.Mx4(r, n, *s["rows"]) if "rows" in s else None
        qt = zo.Mx4(n, r, *s["cols"]) if "cols" in s else None
        zo.zo_mx4_quantize(s["x"], q, qt)
        out = {}
        if q is not None:
            zo.zo_mx4_dequantize(q, s["rows_values"])
            out["rows"] = s["rows_values"]
        if qt is not None:
            zo.zo_mx4_dequantize(qt, s["cols_values"])
            out["cols"] = s["cols_values"]
        return out
    if kind == "linear":
        zo.zo_mx4_linear(s["x"], zo.Mx4(c["n"], c["k"], *s["w"]), s["y"],
                         zo.Mx4(c["m"], c["k"], *s["xq"]))
        return {"y": s["y"]}
    if kind == "train":
        t, n, k = c["t"], c["n"], c["k"]
        xq, xt = zo.Mx4(t, k, *s["xq"]), zo.Mx4(k, t, *s["xt"])
        wq, wt = zo.Mx4(n, k, *s["wq"]), zo.Mx4(k, n, *s["wt"])
        gq, gt = zo.Mx4(t, n, *s["gq"]), zo.Mx4(n, t, *s["gt"])
        zo.zo_mx4_quantize(s["x"], xq, xt)
        zo.zo_mx4_quantize(s["w"], wq, wt)
        zo.zo_mx4_product(xq, wq, s["y"])
        zo.zo_mx4_quantize(s["dy"], gq, gt)
        zo.zo_mx4_product(gq, wt, s["dx"])
        zo.zo_mx4_product(gt, xt, s["dw"])
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}
    if kind == "top":
        zo.zo_top_logits(s["z"], s["values"], s["columns"], s["lse"], tau=c["tau"])
        return {"values": s["values"], "columns": s["columns"], "lse": s["lse"]}
    zo.zo_distill_loss(s["z"], s["values"], s["columns"], s["loss"], s["dz"], tau=c["tau"],
                       teacher_lse=s["lse"] if c["tail"] else None,
                       labels=s["labels"] if c["labels"] else None,
                       kd_weight=0.7 if c["labels"] else 1.0,
                       ce_weight=0.3 if c["labels"] else 0.0, row_weight=s["weight"])
    return {"loss": s["loss"], "dz": s["dz"]}


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _rounded(x):
    """x (32 bits) as its 4-bit form along the last axis holds it."""
    cols = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -cols % 32)).unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    e = torch.where(most == 0, -127, torch.frexp(most).exponent - 3).clamp(-127, 127)
    y = torch.ldexp(b.abs(), -e)
    v = 0.5 * (y > 0.25) + 0.5 * (y >= 0.75) + 0.5 * (y > 1.25) + 0.5 * (y >= 1.75)
    v = v + 1.0 * (y > 2.5) + 1.0 * (y >= 3.5) + 2.0 * (y > 5.0)
    v = torch.ldexp(torch.copysign(v, b), e)
    v = torch.where(torch.isfinite(most), v, math.nan)
    return v.flatten(-2)[..., :cols]


def _read(held, rows, cols):
    """The values of held codes and scales."""
    rp, cp = _padded(rows, cols)
    kt = cp // 128
    codes = held[0].view(rp // 16, kt, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(rp, cp // 2)
    scales = held[1].view(rp // 64, kt, 4, 16, 4).permute(0, 4, 3, 1, 2).reshape(rp, cp // 32)
    codes = torch.stack([codes & 15, codes >> 4], -1).view(rp, cp)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6],
                        device=DEV)
    v = grid[codes.int()].unflatten(-1, (-1, 32))
    v = torch.ldexp(v, scales.int().sub(127).unsqueeze(-1))
    return v.flatten(-2)[:rows, :cols]


def _top_plain(z, k, tau):
    rows, vocab = z.shape
    bits = (z + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    # one whole number for value and column, so that of equal values the lowest column is first
    key = (order << 32) + (0xFFFFFFFF - torch.arange(vocab, device=DEV))
    at = torch.topk(key, k, dim=1).values & 0xFFFFFFFF
    at = 0xFFFFFFFF - at
    s = z / tau
    most = s.amax(1, keepdim=True)
    lse = most[:, 0] + (s - most).exp().sum(1).log()
    return z.gather(1, at), at.int(), lse


def _distill_plain(s):
    c = s["case"]
    tau, vocab = c["tau"], c["vocab"]
    kd, ce = (0.7, 0.3) if c["labels"] else (1.0, 0.0)
    z = s["z"].float()
    used = s["columns"] >= 0
    at = s["columns"].clamp(min=0).long()
    x = z / tau
    most = x.amax(1, keepdim=True)
    total = (x - most).exp().sum(1, keepdim=True)
    logq = x - most - total.log()
    q = logq.exp()
    u = torch.where(used, s["values"] / tau, -math.inf)
    if c["tail"]:
        p = (u - s["lse"][:, None]).exp()
    else:
        p = (u - u.amax(1, keepdim=True)).exp()
        p = p / p.sum(1, keepdim=True)
    # p log(p/q) - p + q: the added parts sum to 0 over all outcomes, and each term is
    # then small where p is near q, so that a small divergence keeps its digits
    qs = q.gather(1, at)
    part = p * (torch.where(p > 0, p, 1.0).log() - logq.gather(1, at)) - p + qs
    kl = torch.where(used, part, 0.0).sum(1)
    # p at its columns, unused slots beyond the last one
    slot = torch.where(used, at, vocab)
    target = torch.zeros((z.shape[0], vocab + 1), device=DEV).scatter_(1, slot, p)[:, :vocab]
    ds = q - target
    if c["tail"]:
        inside = torch.zeros((z.shape[0], vocab + 1), dtype=torch.bool, device=DEV)
        inside = inside.scatter_(1, slot, True)[:, :vocab]
        pr = (1.0 - p.sum(1, keepdim=True)).clamp(min=0)
        qr = torch.where(inside, 0.0, q).sum(1, keepdim=True)
        kl = kl + (pr * (torch.where(pr > 0, pr, 1.0) / qr).log() - pr + qr)[:, 0]
        ds = torch.where(inside, ds, q * (1.0 - pr / qr))
    else:
        kl = kl + 1.0 - torch.where(used, qs, 0.0).sum(1)
    loss, dz = kd * tau * tau * kl, kd * tau * ds
    if c["labels"]:
        has = s["labels"] >= 0
        y = s["labels"].clamp(min=0).long()[:, None]
        top = z.amax(1, keepdim=True)
        lse = top + (z - top).exp().sum(1, keepdim=True).log()
        part = ce * torch.where(has, (lse - z.gather(1, y))[:, 0], 0.0)
        soft = (z - lse).exp()
        soft = soft.scatter_add_(1, y, torch.full_like(lse, -1.0))
        loss, dz = loss + part, dz + ce * torch.where(has[:, None], soft, 0.0)
    w = s["weight"]
    return {"loss": w * loss, "dz": (w[:, None] * dz).to(s["z"].dtype)}


def run(state):
    if own:
        return _run_own(state)
    s = state
    c, kind = s["case"], s["kind"]
    if kind == "quantize":
        x, out = s["x"].float(), {}
        if "rows" in s:
            out["rows"] = _rounded(x).bfloat16()
        if "cols" in s:
            out["cols"] = _rounded(x.t().contiguous()).bfloat16()
        return out
    if kind == "linear":
        w = _read(s["w"], c["n"], c["k"])
        return {"y": (_rounded(s["x"].float()) @ w.t()).to(DTYPES[c["out"]])}
    if kind == "train":
        x, w, dy = s["x"].float(), s["w"], s["dy"].float()
        y = _rounded(x) @ _rounded(w).t()
        dx = _rounded(dy) @ _rounded(w.t().contiguous()).t()
        dw = _rounded(dy.t().contiguous()) @ _rounded(x.t().contiguous()).t()
        return {"y": y.bfloat16(), "dx": dx.bfloat16(), "dw": dw}
    if kind == "top":
        values, columns, lse = _top_plain(s["z"].float(), c["top"], c["tau"])
        return {"values": values, "columns": columns, "lse": lse}
    return _distill_plain(s)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _nearest64(x):
    """The 4-bit form of x (64 bits) along the last axis: the nearest multiple of
    the step that the value's own binade has, half to even, at most 6."""
    rows, cols = x.shape
    full = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=DEV)
    full[:, :cols] = x
    b = full.view(rows, -1, 32)
    most = b.abs().max(-1, keepdim=True).values
    unit = torch.exp2(torch.floor(torch.log2(most.clamp(min=2.0 ** -125))) - 2)
    a = b / unit
    step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=1.0))) - 1)
    v = (torch.round(a / step) * step).clamp(-6, 6) * unit
    return v.reshape(rows, -1)[:, :cols]


def _held64(held, rows, cols):
    rp, cp = _padded(rows, cols)
    r = torch.arange(rows, device=DEV)[:, None]
    k = torch.arange(cols, device=DEV)[None]
    lane = (k % 128) // 32 * 16 + r % 16
    byte = ((r // 16 * (cp // 128) + k // 128) * 64 + lane) * 16 + k % 32 // 2
    code = (held[0][byte] >> (4 * (k % 2)).to(torch.uint8)) & 15
    scale = held[1][((r // 64 * (cp // 128) + k // 128) * 64 + lane) * 4 + r % 64 // 16]
    e, m = (code >> 1 & 3).double(), (code & 1).double()
    v = torch.where(e > 0, torch.exp2(e - 1) * (1 + m / 2), m / 2)
    return torch.where(code > 7, -v, v) * torch.exp2(scale.double() - 127)


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind == "quantize":
        x, out = s["x"].double(), {}
        if "rows" in s:
            out["rows"] = _nearest64(x)
        if "cols" in s:
            out["cols"] = _nearest64(x.t())
        return out
    if kind == "linear":
        return {"y": _nearest64(s["x"].double()) @ _held64(s["w"], c["n"], c["k"]).t()}
    if kind == "train":
        x, w, dy = s["x"].double(), s["w"].double(), s["dy"].double()
        return {"y": _nearest64(x) @ _nearest64(w).t(),
                "dx": _nearest64(dy) @ _nearest64(w.t()).t(),
                "dw": _nearest64(dy.t()) @ _nearest64(x.t()).t()}
    if kind == "top":
        z = s["z"].double()
        values, at = torch.sort(z, dim=1, descending=True, stable=True)
        return {"values": values[:, :c["top"]], "columns": at[:, :c["top"]].int(),
                "lse": torch.logsumexp(z / c["tau"], 1)}
    return _distill64(s)


def _distill64(s):
    """Block by block of rows, by the definition: the teacher's distribution over
    its columns (and the rest as one outcome) against the student's."""
    c = s["case"]
    tau = c["tau"]
    kd, ce = (0.7, 0.3) if c["labels"] else (1.0, 0.0)
    rows, vocab = s["z"].shape
    loss = torch.empty(rows, dtype=torch.float64, device=DEV)
    dz = torch.empty((rows, vocab), dtype=torch.float64, device=DEV)
    for r0 in range(0, rows, 512):
        r = slice(r0, min(rows, r0 + 512))
        z = s["z"][r].double()
        q = torch.softmax(z / tau, 1)
        used, at = s["columns"][r] >= 0, s["columns"][r].long()
        u = s["values"][r].double() / tau
        if c["tail"]:
            p = torch.exp(u - s["lse"][r].double()[:, None]) * used
        else:
            p = torch.softmax(u.masked_fill(~used, -math.inf), 1)
        row, slot = used.nonzero(as_tuple=True)
        col = at[row, slot]
        target = torch.zeros_like(z)
        target[row, col] = p[row, slot]
        seen = torch.zeros_like(z, dtype=torch.bool)
        seen[row, col] = True
        kl = torch.special.xlogy(target, target) - torch.special.xlogy(target, q)
        kl = kl.masked_fill(~seen, 0.0).sum(1)
        ds = q - target
        if c["tail"]:
            rest = (1 - p.sum(1)).clamp(min=0)
            tail = q.masked_fill(seen, 0.0).sum(1)
            kl = kl + torch.special.xlogy(rest, rest) - torch.special.xlogy(rest, tail)
            ds = torch.where(seen, ds, q - q * (rest / tail)[:, None])
        part, grad = kd * tau ** 2 * kl, kd * tau * ds
        if c["labels"]:
            y = s["labels"][r].long()
            has = (y >= 0).nonzero()[:, 0]
            part[has] -= ce * torch.log_softmax(z[has], 1)[torch.arange(len(has)), y[has]]
            grad[has] += ce * torch.softmax(z[has], 1)
            grad[has, y[has]] -= ce
        w = s["weight"][r].double()
        loss[r], dz[r] = w * part, w[:, None] * grad
    return {"loss": loss, "dz": dz}
