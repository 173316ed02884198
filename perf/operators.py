"""The grouped products of an expert layer, their gradients and their 8-bit form: cases, inputs and definitions.

Rows are the kept (token, expert) assignments in expert-major order: expert e owns the rows
[offsets[e], offsets[e+1]) of a matrix that was allocated for `rows` of them before routing was known.
Operators, with `own` as calls of the package, without it as elementary torch operations in fp32:

  mm        y[r] = W[e] x[r]                                    (capmoe.grouped_mm)
  train     the same with dx[r] = W[e]^T dy[r] and dW[e] = sum_r dy[r] x[r]^T
                                                                (grouped_mm, grouped_mm_dx, grouped_mm_dw)
  quantize  e4m3 values with one power-of-two scale per 128 columns of a row, or per 128 x 128 block of a
            weight: the smallest one with which no value passes 448 (quantize_rows, quantize_weights)
  mm8       rows quantised, then the product with 8-bit weights (quantize_rows, grouped_mm_fp8)
  ffn8      W_d (silu(W_g x) * (W_u x)) with 8-bit weights, x and the hidden row quantised (grouped_ffn_fp8)
  ffn_grad  gradients of the SwiGLU expert FFN from x and dy: dx, dW_g, dW_u, dW_d (grouped_ffn_backward)

The plain forms lay the rows out as [E, C] slots (an expert keeps at most C rows, which the host knows from the
capacity) and use one batched product.
"""
import math

import torch

own = False

BLOCK = 128
TOP = 448.0                      # largest e4m3 value: 0.875 * 2^9


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of 128 tokens, top-4 of 60 experts, up projection: about 8 rows an expert, latency
        # and weight bytes count
        dict(name="mm decode", op="mm", dtype="bf16", N=128, k=4, E=60, d=2048, n=1408, gamma=1.5, skew=1.0),
        # prompt batch, down projection of 64 narrow experts (an odd multiple of 128 in)
        dict(name="mm prompt", op="mm", dtype="bf16", N=16384, k=6, E=64, d=1408, n=2048, gamma=1.0, skew=1.2),
        # training step of one product in fp32 with sizes that fit no tile and no 16-byte vector
        dict(name="train odd fp32", op="train", dtype="f32", N=517, k=2, E=7, d=250, n=515, gamma=1.5, skew=1.0),
        # training step of one product, 64 experts of 1024 columns, 4096 tokens, top-8
        dict(name="train bf16", op="train", dtype="bf16", N=4096, k=8, E=64, d=2048, n=1024, gamma=1.0, skew=1.0),
        # activations of a decode step: the smallest call
        dict(name="quantize rows decode", op="quantize", what="rows", dtype="bf16", rows=512, d=2048),
        # weights of 64 experts when a model is loaded
        dict(name="quantize weights", op="quantize", what="weights", dtype="bf16", E=64, n=1024, d=2048),
        # decode step as above with 8-bit weights: half the weight bytes
        dict(name="mm8 decode", op="mm8", N=128, k=4, E=60, d=2048, n=1408, gamma=1.5, skew=1.0),
        # prompt batch, 8 wide experts
        dict(name="mm8 prompt", op="mm8", N=8192, k=2, E=8, d=4096, n=14336, gamma=1.25, skew=0.5),
        # the whole expert FFN of a decode step
        dict(name="ffn8 decode", op="ffn8", N=128, k=4, E=60, d=2048, F=1408, gamma=1.5, skew=1.0),
        # the whole expert FFN of a prompt batch, 64 narrow experts
        dict(name="ffn8 prompt", op="ffn8", N=16384, k=6, E=64, d=2048, F=1408, gamma=1.0, skew=1.2),
        # gradients of a small fp32 layer
        dict(name="ffn grad fp32", op="ffn_grad", dtype="f32", N=512, k=2, E=8, d=256, F=512, gamma=1.0, skew=0.5),
        # gradients of 64 narrow experts, 4096 tokens, top-8
        dict(name="ffn grad bf16", op="ffn_grad", dtype="bf16", N=4096, k=8, E=64, d=2048, F=1024, gamma=1.0, skew=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["mm", "train", "quantize", "mm8", "ffn8", "ffn_grad"])
    dtype = "bf16" if op in ("mm8", "ffn8") else rng.choice(["bf16", "bf16", "f32"])
    step = 16 if op in ("mm8", "ffn8") else 8
    wide = lambda: step * _log(rng, 64 // step, 4096 // step) if dtype == "bf16" else _log(rng, 33, 1024)  # noqa: E731
    if op == "quantize":
        if rng.random() < 0.5:
            return dict(op=op, what="rows", dtype=dtype, rows=_log(rng, 1, 100000), d=8 * _log(rng, 8, 1024))
        return dict(op=op, what="weights", dtype=dtype, E=_log(rng, 1, 64), n=8 * _log(rng, 8, 256), d=8 * _log(rng, 8, 256))
    E = _log(rng, 2, 64)
    k = rng.randint(1, min(8, E))
    N = _log(rng, 1, 16384 if dtype == "bf16" else 2048)
    d, n = wide(), wide()
    while E * d * n > 1 << 28:
        E = max(1, E // 2)
        k = min(k, E)
    cost = {"mm": 2, "train": 6, "mm8": 2, "ffn8": 6, "ffn_grad": 16}[op]
    while cost * N * k * d * n > 1 << 40:
        N //= 2
    c = dict(op=op, N=N, k=k, E=E, d=d, gamma=round(rng.uniform(0.5, 2.0), 2), skew=round(rng.uniform(0.0, 1.3), 2))
    c["F" if op in ("ffn8", "ffn_grad") else "n"] = n
    if op not in ("mm8", "ffn8"):
        c["dtype"] = dtype
    return c


def _capacity(c):
    return max(1, min(c["N"], math.ceil(c["gamma"] * c["N"] * c["k"] / c["E"])))


def _popularity(c):
    p = [1.0 / (e + 1) ** c["skew"] for e in range(c["E"])]
    return [v / sum(p) for v in p]


def work(c):
    if c["op"] == "quantize":
        size = 2 if c["dtype"] == "bf16" else 4
        count = c["rows"] * c["d"] if c["what"] == "rows" else c["E"] * c["n"] * c["d"]
        blocks = count / (BLOCK if c["what"] == "rows" else BLOCK * BLOCK)
        return {"bytes": count * (size + 1) + blocks, "flops": 3.0 * count}
    C, p, total = _capacity(c), _popularity(c), c["N"] * c["k"]
    A = sum(min(total * v, C) for v in p)                       # rows, on average
    used = sum(1.0 - (1.0 - v) ** total for v in p)             # experts with rows, on average
    d, n = c["d"], c.get("n", c.get("F"))
    if c["op"] == "mm8":
        return {"bytes": A * (2 * d + 2 * n) + used * n * d, "flops": 2.0 * A * d * n}
    if c["op"] == "ffn8":
        return {"bytes": A * 4 * d + used * 3 * n * d, "flops": 6.0 * A * d * n}
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "mm":
        return {"bytes": size * (A * (d + n) + used * n * d), "flops": 2.0 * A * d * n}
    if c["op"] == "train":
        return {"bytes": size * (2 * A * (d + n) + (used + c["E"]) * n * d), "flops": 6.0 * A * d * n}
    return {"bytes": size * (3 * A * d + 3 * (used + c["E"]) * n * d), "flops": 16.0 * A * d * n}


# ---------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, std, dtype):
    t = torch.empty(shape, device="cuda", dtype=dtype)
    return t.normal_(0.0, std, generator=gen)


def _codes(w):
    """What a checkpoint with 8-bit weights holds: e4m3 values [E, n, d] and the scale of each 128 x 128 block."""
    E, n, d = w.shape
    p = torch.nn.functional.pad(w.float(), (0, 0, 0, -n % BLOCK))
    q, s = _quantized(p.view(-1, d), BLOCK)
    return q.view(E, -1, d)[:, :n].contiguous(), s.view(E, -1, s.shape[1])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    s = dict(op=c["op"], E=c.get("E"))
    if c["op"] == "quantize":
        s["what"] = c["what"]
        shape = (c["rows"], c["d"]) if c["what"] == "rows" else (c["E"], c["n"], c["d"])
        x = _normal(gen, shape, 1.0 if c["what"] == "rows" else 0.02, dtype)
        # a few columns carry values far above the rest, as activations do
        if c["what"] == "rows":
            x[:, torch.randint(0, c["d"], (max(1, c["d"] // 256),), device="cuda", generator=gen)] *= 50
        s["x"] = x
        return s
    host = torch.Generator().manual_seed(seed)
    C, total, E = _capacity(c), c["N"] * c["k"], c["E"]
    picks = torch.multinomial(torch.tensor(_popularity(c), dtype=torch.float64), total, replacement=True, generator=host)
    counts = torch.bincount(picks, minlength=E).clamp(max=C)
    rows = min(total, E * C)
    offsets = torch.zeros(E + 1, dtype=torch.int64)
    offsets[1:] = torch.cumsum(counts, 0)
    d, n = c["d"], c.get("n", c.get("F"))
    s.update(C=C, rows=rows, offsets=offsets.to("cuda", torch.int32), status=torch.zeros(128, device="cuda", dtype=torch.int32))
    s["x"] = _normal(gen, (rows, d), 1.0, dtype)
    if c["op"] in ("mm", "train"):
        s["w"] = _normal(gen, (E, n, d), 0.02, dtype)
        s["y"] = torch.zeros((rows, n), device="cuda", dtype=dtype)
    if c["op"] == "train":
        s["dy"] = _normal(gen, (rows, n), 1.0, dtype)
        s["dx"] = torch.zeros((rows, d), device="cuda", dtype=dtype)
    if c["op"] == "mm8":
        s["w"] = _codes(_normal(gen, (E, n, d), 0.02, dtype))
        s["y"] = torch.zeros((rows, n), device="cuda", dtype=dtype)
    if c["op"] in ("ffn8", "ffn_grad"):
        s["wg"], s["wu"], s["wd"] = (_normal(gen, sh, 0.02, dtype) for sh in ((E, n, d), (E, n, d), (E, d, n)))
        s["y"] = torch.zeros((rows, d), device="cuda", dtype=dtype)
    if c["op"] == "ffn8":
        s["wg"], s["wu"], s["wd"] = _codes(s["wg"]), _codes(s["wu"]), _codes(s["wd"])
    if c["op"] == "ffn_grad":
        s["dy"] = _normal(gen, (rows, d), 1.0, dtype)
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _quantized(x, tall):
    """e4m3 values and power-of-two scales of x [R, d] in blocks of `tall` rows by 128 columns."""
    R, d = x.shape
    rb, db = -(-R // tall), -(-d // BLOCK)
    p = torch.nn.functional.pad(x, (0, db * BLOCK - d, 0, rb * tall - R)).view(rb, tall, db, BLOCK)
    m, ex = torch.frexp(p.abs().amax(dim=(1, 3)))
    e = torch.where(m == 0, 0, ex - 9 + (m > 0.875)).clamp(min=-127).to(torch.int32)
    inv = ((127 - e) << 23).view(torch.float32)                 # 2^-e
    q = (p * inv[:, None, :, None]).view(rb * tall, db * BLOCK)[:R, :d].to(torch.float8_e4m3fn)
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(q, s, tall):
    """fp32 values of blocks of `tall` rows by 128 columns ([..., n, d])."""
    s = s.float().repeat_interleave(tall, -2)[..., : q.shape[-2], :].repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]
    return q.float() * s


def _slots(s):
    """Place of each row in the [E, C] layout; rows behind the last expert's share one spare place."""
    r = torch.arange(s["rows"], device="cuda")
    off = s["offsets"].long()
    e = torch.searchsorted(off[1:].contiguous(), r, right=True)
    return torch.where(e < s["E"], e * s["C"] + r - off[e], s["E"] * s["C"])


def _spread(x, at, s):
    b = torch.zeros((s["E"] * s["C"] + 1, x.shape[1]), device="cuda", dtype=torch.float32)
    b[at] = x.float()
    return b[:-1].view(s["E"], s["C"], -1)


def _gather(y, at, dtype):
    y = y.reshape(-1, y.shape[-1])
    return torch.cat([y, y.new_zeros((1, y.shape[1]))])[at].to(dtype)


def _swiglu8(s):
    at = _slots(s)
    x = _spread(_values(*_quantized(s["x"].float(), 1), 1), at, s)
    g = torch.bmm(x, _values(*s["wg"], BLOCK).transpose(1, 2))
    u = torch.bmm(x, _values(*s["wu"], BLOCK).transpose(1, 2))
    h = g * torch.sigmoid(g) * u
    hq = _values(*_quantized(h.view(-1, h.shape[2]), 1), 1).view(h.shape)
    return _gather(torch.bmm(hq, _values(*s["wd"], BLOCK).transpose(1, 2)), at, s["y"].dtype)


def _swiglu_grad(s):
    at, dt = _slots(s), s["x"].dtype
    x, dy = _spread(s["x"], at, s), _spread(s["dy"], at, s)
    wg, wu, wd = s["wg"].float(), s["wu"].float(), s["wd"].float()
    g, u, dh = torch.bmm(x, wg.transpose(1, 2)), torch.bmm(x, wu.transpose(1, 2)), torch.bmm(dy, wd)
    sig = torch.sigmoid(g)
    h = g * sig * u
    dg, du = dh * u * sig * (1.0 + g * (1.0 - sig)), dh * g * sig
    dx = torch.bmm(dg, wg) + torch.bmm(du, wu)
    return {"dx": _gather(dx, at, dt), "dw_gate": torch.bmm(dg.transpose(1, 2), x).to(dt),
            "dw_up": torch.bmm(du.transpose(1, 2), x).to(dt), "dw_down": torch.bmm(dy.transpose(1, 2), h).to(dt)}


def _plain(s):
    op = s["op"]
    if op == "quantize":
        x = s["x"]
        if s["what"] == "rows":
            q, sc = _quantized(x.float(), 1)
            return {"q": q, "scale": sc}
        q, sc = _codes(x)
        return {"q": q, "scale": sc}
    if op == "ffn8":
        return {"y": _swiglu8(s)}
    if op == "ffn_grad":
        return _swiglu_grad(s)
    at = _slots(s)
    if op == "mm8":
        x, w = _values(*_quantized(s["x"].float(), 1), 1), _values(*s["w"], BLOCK)
        return {"y": _gather(torch.bmm(_spread(x, at, s), w.transpose(1, 2)), at, s["y"].dtype)}
    x, w, dt = _spread(s["x"], at, s), s["w"].float(), s["x"].dtype
    out = {"y": _gather(torch.bmm(x, w.transpose(1, 2)), at, dt)}
    if op == "train":
        dy = _spread(s["dy"], at, s)
        out["dx"] = _gather(torch.bmm(dy, w), at, dt)
        out["dw"] = torch.bmm(dy.transpose(1, 2), x).to(dt)
    return out


def _framework(s):
    from paper_2503_05066_b200 import capmoe
    op = s["op"]
    if op == "quantize":
        q, sc = capmoe.quantize_rows(s["x"]) if s["what"] == "rows" else capmoe.quantize_weights(s["x"])
        return {"q": q, "scale": sc}
    if op == "ffn8":
        return {"y": capmoe.grouped_ffn_fp8(s["x"], s["offsets"], s["wg"], s["wu"], s["wd"], y_perm=s["y"], dev_status=s["status"])}
    if op == "ffn_grad":
        dx, dwg, dwu, dwd = capmoe.grouped_ffn_backward(s["x"], s["dy"], s["offsets"], s["wg"], s["wu"], s["wd"], dx=s["y"],
                                                        dev_status=s["status"])
        return {"dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    if op == "mm8":
        xq, xs = capmoe.quantize_rows(s["x"], s["offsets"])
        return {"y": capmoe.grouped_mm_fp8(xq, xs, s["offsets"], *s["w"], y=s["y"], dev_status=s["status"])}
    out = {"y": capmoe.grouped_mm(s["x"], s["offsets"], s["w"], y=s["y"], dev_status=s["status"])}
    if op == "train":
        out["dx"] = capmoe.grouped_mm_dx(s["dy"], s["offsets"], s["w"], dx=s["dx"], dev_status=s["status"])
        out["dw"] = capmoe.grouped_mm_dw(s["dy"], s["x"], s["offsets"], dev_status=s["status"])
    return out


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- 64 bits
def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round_e4m3(v):
    """Nearest e4m3 value, ties to even, of |v| <= 448: steps of 2^-3 of the leading power of two, of 2^-9 below 2^-6."""
    step = _two(torch.clamp(torch.frexp(v)[1] - 1, min=-6) - 3)
    return torch.round(v / step) * step


def _exact_quantized(x, tall):
    """Values q and scales of x (64 bits) in blocks of `tall` x 128: the smallest power of two with 448 of it above all."""
    R, d = x.shape
    rb, db = -(-R // tall), -(-d // BLOCK)
    wide = x.new_zeros((rb * tall, db * BLOCK))
    wide[:R, :d] = x
    top = wide.view(rb, tall, db, BLOCK).abs().amax(3).amax(1)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, top.new_tensor(TOP)) / TOP))
    e = torch.where(TOP * _two(e - 1) >= top, e - 1, e)         # where the logarithm was off by a step
    e = torch.where(TOP * _two(e) < top, e + 1, e)
    e = torch.where(top > 0, e, torch.zeros_like(e)).clamp(min=-127)
    sc = _two(e)
    q = _round_e4m3(wide / sc.repeat_interleave(tall, 0).repeat_interleave(BLOCK, 1))
    return q[:R, :d].contiguous(), sc


def _exact_rows(x):
    q, sc = _exact_quantized(x.double(), 1)
    return q * sc.repeat_interleave(BLOCK, 1)[:, : x.shape[1]]


def _exact_weight(w, e):
    n, d = w[0].shape[1:]
    return w[0][e].double() * w[1][e].double().repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :d]


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    f64 = dict(device="cuda", dtype=torch.float64)
    if op == "quantize":
        if s["what"] == "rows":
            q, sc = _exact_quantized(s["x"].double(), 1)
            return {"q": q, "scale": sc}
        parts = [_exact_quantized(w.double(), BLOCK) for w in s["x"]]
        return {"q": torch.stack([p[0] for p in parts]), "scale": torch.stack([p[1] for p in parts])}
    off = s["offsets"].tolist()
    E, rows, d = s["E"], s["rows"], s["x"].shape[1]
    n = case.get("n", case.get("F"))
    spans = [(e, slice(off[e], off[e + 1])) for e in range(E)]
    if op in ("mm", "train", "mm8"):
        out = {"y": torch.zeros((rows, n), **f64)}
        if op == "train":
            out["dx"], out["dw"] = torch.zeros((rows, d), **f64), torch.zeros((E, n, d), **f64)
        for e, r in spans:
            w = _exact_weight(s["w"], e) if op == "mm8" else s["w"][e].double()
            x = _exact_rows(s["x"][r]) if op == "mm8" else s["x"][r].double()
            out["y"][r] = x @ w.T
            if op == "train":
                dy = s["dy"][r].double()
                out["dx"][r], out["dw"][e] = dy @ w, dy.T @ x
        return out
    if op == "ffn8":
        y = torch.zeros((rows, d), **f64)
        for e, r in spans:
            x = _exact_rows(s["x"][r])
            g, u = x @ _exact_weight(s["wg"], e).T, x @ _exact_weight(s["wu"], e).T
            y[r] = _exact_rows(g / (1.0 + torch.exp(-g)) * u) @ _exact_weight(s["wd"], e).T
        return {"y": y}
    out = {"dx": torch.zeros((rows, d), **f64)}
    for name in ("dw_gate", "dw_up", "dw_down"):
        out[name] = torch.zeros((E, d, n) if name == "dw_down" else (E, n, d), **f64)
    for e, r in spans:
        x, dy = s["x"][r].double(), s["dy"][r].double()
        wg, wu, wd = s["wg"][e].double(), s["wu"][e].double(), s["wd"][e].double()
        g, u, dh = x @ wg.T, x @ wu.T, dy @ wd
        p = 1.0 / (1.0 + torch.exp(-g))
        silu = g * p
        dg, du = dh * u * (p + silu * (1.0 - p)), dh * silu
        out["dx"][r] = dg @ wg + du @ wu
        out["dw_gate"][e], out["dw_up"][e], out["dw_down"][e] = dg.T @ x, du.T @ x, dy.T @ (silu * u)
    return out
