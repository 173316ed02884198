"""What stands around the grouped products of an expert layer when it is trained or served in 8 bits: cases, inputs and definitions.

N tokens of d columns are routed to k of E experts; an expert keeps its C best-scored tokens.  slot_row[t, s] is the row that
token t's slot s holds in the expert-major order of the kept (token, expert) pairs, or -1; slots 0..k-1 are the token's top-k
experts, and with D > 0 the slots behind them the E/D experts of the token's own device.  Operators, with `own` as calls of the
package, without it as elementary torch operations:

  norm          h = x + residual, y = h / rms(h) * w, and y's rows as e4m3 codes with one power-of-two scale per 128 columns
                                                                (capmoe.rms_norm)
  norm_grad     gradients of x (and of the residual, the same) and of w from dy and what flows into h from behind
                                                                (rms_norm_backward)
  permute8      rows of codes and scales sorted by expert       (permute_fp8)
  combine_grad  of y[t] = sum_s weight[r] y_perm[r]: dy_perm[r] = weight[r] dy[t], dweight[r] = dy[t] . y_perm[r]
                                                                (combine_backward)
  permute_grad  dx[t] = sum_s dx_perm[slot_row[t, s]] + add[t]  (permute_backward)
  route_grad    from the gradient of the kept pairs' softmax scores (and of all scores, where a balance loss gives it one) to
                those of the logits, the tokens, the router's weights and its bias
                                                                (route_backward)
"""
import math

import torch

own = False

BLOCK = 128
EPS = 1e-5


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # in front of the experts, one decode step of 128 tokens: the smallest call, latency counts
        dict(name="norm decode", op="norm", dtype="bf16", N=128, d=4096, residual=True, codes=True),
        # the same for a prompt batch
        dict(name="norm prompt", op="norm", dtype="bf16", N=16384, d=2048, residual=True, codes=True),
        # a small model in fp32, a width that fits no 16-byte vector
        dict(name="norm grad odd fp32", op="norm_grad", dtype="f32", N=517, d=515, residual=False),
        # training step, wide rows
        dict(name="norm grad bf16", op="norm_grad", dtype="bf16", N=16384, d=4096, residual=True),
        # 8-bit rows of a decode step, top-4 of 60 experts
        dict(name="permute8 decode", op="permute8", N=128, k=4, E=60, D=0, d=2048, gamma=1.5, skew=1.0),
        # 8-bit rows of a prompt batch, top-6 of 64 experts, popular experts overflow
        dict(name="permute8 prompt", op="permute8", N=16384, k=6, E=64, D=0, d=2048, gamma=1.0, skew=1.2),
        # training step of a small fp32 layer
        dict(name="combine grad fp32", op="combine_grad", dtype="f32", N=512, k=2, E=8, D=0, d=256, gamma=1.0, skew=0.5),
        # training step of 64 narrow experts, top-8
        dict(name="combine grad bf16", op="combine_grad", dtype="bf16", N=16384, k=8, E=64, D=0, d=2048, gamma=1.0, skew=1.0),
        # training step of 8 wide experts, tokens also offered to the experts of their own device, gradient of a shared expert added
        dict(name="permute grad expanded", op="permute_grad", dtype="bf16", N=8192, k=2, E=8, D=4, d=4096, gamma=1.25, skew=0.5, add=True),
        # training step, top-6 of 64 experts
        dict(name="permute grad bf16", op="permute_grad", dtype="bf16", N=16384, k=6, E=64, D=0, d=2048, gamma=1.0, skew=1.2, add=False),
        # a small fp32 router, sizes that fit no tile
        dict(name="route grad odd fp32", op="route_grad", dtype="f32", N=517, k=2, E=7, D=0, d=250, gamma=1.5, skew=1.0, aux=False),
        # training step, router of 64 experts with a balance loss
        dict(name="route grad bf16", op="route_grad", dtype="bf16", N=16384, k=8, E=64, D=0, d=2048, gamma=1.0, skew=1.0, aux=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _no_larger(c):
    """The case with as many tokens as keep it below the largest listed ones."""
    while c["N"] > 1 and (work(c)["bytes"] > 6.0e8 or work(c)["flops"] > 8.0e9):
        c["N"] //= 2
    return c


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "permute8", "combine_grad", "permute_grad", "route_grad"])
    c = dict(op=op)
    if op != "permute8":
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    N = _log(rng, 1, 65536)
    if op in ("norm", "norm_grad"):
        d = _log(rng, 33, 8192) if rng.random() < 0.25 else 8 * _log(rng, 8, 1024)
        c.update(N=N, d=d, residual=rng.random() < 0.75)
        if op == "norm":
            c["codes"] = rng.random() < 0.5
        return _no_larger(c)
    E = _log(rng, 2, 256)
    k = rng.randint(1, min(8, E))
    d = 16 * _log(rng, 4, 512)
    if op == "route_grad" and rng.random() < 0.25:
        d = _log(rng, 33, 2048)
    groups = [g for g in (1, 2, 4, 8, 16) if E % g == 0 and E // g <= 8]
    D = rng.choice(groups) if groups and rng.random() < 0.3 else 0
    c.update(N=max(1, min(N, (1 << 22) // E)), k=k, E=E, D=D, d=d, gamma=round(rng.uniform(0.5, 2.0), 2), skew=round(rng.uniform(0.0, 1.3), 2))
    if op == "permute_grad":
        c["add"] = rng.random() < 0.5
    if op == "route_grad":
        c["aux"] = rng.random() < 0.5
    return _no_larger(c)


def _capacity(c):
    return max(1, min(c["N"], math.ceil(c["gamma"] * c["N"] * c["k"] / c["E"])))


def _slots(c):
    return c["k"] + (c["E"] // c["D"] if c["D"] else 0)


def _rows(c):
    """Rows that are allocated before routing is known."""
    return min(c["N"] * _slots(c), c["E"] * _capacity(c))


def _kept(c):
    """Kept pairs, on average: offers of an expert are its share of N * k, with D > 0 also N / D tokens of its device."""
    p = [1.0 / (e + 1) ** c["skew"] for e in range(c["E"])]
    near = c["N"] / c["D"] if c["D"] else 0
    total = 0.0
    for v in p:
        hit = min(c["N"], c["N"] * c["k"] * v / sum(p))
        total += min(hit + near * (1.0 - hit / c["N"]), _capacity(c))
    return total


def work(c):
    size = 4 if c.get("dtype") == "f32" else 2
    N, d, op = c["N"], c["d"], c["op"]
    if op == "norm":
        return {"bytes": N * d * size * (4 if c["residual"] else 2) + (N * (d + d / BLOCK) if c["codes"] else 0) + 4 * N,
                "flops": (8.0 if c["codes"] else 5.0) * N * d}
    if op == "norm_grad":
        return {"bytes": N * d * size * (4 if c["residual"] else 3), "flops": 11.0 * N * d}
    A, slots, E = _kept(c), _slots(c), c["E"]
    if op == "permute8":
        return {"bytes": (N + A) * (d + d / BLOCK) + 4 * N * slots + 12 * A, "flops": 0.0}
    if op == "combine_grad":
        return {"bytes": (N + 2 * A) * d * size + 4 * N * slots + 8 * A, "flops": 3.0 * A * d}
    if op == "permute_grad":
        return {"bytes": (A + N * (2 if c["add"] else 1)) * d * size + 4 * N * slots, "flops": 1.0 * A * d}
    return {"bytes": 2 * N * d * size + 2 * E * d * size + 8 * N * E + 4 * N * (slots + c["k"]) + 4 * A,
            "flops": 4.0 * N * E * d}


# ---------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, std, dtype):
    t = torch.empty(shape, device="cuda", dtype=dtype)
    return t.normal_(0.0, std, generator=gen)


def _activations(gen, N, d, dtype):
    """A few columns carry values far above the rest, as activations do."""
    x = _normal(gen, (N, d), 1.0, dtype)
    x[:, torch.randint(0, d, (max(1, d // 256),), device="cuda", generator=gen)] *= 50
    return x


def _routing(c, gen):
    """Scores, top-k lists and rows of the kept pairs, as the layer's first stages leave them."""
    N, E, k, D = c["N"], c["E"], c["k"], c["D"]
    liked = -c["skew"] * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    scores = torch.softmax(_normal(gen, (N, E), 1.0, torch.float32) + liked, dim=1)
    top = torch.sort(scores, dim=1, descending=True, stable=True)[1][:, :k]
    in_top = torch.zeros((N, E), device="cuda", dtype=torch.bool).scatter_(1, top, True)
    offered = in_top
    if D:
        m = E // D
        home = torch.arange(N, device="cuda") * D // N
        offered = in_top | (torch.arange(E, device="cuda") // m == home[:, None])
    order = torch.argsort(torch.where(offered, scores, -1.0), dim=0, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(0, order, torch.arange(N, device="cuda")[:, None].expand(N, E))
    kept = offered & (rank < _capacity(c))
    count = kept.sum(0)
    offsets = torch.zeros(E + 1, device="cuda", dtype=torch.int64)
    offsets[1:] = torch.cumsum(count, 0)
    row = torch.where(kept, torch.cumsum(kept, 0) - 1 + offsets[:-1], -1)
    slot_row = row.gather(1, top)
    if D:
        near = home[:, None] * m + torch.arange(m, device="cuda")
        slot_row = torch.cat([slot_row, torch.where(in_top.gather(1, near), -1, row.gather(1, near))], 1)
    t, e = torch.nonzero(kept, as_tuple=True)
    r = row[t, e]
    rows = _rows(c)
    token = torch.full((rows,), -1, device="cuda", dtype=torch.int32)
    weight = torch.zeros((rows,), device="cuda", dtype=torch.float32)
    token[r], weight[r] = t.int(), scores[t, e]
    return dict(scores=scores, topk=top.int().contiguous(), slot_row=slot_row.int().contiguous(), token=token, weight=weight,
                offsets=offsets.int(), rows=rows, kept=r.numel())


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    N, d, op = c["N"], c["d"], c["op"]
    s = dict(op=op, codes=c.get("codes"), E=c.get("E"), D=c.get("D"), k=c.get("k"))
    if op == "norm":
        s["x"] = _activations(gen, N, d, dtype)
        s["residual"] = _normal(gen, (N, d), 3.0, dtype) if c["residual"] else None
        s["w"] = (1.0 + _normal(gen, (d,), 0.1, torch.float32)).to(dtype)
        return s
    if op == "norm_grad":
        s["h"] = _activations(gen, N, d, dtype)
        s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
        s["w"] = (1.0 + _normal(gen, (d,), 0.1, torch.float32)).to(dtype)
        s["dy"] = _normal(gen, (N, d), 1.0, dtype)
        s["dh"] = _normal(gen, (N, d), 1.0, dtype) if c["residual"] else None
        return s
    s.update(_routing(c, gen))
    rows = s["rows"]
    if op == "permute8":
        s["q"], s["scale"] = _quantized(_activations(gen, N, d, dtype).float())
        s["out"] = dict(x_q=torch.zeros((rows, d), device="cuda", dtype=torch.float8_e4m3fn),
                        x_scale=torch.ones((rows, -(-d // BLOCK)), device="cuda").to(torch.float8_e8m0fnu),
                        perm_token=torch.full((rows,), -1, device="cuda", dtype=torch.int32),
                        perm_weight=torch.zeros((rows,), device="cuda"))
    if op == "combine_grad":
        s["dy"], s["y_perm"] = _normal(gen, (N, d), 1.0, dtype), _normal(gen, (rows, d), 1.0, dtype)
        s["dy_perm"] = torch.zeros((rows, d), device="cuda", dtype=dtype)
        s["dweight"] = torch.zeros((rows,), device="cuda")
    if op == "permute_grad":
        s["dx_perm"] = _normal(gen, (rows, d), 1.0, dtype)
        s["add"] = _normal(gen, (N, d), 1.0, dtype) if c["add"] else None
    if op == "route_grad":
        s["x"], s["w"] = _activations(gen, N, d, dtype), _normal(gen, (c["E"], d), 0.02, dtype)
        s["dweight"] = _normal(gen, (rows,), 1.0, torch.float32)
        s["dscores"] = None
        if c["aux"]:                      # of 0.01 E * sum_e (share of the pairs) * (mean score): the same for every token
            share = torch.bincount(s["topk"].flatten().long(), minlength=c["E"]).float() / (N * c["k"])
            s["dscores"] = 0.01 * c["E"] / N * share
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _quantized(x):
    """e4m3 codes and power-of-two scales of the rows x [R, d] (fp32): per 128 columns the smallest scale that keeps all below 448."""
    R, d = x.shape
    db = -(-d // BLOCK)
    p = torch.nn.functional.pad(x, (0, db * BLOCK - d)).view(R, db, BLOCK)
    m, ex = torch.frexp(p.abs().amax(dim=2))
    e = torch.where(m == 0, 0, ex - 9 + (m > 0.875)).clamp(min=-127).to(torch.int32)
    inv = ((127 - e) << 23).view(torch.float32)                 # 2^-e
    q = (p * inv[:, :, None]).view(R, db * BLOCK)[:, :d].to(torch.float8_e4m3fn)
    return q.contiguous(), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _expert_of_slots(s):
    """[N, slots] expert ids."""
    e = s["topk"].long()
    if s["D"]:
        N, m = e.shape[0], s["E"] // s["D"]
        home = torch.arange(N, device="cuda") * s["D"] // N
        e = torch.cat([e, home[:, None] * m + torch.arange(m, device="cuda")], 1)
    return e


def _plain(s):
    op = s["op"]
    if op == "norm":
        x = s["x"]
        h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
        hf = h.float()
        rstd = torch.rsqrt(hf.square().mean(1) + EPS)
        y = (hf * rstd[:, None] * s["w"].float()).to(x.dtype)
        out = {"rstd": rstd, "y": y}
        if s["residual"] is not None:
            out["h"] = h
        if s["codes"]:
            out["q"], out["scale"] = _quantized(y.float())
        return out
    if op == "norm_grad":
        xhat = s["h"].float() * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["w"].float()
        dx = s["rstd"][:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["h"].dtype), "dw": (dy * xhat).sum(0)}
    if op == "permute8":
        r = torch.nonzero(s["token"] >= 0).flatten()
        t = s["token"][r].long()
        out = {"x_q": torch.zeros_like(s["out"]["x_q"]), "x_scale": torch.ones_like(s["out"]["x_scale"].float()).to(s["scale"].dtype),
               "perm_token": torch.full_like(s["token"], -1), "perm_weight": torch.zeros_like(s["weight"])}
        out["x_q"].view(torch.uint8)[r] = s["q"].view(torch.uint8)[t]
        out["x_scale"].view(torch.uint8)[r] = s["scale"].view(torch.uint8)[t]
        at = s["slot_row"] >= 0
        n = torch.nonzero(at)[:, 0]
        out["perm_token"][s["slot_row"][at].long()] = n.int()
        out["perm_weight"][s["slot_row"][at].long()] = s["scores"][n, _expert_of_slots(s)[at]]
        return out
    live = s.get("token")
    if op == "combine_grad":
        dy = torch.where((live >= 0)[:, None], s["dy"].float()[live.clamp(min=0).long()], 0.0)
        return {"dy_perm": (dy * s["weight"][:, None]).to(s["dy"].dtype), "dweight": (dy * s["y_perm"].float()).sum(1)}
    if op == "permute_grad":
        N, d = s["slot_row"].shape[0], s["dx_perm"].shape[1]
        dx = torch.zeros((N + 1, d), device="cuda") if s["add"] is None else torch.cat([s["add"].float(), torch.zeros((1, d), device="cuda")])
        dx.index_add_(0, torch.where(live >= 0, live, N).long(), s["dx_perm"].float())
        return {"dx": dx[:N].to(s["dx_perm"].dtype)}
    sr = s["slot_row"].long()
    dS = torch.zeros_like(s["scores"])
    dS.scatter_add_(1, _expert_of_slots(s), torch.where(sr >= 0, s["dweight"][sr.clamp(min=0)], 0.0))
    if s["dscores"] is not None:
        dS = dS + s["dscores"]
    S = s["scores"]
    dl = S * (dS - (S * dS).sum(1, keepdim=True))
    dt = s["x"].dtype
    return {"dlogits": dl, "dx": (dl @ s["w"].float()).to(dt), "dw": (dl.T @ s["x"].float()).to(dt), "dbias": dl.sum(0)}


def _framework(s):
    from paper_2503_05066_b200 import capmoe
    op = s["op"]
    if op == "norm":
        out = capmoe.rms_norm(s["x"], s["w"], s["residual"], eps=EPS, fp8=s["codes"])
        wanted = ["rstd", "y"] + (["h"] if s["residual"] is not None else []) + (["q", "scale"] if s["codes"] else [])
        return {name: out[name] for name in wanted}
    if op == "norm_grad":
        dx, dw = capmoe.rms_norm_backward(s["dy"], s["h"], s["w"], s["rstd"], dh=s["dh"], out_dtype=torch.float32)
        return {"dx": dx, "dw": dw}
    if op == "permute8":
        return capmoe.permute_fp8(s["q"], s["scale"], s["scores"], s["topk"], s["slot_row"], s["rows"], D=s["D"], out=s["out"])
    if op == "combine_grad":
        dy_perm, dweight = capmoe.combine_backward(s["dy"], s["y_perm"], s["slot_row"], s["weight"], dy_perm=s["dy_perm"],
                                                   dweight=s["dweight"])
        return {"dy_perm": dy_perm, "dweight": dweight}
    if op == "permute_grad":
        return {"dx": capmoe.permute_backward(s["dx_perm"], s["slot_row"], add=s["add"])}
    out = capmoe.route_backward(s["x"], s["w"], s["scores"], s["topk"], s["slot_row"], s["dweight"], D=s["D"], dscores=s["dscores"])
    return {name: out[name] for name in ("dlogits", "dx", "dw", "dbias")}


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- 64 bits
def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(y):
    """Codes and scales (64 bits) of y [R, d]: the smallest power of two with 448 of it above all, then the nearest e4m3 value."""
    R, d = y.shape
    wide = y.new_zeros((R, -(-d // BLOCK) * BLOCK))
    wide[:, :d] = y
    top = wide.view(R, -1, BLOCK).abs().amax(2)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, top.new_tensor(448.0)) / 448.0))
    e = torch.where(448.0 * _two(e - 1) >= top, e - 1, e)       # where the logarithm was off by a step
    e = torch.where(448.0 * _two(e) < top, e + 1, e)
    e = torch.where(top > 0, e, torch.zeros_like(e)).clamp(min=-127)
    v = wide / _two(e).repeat_interleave(BLOCK, 1)
    step = _two(torch.clamp(torch.frexp(v)[1] - 1, min=-6) - 3)
    return (torch.round(v / step) * step)[:, :d].contiguous(), _two(e)


def exact(case, seed):
    s = prepare(case, seed)
    op, N, d = s["op"], case["N"], case["d"]
    f64 = dict(device="cuda", dtype=torch.float64)
    if op == "norm":
        # h, and y where it is turned into codes, are defined as rounded to the tokens' type
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        stored = h.to(s["x"].dtype).double()
        rstd = 1.0 / torch.sqrt(torch.sum(stored * stored, 1) / d + EPS)
        y = stored * s["w"].double() * rstd[:, None]
        out = {"rstd": rstd, "y": y}
        if s["residual"] is not None:
            out["h"] = h
        if s["codes"]:
            out["q"], out["scale"] = _exact_codes(y.to(s["x"].dtype).double())
        return out
    if op == "norm_grad":
        h, dy, w, r = s["h"].double(), s["dy"].double(), s["w"].double(), s["rstd"].double()
        dot = torch.einsum("nd,nd,d->n", dy, h, w)
        dx = dy * w * r[:, None] - h * (r ** 3 * dot / d)[:, None]
        if s["dh"] is not None:
            dx += s["dh"].double()
        return {"dx": dx, "dw": torch.einsum("nd,nd,n->d", dy, h, r)}
    if op == "permute8":
        rows, kept = s["rows"], s["kept"]
        t = s["token"][:kept].long()
        q, sc = torch.zeros((rows, d), **f64), torch.ones((rows, s["scale"].shape[1]), **f64)
        q[:kept], sc[:kept] = s["q"].double()[t], s["scale"].double()[t]
        return {"x_q": q, "x_scale": sc, "perm_token": s["token"], "perm_weight": s["weight"]}
    if op == "combine_grad":
        dy_perm, dweight = torch.zeros((s["rows"], d), **f64), torch.zeros((s["rows"],), **f64)
        for slot in s["slot_row"].long().T:
            t = torch.nonzero(slot >= 0).flatten()
            r, dy = slot[t], s["dy"][t].double()
            dy_perm[r] = s["weight"][r].double()[:, None] * dy
            dweight[r] = torch.einsum("nd,nd->n", dy, s["y_perm"][r].double())
        return {"dy_perm": dy_perm, "dweight": dweight}
    if op == "permute_grad":
        dx = torch.zeros((N, d), **f64) if s["add"] is None else s["add"].double()
        for slot in s["slot_row"].long().T:
            t = torch.nonzero(slot >= 0).flatten()
            dx[t] += s["dx_perm"][slot[t]].double()
        return {"dx": dx}
    E, S = s["E"], s["scores"].double()
    dS = torch.zeros((N, E), **f64) if s["dscores"] is None else s["dscores"].double().repeat(N, 1)
    expert = torch.searchsorted(s["offsets"][1:].contiguous().long(), torch.arange(s["kept"], device="cuda"), right=True)
    dS[s["token"][: s["kept"]].long(), expert] += s["dweight"][: s["kept"]].double()
    dl = S * dS - S * torch.einsum("ne,ne->n", S, dS)[:, None]
    return {"dlogits": dl, "dx": dl @ s["w"].double(), "dw": torch.einsum("ne,nd->ed", dl, s["x"].double()),
            "dbias": torch.einsum("ne->e", dl)}
