"""64-bit definitions of the grouped products, their gradients and their 8-bit form, each with an elementwise
bound on what fp32 accumulation and the roundings to the storage type may add.

An fp32 sum of K products in any order differs from the exact one by at most K * 2^-23 * sum |a b| (2^-24 for
each of the K - 1 additions, the same again where an adder truncates instead of rounding); a stored value is off
by half a step more, eps / 2 of it (2^-8 for bf16, 2^-24 for fp32)."""
import torch

BLOCK, TOP = 128, 448.0
F64 = torch.float64


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def offsets_of(counts):
    o = torch.zeros(len(counts) + 1, dtype=torch.int32)
    o[1:] = torch.cumsum(torch.tensor(counts, dtype=torch.int32), 0)
    return o.cuda()


def product(a, b, stored=None):
    """a [R,K] b [C,K]^T in 64 bits with its fp32 bound; `stored`: rounded once more to that type."""
    y = a @ b.T
    e = a.shape[1] * 2.0 ** -23 * (a.abs() @ b.abs().T)
    return y, e if stored is None else e + half_step(stored) * (y.abs() + e) + 1e-38


def rounded(y, e, dtype):
    return e + half_step(dtype) * (y.abs() + e) + 1e-38


def close(got, ref, err):
    d = (got.double() - ref).abs()
    assert bool(torch.isfinite(d).all()), "not finite"
    assert bool((d <= err).all()), f"worst excess {float((d - err).max()):.3e}, worst ratio {float((d / err).max()):.2f}"


# ------------------------------------------------------------------------------------------- 8 bits
def two(e):
    return ((e.long() + 1023) << 52).view(F64)


def round_e4m3(v):
    step = two(torch.clamp(torch.frexp(v)[1] - 1, min=-6) - 3)
    return torch.round(v / step) * step


def scale_exponent(top):
    """Smallest e >= -127 with top <= 448 * 2^e; 0 for zero."""
    m, ex = torch.frexp(top)
    e = (ex - 9 + (m > 0.875).int()).clamp(min=-127)
    return torch.where(top > 0, e, torch.zeros_like(e))


def block_max(x, tall):
    R, d = x.shape
    rb, db = -(-R // tall), -(-d // BLOCK)
    p = torch.zeros((rb * tall, db * BLOCK), dtype=F64, device=x.device)
    p[:R, :d] = x.abs()
    return p.view(rb, tall, db, BLOCK).amax(3).amax(1)


def spread(s, tall, shape):
    return s.repeat_interleave(tall, 0)[: shape[0]].repeat_interleave(BLOCK, 1)[:, : shape[1]]


def quantized(x, tall, e=None):
    """(codes' values, scale exponents) of x [R,d] in 64 bits; `e`: with these exponents.  A block that holds a NaN
    or an infinity has NaN codes and exponent 128 (the scale code of a NaN)."""
    top = block_max(x, tall)
    lost = ~torch.isfinite(top)
    if e is None:
        e = torch.where(lost, torch.full_like(top, 128).int(), scale_exponent(torch.where(lost, 0.0, top)))
    q = round_e4m3((x / spread(two(e), tall, x.shape)).clamp(-TOP, TOP))
    return torch.where(spread(lost, tall, x.shape), float("nan"), q), e


def same_codes(q, s, ref):
    """Codes' values and scales equal to the reference's, NaN for NaN."""
    rq, re = ref
    rs = torch.where(re == 128, float("nan"), two(re))
    return (torch.equal(q.double().nan_to_num(-1e9), rq.nan_to_num(-1e9)) and
            torch.equal(s.double().nan_to_num(-1e9), rs.nan_to_num(-1e9)))


def values(x, tall):
    q, e = quantized(x, tall)
    return q * spread(two(e), tall, x.shape)


def decoded(q, s, tall):
    return q.double() * spread(s.double(), tall, q.shape)


# ------------------------------------------------------------------------------------------- SwiGLU
def swiglu(x, wg, wu):
    """h = silu(x wg^T) * (x wu^T) with its fp32 bound (exponential and division: a few steps of 2^-23)."""
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    p = torch.sigmoid(g)
    a = g * p
    h = a * u
    ea = 1.1 * eg + 2.0 ** -20 * a.abs()                    # |silu'| < 1.1
    return g, u, h, ea * u.abs() + a.abs() * eu + ea * eu + 2.0 ** -22 * h.abs()


def quantized_hidden(h, e):
    """Values of h after the row quantiser and how far they may be off when h is off by e: h moved to either end
    of its interval, and a block's scale taken for either end of its maximum."""
    q = values(h, 1)
    top = block_max(h, 1)
    te = block_max(e, 1)
    worst = torch.zeros_like(h)
    for t in (top - te, top, top + te):
        sc = scale_exponent(t.clamp(min=0))
        for v in (h - e, h, h + e):
            worst = torch.maximum(worst, (quantized(v, 1, sc)[0] * spread(two(sc), 1, h.shape) - q).abs())
    return q, worst


def ffn_gradient(x, dy, wg, wu, wd, dtype):
    """Gradients of one expert's FFN and their bounds, intermediates dg, du and h rounded to `dtype`."""
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    dh, edh = product(dy, wd.T)
    p = torch.sigmoid(g)
    a = g * p
    da = p + a * (1 - p)
    dg, du, h = dh * u * da, dh * a, a * u
    ulp = 2.0 ** -20
    # |silu'| < 1.1, |silu''| <= 0.5
    edg = 1.1 * (edh * u.abs() + dh.abs() * eu + edh * eu) + 0.5 * eg * (dh * u).abs() + ulp * (dh * u).abs()
    edu = edh * (a.abs() + 1.1 * eg) + dh.abs() * 1.1 * eg + ulp * (dh * a).abs() + ulp * dh.abs() * g.abs()
    eh = 1.1 * eg * (u.abs() + eu) + a.abs() * eu + ulp * h.abs() + ulp * (g * u).abs()
    edg, edu, eh = rounded(dg, edg, dtype), rounded(du, edu, dtype), rounded(h, eh, dtype)

    def second(m, em, n, en=None):
        """m^T n over the rows, m off by em (n by en), accumulated in fp32 and stored."""
        y = m.T @ n
        am, an = m.abs() + em, n.abs() + (0 if en is None else en)
        e = em.T @ n.abs() + (0 if en is None else am.T @ en) + m.shape[0] * 2.0 ** -23 * (am.T @ an)
        return y, rounded(y, e, dtype)

    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + 2 * wg.shape[0] * 2.0 ** -23 * ((dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs())
    z = torch.zeros_like(dy)
    return {"dx": (dx, rounded(dx, edx, dtype)), "dw_gate": second(dg, edg, x), "dw_up": second(du, edu, x),
            "dw_down": second(dy, z, h, eh)}
