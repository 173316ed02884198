"""Root-mean-square norm with residual and 8-bit codes, and its gradients, against 64 bits.

Bounds: a sum of K fp32 terms in any order is off by at most K * 2^-23 of the sum of magnitudes, a product or sum of two by
2^-24 of it, rsqrtf by two units (2^-22), a stored value by half a step more (grouped_ref)."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.grouped_ref import close, half_step, rounded

pytestmark = pytest.mark.gpu
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U = 2.0 ** -24


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _normal(shape, std, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=F32).normal_(0.0, std, generator=g).to(dtype)


def _ref(h, w, eps):
    """rstd and y of the stored rows h, with their bounds (before y's rounding to its type)."""
    h, w = h.double(), w.double()
    d = h.shape[1]
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + eps)
    rel = (d + 4) * 2 * U / 2 + 4 * U                       # the sum's error halves under the root; rsqrt and its operand
    y = h * rstd[:, None] * w
    return rstd, rel * rstd + 1e-38, y, (rel + 2.1 * U) * y.abs()


def _check(cm, N, d, dtype, residual, fp8, eps=1e-6, seed=0, scale=1.0):
    x, w = _normal((N, d), scale, dtype, seed), _normal((d,), 1.0, dtype, seed + 1)
    res = _normal((N, d), 2 * scale, dtype, seed + 2) if residual else None
    got = cm.rms_norm(x, w, res, eps=eps, fp8=fp8)
    if residual:
        h = x.double() + res.double()
        close(got["h"], h, U * h.abs() + half_step(dtype) * 1.01 * h.abs() + 1e-38)
    else:
        assert got["h"] is x
    rstd, er, y, ey = _ref(got["h"], w, eps)
    close(got["rstd"], rstd, er)
    close(got["y"], y, rounded(y, ey, dtype))
    if fp8:
        q, s = cm.quantize_rows(got["y"])
        assert torch.equal(got["q"].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got["scale"].view(torch.uint8), s.view(torch.uint8))
    return x, res, w, got


# widths: one vector, odd, one block of 128, borders of it, of a warp's vectors, of a block's, the widest
WIDTHS = [1, 8, 37, 64, 127, 128, 129, 136, 250, 256, 257, 515, 1024, 2048, 2056, 4096, 5000, 8192, 8200, 12295, 16384]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm(cm, d, dtype):
    for N, residual, fp8 in ((1, False, True), (3, True, False), (129, True, True)):
        _check(cm, N, d, dtype, residual, fp8, seed=d + N)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,d", [(5000, 64), (3001, 256), (2500, 1032), (4000, 2048), (2400, 4096), (1300, 515), (1500, 8192)])
def test_norm_of_many_rows(cm, N, d, dtype):
    _check(cm, N, d, dtype, True, True, seed=N)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_no_rows(cm, dtype):
    w = _normal((64,), 1.0, dtype, 1)
    x = torch.empty((0, 64), device="cuda", dtype=dtype)
    got = cm.rms_norm(x, w, x.clone(), fp8=True)
    assert got["y"].shape == (0, 64) and got["q"].shape == (0, 64) and got["scale"].shape == (0, 1) and got["rstd"].shape == (0,)
    dw = torch.full((64,), 7.0, device="cuda", dtype=dtype)
    dx, dw = cm.rms_norm_backward(x, x, w, got["rstd"], dw=dw)
    assert dx.shape == (0, 64) and bool((dw == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_zeros_small_and_large_values(cm, dtype):
    """eps alone under the root; magnitudes whose squares are subnormal or near the largest float."""
    d = 256
    x = _normal((6, d), 1.0, dtype, 3)
    x[0] = 0
    x[1] *= 1e-21
    x[2] *= 1e17
    x[3, 1:] = 0
    w = _normal((d,), 1.0, dtype, 4)
    for eps in (1e-6, 1e-3):
        got = cm.rms_norm(x, w, eps=eps, fp8=True)
        rstd, er, y, ey = _ref(x, w, eps)
        close(got["rstd"], rstd, er)
        close(got["y"], y, rounded(y, ey, dtype))
        assert bool((got["y"][0] == 0).all()) and bool((got["q"][0].float() == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [136, 257, 4096])
def test_nan_and_infinity_stay_in_their_rows(cm, d, dtype):
    x, w, res = _normal((40, d), 1.0, dtype, 5), _normal((d,), 1.0, dtype, 6), _normal((40, d), 1.0, dtype, 7)
    clean = cm.rms_norm(x, w, res, fp8=True)
    x[3, d // 2], x[17, 0], res[29, d - 1] = float("nan"), float("inf"), float("-inf")
    got = cm.rms_norm(x, w, res, fp8=True)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 17, 29]] = True
    for key in ("h", "y", "rstd", "q", "scale"):
        a, b = got[key][~bad], clean[key][~bad]
        assert torch.equal(a.float(), b.float()), key
    assert bool(got["y"][3].isnan().all())
    q, s = cm.quantize_rows(got["y"])
    assert torch.equal(got["q"].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got["scale"].view(torch.uint8), s.view(torch.uint8))
    dy = _normal((40, d), 1.0, dtype, 8)
    dx, _ = cm.rms_norm_backward(dy, got["h"], w, got["rstd"])
    dx0, _ = cm.rms_norm_backward(dy, clean["h"], w, clean["rstd"])
    assert torch.equal(dx[~bad], dx0[~bad]) and bool(dx[3].isnan().all())


def test_in_place_and_into_given_buffers(cm):
    for dtype, d in ((BF16, 1032), (F32, 37)):
        x, res, w, got = _check(cm, 77, d, dtype, True, True, seed=9)
        x2, res2 = x.clone(), res.clone()
        out = {k: torch.empty_like(v) for k, v in got.items()}
        out["h"], out["y"] = res2, x2
        again = cm.rms_norm(x2, w, res2, fp8=True, out=out)
        for k in got:
            assert again[k].data_ptr() == out[k].data_ptr()
            assert torch.equal(again[k].view(torch.uint8), got[k].view(torch.uint8)), k


def _grad_ref(dy, h, w, rstd, dh):
    dy, h, w, r = dy.double(), h.double(), w.double(), rstd.double()[:, None]
    N, d = h.shape
    g, n = dy * w, h * r
    mean, mag = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dx = r * (g - n * mean)
    e = r * (4 * U * (g.abs() + (n * mean).abs()) + n.abs() * ((d + 4) * 2 * U * mag + 4 * U * mean.abs()))
    if dh is not None:
        dx = dx + dh.double()
        e = e + 2 * U * (dh.double().abs() + (r * g).abs() + (r * n * mean).abs())
    dw = (dy * n).sum(0)
    return dx, e, dw, (N + 4) * 2 * U * (dy * n).abs().sum(0)


def _check_grad(cm, N, d, dtype, dh, out_dtype, seed=0):
    h, w = _normal((N, d), 1.5, dtype, seed), _normal((d,), 1.0, dtype, seed + 1)
    dy = _normal((N, d), 1.0, dtype, seed + 2)
    dh = _normal((N, d), 1.0, dtype, seed + 3) if dh else None
    rstd = cm.rms_norm(h, w)["rstd"]
    gx, gw = cm.rms_norm_backward(dy, h, w, rstd, dh=dh, out_dtype=out_dtype)
    dx, e, dw, ew = _grad_ref(dy, h, w, rstd, dh)
    close(gx, dx, rounded(dx, e, dtype))
    assert gw.dtype == (out_dtype or dtype)
    close(gw, dw, rounded(dw, ew, gw.dtype))
    return h, w, dy, dh, rstd, gx, gw


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", WIDTHS)
def test_gradients(cm, d, dtype):
    for N, dh, out in ((1, False, F32), (3, True, None), (130, True, F32)):
        _check_grad(cm, N, d, dtype, dh, out, seed=d + N)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,d", [(5000, 64), (9001, 256), (2500, 1032), (4000, 2048), (2400, 4096), (1300, 515), (1500, 8192)])
def test_gradients_of_many_rows(cm, N, d, dtype):
    _check_grad(cm, N, d, dtype, True, None, seed=N)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,d", [(32, 60), (33, 60), (31, 512), (16, 520), (17, 1024), (4, 4096), (5, 4096), (4, 16384), (2, 8193), (9, 1001), (3000, 24), (2500, 130)])
def test_gradients_of_one_block_and_of_narrow_rows(cm, N, d, dtype):
    for out in (None, F32):
        args = _check_grad(cm, N, d, dtype, True, out, seed=N + d)
    h, w, dy, dh, rstd, gx, gw = args
    room = torch.full((d + 4,), float("nan"), device="cuda")          # dw anywhere on four bytes, and nothing beside it
    x2, w2 = cm.rms_norm_backward(dy, h, w, rstd, dh=dh, dw=room[1:d + 1])
    assert torch.equal(x2, gx) and torch.equal(w2, gw) and bool(room[0].isnan()) and bool(room[d + 1:].isnan().all())


def test_gradients_against_differences(cm):
    """Along random directions: (f(p + s v) - f(p - s v)) / 2s of f = <dy, y> + <dh, h> in 64 bits, whose own error is s^2 and
    rounding / s; the gradient's is its elementwise bound times the direction."""
    N, d, eps, s = 9, 96, 1e-6, 1e-4
    x, res, w = _normal((N, d), 1.0, F32, 1), _normal((N, d), 1.0, F32, 2), _normal((d,), 1.0, F32, 3)
    dy, dh = _normal((N, d), 1.0, F32, 4), _normal((N, d), 1.0, F32, 5)
    got = cm.rms_norm(x, w, res, eps=eps)
    dx, dw = cm.rms_norm_backward(dy, got["h"], w, got["rstd"], dh=dh)

    def f(h, w):
        return ((h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w) * dy.double()).sum() + (h * dh.double()).sum()

    h, w64 = got["h"].double(), w.double()
    for seed in range(4):
        vh, vw = _normal((N, d), 1.0, F32, 10 + seed).double(), _normal((d,), 1.0, F32, 20 + seed).double()
        for grad, v, up, down in ((dx, vh, (h + s * vh, w64), (h - s * vh, w64)), (dw, vw, (h, w64 + s * vw), (h, w64 - s * vw))):
            want = (f(*up) - f(*down)) / (2 * s)
            have = (grad.double() * v).sum()
            # third derivatives are of the order of the gradient itself (rows of unit size): s^2 of the terms; fp32 gradient: d * 2^-23
            assert abs(want - have) <= (100 * s * s + 4 * d * 2 * U) * (grad.double() * v).abs().sum() + 1e-9


def test_workspace_and_gradient_buffers_given(cm):
    h, w, dy, dh, rstd, gx, gw = _check_grad(cm, 300, 1032, BF16, True, F32, seed=4)
    ws = torch.empty((cm.rms_norm_backward_workspace_bytes(300, 1032, BF16),), device="cuda", dtype=torch.uint8)
    for into in (dy.clone(), dh.clone()):
        a = dy if into.data_ptr() != dy.data_ptr() else into
        dw = torch.empty((1032,), device="cuda", dtype=F32)
        x2, w2 = cm.rms_norm_backward(a, h, w, rstd, dh=dh, dx=into, dw=dw, ws=ws)
        assert x2.data_ptr() == into.data_ptr() and torch.equal(x2, gx) and torch.equal(w2, gw)
    dy2 = dy.clone()                                                  # into dy itself
    x2, w2 = cm.rms_norm_backward(dy2, h, w, rstd, dh=dh, dx=dy2, out_dtype=F32)
    assert torch.equal(x2, gx) and torch.equal(w2, gw)
    with pytest.raises(cm.CapmoeError) as e:
        cm.rms_norm_backward(dy, h, w, rstd, ws=ws[:-1])
    assert e.value.status == cm.EWORKSPACE


def test_captured_replayed_and_on_another_stream(cm):
    N, d = 700, 2048
    x, res, w, dy = (_normal(s, 1.0, BF16, i) for i, s in enumerate([(N, d), (N, d), (d,), (N, d)]))

    def run(stream=None):
        f = cm.rms_norm(x, w, res, fp8=True, stream=stream)
        return [f[k] for k in ("h", "y", "rstd", "q", "scale")] + list(cm.rms_norm_backward(dy, f["h"], w, f["rstd"], dh=res, stream=stream))

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = run(side)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):                                                # two graphs, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out))
    first = [a.clone() for a in want]
    for seed in (50, 51):
        x.copy_(_normal((N, d), 1.0, BF16, seed))
        for g, _ in graphs:
            g.replay()
        now = run()
        for _, out in graphs:
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(out, now))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, other))


def test_rows_past_32_bit_offsets(cm):
    d = 16384
    N = (1 << 31) // d + 100
    x = torch.empty((N, d), device="cuda", dtype=BF16)
    x[:3].copy_(_normal((3, d), 1.0, BF16, 1))
    x[3:].fill_(0.25)
    x[-60:].copy_(_normal((60, d), 1.0, BF16, 2))
    w = _normal((d,), 1.0, BF16, 3)
    got = cm.rms_norm(x, w, x, fp8=True)
    part = cm.rms_norm(x[-60:].clone(), w, x[-60:].clone(), fp8=True)
    for k in ("h", "y", "rstd", "q", "scale"):
        assert torch.equal(got[k][-60:].view(torch.uint8), part[k].view(torch.uint8)), k
    dx, _ = cm.rms_norm_backward(x, got["h"], w, got["rstd"], dx=got["y"])
    ref, e, _, _ = _grad_ref(x[-60:], got["h"][-60:], w, got["rstd"][-60:], None)
    close(dx[-60:], ref, rounded(ref, e, BF16))


def test_guard_bands(cm):
    """Nothing around the outputs is written."""
    for dtype, N, d in ((BF16, 5, 136), (F32, 5, 37), (BF16, 3, 515)):
        x, res, w = _normal((N, d), 1.0, dtype, 1), _normal((N, d), 1.0, dtype, 2), _normal((d,), 1.0, dtype, 3)
        held = []

        def buf(shape, t):
            n = 1
            for v in shape:
                n *= v
            size = n * torch.empty((), dtype=t).element_size()
            raw = torch.full((256 + size + 256,), 0x5A, device="cuda", dtype=torch.uint8)
            held.append((raw, size))
            return raw[256:256 + size].view(t).view(shape)

        nb = (d + 127) // 128
        out = dict(h=buf((N, d), dtype), y=buf((N, d), dtype), rstd=buf((N,), F32), q=buf((N, d), cm.FP8), scale=buf((N, nb), cm.SCALE))
        f = cm.rms_norm(x, w, res, fp8=True, out=out)
        cm.rms_norm_backward(x, f["h"], w, f["rstd"], dx=buf((N, d), dtype), dw=buf((d,), F32),
                             ws=buf((cm.rms_norm_backward_workspace_bytes(N, d, dtype),), torch.uint8))
        for raw, size in held:
            assert bool((raw[:256] == 0x5A).all()) and bool((raw[256 + size:] == 0x5A).all())


def test_the_same_bits_every_time(cm):
    h, w, dy = _normal((3000, 1024), 1.0, BF16, 1), _normal((1024,), 1.0, BF16, 2), _normal((3000, 1024), 1.0, BF16, 3)
    rstd = cm.rms_norm(h, w)["rstd"]
    want = cm.rms_norm_backward(dy, h, w, rstd, out_dtype=F32)
    for _ in range(20):
        got = cm.rms_norm_backward(dy, h, w, rstd, out_dtype=F32)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
