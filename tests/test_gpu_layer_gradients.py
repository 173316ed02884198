"""8-bit permute, the gradients of combine, permute and router, and the whole layer's backward pass, against 64 bits.
Bounds as in grouped_ref: K * 2^-23 of the sum of magnitudes for an fp32 sum of K terms, half a step for what is stored."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.grouped_ref import close, ffn_gradient, half_step, rounded

pytestmark = pytest.mark.gpu
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U2 = 2.0 ** -23


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, std, dtype, seed):
    return torch.empty(shape, device="cuda", dtype=F32).normal_(0.0, std, generator=_gen(seed)).to(dtype)


def _slots(N, slots, spare, seed, keep=0.7):
    """slot_row [N, slots] with about `keep` of the slots on rows of their own, in no order; tokens 0, 3, 6 .. of every ten keep
    none; spare rows belong to nobody.  -> (slot_row, rows, [(token, slot, row)] tensors)"""
    g = _gen(seed)
    on = torch.rand((N, slots), device="cuda", generator=g) < keep
    on[torch.arange(N, device="cuda") % 10 == 3] = False
    t, s = torch.nonzero(on, as_tuple=True)
    rows = t.numel() + spare
    r = torch.randperm(rows, device="cuda", generator=g)[: t.numel()]
    slot_row = torch.full((N, slots), -1, device="cuda", dtype=torch.int32)
    slot_row[t, s] = r.int()
    return slot_row, rows, t, s, r


SHAPES = [(1, 1, 8), (1, 4, 64), (3, 2, 136), (33, 8, 256), (200, 3, 1024), (517, 6, 2048), (40, 2, 8192), (64, 33, 264), (20, 288, 128), (300, 1, 4104), (30, 70, 4096), (2, 3, 16384), (5, 40, 1032)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,slots,d", SHAPES + [(9000, 4, 512), (6000, 2, 2048)])
def test_combine_backward(cm, N, slots, d, dtype):
    slot_row, rows, t, s, r = _slots(N, slots, 5, N + slots)
    dy, y_perm = _normal((N, d), 1.0, dtype, 1), torch.full((rows, d), float("nan"), device="cuda", dtype=dtype)
    y_perm[r] = _normal((r.numel(), d), 1.0, dtype, 2)
    w = torch.full((rows,), float("nan"), device="cuda")
    w[r] = torch.rand((r.numel(),), device="cuda", generator=_gen(3))
    dy_perm, dweight = torch.full((rows, d), 9.0, device="cuda", dtype=dtype), torch.full((rows,), 9.0, device="cuda")
    cm.combine_backward(dy, y_perm, slot_row, w, dy_perm=dy_perm, dweight=dweight)
    g, y = dy.double()[t], y_perm.double()[r]
    ref = w.double()[r][:, None] * g
    close(dy_perm[r], ref, half_step(dtype) * ref.abs() * 1.01 + 2.0 ** -24 * ref.abs() + 1e-38)
    close(dweight[r], (g * y).sum(1), d * U2 * (g * y).abs().sum(1) + 1e-38)
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[r] = False
    assert bool((dy_perm[other] == 9).all()) and bool((dweight[other] == 9).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,slots,d", SHAPES + [(9000, 4, 512), (6000, 2, 2048)])
def test_permute_backward(cm, N, slots, d, dtype):
    slot_row, rows, t, s, r = _slots(N, slots, 5, N + slots)
    dx_perm = torch.full((rows, d), float("nan"), device="cuda", dtype=dtype)
    dx_perm[r] = _normal((r.numel(), d), 1.0, dtype, 1)
    a, b = _normal((N, d), 1.0, dtype, 2), _normal((N, d), 1.0, dtype, 3)
    base = torch.zeros((N, d), device="cuda", dtype=F64).index_add_(0, t, dx_perm.double()[r])
    size = torch.zeros((N, d), device="cuda", dtype=F64).index_add_(0, t, dx_perm.double()[r].abs())
    for add in (None, a, (a,), (a, b)):
        terms = () if add is None else (add,) if isinstance(add, torch.Tensor) else add
        ref, mag = base.clone(), size.clone()
        for v in terms:
            ref, mag = ref + v.double(), mag + v.double().abs()
        close(cm.permute_backward(dx_perm, slot_row, add=add), ref, rounded(ref, (slots + 2) * U2 * mag, dtype))
    want = cm.permute_backward(dx_perm, slot_row, add=(a, b))
    for into in (0, 1):                                               # in place of either addend
        pair = [a.clone(), b.clone()]
        got = cm.permute_backward(dx_perm, slot_row, add=pair, dx=pair[into])
        assert got.data_ptr() == pair[into].data_ptr() and torch.equal(got, want)


def _routing(cm, N, E, k, D, seed, gamma=0.8, skew=2.0):
    """Scores and lists as the route and drop stages leave them."""
    lg = _normal((N, E), 1.0, F32, seed) - skew * torch.linspace(0, 1, E, device="cuda")
    r = cm.route(None, None, None, k, logits_in=lg.contiguous())
    C = cm.capacity(N, E, k, gamma)
    dr = cm.expanded_drop(r["scores"], r["topk_idx"], C, D) if D else cm.token_drop(r["topk_score"], r["topk_idx"], E, C)
    return r, dr, cm.max_rows(N, E, k, max(D, 1), C, D > 0)


def _expert_of(r, dr, E, D):
    e = r["topk_idx"].long()
    if D:
        N, m = e.shape[0], E // D
        home = torch.arange(N, device="cuda") * D // N
        e = torch.cat([e, home[:, None] * m + torch.arange(m, device="cuda")], 1)
    return e


@pytest.mark.parametrize("N,E,k,D,d", [(1, 2, 1, 0, 16), (7, 8, 2, 0, 128), (130, 60, 4, 0, 2048), (1000, 64, 6, 0, 272), (500, 8, 2, 4, 4096),
                                       (300, 256, 8, 32, 2064), (900, 130, 6, 10, 48), (100, 64, 2, 1, 160),
                                       (70, 8, 2, 0, 16400), (3000, 16, 4, 0, 512), (40, 4, 1, 0, 40000)])
def test_permute_fp8(cm, N, E, k, D, d):
    r, dr, rows = _routing(cm, N, E, k, D, N)
    rows += 3
    x = _normal((N, d), 1.0, BF16, 1)
    q, sc = cm.quantize_rows(x)
    f16 = cm.permute(x, r["scores"], r["topk_idx"], dr["slot_row"], rows, D=D)
    out = dict(x_q=torch.full((rows, d), 2.0, device="cuda").to(cm.FP8), x_scale=torch.full((rows, (d + 127) // 128), 4.0, device="cuda").to(cm.SCALE),
               perm_token=torch.full((rows,), -7, device="cuda", dtype=torch.int32), perm_weight=torch.full((rows,), -7.0, device="cuda"))
    got = cm.permute_fp8(q, sc, r["scores"], r["topk_idx"], dr["slot_row"], rows, D=D, out=out)
    A = int(dr["offsets"][-1])
    t = f16["perm_token"][:A].long()
    assert torch.equal(got["perm_token"][:A], f16["perm_token"][:A]) and torch.equal(got["perm_weight"][:A], f16["perm_weight"][:A])
    assert torch.equal(got["x_q"].view(torch.uint8)[:A], q.view(torch.uint8)[t]) and torch.equal(got["x_scale"].view(torch.uint8)[:A], sc.view(torch.uint8)[t])
    assert bool((got["perm_token"][A:] == -7).all()) and bool((got["perm_weight"][A:] == -7).all())
    assert bool((got["x_q"][A:].float() == 2).all()) and bool((got["x_scale"][A:].float() == 4).all())


def test_permute_fp8_without_rows(cm):
    """Capacity zero: nobody keeps anything, no buffer is touched."""
    r = cm.route(None, None, None, 2, logits_in=_normal((40, 8), 1.0, F32, 2))
    q, sc = cm.quantize_rows(_normal((40, 64), 1.0, BF16, 1))
    none = torch.full((40, 2), -1, device="cuda", dtype=torch.int32)
    got = cm.permute_fp8(q, sc, r["scores"], r["topk_idx"], none, 0)
    assert got["x_q"].shape == (0, 64) and got["perm_token"].shape == (0,)


def test_sizes_of_other_types(cm):
    """NumPy integers are sizes, floats are not; a size past 32 bits is refused, not cut."""
    import numpy as np
    N, E = 40, 8
    r, dr, rows = _routing(cm, N, E, 2, 0, 1)
    q, sc = cm.quantize_rows(_normal((N, 64), 1.0, BF16, 1))
    args = (q, sc, r["scores"], r["topk_idx"], dr["slot_row"])
    want = cm.permute_fp8(*args, rows)
    A = int(dr["offsets"][-1])
    assert torch.equal(cm.permute_fp8(*args, np.int64(rows))["x_q"][:A].view(torch.uint8), want["x_q"][:A].view(torch.uint8))
    run = cm._binding().run
    y = torch.empty((N, 64), device="cuda")
    good = [y, None, y[0], N, 64, 0, 1e-6, None, y, None, None, None]
    assert run("capmoe_rms_norm", y, *good[:3], N, (1 << 32) + 64, *good[5:]) == cm.EUNSUPPORTED
    for at, bad in ((3, 4.0), (4, "64"), (4, None), (5, y), (6, None)):
        with pytest.raises(TypeError):
            run("capmoe_rms_norm", y, *good[:at], bad, *good[at + 1:])


@pytest.mark.parametrize("N,E,k,d,F", [(1, 8, 2, 2048, 1408), (128, 60, 4, 2048, 1408), (2000, 8, 2, 256, 512), (300, 8, 2, 264, 136), (3000, 4, 2, 1424, 256)])
def test_ffn_from_codes_is_the_ffn_from_rows(cm, N, E, k, d, F):
    """Norm with codes, codes sorted by expert, FFN from codes: the bits of norm, permute, FFN that quantises its rows."""
    x, w, res = _normal((N, d), 1.0, BF16, 1), _normal((d,), 1.0, BF16, 2), _normal((N, d), 1.0, BF16, 3)
    wg, wu, wd = (cm.quantize_weights(_normal(s, 0.05, BF16, 4 + i)) for i, s in enumerate([(E, F, d), (E, F, d), (E, d, F)]))
    n = cm.rms_norm(x, w, res, fp8=True)
    r, dr, rows = _routing(cm, N, E, k, 0, 5)
    perm = cm.permute(n["y"], r["scores"], r["topk_idx"], dr["slot_row"], rows)
    st = torch.zeros((128,), device="cuda", dtype=torch.int32)
    A = int(dr["offsets"][-1])
    for status in (st, None):
        if d % 16 == 0:
            p8 = cm.permute_fp8(n["q"], n["scale"], r["scores"], r["topk_idx"], dr["slot_row"], rows)
            rows8 = (p8["x_q"], p8["x_scale"])
        else:
            rows8 = cm.quantize_rows(perm["x_perm"])
        want = cm.grouped_ffn_fp8(perm["x_perm"], dr["offsets"], wg, wu, wd, dev_status=status)
        got = cm.grouped_ffn_fp8(rows8, dr["offsets"], wg, wu, wd, dev_status=status)
        assert torch.equal(got[:A], want[:A])
    assert int(st[0]) == cm.OK


def _route_ref(x, w, S, expert, slot_row, dweight, dscores, dtype):
    """dlogits, dx, dw, dbias in 64 bits with bounds."""
    S = S.double()
    N, E = S.shape
    dS = torch.zeros((N, E), device="cuda", dtype=F64)
    if dscores is not None:
        dS += dscores.double()
    mag = dS.abs()
    at = slot_row >= 0
    n = torch.nonzero(at)[:, 0]
    dS.index_put_((n, expert[at]), dweight.double()[slot_row[at].long()], accumulate=True)
    mag.index_put_((n, expert[at]), dweight.double()[slot_row[at].long()].abs(), accumulate=True)
    dot, dmag = (S * dS).sum(1, keepdim=True), (S * mag).sum(1, keepdim=True)
    dl = S * (dS - dot)
    edl = S * (U2 * mag + (E + 4) * U2 * dmag + U2 * (dS - dot).abs()) + 1e-38
    x, w = x.double(), w.double()
    into = edl if dtype == F32 else edl + 2.0 ** -16 * dl.abs() * 1.01      # as two bf16 numbers
    amp = dl.abs() + into
    terms = E if dtype == F32 else 2 * E
    dx, edx = dl @ w, into @ w.abs() + terms * U2 * (amp @ w.abs())
    dw, edw = dl.T @ x, into.T @ x.abs() + 2 * N * U2 * (amp.T @ x.abs())
    return (dl, edl), (dx, edx), (dw, edw), (dl.sum(0), edl.sum(0) + N * U2 * amp.sum(0))


def _check_route(cm, N, E, k, D, d, dtype, scores_grad, out_dtype, seed=0, gamma=0.8):
    r, dr, rows = _routing(cm, N, E, k, D, seed, gamma)
    x, w = _normal((N, d), 1.0, dtype, seed + 1), _normal((E, d), 0.1, dtype, seed + 2)
    dweight = torch.full((rows + 2,), float("nan"), device="cuda")
    A = int(dr["offsets"][-1])
    dweight[:A] = _normal((A,), 1.0, F32, seed + 3)
    dscores = None if scores_grad is None else _normal((N, E) if scores_grad == "each" else (E,), 0.3, F32, seed + 4)
    st = torch.zeros((128,), device="cuda", dtype=torch.int32)
    args = (x, w, r["scores"], r["topk_idx"], dr["slot_row"], dweight)
    got = cm.route_backward(*args, D=D, dscores=dscores, out_dtype=out_dtype, dev_status=st)
    ref = _route_ref(x, w, r["scores"], _expert_of(r, dr, E, D), dr["slot_row"], dweight, dscores, dtype)
    close(got["dlogits"], *ref[0])
    close(got["dx"], ref[1][0], rounded(*ref[1], dtype))
    assert got["dw"].dtype == (out_dtype or dtype)
    close(got["dw"], ref[2][0], rounded(*ref[2], got["dw"].dtype))
    close(got["dbias"], ref[3][0], rounded(*ref[3], F32))
    assert int(st[0]) == cm.OK
    return args, dict(D=D, dscores=dscores, out_dtype=out_dtype), got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,E,k,D,d", [(1, 2, 1, 0, 8), (1, 64, 8, 0, 2048), (5, 8, 2, 0, 64), (31, 7, 2, 0, 250), (517, 7, 2, 0, 250), (130, 60, 4, 0, 1408),
                                       (200, 16, 2, 4, 520), (129, 64, 6, 0, 2048), (300, 256, 8, 32, 136), (257, 130, 6, 10, 200),
                                       (1000, 33, 3, 0, 1032), (640, 128, 8, 16, 257), (2100, 8, 2, 0, 4096), (70, 1, 1, 0, 96), (400, 9, 3, 0, 33)])
def test_route_backward(cm, N, E, k, D, d, dtype):
    for i, (scores_grad, out) in enumerate(((None, None), ("each", F32), ("all", None))):
        _check_route(cm, N, E, k, D, d, dtype, scores_grad, out, seed=7 * i + N)


@pytest.mark.parametrize("N,E,k,D,d,dtype", [(9000, 64, 6, 0, 512, BF16), (20000, 8, 2, 0, 256, BF16), (5000, 256, 8, 32, 640, BF16), (6000, 16, 2, 2, 1032, F32),
                                             (7001, 60, 4, 0, 136, F32), (12345, 128, 8, 0, 264, BF16), (4000, 100, 2, 0, 77, BF16)])
def test_route_backward_of_many_tokens(cm, N, E, k, D, d, dtype):
    _check_route(cm, N, E, k, D, d, dtype, "all", None, seed=N)


@pytest.mark.parametrize("N,E,k,D,d,dtype", [(5001, 256, 8, 0, 130, F32), (3000, 200, 4, 0, 257, F32), (4100, 65, 3, 0, 1032, F32), (9001, 256, 8, 0, 259, BF16),
                                             (300, 9, 2, 0, 4099, F32), (300, 3, 1, 0, 4098, BF16), (129, 17, 2, 0, 127, BF16), (65, 129, 2, 0, 1, F32),
                                             (193, 70, 2, 0, 2, BF16), (257, 33, 2, 0, 63, BF16)])
def test_route_backward_of_rows_that_warps_lay_out(cm, N, E, k, D, d, dtype):
    """fp32 in passes of 64 experts; bf16 rows that start between words of four bytes; column slices of one and two columns."""
    _check_route(cm, N, E, k, D, d, dtype, "each", None, seed=N)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,E,d", [(1, 3, 40), (32, 8, 520), (33, 8, 520), (64, 60, 2048), (100, 256, 136), (128, 70, 131), (128, 16, 1032), (129, 16, 1032)])
def test_route_backward_of_few_tokens(cm, N, E, d, dtype):
    """Up to 128 tokens dW and dbias have no parts to join."""
    for out in (None, F32):
        _check_route(cm, N, E, min(E, 4), 0, d, dtype, "each", out, seed=N + d, gamma=4.0)


def test_route_backward_captured_and_on_two_streams(cm):
    """Every form of the products, twice in one graph with workspaces of its own, replayed while the same calls run on another stream."""
    calls = []
    for N, E, d, dtype in ((700, 200, 260, F32), (700, 30, 131, BF16), (900, 64, 512, BF16), (600, 6, 100, F32), (100, 70, 96, F32), (90, 70, 96, BF16)):
        args, kw, want = _check_route(cm, N, E, 2, 0, d, dtype, "all", None, seed=N)
        calls.append((args, kw, want))
    torch.cuda.synchronize()
    g, got = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(g):
        for _ in range(2):
            got += [cm.route_backward(*args, **kw) for args, kw, _ in calls]
    side, eager = torch.cuda.Stream(), []
    for _ in range(3):
        for r in got:
            for v in r.values():
                v.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        g.replay()
        eager = [cm.route_backward(*args, stream=side, **kw) for args, kw, _ in calls]
        torch.cuda.synchronize()
        for r, (_, _, want) in zip(got + eager, calls * 3):
            assert all(torch.equal(r[key], want[key]) for key in want)


def test_long_fp32_sums_of_dw_keep_their_precision(cm):
    """Sums of 9000 terms of one sign, 2300 of them in one thread block.  Sixteen additions a group of 256 tokens that cut off what
    fp32 does not hold (2^-23 of the sum, and as much where terms are aligned), then rounded ones: 9 groups, 4 ranges."""
    N, E, d = 9000, 20, 4096
    r, dr, rows = _routing(cm, N, E, 2, 0, 5, 4.0)
    x, w = _normal((N, d), 1.0, F32, 6).abs() + 0.1, _normal((E, d), 0.1, F32, 7)
    dscores = torch.zeros((E,), device="cuda")
    dscores[3] = 1.0                                                  # one expert's dlogits are positive, the others' negative
    got = cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], torch.zeros((rows,), device="cuda"), dscores=dscores)
    want = got["dlogits"].double().T @ x.double()
    close(got["dw"], want, (2 * 16 + 9 + 4 + 1) * U2 * want.abs())


def test_route_backward_of_large_and_small_numbers(cm):
    """Three bf16 numbers hold an fp32 number of any size: tokens near the largest, W_r far below one."""
    N, E, d = 300, 24, 96
    r, dr, rows = _routing(cm, N, E, 2, 0, 5, 4.0)
    x, w = _normal((N, d), 1.0, F32, 6) * 2.0 ** 121, _normal((E, d), 1.0, F32, 7) * 2.0 ** -90
    dweight = _normal((rows,), 2.0 ** -20, F32, 8)
    got = cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], dweight)
    ref = _route_ref(x, w, r["scores"], _expert_of(r, dr, E, 0), dr["slot_row"], dweight, None, F32)
    close(got["dx"], ref[1][0], rounded(*ref[1], F32))
    close(got["dw"], ref[2][0], rounded(*ref[2], F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_route_backward_without_tokens_and_without_rows(cm, dtype):
    E, d = 8, 64
    w = _normal((E, d), 1.0, dtype, 1)
    i32 = dict(device="cuda", dtype=torch.int32)
    dw, db = torch.full((E, d), 3.0, device="cuda", dtype=dtype), torch.full((E,), 3.0, device="cuda")
    cm.route_backward(torch.empty((0, d), device="cuda", dtype=dtype), w, torch.empty((0, E), device="cuda"), torch.empty((0, 2), **i32),
                      torch.empty((0, 2), **i32), torch.empty((0,), device="cuda"), out=dict(dw=dw, dbias=db))
    assert bool((dw == 0).all()) and bool((db == 0).all())
    r = cm.route(None, None, None, 2, logits_in=_normal((40, E), 1.0, F32, 2))
    none = torch.full((40, 2), -1, **i32)                             # capacity zero: nobody keeps anything
    got = cm.route_backward(_normal((40, d), 1.0, dtype, 3), w, r["scores"], r["topk_idx"], none, torch.empty((0,), device="cuda"))
    assert all(bool((got[k] == 0).all()) for k in got)
    dxp = cm.permute_backward(torch.empty((0, d), device="cuda", dtype=dtype), none)
    assert bool((dxp == 0).all())
    cm.combine_backward(_normal((40, d), 1.0, dtype, 4), torch.empty((0, d), device="cuda", dtype=dtype), none, torch.empty((0,), device="cuda"))


def test_route_backward_against_differences(cm):
    """f = sum of dweight over the kept pairs' scores + <dscores, scores>, in 64 bits as a function of x, W_r and bias, the kept
    set fixed: central differences of step s are off by s^2 (f's third derivatives are of the order of its first)."""
    N, E, k, d, s = 60, 8, 2, 48, 1e-4
    r, dr, rows = _routing(cm, N, E, k, 0, 3)
    x, w, b = _normal((N, d), 0.3, F32, 1), _normal((E, d), 0.3, F32, 2), _normal((E,), 0.3, F32, 4)
    route = cm.route(x, w, b, k)
    dr = cm.token_drop(route["topk_score"], route["topk_idx"], E, cm.capacity(N, E, k, 0.8))
    dweight, dsc = _normal((rows,), 1.0, F32, 5), _normal((N, E), 0.5, F32, 6)
    got = cm.route_backward(x, w, route["scores"], route["topk_idx"], dr["slot_row"], dweight, dscores=dsc)
    at = dr["slot_row"] >= 0
    n, e, v = torch.nonzero(at)[:, 0], route["topk_idx"].long()[at], dweight.double()[dr["slot_row"][at].long()]

    def f(x, w, b):
        S = torch.softmax(x @ w.T + b, 1)
        return (S[n, e] * v).sum() + (S * dsc.double()).sum()

    p = [x.double(), w.double(), b.double()]
    for seed in range(3):
        for i, key in enumerate(("dx", "dw", "dbias")):
            dirn = _normal(p[i].shape, 1.0, F32, 30 + seed).double()
            up, down = list(p), list(p)
            up[i], down[i] = p[i] + s * dirn, p[i] - s * dirn
            want, g = (f(*up) - f(*down)) / (2 * s), got[key].double()
            # a direction moves a logit by up to |x| |dirn| ~ 10: third derivatives up to 1000 times the first;
            # the scores themselves are fp32 (d * 2^-23 of a logit's terms)
            assert abs(want - (g * dirn).sum()) <= (1000 * s * s + 8 * N * U2) * (g * dirn).abs().sum() + 1e-8


def test_nan_of_one_token_stays_out_of_the_others(cm):
    for E, d, dtype in ((60, 136, BF16), (8, 250, F32), (8, 256, BF16)):
        (x, w, S, idx, sr, dwt), kw, clean = _check_route(cm, 150, E, 2, 0, d, dtype, None, None, seed=2, gamma=4.0)
        dwt = dwt.clone()
        dwt[int(sr[11, 0])] = float("nan")
        got = cm.route_backward(x, w, S, idx, sr, dwt)
        ok = torch.arange(150, device="cuda") != 11
        assert torch.equal(got["dx"][ok], clean["dx"][ok]) and torch.equal(got["dlogits"][ok], clean["dlogits"][ok])
        assert bool(got["dx"][11].isnan().all()) and bool(got["dbias"].isnan().all())


def test_rows_outside_the_buffers_count_as_none(cm):
    N, d = 50, 64
    slot_row, rows, t, s, r = _slots(N, 4, 0, 1)
    far = slot_row.clone()
    far[slot_row < 0] = rows + 1000
    far[0, 0] = 2 ** 31 - 1
    near = slot_row.clone()
    near[0, 0] = -1
    dy, yp = _normal((N, d), 1.0, BF16, 1), _normal((rows, d), 1.0, BF16, 2)
    w = torch.rand((rows,), device="cuda")
    out = []
    for sr in (far, near):
        a, b = torch.zeros((rows, d), device="cuda", dtype=BF16), torch.zeros((rows,), device="cuda")
        cm.combine_backward(dy, yp, sr, w, dy_perm=a, dweight=b)
        out.append((a, b, cm.permute_backward(yp, sr)))
    assert all(torch.equal(u, v) for u, v in zip(*out))


def test_rows_past_32_bit_offsets(cm):
    N, slots, d = 64, 4, 4096
    rows = (1 << 31) // d + 5000
    g = _gen(1)
    r = (rows - 1 - torch.randperm(4000, device="cuda", generator=g)[: N * slots]).view(N, slots)
    small = torch.argsort(torch.argsort(r.flatten())).view(N, slots).int()                # the same rows, packed
    big = torch.empty((rows, d), device="cuda", dtype=BF16)
    packed = _normal((N * slots, d), 1.0, BF16, 2)
    big[r.flatten()] = packed[small.flatten().long()]
    dy, wp = _normal((N, d), 1.0, BF16, 3), torch.rand((N * slots,), device="cuda", generator=g)
    w = torch.zeros((rows,), device="cuda")
    w[r.flatten()] = wp[small.flatten().long()]
    a, b = cm.combine_backward(dy, big, r.int().contiguous(), w)
    a0, b0 = cm.combine_backward(dy, packed, small.contiguous(), wp)
    assert torch.equal(a[r.flatten()], a0[small.flatten().long()]) and torch.equal(b[r.flatten()], b0[small.flatten().long()])
    assert torch.equal(cm.permute_backward(big, r.int().contiguous()), cm.permute_backward(packed, small.contiguous()))


def test_captured_replayed_and_on_another_stream(cm):
    N, E, k, d = 600, 64, 6, 1024
    r, dr, rows = _routing(cm, N, E, k, 0, 1)
    x, w, dy = _normal((N, d), 1.0, BF16, 1), _normal((E, d), 0.1, BF16, 2), _normal((N, d), 1.0, BF16, 3)
    yp, q = _normal((rows, d), 1.0, BF16, 4), cm.quantize_rows(x)
    wp = torch.rand((rows,), device="cuda")
    A = int(dr["offsets"][-1])

    def run(stream=None):
        a, b = cm.combine_backward(dy, yp, dr["slot_row"], wp, stream=stream)
        o = cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], b, stream=stream)
        p = cm.permute_fp8(*q, r["scores"], r["topk_idx"], dr["slot_row"], rows, stream=stream)
        return [a[:A], b[:A], cm.permute_backward(a, dr["slot_row"], add=o["dx"], stream=stream), *o.values(), p["x_q"][:A].view(torch.uint8),
                p["x_scale"][:A].view(torch.uint8)]

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = run(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out))
    for seed in (50, 51):
        dy.copy_(_normal((N, d), 1.0, BF16, seed))
        for g, _ in graphs:
            g.replay()
        now = run()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, now))


def test_two_streams_at_once_give_what_one_gives(cm):
    cases = [(900, 64, 6, 1024, BF16), (700, 8, 2, 520, BF16)]
    calls = []
    for N, E, k, d, dt in cases:
        r, dr, rows = _routing(cm, N, E, k, 0, N)
        x, w, dwt = _normal((N, d), 1.0, dt, 1), _normal((E, d), 0.1, dt, 2), _normal((rows,), 1.0, F32, 3)
        calls.append((x, w, r["scores"], r["topk_idx"], dr["slot_row"], dwt))
    want = [cm.route_backward(*c) for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(30):
        for i, c in enumerate(calls):
            got[i].append(cm.route_backward(*c, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(g[k], want[i][k]) for k in g)


def test_guard_bands(cm):
    """Nothing around the outputs and the workspace is written."""
    for dtype, E, d, N in ((BF16, 60, 136, 77), (BF16, 8, 72, 33), (F32, 7, 36, 33), (BF16, 16, 33, 50), (BF16, 130, 264, 300)):
        r, dr, rows = _routing(cm, N, E, 2, 0, 1)
        held = []

        def buf(shape, t):
            n = 1
            for v in shape:
                n *= v
            size = n * torch.empty((), dtype=t).element_size()
            raw = torch.full((256 + size + 256,), 0x5A, device="cuda", dtype=torch.uint8)
            held.append((raw, size))
            return raw[256:256 + size].view(t).view(shape)

        x, w, dwt = _normal((N, d), 1.0, dtype, 1), _normal((E, d), 0.1, dtype, 2), _normal((rows,), 1.0, F32, 3)
        cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], dwt,
                          out=dict(dlogits=buf((N, E), F32), dx=buf((N, d), dtype), dw=buf((E, d), F32), dbias=buf((E,), F32)),
                          ws=buf((cm.route_backward_workspace_bytes(N, d, E, dtype),), torch.uint8))
        if d * x.element_size() % 16 == 0:
            yp = _normal((rows, d), 1.0, dtype, 4)
            cm.combine_backward(x, yp, dr["slot_row"], dwt, dy_perm=buf((rows, d), dtype), dweight=buf((rows,), F32))
            cm.permute_backward(yp, dr["slot_row"], dx=buf((N, d), dtype))
        for raw, size in held:
            assert bool((raw[:256] == 0x5A).all()) and bool((raw[256 + size:] == 0x5A).all())


def test_the_same_bits_every_time(cm):
    args, kw, want = _check_route(cm, 5000, 64, 6, 0, 1024, BF16, "all", F32, seed=1)
    for _ in range(20):
        got = cm.route_backward(*args, **kw)
        assert all(torch.equal(got[k], want[k]) for k in want)


# ------------------------------------------------------------------------------------------- the whole layer
def _layer(cm, N, d, F, E, k, D, mode, dtype, shared, seed=0, **kw):
    x, wr, b = _normal((N, d), 1.0, dtype, seed), _normal((E, d), 0.2, dtype, seed + 1), _normal((E,), 0.2, F32, seed + 2)
    ws = [_normal(s, 0.15, dtype, seed + 3 + i) for i, s in enumerate([(E, F, d), (E, F, d), (E, d, F)])]
    sh = None if not shared else tuple(_normal(s, 0.15, dtype, seed + 9 + i) for i, s in enumerate([(1, F, d), (1, F, d), (1, d, F)]))
    layer = cm.MoELayer(x, wr, b, *ws, k=k, D=D, mode=mode, shared=sh, **kw)
    layer.forward()
    return layer, _normal((N, d), 1.0, dtype, seed + 20)


MODES = [("nodrop", {}), ("token_drop", {}), ("expanded_drop", {}), ("device_token_drop", {}), ("device_expanded_drop", {}),
         ("token_drop", dict(metric="order")), ("expanded_drop", dict(max_experts=3))]


@pytest.mark.parametrize("mode,kw", MODES)
def test_layer_gradients(cm, mode, kw):
    """fp32, against the formulas in 64 bits from what the forward left (scores, kept rows, y_perm).  dy_perm has one rounding
    (2^-24), less than a tenth of what the sums of the products that read it are allowed: their bounds times 1.1."""
    N, d, F, E, k, D = 120, 64, 48, 8, 2, 4
    layer, dy = _layer(cm, N, d, F, E, k, D, mode, F32, shared=True, gamma=0.9, **kw)
    t = layer.t
    dsc = _normal((E,), 0.2, F32, 40)
    g = layer.backward(dy, dscores=dsc)
    layer.check_device_status()
    A = int(t["expert_offsets"][-1])
    off = t["expert_offsets"].tolist()
    tok, wgt = t["perm_token"][:A].long(), t["perm_weight"][:A].double()
    dyp, yp = wgt[:, None] * dy.double()[tok], t["y_perm"][:A].double()
    dweight = (dy.double()[tok] * yp).sum(1)
    edw = d * U2 * (dy.double()[tok] * yp).abs().sum(1)
    dx, edx = torch.zeros((N, d), device="cuda", dtype=F64), torch.zeros((N, d), device="cuda", dtype=F64)
    for e in range(E):
        rows = slice(off[e], off[e + 1])
        ref = ffn_gradient(t["x"].double()[tok[rows]], dyp[rows], t["w_gate"][e].double(), t["w_up"][e].double(), t["w_down"][e].double(), F32)
        for key in ("dw_gate", "dw_up", "dw_down"):
            close(g[key][e], ref[key][0], 1.1 * ref[key][1])
        dx.index_add_(0, tok[rows], ref["dx"][0])
        edx.index_add_(0, tok[rows], 1.1 * ref["dx"][1] + (layer.slots + 2) * U2 * ref["dx"][0].abs())
    sh = ffn_gradient(t["x"].double(), dy.double(), t["ws_gate"][0].double(), t["ws_up"][0].double(), t["ws_down"][0].double(), F32)
    for key, name in (("dw_gate", "dws_gate"), ("dw_up", "dws_up"), ("dw_down", "dws_down")):
        close(g[name][0], *sh[key])
    # the router: the kept pairs' experts from the rows, dweight's own error carried through
    expert = torch.searchsorted(t["expert_offsets"][1:].long().contiguous(), torch.arange(A, device="cuda"), right=True)
    S = t["scores"].double()
    dS, mag = dsc.double().repeat(N, 1), dsc.double().abs().repeat(N, 1)
    dS.index_put_((tok, expert), dweight, accumulate=True)
    mag.index_put_((tok, expert), dweight.abs(), accumulate=True)
    edS = torch.zeros_like(dS).index_put_((tok, expert), edw, accumulate=True)
    dl = S * (dS - (S * dS).sum(1, keepdim=True))
    edl = S * (edS + (S * edS).sum(1, keepdim=True) + U2 * mag + (E + 4) * U2 * (S * mag).sum(1, keepdim=True)) + 2 * U2 * dl.abs() + 1e-38
    x, wr = t["x"].double(), t["w_router"].double()
    amp = dl.abs() + edl
    close(g["dlogits"], dl, edl)
    close(g["dw_router"], dl.T @ x, edl.T @ x.abs() + 2 * N * U2 * (amp.T @ x.abs()))
    close(g["dbias"], dl.sum(0), edl.sum(0) + N * U2 * amp.sum(0))
    rdx, erdx = dl @ wr, edl @ wr.abs() + (E + 1) * U2 * (amp @ wr.abs())
    total = dx + sh["dx"][0] + rdx
    close(g["dx"], total, edx + sh["dx"][1] + erdx + (layer.slots + 3) * U2 * (dx.abs() + sh["dx"][0].abs() + rdx.abs()))


def test_layer_gradients_are_those_of_the_stages_in_bf16(cm):
    layer, dy = _layer(cm, 900, 256, 128, 64, 6, 8, "expanded_drop", BF16, shared=False)
    t = layer.t
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = layer.backward(dy, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    g = layer.backward(dy)
    layer.check_device_status()
    assert all(torch.equal(g[k], other[k]) for k in g)
    dyp, dwt = cm.combine_backward(dy, t["y_perm"], t["slot_row"], t["perm_weight"])
    dxp, dwg, dwu, dwd = cm.grouped_ffn_backward(t["x_perm"], dyp, t["expert_offsets"], t["w_gate"], t["w_up"], t["w_down"])
    r = cm.route_backward(t["x"], t["w_router"], t["scores"], t["topk_idx"], t["slot_row"], dwt, D=8)
    want = dict(dx=cm.permute_backward(dxp, t["slot_row"], add=r["dx"]), dw_router=r["dw"], dbias=r["dbias"], dw_gate=dwg, dw_up=dwu, dw_down=dwd)
    for k, v in want.items():
        assert torch.equal(g[k], v), k


def test_a_step_of_norm_and_layer_against_differences(cm):
    """Norm, router, experts and combine as a training step runs them: the gradient of <dy, y> + <dh, h> by x and by the norm's
    weight, against central differences of the same function in 64 bits with the kept set and the paths' weights recomputed."""
    N, d, F, E, k = 40, 32, 24, 4, 2
    x, res, wn = _normal((N, d), 1.0, F32, 1), _normal((N, d), 1.0, F32, 2), 1 + _normal((d,), 0.1, F32, 3)
    n = cm.rms_norm(x, wn, res)
    wr, b = _normal((E, d), 0.2, F32, 5), _normal((E,), 0.2, F32, 6)
    ws = [_normal(s, 0.2, F32, 7 + i) for i, s in enumerate([(E, F, d), (E, F, d), (E, d, F)])]
    layer = cm.MoELayer(n["y"], wr, b, *ws, k=k, D=1, mode="token_drop", gamma=0.9)
    layer.forward()
    dy, dh = _normal((N, d), 1.0, F32, 11), _normal((N, d), 1.0, F32, 12)
    g = layer.backward(dy)
    dx, dwn = cm.rms_norm_backward(g["dx"], n["h"], wn, n["rstd"], dh=dh)
    sr = layer.t["slot_row"]
    at = sr >= 0
    tok, e = torch.nonzero(at)[:, 0], layer.t["topk_idx"].long()[at]

    def f(x, wn):
        h = x + res.double()
        y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * wn
        S = torch.softmax(y @ wr.double().T + b.double(), 1)
        total = (h * dh.double()).sum()
        for i in range(E):
            t = tok[e == i]
            gate, up = y[t] @ ws[0][i].double().T, y[t] @ ws[1][i].double().T
            out = (gate * torch.sigmoid(gate) * up) @ ws[2][i].double().T
            total = total + (S[t, i][:, None] * out * dy.double()[t]).sum()
        return total

    x64, w64 = x.double(), wn.double()
    for seed in range(3):
        v, u = _normal((N, d), 1.0, F32, 60 + seed).double(), _normal((d,), 1.0, F32, 70 + seed).double()
        for s, grad, dirn, up, down in ((1e-4, dx, v, lambda s: f(x64 + s * v, w64), lambda s: f(x64 - s * v, w64)),
                                        (1e-4, dwn, u, lambda s: f(x64, w64 + s * u), lambda s: f(x64, w64 - s * u))):
            want = (up(s) - down(s)) / (2 * s)
            size = (grad.double() * dirn).abs().sum()
            # Richardson: the differences' own error from a second step; the chain's fp32 sums: 4 products of at most d terms
            coarse = (up(2 * s) - down(2 * s)) / (4 * s)
            assert abs(want - (grad.double() * dirn).sum()) <= abs(want - coarse) + 40 * d * U2 * size
