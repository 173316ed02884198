"""8-bit expert products: quantisers bit for bit, products and the FFN against 64-bit definitions."""
import pytest
import torch

import grouped_ref as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def cm():
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _normal(shape, std, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(0, std, generator=g)


def _spans(counts):
    o = 0
    for e, c in enumerate(counts):
        yield e, slice(o, o + c)
        o += c


def _block(cm):
    return torch.zeros(cm.FFN_STATUS_WORDS, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 128), (3, 8), (5, 127), (17, 129), (64, 2048), (9, 1000), (300, 136), (2, 4104)])
def test_quantize_rows(cm, rows, d, dtype):
    x = _normal((rows, d), 1.0, dtype, 1)
    x[:, ::37] *= 60
    x[0, : min(d, 128)] = 0                                    # a block of zeros
    q, s = cm.quantize_rows(x)
    assert R.same_codes(q, s, R.quantized(x.double(), 1))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,n,d", [(1, 1, 1), (2, 128, 128), (3, 127, 129), (2, 200, 264), (1, 8, 1000), (5, 136, 40)])
def test_quantize_weights(cm, E, n, d, dtype):
    w = _normal((E, n, d), 0.02, dtype, 2)
    q, s = cm.quantize_weights(w)
    for e in range(E):
        assert R.same_codes(q[e], s[e], R.quantized(w[e].double(), 128))


def test_quantize_borders(cm):
    """Maxima on, just above and just below 448 * 2^e; ties between two codes; the smallest and the largest numbers."""
    x = torch.zeros((12, 128), device="cuda", dtype=F32)
    top = torch.tensor([448.0, 449.0, 447.0, 0.875, 0.8750001, 1.0, 3.0e38, 1e-38, 1e-45, 2.0 ** -119, 240.0, 7.0], device="cuda")
    x[:, 0] = top
    x[:, 1:18] = top[:, None] * torch.linspace(-1, 1, 17, device="cuda")
    x[:, 20] = top * 17 / 448                                  # halfway between 16 and 18
    x[:, 21] = top * 19 / 448                                  # halfway between 18 and 20
    q, s = cm.quantize_rows(x)
    assert R.same_codes(q, s, R.quantized(x.double(), 1))
    assert s.view(torch.uint8)[0, 0] == 127 and s.view(torch.uint8)[1, 0] == 128 and s.view(torch.uint8)[8, 0] == 0


def test_quantize_smallest_bf16_numbers(cm):
    """Maxima and values below the smallest normal number, and blocks whose scale is clamped at 2^-127."""
    x = torch.zeros((4, 256), device="cuda", dtype=BF16)
    for i, top in enumerate((2.0 ** -118, 2.0 ** -126, 2.0 ** -133, 1.0)):
        x[i] = (torch.linspace(-1, 1, 256, device="cuda", dtype=torch.float64) * top).to(BF16)
    x[3, 1::2] = (torch.linspace(-1, 1, 128, device="cuda", dtype=torch.float64) * 2.0 ** -127).to(BF16)
    q, s = cm.quantize_rows(x)
    assert R.same_codes(q, s, R.quantized(x.double(), 1))


def test_quantize_largest_numbers(cm):
    x = torch.zeros((3, 128), device="cuda", dtype=F32)
    x[:, ::3] = torch.tensor([3.4e38, -3.0e38, 2.0 ** 127], device="cuda")[:, None]
    x[:, 1::3] = 2.0e38 * torch.linspace(-1, 1, 43, device="cuda")
    q, s = cm.quantize_rows(x)
    assert bool(torch.isfinite(R.decoded(q, s, 1)).all()) and R.same_codes(q, s, R.quantized(x.double(), 1))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_block_with_a_nan_or_an_infinity_becomes_nan(cm, bad):
    x = _normal((4, 300), 1.0, BF16, 3)
    x[2, 130] = bad
    q, s = cm.quantize_rows(x)
    v = R.decoded(q, s, 1)
    assert bool(torch.isnan(v[2, 128:256]).all()) and int(torch.isnan(v).sum()) == 128
    w = _normal((1, 200, 300), 1.0, BF16, 3)
    w[0, 150, 299] = bad
    q, s = cm.quantize_weights(w)
    v = R.decoded(q[0], s[0], 128)
    assert bool(torch.isnan(v[128:, 256:]).all()) and int(torch.isnan(v).sum()) == 72 * 44


def test_rows_behind_the_last_expert_are_not_quantised(cm):
    x = _normal((40, 256), 1.0, BF16, 4)
    out = (torch.full((40, 256), 2.0, device="cuda").to(cm.FP8), torch.full((40, 2), 4.0, device="cuda").to(cm.SCALE))
    q, s = cm.quantize_rows(x, R.offsets_of([10, 0, 13]), out=out)
    assert bool((q[23:].float() == 2).all()) and bool((s[23:].float() == 4).all())
    assert R.same_codes(q[:23], s[:23], R.quantized(x[:23].double(), 1))


COUNTS = {"one row": [1], "all empty": [0, 0], "few": [1, 0, 3, 2, 0, 5, 1], "borders": [16, 15, 17, 0, 64, 63, 65, 128, 127, 129, 1],
          "long": [0, 700, 1, 300, 0], "longer": [1100, 37, 2051], "many": [(7 * e) % 23 for e in range(256)]}


def _mm(cm, counts, d, n, status=True):
    off = R.offsets_of(counts)
    A, E = sum(counts), len(counts)
    rows = A + 4
    x = _normal((rows, d), 1.0, BF16, 5)
    x *= torch.exp2(torch.randint(-6, 7, (rows, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(6)).float()).to(BF16)
    w = _normal((E, n, d), 0.05, BF16, 7)
    w *= torch.exp2((torch.arange(n, device="cuda") // 128 % 5 - 2).float())[:, None].to(BF16)     # blocks of different scales
    w *= torch.exp2((torch.arange(d, device="cuda") // 128 % 7 - 3).float()).to(BF16)
    xq, xs = cm.quantize_rows(x)
    xq.view(torch.uint8)[A:] = 0x7f                            # NaN codes behind the last expert's rows
    wq, ws = cm.quantize_weights(w)
    y = torch.full((rows, n), 3.0, device="cuda", dtype=BF16)
    st = _block(cm) if status else None
    cm.grouped_mm_fp8(xq, xs, off, wq, ws, y=y, dev_status=st)
    assert bool((y[A:] == 3).all())
    for e, r in _spans(counts):
        R.close(y[r], *R.product(R.decoded(xq[r], xs[r], 1), R.decoded(wq[e], ws[e], 128), BF16))
    assert st is None or int(st[0]) == 0


@pytest.mark.parametrize("d,n", [(128, 128), (256, 512), (1024, 256), (16, 16), (144, 272), (400, 48), (640, 1040), (33, 65), (250, 130), (1, 7)])
@pytest.mark.parametrize("name", ["one row", "all empty", "few", "borders"])
def test_product(cm, name, d, n):
    _mm(cm, COUNTS[name], d, n)


@pytest.mark.parametrize("d,n", [(256, 512), (144, 272), (1936, 400), (400, 48)])
@pytest.mark.parametrize("name", ["long", "longer", "many"])
def test_product_long_and_many_segments(cm, name, d, n):
    _mm(cm, COUNTS[name], d, n)


@pytest.fixture
def forced(cm):
    yield lambda name: cm.debug_ffn_variant(name)
    cm.debug_ffn_variant("auto")


def test_product_without_a_status_block(cm):
    _mm(cm, COUNTS["borders"], 384, 320, status=False)
    _mm(cm, COUNTS["longer"], 384, 320, status=False)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_scales_need_no_alignment(cm, shift):
    """Scales are bytes: a scale tensor may start anywhere."""
    counts, d, n = [40, 0, 150], 1024, 256
    off = R.offsets_of(counts)
    x, w = _normal((190, d), 1.0, BF16, 21), _normal((3, n, d), 0.05, BF16, 22)
    (xq, xs), (wq, ws) = cm.quantize_rows(x), cm.quantize_weights(w)

    def moved(s):
        raw = torch.zeros(s.numel() + 4, device="cuda", dtype=torch.uint8)
        raw[shift:shift + s.numel()] = s.view(torch.uint8).reshape(-1)
        return raw[shift:shift + s.numel()].view(cm.SCALE).view(s.shape)

    y = cm.grouped_mm_fp8(xq, xs, off, wq, ws)
    assert torch.equal(cm.grouped_mm_fp8(xq, moved(xs), off, wq, moved(ws)), y)


def test_a_nan_row_stays_a_row(cm):
    counts = [40, 0, 90]
    off = R.offsets_of(counts)
    x, w = _normal((130, 256), 1.0, BF16, 8), _normal((3, 128, 256), 0.05, BF16, 9)
    x[77, 5] = float("inf")
    y = cm.grouped_mm_fp8(*cm.quantize_rows(x), off, *cm.quantize_weights(w))
    nan = torch.isnan(y)
    assert bool(nan[77].all()) and int(nan.sum()) == 128 and bool(torch.isfinite(y[:77].float()).all())


FFN_CASES = [([1], 128, 128), ([0, 0], 128, 128), ([3, 0, 70, 129, 1], 256, 192), ([65, 64, 17], 144, 80),
                                        ([5, 9, 0, 33], 33, 45), ([300, 0, 513], 256, 320), ([1] * 60, 256, 384), ([1100, 1400], 384, 256)]


@pytest.mark.parametrize("form", ["auto", "pair", "short"])
@pytest.mark.parametrize("counts,d,F", FFN_CASES)
def test_ffn(cm, forced, counts, d, F, form):
    forced(form)
    off = R.offsets_of(counts)
    A, E = sum(counts), len(counts)
    rows = A + 3
    x = _normal((rows, d), 1.0, BF16, 10)
    x[A:] = float("nan")
    w = [cm.quantize_weights(_normal(s, 0.08, BF16, 11 + i)) for i, s in enumerate(((E, F, d), (E, F, d), (E, d, F)))]
    y = torch.full((rows, d), 3.0, device="cuda", dtype=BF16)
    st = _block(cm)
    cm.grouped_ffn_fp8(x, off, *w, y_perm=y, dev_status=st)
    assert int(st[0]) == 0 and bool((y[A:] == 3).all())
    for e, r in _spans(counts):
        if r.start == r.stop:
            continue
        wg, wu, wd = (R.decoded(q[e], s[e], 128) for q, s in w)
        _, _, h, eh = R.swiglu(R.values(x[r].double(), 1), wg, wu)
        hq, ehq = R.quantized_hidden(h, eh)
        ref, e1 = R.product(hq, wd)
        R.close(y[r], ref, R.rounded(ref, e1 * 1.2 + ehq @ wd.abs().T, BF16))


def test_ffn_follows_the_16_bit_ffn(cm):
    """The 8-bit FFN of a layer's own rows next to grouped_ffn: the quantisers' errors are independent and at most
    2^-4 of a value (about 2.5 % rms), four of them on the way to an output: below 10 % of the outputs' norm."""
    from paper_2503_05066_b200 import synth
    cfg = synth.CONFIGS["olmoe"].with_(N=400, d=256, F=256, E=8, k=2, D=2)
    inp = synth.make_layer_inputs(cfg)
    x, wr, wg, wu, wd = (t.cuda() for t in (inp.x, inp.w_router, inp.w_gate, inp.w_up, inp.w_down))
    r = cm.route(x, wr, None, cfg.k)
    C = cm.capacity(cfg.N, cfg.E, cfg.k, 1.0)
    dr = cm.token_drop(r["topk_score"], r["topk_idx"], cfg.E, C)
    A_max = cm.max_rows(cfg.N, cfg.E, cfg.k, cfg.D, C, False)
    p = cm.permute(x, r["scores"], r["topk_idx"], dr["slot_row"], A_max)
    y16 = cm.grouped_ffn(p["x_perm"], dr["offsets"], wg, wu, wd)
    y8 = cm.grouped_ffn_fp8(p["x_perm"], dr["offsets"], *(cm.quantize_weights(w) for w in (wg, wu, wd)),
                            y_perm=torch.zeros_like(y16))
    out = cm.combine(y8, dr["slot_row"], p["perm_weight"])
    ref = cm.combine(y16, dr["slot_row"], p["perm_weight"])
    assert float((y8 - y16).float().norm() / y16.float().norm()) < 0.1
    assert float((out - ref).float().norm() / ref.float().norm()) < 0.1


def test_captured_and_replayed(cm):
    counts = [70, 0, 5, 200]
    off = R.offsets_of(counts)
    x = _normal((275, 256), 1.0, BF16, 14)
    w = [cm.quantize_weights(_normal(s, 0.08, BF16, 15 + i)) for i, s in enumerate(((4, 384, 256), (4, 384, 256), (4, 256, 384)))]
    q = (torch.zeros((275, 256), device="cuda").to(cm.FP8), torch.zeros((275, 2), device="cuda").to(cm.SCALE))
    y, z = torch.zeros((275, 384), device="cuda", dtype=BF16), torch.zeros((275, 256), device="cuda", dtype=BF16)
    ws = torch.empty(cm.ffn_fp8_workspace_bytes(275, 256, 384), device="cuda", dtype=torch.uint8)
    st = _block(cm)

    def calls():
        cm.quantize_rows(x, off, out=q)
        cm.grouped_mm_fp8(*q, off, *w[0], y=y, dev_status=st)
        cm.grouped_ffn_fp8(x, off, *w, y_perm=z, ws=ws, dev_status=st)

    calls()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        calls()
    x.copy_(_normal((275, 256), 1.0, BF16, 20))
    off.copy_(R.offsets_of([0, 100, 75, 100]))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    got = y.clone(), z.clone()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    assert torch.equal(got[0], y) and torch.equal(got[1], z) and int(st[0]) == 0


def test_guard_bands(cm):
    G = 4096
    for d, n in ((144, 272), (33, 65)):
        counts = [37, 0, 130]
        off = R.offsets_of(counts)
        x, w = _normal((167, d), 1.0, BF16, 1), _normal((3, n, d), 0.1, BF16, 2)
        shapes = [((167, d), cm.FP8), ((167, -(-d // 128)), cm.SCALE), ((3, n, d), cm.FP8), ((3, -(-n // 128), -(-d // 128)), cm.SCALE),
                  ((167, n), BF16)]
        raws, views = [], []
        for shape, dt in shapes:
            size = 2 if dt == BF16 else 1
            for v in shape:
                size *= v
            raw = torch.full((size + 2 * G,), 0xA5, device="cuda", dtype=torch.uint8)
            raws.append(raw)
            views.append(raw[G:G + size].view(dt).view(shape))
        cm.quantize_rows(x, out=(views[0], views[1]))
        cm.quantize_weights(w, out=(views[2], views[3]))
        cm.grouped_mm_fp8(views[0], views[1], off, views[2], views[3], y=views[4])
        torch.cuda.synchronize()
        for raw in raws:
            assert bool((raw[:G] == 0xA5).all()) and bool((raw[-G:] == 0xA5).all())


def test_two_streams_at_once_give_what_one_gives(cm):
    counts = [300, 0, 77, 1200, 5, 640]
    off = R.offsets_of(counts)
    A = sum(counts)
    x = _normal((A, 512), 1.0, BF16, 40)
    w = [cm.quantize_weights(_normal(s, 0.08, BF16, 41 + i)) for i, s in enumerate(((6, 768, 512), (6, 768, 512), (6, 512, 768)))]

    def calls(st):
        q = cm.quantize_rows(x, off)
        return cm.grouped_mm_fp8(*q, off, *w[0], dev_status=st), cm.grouped_ffn_fp8(x, off, *w, dev_status=st)

    want = calls(_block(cm))
    torch.cuda.synchronize()
    streams, blocks = [torch.cuda.Stream() for _ in range(3)], [_block(cm) for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for s, b in zip(streams, blocks):
            with torch.cuda.stream(s):
                got.append(calls(b))
        torch.cuda.synchronize()
        for g in got:
            assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])
    assert all(int(b[0]) == 0 for b in blocks)


def test_matrices_past_32_bit_offsets(cm):
    rows, d = 1_100_000, 2048
    x = torch.empty((rows, d), device="cuda", dtype=BF16)
    x[:] = _normal((1, d), 1.0, BF16, 50)
    x[-400:] = _normal((400, d), 1.0, BF16, 51)
    q, s = cm.quantize_rows(x)
    assert R.same_codes(q[-400:], s[-400:], R.quantized(x[-400:].double(), 1))
    assert R.same_codes(q[rows // 2:][:8], s[rows // 2:][:8], R.quantized(x[rows // 2:][:8].double(), 1))
    wq, ws = cm.quantize_weights(_normal((2, 64, d), 0.05, BF16, 52))
    off = R.offsets_of([rows - 400, 400])
    y = cm.grouped_mm_fp8(q, s, off, wq, ws)
    for e, r in ((0, slice(rows - 500, rows - 400)), (1, slice(rows - 400, rows))):
        R.close(y[r], *R.product(R.decoded(q[r], s[r], 1), R.decoded(wq[e], ws[e], 128), BF16))


def test_a_call_on_another_stream_keeps_its_workspace(cm):
    """The call is queued behind 10 ms of waiting on its own stream; meanwhile the current stream takes memory of the
    workspace's size and writes to it.  Workspaces made inside a call belong to the call's stream, so nothing changes."""
    counts, d, F = [70, 0, 5, 200], 256, 384
    off = R.offsets_of(counts)
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s, dtype: torch.randn(s, device="cuda", generator=g).mul_(0.3).to(dtype)
    x8, w8 = rand(275, d, dtype=torch.bfloat16), [cm.quantize_weights(rand(4, *s, dtype=torch.bfloat16)) for s in ((F, d), (F, d), (d, F))]
    x, dy = rand(275, d, dtype=torch.float32), rand(275, d, dtype=torch.float32)
    w = [rand(4, *s, dtype=torch.float32) for s in ((F, d), (F, d), (d, F))]
    for need, call in ((cm.ffn_fp8_workspace_bytes(275, d, F), lambda **kw: (cm.grouped_ffn_fp8(x8, off, *w8, **kw),)),
                       (cm.ffn_backward_workspace_bytes(275, 4, F, torch.float32),
                        lambda **kw: cm.grouped_ffn_backward(x, dy, off, *w, **kw))):
        want = call()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = call(stream=side)
        taken = [torch.full((need,), 0x5a, device="cuda", dtype=torch.uint8) for _ in range(8)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        del taken
