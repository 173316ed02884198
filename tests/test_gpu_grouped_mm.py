"""Grouped products over expert-major rows and their gradients against 64-bit definitions."""
import ctypes

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


def _rows(shape, used, std, dtype, seed):
    """Random rows; those behind the last expert's hold NaN, which no result may show."""
    t = _normal(shape, std, dtype, seed)
    t[used:] = float("nan")
    return t


# rows per expert: none at all, one, tile borders and their neighbours, long next to empty
COUNTS = {
    "one row": [1],
    "all empty": [0, 0, 0],
    "few": [1, 0, 3, 2, 0, 5, 1],
    "borders": [16, 15, 17, 0, 64, 63, 65, 128, 127, 129, 1],
    "long": [0, 700, 1, 300, 0],
    "longer": [1100, 37, 2051],
    "many": [(7 * e) % 23 for e in range(256)],
}
# (d, n): whole tiles, multiples of 64 and of 8 that leave ragged tiles, and sizes with no 16-byte rows
SIZES = [(256, 512), (64, 64), (192, 320), (136, 72), (8, 264), (520, 24), (33, 65), (250, 515), (1, 7), (7, 1), (64, 33), (33, 64)]


def _case(counts, d, n, dtype, spare=5):
    off = R.offsets_of(counts)
    A = sum(counts)
    rows = A + spare
    E = len(counts)
    return off, A, rows, _rows((rows, d), A, 1.0, dtype, 1), _rows((rows, n), A, 1.0, dtype, 2), _normal((E, n, d), 0.1, dtype, 3)


def _spans(counts):
    o = 0
    for e, c in enumerate(counts):
        yield e, slice(o, o + c)
        o += c


def _block(cm):
    return torch.zeros(cm.FFN_STATUS_WORDS, device="cuda", dtype=torch.int32)


def _check_all(cm, counts, d, n, dtype, status=True):
    off, A, rows, x, dy, w = _case(counts, d, n, dtype)
    st = _block(cm) if status else None
    y = torch.full((rows, n), 3.0, device="cuda", dtype=dtype)
    dx = torch.full((rows, d), 3.0, device="cuda", dtype=dtype)
    dw = torch.full((len(counts), n, d), float("nan"), device="cuda", dtype=dtype)
    cm.grouped_mm(x, off, w, y=y, dev_status=st)
    cm.grouped_mm_dx(dy, off, w, dx=dx, dev_status=st)
    cm.grouped_mm_dw(dy, x, off, dw=dw, dev_status=st)
    assert bool((y[A:] == 3).all()) and bool((dx[A:] == 3).all()), "rows behind the last expert's were written"
    for e, r in _spans(counts):
        w64, x64, dy64 = w[e].double(), x[r].double(), dy[r].double()
        R.close(y[r], *R.product(x64, w64, dtype))
        R.close(dx[r], *R.product(dy64, w64.T, dtype))
        R.close(dw[e], *R.product(dy64.T, x64.T, dtype))
    if st is not None:
        assert int(st[0]) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,n", SIZES)
@pytest.mark.parametrize("name", ["one row", "all empty", "few", "borders"])
def test_products_and_gradients(cm, name, d, n, dtype):
    _check_all(cm, COUNTS[name], d, n, dtype)


@pytest.mark.parametrize("d,n", [(256, 512), (136, 72), (1032, 264), (320, 1032), (250, 515)])
@pytest.mark.parametrize("name", ["long", "longer", "many"])
def test_long_and_many_segments(cm, name, d, n):
    _check_all(cm, COUNTS[name], d, n, BF16)


def test_many_segments_fp32(cm):
    _check_all(cm, COUNTS["many"], 40, 72, F32)


@pytest.mark.parametrize("counts,d,n,dtype", [([1300, 0, 1270, 10], 37, 1921, F32), ([1300, 0, 1270, 10], 1921, 37, F32),
                                              ([1300, 0, 1270, 10], 64, 1924, F32), ([70, 0, 200], 1300, 1301, F32),
                                              ([1300, 0, 1270, 10], 37, 1921, BF16), ([70, 0, 200], 1301, 1300, BF16)])
def test_large_tiles_of_the_fma_kernels(cm, counts, d, n, dtype):
    """So many 128 x 128 tiles that one direction's product runs on them (fp32, and bf16 of odd sizes)."""
    _check_all(cm, counts, d, n, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,d,n", [([1], 1021, 37), ([3, 0, 1], 64, 1001), ([2, 5], 511, 130), ([1, 40], 65, 300), ([7], 4099, 5)])
def test_few_rows_with_long_sums(cm, counts, d, n, dtype):
    """So few tiles that the reduction is split over a cluster's blocks, in 2, 4 and 8 parts."""
    _check_all(cm, counts, d, n, dtype)


@pytest.mark.parametrize("counts", [COUNTS["borders"], COUNTS["longer"]])
def test_without_a_status_block(cm, counts):
    _check_all(cm, counts, 192, 320, BF16, status=False)


@pytest.mark.parametrize("d,n", [(256, 512), (136, 72), (33, 65)])
def test_weight_gradient_in_fp32(cm, d, n):
    """bf16 rows, fp32 gradient: nothing but the fp32 sum's own error."""
    counts = COUNTS["borders"] + [300]
    off, A, rows, x, dy, _ = _case(counts, d, n, BF16)
    dw = cm.grouped_mm_dw(dy, x, off, out_dtype=F32, dev_status=_block(cm))
    assert dw.dtype == F32
    for e, r in _spans(counts):
        R.close(dw[e], *R.product(dy[r].double().T, x[r].double().T, F32))


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("counts,d,n,in_parts", [([3000], 136, 72, True), ([700, 0, 5000], 264, 256, True), ([0, 9000], 512, 320, True),
                                                 ([1, 1, 2600, 40], 64, 1032, False)])
def test_weight_gradient_in_parts(cm, counts, d, n, in_parts, out_dtype):
    """Few output tiles and long segments, on the average of the allocated rows: the sums are split into parts when the
    workspace has room for them."""
    off, A, rows, x, dy, _ = _case(counts, d, n, BF16)
    extra = cm.dw_split_bytes(rows, len(counts), d, n, BF16)
    assert extra >= 2 * 4 * len(counts) * d * n if in_parts else extra == 0
    small = torch.empty(1 << 12, device="cuda", dtype=torch.uint8)
    whole = cm.grouped_mm_dw(dy, x, off, out_dtype=out_dtype, dev_status=_block(cm), ws=small)
    before = cm.launch_count()
    split = cm.grouped_mm_dw(dy, x, off, out_dtype=out_dtype, dev_status=_block(cm))
    assert cm.launch_count() - before == (3 if in_parts else 2)  # maps, products, the sum of the parts
    assert torch.equal(split, cm.grouped_mm_dw(dy, x, off, out_dtype=out_dtype))
    for e, r in _spans(counts):
        want = R.product(dy[r].double().T, x[r].double().T, out_dtype)
        R.close(split[e], *want)
        R.close(whole[e], *want)


def test_parts_captured_and_replayed(cm):
    """Split sums (bf16 parts in the workspace, fp32 clusters) in one graph, replayed after the offsets have moved."""
    off, A, rows, x, dy, _ = _case([700, 0, 5000], 264, 256, BF16)
    dy2, w2, off2 = _normal((9, 1021), 1.0, F32, 41), _normal((2, 37, 1021), 0.1, F32, 42), R.offsets_of([4, 5])

    def calls():
        return [cm.grouped_mm_dw(dy, x, off), cm.grouped_mm(dy2, off2, w2)]

    calls()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = calls()
    off.copy_(R.offsets_of([2000, 3000, 700]))
    off2.copy_(R.offsets_of([8, 1]))
    torch.cuda.synchronize()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, calls()):
        assert torch.equal(a, b)


def test_few_tiles_but_short_segments_are_not_split(cm):
    assert cm.dw_split_bytes(900, 1, 256, 256, BF16) == 0 and cm.dw_split_bytes(1 << 20, 64, 2048, 1024, BF16) == 0
    assert cm.dw_split_bytes(1 << 20, 1, 256, 256, F32) == 0


def test_weight_gradient_with_no_rows_allocated(cm):
    x = torch.empty((0, 64), device="cuda", dtype=BF16)
    dy = torch.empty((0, 32), device="cuda", dtype=BF16)
    dw = torch.full((2, 32, 64), 5.0, device="cuda", dtype=BF16)
    cm.grouped_mm_dw(dy, x, R.offsets_of([0, 0]), dw=dw)
    assert bool((dw == 0).all())
    assert cm.grouped_mm(x, R.offsets_of([0, 0]), torch.zeros((2, 32, 64), device="cuda", dtype=BF16)).shape == (0, 32)


def test_infinities_stay_in_their_rows_and_experts(cm):
    """A NaN or an infinity in one row shows in that row's results and in its expert's weight gradient only."""
    counts = [40, 30, 0, 50]
    off, A, rows, x, dy, w = _case(counts, 128, 64, BF16)
    x[45, 7] = float("inf")
    dy[45, 3] = float("nan")
    y = cm.grouped_mm(x, off, w)
    dx = cm.grouped_mm_dx(dy, off, w)
    dw = cm.grouped_mm_dw(dy, x, off)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[45] = True
    assert bool((~torch.isfinite(y[:A])).any(1).eq(bad[:A]).all()) and bool((~torch.isfinite(dx[:A])).any(1).eq(bad[:A]).all())
    fine = torch.isfinite(dw.double()).all(2).all(1)
    assert fine.tolist() == [True, False, True, True]


def _check_ffn_gradient(cm, counts, d, F, dtype):
    off = R.offsets_of(counts)
    A, E = sum(counts), len(counts)
    rows = A + 3
    x, dy = _rows((rows, d), A, 1.0, dtype, 4), _rows((rows, d), A, 1.0, dtype, 5)
    wg, wu, wd = _normal((E, F, d), 0.1, dtype, 6), _normal((E, F, d), 0.1, dtype, 7), _normal((E, d, F), 0.1, dtype, 8)
    st = _block(cm)
    dx0 = torch.full((rows, d), 3.0, device="cuda", dtype=dtype)
    got = dict(zip(("dx", "dw_gate", "dw_up", "dw_down"),
                   cm.grouped_ffn_backward(x, dy, off, wg, wu, wd, dx=dx0, dev_status=st)))
    assert int(st[0]) == 0 and bool((got["dx"][A:] == 3).all())
    for e, r in _spans(counts):
        ref = R.ffn_gradient(x[r].double(), dy[r].double(), wg[e].double(), wu[e].double(), wd[e].double(), dtype)
        R.close(got["dx"][r], *ref["dx"])
        for k in ("dw_gate", "dw_up", "dw_down"):
            R.close(got[k][e], *ref[k])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,d,F", [([1], 64, 64), ([0, 0], 64, 64), ([3, 0, 70, 129, 1], 128, 192), ([65, 64, 17], 136, 72),
                                        ([5, 9, 0, 33], 33, 45), ([300, 0, 513], 256, 320), ([1] * 30, 64, 264),
                                        ([1200, 0, 33], 136, 192)])
def test_ffn_gradient(cm, counts, d, F, dtype):
    _check_ffn_gradient(cm, counts, d, F, dtype)


@pytest.mark.parametrize("counts,d,F", [([2100], 136, 192), ([5, 4000], 256, 264)])
def test_ffn_gradient_in_parts(cm, counts, d, F):
    assert cm.dw_split_bytes(sum(counts) + 3, len(counts), d, F, BF16, products=3) > 0
    _check_ffn_gradient(cm, counts, d, F, BF16)


@pytest.mark.parametrize("counts,d,F", [([1300, 0, 1270, 10], 1921, 37), ([70, 0, 200], 1285, 650)])
def test_ffn_gradient_of_large_fp32_tiles(cm, counts, d, F):
    _check_ffn_gradient(cm, counts, d, F, F32)


@pytest.mark.parametrize("counts,d,F", [([1], 1001, 33), ([2, 0, 5], 300, 70), ([33, 1], 515, 96), ([4], 70, 999)])
def test_ffn_gradient_of_few_rows(cm, counts, d, F):
    _check_ffn_gradient(cm, counts, d, F, F32)


def test_ffn_gradient_against_differences(cm):
    """Directional differences of the forward layer in 64 bits against the gradients' inner products.  With step t the
    symmetric difference of a smooth function is off by O(t^2); the loss is a sum of about 10^3 terms of size 1."""
    counts, d, F = [9, 0, 14], 48, 40
    off = R.offsets_of(counts)
    A, E = sum(counts), len(counts)
    x, dy = _normal((A, d), 1.0, F32, 1), _normal((A, d), 1.0, F32, 2)
    wg, wu, wd = _normal((E, F, d), 0.2, F32, 3), _normal((E, F, d), 0.2, F32, 4), _normal((E, d, F), 0.2, F32, 5)
    grads = cm.grouped_ffn_backward(x, dy, off, wg, wu, wd)

    def loss(x, wg, wu, wd):
        s = 0.0
        for e, r in _spans(counts):
            g, u = x[r] @ wg[e].T, x[r] @ wu[e].T
            s = s + (((g * torch.sigmoid(g) * u) @ wd[e].T) * dy[r].double()).sum()
        return s

    args = [t.double() for t in (x, wg, wu, wd)]
    t = 1e-4
    for i, grad in enumerate(grads):
        v = _normal(args[i].shape, 1.0, F32, 20 + i).double()
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + t * v, args[i] - t * v
        num = float((loss(*up) - loss(*down)) / (2 * t))
        ana = float((grad.double() * v).sum())
        # fp32 gradients: 2^-23 times a few hundred roundings of the terms; the difference: t^2 of the third derivative
        assert abs(num - ana) <= 1e-4 * float((grad.double() * v).abs().sum()), (i, num, ana)


def test_runs_with_the_layers_own_stages(cm):
    """A training step of the expert part as a program runs it: route, drop, permute, FFN, then its gradients; the
    product calls reproduce the FFN's down projection."""
    from paper_2503_05066_b200 import synth
    cfg = synth.CONFIGS["olmoe"].with_(N=300, d=128, F=192, E=8, k=2, D=2)
    inp = synth.make_layer_inputs(cfg)
    x, wr, wg, wu, wd = (t.cuda() for t in (inp.x, inp.w_router, inp.w_gate, inp.w_up, inp.w_down))
    r = cm.route(x, wr, None, cfg.k)
    C = cm.capacity(cfg.N, cfg.E, cfg.k, 1.0)
    dr = cm.token_drop(r["topk_score"], r["topk_idx"], cfg.E, C)
    A_max = cm.max_rows(cfg.N, cfg.E, cfg.k, cfg.D, C, False)
    p = cm.permute(x, r["scores"], r["topk_idx"], dr["slot_row"], A_max)
    h = torch.zeros((A_max, cfg.F), device="cuda", dtype=BF16)
    y = cm.grouped_ffn(p["x_perm"], dr["offsets"], wg, wu, wd, h_ws=h)
    again = cm.grouped_mm(h, dr["offsets"], wd, y=torch.zeros_like(y))
    A = int(dr["offsets"][-1])
    dy = _normal((A_max, cfg.d), 1.0, BF16, 9)
    dx, dwg, dwu, dwd = cm.grouped_ffn_backward(p["x_perm"], dy, dr["offsets"], wg, wu, wd)
    off = dr["offsets"].tolist()
    for e in range(cfg.E):
        s = slice(off[e], off[e + 1])
        R.close(again[s], *R.product(h[s].double(), wd[e].double(), BF16))
        ref = R.ffn_gradient(p["x_perm"][s].double(), dy[s].double(), wg[e].double(), wu[e].double(), wd[e].double(), BF16)
        R.close(dx[s], *ref["dx"])
        R.close(dwd[e], *ref["dw_down"])
    assert A <= A_max and bool((again[A:] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_replayed_and_on_another_stream(cm, dtype):
    """One graph of all calls, replayed on new data in the same buffers, equals the eager calls bit for bit."""
    counts = [70, 0, 5, 200]
    off, A, rows, x, dy, w = _case(counts, 128, 192, dtype)
    wd = _normal((4, 128, 192), 0.1, dtype, 11)
    st = _block(cm)
    out = [torch.zeros((rows, 192), device="cuda", dtype=dtype), torch.zeros((rows, 128), device="cuda", dtype=dtype),
           torch.zeros((4, 192, 128), device="cuda", dtype=dtype)]
    ws = torch.empty(1 << 16, device="cuda", dtype=torch.uint8)
    fx = torch.zeros((rows, 128), device="cuda", dtype=dtype)
    fdw = [torch.zeros((4, 192, 128), device="cuda", dtype=dtype), torch.zeros((4, 192, 128), device="cuda", dtype=dtype),
           torch.zeros((4, 128, 192), device="cuda", dtype=dtype)]
    fws = torch.empty(cm.ffn_backward_workspace_bytes(rows, 4, 192, dtype), device="cuda", dtype=torch.uint8)
    dxs = _normal((rows, 128), 1.0, dtype, 12)

    def calls():
        cm.grouped_mm(x, off, w, y=out[0], dev_status=st)
        cm.grouped_mm_dx(dy, off, w, dx=out[1], dev_status=st)
        cm.grouped_mm_dw(dy, x, off, dw=out[2], ws=ws, dev_status=st)
        cm.grouped_ffn_backward(x, dxs, off, w, w, wd, dx=fx, dw=fdw, ws=fws, dev_status=st)

    calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        calls()
    x[:A] = _normal((A, 128), 1.0, dtype, 13)
    dy[:A] = _normal((A, 192), 1.0, dtype, 14)
    off.copy_(R.offsets_of([0, 100, 75, 100]))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in out + [fx] + fdw]
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    for a, b in zip(got, out + [fx] + fdw):
        assert torch.equal(a, b)
    assert int(st[0]) == 0


def test_offsets_past_the_allocated_rows_are_clamped(cm):
    """Offsets that claim more rows than were allocated never reach memory behind the buffers."""
    for dtype in (F32, BF16):
        x, dy = _normal((50, 64), 1.0, dtype, 1), _normal((50, 64), 1.0, dtype, 2)
        w = _normal((2, 64, 64), 0.1, dtype, 3)
        off = torch.tensor([0, 30, 90], device="cuda", dtype=torch.int32)
        y = cm.grouped_mm(x, off, w)
        dw = cm.grouped_mm_dw(dy, x, off)
        R.close(y[30:], *R.product(x[30:].double(), w[1].double(), dtype))
        R.close(dw[1], *R.product(dy[30:].double().T, x[30:].double().T, dtype))


def test_guard_bands(cm):
    """Every output between canaries."""
    for dtype, d, n in ((BF16, 136, 72), (F32, 33, 65), (BF16, 192, 320)):
        counts = [37, 0, 130]
        off, A, rows, x, dy, w = _case(counts, d, n, dtype, spare=0)
        G = 1024

        def guarded(shape):
            size = 1
            for v in shape:
                size *= v
            raw = torch.full((size + 2 * G,), 7.0, device="cuda", dtype=dtype)
            return raw, raw[G:G + size].view(shape)

        raws = []
        for shape, call in (((rows, n), lambda t: cm.grouped_mm(x, off, w, y=t)), ((rows, d), lambda t: cm.grouped_mm_dx(dy, off, w, dx=t)),
                            ((3, n, d), lambda t: cm.grouped_mm_dw(dy, x, off, dw=t))):
            raw, t = guarded(shape)
            call(t)
            raws.append(raw)
        torch.cuda.synchronize()
        for raw in raws:
            assert bool((raw[:G] == 7).all()) and bool((raw[-G:] == 7).all())
            assert not bool((raw[G:-G] == 7).all())


def _at(t, shift):
    """The tensor's values in memory that starts `shift` bytes behind an allocation's start."""
    raw = torch.zeros(t.numel() * t.element_size() + shift, device="cuda", dtype=torch.uint8)
    v = raw[shift:].view(t.dtype).view(t.shape)
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype,d,n", [(BF16, 136, 72), (BF16, 33, 65), (F32, 64, 96), (F32, 33, 65)])
def test_buffers_that_start_on_16_bytes(cm, dtype, d, n):
    counts = [70, 0, 5, 200]
    off, A, rows, x, dy, w = _case(counts, d, n, dtype)
    want = cm.grouped_mm(x, off, w)[:A], cm.grouped_mm_dx(dy, off, w)[:A], cm.grouped_mm_dw(dy, x, off)
    x2, dy2, w2 = _at(x, 16), _at(dy, 48), _at(w, 16)
    ws = torch.empty(1 << 16, device="cuda", dtype=torch.uint8)[16:]
    got = (cm.grouped_mm(x2, off, w2, y=_at(torch.zeros((rows, n), device="cuda", dtype=dtype), 16))[:A],
           cm.grouped_mm_dx(dy2, off, w2, dx=_at(torch.zeros((rows, d), device="cuda", dtype=dtype), 80))[:A],
           cm.grouped_mm_dw(dy2, x2, off, dw=_at(torch.zeros((4, n, d), device="cuda", dtype=dtype), 16), ws=ws))
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_misaligned_buffers_are_refused(cm):
    off = R.offsets_of([3, 4])
    x, w = _normal((7, 64), 1.0, BF16, 1), _normal((2, 32, 64), 0.1, BF16, 2)
    with pytest.raises(cm.CapmoeError) as err:
        cm.grouped_mm(_at(x, 8), off, w)
    assert err.value.status == cm.EINVAL


def test_two_streams_at_once_give_what_one_gives(cm):
    """Calls that overlap on the GPU, each with its own status block and workspace; the tiles are handed out differently
    every time and every result is the same bits."""
    counts = [300, 0, 77, 1200, 5, 640]
    off, A, rows, x, dy, w = _case(counts, 512, 768, BF16)
    wd, dyx = _normal((6, 512, 768), 0.1, BF16, 30), _rows((rows, 512), A, 1.0, BF16, 31)

    def calls(st):
        return [cm.grouped_mm(x, off, w, dev_status=st)[:A], cm.grouped_mm_dx(dy, off, w, dev_status=st)[:A],
                cm.grouped_mm_dw(dy, x, off, dev_status=st),
                *(t[:A] if i == 0 else t for i, t in enumerate(cm.grouped_ffn_backward(x, dyx, off, w, w, wd, dev_status=st)))]

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
            assert all(torch.equal(a, b) for a, b in zip(want, g))
    assert all(int(b[0]) == 0 for b in blocks)


def test_matrices_past_32_bit_offsets(cm):
    """More than 2^31 elements in the rows of one side."""
    rows, d, n = 1_100_000, 64, 2048
    counts = [rows - 300, 0, 300]
    off = R.offsets_of(counts)
    x, w = _normal((rows, d), 1.0, BF16, 1), _normal((3, n, d), 0.1, BF16, 2)
    y = cm.grouped_mm(x, off, w)
    at = torch.tensor([0, 1, rows // 2, rows - 301, rows - 300, rows - 1], device="cuda")
    for e, r in ((0, at[:4]), (2, at[4:])):
        R.close(y[r], *R.product(x[r].double(), w[e].double(), BF16))
    dx = cm.grouped_mm_dx(y, off, w)
    for e, r in ((0, at[:4]), (2, at[4:])):
        R.close(dx[r], *R.product(y[r].double(), w[e].double().T, BF16))
    dw = cm.grouped_mm_dw(y, x, off)
    R.close(dw[2], *R.product(y[-300:].double().T, x[-300:].double().T, BF16))
    assert bool((dw[1] == 0).all()) and bool(torch.isfinite(dw.float()).all())


def test_the_same_bits_every_time(cm):
    """Tiles are handed from one CTA of a pair to the other while they run; with many experts without rows the hand-overs
    follow each other closely.  Any that went wrong would leave half a tile unwritten or mixed with another one."""
    counts = [0, 1, 0, 0, 0, 1] + [0] * 12 + [1, 0, 0, 0]
    E, d, F = len(counts), 2712, 3456
    off = R.offsets_of(counts)
    x, dy = _normal((3, d), 1.0, BF16, 50), _normal((3, d), 1.0, BF16, 51)
    w = [_normal((E, *s), 0.02, BF16, 52 + i) for i, s in enumerate(((F, d), (F, d), (d, F)))]
    st = _block(cm)
    dw = [torch.empty_like(t) for t in w]
    want, same = None, torch.ones((), device="cuda", dtype=torch.bool)
    for _ in range(300):
        for t in dw:
            t[0].fill_(7.0)
            t[4].fill_(7.0)
            t[6:9].fill_(7.0)
        cm.grouped_ffn_backward(x, dy, off, *w, dw=dw, dev_status=st)
        got = [t[4:9] for t in dw]
        if want is None:
            want = [t.clone() for t in got]
            assert all(bool((t[0] == 0).all()) and bool((t[2:] == 0).all()) for t in want)
        for a, b in zip(got, want):
            same &= (a == b).all()
    assert bool(same) and int(st[0]) == 0
