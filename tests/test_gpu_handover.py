"""Tiles that one CTA of a pair takes from a counter and hands to the other: a hand-over that went wrong would leave half a
tile unwritten or mix it with another one.  Every call here has thousands of the shortest tiles, so millions of hand-overs
run in a test; the first call is held against a 64-bit definition, every later one, into buffers filled anew, has to give
the same bits."""
import pytest
import torch

import grouped_ref as R

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
E = 256


@pytest.fixture(scope="module")
def cm():
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


@pytest.fixture
def forced(cm):
    yield lambda name: cm.debug_ffn_variant(name)
    cm.debug_ffn_variant("auto")


def _normal(shape, std, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=BF16).normal_(0, std, generator=g)


def _repeat(cm, calls, outs, run, first):
    """run(status block) into `outs`, again and again; first() checks what the first call left there."""
    st = torch.zeros(cm.FFN_STATUS_WORDS, device="cuda", dtype=torch.int32)
    same = torch.ones((), device="cuda", dtype=torch.bool)
    want = None
    for _ in range(calls):
        for t in outs:
            t.fill_(7.0)
        run(st)
        if want is None:
            first()
            want = [t.clone() for t in outs]
        for t, w in zip(outs, want):
            same &= (t == w).all()
    assert int(st[0]) == 0 and bool(same)


@pytest.mark.parametrize("d,F", [(64, 4096), (4096, 64)])
@pytest.mark.parametrize("form", ["pair", "short"])
def test_ffn(cm, forced, form, d, F):
    """One row per expert: 4096 tiles and more of one k-block in the gate/up launch (in the down launch with d = 4096)."""
    forced(form)
    off = torch.arange(E + 1, device="cuda", dtype=torch.int32)
    x = _normal((E, d), 1.0, 1)
    w = [_normal((E, *s), 0.4 / d ** 0.5, 2 + i) for i, s in enumerate(((F, d), (F, d), (d, F)))]
    h, y = torch.empty((E, F), device="cuda", dtype=BF16), torch.empty((E, d), device="cuda", dtype=BF16)

    def first():
        for e in range(E):
            wg, wu, wd = (t[e].double() for t in w)
            _, _, ref, err = R.swiglu(x[e:e + 1].double(), wg, wu)
            R.close(h[e:e + 1], ref, R.rounded(ref, err, BF16))
            R.close(y[e:e + 1], *R.product(h[e:e + 1].double(), wd, BF16))

    _repeat(cm, 3000, [h, y], lambda st: cm.grouped_ffn(x, off, *w, h_ws=h, y_perm=y, dev_status=st), first)


def test_weight_gradients(cm):
    """16 tiles for each of 256 experts, most of them empty sums; a row's outer product is exact before its rounding."""
    d = n = 1024
    counts = [1 if e % 9 == 4 else 0 for e in range(E)]
    off, A = R.offsets_of(counts), sum(counts)
    x, dy = _normal((A, d), 1.0, 10), _normal((A, n), 1.0, 11)
    dw = torch.empty((E, n, d), device="cuda", dtype=BF16)

    def first():
        r = 0
        for e, c in enumerate(counts):
            assert torch.equal(dw[e], (dy[r].float()[:, None] * x[r].float()).to(BF16) if c else torch.zeros_like(dw[e]))
            r += c

    _repeat(cm, 1500, [dw], lambda st: cm.grouped_mm_dw(dy, x, off, dw=dw, dev_status=st), first)


@pytest.mark.parametrize("direction", ["y", "dx"])
def test_row_products(cm, direction):
    """One row per expert in buffers for many more (the products of a few allocated rows take no counter)."""
    rows, k, m = 65 * E, 64, 4096
    off = torch.arange(E + 1, device="cuda", dtype=torch.int32)
    x = _normal((rows, k), 1.0, 20)
    w = _normal((E, m, k) if direction == "y" else (E, k, m), 0.1, 21)
    y = torch.full((rows, m), 7.0, device="cuda", dtype=BF16)
    run = (lambda st: cm.grouped_mm(x, off, w, y=y, dev_status=st)) if direction == "y" else (
        lambda st: cm.grouped_mm_dx(x, off, w, dx=y, dev_status=st))

    def first():
        for e in range(E):
            R.close(y[e:e + 1], *R.product(x[e:e + 1].double(), w[e].double() if direction == "y" else w[e].double().T, BF16))

    _repeat(cm, 3000, [y[:E]], run, first)
    assert bool((y[E:] == 7).all())


def test_ffn_gradients(cm):
    """All three launches: hidden gradients, dx and the three weight gradients, whole."""
    d = F = 512
    counts = [1 if e % 4 == 1 else 0 for e in range(E)]
    off, A = R.offsets_of(counts), sum(counts)
    x, dy = _normal((A, d), 1.0, 30), _normal((A, d), 1.0, 31)
    w = [_normal((E, *s), 0.05, 32 + i) for i, s in enumerate(((F, d), (F, d), (d, F)))]
    dx, dw = torch.empty_like(x), [torch.empty_like(t) for t in w]

    def first():
        r = 0
        for e, c in enumerate(counts):
            if c == 0:
                assert all(bool((t[e] == 0).all()) for t in dw)
                continue
            ref = R.ffn_gradient(x[r:r + 1].double(), dy[r:r + 1].double(), *(t[e].double() for t in w), BF16)
            for got, name in ((dx[r:r + 1], "dx"), (dw[0][e], "dw_gate"), (dw[1][e], "dw_up"), (dw[2][e], "dw_down")):
                R.close(got, *ref[name])
            r += 1

    _repeat(cm, 1500, [dx, *dw], lambda st: cm.grouped_ffn_backward(x, dy, off, *w, dx=dx, dw=dw, dev_status=st), first)


@pytest.mark.parametrize("d,F", [(128, 2048), (2048, 128)])
@pytest.mark.parametrize("form", ["pair", "short"])
def test_8_bit_ffn(cm, forced, form, d, F):
    """One row per expert in buffers for many more; the gate/up launch (the down launch with d = 2048) has the short tiles."""
    forced(form)
    rows = 65 * E
    off = torch.arange(E + 1, device="cuda", dtype=torch.int32)
    x = _normal((rows, d), 1.0, 40)
    w = [cm.quantize_weights(_normal((E, *s), 0.08, 41 + i)) for i, s in enumerate(((F, d), (F, d), (d, F)))]
    y = torch.full((rows, d), 7.0, device="cuda", dtype=BF16)

    def first():
        for e in range(E):
            wg, wu, wd = (R.decoded(q[e], s[e], 128) for q, s in w)
            _, _, h, eh = R.swiglu(R.values(x[e:e + 1].double(), 1), wg, wu)
            hq, ehq = R.quantized_hidden(h, eh)
            ref, e1 = R.product(hq, wd)
            R.close(y[e:e + 1], ref, R.rounded(ref, e1 * 1.2 + ehq @ wd.abs().T, BF16))

    _repeat(cm, 3000, [y[:E]], lambda st: cm.grouped_ffn_fp8(x, off, *w, y_perm=y, dev_status=st), first)
    assert bool((y[E:] == 7).all())
