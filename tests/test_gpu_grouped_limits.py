"""Grouped products at the largest row counts that they accept: nearly all rows in one expert, a few before and behind it."""
import pytest
import torch

import grouped_ref as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROWS = (1 << 31) - 512
COUNTS = [5, ROWS - 12, 7]


@pytest.fixture(scope="module")
def cm():
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


@pytest.fixture(autouse=True)
def room():
    def need(gigabytes):
        torch.cuda.empty_cache()
        if torch.cuda.mem_get_info()[0] < (gigabytes + 4) * 1e9:
            pytest.skip("not enough free memory on this device")
    yield need
    torch.cuda.empty_cache()


def _normal(shape, std, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(0, std, generator=g)


def _sample():
    """Row numbers next to every border and all over, and the expert of each."""
    g = torch.Generator(device="cuda").manual_seed(9)
    any_row = torch.randint(0, ROWS, (200_000,), device="cuda", generator=g)
    at = torch.cat([torch.arange(600, device="cuda"), any_row, torch.arange(ROWS - 600, ROWS, device="cuda")])
    e = (at >= 5).long() + (at >= ROWS - 7).long()
    return [(i, at[e == i]) for i in range(3)]


def _finite(t):
    return all(bool(torch.isfinite(c.float()).all()) for c in t.split(1 << 26))


@pytest.mark.parametrize("dtype,size", [(BF16, 8), (F32, 1)])
def test_products(cm, room, dtype, size):
    """All rows are written (the outputs start as NaN), and those at every border are right."""
    room(2e-9 * ROWS * size * dtype.itemsize)
    off = R.offsets_of(COUNTS)
    x, w = _normal((ROWS, size), 1.0, dtype, 1), _normal((3, size, size), 1.0, dtype, 2)
    y = torch.full_like(x, float("nan"))
    cm.grouped_mm(x, off, w, y=y)
    assert _finite(y)
    for e, r in _sample():
        R.close(y[r], *R.product(x[r].double(), w[e].double(), dtype))
    x.fill_(float("nan"))
    cm.grouped_mm_dx(y, off, w, dx=x)
    assert _finite(x)
    for e, r in _sample():
        R.close(x[r], *R.product(y[r].double(), w[e].double().T, dtype))


def test_8_bit_product(cm, room):
    size = 16
    room(1e-9 * ROWS * (size + 1 + 2 * size))
    off = R.offsets_of(COUNTS)
    g = torch.Generator(device="cuda").manual_seed(3)
    code = torch.empty((ROWS, size), device="cuda", dtype=torch.uint8).random_(0, 0x7f, generator=g)       # finite, positive
    scale = torch.empty((ROWS, 1), device="cuda", dtype=torch.uint8).random_(120, 130, generator=g)
    xq, xs = code.view(cm.FP8), scale.view(cm.SCALE)
    wq, ws = cm.quantize_weights(_normal((3, size, size), 1.0, BF16, 4))
    y = torch.full((ROWS, size), float("nan"), device="cuda", dtype=BF16)
    cm.grouped_mm_fp8(xq, xs, off, wq, ws, y=y)
    assert _finite(y)
    for e, r in _sample():
        at = R.decoded(code[r].view(cm.FP8), scale[r].view(cm.SCALE), 1)
        R.close(y[r], *R.product(at, R.decoded(wq[e], ws[e], 128), BF16))


def test_weight_gradient_of_a_very_long_segment(cm, room):
    """One of many experts has 805 million rows: its reduction, which is not split, takes about four seconds, longer than a
    wait may usually last.  Sums of -1, 0 and 1 far below 2^24: every order gives the same."""
    rows, E, size = 3 << 28, 40, 8
    room(4e-9 * rows * size)
    off = torch.full((E + 1,), rows, device="cuda", dtype=torch.int32)
    off[:18] = 0
    off[18:21] = rows - 5                                       # two experts without rows behind it, then one with five
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.empty((rows, size), device="cuda", dtype=BF16) for _ in range(2))
    for t in (x, dy):
        for c in t.split(1 << 26):
            c.copy_(torch.empty(c.shape, device="cuda", dtype=torch.int8).random_(-1, 2, generator=g))
    st = torch.zeros(cm.FFN_STATUS_WORDS, device="cuda", dtype=torch.int32)
    want = torch.zeros((E, size, size), device="cuda", dtype=F32)
    for a, b in zip(dy[:-5].split(1 << 24), x[:-5].split(1 << 24)):
        want[17] += a.float().T @ b.float()
    want[20] = dy[-5:].float().T @ x[-5:].float()
    for status in (st, None):
        dw = cm.grouped_mm_dw(dy, x, off, out_dtype=F32, dev_status=status)
        assert torch.equal(dw, want)
    assert int(st[0]) == 0 and float(want[17].abs().max()) < 2 ** 22


def test_quantisers_of_the_longest_rows(cm, room):
    """One row (one column of a weight) of 2^31 - 1024 elements has the blocks of as many rows of 128."""
    size = (1 << 31) - 1024
    room(2e-9 * size * 4)
    x = _normal((1, size), 1.0, BF16, 6)
    q, s = (t.view(torch.uint8) for t in cm.quantize_rows(x.view(-1, 128)))
    for view, got in ((x.shape, cm.quantize_rows(x)), ((1, size, 1), cm.quantize_weights(x.view(1, size, 1)))):
        assert got[0].shape == view
        assert torch.equal(got[0].view(torch.uint8).view(q.shape), q) and torch.equal(got[1].view(torch.uint8).view(s.shape), s)
