"""What the router's gradient keeps of its sums, in every form of its products: all bits of dlogits, long sums of dW, every stage of
tokens in its place.

Bounds.  An MMA adds up to 16 products to an accumulator and cuts off where fp32 ends: 2^-23 of the sum, and as much where the products
are aligned to it.  A rounded addition is off by 2^-24 of its sum."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.grouped_ref import close
from tests.test_gpu_layer_gradients import _normal, _routing

pytestmark = pytest.mark.gpu
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U2 = 2.0 ** -23
PARTS = 3                                     # bf16 numbers of dlogits: MMAs per 16 terms


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _inputs(cm, N, E, d, dtype, dscores, seed=5, positive=False):
    r, dr, rows = _routing(cm, N, E, min(E, 2), 0, seed, 4.0)
    x, w = _normal((N, d), 1.0, dtype, seed + 1), _normal((E, d), 0.1, dtype, seed + 2)
    if positive:
        x = (x.float().abs() + 0.1).to(dtype)
    return cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], torch.zeros((rows,), device="cuda"), dscores=dscores,
                             out_dtype=F32), x.double(), w.double()


# rows that TMA addresses and rows that warps lay out, with 64, 128 and 256 experts at most
BF16_FORMS = [(2, 64), (16, 2048), (60, 264), (100, 264), (256, 136), (2, 33), (31, 33), (64, 2047), (100, 257), (200, 131)]


@pytest.mark.parametrize("E,d", BF16_FORMS)
@pytest.mark.parametrize("N", [1, 16])
def test_dw_of_bf16_tokens_has_every_bit_of_dlogits(cm, N, E, d):
    """One MMA for each of the three numbers of dlogits; their products with bf16 tokens are exact."""
    got, x, w = _inputs(cm, N, E, d, BF16, _normal((N, E), 1.0, F32, 3))
    dl = got["dlogits"].double()
    close(got["dw"], dl.T @ x, PARTS * (1 if N == 1 else 2) * U2 * (dl.abs().T @ x.abs()) + 1e-38)


@pytest.mark.parametrize("E,d", BF16_FORMS)
@pytest.mark.parametrize("N", [1, 65, 300])
def test_dx_of_bf16_tokens_has_every_bit_of_dlogits(cm, N, E, d):
    """dx is one rounding of a sum that is as good as fp32's: it lies between the roundings of the sum's bounds."""
    got, x, w = _inputs(cm, N, E, d, BF16, _normal((N, E), 1.0, F32, 3))
    dl = got["dlogits"].double()
    dx, e = dl @ w, 2 * PARTS * -(-E // 16) * U2 * (dl.abs() @ w.abs()) + 1e-38
    assert bool((got["dx"] >= (dx - e).to(BF16)).all()) and bool((got["dx"] <= (dx + e).to(BF16)).all())


@pytest.mark.parametrize("E,d,dtype,adds", [(16, 18944, BF16, 48), (64, 18944, BF16, 48), (128, 9472, BF16, 48), (256, 9472, BF16, 48),
                                            (20, 9471, BF16, 48), (100, 9471, BF16, 192), (200, 9471, BF16, 192), (20, 9472, F32, 128), (8, 9472, F32, 0)])
def test_long_sums_of_dw_keep_their_precision(cm, E, d, dtype, adds):
    """Sums of 16,400 terms of one sign, up to 8,192 of them in one thread block.  `adds`: MMAs into an accumulator before it is added up in
    registers (256 tokens; of bf16 tokens that warps lay out, more than 64 experts: a part of 1024).  Their sum grows by equal steps, so
    that on average a cut is of half of it; then up to 65 rounded additions, of the groups and of the ranges.  (Plain FMAs: 8,200 rounded
    ones, of sums that grow, fall to either side: the bound of the others, 48.)"""
    N = 16400
    dscores = torch.zeros((E,), device="cuda")
    dscores[1] = 1.0                                                  # one expert's dlogits are positive, the others' negative
    got, x, w = _inputs(cm, N, E, d, dtype, dscores, positive=True)
    want = got["dlogits"].double().T @ x
    close(got["dw"], want, ((adds or 48) + 65 / 2) * U2 * want.abs())


@pytest.mark.parametrize("N,E,d,dtype", [(20000, 8, 256, BF16), (12345, 64, 2048, BF16), (9001, 128, 264, BF16), (9001, 256, 640, BF16), (12345, 30, 131, BF16),
                                         (9001, 100, 77, BF16), (9001, 256, 259, BF16), (20000, 8, 250, F32), (7001, 60, 136, F32), (5001, 200, 257, F32)])
def test_every_stage_of_tokens_counts_once(cm, N, E, d, dtype):
    """dlogits of 64 neighbouring tokens alone: dW is their sum, however many ranges and stages there are (a sum over all tokens
    would hide one that is lost in what it may be off)."""
    last = (N - 1) // 64
    for stage in (0, 1, last // 3, last // 2 + 1, last - 1, last):
        at = slice(64 * stage, min(N, 64 * stage + 64))
        dscores = torch.zeros((N, E), device="cuda")
        dscores[at] = _normal((at.stop - at.start, E), 1.0, F32, stage)
        got, x, w = _inputs(cm, N, E, d, dtype, dscores)
        dl = got["dlogits"].double()
        rest = dl.clone()
        rest[at] = 0
        assert bool((rest == 0).all())
        close(got["dw"], dl[at].T @ x[at], 64 * U2 * (dl[at].abs().T @ x[at].abs()) + 1e-38)
        close(got["dbias"], dl[at].sum(0), 64 * U2 * dl[at].abs().sum(0) + 1e-38)
