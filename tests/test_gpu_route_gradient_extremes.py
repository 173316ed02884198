"""Infinities and NaN in the router's gradient, in every form of its products: what the definition makes of them is not finite in
the result either (an infinity may have become a NaN), and nothing else is touched."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.test_gpu_layer_gradients import _normal, _routing

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


FORMS = [(8, 250, F32), (8, 256, F32), (20, 96, F32), (100, 97, F32), (16, 64, BF16), (64, 2048, BF16), (8, 38400, BF16), (100, 264, BF16), (256, 136, BF16),
         (31, 33, BF16), (100, 257, BF16), (200, 131, BF16)]


@pytest.mark.parametrize("E,d,dtype", FORMS)
def test_what_is_not_finite_stays_where_it_belongs(cm, E, d, dtype):
    N = 300
    r, dr, rows = _routing(cm, N, E, 2, 0, 1, 4.0)
    x, w, dsc = _normal((N, d), 1.0, dtype, 2), _normal((E, d), 0.1, dtype, 3), _normal((N, E), 0.5, F32, 4)
    dwt = _normal((rows,), 1.0, F32, 5)

    def run(x, w, dsc):
        return cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], dwt, dscores=dsc, out_dtype=F32)

    def as_defined(got, x, w):
        dl = got["dlogits"].double()
        assert torch.equal(got["dx"].isfinite(), (dl @ w.double()).isfinite())
        assert torch.equal(got["dw"].isfinite(), (dl.T @ x.double()).isfinite())
        assert torch.equal(got["dbias"].isfinite(), dl.sum(0).isfinite())

    clean = run(x, w, dsc)
    assert all(bool(v.isfinite().all()) for v in clean.values())
    for value in (INF, -INF, NAN):
        # a token's column: dW of that column alone
        x1 = x.clone()
        x1[11, d // 2] = x1[N - 1, 0] = value
        got = run(x1, w, dsc)
        as_defined(got, x1, w)
        cols = torch.ones(d, dtype=torch.bool, device="cuda")
        cols[[0, d // 2]] = False
        assert all(torch.equal(got[k], clean[k]) for k in ("dlogits", "dx", "dbias")) and torch.equal(got["dw"][:, cols], clean["dw"][:, cols])
        # an expert's column: dx of that column alone
        w1 = w.clone()
        w1[1, d - 1] = value
        got = run(x, w1, dsc)
        as_defined(got, x, w1)
        assert all(torch.equal(got[k], clean[k]) for k in ("dlogits", "dw", "dbias")) and torch.equal(got["dx"][:, :-1], clean["dx"][:, :-1])
        # a score's gradient: that token's dlogits, with them its dx, and all sums over tokens
        d1 = dsc.clone()
        d1[130, 1] = value
        got = run(x, w, d1)
        as_defined(got, x, w)
        ok = torch.arange(N, device="cuda") != 130
        assert not bool(got["dlogits"][130].isfinite().any())
        assert torch.equal(got["dlogits"][ok], clean["dlogits"][ok]) and torch.equal(got["dx"][ok], clean["dx"][ok])
