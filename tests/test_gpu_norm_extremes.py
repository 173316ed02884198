"""Gradients of the norm where rstd is far from one.  Bounds as in test_gpu_norm."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.grouped_ref import close, rounded
from tests.test_gpu_norm import _grad_ref, _normal

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 258, 515, 4096])
def test_gradients_of_rows_of_any_size(cm, d, dtype):
    """Without eps, rows of 1e-20 to 1e17: rstd^2 alone would pass fp32, what it is multiplied with brings it back."""
    h, w = _normal((40, d), 1.0, dtype, 1), _normal((d,), 1.0, dtype, 2)
    h *= 10.0 ** torch.linspace(-20, 17, 40, device="cuda")[:, None].to(dtype)
    rstd = (1.0 / torch.sqrt((h.double() ** 2).mean(1))).float()
    dy = _normal((40, d), 1.0, dtype, 3)
    for dh in (None, _normal((40, d), 1.0, dtype, 4)):
        gx, gw = cm.rms_norm_backward(dy, h, w, rstd, dh=dh, out_dtype=F32)
        dx, e, dw, ew = _grad_ref(dy, h, w, rstd, dh)
        close(gx, dx, rounded(dx, e, dtype))
        close(gw, dw, rounded(dw, ew, F32))
