"""Home groups from a table, not from a token's place: which experts the slots behind the top-k ones belong to."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.grouped_ref import close, rounded
from tests.test_gpu_layer_gradients import _normal, _route_ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _routing(cm, N, E, k, D, seed):
    """Scores, top-k lists and rows with a random table; -> also every slot's expert and the rows that are used."""
    r = cm.route(None, None, None, k, logits_in=_normal((N, E), 1.0, F32, seed))
    group = torch.randint(0, D, (N,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).int()
    C = cm.capacity(N, E, k, 0.9)
    dr = cm.expanded_drop(r["scores"], r["topk_idx"], C, D, token_group=group)
    plain = cm.expanded_drop(r["scores"], r["topk_idx"], C, D)
    assert not torch.equal(dr["slot_row"], plain["slot_row"])         # the table matters
    m = E // D
    expert = torch.cat([r["topk_idx"].long(), group.long()[:, None] * m + torch.arange(m, device="cuda")], 1)
    return r, dr, group, expert, cm.max_rows(N, E, k, D, C, True)


@pytest.mark.parametrize("N,E,k,D,d", [(500, 8, 2, 4, 4096), (300, 256, 8, 32, 2064), (900, 130, 6, 10, 48), (33, 16, 1, 16, 160)])
def test_permute_fp8(cm, N, E, k, D, d):
    r, dr, group, expert, rows = _routing(cm, N, E, k, D, N)
    x = _normal((N, d), 1.0, BF16, 1)
    q, sc = cm.quantize_rows(x)
    want = cm.permute(x, r["scores"], r["topk_idx"], dr["slot_row"], rows, D=D, token_group=group)
    got = cm.permute_fp8(q, sc, r["scores"], r["topk_idx"], dr["slot_row"], rows, D=D, token_group=group)
    A = int(dr["offsets"][-1])
    t, s = torch.nonzero(dr["slot_row"] >= 0, as_tuple=True)
    weight = torch.empty((A,), device="cuda")
    weight[dr["slot_row"][t, s].long()] = r["scores"][t, expert[t, s]]
    assert torch.equal(got["perm_weight"][:A], weight) and torch.equal(got["perm_weight"][:A], want["perm_weight"][:A])
    assert torch.equal(got["perm_token"][:A], want["perm_token"][:A])
    at = want["perm_token"][:A].long()
    assert torch.equal(got["x_q"].view(torch.uint8)[:A], q.view(torch.uint8)[at]) and torch.equal(got["x_scale"].view(torch.uint8)[:A], sc.view(torch.uint8)[at])


@pytest.mark.parametrize("N,E,k,D,d,dtype", [(300, 8, 2, 4, 100, F32), (700, 8, 1, 2, 256, F32), (300, 60, 4, 12, 136, F32), (200, 130, 3, 13, 66, F32),
                                             (300, 64, 6, 16, 512, BF16), (200, 256, 8, 32, 136, BF16), (300, 32, 2, 8, 77, BF16), (200, 100, 2, 20, 33, BF16)])
def test_route_backward(cm, N, E, k, D, d, dtype):
    r, dr, group, expert, rows = _routing(cm, N, E, k, D, N)
    x, w, dsc = _normal((N, d), 1.0, dtype, 1), _normal((E, d), 0.1, dtype, 2), _normal((E,), 0.3, F32, 3)
    dweight = torch.full((rows,), float("nan"), device="cuda")
    A = int(dr["offsets"][-1])
    dweight[:A] = _normal((A,), 1.0, F32, 4)
    got = cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], dweight, D=D, token_group=group, dscores=dsc, out_dtype=F32)
    ref = _route_ref(x, w, r["scores"], expert, dr["slot_row"], dweight, dsc, dtype)
    close(got["dlogits"], *ref[0])
    close(got["dx"], ref[1][0], rounded(*ref[1], dtype))
    close(got["dw"], ref[2][0], rounded(*ref[2], F32))
    close(got["dbias"], ref[3][0], rounded(*ref[3], F32))
