"""The operators around the expert products past 32-bit offsets, with rows of dscores further apart than experts, and with more column
slices than the device has SMs."""
import ctypes

import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build
from tests.grouped_ref import close, rounded
from tests.test_gpu_layer_gradients import _expert_of, _normal, _route_ref, _routing

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U2 = 2.0 ** -23


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


@pytest.mark.parametrize("N,E,d,dtype", [((1 << 31) // 2048 + 1000, 8, 2048, BF16), ((1 << 31) // 1024 + 1001, 8, 1024, F32), ((1 << 31) // 1024 + 1001, 9, 1024, F32),
                                         ((1 << 31) // 1023 + 1001, 16, 1023, BF16), ((1 << 31) // 256 + 777, 256, 16, BF16), ((1 << 31) // 256 + 777, 256, 12, F32),
                                         ((1 << 31) // 256 + 777, 256, 15, BF16)])
def test_route_backward_past_32_bit_offsets(cm, N, E, d, dtype):
    """Elements of x and dx, or of scores and dlogits, past 2^31: dlogits of the last tokens alone, of two slots of which one keeps a row."""
    n, at = 200, N - 200
    scores = torch.empty((N, E), device="cuda").fill_(1.0 / E)
    scores[at:] = torch.softmax(_normal((n, E), 1.0, F32, 1), 1)
    topk = torch.zeros((N, 2), device="cuda", dtype=torch.int32)
    topk[at:, 1] = 1 + torch.arange(n, device="cuda", dtype=torch.int32) % (E - 1)
    slot_row = torch.full((N, 2), -1, device="cuda", dtype=torch.int32)
    slot_row[at:, 1] = torch.randperm(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).int()
    x = torch.ones((N, d), device="cuda", dtype=dtype)
    x[at:] = _normal((n, d), 1.0, dtype, 3)
    w, dweight = _normal((E, d), 0.1, dtype, 4), _normal((n,), 1.0, F32, 5)
    got = cm.route_backward(x, w, scores, topk, slot_row, dweight, out_dtype=F32)
    ref = _route_ref(x[at:], w, scores[at:], topk[at:].long(), slot_row[at:], dweight, None, dtype)
    assert not bool(got["dlogits"][:at].any()) and not bool(got["dx"][:at].any())
    close(got["dlogits"][at:], *ref[0])
    close(got["dx"][at:], ref[1][0], rounded(*ref[1], dtype))
    close(got["dw"], ref[2][0], rounded(*ref[2], F32))
    close(got["dbias"], ref[3][0], rounded(*ref[3], F32))


def test_permute_fp8_past_32_bit_offsets(cm):
    """Tokens and rows whose codes lie past 2^32."""
    d, n = 4096, 100
    N, rows = (1 << 32) // d + 1000, (1 << 32) // d + 5000
    slots = 2
    q = torch.zeros((N, d), device="cuda", dtype=torch.uint8)
    q[N - n:] = torch.randint(0, 120, (n, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.uint8)
    sc = torch.randint(120, 130, (N, d // 128), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(torch.uint8)
    E = slots
    scores = torch.rand((N, E), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    topk = torch.arange(slots, device="cuda", dtype=torch.int32).repeat(N, 1)
    slot_row = torch.full((N, slots), -1, device="cuda", dtype=torch.int32)
    r = rows - 1 - torch.randperm(2000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))[:n]
    slot_row[N - n:, slots - 1] = r.int()
    got = cm.permute_fp8(q.view(cm.FP8), sc.view(cm.SCALE), scores, topk, slot_row, rows)
    assert torch.equal(got["x_q"].view(torch.uint8)[r], q[N - n:]) and torch.equal(got["x_scale"].view(torch.uint8)[r], sc[N - n:])
    assert torch.equal(got["perm_token"][r].long(), torch.arange(N - n, N, device="cuda")) and torch.equal(got["perm_weight"][r], scores[N - n:, slots - 1])


@pytest.mark.parametrize("E,d,dtype", [(8, 250, F32), (40, 96, F32), (64, 512, BF16), (33, 77, BF16)])
@pytest.mark.parametrize("ld", [0, 1, 37])
def test_rows_of_dscores_further_apart_than_experts(cm, E, d, dtype, ld):
    """The C entry point's dscores_ld: E + ld, or (0) the same row for every token."""
    N, k = 300, 2
    r, dr, rows = _routing(cm, N, E, k, 0, 3)
    x, w, dwt = _normal((N, d), 1.0, dtype, 1), _normal((E, d), 0.1, dtype, 2), _normal((rows,), 1.0, F32, 3)
    wide = torch.full((N, E + ld), float("nan"), device="cuda")
    wide[:, :E] = _normal((N, E), 0.3, F32, 4)
    dscores = wide[:, :E] if ld else wide[0, :E].expand(N, E)
    want = cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], dwt, dscores=dscores.contiguous())
    got = {key: torch.zeros_like(v) for key, v in want.items()}
    ws = torch.empty((cm.route_backward_workspace_bytes(N, d, E, dtype),), device="cuda", dtype=torch.uint8)
    p = lambda t: ctypes.c_void_p(t.data_ptr())                       # noqa: E731
    code = cm.F32 if dtype == F32 else cm.BF16
    rc = cm.lib().capmoe_route_backward(p(x), p(w), p(r["scores"]), p(r["topk_idx"]), p(dr["slot_row"]), p(dwt), N, d, E, k, k, 0, None, p(wide),
                                        E + ld if ld else 0, code, code, rows, p(got["dlogits"]), p(got["dx"]), p(got["dw"]), p(got["dbias"]), p(ws),
                                        ws.numel(), None, torch.cuda.current_stream().cuda_stream)
    assert rc == cm.OK
    torch.cuda.synchronize()
    assert all(torch.equal(got[key], want[key]) for key in want)


@pytest.mark.parametrize("N,E,d,dtype", [(300, 8, 38400, BF16), (700, 60, 38408, BF16), (300, 70, 19464, BF16), (300, 200, 19464, BF16), (300, 20, 19457, F32),
                                         (300, 100, 19458, F32), (1300, 20, 19457, BF16), (1300, 100, 19457, BF16), (300, 8, 152000, F32)])
def test_more_column_slices_than_sms(cm, N, E, d, dtype):
    r, dr, rows = _routing(cm, N, E, 2, 0, 3)
    x, w, dsc = _normal((N, d), 1.0, dtype, 1), _normal((E, d), 0.1, dtype, 2), _normal((E,), 0.3, F32, 4)
    dwt = _normal((rows,), 1.0, F32, 3)
    got = cm.route_backward(x, w, r["scores"], r["topk_idx"], dr["slot_row"], dwt, dscores=dsc, out_dtype=F32)
    ref = _route_ref(x, w, r["scores"], _expert_of(r, dr, E, 0), dr["slot_row"], dwt, dsc, dtype)
    close(got["dlogits"], *ref[0])
    close(got["dx"], ref[1][0], rounded(*ref[1], dtype))
    close(got["dw"], ref[2][0], rounded(*ref[2], F32))
    close(got["dbias"], ref[3][0], rounded(*ref[3], F32))
