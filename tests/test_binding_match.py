"""Every check of types and sizes in front of the operators around the expert products, by its own message: on a machine without a GPU a
call that passes them all still ends in the refusal of its device, with the same status."""
import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build

F32, BF16, F64, I32, I64 = torch.float32, torch.bfloat16, torch.float64, torch.int32, torch.int64
N, D, E, K, A = 4, 64, 8, 2, 6


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _t(*shape, dtype=F32, device="cpu"):
    return torch.zeros(shape, dtype=F32, device=device).to(dtype)


def calls(cm, device="cpu"):
    """name -> (call, good arguments, {argument: other values that must be refused}, words that the refusals of the wrapper hold)."""
    t = lambda *s, dtype=F32: _t(*s, dtype=dtype, device=device)      # noqa: E731
    f8, sc = cm.FP8, cm.SCALE
    lists = dict(scores=t(N, E), topk_idx=t(N, K, dtype=I32), slot_row=t(N, K, dtype=I32))
    bad_lists = dict(scores=[t(N, E, dtype=BF16), t(N + 1, E), t(N)], topk_idx=[t(N, K, dtype=I64), t(N - 1, K, dtype=I32), t(N, dtype=I32)],
                     slot_row=[t(N, K, dtype=I64), t(N + 1, K, dtype=I32), t(N, dtype=I32)], token_group=[t(N - 1, dtype=I32), t(N, dtype=I64), t(N, 1, dtype=I32)])
    return {
        "rms_norm": (cm.rms_norm, dict(x=t(N, D), w=t(D), residual=t(N, D)),
                     dict(x=[t(N, D, dtype=BF16), t(N, D + 1), t(N)], w=[t(D - 1), t(D, dtype=BF16), t(1, D)], residual=[t(N, D - 1), t(N + 1, D), t(N, D, dtype=BF16)],
                          out=[dict(y=t(N - 1, D)), dict(rstd=t(N + 1)), dict(h=t(N, D, dtype=BF16)), dict(rstd=t(N, dtype=F64))])),
        "rms_norm_codes": (cm.rms_norm, dict(x=t(N, D), w=t(D), fp8=True),
                           dict(out=[dict(q=t(N, D)), dict(q=t(N, D + 1, dtype=f8)), dict(scale=t(N, 2, dtype=sc)), dict(scale=t(N, 1))])),
        "rms_norm_backward": (cm.rms_norm_backward, dict(dy=t(N, D), h=t(N, D), w=t(D), rstd=t(N), dh=t(N, D)),
                              dict(dy=[t(N + 1, D), t(N, D - 1), t(N, D, dtype=BF16)], h=[t(N - 1, D), t(N, D, dtype=BF16), t(D)], w=[t(D + 1), t(D, dtype=BF16), t(1, D)],
                                   rstd=[t(N - 1), t(N, dtype=F64), t(N, 1)], dh=[t(N, D + 1), t(N - 1, D), t(N, D, dtype=BF16)],
                                   dx=[t(N - 1, D), t(N, D, dtype=BF16)], dw=[t(D - 1)])),
        "permute_fp8": (cm.permute_fp8, dict(x_q=t(N, D, dtype=f8), x_scale=t(N, 1, dtype=sc), **lists, A_max=A, token_group=t(N, dtype=I32)),
                        dict(x_q=[t(N, D), t(N - 1, D, dtype=f8), t(N, 3 * D, dtype=f8)], x_scale=[t(N, 2, dtype=sc), t(N - 1, 1, dtype=sc), t(N, 1)], **bad_lists,
                             out=[dict(x_q=t(A - 1, D, dtype=f8)), dict(x_scale=t(A, 2, dtype=sc)), dict(perm_token=t(A, dtype=I64)), dict(perm_weight=t(A + 1))])),
        "combine_backward": (cm.combine_backward, dict(dy=t(N, D), y_perm=t(A, D), slot_row=t(N, K, dtype=I32), perm_weight=t(A)),
                             dict(dy=[t(N + 1, D), t(N, D, dtype=BF16), t(D)], y_perm=[t(A, D - 4), t(A - 1, D), t(A, D, dtype=BF16)],
                                  slot_row=bad_lists["slot_row"], perm_weight=[t(A - 1), t(A, dtype=F64), t(A, 1)],
                                  dy_perm=[t(A - 1, D), t(A, D, dtype=BF16)], dweight=[t(A - 1), t(A, dtype=F64)])),
        "permute_backward": (cm.permute_backward, dict(dx_perm=t(A, D), slot_row=t(N, K, dtype=I32), add=(t(N, D), t(N, D))),
                             dict(dx_perm=[t(A, D + 4), t(A, D, dtype=BF16), t(D)], slot_row=bad_lists["slot_row"],
                                  add=[t(N + 1, D), (t(N, D), t(N, D - 4)), t(N, D, dtype=BF16)], dx=[t(N - 1, D), t(N, D, dtype=BF16)])),
        "route_backward": (cm.route_backward, dict(x=t(N, D), w_router=t(E, D), **lists, dweight=t(A), token_group=t(N, dtype=I32), dscores=t(N, E)),
                           dict(x=[t(N + 1, D), t(N, D - 1), t(N, D, dtype=BF16), t(D)], w_router=[t(E - 1, D), t(E, D + 1), t(E, D, dtype=BF16)], **bad_lists,
                                dweight=[t(A, dtype=F64), t(A, 1)], dscores=[t(N, E - 1), t(N + 1, E), t(E + 1), t(N, E, dtype=F64)],
                                out=[dict(dlogits=t(N, E - 1)), dict(dx=t(N, D, dtype=BF16)), dict(dw=t(E, D + 1)), dict(dbias=t(E, dtype=F64))])),
    }


NAMES = ["rms_norm", "rms_norm_codes", "rms_norm_backward", "permute_fp8", "combine_backward", "permute_backward", "route_backward"]


@pytest.mark.parametrize("name", NAMES)
def test_each_argument_that_does_not_fit_is_refused_for_that(cm, name):
    call, good, bad = calls(cm)[name]
    with pytest.raises(cm.CapmoeError, match="CUDA tensors on one device expected"):       # the only thing wrong with the good ones
        call(**good)
    for key, values in bad.items():
        for v in values:
            with pytest.raises(cm.CapmoeError) as err:
                call(**{**good, key: v})
            assert err.value.status == cm.EINVAL and "on one device" not in str(err.value), (key, str(err.value))


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_nothing_is_launched_for_arguments_that_do_not_fit(cm, name):
    """The same with CUDA tensors: a size that slipped through would be read out of range, so only refusals are tried here that the CPU
    test has shown."""
    call, good, bad = calls(cm, "cuda")[name]
    before = cm.launch_count()
    for key, values in bad.items():
        for v in values:
            with pytest.raises(cm.CapmoeError) as err:
                call(**{**good, key: v})
            assert err.value.status == cm.EINVAL, key
        for v in values[:1] if key not in ("out", "add") else ():                          # a tensor that stayed on the host
            with pytest.raises(cm.CapmoeError):
                call(**{**good, key: good[key].cpu() if key in good else v.cpu()})
    assert cm.launch_count() == before


def test_match_alone(cm):
    """A letter is one number wherever it stands, T one type, `?` may be None; anything else does not match."""
    match = cm._binding().match
    x, w = _t(3, 5), _t(5)
    assert match("T[N,d] T[d]", x, w) == (cm.F32, 3, 5)
    assert match("T[N,d] T[d] T?[N,d]", x.bfloat16(), w.bfloat16(), None) == (cm.BF16, 3, 5)
    assert match("i[N,k] f[N]", _t(3, 2, dtype=I32), _t(3)) == (-1, 3, 2)
    assert match("q[N,d] s[N,B]", _t(3, 129, dtype=cm.FP8), _t(3, 2, dtype=cm.SCALE)) == (-1, 3, 129)
    for pattern, args in (("T[N,d] T[d]", (x, _t(4))), ("T[N,d] T[d]", (x, w.bfloat16())), ("T[N,d] T[d]", (x, None)), ("T[N,d] T[d]", (x.half(), w.half())),
                          ("T[N,d] T[d]", (x.double(), w.double())), ("T[N,d] T[d]", (x, _t(1, 5))), ("T[N,d]", (_t(3),)), ("f[N]", (_t(3, dtype=BF16),)),
                          ("i[N]", (_t(3, dtype=I64),)), ("q[N]", (_t(3, dtype=torch.uint8),)), ("s[N]", (_t(3, dtype=torch.uint8),)), ("T[N,N]", (x,)),
                          ("q[N,d] s[N,B]", (_t(3, 128, dtype=cm.FP8), _t(3, 2, dtype=cm.SCALE))), ("T[N,d] T?[N,d]", (x, _t(3, 4))), ("T[d]", ([1.0],))):
        assert match(pattern, *args) is None, (pattern, [getattr(a, "shape", a) for a in args])
    with pytest.raises(TypeError):
        match("T[N,d] T[d]", x)
