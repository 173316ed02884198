"""What the norm, the 8-bit permute and the gradients around the expert products refuse, on a machine without a GPU: every bad
call returns its status before anything is launched (no pointer here is ever dereferenced)."""
import ctypes

import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build

Z, P = ctypes.c_void_p(0), ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)                     # not 16-byte aligned
I = ctypes.c_int64
BIG = ctypes.c_size_t(1 << 40)


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _calls(cm):
    """name -> (call, good arguments)."""
    L = cm.lib()
    f = ctypes.c_float
    return {
        "norm": (L.capmoe_rms_norm, dict(x=P, res=P, w=P, N=I(8), d=64, dt=1, eps=f(1e-6), h=P, y=P, rstd=P, q=P, sc=P, s=Z)),
        "norm_bwd": (L.capmoe_rms_norm_backward, dict(dy=P, h=P, w=P, rstd=P, dh=P, N=I(8), d=64, dt=1, odt=1, dx=P, dw=P, ws=P, wsb=BIG, s=Z)),
        "perm8": (L.capmoe_permute_fp8, dict(x=P, xs=P, N=I(8), d=64, E=4, k=2, slots=2, D=0, rows=I(16), sc=P, idx=P, tg=Z, sr=P, q=P, qs=P,
                                             pt=P, pw=P, st=Z, s=Z)),
        "comb_bwd": (L.capmoe_combine_backward, dict(dy=P, yp=P, sr=P, pw=P, N=I(8), d=64, slots=2, dt=1, rows=I(16), dyp=P, dwt=P, s=Z)),
        "perm_bwd": (L.capmoe_permute_backward, dict(dxp=P, sr=P, N=I(8), d=64, slots=2, dt=1, rows=I(16), a=P, b=P, dx=P, s=Z)),
        "route_bwd": (L.capmoe_route_backward, dict(x=P, w=P, sc=P, idx=P, sr=P, dwt=P, N=I(8), d=64, E=4, k=2, slots=2, D=0, tg=Z, ds=Z, ld=I(0), dt=1,
                                                    odt=1, rows=I(16), dl=P, dx=P, dw=P, db=P, ws=P, wsb=BIG, st=Z, s=Z)),
        "ffn8_codes": (L.capmoe_grouped_ffn_fp8_codes, dict(x=P, xs=P, off=P, E=4, d=64, F=64, wg=P, wgs=P, wu=P, wus=P, wd=P, wds=P, y=P, rows=I(8), ws=P,
                                                            wsb=BIG, st=Z, s=Z)),
    }


MAY_BE_ABSENT = {"norm": ("rstd",), "norm_bwd": ("dh",), "perm_bwd": ("a", "b")}
ANY_ALIGNMENT = {"norm": ("rstd", "sc"), "norm_bwd": ("rstd", "dw"), "perm8": ("xs", "sc", "idx", "sr", "qs", "pt", "pw"), "comb_bwd": ("sr", "pw", "dwt"),
                 "perm_bwd": ("sr",), "route_bwd": ("sc", "idx", "sr", "dwt", "db"), "ffn8_codes": ("xs", "off", "wgs", "wus", "wds")}


@pytest.mark.parametrize("name", ["norm", "norm_bwd", "perm8", "comb_bwd", "perm_bwd", "route_bwd", "ffn8_codes"])
def test_bad_arguments(cm, name):
    fn, good = _calls(cm)[name]
    before = cm.launch_count()

    def status(**change):
        return fn(*{**good, **change}.values())

    for key in ("d", "E", "F", "k"):
        if key in good:
            assert status(**{key: 0}) == cm.EINVAL and status(**{key: -1}) == cm.EINVAL, key
    count = "rows" if name == "ffn8_codes" else "N"
    assert status(**{count: I(-1)}) == cm.EINVAL
    if "rows" in good:
        assert status(rows=I(-1)) == cm.EINVAL and status(rows=I(1 << 31)) == cm.EUNSUPPORTED
    if "dt" in good:
        assert status(dt=2) == cm.EUNSUPPORTED
    if "odt" in good:
        assert status(odt=5) == cm.EUNSUPPORTED and status(dt=0, odt=1) == cm.EUNSUPPORTED
    for key, v in good.items():
        if v is P:
            if key not in MAY_BE_ABSENT.get(name, ()):
                assert status(**{key: Z}) == cm.EINVAL, key
            if key not in ANY_ALIGNMENT[name]:
                assert status(**{key: ODD}) == cm.EINVAL, key
    if "wsb" in good:
        assert status(wsb=ctypes.c_size_t(0)) == cm.EWORKSPACE
    if name not in ("norm_bwd", "route_bwd"):                       # (those write zeros then)
        assert status(**{count: I(0)}) == cm.OK
    assert cm.launch_count() == before


def test_sizes_and_lists(cm):
    calls = _calls(cm)

    def status(name, **change):
        fn, good = calls[name]
        return fn(*{**good, **change}.values())

    before = cm.launch_count()
    f = ctypes.c_float
    assert status("norm", d=16385) == cm.EUNSUPPORTED and status("norm_bwd", d=16385) == cm.EUNSUPPORTED
    assert status("norm", eps=f(-1.0)) == cm.EINVAL and status("norm", eps=f(float("nan"))) == cm.EINVAL
    assert status("norm", h=Z) == cm.EINVAL and status("norm", res=Z) == cm.EINVAL       # h comes with a residual
    assert status("norm", q=Z) == cm.EINVAL and status("norm", sc=Z) == cm.EINVAL
    for name in ("perm8", "route_bwd"):
        assert status(name, k=5) == cm.EINVAL and status(name, D=-1) == cm.EINVAL
        assert status(name, slots=3) == cm.EINVAL and status(name, D=3, slots=3) == cm.EINVAL and status(name, D=2, slots=2) == cm.EINVAL
    assert status("perm8", d=72) == cm.EUNSUPPORTED                 # rows of whole 16-byte vectors
    assert status("comb_bwd", d=60) == cm.EUNSUPPORTED and status("perm_bwd", d=60) == cm.EUNSUPPORTED
    assert status("comb_bwd", slots=0) == cm.EINVAL and status("comb_bwd", slots=289) == cm.EUNSUPPORTED
    assert status("perm_bwd", slots=0) == cm.EINVAL and status("perm_bwd", slots=289) == cm.EUNSUPPORTED
    assert status("comb_bwd", N=I(1 << 31)) == cm.EUNSUPPORTED and status("perm_bwd", N=I(1 << 31)) == cm.EUNSUPPORTED
    assert status("route_bwd", E=257) == cm.EUNSUPPORTED and status("route_bwd", N=I(1 << 31)) == cm.EUNSUPPORTED
    assert status("route_bwd", E=64, k=33, slots=33) == cm.EUNSUPPORTED
    assert status("route_bwd", ds=P, ld=I(3)) == cm.EINVAL and status("route_bwd", ds=P, ld=I(-4)) == cm.EINVAL
    assert status("ffn8_codes", E=257) == cm.EUNSUPPORTED
    n = ctypes.c_size_t(0)
    L = cm.lib()
    assert L.capmoe_rms_norm_backward_workspace_bytes(I(8), 64, 1, None) == cm.EINVAL
    assert L.capmoe_rms_norm_backward_workspace_bytes(I(8), 0, 1, ctypes.byref(n)) == cm.EINVAL
    assert L.capmoe_route_backward_workspace_bytes(I(8), 64, 257, 1, ctypes.byref(n)) == cm.EUNSUPPORTED
    assert L.capmoe_route_backward_workspace_bytes(I(8), 64, 4, 1, None) == cm.EINVAL
    assert cm.rms_norm_backward_workspace_bytes(0, 64, torch.float32) == 0
    assert cm.route_backward_workspace_bytes(16384, 2048, 64, torch.bfloat16) > 0
    assert cm.launch_count() == before


def test_the_binding_refuses_before_the_library(cm):
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)      # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)                     # noqa: E731

    def refused(status, fn, *a, **k):
        with pytest.raises(cm.CapmoeError) as e:
            fn(*a, **k)
        assert e.value.status == status

    x, w = t(4, 64), t(64)
    refused(cm.EINVAL, cm.rms_norm, x, t(63))
    refused(cm.EINVAL, cm.rms_norm, x, t(64, dtype=torch.bfloat16))
    refused(cm.EINVAL, cm.rms_norm, x, w, t(4, 63))
    refused(cm.EINVAL, cm.rms_norm, x, w, out=dict(y=t(3, 64)))
    refused(cm.EINVAL, cm.rms_norm, x, w)                                # not on a GPU
    refused(cm.EUNSUPPORTED, cm.rms_norm, x.half(), w.half())
    refused(cm.EINVAL, cm.rms_norm_backward, x, x, w, t(3))
    refused(cm.EINVAL, cm.rms_norm_backward, t(4, 60), x, w, t(4))
    refused(cm.EINVAL, cm.combine_backward, x, t(8, 60), i(4, 2), t(8))
    refused(cm.EINVAL, cm.combine_backward, x, t(8, 64), i(3, 2), t(8))
    refused(cm.EINVAL, cm.combine_backward, x, t(8, 64), i(4, 2), t(7))
    refused(cm.EINVAL, cm.permute_backward, t(8, 64), i(4, 2), add=t(5, 64))
    refused(cm.EUNSUPPORTED, cm.permute_backward, t(8, 64), i(4, 2), add=(x, x, x))
    lists = (t(4, 8), i(4, 2), i(4, 2))
    refused(cm.EINVAL, cm.route_backward, x, t(7, 64), *lists, t(8))
    refused(cm.EINVAL, cm.route_backward, x, t(8, 64), *lists, t(8).double())
    refused(cm.EINVAL, cm.route_backward, x, t(8, 64), *lists, t(8), dscores=t(7))
    refused(cm.EINVAL, cm.route_backward, x, t(8, 64), *lists, t(8), token_group=i(3))
    refused(cm.EINVAL, cm.permute_fp8, x, t(4, 1), *lists, 8)
    refused(cm.EINVAL, cm.grouped_ffn_fp8, (x, x), i(5), (t(4, 8, 64), x), (x, x), (x, x))


def test_the_compiled_binding_takes_what_the_entry_points_take(cm):
    """Types and ranges of its arguments, on calls that end in a check of the library or before it."""
    run = cm._binding().run
    x = torch.zeros((4, 64))
    with pytest.raises(TypeError):
        run("capmoe_rms_norm")
    with pytest.raises(TypeError):
        run("capmoe_nothing", x)
    with pytest.raises(TypeError):
        run("capmoe_rms_norm", x, x)                                     # too few
    assert run("capmoe_rms_norm", x, *([None] * 12)) is None             # not on a GPU: nothing is looked at
