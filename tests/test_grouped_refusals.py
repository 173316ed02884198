"""What the grouped products refuse, on a machine without a GPU: every bad call returns its status before anything
is launched (no pointer here is ever dereferenced)."""
import ctypes

import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build

Z, P = ctypes.c_void_p(0), ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)                     # not 16-byte aligned
I = ctypes.c_int64
S = ctypes.c_size_t


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def _calls(cm):
    """name -> (call, good arguments); every argument list is complete and valid."""
    L = cm.lib()
    big = S(1 << 40)
    return {
        "mm": (L.capmoe_grouped_mm, dict(x=P, off=P, w=P, E=4, d=64, n=64, dt=1, y=P, rows=I(8), st=Z, s=Z)),
        "dx": (L.capmoe_grouped_mm_dx, dict(x=P, off=P, w=P, E=4, d=64, n=64, dt=1, y=P, rows=I(8), st=Z, s=Z)),
        "dw": (L.capmoe_grouped_mm_dw, dict(dy=P, x=P, off=P, E=4, d=64, n=64, dt=1, odt=1, y=P, rows=I(8), ws=P, wsb=big, st=Z, s=Z)),
        "bwd": (L.capmoe_grouped_ffn_backward, dict(x=P, dy=P, off=P, E=4, d=64, n=64, dt=1, wg=P, wu=P, wd=P, y=P, a=P, b=P, c=P,
                                                    rows=I(8), ws=P, wsb=big, st=Z, s=Z)),
        "mm8": (L.capmoe_grouped_mm_fp8, dict(x=P, xs=P, off=P, w=P, wsc=P, E=4, d=64, n=64, y=P, rows=I(8), st=Z, s=Z)),
        "ffn8": (L.capmoe_grouped_ffn_fp8, dict(x=P, off=P, E=4, d=64, n=64, wg=P, wgs=P, wu=P, wus=P, wd=P, wds=P, y=P, rows=I(8),
                                                ws=P, wsb=big, st=Z, s=Z)),
    }


@pytest.mark.parametrize("name", ["mm", "dx", "dw", "bwd", "mm8", "ffn8"])
def test_bad_arguments(cm, name):
    fn, good = _calls(cm)[name]
    before = cm.launch_count()

    def status(**change):
        return fn(*{**good, **change}.values())

    for key in ("E", "d", "n"):
        assert status(**{key: 0}) == cm.EINVAL and status(**{key: -1}) == cm.EINVAL, key
    assert status(rows=I(-1)) == cm.EINVAL
    assert status(E=257) == cm.EUNSUPPORTED
    assert status(rows=I(1 << 31)) == cm.EUNSUPPORTED
    if "dt" in good:
        assert status(dt=2) == cm.EUNSUPPORTED
    for key, v in good.items():
        if v is P:
            assert status(**{key: Z}) == cm.EINVAL, key
            if key not in ("off", "xs", "wsc", "wgs", "wus", "wds"):
                assert status(**{key: ODD}) == cm.EINVAL, key
    if "wsb" in good:
        assert status(wsb=S(0)) == cm.EWORKSPACE
    if name == "dw":
        assert status(odt=5) == cm.EUNSUPPORTED and status(dt=0, odt=1) == cm.EUNSUPPORTED
    if name in ("mm", "dx", "mm8", "ffn8"):
        assert status(rows=I(0)) == cm.OK            # nothing to do
    assert cm.launch_count() == before


def test_quantisers(cm):
    L = cm.lib()
    before = cm.launch_count()
    assert L.capmoe_quantize_rows(P, Z, I(-1), 64, 1, P, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_rows(P, Z, I(4), 0, 1, P, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_rows(P, Z, I(4), 64, 3, P, P, Z) == cm.EUNSUPPORTED
    assert L.capmoe_quantize_rows(P, Z, I(1 << 31), 64, 1, P, P, Z) == cm.EUNSUPPORTED
    assert L.capmoe_quantize_rows(Z, Z, I(4), 64, 1, P, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_rows(ODD, Z, I(4), 64, 1, P, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_rows(P, Z, I(4), 64, 1, Z, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_rows(P, Z, I(4), 64, 1, P, Z, Z) == cm.EINVAL
    assert L.capmoe_quantize_rows(Z, Z, I(0), 64, 1, Z, Z, Z) == cm.OK
    for E, n, d in ((0, 8, 8), (1, 0, 8), (1, 8, 0)):
        assert L.capmoe_quantize_weights(P, E, n, d, 1, P, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_weights(P, 1, 8, 8, 9, P, P, Z) == cm.EUNSUPPORTED
    assert L.capmoe_quantize_weights(Z, 1, 8, 8, 1, P, P, Z) == cm.EINVAL
    assert L.capmoe_quantize_weights(P, 1, 8, 8, 1, ODD, P, Z) == cm.EINVAL
    assert cm.launch_count() == before


def test_workspace_sizes(cm):
    assert cm.ffn_backward_workspace_bytes(1000, 8, 96, torch.bfloat16) >= 3 * 1000 * 96 * 2
    assert cm.ffn_backward_workspace_bytes(1000, 8, 96, torch.float32) >= 3 * 1000 * 96 * 4
    assert cm.ffn_fp8_workspace_bytes(1000, 256, 96) >= 1000 * (256 + 2 + 96 + 1)
    L = cm.lib()
    out = S(0)
    assert L.capmoe_ffn_backward_workspace_bytes(I(-1), 4, 4, 1, ctypes.byref(out)) == cm.EINVAL
    assert L.capmoe_ffn_backward_workspace_bytes(I(1), 4, 4, 7, ctypes.byref(out)) == cm.EUNSUPPORTED
    assert L.capmoe_ffn_backward_workspace_bytes(I(1), 4, 4, 1, Z) == cm.EINVAL
    assert L.capmoe_grouped_mm_dw_workspace_bytes(0, ctypes.byref(out)) == cm.EINVAL
    assert L.capmoe_ffn_fp8_workspace_bytes(I(1), 0, 4, ctypes.byref(out)) == cm.EINVAL


def test_binding_checks_shapes_and_types(cm):
    """The binding refuses tensors that do not fit together before it asks for a device."""
    bf, f32 = torch.bfloat16, torch.float32
    off = torch.zeros(3, dtype=torch.int32)
    x, w = torch.zeros((4, 64), dtype=bf), torch.zeros((2, 32, 64), dtype=bf)
    dy = torch.zeros((4, 32), dtype=bf)
    q8, s8 = torch.zeros((4, 64)).to(cm.FP8), torch.ones((4, 1)).to(cm.SCALE)
    w8 = (torch.zeros((2, 32, 64)).to(cm.FP8), torch.ones((2, 1, 1)).to(cm.SCALE))
    d8 = (torch.zeros((2, 64, 32)).to(cm.FP8), torch.ones((2, 1, 1)).to(cm.SCALE))
    wd = torch.zeros((2, 64, 32), dtype=bf)
    bad = [
        lambda: cm.grouped_mm(x, off.long(), w), lambda: cm.grouped_mm(x, off[:2], w), lambda: cm.grouped_mm(x.float(), off, w),
        lambda: cm.grouped_mm(x[:, :32], off, w), lambda: cm.grouped_mm(x, off, w, y=torch.zeros((4, 33), dtype=bf)),
        lambda: cm.grouped_mm(x, off, w, y=torch.zeros((4, 32), dtype=f32)),
        lambda: cm.grouped_mm_dx(x, off, w), lambda: cm.grouped_mm_dw(dy[:3], x, off), lambda: cm.grouped_mm_dw(dy.float(), x, off),
        lambda: cm.grouped_ffn_backward(x, dy, off, w, w, wd), lambda: cm.grouped_ffn_backward(x, x, off, w, w, w),
        lambda: cm.grouped_ffn_backward(x, x, off, w, w, wd.float()),
        lambda: cm.quantize_rows(x[0]), lambda: cm.quantize_weights(x), lambda: cm.quantize_rows(x, out=(q8, s8[:3])),
        lambda: cm.grouped_mm_fp8(x, s8, off, *w8), lambda: cm.grouped_mm_fp8(q8, s8.float(), off, *w8),
        lambda: cm.grouped_mm_fp8(q8, s8, off, w8[0], s8), lambda: cm.grouped_ffn_fp8(x.float(), off, w8, w8, d8),
        lambda: cm.grouped_ffn_fp8(x, off, w8, w8, w8),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(cm.CapmoeError) as err:
            call()
        assert err.value.status == cm.EINVAL, i
    with pytest.raises(cm.CapmoeError) as err:
        cm.quantize_rows(torch.zeros((2, 8), dtype=torch.float16), out=(torch.zeros((2, 8)).to(cm.FP8), torch.ones((2, 1)).to(cm.SCALE)))
    assert err.value.status in (cm.EUNSUPPORTED, cm.EINVAL)


def test_strided_offsets_are_refused(cm):
    with pytest.raises(AssertionError, match="contiguous"):
        cm.quantize_rows(torch.zeros((4, 64)), offsets=torch.zeros(10, dtype=torch.int32)[::2])


def test_split_bytes_refuses_bad_sizes(cm):
    out = ctypes.c_size_t(1)
    good = dict(rows=I(1 << 20), E=2, d=512, n=512, dt=1, products=1)
    for change in (dict(rows=I(-1)), dict(E=0), dict(d=0), dict(n=0), dict(products=0), dict(products=4)):
        assert cm.lib().capmoe_dw_split_bytes(*{**good, **change}.values(), ctypes.byref(out)) == cm.EINVAL
    assert cm.lib().capmoe_dw_split_bytes(*good.values(), None) == cm.EINVAL
    assert cm.lib().capmoe_dw_split_bytes(*{**good, "d": 33}.values(), ctypes.byref(out)) == cm.OK and out.value == 0


@pytest.mark.parametrize("name", ["mm", "dx", "dw", "bwd", "mm8", "ffn8"])
def test_rows_that_round_up_past_32_bits(cm, name):
    """Segments are rounded up to whole tiles in 32 bits: the last 511 row counts below 2^31 are refused."""
    fn, good = _calls(cm)[name]
    before = cm.launch_count()
    for rows in ((1 << 31) - 511, (1 << 31) - 1):
        assert fn(*{**good, "rows": I(rows)}.values()) == cm.EUNSUPPORTED
    assert cm.launch_count() == before


def test_quantisers_refuse_sizes_that_pass_32_bits(cm):
    """Columns (rows of a weight) are rounded up to whole warps' shares in 32 bits."""
    L = cm.lib()
    before = cm.launch_count()
    for v in ((1 << 31) - 1023, (1 << 31) - 1):
        for dt in (cm.F32, cm.BF16):
            assert L.capmoe_quantize_rows(P, Z, I(1), v, dt, P, P, Z) == cm.EUNSUPPORTED
            assert L.capmoe_quantize_weights(P, 1, v, 1, dt, P, P, Z) == cm.EUNSUPPORTED
            assert L.capmoe_quantize_weights(P, 1, 1, v, dt, P, P, Z) == cm.EUNSUPPORTED
    assert cm.launch_count() == before


def test_binding_refuses_sizes_that_do_not_fit_a_c_int(cm):
    """2^32 + 64 columns must not reach the library as 64."""
    bf, i32, big = torch.bfloat16, torch.int32, (1 << 32) + 64

    def meta(*shape, dtype=bf):
        return torch.empty(shape, device="meta", dtype=dtype)

    off = meta(3, dtype=i32)
    w8 = (meta(2, 64, big, dtype=cm.FP8), meta(2, 1, big // 128 + 1, dtype=cm.SCALE))
    d8 = (meta(2, big, 64, dtype=cm.FP8), meta(2, big // 128 + 1, 1, dtype=cm.SCALE))
    calls = [
        lambda: cm.grouped_mm(meta(4, big), off, meta(2, 64, big)), lambda: cm.grouped_mm(meta(4, 64), off, meta(2, big, 64)),
        lambda: cm.grouped_mm_dx(meta(4, big), off, meta(2, big, 64)), lambda: cm.grouped_mm_dw(meta(4, big), meta(4, 64), off),
        lambda: cm.grouped_ffn_backward(meta(4, 64), meta(4, 64), off, meta(2, big, 64), meta(2, big, 64), meta(2, 64, big)),
        lambda: cm.quantize_rows(meta(4, big)), lambda: cm.quantize_weights(meta(2, big, 64)),
        lambda: cm.quantize_weights(meta(2, 64, big)), lambda: cm.quantize_weights(meta(big, 64, 64)),
        lambda: cm.grouped_mm_fp8(meta(4, big, dtype=cm.FP8), meta(4, big // 128 + 1, dtype=cm.SCALE), off, *w8),
        lambda: cm.grouped_ffn_fp8(meta(4, 64), off, d8, d8, w8),
        lambda: cm.grouped_mm(meta(4, 64), meta((1 << 32) + 3, dtype=i32), meta((1 << 32) + 2, 64, 64)),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(cm.CapmoeError) as err:
            call()
        assert err.value.status == cm.EUNSUPPORTED, i


def test_workspaces_are_sized_for_their_device(cm, monkeypatch):
    """The size depends on the device's SM count: one device's must not serve another."""
    class On(torch.Tensor):
        index = 0

        def get_device(self):
            return On.index

    sizes = {"capmoe_grouped_mm_dw_workspace_bytes": 512, "capmoe_ffn_backward_workspace_bytes": 512, "capmoe_dw_split_bytes": 0}
    seen = []
    monkeypatch.setattr(cm, "_bytes", lambda fn, *args: sizes[fn] + (On.index + 1) * 1000)
    monkeypatch.setattr(cm, "_run", lambda name, like, *args: seen.append(next(v for v in args if isinstance(v, torch.Tensor) and
                                                                              v.dtype == torch.uint8).numel()))
    off = torch.zeros(4, dtype=torch.int32)
    x, w, wd = torch.zeros((17, 24)).as_subclass(On), torch.zeros((3, 40, 24)), torch.zeros((3, 24, 40))
    for On.index in (0, 1, 0, 1):
        cm.grouped_mm_dw(x, x, off)
        cm.grouped_ffn_backward(x, x, off, w, w, wd)
    cm._dw_bytes.cache_clear()
    cm._ffn_backward_bytes.cache_clear()
    assert seen == [2512, 2512, 4512, 4512] * 2
