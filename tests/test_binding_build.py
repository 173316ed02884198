"""The compiled binding belongs to one interpreter and one torch; the library does not."""
import os
import sysconfig

import pytest
import torch

from paper_2503_05066_b200 import build as capmoe_build


@pytest.fixture(scope="module")
def cm():
    capmoe_build.build()
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


def test_another_torch_or_interpreter_has_a_binding_of_its_own(cm, monkeypatch):
    here = capmoe_build.bind_path()
    assert os.path.exists(here)
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0")
        assert capmoe_build.bind_path() != here
    with monkeypatch.context() as m:
        m.setattr(sysconfig, "get_config_var", lambda name: "cpython-300")
        assert capmoe_build.bind_path() != here
    assert capmoe_build.bind_path() == here


def test_a_binding_that_is_up_to_date_but_another_torch_s_is_built(cm, monkeypatch, tmp_path):
    built = tmp_path / "_bind.other.so"
    calls = []

    def command():
        calls.append(1)
        return ["touch", str(built)]

    monkeypatch.setattr(capmoe_build, "_bind_cmd", command)
    capmoe_build.build()
    assert not calls                                                     # this torch's is there
    monkeypatch.setattr(capmoe_build, "bind_path", lambda: str(built))
    capmoe_build.build()
    assert calls == [1] and built.exists()
    capmoe_build.build()
    assert calls == [1]


def test_without_a_binding(cm, monkeypatch, tmp_path):
    """The grouped products go by ctypes, with the same refusals; the operators that need the binding say what is missing."""
    monkeypatch.setattr(cm, "_bind", None)
    monkeypatch.setattr(cm, "bind_path", lambda: str(tmp_path / "_bind.none.so"))
    x, off = torch.zeros((4, 64)), torch.zeros((3,), dtype=torch.int32)
    with pytest.raises(cm.CapmoeError, match="CUDA tensors on one device expected"):
        cm.grouped_mm(x, off, torch.zeros((2, 8, 64)))
    with pytest.raises(RuntimeError, match="_bind.none.so is missing"):
        cm.rms_norm(x, torch.zeros((64,)))


@pytest.mark.gpu
def test_grouped_products_without_a_binding_on_a_gpu(cm, monkeypatch, tmp_path):
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.empty(s, device="cuda").normal_(0, 1, generator=g).bfloat16()      # noqa: E731
    x, w, off = n(200, 128), n(3, 64, 128), torch.tensor([0, 70, 70, 200], device="cuda", dtype=torch.int32)
    q = cm.quantize_rows(x)
    want = (cm.grouped_mm(x, off, w), cm.grouped_mm_dw(n(200, 64), x, off), q[0].view(torch.uint8))
    g.manual_seed(1)
    x, w = n(200, 128), n(3, 64, 128)
    monkeypatch.setattr(cm, "_bind", None)
    monkeypatch.setattr(cm, "bind_path", lambda: str(tmp_path / "_bind.none.so"))
    got = (cm.grouped_mm(x, off, w), cm.grouped_mm_dw(n(200, 64), x, off), cm.quantize_rows(x)[0].view(torch.uint8))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(cm.CapmoeError, match="CUDA tensors on one device expected"):
        cm.grouped_mm(x, off, w.cpu())


def test_a_refused_call_leaves_no_size_for_its_device(cm, monkeypatch):
    """Sizes come from the current device's SM count and are remembered for the tensors' device: a call that is refused because the two
    differ must not leave one behind."""
    class On1(torch.Tensor):
        def get_device(self):
            return 1

    current, seen = [0], []

    class Bind:
        match = staticmethod(lambda pattern, *tensors: cm_match(pattern, *tensors))

        @staticmethod
        def new(like, dtype, *sizes):
            t = torch.empty(sizes or like.shape, dtype=dtype or like.dtype)
            if dtype == torch.uint8:
                seen.append(t.numel())
            return t.as_subclass(On1)

        @staticmethod
        def run(name, like, *args):
            return None if current[0] != like.get_device() else 0

    cm_match = cm._binding().match
    monkeypatch.setattr(cm, "_bind", Bind)
    monkeypatch.setattr(cm, "_bytes", lambda fn, *args: 512 + 1000 * current[0])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    f, i = (lambda *s: torch.zeros(s).as_subclass(On1)), (lambda *s: torch.zeros(s, dtype=torch.int32).as_subclass(On1))
    calls = [lambda: cm.rms_norm_backward(f(4, 64), f(4, 64), f(64), f(4)),
             lambda: cm.route_backward(f(4, 64), f(8, 64), f(4, 8), i(4, 2), i(4, 2), f(8))]
    for call in calls:
        current[0] = 0
        with pytest.raises(cm.CapmoeError, match="tensors on cuda:1, but cuda:0 is the current device"):
            call()
        current[0] = 1
        call()
    cm._norm_backward_bytes.cache_clear()
    cm._route_backward_bytes.cache_clear()
    assert seen == [512, 1512, 512, 1512]
