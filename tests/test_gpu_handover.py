"""Tiles that one CTA of a pair takes from a counter and hands to the other: a hand-over that went wrong would leave half a
tile unwritten or mix it with another one.  Every call here has thousands of the shortest tiles, so millions of hand-overs
run in a test; the first call is held against a 64-bit definition, every later one, into buffers filled anew, has to give
the same bits."""
import pytest
import torch

import grouped_ref as R

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
E = 256


@pytest.fixture(scope="module")
def cm():
    from paper_2503_05066_b200 import capmoe
    capmoe.lib()
    return capmoe


@pytest.fixture
def forced(cm):
    yield lambda name: cm.debug_ffn_variant(name)
    cm.debug_ffn_variant("auto")


def _normal(shape, std, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=BF16).normal_(0, std, generator=g)


def _repeat(cm, calls, outs, run, first):
    """run(status block) into `outs`, again and again; first() checks what the first call left there."""
    st = torch.zeros(cm.FFN_STATUS_WORDS, device="cuda", dtype=torch.int32)
    same = torch.ones((), device="cuda", dtype=torch.bool)
    want = None
    for _ in range(calls):
        for t in outs:
            t.fill_(7.0)
        run(st)
        if want is None:
            first()
            want = [t.clone() for t in outs]
        for t, w in zip(outs, want):
            same &= (t == w).all()
    assert int(st[0]) == 0 and bool(same)


@pytest.mark.parametrize("d,F", [(64, 4096), (4096, 64)])
@pytest.mark.parametrize("form", ["pair", "short"])
def test_ffn(cm, forced, form, d, F):
    """One row per expert: 4096 tiles and more of one k-block in the gate/up launch (in the down launch with d = 4096)."""
    forced(form)
    off = torch.arange(E + 1, device="cuda", dtype=torch.int32)
    x = _normal((E, d), 1.0, 1)
    w = [_normal((E, *s), 0.4 / d ** 0.5, 2 + i) for i, s in enumerate(((F, d), (F, d), (d, F)))]
    h, y = torch.empty((E, F), device="cuda", dtype=BF16), torch.empty((E, d), device="cuda", dtype=BF16)

    def first():
        for e in range(E):
            wg, wu, wd = (t[e].double() for t in w)
            _, _, ref, err = R.swiglu(x[e:e + 1].double(), wg, wu)
            R.close(h[e:e + 1], ref, R.rounded(ref, err, BF16))
            R.close(y[e:e + 1], *R.product(h[e:e + 1].double(), wd, BF16))

    _repeat(cm, 3000, [h, y], lambda st: cm.grouped_ffn(x, off, *w, h_ws=h, y_perm=y, dev_status=st), first)
