"""The recurrence with given coefficients above one: what is zero passes products of any size, and products within f32's range lose nothing."""
import numpy as np
import pytest

from oracle import learn_oracle as orc
from tests.learn_util import check

pytestmark = pytest.mark.gpu

# within a wavefront, a workgroup, a workgroup's chunks in turn, chunks that hand on, groups of chunks that hand on, one channel
SHAPES = [(3, 40, 12), (2, 600, 12), (300, 1400, 64), (1, 5000, 4), (1, 9000, 64), (1, 9000, 1)]


def _n(t):
    return None if t is None else t.double().cpu().numpy()


def _both(gate, u, dh, first=None, h0=None):
    from paper_2502_20168_amd import learn
    f = learn.ssm_gated_scan_fwd(gate, u, first, h0, linear=True)
    return f, learn.ssm_gated_scan_bwd(gate, u, first, h0, f["carry"], dh, linear=True)


@pytest.mark.parametrize("value", (2.0, -1.3, 1e20))
@pytest.mark.parametrize("Bt,L,D", SHAPES)
def test_padding_in_front_of_a_sequence(Bt, L, D, value):
    """Steps of a zero input from a zero state, then an episode that decays: with a reset where it begins, and (forwards) without."""
    import torch
    gen = torch.Generator().manual_seed(1)
    start = L - 30
    gate, u, dh = torch.full((Bt, L, D), value), torch.zeros(Bt, L, D), torch.zeros(Bt, L, D)
    gate[:, start:] = 0.5
    u[:, start:], dh[:, start:] = torch.randn(Bt, 30, D, generator=gen), torch.randn(Bt, 30, D, generator=gen)
    first = torch.zeros(Bt, L, dtype=torch.uint8)
    first[:, start] = 1
    gate, u, dh, first = (t.cuda() for t in (gate, u, dh, first))
    f, b = _both(gate, u, dh, first)
    part = [_n(t[:, start:]) for t in (gate, u, first, dh)]
    h = orc.gated_fwd(*part[:3], linear=True)
    g = orc.gated_bwd(part[0], part[1], part[2], None, part[3], linear=True)
    for t in (f["h"], b["dgate"], b["du"]):
        assert not t[:, :start].any()
    check(f["h"][:, start:], h, 1e-6, "h")
    check(f["h_last"], h[:, -1], 1e-6, "h_last")
    check(b["dgate"][:, start:], g["dgate"], 1e-6, "dgate")
    check(b["du"][:, start:], g["du"], 1e-6, "du")
    assert not b["dh0"].any()
    f, _ = _both(gate, u, dh)
    assert not f["h"][:, :start].any()
    check(f["h"][:, start:], h, 1e-6, "h without a reset")


@pytest.mark.parametrize("Bt,L,D", SHAPES)
def test_products_up_to_the_range(Bt, L, D):
    """Coefficients of either sign that multiply up to 2^100, down again and up: states and gradients element by element."""
    import torch
    gen = torch.Generator().manual_seed(3)
    up = (torch.arange(L) // 100) % 2 == 0
    gate = torch.where(up, 2.0, 0.5)[None, :, None] * torch.where(torch.rand(Bt, L, D, generator=gen) < 0.3, -1.0, 1.0)
    u, dh = torch.zeros(Bt, L, D), torch.zeros(Bt, L, D)
    dh[:, -1] = 1.0 + torch.rand(Bt, D, generator=gen)
    h0 = 1.0 + torch.rand(Bt, D, generator=gen)
    f, b = _both(gate.cuda(), u.cuda(), dh.cuda(), None, h0.cuda())
    h = orc.gated_fwd(_n(gate), _n(u), None, _n(h0), linear=True)
    g = orc.gated_bwd(_n(gate), _n(u), None, _n(h0), _n(dh), linear=True)
    for got, ref in ((f["h"], h), (b["dgate"], g["dgate"]), (b["du"], g["du"]), (b["dh0"], g["dh0"])):
        assert np.all(np.abs(_n(got) - ref) <= 1e-6 * np.abs(ref))


@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
@pytest.mark.parametrize("Bt,L,D", SHAPES)
def test_a_coefficient_that_is_not_finite(Bt, L, D, bad):
    """It is no product: beside a zero state it makes NaN, as the definition does."""
    import torch
    gate, u, dh = torch.full((Bt, L, D), 0.5), torch.zeros(Bt, L, D), torch.zeros(Bt, L, D)
    gate[0, 21, 0] = bad
    f, b = _both(gate.cuda(), u.cuda(), dh.cuda())
    assert torch.isnan(f["h"][0, 21:, 0]).all() and not f["h"][0, :21].any() and not f["h"][0, :, 1:].any()
    assert torch.isnan(b["du"][0, :21, 0]).all() and not b["du"][0, 21:].any()
