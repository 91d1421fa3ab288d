"""The gated linear recurrence where gates are near one and inputs are sparse: states are small beside the inputs they come from."""
import numpy as np
import pytest

from oracle import learn_oracle as orc

pytestmark = pytest.mark.gpu

# 1 - f is good to 10^-6 of itself at gates up to 17 (the exponent, 24.5 in powers of two, is rounded by 2^-20), a gradient has two such factors; 1500 roundings of
# 2^-25 in either direction add up to 10^-6.  Everything is positive, nothing cancels.
ELEMENTWISE = 1e-5


@pytest.mark.parametrize("L,resets", [(40, False), (200, True), (1500, True), (5000, True)])
def test_gradient_of_the_gates_behind_an_impulse(L, resets):
    """Every 40th input is not zero: behind it, the gradient of a gate is the state times what flows back, element by element."""
    import torch
    from paper_2502_20168_amd import learn
    gen = torch.Generator().manual_seed(2)
    uniform = lambda lo, hi, *s: torch.rand(s, generator=gen) * (hi - lo) + lo
    gate, u, dh = uniform(10, 17, 2, L, 12), torch.zeros(2, L, 12), uniform(0.5, 1.5, 2, L, 12)
    u[:, ::40] = uniform(1, 2, 2, len(range(0, L, 40)), 12)
    first = torch.zeros(2, L, dtype=torch.uint8)
    if resets:
        first[:, 120::400] = 1
    n = lambda t: t.double().numpy()
    ref = orc.gated_bwd(n(gate), n(u), first.numpy(), None, n(dh))
    gate, u, dh, first = (t.cuda() for t in (gate, u, dh, first))
    f = learn.ssm_gated_scan_fwd(gate, u, first)
    g = learn.ssm_gated_scan_bwd(gate, u, first, None, f["carry"], dh)
    for k in ("dgate", "du"):
        got = n(g[k].cpu())
        assert np.all(np.abs(got - ref[k]) <= ELEMENTWISE * np.abs(ref[k])), (k, np.max(np.abs(got - ref[k]) / np.maximum(np.abs(ref[k]), 1e-300)))
