"""AdamW over the parameters of the layer, the complex ones as pairs of real numbers that share their memory."""
import numpy as np
import pytest

from oracle import learn_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", (8, 32))
def test_complex_parameters_through_their_real_views(bits):
    import torch
    from paper_2502_20168_amd import learn
    torch.manual_seed(1)
    layer = [torch.randn(s, dtype=dt, device="cuda") for s, dt in (((12,), torch.complex64), ((12, 20), torch.complex64), ((20,), torch.float32))]
    grads = [torch.randn_like(p) for p in layer]
    real = lambda ts: [torch.view_as_real(t) if t.is_complex() else t for t in ts]
    before = [p.double().cpu().numpy() for p in real(layer)]
    state = learn.ssm_adamw_state(real(layer), bits)
    learn.ssm_adamw_step(real(layer), real(grads), **state, lr=1e-2, step=1)
    for p, b, g in zip(real(layer), before, real(grads)):
        want, _, _ = orc.adamw(b, g.double().cpu().numpy(), 0 * b, 0 * b, 1e-2, 0.9, 0.999, 1e-8, 0.0, 1)
        # one rounding of the parameter, some 20 of an update of 10^-2
        assert np.all(np.abs(p.double().cpu().numpy() - want) <= 2.0 ** -23 * np.abs(want) + 20 * 2.0 ** -24 * 1e-2)
