"""A workspace given by the caller: memory of the GPU without gaps, or an error before anything is launched (CPU only; fake tensors on the GPU)."""
import types

import pytest

from tests.test_binding import _calls as layer_calls
from tests.test_learn_boundary import _calls as learn_calls

LAYER = ("scan_fwd", "scan_bwd", "block_fwd", "block_bwd", "scan_states", "scan_states_reverse", "half_glu_fwd", "half_glu_bwd")
LEARN = ("gated_scan_fwd", "gated_scan_bwd", "policy_loss_fwd", "policy_loss_grad")


def test_every_call_with_a_workspace_is_here():
    import inspect
    for names, calls in ((LAYER, layer_calls("cpu", run=False)), (LEARN, learn_calls("cpu"))):
        assert sorted(names) == sorted(n for n, c in calls.items() if "workspace" in inspect.signature(c[0]).parameters)


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("wrong", ("device", "gaps", "one element for all"))
@pytest.mark.parametrize("call", LAYER + LEARN)
def test_a_workspace_that_kernels_cannot_use_is_refused(call, wrong, native, monkeypatch):
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    from paper_2502_20168_amd import binding, learn
    if not native:
        monkeypatch.setattr(binding, "_native", binding._GeneralPathOnly())
        monkeypatch.setattr(learn, "_native", binding._GeneralPathOnly())
    with FakeTensorMode(allow_non_fake_inputs=True):
        fn, kw, _ = layer_calls("cuda", run=False)[call] if call in LAYER else learn_calls("cuda")[call]
        bytes_ = lambda n, device="cuda": torch.empty(n, dtype=torch.uint8, device=device)
        ws = {"device": bytes_(1 << 20, "cpu"), "gaps": bytes_(1 << 21)[::2], "one element for all": bytes_(1).expand(1 << 20)}[wrong]
        with pytest.raises(ValueError, match="^workspace must be a contiguous cuda tensor"):
            fn(**kw, workspace=ws, stream=types.SimpleNamespace(cuda_stream=0))


def test_the_status_of_memory_that_is_none():
    import torch
    from paper_2502_20168_amd import binding
    with pytest.raises(ValueError, match="^workspace must be a contiguous cuda tensor"):
        binding.ssm_workspace_status(torch.zeros(256, dtype=torch.uint8))
