"""The two halves of the binding of the learner's operators: the native one makes the call, the general one returns the same."""
import pytest

from tests.test_learn_boundary import _calls

NAMES = ("gated_scan_fwd", "gated_scan_bwd", "gated_step", "policy_loss_fwd", "policy_loss_bwd", "policy_loss_grad")


def test_every_native_entry_point_is_among_the_calls():
    from paper_2502_20168_amd import _ssmlearn
    assert sorted(NAMES + ("adamw_step", "adamw_values")) == sorted(n for n in dir(_ssmlearn) if not n.startswith("_"))
    assert sorted(NAMES) == sorted(_calls("cpu"))


def _flat(r):
    import torch
    return [r] if torch.is_tensor(r) or r is None else [t for k in (sorted(r) if isinstance(r, dict) else range(len(r))) for t in _flat(r[k])]


class _Watched:
    def __init__(self, native):
        self.native, self.made = native, []

    def __getattr__(self, name):
        return lambda *a: self.made.append(getattr(self.native, name)(*a)) or self.made[-1]


def _both(call, monkeypatch):
    import torch
    from paper_2502_20168_amd import binding, learn
    from paper_2502_20168_amd import _ssmlearn
    watched = _Watched(_ssmlearn)
    monkeypatch.setattr(learn, "_native", watched)
    got = _flat(call())
    assert watched.made and all(m is not None and type(m) is not int for m in watched.made)
    monkeypatch.setattr(learn, "_native", binding._GeneralPathOnly())
    ref = _flat(call())
    torch.cuda.synchronize()
    assert len(got) == len(ref)
    for g, r in zip(got, ref):
        assert (g is None) == (r is None)
        assert g is None or (g.dtype == r.dtype and g.shape == r.shape and g.stride() == r.stride() and torch.equal(g, r))


@pytest.mark.gpu
@pytest.mark.parametrize("call", NAMES)
def test_native_and_general_path_return_the_same(call, monkeypatch):
    import torch
    torch.manual_seed(1)
    fn, kw, _ = _calls("cuda")[call]
    _both(lambda: fn(**kw), monkeypatch)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ("halves", "time", "odd"))
def test_outputs_lie_in_memory_as_on_the_general_path(layout, monkeypatch):
    import torch
    from paper_2502_20168_amd import learn
    from tests.learn_util import laid_out
    torch.manual_seed(1)
    z, u, d = (laid_out(torch.randn(3, 140, 6, device="cuda"), layout) for _ in range(3))
    _both(lambda: learn.ssm_gated_scan_fwd(z, u), monkeypatch)
    carry = learn.ssm_gated_scan_fwd(z, u)["carry"]
    _both(lambda: learn.ssm_gated_scan_bwd(z, u, None, None, carry, d), monkeypatch)
    x = torch.randn(5, 12, device="cuda")[:, :9]
    row = (x, torch.zeros(5, dtype=torch.int64, device="cuda")) + tuple(torch.randn(5, device="cuda") for _ in range(2))
    _both(lambda: learn.ssm_policy_loss_grad(*row), monkeypatch)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", (8, 32))
def test_adamw_through_both(bits, monkeypatch):
    import torch
    from paper_2502_20168_amd import learn
    torch.manual_seed(1)
    grads = [torch.randn(s, device="cuda") for s in (5, 700, 3)]

    def call():
        params = [torch.ones_like(g) for g in grads]
        st = learn.ssm_adamw_state(params, bits)
        for t in (1, 2):
            learn.ssm_adamw_step(params, grads, **st, lr=0.1, step=t, grad_scale=torch.full((), 0.5, device="cuda"))
        values = learn.ssm_adamw_values(**st) if bits == 8 else ()
        return params + st["m"] + st["v"] + [t for v in values for t in v]

    _both(call, monkeypatch)


def test_without_its_native_half_the_binding_takes_the_general_path(monkeypatch):
    import sys
    import torch
    import paper_2502_20168_amd as package
    from paper_2502_20168_amd import learn
    monkeypatch.setattr(learn, "_native", None)
    monkeypatch.delattr(package, "_ssmlearn", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2502_20168_amd._ssmlearn", None)     # (its import raises ImportError)
    with pytest.warns(RuntimeWarning, match="native half"), pytest.raises(ValueError, match="gate must be a cuda tensor"):
        learn.ssm_gated_step(torch.zeros(2, 3), torch.zeros(2, 3))


def test_a_tensor_without_storage_raises_torchs_error():
    import types
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    from paper_2502_20168_amd import learn
    with FakeTensorMode(allow_non_fake_inputs=True):
        f = lambda *s: torch.zeros(s, device="cuda")
        batch, k = f(7, 2, 3), {"stream": types.SimpleNamespace(cuda_stream=0)}
        with pytest.raises(RuntimeError, match="data pointer"):
            torch.func.vmap(lambda u: learn.ssm_gated_step(f(2, 3), u, h=f(2, 3), y=f(2, 3), **k))(batch)
