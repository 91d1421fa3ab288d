"""Inputs that overlap themselves (windows over one array, repeats): they are read where they lie, the outputs are dense."""
import pytest

pytestmark = pytest.mark.gpu


def _windows(kind, Bt, L, D):
    import torch
    torch.manual_seed(1)
    x = torch.randn(Bt * L * D, device="cuda")
    seq, step = {"by one": (L * D, 1), "of both": (1, 2), "repeated steps": (1, 0), "repeated sequences": (0, 1)}[kind]
    return x.as_strided((Bt, L, D), (seq, step, 1))


@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("kind", ("by one", "of both", "repeated steps", "repeated sequences"))
def test_recurrence(kind, native, monkeypatch):
    import torch
    from paper_2502_20168_amd import binding, learn
    if not native:
        monkeypatch.setattr(learn, "_native", binding._GeneralPathOnly())
    z, u, d = (_windows(kind, 3, 140, 6) for _ in range(3))
    dense = [t.contiguous() for t in (z, u, d)]
    f, want = learn.ssm_gated_scan_fwd(z, u), learn.ssm_gated_scan_fwd(*dense[:2])
    b = learn.ssm_gated_scan_bwd(z, u, None, None, f["carry"], d)
    back = learn.ssm_gated_scan_bwd(*dense[:2], None, None, want["carry"], dense[2])
    for got, ref in ((f, want), (b, back)):
        for k in ref:
            assert torch.equal(got[k], ref[k]), k


@pytest.mark.parametrize("native", (True, False))
def test_policy_loss(native, monkeypatch):
    import torch
    from paper_2502_20168_amd import binding, learn
    if not native:
        monkeypatch.setattr(learn, "_native", binding._GeneralPathOnly())
    torch.manual_seed(1)
    x = torch.randn(40, device="cuda").as_strided((9, 7), (1, 1))
    row = (torch.zeros(9, dtype=torch.int64, device="cuda"),) + tuple(torch.randn(9, device="cuda") for _ in range(2))
    r, want = learn.ssm_policy_loss_grad(x, *row), learn.ssm_policy_loss_grad(x.contiguous(), *row)
    b = learn.ssm_policy_loss_bwd(x, *row, None, None, r["logp"], r["entropy"], r["lse"])
    for k in want:
        assert torch.equal(r[k], want[k]), k
    assert torch.equal(b, learn.ssm_policy_loss_bwd(x.contiguous(), *row, None, None, r["logp"], r["entropy"], r["lse"]))
