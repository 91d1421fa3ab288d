"""The clipped policy loss where the row's own action has a logit far below the others, or one that cannot be taken at all."""
import numpy as np
import pytest

from tests.learn_util import check, tolerance
from tests.test_policy_gpu import ARITHMETIC, _inputs, _oracle

pytestmark = pytest.mark.gpu

# a row in part of a wavefront, in one, in a workgroup's registers, read again, in pieces
HOLDERS = [(9, 6), (9, 70), (5, 3001), (66, 70001), (4, 70001)]


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("eta", (0.0, 0.05))
@pytest.mark.parametrize("N,K", HOLDERS)
def test_own_action_at_minus_infinity(N, K, eta, dtype):
    """rho = 0 there: no term of the ratio for a positive advantage, the lower bound's for a negative one, the entropy's as ever."""
    import torch
    from paper_2502_20168_amd import learn
    terms = {"clip_low": 0.2, "clip_high": 0.3, "kl_coef": 0.0, "entropy_coef": eta}
    s = _inputs(N, K, dtype, masked=0.2, ref=False)
    rows = torch.tensor([0, 1, N - 1], device="cuda")
    s["logits"][rows, s["action"][rows]] = -float("inf")
    s["advantage"][:3] = torch.tensor([1.5, -1.5, 0.5], device="cuda")
    ref, args = _oracle(s, 1.0, terms), tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **terms)
    g = learn.ssm_policy_loss_grad(*args, **terms)
    b = learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **terms)
    assert np.isfinite(ref["loss"]) and np.all(np.isneginf(ref["logp"][rows.cpu().numpy()]))
    finite = np.isfinite(ref["logp"])
    for r in (f, g):
        assert abs(float(r["loss"]) - ref["loss"]) <= ARITHMETIC * float(s["weight"].sum()) * 8
        assert torch.isneginf(r["logp"][rows]).all()
        check(r["logp"][torch.from_numpy(finite).cuda()], ref["logp"][finite], ARITHMETIC, "logp")
        check(r["entropy"], ref["entropy"], ARITHMETIC, "entropy")
        check(r["lse"], ref["lse"], ARITHMETIC, "lse")
    for d in (g["dlogits"], b):
        check(d, ref["dlogits"], tolerance(dtype, 3 * ARITHMETIC), "dlogits")


@pytest.mark.parametrize("N,K", HOLDERS)
def test_no_such_action_beside_an_advantage_of_zero(N, K):
    """An action >= K makes its row NaN whatever the advantage is, and no other row."""
    import torch
    from paper_2502_20168_amd import learn
    terms = {"clip_low": 0.2, "clip_high": 0.3, "kl_coef": 0.0, "entropy_coef": 0.05}
    s = _inputs(N, K, ref=False)
    s["action"][1], s["advantage"][1] = K, 0.0
    args = tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **terms)
    g = learn.ssm_policy_loss_grad(*args, **terms)
    b = learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **terms)
    others = [0] + list(range(2, N))
    for r in (f, g):
        assert torch.isnan(r["loss"]) and torch.isnan(r["logp"][1]) and torch.isfinite(r["logp"][others]).all()
    for d in (g["dlogits"], b):
        assert torch.isnan(d[1]).all() and torch.isfinite(d[others]).all()


@pytest.mark.parametrize("dtype,low", [("f32", -1e4), ("f32", -1e6), ("f32", -1e9), ("f32", None), ("bf16", -1e4), ("bf16", None), ("f16", None)])
@pytest.mark.parametrize("N,K", HOLDERS)
def test_gradient_from_stored_statistics_where_the_own_action_is_far_below(N, K, dtype, low):
    """Finite logits of the own action down to the type's lowest: the gradient on its own is that of the definition, and that of loss and gradient in one call."""
    import torch
    from paper_2502_20168_amd import learn
    terms = {"clip_low": 0.2, "clip_high": 0.3, "kl_coef": 0.0, "entropy_coef": 0.05}
    s = _inputs(N, K, dtype, masked=0.2, ref=False)
    rows = torch.tensor([0, 1, N - 1], device="cuda")
    s["logits"][rows, s["action"][rows]] = torch.finfo(s["logits"].dtype).min if low is None else low
    s["advantage"][:3] = torch.tensor([1.5, -1.5, 0.5], device="cuda")
    if low is not None and low >= -1e6:                      # taken where it was as unlikely: the ratio is not zero
        s["logp_old"][0] = s["logits"][0, s["action"][0]].float()
    ref, args = _oracle(s, 1.0, terms), tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **terms)
    g = learn.ssm_policy_loss_grad(*args, **terms)
    b = learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **terms)
    assert abs(float(f["loss"]) - ref["loss"]) <= ARITHMETIC * float(s["weight"].sum()) * 8
    for name, d in (("one call", g["dlogits"]), ("on its own", b)):
        for n in range(min(N, 5)):                           # (row by row: no row hides behind a larger one)
            check(d[n], ref["dlogits"][n], tolerance(dtype, 3 * ARITHMETIC), "%s, row %d" % (name, n))


@pytest.mark.parametrize("N,K", HOLDERS)
def test_gradient_from_stored_statistics_at_large_logits(N, K):
    """Logits of 10^4: lse is rounded by 5e-4, the logit of an ordinary own action is the reference."""
    from paper_2502_20168_amd import learn
    terms = {"clip_low": 0.2, "clip_high": 0.3, "kl_coef": 0.0, "entropy_coef": 0.05}
    s = _inputs(N, K, ref=False)
    s["logits"] += 1e4
    ref, args = _oracle(s, 1.0, terms), tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **terms)
    check(learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **terms), ref["dlogits"], tolerance("f32", 3 * ARITHMETIC), "dlogits")


@pytest.mark.parametrize("low", (-1e4, -float("inf")))
@pytest.mark.parametrize("N,K", HOLDERS)
def test_a_reference_without_a_coefficient(N, K, low):
    """kl_coef 0: no KL term, also where the distance from the reference overflows."""
    import torch
    from paper_2502_20168_amd import learn
    terms = {"clip_low": 0.2, "clip_high": 0.3, "kl_coef": 0.0, "entropy_coef": 0.05}
    s = _inputs(N, K, masked=0.2)
    s["logits"][1, s["action"][1]] = low
    args = tuple(s.values())
    bare = args[:-1] + (None,)
    for call in (learn.ssm_policy_loss_fwd, learn.ssm_policy_loss_grad):
        r, want = call(*args, **terms), call(*bare, **terms)
        assert torch.isfinite(r["loss"])
        for k in r:
            assert torch.equal(r[k], want[k]), k
    b = [learn.ssm_policy_loss_bwd(*a, r["logp"], r["entropy"], r["lse"], **terms) for a in (args, bare)]
    assert torch.isfinite(b[0]).all() and torch.equal(*b)
    assert abs(float(r["loss"]) - _oracle(s, 1.0, terms)["loss"]) <= ARITHMETIC * float(s["weight"].sum()) * 8
