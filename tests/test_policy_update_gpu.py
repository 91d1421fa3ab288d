"""The example that runs the learner's operators together: its gradients against automatic differentiation in 64 bits, and that it learns."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _plain_gradients(policy, o, t, h0):
    """The loss and its gradients with respect to policy.params() plus the value's squared error, by torch in float64 on the CPU."""
    import torch
    import policy_update as ex
    d = lambda v: v.detach().cpu().double()
    w_in, b_in, w_out, w_value = (d(p).requires_grad_() for p in policy.params())
    x, first, D = d(o["x"]), o["first"].cpu().t(), policy.D
    h, hs = d(h0), []
    for k in range(x.shape[0]):
        both = x[k] @ w_in + b_in
        f = torch.sigmoid(both[:, :D])
        h = torch.where(first[k][:, None] != 0, torch.zeros_like(h), f * h) + (1 - f) * both[:, D:]
        hs.append(h)
    h = torch.stack(hs).view(-1, D)
    logits = (h @ w_out)[:, :ex.CUES]
    logp_all = torch.log_softmax(logits, 1)
    logp = logp_all.gather(1, t["action"].cpu()[:, None])[:, 0]
    entropy = -(logp_all.exp() * logp_all).sum(1)
    weight, A = d(t["weight"]), d(t["advantage"])
    rho = torch.exp(logp - d(t["logp"]))
    loss = (weight * (-torch.minimum(rho * A, rho.clamp(0.8, 1.25) * A) - 1e-3 * entropy)).sum()
    value = 0.5 * (weight * ((h @ w_value)[:, 0] - d(t["ret"])) ** 2).sum()
    (loss + value).backward()
    return float(loss.detach()), [p.grad for p in (w_in, b_in, w_out, w_value)]


def test_gradients_of_one_update():
    """Chains of at most 40 roundings, sums of at most 64 terms in each dense layer: 64 * 40 * 2^-24 of a gradient's norm."""
    import torch
    import policy_update as ex
    gen = torch.Generator(device="cuda").manual_seed(3)
    policy, env = ex.Policy(12, torch.float32, gen, 32), ex.Recall(6, gen)
    policy.w_value.normal_(generator=gen)
    h = torch.randn(6, 12, generator=gen, device="cuda")
    h0 = h.clone()
    o = ex.roll_out(policy, env, h, 30, gen)
    t = ex.targets(policy, o)
    policy.w_out.add_(0.3 * torch.randn(policy.w_out.shape, generator=gen, device="cuda"))       # ratios away from 1
    loss, grads = ex.gradients(policy, o, t, h0)
    ref_loss, ref = _plain_gradients(policy, o, t, h0)
    bound = 64 * 40 * 2.0 ** -24
    assert abs(float(loss) - ref_loss) <= bound * max(1.0, abs(ref_loss))
    for g, r in zip(grads, ref):
        r = r.reshape(g.shape)
        if g.shape[-1] == ex.ACTIONS:
            assert torch.equal(g[:, ex.CUES:], torch.zeros_like(g[:, ex.CUES:]))                 # actions that cannot be taken
        assert float((g.cpu().double() - r).norm()) <= bound * float(r.norm())


@pytest.mark.parametrize("dtype,bits", (("float32", 32), ("bfloat16", 8)))
def test_it_learns(dtype, bits):
    """By chance an eighth of the answers is right; remembering the cue makes nearly all right."""
    import torch
    import policy_update as ex
    right = ex.train(updates=60, dtype=getattr(torch, dtype), bits=bits)
    assert right[0] < 0.25 and right[-1] > 0.9, right
