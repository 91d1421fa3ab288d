"""A recurrent policy that learns to remember, with the library's learner operators: python examples/policy_update.py

Episodes of 4 to 12 steps run back to back in many environments.  The first observation of an episode shows a cue, the ones after
it show noise, the last one asks for the cue back: the action taken there earns 1 if it names the cue.  Two of the actions are
never allowed.  The policy is one gated linear recurrence between two dense layers:

    acting     ssm_gated_step, one step of every environment, the state updated in place
    returns    ssm_policy_loss_fwd for the log-probabilities of what was done, ssm_lambda_return for what it earned
    update     ssm_gated_scan_fwd over the time-major observations, ssm_policy_loss_grad for loss and gradient in one pass (only steps
               that ask count, the others are idle rows), ssm_gated_scan_bwd, ssm_adamw_step over all parameters at once

The dense layers are plain matrix products.  Gradients are clipped without a pass of their own: their norm's factor goes to
ssm_adamw_step as grad_scale, and a step whose norm is not finite is skipped on the device.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_20168_amd import binding as ssm      # noqa: E402
from paper_2502_20168_amd import learn               # noqa: E402

CUES, ILLEGAL = 8, 2
ACTIONS = CUES + ILLEGAL
INPUTS = CUES + 2                                    # cue, asked, noise


class Recall:
    """N environments; observation [N, INPUTS], is_first [N] uint8 and asked [N] float32 of the present step."""

    def __init__(self, N, gen):
        self.N, self.gen = N, gen
        self.left = torch.zeros(N, dtype=torch.int64, device="cuda")
        self.cue = torch.zeros(N, dtype=torch.int64, device="cuda")
        self.first = torch.ones(N, dtype=torch.bool, device="cuda")
        self._begin()

    def _begin(self):
        draw = lambda lo, hi: torch.randint(lo, hi, (self.N,), generator=self.gen, device="cuda")
        self.left = torch.where(self.first, draw(3, 12), self.left)
        self.cue = torch.where(self.first, draw(0, CUES), self.cue)

    def observe(self):
        cue = torch.nn.functional.one_hot(self.cue, CUES) * self.first[:, None]
        noise = torch.randn(self.N, 1, generator=self.gen, device="cuda")
        asked = (self.left == 0).float()
        return torch.cat((cue.float(), asked[:, None], noise), 1), self.first.to(torch.uint8), asked

    def act(self, action):
        """Reward of this step and whether the episode goes on."""
        asked = self.left == 0
        reward = (asked & (action == self.cue)).float()
        self.first = asked
        self.left = self.left - 1
        self._begin()
        return reward, (~asked).float()


class Policy:
    def __init__(self, D, dtype, gen, bits):
        normal = lambda fan, *shape: (torch.randn(shape, generator=gen, device="cuda") / math.sqrt(fan)).to(dtype)
        self.D = D
        self.w_in = normal(INPUTS, INPUTS, 2 * D)
        self.b_in = torch.cat((torch.linspace(0, 4, D, device="cuda"), torch.zeros(D, device="cuda"))).to(dtype)   # decays over 2 to 50 steps
        self.w_out = normal(D, D, ACTIONS)
        self.w_value = torch.zeros(D, 1, dtype=dtype, device="cuda")
        self.bar = torch.zeros(ACTIONS, device="cuda", dtype=dtype)
        self.bar[CUES:] = float("-inf")
        self.state = learn.ssm_adamw_state(self.params(), bits)
        self.step = 0

    def params(self):
        return [self.w_in, self.b_in, self.w_out, self.w_value]

    def project(self, x):
        """Gate and input of the recurrence: the halves of one product."""
        both = torch.addmm(self.b_in, x.reshape(-1, INPUTS).to(self.w_in.dtype), self.w_in).view(*x.shape[:-1], 2 * self.D)
        return both[..., :self.D], both[..., self.D:]

    def logits(self, h):
        return torch.addmm(self.bar, h, self.w_out)


def roll_out(policy, env, h, T, gen):
    """T steps of acting from the states h [N, D], which end as those behind the last step.  Everything time-major."""
    x, first, asked, action, reward, cont, logits, value = ([] for _ in range(8))
    for _ in range(T):
        obs, is_first, ask = env.observe()
        gate, u = policy.project(obs)
        y, _ = learn.ssm_gated_step(gate, u, h, is_first, h=h)
        score = policy.logits(y)
        a = torch.multinomial(torch.softmax(score.float(), 1), 1, generator=gen)[:, 0]
        r, c = env.act(a)
        for to, what in ((x, obs), (first, is_first), (asked, ask), (action, a), (reward, r), (cont, c), (logits, score),
                         (value, (y @ policy.w_value).float()[:, 0])):
            to.append(what)
    return {"x": torch.stack(x), "first": torch.stack(first, 1).contiguous(), "asked": torch.stack(asked), "action": torch.stack(action),
            "reward": torch.stack(reward), "cont": torch.stack(cont), "logits": torch.stack(logits), "value": torch.stack(value)}


def targets(policy, o):
    """Log-probabilities of what was done, weights, returns and advantages, flat over [T, N]."""
    weight = (o["asked"] / o["asked"].sum().clamp(min=1.0)).view(-1)
    flat = o["action"].view(-1)
    zero = torch.zeros_like(weight)
    done = learn.ssm_policy_loss_fwd(o["logits"].view(-1, ACTIONS), flat, zero, zero, weight)
    ret = ssm.ssm_lambda_return(o["reward"], o["cont"], o["value"], 0.97, 0.95)
    return {"weight": weight, "action": flat, "logp": done["logp"], "ret": ret.view(-1), "advantage": (ret - o["value"]).view(-1)}


def gradients(policy, o, t, h0):
    """Loss and the gradients of policy.params(), of one pass over the whole roll-out."""
    T, N, D = o["x"].shape[0], o["x"].shape[1], policy.D
    gate, u = policy.project(o["x"])
    by_seq = lambda v: v.transpose(0, 1)                       # [T, N, D] as the recurrence's [N, T, D]: strides, no copy
    s = learn.ssm_gated_scan_fwd(by_seq(gate), by_seq(u), o["first"], h0)
    h = s["h"].transpose(0, 1).reshape(T * N, D)
    score = policy.logits(h)
    r = learn.ssm_policy_loss_grad(score, t["action"], t["logp"], t["advantage"], t["weight"], clip_low=0.2, clip_high=0.25,
                                   entropy_coef=1e-3, out={"dlogits": score})
    dscore = r["dlogits"]
    value = h @ policy.w_value
    dvalue = ((value.float()[:, 0] - t["ret"]) * t["weight"]).to(h.dtype)[:, None]
    dh = torch.addmm(dvalue @ policy.w_value.t(), dscore, policy.w_out.t())
    both = torch.empty(T, N, 2 * D, dtype=h.dtype, device="cuda")
    learn.ssm_gated_scan_bwd(by_seq(gate), by_seq(u), o["first"], h0, s["carry"], by_seq(dh.view(T, N, D)), want_dh0=False,
                             out={"dgate": by_seq(both[..., :D]), "du": by_seq(both[..., D:])})
    both = both.view(T * N, 2 * D)
    return r["loss"], [o["x"].view(-1, INPUTS).to(h.dtype).t() @ both, both.sum(0), h.t() @ dscore, h.t() @ dvalue]


def update(policy, o, t, h0, lr):
    loss, grads = gradients(policy, o, t, h0)
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.float()) for g in grads]))
    policy.step += 1
    learn.ssm_adamw_step(policy.params(), grads, policy.state["m"], policy.state["v"], policy.state["m_scale"], policy.state["v_scale"],
                         lr=lr, weight_decay=1e-4, step=policy.step, grad_scale=torch.clamp(1.0 / norm, max=1.0),
                         skip=(~torch.isfinite(norm)).float())
    return loss


def train(updates=60, N=256, T=64, D=64, epochs=2, lr=1e-2, dtype=torch.float32, bits=32, seed=0, report=0):
    """Share of right answers of every roll-out."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    policy, env = Policy(D, dtype, gen, bits), Recall(N, gen)
    h = torch.zeros(N, D, device="cuda")
    right = []
    for i in range(updates):
        begin = time.perf_counter()
        h0 = h.clone()
        o = roll_out(policy, env, h, T, gen)
        t = targets(policy, o)
        for _ in range(epochs):
            update(policy, o, t, h0, lr)
        right.append(float(o["reward"].sum() / o["asked"].sum()))
        if report and (i + 1) % report == 0:
            print("update %4d: %5.1f %% right, %.1f ms" % (i + 1, 100 * right[-1], 1e3 * (time.perf_counter() - begin)), flush=True)
    return right


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--updates", type=int, default=60)
    p.add_argument("--envs", type=int, default=256)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--width", type=int, default=64)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    p.add_argument("--bits", type=int, choices=(8, 32), default=32, help="of the optimizer's states")
    a = p.parse_args()
    right = train(a.updates, a.envs, a.steps, a.width, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype], bits=a.bits, report=10)
    print("right at the start %.1f %% (by chance %.1f %%), at the end %.1f %%" % (100 * right[0], 100 / CUES, 100 * right[-1]))


if __name__ == "__main__":
    main()
