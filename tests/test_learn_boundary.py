"""Host-side contract of include/ssm_learn.h and its binding: exports, and errors before any launch (no GPU needed)."""
import ctypes
import os
import re

import pytest

from paper_2502_20168_amd import binding as ssm
from paper_2502_20168_amd import build as ssm_build
from paper_2502_20168_amd import learn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000                       # never dereferenced: every check below fails before a launch
BAD, WS, BIG = ssm.SSM_ERR_INVALID_ARG, ssm.SSM_ERR_WORKSPACE, ssm.SSM_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if ssm_build.is_stale():
        ssm_build.build()
    return learn._lib()


def test_every_declared_symbol_is_exported(lib):
    header = open(os.path.join(ROOT, "include", "ssm_learn.h")).read()
    declared = set(re.findall(r"^(?:size_t|ssm_status|int64_t) (ssm_[a-z0-9_]+)\(", header, re.M))
    assert declared == set(learn.EXPORTS)
    assert all(hasattr(lib, name) for name in declared)


def test_carry_rows(lib):
    assert [learn.ssm_gated_carry_rows(L) for L in (-1, 0, 1, 128, 129, 256, 257)] == [0, 0, 0, 0, 1, 1, 2]


DENSE = learn._Strides(32, 4)


def _gated(lib, fn, **over):
    a = dict(gate=FAKE, gs=DENSE, u=FAKE, us=DENSE, is_first=None, h0=None, carry=FAKE, dh=FAKE, dhs=DENSE, dh_last=None, dtype=0, linear=0,
             Bt=2, L=8, D=4, h=FAKE, hs=DENSE, h_last=None, dgate=FAKE, dgs=DENSE, du=FAKE, dus=DENSE, dh0=None, ws=None, n=0, stream=None)
    a.update(over)
    names = {"ssm_gated_scan_fwd": "gate gs u us is_first h0 dtype linear Bt L D h hs h_last carry ws n stream",
             "ssm_gated_scan_bwd": "gate gs u us is_first h0 carry dh dhs dh_last dtype linear Bt L D dgate dgs du dus dh0 ws n stream"}[fn]
    return getattr(lib, fn)(*[a[k] for k in names.split()])


@pytest.mark.parametrize("fn,needed", [("ssm_gated_scan_fwd", ("gate", "u", "h")), ("ssm_gated_scan_bwd", ("gate", "u", "dh", "dgate", "du"))])
def test_gated_argument_errors(lib, fn, needed):
    for name in needed:
        assert _gated(lib, fn, **{name: None}) == BAD, name
        assert _gated(lib, fn, **{name: FAKE + 2}) == BAD, name
        assert _gated(lib, fn, dtype=1, **{name: FAKE + 1}) == BAD, name
    for dim in ("Bt", "L", "D"):
        assert _gated(lib, fn, **{dim: 0}) == BAD and _gated(lib, fn, **{dim: -1}) == BAD
    assert _gated(lib, fn, dtype=3) == BAD and _gated(lib, fn, h0=FAKE + 2) == BAD
    assert _gated(lib, fn, D=1 << 17) == BIG and _gated(lib, fn, Bt=1 << 31, L=2) == BIG
    assert _gated(lib, fn, gs=learn._Strides(-32, 4)) == BAD and _gated(lib, fn, us=learn._Strides(32, -4)) == BAD
    assert _gated(lib, fn, gs=learn._Strides(1 << 62, 4)) == BIG
    for out in ("hs",) if fn.endswith("fwd") else ("dgs", "dus"):
        for s in ((32, 3), (3, 32), (8, 4), (0, 4), (32, 0)):        # two elements in one place
            assert _gated(lib, fn, **{out: learn._Strides(*s)}) == BAD, s
    if fn.endswith("bwd"):
        assert _gated(lib, fn, L=129, carry=None, dgs=learn._Strides(516, 4), dus=learn._Strides(516, 4)) == BAD


def test_gated_step_argument_errors(lib):
    f = lib.ssm_gated_step
    assert f(None, 4, FAKE, 4, None, None, 0, 0, 2, 4, FAKE, None, None) == BAD
    assert f(FAKE, 4, None, 4, None, None, 0, 0, 2, 4, FAKE, None, None) == BAD
    assert f(FAKE, 4, FAKE, 4, None, None, 0, 0, 2, 4, None, FAKE, None) == BAD
    assert f(FAKE, -4, FAKE, 4, None, None, 0, 0, 2, 4, FAKE, None, None) == BAD
    assert f(FAKE, 4, FAKE, 4, None, None, 5, 0, 2, 4, FAKE, None, None) == BAD
    assert f(FAKE, 4, FAKE, 4, None, None, 0, 0, 0, 4, FAKE, None, None) == BAD
    assert f(FAKE, 4, FAKE, 4, None, None, 0, 0, 2, 1 << 17, FAKE, None, None) == BIG


def _policy(lib, fn, **over):
    a = dict(x=FAKE, pitch=8, action=FAKE, old=FAKE, adv=FAKE, w=None, ref=None, terms=learn._Terms(0.2, 0.2, 0.0, 0.0), dtype=0, N=4, K=8,
             loss=FAKE, logp=FAKE, entropy=FAKE, lse=FAKE, dloss=None, dx=FAKE + 4096, dpitch=8, ws=FAKE, n=256, stream=None)
    a.update(over)
    names = {"ssm_policy_loss_fwd": "x pitch action old adv w ref terms dtype N K loss logp entropy lse ws n stream",
             "ssm_policy_loss_bwd": "x pitch action old adv w ref terms dtype N K logp entropy lse dloss dx dpitch stream",
             "ssm_policy_loss_grad": "x pitch action old adv w ref terms dtype N K dloss loss logp entropy lse dx dpitch ws n stream"}[fn]
    return getattr(lib, fn)(*[a[k] for k in names.split()])


@pytest.mark.parametrize("fn", ("ssm_policy_loss_fwd", "ssm_policy_loss_bwd", "ssm_policy_loss_grad"))
def test_policy_argument_errors(lib, fn):
    for name in ("x", "action", "old", "adv", "logp", "entropy", "lse"):
        assert _policy(lib, fn, **{name: None}) == BAD, name
        assert _policy(lib, fn, **{name: FAKE + 1}) == BAD, name
    for name in ("w", "ref"):
        assert _policy(lib, fn, **{name: FAKE + 2}) == BAD, name
    for dim in ("N", "K"):
        assert _policy(lib, fn, **{dim: 0}) == BAD
    assert _policy(lib, fn, dtype=-1) == BAD and _policy(lib, fn, pitch=-1) == BAD
    assert _policy(lib, fn, K=(1 << 30) + 1, dpitch=1 << 31) == BIG and _policy(lib, fn, N=1 << 31) == BIG
    nan = float("nan")
    for t in ((-0.1, 0.2, 0, 0), (nan, 0.2, 0, 0), (0.2, nan, 0, 0), (0.2, 0.2, nan, 0), (0.2, 0.2, 0, nan)):
        assert _policy(lib, fn, terms=learn._Terms(*t)) == BAD
    if fn != "ssm_policy_loss_bwd":
        assert _policy(lib, fn, loss=None) == BAD
        assert _policy(lib, fn, ws=None) == WS and _policy(lib, fn, ws=FAKE + 64) == WS and _policy(lib, fn, n=0) == WS
    if fn != "ssm_policy_loss_fwd":
        assert _policy(lib, fn, dx=None) == BAD and _policy(lib, fn, dpitch=7) == BAD and _policy(lib, fn, dloss=FAKE + 1) == BAD
        assert _policy(lib, fn, dx=FAKE, dpitch=9) == BAD            # over the logits, but with rows elsewhere


def test_policy_workspace_bytes(lib):
    assert learn.ssm_policy_loss_workspace_bytes(1, 5) > 0
    for bad in ((0, 5), (5, 0), (-1, 5), (1 << 31, 5), (5, (1 << 30) + 1)):
        assert learn.ssm_policy_loss_workspace_bytes(*bad) == 0


def _tensor(**over):
    t = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, n=10)
    t.update(over)
    return t


def _adamw(lib, rows=None, bits=32, p=0, g=0, scale=None, skip=None, count=None, **rates):
    rows = [_tensor()] if rows is None else rows
    arr = (learn._AdamwTensor * len(rows))(*[learn._AdamwTensor(**r) for r in rows])
    r = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
    r.update(rates)
    return lib.ssm_adamw_step(arr, len(rows) if count is None else count, learn._AdamwRates(**r), p, g, bits, scale, skip, None)


def test_adamw_argument_errors(lib):
    for name in ("param", "grad", "m", "v"):
        assert _adamw(lib, [_tensor(), _tensor(**{name: None})]) == BAD, name
        assert _adamw(lib, [_tensor(**{name: FAKE + 2})]) == BAD, name
    for name in ("m_scale", "v_scale"):
        assert _adamw(lib, [_tensor(**{name: None})], bits=8) == BAD, name
        assert _adamw(lib, [_tensor(**{name: FAKE + 2})], bits=8) == BAD, name
    assert _adamw(lib, [_tensor(n=-1)]) == BAD and _adamw(lib, [_tensor(n=1 << 41)]) == BIG
    assert _adamw(lib, count=0) == BAD and _adamw(lib, bits=16) == BAD
    assert _adamw(lib, p=1, g=0) == BAD and _adamw(lib, p=1, g=2) == BAD and _adamw(lib, p=3) == BAD and _adamw(lib, g=3) == BAD
    assert _adamw(lib, scale=FAKE + 2) == BAD and _adamw(lib, skip=FAKE + 1) == BAD
    nan = float("nan")
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1.0), dict(eps=nan), dict(step=0), dict(lr=nan),
                dict(weight_decay=nan)):
        assert _adamw(lib, **bad) == BAD, bad
    assert lib.ssm_adamw_step(None, 1, learn._AdamwRates(0.1, 0.9, 0.9, 0, 0, 1), 0, 0, 32, None, None, None) == BAD
    one = (learn._AdamwStored * 1)(learn._AdamwStored(FAKE, FAKE, FAKE, None, FAKE, FAKE, 3))
    assert lib.ssm_adamw_values(one, 1, None) == BAD and lib.ssm_adamw_values(None, 1, None) == BAD and lib.ssm_adamw_values(one, 0, None) == BAD


def test_empty_tensors_alone_launch_nothing(lib):
    assert _adamw(lib, [_tensor(n=0, param=None)]) == ssm.SSM_OK


def test_what_no_grid_holds(lib):
    """A grid holds fewer than 2^32 threads; a sequence's last chunk ends within 31 bits."""
    import torch
    far = learn._Strides(1 << 40, 1)
    for fn in ("ssm_gated_scan_fwd", "ssm_gated_scan_bwd"):
        strides = dict(gs=far, us=far, hs=far) if fn.endswith("fwd") else dict(gs=far, us=far, dhs=far, dgs=far, dus=far)
        assert _gated(lib, fn, Bt=1, L=(1 << 31) - 1, D=1, **strides) == BIG
        assert _gated(lib, fn, Bt=1, L=(1 << 31) - 8192, D=1, **strides) == BIG
    assert learn.ssm_gated_workspace_bytes(1, (1 << 31) - 1, 1, torch.float32, False) == 0
    assert lib.ssm_gated_step(FAKE, 4, FAKE, 4, None, None, 0, 0, 1 << 20, 4097, FAKE, None, None) == BIG
    for fn in ("ssm_policy_loss_fwd", "ssm_policy_loss_bwd", "ssm_policy_loss_grad"):
        for N, K in ((1 << 26, 1000), (1 << 24, 9000)):
            assert _policy(lib, fn, N=N, K=K, pitch=K, dpitch=K, n=1 << 40) == BIG, (fn, N, K)
    for bits, chunk in ((32, 1024), (8, 4096)):
        assert _adamw(lib, [_tensor(n=(1 << 24) * chunk)], bits=bits) == BIG
    one = (learn._AdamwStored * 1)(learn._AdamwStored(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 35))
    assert lib.ssm_adamw_values(one, 1, None) == BIG


WRONG = {"shape": lambda t: t[..., :-1].contiguous(), "stride": lambda t: t.repeat_interleave(2, -1)[..., ::2], "device": lambda t: t.cpu(),
         "type": lambda t: t.double() if t.is_floating_point() else t.short()}


def _calls(device):
    """name -> (function, keyword arguments, names of the tensors whose errors name them)"""
    import torch
    Bt, L, D, N, K = 2, 130, 6, 5, 7
    f = lambda *s: torch.randn(s, device=device)
    flags = lambda *s: torch.zeros(s, dtype=torch.uint8, device=device)
    scan = {"gate": f(Bt, L, D), "u": f(Bt, L, D), "is_first": flags(Bt, L), "h0": f(Bt, D)}
    row = {"logits": f(N, K), "action": torch.zeros(N, dtype=torch.int64, device=device), "logp_old": f(N), "advantage": f(N), "weight": f(N), "logp_ref": f(N)}
    stats = {"logp": f(N), "entropy": f(N), "lse": f(N)}
    return {
        "gated_scan_fwd": (learn.ssm_gated_scan_fwd, scan, ("u", "is_first", "h0")),
        "gated_scan_bwd": (learn.ssm_gated_scan_bwd, {**scan, "carry": f(Bt, 1, D), "dh": f(Bt, L, D), "dh_last": f(Bt, D)},
                           ("u", "is_first", "h0", "carry", "dh", "dh_last")),
        "gated_step": (learn.ssm_gated_step, {"gate": f(Bt, D), "u": f(Bt, D), "h_prev": f(Bt, D), "is_first": flags(Bt)}, ("u", "h_prev", "is_first")),
        "policy_loss_fwd": (learn.ssm_policy_loss_fwd, row, ("action", "logp_old", "advantage", "weight", "logp_ref")),
        "policy_loss_bwd": (learn.ssm_policy_loss_bwd, {**row, **stats}, ("action", "logp_old", "advantage", "weight", "logp_ref", "logp", "entropy", "lse")),
        "policy_loss_grad": (learn.ssm_policy_loss_grad, row, ("action", "logp_old", "advantage", "weight", "logp_ref")),
    }


@pytest.mark.parametrize("wrong", sorted(WRONG))
@pytest.mark.parametrize("call", ("gated_scan_fwd", "gated_scan_bwd", "gated_step", "policy_loss_fwd", "policy_loss_bwd", "policy_loss_grad"))
def test_a_wrong_argument_is_named(call, wrong):
    """Fake tensors on the GPU: a call that is not refused cannot reach one."""
    import types
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode(allow_non_fake_inputs=True):
        fn, kw, names = _calls("cuda")[call]
        kw["stream"] = types.SimpleNamespace(cuda_stream=0)
        for name in names:
            with pytest.raises(ValueError, match="^%s must be a .*cuda tensor" % name):
                fn(**{**kw, name: WRONG[wrong](kw[name])})


def test_a_wrong_type_or_dimension_of_the_first_argument_is_named():
    import torch
    with pytest.raises(ValueError, match="gate must be float32, bfloat16 or float16"):
        learn.ssm_gated_scan_fwd(torch.zeros(1, 2, 3, dtype=torch.float64), torch.zeros(1, 2, 3))
    with pytest.raises(ValueError, match=r"gate must be \[Bt,L,D\]"):
        learn.ssm_gated_scan_fwd(torch.zeros(2, 3), torch.zeros(2, 3))
    with pytest.raises(ValueError, match="gate must be a cuda tensor"):
        learn.ssm_gated_scan_fwd(torch.zeros(1, 2, 3), torch.zeros(1, 2, 3))
    with pytest.raises(ValueError, match=r"logits must be \[N,K\]"):
        learn.ssm_policy_loss_fwd(torch.zeros(3), *[torch.zeros(3)] * 3)
    with pytest.raises(ValueError, match="logits must be a cuda tensor"):
        learn.ssm_policy_loss_fwd(torch.zeros(3, 2), torch.zeros(3, dtype=torch.int64), torch.zeros(3), torch.zeros(3))


def test_adamw_lists_are_checked():
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode(allow_non_fake_inputs=True):
        t = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
        good = {"params": [t(5), t(3, 2)], "grads": [t(5), t(3, 2)], "m": [t(5), t(3, 2)], "v": [t(5), t(3, 2)]}
        call = lambda **over: learn.ssm_adamw_step(**{**good, **over}, lr=0.1, step=1)
        with pytest.raises(ValueError, match="grads must have one tensor per parameter"):
            call(grads=good["grads"][:1])
        for name in ("grads", "m", "v"):
            with pytest.raises(ValueError, match=r"%s\[1\] must be a contiguous cuda tensor" % name):
                call(**{name: [t(5), t(2, 3)]})
        with pytest.raises(ValueError, match=r"params\[1\] must be"):
            call(params=[t(5), t(2, 3).t()])
        with pytest.raises(ValueError, match="m_scale and v_scale must be given"):
            call(m=[t(5, dt=torch.uint8), t(3, 2, dt=torch.uint8)])
        with pytest.raises(ValueError, match=r"m_scale\[0\] must be"):
            b = [t(5, dt=torch.uint8), t(3, 2, dt=torch.uint8)]
            call(m=b, v=b, m_scale=[t(2), t(1)], v_scale=[t(1), t(1)])
        with pytest.raises(ValueError, match="grad_scale must be"):
            call(grad_scale=t(2))
        with pytest.raises(ValueError, match="at least one tensor"):
            call(params=[])
        with pytest.raises(ValueError, match="bits must be"):
            learn.ssm_adamw_state(good["params"], 16)
