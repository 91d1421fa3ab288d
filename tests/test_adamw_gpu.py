"""AdamW over many tensors on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import learn_oracle as orc
from tests.learn_util import ROUND, torch_dtype

pytestmark = pytest.mark.gpu

RATES = {"lr": 1e-2, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "weight_decay": 0.1}
SIZES = [1, 2, 3, 4, 5, 255, 256, 257, 1023, 2048, 2049, 5000, 0, 70001]
TYPES = [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")]
ULP = 2.0 ** -24


def _lists(sizes, pdt, gdt, bits, seed=0, offset=0, history=True):
    """Lists of tensors of these sizes; offset: every tensor starts that many elements into its memory."""
    import torch
    from paper_2502_20168_amd import learn
    gen = torch.Generator().manual_seed(seed)
    at = lambda t: torch.cat((t.new_zeros(offset), t)).cuda()[offset:]
    s = {"params": [at(torch.randn(n, generator=gen).to(torch_dtype(pdt))) for n in sizes],
         "grads": [at((torch.randn(n, generator=gen) * 0.1).to(torch_dtype(gdt))) for n in sizes]}
    s.update(learn.ssm_adamw_state(s["params"], bits))
    if bits == 32 and history:
        s["m"] = [at(torch.randn(n, generator=gen) * 0.05) for n in sizes]
        s["v"] = [at(torch.rand(n, generator=gen) * 0.01) for n in sizes]
    elif history:
        for n in range(len(sizes)):
            k = sizes[n]
            s["m"][n] = at(torch.randint(0, 127, (k,), generator=gen).to(torch.uint8) + 128 * torch.randint(0, 2, (k,), generator=gen).to(torch.uint8))
            s["v"][n] = at(torch.randint(60, 256, (k,), generator=gen).to(torch.uint8))
            s["m_scale"][n] = (torch.rand(s["m_scale"][n].numel(), generator=gen) * 1e-4 + 1e-5).cuda()
            s["v_scale"][n] = (torch.rand(s["v_scale"][n].numel(), generator=gen) * 0.1 + 0.05).cuda()
    return s


def _host(s):
    return {k: None if v is None else [t.double().cpu().numpy() if t.dtype.is_floating_point else t.cpu().numpy() for t in v] for k, v in s.items()}


def _step(s, step=5, **kw):
    from paper_2502_20168_amd import learn
    learn.ssm_adamw_step(s["params"], s["grads"], s["m"], s["v"], s["m_scale"], s["v_scale"], **{**RATES, **kw}, step=step)


def _check_params(got, before, ref, pdt, m_terms, v, what):
    # the update in fp32: about ten roundings, and three of the terms of m, which may cancel; its result rounded once more where the parameter has fewer bits
    rate = RATES["lr"] / (1 - RATES["beta1"] ** 5) * np.sqrt(1 - RATES["beta2"] ** 5)
    allow = (ROUND[pdt] * 1.01 + 4 * ULP) * np.abs(ref) + 20 * ULP * np.abs(ref - before) + (2.0 ** -25 if pdt == "f16" else 0)
    allow = allow + rate * 3 * ULP * m_terms / np.maximum(np.sqrt(v), 1e-30)
    assert np.all(np.abs(got - ref) <= allow), (what, np.max(np.abs(got - ref) - allow))


def _check_codes(code, scale, want, kind, what):
    """Every stored value is one that its block's codes offer next to the value wanted: within half a step, relative to the block's scale."""
    bits, (mantissa, bias, top) = (orc.M_BITS, orc.M_BITS) if kind == "m" else (orc.R_BITS, orc.R_BITS)
    want = np.abs(want) if kind == "m" else np.sqrt(want)
    n = want.size
    blocks = np.concatenate((want, np.zeros(-n % orc.BLOCK))).reshape(-1, orc.BLOCK).max(1)
    np.testing.assert_allclose(scale, blocks / top, rtol=4e-6, err_msg=what)
    per = np.repeat(scale, orc.BLOCK)[:n]
    value = orc.code_values(bits)[code & 127 if kind == "m" else code] * per
    half = np.maximum(want * 2.0 ** -(mantissa + 1), per * 2.0 ** (-bias - mantissa))
    floor = (per * 2.0 ** (1 - bias - mantissa)) if kind == "v" else 0.0            # (a positive v takes at least the smallest code)
    assert np.all(np.abs(value - want) <= half * (1 + 1e-4) + want * 4e-6 + np.where(want < floor, floor - want, 0)), what
    if kind == "v":
        assert np.all(code[want > 0] > 0), what


@pytest.mark.parametrize("offset", (0, 1, 3))
@pytest.mark.parametrize("bits", (32, 8))
@pytest.mark.parametrize("pdt,gdt", TYPES)
def test_step(pdt, gdt, bits, offset):
    s = _lists(SIZES, pdt, gdt, bits, offset=offset)
    b = _host(s)
    _step(s)
    a = _host(s)
    for k, n in enumerate(SIZES):
        if bits == 32:
            m0, v0 = b["m"][k], b["v"][k]
        else:
            m0, v0 = orc.stored_m(b["m"][k], b["m_scale"][k]), orc.stored_v(b["v"][k], b["v_scale"][k])
        p, m, v = orc.adamw(b["params"][k], b["grads"][k], m0, v0, step=5, **RATES)
        _check_params(a["params"][k], b["params"][k], p, pdt, np.abs(m0) + np.abs(b["grads"][k]), v, "params of %d" % n)
        if n == 0:
            continue
        if bits == 32:
            assert np.all(np.abs(a["m"][k] - m) <= 3 * ULP * (np.abs(m0) + np.abs(b["grads"][k]))) and np.all(np.abs(a["v"][k] - v) <= 4 * ULP * v + 1e-38)
        else:
            _check_codes(a["m"][k], a["m_scale"][k], m, "m", "m of %d" % n)
            _check_codes(a["v"][k], a["v_scale"][k], v, "v", "v of %d" % n)
            wrong_sign = (a["m"][k] >= 128) != (m < 0)
            assert np.all(np.abs(m[wrong_sign]) <= 3 * ULP * (np.abs(m0) + np.abs(b["grads"][k]))[wrong_sign])


@pytest.mark.parametrize("bits", (32, 8))
def test_many_tensors_are_many_single_steps(bits):
    """More tensors than one launch describes, in one call and one by one."""
    import torch
    from paper_2502_20168_amd import learn
    rng = np.random.default_rng(0)
    sizes = [int(x) for x in rng.integers(0, 6000, size=131)]
    one, many = _lists(sizes, "f32", "f32", bits), _lists(sizes, "f32", "f32", bits)
    _step(many)
    for k in range(len(sizes)):
        pick = lambda key: None if one[key] is None else [one[key][k]]
        learn.ssm_adamw_step(pick("params"), pick("grads"), pick("m"), pick("v"), pick("m_scale"), pick("v_scale"), **RATES, step=5)
    for key in ("params", "m", "v", "m_scale", "v_scale"):
        for x, y in zip(one[key] or [], many[key] or []):
            assert torch.equal(x, y), key


@pytest.mark.parametrize("bits", (32, 8))
def test_neighbours_are_left_alone(bits):
    """Tensors that share memory with others: nothing outside them changes."""
    import torch
    s = _lists([1000], "f32", "bf16", bits)
    wide = {k: [torch.cat((t[0].new_full((7,), 3), t[0], t[0].new_full((9,), 3)))] for k, t in s.items() if t is not None}
    part = {k: [t[0][7:-9]] for k, t in wide.items()}
    part.setdefault("m_scale", None), part.setdefault("v_scale", None)
    _step(part)
    for k, t in wide.items():
        assert (t[0][:7] == 3).all() and (t[0][-9:] == 3).all(), k


@pytest.mark.parametrize("bits", (32, 8))
def test_grad_scale_and_skip(bits):
    import torch
    s, r = _lists([300, 5000], "f32", "f32", bits), _lists([300, 5000], "f32", "f32", bits)
    r["grads"] = [g * 0.25 for g in r["grads"]]
    _step(s, grad_scale=torch.tensor([0.25], device="cuda"), skip=torch.zeros(1, device="cuda"))
    _step(r)
    keep = _host(s)
    for k in ("params", "m", "v"):
        assert all(torch.equal(x, y) for x, y in zip(s[k], r[k]))
    _step(s, grad_scale=torch.tensor(float("nan"), device="cuda"), skip=torch.ones((), device="cuda"))
    for k, v in _host(s).items():
        assert v is None or all(np.array_equal(x, y) for x, y in zip(v, keep[k]))


def test_values_of_stored_states():
    import torch
    from paper_2502_20168_amd import learn
    s = _lists(SIZES, "f32", "f32", 8)
    m, v = learn.ssm_adamw_values(s["m"], s["v"], s["m_scale"], s["v_scale"])
    h = _host(s)
    for k in range(len(SIZES)):
        np.testing.assert_allclose(m[k].cpu().numpy(), orc.stored_m(h["m"][k], h["m_scale"][k]), rtol=2.0 ** -23)
        np.testing.assert_allclose(v[k].cpu().numpy(), orc.stored_v(h["v"][k], h["v_scale"][k]), rtol=2.0 ** -22)
    # every code, both signs
    code = torch.arange(256, dtype=torch.uint8, device="cuda")
    one = torch.ones(1, device="cuda")
    m, v = learn.ssm_adamw_values([code], [code], [one], [one])
    np.testing.assert_array_equal(m[0].cpu().numpy(), orc.stored_m(np.arange(256), [1.0]))
    np.testing.assert_array_equal(v[0].cpu().numpy(), orc.stored_v(np.arange(256), [1.0]))


def test_stored_states_are_rounded_to_nearest_even():
    """beta 0: m is the gradient itself and v its square, so the codes are those of the gradients."""
    import torch
    from paper_2502_20168_amd import learn
    vals = orc.code_values(orc.M_BITS)[:127]
    mid = (vals[1:] + vals[:-1]) / 2                                  # ties go to the even code
    g = np.concatenate((vals, mid, [448.0], [0.0]))
    s = {"params": [torch.zeros(g.size, device="cuda")], "grads": [torch.tensor(g, dtype=torch.float32, device="cuda")]}
    s.update(learn.ssm_adamw_state(s["params"], 8))
    _step(s, beta1=0.0, beta2=0.0)
    code = s["m"][0].cpu().numpy()
    np.testing.assert_array_equal(code[:127], np.arange(127))
    even = np.where(np.arange(126) % 2 == 0, np.arange(126), np.arange(1, 127))
    np.testing.assert_array_equal(code[127:253], even)
    assert float(s["m_scale"][0][0]) == 1.0


@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
def test_what_is_not_finite_reaches_the_state(bad):
    import torch
    from paper_2502_20168_amd import learn
    s = _lists([600], "f32", "f32", 8)
    s["grads"][0][300] = bad
    _step(s)
    m, v = learn.ssm_adamw_values(s["m"], s["v"], s["m_scale"], s["v_scale"])
    assert not torch.isfinite(m[0][256:512]).any() and not torch.isfinite(v[0][256:512]).any()
    for t in (m[0], v[0], s["params"][0]):
        assert torch.isfinite(t[:256]).all() and torch.isfinite(t[512:]).all()
    assert not torch.isfinite(s["params"][0][300])


def test_zero_gradients_and_tiny_ones():
    import torch
    from paper_2502_20168_amd import learn
    s = _lists([1024], "f32", "f32", 8, history=False)
    s["grads"][0].zero_()
    s["grads"][0][256:512] = 1e-44
    s["grads"][0][512:768] = torch.logspace(-14, 0, 256, device="cuda")
    before = s["params"][0].clone()
    _step(s, step=1, weight_decay=0.0)
    m, v = learn.ssm_adamw_values(s["m"], s["v"], s["m_scale"], s["v_scale"])
    assert not m[0][:512].any() and not v[0][:512].any() and torch.equal(s["params"][0][:256], before[:256])
    assert (v[0][514:768] > 0).all() and torch.isfinite(s["params"][0]).all()


@pytest.mark.parametrize("bits", (32, 8))
def test_a_quadratic_is_minimised(bits):
    import torch
    from paper_2502_20168_amd import learn
    gen = torch.Generator(device="cuda").manual_seed(0)
    target = torch.randn(5000, generator=gen, device="cuda")
    p = torch.zeros(5000, device="cuda")
    st = learn.ssm_adamw_state([p], bits)
    for t in range(1, 401):
        g = p - target
        learn.ssm_adamw_step([p], [g], st["m"], st["v"], st["m_scale"], st["v_scale"], lr=0.05 if t < 300 else 0.005, step=t)
    assert (p - target).abs().max() < 0.05


def test_a_captured_graph_replays_as_the_eager_calls():
    import torch
    s, r = _lists([3000, 77], "f32", "f32", 8), _lists([3000, 77], "f32", "f32", 8)
    _step(_lists([3000, 77], "f32", "f32", 8))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(s)
    for i in range(3):
        new = [torch.randn_like(g) for g in s["grads"]]
        for x, y, z in zip(s["grads"], r["grads"], new):
            x.copy_(z), y.copy_(z)
        graph.replay()
        torch.cuda.synchronize()
        _step(r)
        for k in ("params", "m", "v", "m_scale", "v_scale"):
            assert all(torch.equal(x, y) for x, y in zip(s[k], r[k])), (i, k)
