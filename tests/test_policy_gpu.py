"""The clipped policy loss on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import learn_oracle as orc
from tests.learn_util import DTYPES, check, tolerance, torch_dtype

pytestmark = pytest.mark.gpu

# exponents up to about 20 carry 20 * 2^-24 into a probability and a logarithm; sums of positive terms add little
ARITHMETIC = 1e-5
TERMS = {"clip_low": 0.2, "clip_high": 0.3, "kl_coef": 0.1, "entropy_coef": 0.05}


def _inputs(N, K, dtype="f32", pad=0, masked=0.0, idle=0.0, ref=True, seed=0, scale=2.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(N, K + pad, generator=gen) * scale).to(torch_dtype(dtype))
    a = torch.randint(K, (N,), generator=gen)
    if masked:
        out = torch.rand(N, K + pad, generator=gen) < masked
        out[torch.arange(N), a] = False
        x[out] = -float("inf")
    x[:, K:] = float("nan")
    logp = torch.log_softmax(x[:, :K].double(), 1).gather(1, a[:, None])[:, 0].float()
    w = torch.rand(N, generator=gen) / N
    w[torch.rand(N, generator=gen) < idle] = 0
    s = {"logits": x.cuda()[:, :K], "action": a.cuda(), "logp_old": (logp + 0.3 * torch.randn(N, generator=gen)).cuda(),
         "advantage": torch.randn(N, generator=gen).cuda(), "weight": w.cuda(), "logp_ref": (logp + 0.3 * torch.randn(N, generator=gen)).cuda() if ref else None}
    return s


def _oracle(s, dloss=1.0, terms=TERMS):
    n = lambda t: None if t is None else t.double().cpu().numpy()
    return orc.policy_loss(n(s["logits"]), s["action"].cpu().numpy(), n(s["logp_old"]), n(s["advantage"]), n(s["weight"]), n(s["logp_ref"]),
                           dloss=dloss, **terms)


def _finite(t):
    import torch
    return torch.where(t == -float("inf"), torch.zeros_like(t), t)


def _compare(s, dtype, terms=TERMS):
    import torch
    from paper_2502_20168_amd import learn
    ref = _oracle(s, 1.0, terms)
    args = tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **terms)
    g = learn.ssm_policy_loss_grad(*args, **terms)
    b = learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **terms)
    for r in (f, g):
        assert abs(float(r["loss"]) - ref["loss"]) <= ARITHMETIC * np.sum(np.abs(s["weight"].cpu().numpy() if s["weight"] is not None else 1.0)) * 8
        check(r["logp"], ref["logp"], ARITHMETIC, "logp")
        check(r["entropy"], ref["entropy"], ARITHMETIC, "entropy")
        assert np.array_equal(np.isinf(ref["lse"]), torch.isinf(r["lse"]).cpu().numpy())
        check(_finite(r["lse"]), np.where(np.isinf(ref["lse"]), 0, ref["lse"]), ARITHMETIC, "lse")
    for d in (g["dlogits"], b):
        assert d.dtype == s["logits"].dtype
        check(d, ref["dlogits"], tolerance(dtype, 3 * ARITHMETIC), "dlogits")
    return f, g, b


SHAPES = [(1, 1), (3, 2), (5, 3), (64, 7), (33, 32), (17, 33), (9, 64), (300, 65), (4, 255), (6, 256), (2, 1000), (3, 1025), (2, 2048), (7, 5003),
          (1, 16384), (2, 20001), (1, 40000), (2, 70001), (1, 140000), (1, 300001),
          (64, 9001), (65, 9001), (40, 16400), (2, 1200003), (66, 33000), (70, 70001), (513, 33000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K", SHAPES)
def test_shapes(N, K, dtype):
    _compare(_inputs(N, K, dtype, masked=0.2 if K > 3 else 0.0), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K,pad", [(40, 5, 1), (11, 130, 3), (3, 3000, 7), (2, 33000, 5), (66, 70001, 3)])
def test_rows_in_a_padded_array(N, K, pad, dtype):
    _compare(_inputs(N, K, dtype, pad=pad, idle=0.3), dtype)


@pytest.mark.parametrize("kl,eta", [(0.0, 0.0), (0.2, 0.0), (0.0, 0.1)])
@pytest.mark.parametrize("N,K", [(200, 18), (5, 3000)])
def test_terms(N, K, kl, eta):
    _compare(_inputs(N, K, ref=kl > 0), "f32", {"clip_low": 0.1, "clip_high": 0.4, "kl_coef": kl, "entropy_coef": eta})


def test_many_rows_and_the_mean():
    s = _inputs(70000, 6, ref=False)
    s["weight"] = None
    _compare(s, "f32")


@pytest.mark.parametrize("K", (6, 70, 3001, 70001))
def test_idle_rows_hold_anything(K):
    """Weight zero, a negative action, no action that can be taken: nothing of the row's logits reaches a result."""
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(8, K)
    s["logits"][1] = float("nan")
    s["weight"][1] = 0
    s["logits"][3] = float("inf")
    s["action"][3] = -1
    s["logits"][5] = -float("inf")
    clean = dict(s, logits=s["logits"].clone())
    clean["logits"][[1, 3, 5]] = 0
    clean["weight"] = s["weight"].clone()
    clean["weight"][[1, 3, 5]] = 0
    _compare(clean, "f32")
    args = tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **TERMS)
    g = learn.ssm_policy_loss_grad(*args, **TERMS)
    b = learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **TERMS)
    ref = learn.ssm_policy_loss_grad(*clean.values(), **TERMS)
    for k in ("loss", "logp", "entropy", "lse"):
        assert torch.equal(f[k], ref[k]) and torch.equal(g[k], ref[k]), k
    assert torch.equal(g["dlogits"], ref["dlogits"])
    for d in (g["dlogits"], b):
        assert not d[[1, 3, 5]].any() and torch.isfinite(d).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", (9, 400, 9000))
def test_the_types_lowest_value_masks(K, dtype):
    import torch
    s = _inputs(4, K, dtype)
    low = torch.finfo(s["logits"].dtype).min
    out = torch.rand(4, K, device="cuda") < 0.4
    out[torch.arange(4), s["action"].cuda()] = False
    s["logits"][out] = low
    s["logits"][2] = low                                 # a row of nothing but the lowest value is uniform
    s["logp_old"][2] = s["logp_ref"][2] = -float(np.log(K))
    _, g, _ = _compare(s, dtype)
    keep = out.clone()
    keep[2] = False
    assert not g["dlogits"][keep].any()


@pytest.mark.parametrize("K", (5, 300, 9000))
def test_what_is_not_a_number_reaches_the_results(K):
    import torch
    from paper_2502_20168_amd import learn
    for bad, where in ((float("nan"), "one"), (float("inf"), "one"), (float("nan"), "beside nothing"), (0.0, "action")):
        s = _inputs(3, K)
        if where == "beside nothing":
            s["logits"][1] = -float("inf")
        if where == "action":
            s["action"][1] = K
        else:
            s["logits"][1, K - 2] = bad
        f = learn.ssm_policy_loss_fwd(*s.values(), **TERMS)
        g = learn.ssm_policy_loss_grad(*s.values(), **TERMS)
        for r in (f, g):
            assert torch.isnan(r["loss"]) and torch.isnan(r["logp"][1]) and torch.isfinite(r["logp"][[0, 2]]).all()
        assert torch.isnan(g["dlogits"][1]).any() and torch.isfinite(g["dlogits"][[0, 2]]).all()


def test_ratios_that_overflow():
    """exp(logp - logp_old) beyond the range: a positive advantage is clipped, one of zero adds nothing, a negative one is infinite."""
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(3, 12, ref=False)
    s["logp_old"][:] = -200.0
    s["weight"][:] = 1.0
    terms = {"clip_low": 0.2, "clip_high": 0.3}
    for A, want in ((2.0, -2.6), (0.0, 0.0), (-1.0, float("inf"))):
        s["advantage"][:] = A
        g = learn.ssm_policy_loss_grad(*(t[:1] if t is not None else None for t in s.values()), **terms)
        assert float(g["loss"]) == pytest.approx(want, rel=1e-6)
        if A >= 0:
            assert not g["dlogits"].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K", [(50, 20), (4, 700), (3, 5003), (2, 50001), (1, 200003), (66, 70001)])
def test_gradient_over_the_logits(N, K, dtype):
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(N, K, dtype, pad=3, idle=0.2)
    ref = learn.ssm_policy_loss_grad(*s.values(), **TERMS)
    args = tuple(s.values())
    f = learn.ssm_policy_loss_fwd(*args, **TERMS)
    b = learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], **TERMS)
    keep = s["logits"].clone()
    got = learn.ssm_policy_loss_grad(*args, out={"dlogits": s["logits"]}, **TERMS)
    assert got["dlogits"] is s["logits"] and torch.equal(s["logits"], ref["dlogits"])
    s["logits"].copy_(keep)
    assert torch.equal(learn.ssm_policy_loss_bwd(*args, f["logp"], f["entropy"], f["lse"], dlogits=s["logits"], **TERMS), b)


def test_gradient_times_a_scalar_streams_and_repeats():
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(37, 1500)
    d = torch.tensor(-2.5, device="cuda")
    ref = _oracle(s, -2.5)["dlogits"]
    g = learn.ssm_policy_loss_grad(*s.values(), d, **TERMS)
    f = learn.ssm_policy_loss_fwd(*s.values(), **TERMS)
    b = learn.ssm_policy_loss_bwd(*s.values(), f["logp"], f["entropy"], f["lse"], d, **TERMS)
    check(g["dlogits"], ref, 4e-5, "dlogits")
    check(b, ref, 4e-5, "dlogits")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h = learn.ssm_policy_loss_grad(*s.values(), d, stream=side, **TERMS)
    torch.cuda.synchronize()
    for k in g:
        assert torch.equal(g[k], h[k]), k


def test_a_captured_graph_replays_as_the_eager_calls():
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(100, 700)
    run = lambda: learn.ssm_policy_loss_grad(*s.values(), **TERMS)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = run()
    for seed in (5, 6, 7):
        for k, v in _inputs(100, 700, seed=seed).items():
            s[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        e = run()
        for k in r:
            assert torch.equal(r[k], e[k]), k
