"""The gated linear recurrence on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import learn_oracle as orc
from tests.learn_util import DTYPES, check, laid_out, tolerance, torch_dtype

pytestmark = pytest.mark.gpu

# Before the rounding of a result: a gate is good to about 4 units of 2^-24 and the state forgets within 1 / (1 - f) steps, 8 at the mean of the gates
# drawn here and some hundreds in their tail; rounding adds up like the square root of those.
ARITHMETIC = 1e-5


def _inputs(Bt, L, D, dtype, linear, flags, h0, layout="dense", seed=0, bias=2.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen)
    z = rand(Bt, L, D) + bias
    z = torch.sigmoid(z) if linear else z
    dt = torch_dtype(dtype)
    dev = lambda t: laid_out(t.to(dt).cuda(), layout)
    first = {"none": None, "some": torch.rand(Bt, L, generator=gen) < 0.1, "all": torch.ones(Bt, L, dtype=torch.bool)}[flags]
    return {"gate": dev(z), "u": dev(rand(Bt, L, D)), "is_first": None if first is None else first.to(torch.uint8).cuda(),
            "h0": rand(Bt, D).cuda() if h0 else None, "dh": dev(rand(Bt, L, D)), "dh_last": rand(Bt, D).cuda() if h0 else None, "linear": linear}


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _run(s):
    from paper_2502_20168_amd import learn
    f = learn.ssm_gated_scan_fwd(s["gate"], s["u"], s["is_first"], s["h0"], linear=s["linear"])
    b = learn.ssm_gated_scan_bwd(s["gate"], s["u"], s["is_first"], s["h0"], f["carry"], s["dh"], s["dh_last"], linear=s["linear"])
    return f, b


def _compare(s, dtype, arithmetic=ARITHMETIC):
    f, b = _run(s)
    args = [_np(s[k]) for k in ("gate", "u", "is_first", "h0")]
    h = orc.gated_fwd(*args, linear=s["linear"])
    g = orc.gated_bwd(*args, _np(s["dh"]), _np(s["dh_last"]), linear=s["linear"])
    tol = tolerance(dtype, arithmetic)
    check(f["h"], h, tol, "h")
    check(f["h_last"], h[:, -1], arithmetic, "h_last")
    if f["carry"] is not None:
        check(f["carry"], h[:, 127:-1:128][:, :f["carry"].shape[1]], arithmetic, "carry")
    for k in ("dgate", "du"):
        check(b[k], g[k], tol, k)
    check(b["dh0"], g["dh0"], arithmetic, "dh0")


SHAPES = [(1, 1, 1), (2, 1, 3), (3, 2, 5), (1, 3, 2), (70, 7, 9), (4, 16, 64), (1, 127, 64), (2, 128, 66), (2, 129, 4), (1, 257, 130), (5, 300, 250),
          (2, 1025, 16), (1, 4100, 20), (300, 5, 3), (9, 33, 257), (130, 64, 12), (1, 640, 512), (64, 1100, 40), (30, 300, 500), (20, 1030, 250)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Bt,L,D", SHAPES)
def test_shapes(Bt, L, D, dtype):
    _compare(_inputs(Bt, L, D, dtype, False, "some", True), dtype)


@pytest.mark.parametrize("linear", (False, True))
@pytest.mark.parametrize("flags", ("none", "some", "all"))
@pytest.mark.parametrize("h0", (False, True))
@pytest.mark.parametrize("Bt,L,D", [(3, 200, 36), (2, 9, 7)])
def test_resets_and_initial_states(Bt, L, D, flags, h0, linear):
    _compare(_inputs(Bt, L, D, "f32", linear, flags, h0), "f32")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ("halves", "time", "odd"))
@pytest.mark.parametrize("Bt,L,D", [(3, 150, 70), (2, 5, 3), (4, 260, 64)])
def test_layouts(Bt, L, D, layout, dtype):
    _compare(_inputs(Bt, L, D, dtype, False, "some", True, layout), dtype)


@pytest.mark.parametrize("bias", (6.0, 30.0, -30.0, 200.0, -200.0))
def test_gates_near_one_and_zero(bias):
    # near one the state sums its inputs' remainders over the whole sequence: sqrt(600) roundings more than a state that forgets
    _compare(_inputs(2, 600, 20, "f32", False, "some", True, bias=bias), "f32", 5e-5)


def test_a_long_sequence_of_a_few_channels():
    _compare(_inputs(1, 20000, 4, "f32", False, "none", True, bias=4.0), "f32", 5e-5)
    _compare(_inputs(2, 9000, 24, "bf16", True, "some", True, bias=3.0), "bf16", 5e-5)


def test_chunks_groups_and_blocks_of_groups_hand_states_on():
    """One channel block, 128 steps to a chunk of 16 rows, 16 chunks to a group, 16 groups to a block: a sequence over three blocks, its carries compared with the
    oracle's states and the gradient with the definition in 64 bits, where resets lie in few places and the state forgets slowly."""
    import torch
    L = 2 * 128 * 256 + 5 * 128 * 16 + 3 * 128 + 17
    s = _inputs(1, L, 64, "f32", False, "none", True, bias=7.0)
    s["is_first"] = torch.zeros(1, L, dtype=torch.uint8, device="cuda")
    s["is_first"][0, [40000, 65535, 65536 + 3]] = 1
    _compare(s, "f32", 1e-4)                 # a state of 1100 steps: a gate near one is good to 2^-24, times the steps it is raised to, times the root of what is added up


def test_a_sequence_in_two_parts():
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(3, 700, 40, "f32", False, "some", True)
    whole, _ = _run(s)
    cut = lambda t, a, b: t[:, a:b]
    one = learn.ssm_gated_scan_fwd(cut(s["gate"], 0, 301), cut(s["u"], 0, 301), s["is_first"][:, :301].contiguous(), s["h0"])
    two = learn.ssm_gated_scan_fwd(cut(s["gate"], 301, 700), cut(s["u"], 301, 700), s["is_first"][:, 301:].contiguous(), one["h_last"])
    got = torch.cat((one["h"], two["h"]), 1)
    assert (got - whole["h"]).abs().max() <= 1e-5 * whole["h"].abs().max()
    assert (two["h_last"] - whole["h_last"]).abs().max() <= 1e-5 * whole["h_last"].abs().max()


@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
@pytest.mark.parametrize("linear", (False, True))
@pytest.mark.parametrize("L", (40, 500))
def test_a_reset_drops_what_is_not_finite(L, linear, bad):
    """Before step 21 forwards, and behind it backwards, everything that is not finite stays on its side of the reset."""
    import torch
    s = _inputs(2, L, 12, "f32", linear, "none", True)
    clean = {k: v.clone() if torch.is_tensor(v) else v for k, v in s.items()}
    first = torch.zeros(2, L, dtype=torch.uint8, device="cuda")
    first[:, 21] = 1
    s["is_first"] = clean["is_first"] = first
    s["u"][:, 20] = bad
    s["h0"][0] = bad
    f, _ = _run(s)
    ref, _ = _run(clean)
    assert torch.equal(f["h"][:, 21:], ref["h"][:, 21:]) and torch.equal(f["h_last"], ref["h_last"])
    assert not torch.isfinite(f["h"][:, 20]).any()
    s["u"], s["h0"] = clean["u"], clean["h0"]
    s["dh"][:, 21:] = bad
    _, b = _run(s)
    _, ref = _run(clean)
    for k in ("du", "dgate"):
        assert torch.equal(b[k][:, :21], ref[k][:, :21])
    assert torch.equal(b["dh0"], ref["dh0"])


def test_not_a_number_reaches_the_results():
    """Without a reset a NaN in the gate, the input or the initial state is seen to the end, through every decay."""
    import torch
    for key in ("gate", "u", "h0"):
        s = _inputs(1, 1500, 8, "f32", False, "none", True, bias=-3.0)
        (s[key] if key == "h0" else s[key][:, 1])[0, 3] = float("nan")
        f, b = _run(s)
        assert torch.isnan(f["h_last"][0, 3]) and torch.isfinite(f["h_last"][0, :3]).all()
        assert torch.isnan(b["dgate"][0, 2:, 3]).all() and torch.isfinite(b["dgate"][0, :, 4:]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("linear", (False, True))
@pytest.mark.parametrize("Bt,D,pitch", [(1, 1, 1), (3, 5, 5), (16, 512, 512), (7, 33, 70), (1000, 130, 131)])
def test_step(Bt, D, pitch, linear, dtype):
    import torch
    from paper_2502_20168_amd import learn
    gen = torch.Generator().manual_seed(4)
    dt = torch_dtype(dtype)
    z, u = (torch.randn(Bt, pitch, generator=gen).to(dt).cuda()[:, :D] for _ in range(2))
    h, first = torch.randn(Bt, D, generator=gen).cuda(), (torch.rand(Bt, generator=gen) < 0.3).to(torch.uint8).cuda()
    ref = orc.gated_fwd(_np(z)[:, None], _np(u)[:, None], _np(first)[:, None], _np(h), linear)[:, 0]
    y, new = learn.ssm_gated_step(z, u, h, first, linear=linear)
    check(y, ref, tolerance(dtype, 2e-6), "y")
    check(new, ref, 2e-6, "h")
    _, same = learn.ssm_gated_step(z, u, h, first, linear=linear, h=h)              # in place
    assert same is h and torch.equal(h, new)
    y0, _ = learn.ssm_gated_step(z, u, linear=linear)
    check(y0, orc.gated_fwd(_np(z)[:, None], _np(u)[:, None], linear=linear)[:, 0], tolerance(dtype, 2e-6), "y from nothing")


def test_steps_one_by_one_are_the_scan():
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(4, 12, 20, "f32", False, "some", True)
    f, _ = _run(s)
    h = s["h0"].clone()
    for t in range(12):
        y, h = learn.ssm_gated_step(s["gate"][:, t], s["u"][:, t], h, s["is_first"][:, t].contiguous())
        assert (y - f["h"][:, t]).abs().max() <= 1e-6 * f["h"].abs().max()
    assert (h - f["h_last"]).abs().max() <= 1e-6 * f["h"].abs().max()


def test_given_outputs_streams_and_repeats():
    import torch
    from paper_2502_20168_amd import learn
    s = _inputs(4, 1300, 72, "bf16", False, "some", True)
    f, b = _run(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = {"h": torch.empty(1300, 4, 72, dtype=torch.bfloat16, device="cuda").transpose(0, 1)}
    g = learn.ssm_gated_scan_fwd(s["gate"], s["u"], s["is_first"], s["h0"], out=out, stream=side)
    c = learn.ssm_gated_scan_bwd(s["gate"], s["u"], s["is_first"], s["h0"], g["carry"], s["dh"], s["dh_last"], stream=side, want_dh0=False)
    torch.cuda.synchronize()
    assert g["h"] is out["h"] and c["dh0"] is None
    for x, y in ((f, g), (b, c)):
        for k in x:
            if y[k] is not None:
                assert torch.equal(x[k], y[k]), k


def test_a_captured_graph_replays_as_the_eager_calls():
    import torch
    s = _inputs(3, 1300, 40, "f32", False, "some", True)
    _run(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f, b = _run(s)
    for seed in (5, 6, 7):
        new = _inputs(3, 1300, 40, "f32", False, "some", True, seed=seed)
        for k, v in new.items():
            if torch.is_tensor(v):
                s[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        g, c = _run(s)
        for x, y in ((f, g), (b, c)):
            for k in x:
                assert torch.equal(x[k], y[k]), k


@pytest.mark.parametrize("flags", ("none", "some"))
@pytest.mark.parametrize("L", (4000, 9000))
def test_a_wait_that_gives_up_hands_on_nan(L, flags):
    """A poll bound of zero: a chunk whose predecessor is not ready yet gives up at once, every channel for itself.  Whatever happened, the states and gradients are
    right or NaN, never something else, and the workspace says so."""
    import torch
    from paper_2502_20168_amd import binding, learn
    s = _inputs(2, L, 64, "f32", False, flags, True)
    ref, back = _run(s)
    n = learn.ssm_gated_workspace_bytes(2, L, 64, torch.float32, False)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    fwd = lambda: learn.ssm_gated_scan_fwd(s["gate"], s["u"], s["is_first"], s["h0"], workspace=ws)
    bwd = lambda: learn.ssm_gated_scan_bwd(s["gate"], s["u"], s["is_first"], s["h0"], ref["carry"], s["dh"], s["dh_last"], workspace=ws)
    for call, right in ((fwd, ref), (bwd, back)):
        for _ in range(4):
            old = binding.ssm_set_spin_limit(0)
            try:
                r = call()
                status = learn.ssm_workspace_status(ws)
            finally:
                binding.ssm_set_spin_limit(old)
            seen = False
            for k, t in r.items():
                bad = torch.isnan(t)
                seen |= bool(bad.any())
                assert torch.equal(t[~bad], right[k][~bad]), k
            assert status == binding.SSM_ERR_SCAN_TIMEOUT or not seen
        r = call()
        assert learn.ssm_workspace_status(ws) == binding.SSM_OK
        for k, t in r.items():
            assert torch.equal(t, right[k]), k


def test_a_workspace_too_small_is_refused():
    import torch
    from paper_2502_20168_amd import binding, learn
    s = _inputs(2, 4000, 64, "f32", False, "none", True)
    n = learn.ssm_gated_workspace_bytes(2, 4000, 64, torch.float32, False)
    with pytest.raises(learn.SsmError) as e:
        learn.ssm_gated_scan_fwd(s["gate"], s["u"], workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.SSM_ERR_WORKSPACE
