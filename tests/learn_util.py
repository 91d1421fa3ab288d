"""Helpers of the tests of the learner's operators: types, layouts, tolerances."""
import numpy as np

DTYPES = ("f32", "bf16", "f16")
# Relative rounding of one store: half a unit in the last place (24, 8 and 11 significant bits).
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def torch_dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def tolerance(dtype, arithmetic):
    """One rounding to the type of the result, and `arithmetic` for what fp32 operations lose before it."""
    return ROUND[dtype] * 1.01 + arithmetic


def check(got, ref, tol, name):
    """max|got - ref| <= tol max|ref| and the same of the norms, and half a step where numbers of the type become fixed-point (f16), or for
    f32 and bf16 what a factor below 2^-126 that was taken for zero leaves behind after products with others of up to 2^10."""
    import torch
    step = 2.0 ** -25 * 1.01 if got.dtype == torch.float16 else 2.0 ** -116
    got = got.detach().double().cpu().numpy()
    ref = np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.all(np.isfinite(got)), name + " has non-finite values"
    d = np.abs(got - ref)
    big, norm = np.abs(ref).max(), np.linalg.norm(ref)
    assert d.max() <= tol * big + step, "%s: off by %.3e where the largest value is %.3e (allowed %.3e of it)" % (name, d.max(), big, tol)
    assert np.linalg.norm(d) <= tol * norm + step * d.size ** 0.5, "%s: off by %.3e where the norm is %.3e (allowed %.3e of it)" % (name, np.linalg.norm(d), norm, tol)


def laid_out(x, layout):
    """A tensor [Bt, L, D] with the values of x in memory as the layout says."""
    import torch
    if layout == "dense":
        return x.contiguous()
    if layout == "halves":
        return torch.cat((x, torch.full_like(x, float("nan"))), -1)[..., :x.shape[-1]]
    if layout == "time":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "odd":                                  # rows of no aligned length that start at an odd element
        Bt, L, D = x.shape
        buf = torch.full((Bt * (L * (D + 3) + 5) + 1,), float("nan"), dtype=x.dtype, device=x.device)
        v = buf[1:].as_strided((Bt, L, D), (L * (D + 3) + 5, D + 3, 1), 1)
        v.copy_(x)
        return v
    raise ValueError(layout)
