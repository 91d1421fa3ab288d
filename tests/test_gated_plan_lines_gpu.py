"""The gated recurrence on both sides of every line of the rule that spreads it over the GPU (whether chunks hand states on shows in the workspace)."""
import pytest

from tests.test_gated_gpu import _compare, _inputs

# (Bt, L, D), chunks in workgroups of their own; in pairs, one on either side
LINES = [
    ((3, 64, 16), False), ((3, 65, 16), False),              # a sequence within a wavefront: 8 vectors of channels x 8 threads along time
    ((64, 70, 256), False), ((65, 70, 256), False),          # 256 chains of 64 channels
    ((4, 2048, 64), False), ((4, 2049, 64), True),           # a CU's share is one workgroup of 1024 threads
    ((20, 6144, 64), False), ((20, 6145, 64), True),         # three of them,
    ((20, 6100, 64), False), ((19, 6100, 64), True),         # with 160 chains at least
    ((7, 2000, 1024), False), ((6, 2000, 1024), True),       # 224 chains of 32 channels
    ((1, 4096, 64), True), ((1, 4097, 64), True),            # more than two groups of chunks
    ((20, 6200, 64), True), ((21, 6200, 64), True),          # 1024 workgroups
    ((63, 3200, 64), True), ((64, 3200, 64), True),          # 64 chains: neighbours on one XCD
]


def test_the_sides_of_the_lines():
    import torch
    from paper_2502_20168_amd import learn
    for shape, handed_on in LINES:
        assert (learn.ssm_gated_workspace_bytes(*shape, torch.float32, False) > 0) == handed_on, shape


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("shape", [s for s, _ in LINES])
def test_shapes_at_the_lines(shape, dtype):
    _compare(_inputs(*shape, dtype, False, "some", True), dtype)
