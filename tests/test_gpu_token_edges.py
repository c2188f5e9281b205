"""Calls at the edge of what the token side's entry points document, each against its definition in float64."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_token_ops import FP32, SHAPES, Heads, within  # noqa: E402


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


# ---------------------------------------------------------------------------------------------
# per-head norm and rotation
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("t,hq,hkv,hd", SHAPES)
def test_one_gradient_for_both_gains(B, t, hq, hkv, hd, rotate):
    """Queries and keys with one gain: its gradient is the sum of both, overwritten or added."""
    p = Heads(B, t, hq, hkv, hd, rotate)
    _, _, sums, sizes = p.want_bwd()
    dx, q, k = torch.empty_like(p.x), torch.empty(hd, device="cuda"), torch.empty(hd, device="cuda")
    p.bwd(p.dy, p.x, dx, q, k)
    both = torch.full((hd,), float("nan"), device="cuda")
    p.bwd(p.dy, p.x, dx, both, both)
    assert torch.equal(both, q + k)                          # the terms of two buffers, added once
    want, bound = sums[0] + sums[1], sizes[0] + sizes[1] + (sums[0].abs() + sums[1].abs()) * FP32
    within(both, want, bound)
    p.bwd(p.dy, p.x, dx, both, both, accumulate=1)
    within(both, 2 * want, 2 * bound + 4 * (sums[0].abs() + sums[1].abs()) * FP32)      # two more additions
