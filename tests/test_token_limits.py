"""Sizes and buffers at the edge of what the token side's entry points take: host only, nothing is launched."""
import os

import pytest

SHAPE, UNSUPPORTED = 3, 8
P = 0x10000        # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_25120_amd import build
        build.build()
    binding.lib()
    return binding


def refused(B, status, call, **kw):
    with pytest.raises(B.MllmError) as e:
        call(**kw, stream=1)
    assert e.value.status == status, str(e.value)


def qk(t, hq, hkv, head_dim):
    width = (hq + hkv) * head_dim
    return dict(x=P, gamma_q=P, gamma_k=P, t=t, n_q_heads=hq, n_kv_heads=hkv, head_dim=head_dim, x_stride=width, eps=1e-6)


@pytest.mark.parametrize("head_dim", [64, 144, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 1), (4, 1), (14, 1)])
def test_more_heads_than_a_launch_has_threads_for(B, hq, hkv, head_dim):
    """Wide heads take 16 lanes: from 2^28 - 15 heads on, whole workgroups of 256 threads hold 2^32 of them, which no launch has."""
    t = ((1 << 28) - 1) // (hq + hkv)
    assert t * (hq + hkv) == (1 << 28) - 1
    width = (hq + hkv) * head_dim
    refused(B, SHAPE, B.mllm_op_qk_norm_rope_fwd, **qk(t, hq, hkv, head_dim), y=P, y_stride=width)
    refused(B, SHAPE, B.mllm_op_qk_norm_rope_bwd, **qk(t, hq, hkv, head_dim), dy=P, dx=P, dgamma_q=P, dgamma_k=P + 4096, dy_stride=width,
            dx_stride=width, partial=P)


def test_no_scratch_for_more_heads_than_a_call_takes(B):
    size = B.mllm_op_qk_norm_rope_bwd_partial_bytes
    assert size(4, 65536, 65536, 64) > 0
    for hq, hkv in ((65537, 1), (1, 65537), ((1 << 31) - 1, (1 << 31) - 1)):
        assert size(4, hq, hkv, 64) == 0


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("offset", [16, 240, -16, -240])
def test_gains_gradients_that_overlap_in_part(B, offset, accumulate):
    """One buffer for both takes the sum; 64 values each, some of them shared, mean nothing."""
    refused(B, UNSUPPORTED, B.mllm_op_qk_norm_rope_bwd, **qk(4, 4, 2, 64), dy=P, dx=P, dgamma_q=2 * P, dgamma_k=2 * P + offset, dy_stride=384,
            dx_stride=384, partial=P, accumulate=accumulate)
