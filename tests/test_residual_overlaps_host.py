"""Overlapping buffers that the residual norms refuse: host only, nothing is launched."""
import os

import pytest

UNSUPPORTED = 8
P = 0x100000       # never dereferenced: validation fails first
T, D = 4, 64
ROWS, VECTOR, STATS = 2 * T * D, 4 * D, 16 * T       # bytes of a matrix, of a gradient, of the statistics


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_25120_amd import build
        build.build()
    binding.lib()
    return binding


INPUTS = dict(dn=P, dy=2 * P, y=3 * P, o=4 * P, stats=5 * P)
PARAMETERS = dict(post_g=20 * P, post_b=21 * P, scale=22 * P, pre_g=23 * P, pre_b=24 * P, gate=25 * P)
GRADS = dict(post_g=10 * P, post_b=11 * P, scale=12 * P, pre_g=13 * P, pre_b=14 * P, gate=15 * P)
OUTPUTS = dict(dx=6 * P, d_o=7 * P, partial=8 * P)


def backward(B, block=None, grads=None, **change):
    """Status and message of a backward call."""
    b = B.ResidualNorm(**{**dict(post_kind=0, pre_kind=0, post_eps=1e-6, pre_eps=1e-6), **PARAMETERS, **(block or {})})
    g = B.ResidualNormGrads(**{**GRADS, **(grads or {})})
    try:
        B.mllm_op_residual_norm_bwd(b, grads=g, t=T, d=D, stream=1, **{**INPUTS, **OUTPUTS, **change})
    except B.MllmError as e:
        return e.status, str(e)
    return 0, ""


def overlaps(result):
    return result[0] == UNSUPPORTED and "overlap" in result[1]


@pytest.mark.parametrize("name,at", [(k, v) for k, v in INPUTS.items()] + [(k, v) for k, v in PARAMETERS.items()])
def test_gradients_and_scratch_that_reach_into_inputs(B, name, at):
    size = STATS if name == "stats" else 4 if name == "gate" else ROWS if name in INPUTS else 2 * D
    for grad in GRADS:
        own = 4 if grad == "gate" else VECTOR
        assert overlaps(backward(B, grads={grad: at})), (grad, name)
        if size >= 16:
            assert overlaps(backward(B, grads={grad: at + size - 16})), (grad, name, "its last bytes")
        if own >= 16:
            assert overlaps(backward(B, grads={grad: at - own + 16})), (grad, name, "from the front")
    assert overlaps(backward(B, partial=at))
    assert overlaps(backward(B, partial=at - B.mllm_op_residual_norm_bwd_partial_bytes(T, D) // 16 * 16))
    for out in ("dx", "d_o"):
        if name not in ("dn", "dy"):            # those two are the ones that they may be
            assert overlaps(backward(B, **{out: at})), (out, name)
        assert overlaps(backward(B, **{out: at - ROWS + 16})), (out, name)


@pytest.mark.parametrize("out", ("dx", "d_o", "partial"))
def test_gradients_that_reach_into_other_outputs(B, out):
    at = OUTPUTS[out]
    size = B.mllm_op_residual_norm_bwd_partial_bytes(T, D) if out == "partial" else ROWS
    for grad in GRADS:
        assert overlaps(backward(B, grads={grad: at}))
        assert overlaps(backward(B, grads={grad: at + (size - 1) // 16 * 16}))
    for other in ("dx", "d_o"):
        if other != out:
            assert overlaps(backward(B, **{out: OUTPUTS[other] + 16}))


def test_gate_of_every_row(B):
    """It has t values, and so has its gradient."""
    each = dict(gate_per_row=True)
    for out in ("dx", "partial"):
        assert overlaps(backward(B, block=each, **{out: PARAMETERS["gate"] + 4 * T - 16}))
    assert overlaps(backward(B, block=each, grads=dict(gate=PARAMETERS["gate"] + 4 * T - 4)))
    assert overlaps(backward(B, block=each, grads=dict(gate=INPUTS["stats"] - 4 * T + 4)))


FORWARD = dict(x=P, o=2 * P, y=3 * P, n=4 * P, stats=5 * P)


def test_forward_results_that_reach_into_parameters(B):
    for name, at in PARAMETERS.items():
        for out, size in (("y", ROWS), ("n", ROWS), ("stats", STATS)):
            for where in (at, at - size + 16):
                b = B.ResidualNorm(post_kind=0, pre_kind=0, post_eps=1e-6, pre_eps=1e-6, **PARAMETERS)
                with pytest.raises(B.MllmError) as e:
                    B.mllm_op_residual_norm_fwd(b, t=T, d=D, stream=1, **{**FORWARD, out: where})
                assert e.value.status == UNSUPPORTED and "overlap" in str(e.value), (out, name)
