"""What the entry points of the token side refuse, and the sizes they ask for: host only, nothing is launched."""
import os

import pytest

NULL, SHAPE, WORKSPACE, UNSUPPORTED = 1, 3, 7, 8
P = 0x10000        # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_25120_amd import build
        build.build()
    binding.lib()
    return binding


def refused(B, status, call, *args, **kw):
    with pytest.raises(B.MllmError) as e:
        call(*args, stream=1, **kw)
    assert e.value.status == status, str(e.value)


@pytest.mark.parametrize("status,change", [
    (NULL, dict(table=None)), (NULL, dict(ids=None)), (NULL, dict(y=None)),
    (SHAPE, dict(t=-1)), (SHAPE, dict(t=1 << 31)), (SHAPE, dict(vocab=0)), (SHAPE, dict(vocab=1 << 31)),
    (SHAPE, dict(d=0)), (SHAPE, dict(d=60)), (SHAPE, dict(d=-64)), (SHAPE, dict(d=(1 << 20) + 8)),
    (SHAPE, dict(y_stride=56)), (SHAPE, dict(y_stride=68)),
    (UNSUPPORTED, dict(table=P + 8)), (UNSUPPORTED, dict(y=P + 2)),
])
def test_embed_fwd_refusals(B, status, change):
    refused(B, status, B.mllm_op_embed_fwd, **{**dict(table=P, ids=P, y=P, t=4, vocab=10, d=64), **change})


@pytest.mark.parametrize("status,change", [
    (NULL, dict(dy=None)), (NULL, dict(ids=None)), (NULL, dict(dtable=None)), (NULL, dict(workspace=None)),
    (SHAPE, dict(t=-1)), (SHAPE, dict(vocab=0)), (SHAPE, dict(d=60)), (SHAPE, dict(dy_stride=56)), (SHAPE, dict(dy_stride=65)),
    (UNSUPPORTED, dict(dy=P + 8)), (UNSUPPORTED, dict(dtable=P + 4)),
    (WORKSPACE, dict(workspace=P + 16)), (WORKSPACE, dict(short=1)),
])
def test_embed_bwd_refusals(B, status, change):
    need = B.mllm_op_embed_bwd_workspace_bytes(4, 10, 64)
    kw = {**dict(dy=P, ids=P, dtable=P, t=4, vocab=10, d=64, workspace=P, workspace_bytes=need), **change}
    kw["workspace_bytes"] -= kw.pop("short", 0)
    refused(B, status, B.mllm_op_embed_bwd, **kw)


def test_embed_bwd_workspace_serves_fewer_tokens(B):
    """One buffer sized for the longest microbatch serves every shorter one."""
    for vocab, d in ((10, 64), (50257, 3584), (131072, 4096), (1000000, 8)):
        sizes = [B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d) for t in (0, 1, 2, 31, 64, 65, 1000, 5000, 32768, 1000000)]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[1] > 0
    assert B.mllm_op_embed_bwd_workspace_bytes(-1, 10, 64) == 0 and B.mllm_op_embed_bwd_workspace_bytes(4, 0, 64) == 0


QK = dict(x=P, gamma_q=P, gamma_k=P, t=4, n_q_heads=4, n_kv_heads=2, head_dim=64, x_stride=512, eps=1e-6, pos=P, rope_table=P, n_pos=8)
QK_BOTH = [
    (NULL, dict(x=None)), (NULL, dict(gamma_q=None)), (NULL, dict(gamma_k=None)), (NULL, dict(pos=None)),
    (SHAPE, dict(t=-1)), (SHAPE, dict(t=1 << 29)), (SHAPE, dict(n_q_heads=0)), (SHAPE, dict(n_kv_heads=-1)), (SHAPE, dict(n_q_heads=1 << 17)),
    (UNSUPPORTED, dict(head_dim=0)), (UNSUPPORTED, dict(head_dim=72)), (UNSUPPORTED, dict(head_dim=272)),
    (SHAPE, dict(x_stride=376)), (SHAPE, dict(x_stride=388)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=float("nan"))), (SHAPE, dict(n_pos=-1)),
    (UNSUPPORTED, dict(x=P + 8)), (UNSUPPORTED, dict(gamma_q=P + 2)), (UNSUPPORTED, dict(gamma_k=P + 2)), (UNSUPPORTED, dict(rope_table=P + 4)),
]


@pytest.mark.parametrize("status,change", QK_BOTH + [(NULL, dict(y=None)), (SHAPE, dict(y_stride=380)), (UNSUPPORTED, dict(y=P + 8))])
def test_qk_norm_rope_fwd_refusals(B, status, change):
    refused(B, status, B.mllm_op_qk_norm_rope_fwd, **{**QK, **dict(y=P, y_stride=512), **change})


@pytest.mark.parametrize("status,change", QK_BOTH + [
    (NULL, dict(dy=None)), (NULL, dict(dx=None)), (NULL, dict(dgamma_q=None)), (NULL, dict(dgamma_k=None)), (NULL, dict(partial=None)),
    (SHAPE, dict(dy_stride=380)), (SHAPE, dict(dx_stride=380)), (UNSUPPORTED, dict(dy=P + 8)), (UNSUPPORTED, dict(dx=P + 8)),
    (UNSUPPORTED, dict(dgamma_q=P + 4)), (UNSUPPORTED, dict(dgamma_k=P + 4)), (UNSUPPORTED, dict(partial=P + 4))])
def test_qk_norm_rope_bwd_refusals(B, status, change):
    refused(B, status, B.mllm_op_qk_norm_rope_bwd,
            **{**QK, **dict(dy=P, dx=P, dgamma_q=P, dgamma_k=P, dy_stride=512, dx_stride=512, partial=P), **change})


def test_qk_norm_rope_partial_bytes(B):
    assert B.mllm_op_qk_norm_rope_bwd_partial_bytes(-1, 4, 2, 64) == 0 and B.mllm_op_qk_norm_rope_bwd_partial_bytes(4, 0, 2, 64) == 0
    sizes = [B.mllm_op_qk_norm_rope_bwd_partial_bytes(t, 32, 8, 128) for t in (0, 1, 100, 10000, 1000000)]
    assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] <= 4 << 20      # does not grow with the tokens for good


@pytest.mark.parametrize("status,change", [
    (NULL, dict(logits=None)), (NULL, dict(targets=None)), (NULL, dict(loss=None)),
    (SHAPE, dict(t=-1)), (SHAPE, dict(t=1 << 31)), (SHAPE, dict(vocab=0)), (SHAPE, dict(vocab=65)), (SHAPE, dict(cols=60, vocab=50)),
    (SHAPE, dict(logits_stride=56)), (SHAPE, dict(logits_stride=68)), (SHAPE, dict(dlogits_stride=56)),
    (UNSUPPORTED, dict(logits=P + 8)), (UNSUPPORTED, dict(dlogits=P + 4)),
    (UNSUPPORTED, dict(dlogits=P + 16)),                                   # overlaps the logits
    (UNSUPPORTED, dict(dlogits=P, logits_fp32=1)),                         # in place, another type
    (UNSUPPORTED, dict(dlogits=P, dlogits_stride=72)),                     # in place, another stride
])
def test_xent_refusals(B, status, change):
    refused(B, status, B.mllm_op_xent, **{**dict(logits=P, targets=P, loss=P, dlogits=2 * P, t=4, vocab=61, cols=64), **change})
