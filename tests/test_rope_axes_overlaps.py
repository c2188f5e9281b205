"""Buffers of the rotation by several axes that lie in one another: what is refused (host only, nothing is launched) and what is not."""
import os

import pytest

UNSUPPORTED = 8
P = 0x100000       # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_25120_amd import build
        build.build()
    binding.lib()
    return binding


CALL = dict(x=P, y=2 * P, pos=3 * P, axes=[0, 1] * 16, table=4 * P, n_pos=8, t=4, n_heads=4, head_dim=64, x_stride=256, y_stride=256)
LAST_Y = 2 * P + 2 * 4 * 256 - 16          # the result's last 16 bytes


def overlaps(B, **change):
    kw = {**CALL, **change}
    with pytest.raises(B.MllmError) as e:
        B.mllm_op_rope_axes(**{**kw, "axes": B.pair_axes(kw["axes"])}, stream=1)
    return e.value.status == UNSUPPORTED and "overlap" in str(e.value)


@pytest.mark.parametrize("change", [
    dict(pos=2 * P), dict(pos=LAST_Y + 12), dict(pos=2 * P - 2 * 4 * 4 + 4),                            # two axes of four positions
    dict(pos=2 * P - 10 * 4 * 4, pos_stride=40), dict(pos=2 * P - 4 * 4 + 4, axes=[0] * 32),
    dict(table=2 * P), dict(table=LAST_Y), dict(table=2 * P - 8 * 64 * 4 + 16),
    dict(x=2 * P, pos=2 * P),                                                                          # in place
])
def test_result_over_positions_or_table(B, change):
    assert overlaps(B, **change)


@pytest.mark.parametrize("change", [
    dict(y=P + 2 * 248, x_stride=512, y_stride=512),            # eight columns short of the next ones
    dict(y=P + 2 * 264, x_stride=512, y_stride=512),            # the last eight reach into the next row
    dict(x=P + 2 * 264, y=P, x_stride=512, y_stride=512),
    dict(y=P + 2 * 512 + 16, x_stride=512, y_stride=512),
    dict(y=P + 2 * 256, x_stride=512, y_stride=520),            # another stride: the columns move from row to row
])
def test_columns_of_one_buffer_that_do_overlap(B, change):
    assert overlaps(B, **change)


@pytest.mark.gpu
@pytest.mark.parametrize("first,second", [(0, 256), (256, 0), (0, 320), (8, 264), (312, 0)])
@pytest.mark.parametrize("t", [1, 5, 3000])
def test_other_columns_of_one_buffer(B, t, first, second):
    """Heads turned from one part of a buffer's rows into another: they share no byte.  The same bits as into a buffer of its own, and nothing else changes."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(t)
    buffer = torch.randn(t, 576, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, 50, (2, t), generator=g, device="cuda", dtype=torch.int32)
    table = torch.empty(50, 64, device="cuda")
    B.mllm_op_rope_freq_table(table, 50, [1.0 / (1 + i) for i in range(32)])
    x, axes = buffer[:, first:first + 256].contiguous(), B.pair_axes([0, 1] * 16)
    want = torch.empty_like(x)
    B.mllm_op_rope_axes(x, want, pos, axes, table, 50, t, 4, 64, 256, 256)
    expected = buffer.clone()
    expected[:, second:second + 256] = want
    B.mllm_op_rope_axes(buffer[:, first:], buffer[:, second:], pos, axes, table, 50, t, 4, 64, 576, 576)
    assert torch.equal(buffer, expected)
