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
