"""What the entry points around a layer's products refuse, and the sizes they ask for: host only, nothing is launched."""
import os

import numpy as np
import pytest

NULL, SHAPE, CU_SEQLENS, INDEX, WORKSPACE, UNSUPPORTED = 1, 3, 4, 6, 7, 8
P = 0x100000       # never dereferenced: validation fails first


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


GRID = (2, 1, 2, 2, 1)


@pytest.mark.parametrize("status,cu,grids", [
    (CU_SEQLENS, [1, 8], []), (CU_SEQLENS, [0, 8, 7], []),
    (INDEX, [0, 8], [(5, 1, 2, 2, 1)]),                       # goes beyond its sample
    (INDEX, [0, 5, 8], [(4, 1, 2, 1, 1)]),                    # into the next one
    (INDEX, [0, 8], [GRID, (5, 1, 1, 1, 1)]),                 # begins inside the one in front
    (INDEX, [0, 8], [GRID, GRID]), (INDEX, [0, 8], [(6, 1, 1, 1, 1), (1, 1, 1, 1, 1)]),
    (INDEX, [0, 8], [(8, 1, 1, 1, 1)]), (INDEX, [0, 8], [(-1, 1, 1, 1, 1)]), (INDEX, [0], [(0, 1, 1, 1, 1)]),
    (SHAPE, [0, 8], [(2, 0, 2, 2, 1)]), (SHAPE, [0, 8], [(2, 1, -2, -2, 1)]), (SHAPE, [0, 8], [(2, 1, 2, 0, 1)]), (SHAPE, [0, 8], [(2, 2, 1, 2, -1)]),
    (INDEX, [0, 1 << 30], [(2, 1 << 20, 1 << 20, 1 << 20, 1)]),   # a product of 2^60 rows
    (INDEX, [0, 1 << 30], [(2, 3, (1 << 31) - 1, (1 << 31) - 1, 1)]),
    (SHAPE, [0, 100], [(0, 50, 1, 1, 1 << 27), (60, 3, 1, 1, 1)]),    # positions beyond 32 bits
])
def test_positions_refusals(B, status, cu, grids):
    plan = B.PositionGrids(cu, grids)
    refused(B, status, B.mllm_op_grid_positions, plan, P)
    with pytest.raises(B.MllmError) as e:
        B.mllm_grid_positions_count(plan)
    assert e.value.status == status


def test_positions_refuse_buffers(B):
    plan = B.PositionGrids([0, 8], [GRID])
    refused(B, NULL, B.mllm_op_grid_positions, plan, None)
    refused(B, SHAPE, B.mllm_op_grid_positions, plan, P, pos_stride=7)
    assert B.mllm_grid_positions_count(plan) == 6            # two of text, two steps of the grid, two of text
    assert B.mllm_grid_positions_count(B.PositionGrids([0, 0])) == 0


def test_section_axes(B):
    assert B.section_axes([2, 3, 1]).axes.tolist() == [0, 0, 1, 1, 1, 2]
    assert B.section_axes([2, 3, 1], dealt=True).axes.tolist() == [0, 1, 2, 0, 1, 1]
    dealt = B.section_axes([24, 20, 20], dealt=True).axes
    assert np.bincount(dealt).tolist() == [24, 20, 20] and dealt[:60].tolist() == [0, 1, 2] * 20 and set(dealt[60:]) == {0}


@pytest.mark.parametrize("status,change", [
    (NULL, dict(table=None)), (SHAPE, dict(n_pos=-1)), (SHAPE, dict(frequencies=[])), (SHAPE, dict(frequencies=[1.0] * 129)),
    (SHAPE, dict(frequencies=[1.0, float("inf")])), (SHAPE, dict(frequencies=[float("nan")])), (SHAPE, dict(n_pos=1 << 31)),
    (SHAPE, dict(n_pos=1 << 26, frequencies=[1.0] * 64)),
])
def test_table_refusals(B, status, change):
    refused(B, status, B.mllm_op_rope_freq_table, **{**dict(table=P, n_pos=4, frequencies=[1.0, 0.5]), **change})


@pytest.mark.parametrize("status,change", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(pos=None)), (NULL, dict(table=None)),
    (SHAPE, dict(t=-1)), (SHAPE, dict(t=1 << 31)), (SHAPE, dict(n_heads=-1)), (SHAPE, dict(n_heads=65536)), (SHAPE, dict(n_pos=-1)),
    (UNSUPPORTED, dict(head_dim=0)), (UNSUPPORTED, dict(head_dim=60)), (UNSUPPORTED, dict(head_dim=264)),
    (SHAPE, dict(axes=[])), (SHAPE, dict(axes=[0] * 12)), (SHAPE, dict(axes=[0] * 40)), (UNSUPPORTED, dict(axes=[0] * 7 + [4])),
    (SHAPE, dict(pos_stride=3, axes=[0, 1] * 8)),
    (SHAPE, dict(x_stride=248)), (SHAPE, dict(x_stride=260)), (SHAPE, dict(y_stride=248)),
    (UNSUPPORTED, dict(x=P + 8)), (UNSUPPORTED, dict(y=2 * P + 8)), (UNSUPPORTED, dict(table=P + 4)),
    (UNSUPPORTED, dict(y=P + 16)), (UNSUPPORTED, dict(y=P + 3 * 512)), (UNSUPPORTED, dict(y=P, y_stride=264)),
])
def test_rope_axes_refusals(B, status, change):
    kw = {**dict(x=P, y=2 * P, pos=P, axes=[0] * 32, table=P, n_pos=8, t=4, n_heads=4, head_dim=64, x_stride=256, y_stride=256), **change}
    refused(B, status, B.mllm_op_rope_axes, **{**kw, "axes": B.pair_axes(kw["axes"])})


BLOCK = dict(post_kind=0, post_g=P, post_b=P, post_eps=1e-6, scale=P, gate=P, pre_kind=0, pre_g=P, pre_b=P, pre_eps=1e-6)
BOTH = [
    (NULL, dict(post_g=None)), (NULL, dict(post_b=None)), (NULL, dict(pre_g=None)), (NULL, dict(pre_b=None)), (NULL, dict(post_kind=1, post_g=None)),
    (SHAPE, dict(post_kind=3)), (SHAPE, dict(pre_kind=-1)), (SHAPE, dict(gate_act=3)), (SHAPE, dict(gate_act=-1)),
    (SHAPE, dict(post_eps=-1.0)), (SHAPE, dict(pre_eps=float("nan"))),
    (UNSUPPORTED, dict(post_g=P + 2)), (UNSUPPORTED, dict(pre_b=P + 8)), (UNSUPPORTED, dict(scale=P + 4)),
    (SHAPE, dict(t=-1)), (SHAPE, dict(t=1 << 31)), (SHAPE, dict(d=0)), (SHAPE, dict(d=60)), (SHAPE, dict(d=8200)),
]


def split(B, change, call):
    kw = {**dict(t=4, d=64), **change}
    return B.ResidualNorm(**{**BLOCK, **{k: v for k, v in kw.items() if k in BLOCK or k in ("gate_act", "gate_per_row")}}), {
        **call, **{k: v for k, v in kw.items() if k not in BLOCK and k not in ("gate_act", "gate_per_row")}}


@pytest.mark.parametrize("status,change", BOTH + [
    (NULL, dict(x=None)), (NULL, dict(o=None)), (NULL, dict(y=None)), (NULL, dict(n=None)), (NULL, dict(stats=None)),
    (UNSUPPORTED, dict(x=P + 8)), (UNSUPPORTED, dict(o=2 * P + 2)), (UNSUPPORTED, dict(y=3 * P + 4)), (UNSUPPORTED, dict(n=4 * P + 4)),
    (UNSUPPORTED, dict(y=P + 16)), (UNSUPPORTED, dict(y=2 * P)), (UNSUPPORTED, dict(n=P)), (UNSUPPORTED, dict(n=2 * P)), (UNSUPPORTED, dict(n=3 * P + 496)),
    (UNSUPPORTED, dict(stats=3 * P)), (UNSUPPORTED, dict(stats=P)),
])
def test_residual_fwd_refusals(B, status, change):
    block, kw = split(B, change, dict(x=P, o=2 * P, y=3 * P, n=4 * P, stats=5 * P))
    refused(B, status, B.mllm_op_residual_norm_fwd, block, **kw)


GRADS = dict(post_g=10 * P, post_b=11 * P, scale=12 * P, pre_g=13 * P, pre_b=14 * P, gate=15 * P)


@pytest.mark.parametrize("status,change", BOTH + [
    (NULL, dict(dn=None)), (NULL, dict(y=None)), (NULL, dict(o=None)), (NULL, dict(stats=None)), (NULL, dict(dx=None)), (NULL, dict(d_o=None)),
    (NULL, dict(partial=None)), (NULL, dict(pre_kind=2, dy=None)),
    (UNSUPPORTED, dict(dn=P + 8)), (UNSUPPORTED, dict(dy=2 * P + 8)), (UNSUPPORTED, dict(dx=6 * P + 8)), (UNSUPPORTED, dict(partial=8 * P + 4)),
    (UNSUPPORTED, dict(dx=7 * P)), (UNSUPPORTED, dict(dx=P + 16)), (UNSUPPORTED, dict(d_o=2 * P + 496)), (UNSUPPORTED, dict(dx=3 * P)),
    (UNSUPPORTED, dict(d_o=4 * P)), (UNSUPPORTED, dict(dx=P, d_o=P)),
    (UNSUPPORTED, dict(grads=dict(GRADS, pre_g=10 * P))), (UNSUPPORTED, dict(grads=dict(GRADS, gate=14 * P + 252))),
    (UNSUPPORTED, dict(grads=dict(GRADS, scale=11 * P + 16))), (UNSUPPORTED, dict(grads=dict(GRADS, pre_b=14 * P + 8))),
    (UNSUPPORTED, dict(grads=dict(GRADS, post_g=10 * P + 4))),
])
def test_residual_bwd_refusals(B, status, change):
    change = dict(change)
    grads = B.ResidualNormGrads(**change.pop("grads", GRADS))
    block, kw = split(B, change, dict(dn=P, dy=2 * P, y=3 * P, o=4 * P, stats=5 * P, dx=6 * P, d_o=7 * P, partial=8 * P))
    refused(B, status, B.mllm_op_residual_norm_bwd, block, grads=grads, **kw)


def test_residual_partial_bytes(B):
    size = B.mllm_op_residual_norm_bwd_partial_bytes
    assert size(-1, 64) == 0 and size(4, 0) == 0 and size(4, 60) == 0 and size(4, 8200) == 0
    for d in (8, 64, 512, 520, 1024, 4096, 8192):
        sizes = [size(t, d) for t in (0, 1, 7, 100, 1000, 10000, 1000000)]
        assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] <= 1024 * (4 * d + 1) * 4


KEEP = dict(q=2 * P, exponents=3 * P, t=4, format=0)


@pytest.mark.parametrize("status,change", [
    (NULL, dict(x=None)), (NULL, dict(q=None)), (NULL, dict(exponents=None)), (SHAPE, dict(t=-1)), (SHAPE, dict(width=0)), (SHAPE, dict(width=60)),
    (SHAPE, dict(width=(1 << 30) + 8)), (SHAPE, dict(format=2)), (SHAPE, dict(format=-1)), (SHAPE, dict(x_stride=56)), (SHAPE, dict(x_stride=68)),
    (UNSUPPORTED, dict(x=P + 8)), (UNSUPPORTED, dict(q=2 * P + 8)),
    (UNSUPPORTED, dict(q=P + 496)), (UNSUPPORTED, dict(exponents=P + 511)), (UNSUPPORTED, dict(exponents=2 * P + 255)),
])
def test_keep8_refusals(B, status, change):
    refused(B, status, B.mllm_op_keep8, **{**KEEP, **dict(x=P, width=64), **change})
    change = {dict(x="y", x_stride="y_stride").get(k, k): v for k, v in change.items()}
    refused(B, status, B.mllm_op_keep8_load, **{**KEEP, **dict(y=P, width=64), **change})


@pytest.mark.parametrize("status,change", [
    (NULL, dict(pre=None)), (NULL, dict(a=None)), (NULL, dict(q=None)), (NULL, dict(exponents=None)), (SHAPE, dict(act=3)), (SHAPE, dict(act=-1)),
    (SHAPE, dict(f=60)), (SHAPE, dict(format=5)), (UNSUPPORTED, dict(pre=P + 8)), (UNSUPPORTED, dict(a=4 * P + 8)), (UNSUPPORTED, dict(q=2 * P + 8)),
    (UNSUPPORTED, dict(a=P)), (UNSUPPORTED, dict(q=P + 1008)), (UNSUPPORTED, dict(exponents=4 * P)), (UNSUPPORTED, dict(exponents=2 * P + 511)),
])
def test_act_fwd_keep8_refusals(B, status, change):
    refused(B, status, B.mllm_op_act_fwd_keep8, **{**KEEP, **dict(act=2, pre=P, a=4 * P, f=64), **change})


@pytest.mark.parametrize("status,change", [
    (NULL, dict(da=None)), (NULL, dict(dpre=None)), (NULL, dict(da=None, dpre=None, a=None)), (NULL, dict(q=None)), (SHAPE, dict(act=3)), (SHAPE, dict(f=4)),
    (UNSUPPORTED, dict(da=P + 8)), (UNSUPPORTED, dict(dpre=5 * P + 4)), (UNSUPPORTED, dict(a=4 * P + 2)),
    (UNSUPPORTED, dict(dpre=P)), (UNSUPPORTED, dict(a=P)), (UNSUPPORTED, dict(a=5 * P + 16)), (UNSUPPORTED, dict(act=0, dpre=P + 16)),
    (UNSUPPORTED, dict(q=P)), (UNSUPPORTED, dict(a=2 * P + 496)), (UNSUPPORTED, dict(exponents=5 * P + 1023)),
])
def test_act_bwd_keep8_refusals(B, status, change):
    refused(B, status, B.mllm_op_act_bwd_keep8, **{**KEEP, **dict(act=2, da=P, dpre=5 * P, a=4 * P, f=64), **change})


@pytest.mark.parametrize("status,change", [
    (NULL, dict(dy=None)), (NULL, dict(w=None)), (NULL, dict(dx=None)), (NULL, dict(dw=None)), (NULL, dict(q=None)), (NULL, dict(workspace=None)),
    (SHAPE, dict(k=60)), (SHAPE, dict(n=60)), (SHAPE, dict(n=0)), (SHAPE, dict(t=-1)), (SHAPE, dict(format=2)),
    (SHAPE, dict(t=1 << 20, k=2048)), (SHAPE, dict(t=1 << 20, n=2048)),
    (WORKSPACE, dict(workspace=P + 16)), (WORKSPACE, dict(workspace_bytes=511)), (UNSUPPORTED, dict(q=2 * P + 8)),
    (UNSUPPORTED, dict(dx=P)), (UNSUPPORTED, dict(dw=4 * P + 16)), (UNSUPPORTED, dict(dx=6 * P)), (UNSUPPORTED, dict(workspace=2 * P)), (UNSUPPORTED, dict(dx=7 * P)),
    (UNSUPPORTED, dict(dw=2 * P - 16)), (UNSUPPORTED, dict(dy=P + 8)), (UNSUPPORTED, dict(w=4 * P + 2)), (UNSUPPORTED, dict(dx=5 * P + 4)), (UNSUPPORTED, dict(dw=6 * P + 8)),
])
def test_linear_bwd_keep8_refusals(B, status, change):
    refused(B, status, B.mllm_op_linear_bwd_keep8,
            **{**KEEP, **dict(dy=P, w=4 * P, dx=5 * P, dw=6 * P, k=64, n=64, workspace=7 * P, workspace_bytes=1 << 16), **change})


def test_linear_bwd_keep8_workspace(B):
    size = B.mllm_op_linear_bwd_keep8_workspace_bytes
    assert size(-1, 64, 64) == 0 and size(4, 0, 64) == 0 and size(4, 64, -8) == 0
    up = lambda v: (v + 255) // 256 * 256
    for t, k, n in ((1, 64, 64), (777, 3584, 4608), (8192, 4096, 6144)):
        assert size(t, k, n) - up(2 * t * k) == B.mllm_linear_bwd_form(t, k, n)[1]
    for t, k, n in ((1, 8, 8), (777, 1000, 3000), (20000, 512, 72)):            # copies of dy and w with whole tiles of columns
        wide = (n + 63) // 64 * 64
        assert size(t, k, n) >= up(2 * t * k) + up(2 * t * wide) + up(2 * k * wide)
    for k, n in ((72, 7000), (256, 136), (600, 1000)):                          # a buffer for more rows has what fewer rows want
        sizes = [size(t, k, n) - up(2 * t * k) - B.mllm_linear_bwd_form(t, k, (n + 63) // 64 * 64)[1] for t in (1, 1000, 4096, 4097, 30000)]
        assert sizes == sorted(sizes)


def test_layers_that_keep_in_8_bits(B):
    import dataclasses

    import workloads as W
    vit, proj, dec = W.tiny_stage_layers()
    for layers in ([dataclasses.replace(dec, keep8=3)], [dataclasses.replace(dec, keep8=-1)], [dataclasses.replace(vit, keep8=4)],
                   [vit, dataclasses.replace(proj, keep8=1), dec]):
        with pytest.raises(B.MllmError) as e:
            B.mllm_stage_create(layers)
        assert e.value.status == 2
    for keep8 in (0, 1, 2):
        B.mllm_stage_destroy(B.mllm_stage_create([dataclasses.replace(vit, keep8=keep8), proj, dataclasses.replace(dec, keep8=keep8)]))


def test_arguments_of_the_extension_module(B):
    """What the header's types do not take is refused before the call; None, addresses, tensors and NumPy's numbers are taken."""
    calls = B._fast()
    assert set(B.FAST) <= set(B.EXPORTS) and all(callable(getattr(calls, name)) for name in B.FAST)

    class Tensor:
        def data_ptr(self):
            return P

    ok = (Tensor(), 2 * P, 3 * P, np.int64(0), np.int32(64), 64, 0, None)         # no rows: nothing is launched
    assert calls.mllm_op_keep8(*ok) == 0
    assert calls.mllm_op_keep8(None, None, None, *ok[3:]) == 0
    assert calls.mllm_op_keep8(None, 2 * P, 3 * P, 4, *ok[4:]) == NULL and "NULL" in B.mllm_last_error()
    with pytest.raises(TypeError):
        calls.mllm_op_keep8(*ok[:-1])
    with pytest.raises(TypeError):
        calls.mllm_op_keep8(*ok[:4], 64.0, *ok[5:])
    with pytest.raises(AttributeError):
        calls.mllm_op_keep8("x", *ok[1:])
    with pytest.raises(OverflowError):
        calls.mllm_op_keep8(*ok[:6], 1 << 31, None)
    with pytest.raises(OverflowError):
        calls.mllm_op_keep8(*ok[:3], 1 << 63, *ok[4:])
    with pytest.raises(KeyError):
        calls.bind("mllm_op_gemm", P)
    with pytest.raises(ValueError):
        calls.bind("mllm_op_keep8", 0)
    assert calls.mllm_op_keep8(*ok) == 0


def test_calls_from_several_threads(B):
    """The status and its message belong to the thread that called."""
    import threading
    seen = {}

    def work(i):
        for _ in range(200):
            try:
                if i % 2:
                    B.mllm_op_keep8(P, 2 * P, 3 * P, 4, 60, 0, stream=1)
                else:
                    B.mllm_op_keep8(None, 2 * P, 3 * P, 4, 64, 0, stream=1)
            except B.MllmError as e:
                seen.setdefault(i, set()).add((e.status, str(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(len(v) == 1 and next(iter(v))[0] == (SHAPE if i % 2 else NULL) for i, v in seen.items()) and len(seen) == 6
