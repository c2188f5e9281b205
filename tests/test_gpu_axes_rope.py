"""Positions on several axes, tables of rotary factors and the rotation by them, against their definitions in float64."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


def walked(cu, grids):
    """Positions row by row, as the definition says them, and one more than the largest."""
    pos, starts = np.full((3, cu[-1]), -7, dtype=np.int64), {g[0]: g[1:] for g in grids}
    for first, end in zip(cu, cu[1:]):
        row, p = first, 0
        while row < end:
            if row in starts:
                f, h, w, step = starts[row]
                for i in range(f):
                    for j in range(h):
                        for k in range(w):
                            pos[:, row] = p + i * step, p + j, p + k
                            row += 1
                p += max((f - 1) * step + 1, h, w)
            else:
                pos[:, row] = p
                row, p = row + 1, p + 1
    return pos


LAYOUTS = {
    "nothing": ([0], []),
    "empty samples": ([0, 0, 0], []),
    "one token": ([0, 1], []),
    "one token as a grid": ([0, 1], [(0, 1, 1, 1, 1)]),
    "text": ([0, 5, 5, 300], []),
    "image alone": ([0, 24], [(0, 1, 4, 6, 1)]),
    "images side by side": ([0, 60, 110], [(0, 1, 5, 5, 1), (25, 1, 7, 5, 1), (70, 1, 4, 10, 1)]),
    "clip, frames far apart": ([0, 100], [(3, 8, 2, 3, 9)]),
    "clip, frames at one time": ([0, 100], [(3, 8, 2, 3, 0)]),
    "a sample each": ([0, 9, 9, 18, 30], [(0, 1, 3, 3, 1), (9, 1, 3, 3, 1), (20, 2, 5, 1, 2)]),
    "more runs than a launch takes": (list(range(0, 2001, 8)), [(8 * i + 2, 1, 2, 2, 1) for i in range(250)]),
}
LAYOUTS["as many runs as a small launch takes"] = ([0, 24 * 3], [(3 * i, 1, 1, 3, 1) for i in range(24)])
LAYOUTS["one more than that"] = ([0, 25 * 3], [(3 * i, 1, 1, 3, 1) for i in range(25)])
LAYOUTS["as many runs as a launch takes"] = ([0, 192 * 3], [(3 * i, 1, 1, 3, 1) for i in range(192)])
LAYOUTS["one more, and an empty sample behind"] = ([0, 193 * 3, 193 * 3], [(3 * i, 1, 1, 3, 1) for i in range(193)])


@pytest.mark.parametrize("name", sorted(LAYOUTS))
def test_positions(B, name):
    cu, grids = LAYOUTS[name]
    rows, stride = cu[-1], cu[-1] + 5
    want = walked(cu, grids)
    plan = B.PositionGrids(cu, grids)
    assert B.mllm_grid_positions_count(plan) == (want.max() + 1 if rows else 0)
    pos = torch.full((3, stride), -99, dtype=torch.int32, device="cuda")
    B.mllm_op_grid_positions(plan, pos, pos_stride=stride)
    got = pos.cpu().numpy()
    np.testing.assert_array_equal(got[:, :rows], want)
    assert (got[:, rows:] == -99).all()          # rows behind the last sample stay as they were
    if rows:
        dense = torch.empty(3, rows, dtype=torch.int32, device="cuda")
        B.mllm_op_grid_positions(plan, dense)
        np.testing.assert_array_equal(dense.cpu().numpy(), want)


def test_positions_far_on(B):
    """The last position that fits, and the last that does not (refused on the host)."""
    last = (1 << 31) - 2
    cu, grids = [0, 3], [(1, 2, 1, 1, last)]       # p = 1: the second frame is at 1 + last, and it takes last + 1 steps
    with pytest.raises(B.MllmError):
        B.mllm_grid_positions_count(B.PositionGrids(cu, grids))
    grids = [(1, 2, 1, 1, last - 1)]
    assert B.mllm_grid_positions_count(B.PositionGrids(cu, grids)) == last + 1
    pos = torch.empty(3, 3, dtype=torch.int32, device="cuda")
    B.mllm_op_grid_positions(B.PositionGrids(cu, grids), pos)
    assert pos.cpu().tolist() == [[0, 1, last], [0, 1, 1], [0, 1, 1]]


@pytest.mark.parametrize("n_pairs,n_pos", [(1, 5), (8, 1), (40, 1000), (64, 70000), (128, 300)])
def test_table(B, n_pairs, n_pos):
    freq = [3.0 * 500000.0 ** (-i / n_pairs) * (-1) ** (i % 3) for i in range(n_pairs)]
    table = torch.empty(n_pos, 2 * n_pairs, device="cuda")
    B.mllm_op_rope_freq_table(table, n_pos, freq)
    angle = np.arange(n_pos)[:, None] * np.asarray(freq)
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    # the factor's own rounding to fp32, 2^-25 near 1, and the angle's in fp64: 2^-53 of 2.1e5
    assert np.abs(table.cpu().numpy() - want).max() <= 2 ** -25 + 2e5 * 2 ** -52


def test_table_of_one_axis(B):
    """With the frequencies of mllm_op_rope_table the tables agree to a rounding (the exponential may differ in its last bit)."""
    table, other = torch.empty(3000, 128, device="cuda"), torch.empty(3000, 128, device="cuda")
    B.mllm_op_rope_table(table, 3000, 128, 500000.0)
    B.mllm_op_rope_freq_table(other, 3000, [500000.0 ** (-2 * i / 128) for i in range(64)])
    assert (table - other).abs().max().item() <= 2 ** -24 + 3000 * 2 ** -50


def rotated(x, pos, axes, table, heads, hd, inverse):
    """(result, size of its terms) in float64; rows of pairs outside the table NaN."""
    t, pairs = x.shape[0], len(axes)
    v = x.double()[:, :heads * hd].reshape(t, heads, hd)
    out, size = v.clone(), v.abs().clone()
    p = pos.long()[torch.tensor(axes, device=x.device)].T                      # [t, pairs]
    inside = (p >= 0) & (p < table.shape[0])
    p = p.clamp(0, max(0, table.shape[0] - 1))
    i = torch.arange(pairs, device=x.device)
    cos, sin = table.double()[p, i], table.double()[p, pairs + i]
    nan = torch.full_like(cos, NAN)
    cos, sin = torch.where(inside, cos, nan)[:, None], torch.where(inside, sin, nan)[:, None]
    if inverse:
        sin = -sin
    a, b = v[..., :pairs], v[..., pairs:2 * pairs]
    out[..., :pairs], out[..., pairs:2 * pairs] = a * cos - b * sin, b * cos + a * sin
    size[..., :pairs] = size[..., pairs:2 * pairs] = a.abs() + b.abs()
    return out.reshape(t, -1), size.reshape(t, -1)


def inputs(t, width, n_axes, n_pos, pairs, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, width, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, n_pos, (n_axes, t), generator=g, device="cuda", dtype=torch.int32)
    angle = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
    return x, pos, torch.cat([angle.cos(), angle.sin()], 1).float()


def close(got, want, size):
    # one rounding to bf16, 2^-8 of the value; two products and a sum in fp32, three roundings of 2^-24 of the terms
    assert torch.equal(torch.isnan(got.double()), torch.isnan(want))
    fine = ~torch.isnan(want)
    excess = ((got.double() - want).abs() - (2 ** -8 * want.abs() + 4 * 2 ** -24 * size))[fine]
    assert excess.numel() == 0 or excess.max().item() <= 0, excess.max().item()


SHAPES = [  # tokens, heads, head_dim, axes of the pairs
    (1, 1, 16, [0] * 8),
    (1, 40, 128, [i % 3 for i in range(64)]),
    (7, 3, 80, [0] * 13 + [1] * 20 + [2] * 7),
    (300, 6, 64, [0] * 8 + [1] * 12 + [2] * 12),
    (300, 6, 64, [1] * 16 + [2] * 16),                   # an axis that no pair follows
    (513, 5, 96, [(i * 7) % 4 for i in range(32)]),      # four axes, the last elements of a head not rotated
    (1000, 9, 256, [2] * 128),
    (777, 35, 128, [i % 2 for i in range(64)]),
    (64, 2, 248, [0] * 8),                               # most of a head not rotated
    (5000, 32, 64, [0] * 8 + [1] * 12 + [2] * 12),
]


@pytest.mark.parametrize("inverse", [0, 1])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rotation(B, shape, inverse):
    t, heads, hd, axes = SHAPES[shape]
    width, n_axes, n_pos = heads * hd, max(axes) + 1, 900
    x, pos, table = inputs(t, width + 24, n_axes, n_pos, len(axes), shape)
    want, size = rotated(x, pos, axes, table, heads, hd, inverse)
    y = torch.full((t, width + 40), 3.5, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_rope_axes(x, y, pos, B.pair_axes(axes), table, n_pos, t, heads, hd, width + 24, width + 40, inverse=inverse)
    close(y[:, :width], want, size)
    assert bool((y[:, width:] == 3.5).all())             # other columns are not touched
    rest = y[:, :width].reshape(t, heads, hd)[..., 2 * len(axes):]
    assert torch.equal(rest, x[:, :width].reshape(t, heads, hd)[..., 2 * len(axes):])
    place = x.clone()                                    # in place: the same bits
    B.mllm_op_rope_axes(place, place, pos, B.pair_axes(axes), table, n_pos, t, heads, hd, width + 24, width + 24, inverse=inverse)
    assert torch.equal(place[:, :width], y[:, :width]) and torch.equal(place[:, width:], x[:, width:])


def test_inverse_is_the_gradient(B):
    """<dy, R x> = <R^-1 dy, x>, as the rotation is orthogonal."""
    t, heads, hd, axes = 50, 3, 64, [i % 3 for i in range(24)]
    x, pos, table = inputs(t, heads * hd, 3, 40, 24, 5)
    dy = torch.randn(t, heads * hd, device="cuda").bfloat16()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    call = lambda a, b, inverse: B.mllm_op_rope_axes(a, b, pos, B.pair_axes(axes), table, 40, t, heads, hd, heads * hd, heads * hd, inverse=inverse)
    call(x, y, 0)
    call(dy, dx, 1)
    left, right = (dy.double() * y.double()).sum(1), (dx.double() * x.double()).sum(1)
    size = (dy.double().abs() * y.double().abs()).sum(1) + (dx.double().abs() * x.double().abs()).sum(1)
    assert bool(((left - right).abs() <= 1.01 * 2 ** -8 * size).all())        # every element of y and dx is off by 2^-8 of itself at most


def test_positions_outside_the_table(B):
    """Each of the axes by itself: its pairs are NaN, those of the other axes are turned."""
    axes = [0] * 5 + [1] * 6 + [2] * 5
    t, heads, hd = 6, 2, 40
    x, pos, table = inputs(t, heads * hd, 3, 10, 16, 9)
    pos[0, 0], pos[1, 1], pos[2, 2], pos[0, 3], pos[1, 4] = -1, 10, (1 << 31) - 1, -(1 << 31), 9
    want, size = rotated(x, pos, axes, table, heads, hd, 0)
    assert torch.isnan(want).sum().item() == heads * 2 * (5 + 6 + 5 + 5)
    y = torch.empty_like(x)
    B.mllm_op_rope_axes(x, y, pos, B.pair_axes(axes), table, 10, t, heads, hd, heads * hd, heads * hd)
    close(y, want, size)
    B.mllm_op_rope_axes(x, y, pos, B.pair_axes(axes), table, 0, t, heads, hd, heads * hd, heads * hd)       # an empty table
    assert torch.isnan(y.view(t, heads, hd)[..., :32]).all() and torch.equal(y.view(t, heads, hd)[..., 32:], x.view(t, heads, hd)[..., 32:])


def test_strides_of_positions_and_nothing_to_do(B):
    t, heads, hd, axes = 33, 2, 32, [i % 2 for i in range(16)]
    x, pos, table = inputs(t, heads * hd, 2, 50, 16, 2)
    wide = torch.full((2, t + 13), -1, dtype=torch.int32, device="cuda")
    wide[:, :t] = pos
    y, other = torch.empty_like(x), torch.empty_like(x)
    B.mllm_op_rope_axes(x, y, pos, B.pair_axes(axes), table, 50, t, heads, hd, heads * hd, heads * hd)
    B.mllm_op_rope_axes(x, other, wide, B.pair_axes(axes), table, 50, t, heads, hd, heads * hd, heads * hd, pos_stride=t + 13)
    assert torch.equal(y, other)
    B.mllm_op_rope_axes(None, None, None, B.pair_axes(axes), table, 50, 0, heads, hd, heads * hd, heads * hd)
    B.mllm_op_rope_axes(x, other, pos, B.pair_axes(axes), table, 50, t, 0, hd, heads * hd, heads * hd)
    torch.cuda.synchronize()
    assert torch.equal(y, other)


def test_special_values(B):
    """Infinities and NaN stay in their pairs; other heads and rows have the bits that they have without."""
    t, heads, hd, axes = 40, 4, 64, [i % 3 for i in range(32)]
    x, pos, table = inputs(t, heads * hd, 3, 50, 32, 3)
    clean, y = torch.empty_like(x), torch.empty_like(x)
    call = lambda a, b: B.mllm_op_rope_axes(a, b, pos, B.pair_axes(axes), table, 50, t, heads, hd, heads * hd, heads * hd)
    call(x, clean)
    bad = x.clone()
    bad[3, 64 + 5], bad[7, 10], bad[8, 200] = float("inf"), NAN, -float("inf")
    call(bad, y)
    same = torch.ones_like(y, dtype=torch.bool)
    for row, first in ((3, 64 + 5), (7, 10), (8, 200)):     # 200: element 8 of the head that begins at 192
        same[row, first] = same[row, first + 32] = False
        assert not torch.isfinite(y[row, first]) and not torch.isfinite(y[row, first + 32])
    assert torch.equal(y[same], clean[same])


def test_more_workgroups_than_a_dimension_of_a_grid_takes(B):
    """A token a workgroup and 2^20 + 5 of them, 9 GB: rows that repeat have the same results, bit for bit."""
    heads, hd, axes, period = 33, 128, [i % 3 for i in range(64)], 1024
    t, width = (1 << 20) + 5, heads * hd
    part, pos, table = inputs(period, width, 3, 613, 64, 1)
    x = part.repeat(t // period + 1, 1)[:t].contiguous()
    every = pos.repeat(1, t // period + 1)[:, :t].contiguous()
    B.mllm_op_rope_axes(x, x, every, B.pair_axes(axes), table, 613, t, heads, hd, width, width)
    B.mllm_op_rope_axes(part, part, pos, B.pair_axes(axes), table, 613, period, heads, hd, width, width)
    for r in (0, 100 * period, 508 * period, 1023 * period):        # 508 periods: beyond 2^32 bytes
        assert torch.equal(x[r:r + period], part)
    assert torch.equal(x[1 << 20:], part[:5])
