"""Matrices kept in 8 bits and what is computed from them, against the format's definition (bit for bit) and the formulas in float64."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HALF, FP32 = 2.0 ** -8, 2.0 ** -24
FORMATS = ("int8", "e4m3")


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


def fmt(B, name):
    return dict(int8=B.KEEP_INT8, e4m3=B.KEEP_E4M3)[name]


E4M3 = np.array([(1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6 for e in range(16) for m in range(8)][:127])    # its values up to 448


def kept(x, name):
    """(values, exponent bytes, values of the format) of float64 x [t, width], by the definition."""
    t, width = x.shape
    blocks = -(-width // 32)
    v = np.zeros((t, blocks * 32))
    v[:, :width] = x
    v = v.reshape(t, blocks, 32)
    top = np.abs(v).max(2)
    most = dict(int8=127.0, e4m3=448.0)[name]
    e, finite = np.full(top.shape, -112), np.where(np.isfinite(top), top, 0.0)
    while (finite > most * 2.0 ** e).any():
        e = e + (finite > most * 2.0 ** e)
    bad = ~np.isfinite(v).all(2)
    with np.errstate(invalid="ignore"):
        q = v * 2.0 ** -e[..., None].astype(float)
    q = np.where(bad[..., None], 0.0, q)
    if name == "int8":
        q = np.rint(q)
    else:                                # the nearest of the list, an even place between two that are as near
        a = np.abs(q)
        hi = np.searchsorted(E4M3, a).clip(max=126)
        lo = (hi - 1).clip(min=0)
        down, up = a - E4M3[lo], E4M3[hi] - a
        place = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
        q = np.copysign(E4M3[place], q)
    value = q * 2.0 ** e[..., None].astype(float)
    value[bad] = np.nan
    # 2^128, to which the largest bf16 numbers are rounded beside one of 255/128 2^127 (int8 64 * 2^122, e4m3 256 * 2^120), is no bf16 number: infinity
    value = np.where(np.abs(value) >= 2.0 ** 128, np.copysign(np.inf, value), value)
    return value.reshape(t, -1)[:, :width], np.where(bad, 255, e + 127), q.reshape(t, -1)[:, :width]


def wide(t, width, seed, low=-40, high=40):
    """bf16 values whose sizes go over many binades, blocks of zeros and single values among them."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((t, width)) * 2.0 ** g.integers(low, high, (t, 1)) * 2.0 ** g.integers(-9, 1, (t, width))
    x[g.random((t, width)) < 0.05] = 0
    x[:, :32][g.random(t) < 0.2] = 0
    return torch.from_numpy(x).to(torch.bfloat16).cuda()


def borders():
    """Blocks whose largest value is at the formats' limits, and values between two of the formats'."""
    rows = []
    for scale in (1.0, 2.0 ** -60, 2.0 ** 90):
        for top in (127.0, 127.5, 126.5, 128.0, 255.0, 254.0, 448.0, 450.0, 446.0, 464.0, 512.0, 511.0, 1.0, 1.9921875):
            for sign in (1, -1):
                row = np.concatenate([[sign * top], np.arange(0.5, 16, 1) * (top / 127), np.arange(1, 16) * top / 448 / 16])[:32] * scale
                rows.append(row)
    return torch.tensor(np.array(rows), device="cuda").bfloat16()


def store(B, x, name, x_stride=None):
    t, width = x.shape
    q = torch.full((t, width), 0xA5, dtype=torch.uint8, device="cuda")
    e = torch.full((t, -(-width // 32)), 0xA5, dtype=torch.uint8, device="cuda")
    B.mllm_op_keep8(x, q, e, t, width, fmt(B, name), x_stride=x_stride)
    return q, e


def check_store(B, x, name):
    t, width = x.shape
    q, e = store(B, x, name)
    value, byte, number = kept(x.double().cpu().numpy(), name)
    np.testing.assert_array_equal(e.cpu().numpy(), byte)
    got = q.view(torch.int8).double().cpu().numpy() if name == "int8" else q.view(torch.float8_e4m3fn).double().cpu().numpy()
    np.testing.assert_array_equal(got, number)
    y = torch.empty_like(x)
    B.mllm_op_keep8_load(q, e, y, t, width, fmt(B, name))
    np.testing.assert_array_equal(y.double().cpu().numpy(), value)
    return y


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("t,width", [(1, 8), (1, 32), (3, 40), (65, 24), (70, 256), (129, 1000), (33, 4096), (1, 28672), (2000, 72)])
def test_every_value(B, name, t, width):
    check_store(B, wide(t, width, t + width), name)


@pytest.mark.parametrize("name", FORMATS)
def test_borders(B, name):
    check_store(B, borders(), name)
    check_store(B, wide(500, 64, 1, low=-133, high=-90), name)        # down to subnormal numbers
    check_store(B, wide(500, 64, 2, low=100, high=118), name)
    x = torch.full((3, 64), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16, device="cuda")
    x[1] = -x[1]
    x[2, ::2] = 2.0 ** -133
    check_store(B, x, name)


@pytest.mark.parametrize("name", FORMATS)
def test_every_bf16_number(B, name):
    """All finite ones, one in a block of its own, and all of them in blocks with a larger neighbour."""
    every = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()
    every = every[torch.isfinite(every.float())]
    x = torch.zeros(len(every), 32, dtype=torch.bfloat16, device="cuda")
    x[torch.arange(len(every)), torch.arange(len(every)) % 32] = every
    y = check_store(B, x, name)
    v, w = x.double().abs().amax(1), (x.double() - y.double()).abs().amax(1)
    small = v < 3.28e38                      # larger ones may be rounded to 2^128, which is an infinity
    assert bool((w <= v * (1 / 127 if name == "int8" else 2 ** -4) + 2.0 ** -113)[small].all()) and (~small).sum().item() == 2 * 9
    check_store(B, every.view(-1, 8).repeat(1, 4)[:, :32].contiguous(), name)


@pytest.mark.parametrize("name", FORMATS)
def test_infinities_and_nan(B, name):
    """The block that holds one is NaN as a whole, its neighbours are what they are without."""
    x = wide(6, 104, 4, -3, 3)
    clean = check_store(B, x, name)
    x[0, 5], x[1, 40], x[2, 103], x[3, 31] = float("inf"), -float("inf"), float("nan"), float("nan")
    y = check_store(B, x, name)
    bad = torch.zeros(6, 104, dtype=torch.bool, device="cuda")
    bad[0, :32] = bad[1, 32:64] = bad[2, 96:] = bad[3, :32] = True
    assert bool(torch.isnan(y[bad]).all()) and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("name", FORMATS)
def test_strides(B, name):
    base = wide(50, 200, 7)
    x = base[:, 16:16 + 72]                          # columns of a wider matrix
    q, e = store(B, x, name, x_stride=200)
    q2, e2 = store(B, x.contiguous(), name)
    assert torch.equal(q, q2) and torch.equal(e, e2)
    y = torch.full((50, 88), 2.5, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_keep8_load(q, e, y, 50, 72, fmt(B, name), y_stride=88)
    np.testing.assert_array_equal(y[:, :72].double().cpu().numpy(), kept(x.double().cpu().numpy(), name)[0])
    assert bool((y[:, 72:] == 2.5).all())
    B.mllm_op_keep8(None, None, None, 0, 72, fmt(B, name))
    B.mllm_op_keep8_load(None, None, None, 0, 72, fmt(B, name))


def activation(act, v):
    """(value, slopes, sizes of the slopes' terms) in float64; SwiGLU of [gate | up]."""
    if act == 2:
        gate, up = v.chunk(2, 1)
        s = torch.special.expit(gate)
        c = torch.special.expit(-gate)
        return gate * s * up, [up * (s + gate * s * c), gate * s], [up.abs() * (s + gate.abs() * s * c), (gate * s).abs()]
    if act == 0:
        below = 0.5 * torch.special.erfc(-v / math.sqrt(2))
        phi = torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        return v * below, [below + v * phi], [below + v.abs() * phi]
    u = math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    s, c = torch.special.expit(2 * u), torch.special.expit(-2 * u)
    rise = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)
    return v * s, [s + v * s * c * rise], [s + v.abs() * s * c * rise]


# The arithmetic in fp32: exp2 of an argument of up to 2^7 that is off by 2 FP32 of itself, so 2^8 ln 2 FP32 = 1.1e-5 of the result; the fit of the
# normal distribution 1.2e-6; a dozen roundings.  Below 2^-120 the hardware's powers and reciprocals end in zero.
EXP, TINY = 1.5e-5, 2.0 ** -115


def values(t, width, seed):
    """Activations of every size that matters: normal ones, tails, zeros."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, width, generator=g, device="cuda") * torch.exp(0.8 * torch.randn(width, generator=g, device="cuda"))
    x[::5] *= 6
    x[::7, ::3] = 0
    return x.clamp(-60, 60).bfloat16()


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("t,f", [(1, 8), (2, 40), (77, 512), (300, 1000), (33, 14336), (5, 56)])
def test_activations(B, name, act, t, f):
    halves = 2 if act == 2 else 1
    pre, da = values(t, halves * f, t + f), torch.randn(t, f, device="cuda").bfloat16()
    q = torch.full((t, halves * f), 0xA5, dtype=torch.uint8, device="cuda")
    e = torch.full((t, halves * -(-f // 32)), 0xA5, dtype=torch.uint8, device="cuda")
    a = torch.full((t, f), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.mllm_op_act_fwd_keep8(act, pre, a, q, e, t, f, fmt(B, name))
    want, _, _ = activation(act, pre.double())
    assert bool(((a.double() - want).abs() <= (HALF + EXP) * want.abs() + TINY).all())
    # kept as mllm_op_keep8 keeps each half
    parts = [store(B, half.contiguous(), name) for half in pre.split(f, 1)]
    assert torch.equal(q, torch.cat([p[0] for p in parts], 1)) and torch.equal(e, torch.cat([p[1] for p in parts], 1))
    value = torch.from_numpy(np.concatenate([kept(half.double().cpu().numpy(), name)[0] for half in pre.split(f, 1)], 1)).cuda()
    want, slopes, sizes = activation(act, value)
    dpre, again = torch.full_like(pre, float("nan")), torch.full_like(a, float("nan"))
    B.mllm_op_act_bwd_keep8(act, da, q, e, dpre, t, f, fmt(B, name), a=again)
    assert bool(((again.double() - want).abs() <= (HALF + EXP) * want.abs() + TINY).all())
    grad, size = torch.cat([da.double() * s for s in slopes], 1), torch.cat([da.double().abs() * s for s in sizes], 1)
    assert bool(((dpre.double() - grad).abs() <= HALF * grad.abs() + 4 * EXP * size + TINY).all())
    alone, only = torch.empty_like(a), torch.empty_like(pre)          # either of the two results by itself, the GELU kinds in place
    B.mllm_op_act_bwd_keep8(act, None, q, e, None, t, f, fmt(B, name), a=alone)
    B.mllm_op_act_bwd_keep8(act, da, q, e, only, t, f, fmt(B, name))
    assert torch.equal(alone, again) and torch.equal(only, dpre)
    if act != 2:
        B.mllm_op_act_bwd_keep8(act, da, q, e, da, t, f, fmt(B, name))
        assert torch.equal(da, dpre)


@pytest.mark.parametrize("act", [0, 1, 2])
def test_activations_far_out_and_empty(B, act):
    """Every finite bf16 number as an activation's input is finite or as large as it; no rows; NaN stays in its block."""
    every = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()
    every = every[torch.isfinite(every.float())]
    f, halves = 32, 2 if act == 2 else 1
    x = torch.zeros(len(every), halves * f, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = every
    if act == 2:
        x[:, f] = 1
    t = len(every)
    q, e, a = torch.empty_like(x, dtype=torch.uint8), torch.empty(t, halves, dtype=torch.uint8, device="cuda"), torch.empty(t, f, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_act_fwd_keep8(act, x, a, q, e, t, f, B.KEEP_INT8)
    far = every.double().abs() < 2.0 ** 40
    want = activation(act, x.double())[0]
    assert bool(((a.double() - want).abs() <= (HALF + EXP) * want.abs() + TINY)[far].all())
    up = every.double() >= 2.0 ** 40
    assert torch.equal(a[up, 0], every[up])
    # and backward: the slopes at the kept values, whatever their size (2^128, which the largest are rounded to, aside)
    value = torch.empty_like(x)
    B.mllm_op_keep8_load(q, e, value, t, halves * f, B.KEEP_INT8)
    rows = torch.isfinite(value.float()).all(1)
    assert (~rows).sum().item() <= 2 * 9
    da, dpre = torch.ones(t, f, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    B.mllm_op_act_bwd_keep8(act, da, q, e, dpre, t, f, B.KEEP_INT8)
    rows &= value.double().abs().amax(1) < (2.0 ** 40 if act == 1 else 2.0 ** 126)      # (the formula in float64 ends at 2^1024: cubes of 2^340)
    _, slopes, sizes = activation(act, value[rows].double())
    grad, size = torch.cat(slopes, 1), torch.cat(sizes, 1)
    assert bool(((dpre[rows].double() - grad).abs() <= HALF * grad.abs() + 4 * EXP * size + TINY).all())
    far = value.double()[:, 0].abs() >= 2.0 ** 40
    far &= torch.isfinite(value.double()[:, 0])
    assert torch.equal(dpre[far, 0].double(), (value[far, 0].double() > 0).double())
    B.mllm_op_act_fwd_keep8(act, None, None, None, None, 0, f, B.KEEP_INT8)
    B.mllm_op_act_bwd_keep8(act, None, None, None, None, 0, f, B.KEEP_INT8)
    x = values(4, halves * 64, 1)
    x[1, 3] = float("nan")
    q, e = torch.empty_like(x, dtype=torch.uint8), torch.empty(4, 2 * halves, dtype=torch.uint8, device="cuda")
    a, da, dpre = torch.empty(4, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    B.mllm_op_act_fwd_keep8(act, x, a, q, e, 4, 64, B.KEEP_INT8)
    assert torch.isnan(a).sum().item() == 1
    B.mllm_op_act_bwd_keep8(act, da, q, e, dpre, 4, 64, B.KEEP_INT8)
    assert torch.isnan(dpre[1, :32]).all() and torch.isnan(dpre).sum().item() == 32 * halves


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("t,k,n", [(1, 8, 8), (7, 64, 40), (128, 256, 192), (333, 520, 264), (1000, 1024, 512), (2048, 512, 4096),
                                   (1, 1000, 3000), (100, 72, 1000), (2000, 64, 200), (513, 1000, 72), (4097, 256, 136), (4500, 520, 88), (3, 8, 4088)])
def test_linear_gradients(B, name, t, k, n):
    g = torch.Generator(device="cuda").manual_seed(t)
    x = values(t, k, t)
    w, dy = (0.05 * torch.randn(k, n, generator=g, device="cuda")).bfloat16(), torch.randn(t, n, generator=g, device="cuda").bfloat16()
    q, e = store(B, x, name)
    ws = torch.full((B.mllm_op_linear_bwd_keep8_workspace_bytes(t, k, n),), 0xFF, dtype=torch.uint8, device="cuda")
    value = torch.from_numpy(kept(x.double().cpu().numpy(), name)[0]).cuda()
    wide_dy, wide_w = dy.double(), w.double()
    dx_want, dx_size = wide_dy @ wide_w.T.contiguous(), wide_dy.abs() @ wide_w.abs().T.contiguous()
    dw_want, dw_size = value.T.contiguous() @ wide_dy, value.abs().T.contiguous() @ wide_dy.abs()
    dx, dw = torch.full_like(x, float("nan")), torch.full((k, n), float("nan"), device="cuda")
    B.mllm_op_linear_bwd_keep8(dy, q, e, w, dx, dw, t, k, n, fmt(B, name), ws)
    # sums of products in fp32, in any order: the contraction's length times FP32 of the terms
    assert bool(((dx.double() - dx_want).abs() <= HALF * dx_want.abs() + 2 * n * FP32 * dx_size).all())
    assert bool(((dw.double() - dw_want).abs() <= 2 * t * FP32 * dw_size).all())
    once = dw.clone()
    B.mllm_op_linear_bwd_keep8(dy, q, e, w, dx, dw, t, k, n, fmt(B, name), ws, accumulate=1)
    assert bool(((dw.double() - 2 * dw_want).abs() <= 4 * (t + 2) * FP32 * dw_size).all())
    # the same gradients, bit for bit, as from the loaded matrix, where the products are the same (n a multiple of 64)
    y, dx2, dw2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(dw)
    B.mllm_op_keep8_load(q, e, y, t, k, fmt(B, name))
    _, want = B.mllm_linear_bwd_form(t, k, n)
    scratch = torch.empty(max(want, 256), dtype=torch.uint8, device="cuda")
    B.mllm_op_linear_bwd(dy, y, w, dx2, dw2, t, k, n, workspace=scratch, scratch_bytes=want)
    assert n % 64 or (torch.equal(dx, dx2) and torch.equal(once, dw2))
    least = -(-2 * t * k // 256) * 256          # no more than it cannot do without
    B.mllm_op_linear_bwd_keep8(dy, q, e, w, dx, dw, t, k, n, fmt(B, name), ws, workspace_bytes=least)
    assert bool(((dw.double() - dw_want).abs() <= 2 * t * FP32 * dw_size).all())
    with pytest.raises(B.MllmError):
        B.mllm_op_linear_bwd_keep8(dy, q, e, w, dx, dw, t, k, n, fmt(B, name), ws, workspace_bytes=least - 256)


@pytest.mark.parametrize("t,k,n", [(9, 64, 72), (300, 520, 1000), (5000, 64, 72)])
def test_bad_rows_of_a_linear_map(B, t, k, n):
    """NaN and infinity in one row of dy: that row of dx, and with the kept values all of dw's columns that it touches; nothing else of dx has other bits."""
    x, w, dy = values(t, k, 1), (0.05 * torch.randn(k, n, device="cuda")).bfloat16(), torch.randn(t, n, device="cuda").bfloat16()
    q, e = store(B, x, "int8")
    ws = torch.full((B.mllm_op_linear_bwd_keep8_workspace_bytes(t, k, n),), 0xFF, dtype=torch.uint8, device="cuda")
    dx, dw, clean = torch.empty_like(x), torch.empty(k, n, device="cuda"), torch.empty_like(x)
    B.mllm_op_linear_bwd_keep8(dy, q, e, w, clean, dw, t, k, n, B.KEEP_INT8, ws)
    before = dw.clone()
    dy[4, 0], dy[6, n - 1] = float("nan"), float("inf")
    B.mllm_op_linear_bwd_keep8(dy, q, e, w, dx, dw, t, k, n, B.KEEP_INT8, ws)
    rows = torch.ones(t, dtype=torch.bool, device="cuda")
    rows[[4, 6]] = False
    assert torch.equal(dx[rows], clean[rows]) and torch.isnan(dx[4]).all() and not torch.isfinite(dx[6]).any()
    assert torch.isnan(dw[:, 0]).all() and torch.equal(dw[:, 1:n - 1], before[:, 1:n - 1])


def test_linear_gradients_of_no_rows(B):
    w, dw = torch.zeros(16, 24, dtype=torch.bfloat16, device="cuda"), torch.full((16, 24), 3.0, device="cuda")
    B.mllm_op_linear_bwd_keep8(None, None, None, w, None, dw, 0, 16, 24, B.KEEP_INT8, None, accumulate=1)
    assert bool((dw == 3).all())
    B.mllm_op_linear_bwd_keep8(None, None, None, w, None, dw, 0, 16, 24, B.KEEP_INT8, None)
    assert bool((dw == 0).all())


def test_offsets_beyond_32_bits(B):
    """A matrix of more than 2^32 bytes: the last rows and those around the 2^31st and 2^32nd byte."""
    t, width = 300_000, 8192
    x = torch.empty(t, width, dtype=torch.bfloat16, device="cuda")
    pattern = wide(1000, width, 3, -4, 4)
    for r in range(0, t, 1000):
        x[r:r + 1000] = pattern
    q, e = store(B, x, "int8")
    pq, pe = store(B, pattern, "int8")
    for r in (0, 131_000, 262_000, 299_000):
        assert torch.equal(q[r:r + 1000], pq) and torch.equal(e[r:r + 1000], pe)
    py = torch.empty_like(pattern)
    B.mllm_op_keep8_load(pq, pe, py, 1000, width, B.KEEP_INT8)
    B.mllm_op_keep8_load(q, e, x, t, width, B.KEEP_INT8)
    for r in (0, 131_000, 262_000, 299_000):
        assert torch.equal(x[r:r + 1000], py)
