"""The token side of a language model on the GPU, each entry point against its definition in float64.

Tolerances count roundings: a bf16 result is off by at most half a step, 2^-8 of its value, beside the fp32 arithmetic in front
of it; an fp32 sum of n terms by n 2^-24 of the sum of their absolute values."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP32 = 2.0 ** -8, 2.0 ** -24
INT32_MAX = (1 << 31) - 1


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def garbage(nbytes):
    """Scratch whose contents must not matter."""
    return torch.full((max(nbytes, 256),), 0xAB, dtype=torch.uint8, device="cuda")


def within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan), what
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), what
    far = (got - want).abs() - bound
    far[nan | inf] = -1.0
    assert not bool((far > 0).any()), (what, float(far.max()), int((far > 0).sum()), far.numel())


# ---------------------------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("t,vocab,d,pad,scale", [
    (1, 1, 8, 0, 1.0), (5, 7, 24, 8, 2.5), (64, 9, 64, 0, 1.0), (333, 50257, 136, 0, 11.6), (129, 1000, 256, 0, 0.5), (67, 300, 520, 24, 1.0),
    (130, 1000, 4096, 0, 64.0), (3, 11, 8200, 16, 1.0), (1, 50, 16392, 0, 1.0),
])
def test_embed_rows(B, t, vocab, d, pad, scale, fp32):
    g = gen(t + d)
    table = randn(g, vocab, d, dtype=torch.float32 if fp32 else torch.bfloat16)
    ids = torch.randint(0, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    odd = {1: -1, 2: -100, 3: vocab, 4: INT32_MAX}          # no token, no token, beyond the table, far beyond it
    for i, v in odd.items():
        if i < t:
            ids[i] = v
    y = torch.full((t, d + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_embed_fwd(table, ids, y, t, vocab, d, y_stride=d + pad, scale=scale, table_fp32=fp32)
    want = table[ids.clamp(0, vocab - 1).long()].double() * float(torch.tensor(scale, dtype=torch.float32))
    want[ids < 0], want[ids >= vocab] = 0.0, float("nan")
    # the product in fp32, then bf16
    within(y[:, :d], want, want.abs() * (BF16 + FP32))
    assert bool((y[:, d:] == 7.0).all())
    if scale == 1.0 and not fp32:
        there = (ids >= 0) & (ids < vocab)
        assert torch.equal(y[:, :d][there], table[ids[there].long()])


def test_embed_rows_beyond_32_bit_offsets(B):
    vocab, d = 540000, 8192                                  # 4.4e9 elements
    table = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([vocab - 1, 0, 262144, 524288, vocab - 2, 262143], dtype=torch.int32, device="cuda")
    for i, v in enumerate(ids.tolist()):
        table[v] = randn(gen(i), d)
    y = torch.empty(len(ids), d, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_embed_fwd(table, ids, y, len(ids), vocab, d)
    assert torch.equal(y, torch.stack([table[v] for v in ids.tolist()]))


def draw_ids(how, t, vocab, g):
    u = torch.rand(t, generator=g, device="cuda", dtype=torch.float64)
    if how == "uniform":
        ids = (u * vocab).int()
    elif how == "zipf":
        ids = (torch.exp(u * math.log(vocab + 1)) - 1).int().clamp(0, vocab - 1)
    elif how == "one":
        ids = torch.full((t,), vocab // 2, dtype=torch.int32, device="cuda")
    elif how == "two":                                       # long runs of two, in turn
        ids = torch.where(torch.arange(t, device="cuda") // 100 % 2 == 0, 0, vocab - 1).int()
    elif how == "none":
        ids = torch.full((t,), -1, dtype=torch.int32, device="cuda")
    elif how == "ascending":
        ids = (torch.arange(t, device="cuda") % vocab).int()
    elif how == "bucket":                                    # ids that differ by multiples of 1024
        ids = ((u * max(1, vocab // 1024)).int() * 1024).clamp(max=vocab - 1)
    else:                                                    # tokens, image rows and ids that no table holds
        ids = (u * vocab).int()
        ids[u < 0.4] = -1
        ids[u > 0.9] = vocab
        ids[u > 0.95] = INT32_MAX
        ids[u < 0.05] = -INT32_MAX - 1
    return ids.int()


def embed_grad(dy, ids, vocab, scale, before=None):
    """(gradient, bound of its error) from the definition."""
    there = (ids >= 0) & (ids < vocab)
    at, f = ids[there].long(), dy[there].double() * float(torch.tensor(scale, dtype=torch.float32))
    d = dy.shape[1]
    zero = torch.zeros(vocab, d, dtype=torch.float64, device="cuda")
    want, mass = zero.clone().index_add_(0, at, f), zero.clone().index_add_(0, at, f.abs())
    count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones(len(at), dtype=torch.float64, device="cuda"))
    bound = mass * (count[:, None] + 2) * FP32               # the sum, the scale
    if before is not None:
        want += before.double()
        bound += torch.where(count[:, None] > 0, want.abs() * FP32, zero)     # the addition; other rows stay
    return want, bound


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("how", ["uniform", "zipf", "one", "two", "none", "ascending", "bucket", "mixed"])
@pytest.mark.parametrize("t,vocab,d", [(1, 1, 8), (2, 3, 24), (63, 300, 64), (65, 1000, 136), (1000, 70, 264), (1000, 70000, 8), (4097, 3000, 520)])
def test_embed_gradient(B, t, vocab, d, how, accumulate):
    g = gen(t + d + len(how))
    ids, dy, scale = draw_ids(how, t, vocab, g), randn(g, t, d), 3.7
    before = randn(g, vocab, d, dtype=torch.float32)
    got = before.clone() if accumulate else torch.full_like(before, float("nan"))
    ws = garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d))
    B.mllm_op_embed_bwd(dy, ids, got, t, vocab, d, ws, scale=scale, accumulate=accumulate)
    want, bound = embed_grad(dy, ids, vocab, scale, before if accumulate else None)
    within(got, want, bound)
    again = before.clone() if accumulate else torch.full_like(before, float("nan"))
    B.mllm_op_embed_bwd(dy, ids, again, t, vocab, d, ws, scale=scale, accumulate=accumulate)
    assert torch.equal(got, again)                           # the order of the sums does not change


@pytest.mark.parametrize("t,vocab,d,how", [(20000, 131072, 64, "zipf"), (70000, 50257, 40, "zipf"), (100000, 300000, 8, "uniform"),
                                           (50000, 600000, 8, "bucket"), (30000, 500, 136, "one"), (2999, 50257, 2056, "mixed")])
def test_embed_gradient_large(B, t, vocab, d, how):
    g = gen(t)
    ids, dy = draw_ids(how, t, vocab, g), randn(g, t, d)
    got = torch.full((vocab, d), float("nan"), device="cuda")
    ws = garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d))
    B.mllm_op_embed_bwd(dy, ids, got, t, vocab, d, ws)
    want, bound = embed_grad(dy, ids, vocab, 1.0)
    within(got, want, bound)


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("how", ["uniform", "one", "two", "mixed", "none"])
@pytest.mark.parametrize("t,vocab,d", [(1, 7, 8), (2, 3, 16), (31, 5, 8), (33, 40, 512), (63, 1000, 520), (64, 2, 24), (64, 300000, 8), (64, 33, 2056), (65, 33, 2056)])
def test_embed_gradient_of_few_tokens(B, t, vocab, d, how, accumulate):
    g = gen(t + vocab + d)
    ids, wide, scale = draw_ids(how, t, vocab, g), randn(g, t, d + 8), -1.3
    dy = wide[:, :d].clone()
    wide[(ids < 0) | (ids >= vocab)] = float("nan")          # not read
    before = randn(g, vocab, d, dtype=torch.float32)
    got = before.clone() if accumulate else torch.full_like(before, float("nan"))
    B.mllm_op_embed_bwd(wide, ids, got, t, vocab, d, garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d)), dy_stride=d + 8, scale=scale,
                        accumulate=accumulate)
    want, bound = embed_grad(dy, ids, vocab, scale, before if accumulate else None)
    within(got, want, bound)


def test_embed_gradient_of_strided_rows_and_of_no_rows(B):
    g = gen(5)
    t, vocab, d = 200, 40, 72
    wide, ids = randn(g, t, d + 40), draw_ids("uniform", t, vocab, g)
    got = torch.empty(vocab, d, device="cuda")
    ws = garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d))
    B.mllm_op_embed_bwd(wide, ids, got, t, vocab, d, ws, dy_stride=d + 40)
    want, bound = embed_grad(wide[:, :d], ids, vocab, 1.0)
    within(got, want, bound)
    B.mllm_op_embed_bwd(None, None, got, 0, vocab, d, None, accumulate=1)
    within(got, want, bound)
    B.mllm_op_embed_bwd(None, None, got, 0, vocab, d, None)
    assert not bool(got.any())


def test_embed_gradient_reads_no_row_without_an_id(B):
    """Rows of image tokens and of ids that no table holds may be anything."""
    g = gen(17)
    t, vocab, d = 1500, 900, 136
    ids, dy = draw_ids("mixed", t, vocab, g), randn(g, t, d)
    want, bound = embed_grad(dy, ids, vocab, 1.0)
    dy[(ids < 0) | (ids >= vocab)] = float("nan")
    got = torch.full((vocab, d), float("nan"), device="cuda")
    B.mllm_op_embed_bwd(dy, ids, got, t, vocab, d, garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d)))
    within(got, want, bound)


def test_embed_gradient_with_a_longer_microbatch_s_scratch(B):
    """A buffer sized for the longest microbatch, its contents left by other calls, serves shorter ones."""
    g = gen(19)
    vocab, d = 5000, 264
    ws = garbage(B.mllm_op_embed_bwd_workspace_bytes(40000, vocab, d))
    for t in (40000, 3, 33, 9000, 31, 32, 1):
        ids, dy = draw_ids("zipf", t, vocab, g), randn(g, t, d)
        got = torch.full((vocab, d), float("nan"), device="cuda")
        B.mllm_op_embed_bwd(dy, ids, got, t, vocab, d, ws)
        want, bound = embed_grad(dy, ids, vocab, 1.0)
        within(got, want, bound, t)


def test_embed_gradient_beyond_32_bit_offsets(B):
    vocab, d = 540000, 8192
    got = torch.full((vocab, d), 3.0, device="cuda")
    ids = torch.tensor([vocab - 1, 0, 262144, vocab - 1, 524288, 262143], dtype=torch.int32, device="cuda")
    dy = randn(gen(1), len(ids), d)
    B.mllm_op_embed_bwd(dy, ids, got, len(ids), vocab, d, garbage(B.mllm_op_embed_bwd_workspace_bytes(len(ids), vocab, d)))
    assert torch.equal(got[vocab - 1], dy[0].float() + dy[3].float())
    for i in (1, 2, 4, 5):
        assert torch.equal(got[int(ids[i])], dy[i].float())
        got[int(ids[i])] = 0
    got[vocab - 1] = 0
    assert not bool(got.any())


# ---------------------------------------------------------------------------------------------
# per-head norm and rotation
# ---------------------------------------------------------------------------------------------
def turned(v, table, pos, sign):
    if table is None:
        return v
    half = v.shape[-1] // 2
    f = table.double()[pos.long()][:, None]
    a, b, c, s = v[..., :half], v[..., half:], f[..., :half], sign * f[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def pair_size(v):
    """|a| + |b| of every half-split pair, at both of its places: what a rotation's rounding is relative to."""
    half = v.shape[-1] // 2
    m = v[..., :half].abs() + v[..., half:].abs()
    return torch.cat([m, m], -1)


class Heads:
    def __init__(self, B, t, hq, hkv, hd, rotate, tail=16, eps=1e-5):
        g = gen(t + 7 * hq + hd)
        self.B, self.t, self.hq, self.hkv, self.hd, self.eps = B, t, hq, hkv, hd, eps
        self.width, self.h = (hq + hkv) * hd, hq + hkv
        self.stride = self.width + tail
        self.x, self.dy = randn(g, t, self.stride, scale=1.7), randn(g, t, self.stride, scale=0.3)
        self.gq, self.gk = ((1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).bfloat16() for _ in range(2))
        self.n_pos = 37
        self.table = self.pos = None
        if rotate:
            self.table = torch.empty(self.n_pos, hd, device="cuda")
            B.mllm_op_rope_table(self.table, self.n_pos, hd, 10000.0)
            self.pos = torch.randint(0, self.n_pos, (t,), generator=g, device="cuda", dtype=torch.int32)

    def rope(self):
        return dict(pos=self.pos, rope_table=self.table, n_pos=self.n_pos if self.table is not None else 0)

    def fwd(self, x, y, y_stride=None):
        self.B.mllm_op_qk_norm_rope_fwd(x, self.gq, self.gk, y, self.t, self.hq, self.hkv, self.hd, self.stride, y_stride or self.stride, self.eps,
                                        **self.rope())

    def bwd(self, dy, x, dx, dgq, dgk, accumulate=0):
        partial = torch.full((self.B.mllm_op_qk_norm_rope_bwd_partial_bytes(self.t, self.hq, self.hkv, self.hd) // 4,), float("nan"), device="cuda")
        self.B.mllm_op_qk_norm_rope_bwd(dy, x, self.gq, self.gk, dx, dgq, dgk, self.t, self.hq, self.hkv, self.hd, self.stride, self.stride,
                                        self.stride, self.eps, partial, accumulate=accumulate, **self.rope())

    def heads(self, v):
        return v[:, :self.width].double().reshape(self.t, self.h, self.hd)

    def gain(self):
        return torch.cat([self.gq.double().expand(self.hq, -1), self.gk.double().expand(self.hkv, -1)])

    def want_fwd(self):
        x = self.heads(self.x)
        n = x / ((x * x).mean(-1, keepdim=True) + self.eps).sqrt() * self.gain()
        y = turned(n, self.table, self.pos, 1)
        return y, y.abs() * BF16 + pair_size(n) * 16 * FP32          # one bf16 rounding behind a dozen fp32 ones

    def want_bwd(self):
        x = self.heads(self.x)
        r = 1 / ((x * x).mean(-1, keepdim=True) + self.eps).sqrt()
        n, d = x * r, turned(self.heads(self.dy), self.table, self.pos, -1)
        dn, size = d * n, pair_size(self.heads(self.dy)) * n.abs()
        e = d * self.gain()
        m = (e * n).mean(-1, keepdim=True)
        dx = r * (e - n * m)
        mass = r * (pair_size(self.heads(self.dy)) * self.gain().abs() + n.abs() * (size * self.gain().abs()).mean(-1, keepdim=True))
        bound = dx.abs() * BF16 + mass * (16 + self.hd) * FP32
        sums = [v.sum((0, 1)) for v in (dn[:, :self.hq], dn[:, self.hq:])]
        sizes = [v.sum((0, 1)) * (self.t * self.h + 24) * FP32 for v in (size[:, :self.hq], size[:, self.hq:])]
        return dx, bound, sums, sizes


SHAPES = [(1, 1, 1, 16), (3, 4, 2, 64), (130, 5, 3, 32), (65, 2, 1, 48), (33, 7, 1, 80), (70, 3, 3, 96), (19, 4, 4, 112), (257, 32, 8, 128),
          (40, 25, 25, 128), (21, 2, 2, 144), (64, 9, 3, 256), (1500, 28, 4, 128)]


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("t,hq,hkv,hd", SHAPES)
def test_qk_norm_rope(B, t, hq, hkv, hd, rotate):
    p = Heads(B, t, hq, hkv, hd, rotate)
    y = torch.full_like(p.x, 7.0)
    p.fwd(p.x, y)
    want, bound = p.want_fwd()
    within(p.heads(y), want, bound)
    assert bool((y[:, p.width:] == 7.0).all())
    place = p.x.clone()
    p.fwd(place, place)
    assert torch.equal(place[:, :p.width], y[:, :p.width]) and torch.equal(place[:, p.width:], p.x[:, p.width:])
    dense = torch.empty(t, p.width, dtype=torch.bfloat16, device="cuda")
    p.fwd(p.x, dense, y_stride=p.width)
    assert torch.equal(dense, y[:, :p.width])


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("t,hq,hkv,hd", SHAPES)
def test_qk_norm_rope_gradients(B, t, hq, hkv, hd, rotate):
    p = Heads(B, t, hq, hkv, hd, rotate)
    want, bound, sums, sizes = p.want_bwd()
    dx = torch.full_like(p.x, 7.0)
    dgq, dgk = (torch.full((hd,), float("nan"), device="cuda") for _ in range(2))
    p.bwd(p.dy, p.x, dx, dgq, dgk)
    within(p.heads(dx), want, bound, "dx")
    within(dgq, sums[0], sizes[0], "dgamma_q")
    within(dgk, sums[1], sizes[1], "dgamma_k")
    assert bool((dx[:, p.width:] == 7.0).all())
    for over in ("dy", "x"):                                 # written over an input; gradients added up
        dy, x = p.dy.clone(), p.x.clone()
        gq, gk = dgq.clone(), dgk.clone()
        p.bwd(dy, x, dy if over == "dy" else x, gq, gk, accumulate=1)
        assert torch.equal((dy if over == "dy" else x)[:, :p.width], dx[:, :p.width])
        assert torch.equal(gq, dgq + dgq) and torch.equal(gk, dgk + dgk)
    both = torch.zeros(hd, device="cuda")                    # one gain for q and k: its gradients add up in one place
    p.bwd(p.dy, p.x, dx, both, both, accumulate=1)
    within(both, sums[0] + sums[1], sizes[0] + sizes[1] + (sums[0].abs() + sums[1].abs()) * FP32, "shared")


def test_qk_norm_rope_gradient_against_differences(B):
    """The derivative of sum(y * w) along random directions, from the forward definition in float64."""
    p = Heads(B, 5, 3, 2, 64, True)
    dx = torch.zeros_like(p.x)
    dgq, dgk = (torch.empty(64, device="cuda") for _ in range(2))
    p.bwd(p.dy, p.x, dx, dgq, dgk)
    w, x0, gq0, gk0 = p.heads(p.dy), p.x.double(), p.gq.double(), p.gk.double()

    def value(x, gq, gk):
        x = x[:, :p.width].reshape(p.t, p.h, p.hd)
        n = x / ((x * x).mean(-1, keepdim=True) + p.eps).sqrt() * torch.cat([gq.expand(p.hq, -1), gk.expand(p.hkv, -1)])
        return float((turned(n, p.table, p.pos, 1) * w).sum())

    g, h = gen(3), 1e-4
    for _ in range(4):
        vx, vq, vk = (torch.randn(v.shape, generator=g, device="cuda", dtype=torch.float64) for v in (x0, gq0, gk0))
        slope = (value(x0 + h * vx, gq0 + h * vq, gk0 + h * vk) - value(x0 - h * vx, gq0 - h * vq, gk0 - h * vk)) / (2 * h)
        parts = [dx[:, :p.width].double() * vx[:, :p.width], dgq.double() * vq, dgk.double() * vk]
        got = sum(float(v.sum()) for v in parts)
        # dx in bf16: half a step each, and the differences' own error (second order in h, of a function of order one)
        assert abs(got - slope) <= BF16 * float(parts[0].abs().sum()) + 1e-5 * sum(float(v.abs().sum()) for v in parts)


def test_positions_outside_the_table_make_their_rows_nan(B):
    p = Heads(B, 40, 3, 1, 64, True)
    good = torch.empty_like(p.x)
    p.fwd(p.x, good)
    for row, v in ((0, -1), (7, p.n_pos), (39, INT32_MAX)):
        p.pos[row] = v
    y = torch.empty_like(p.x)
    p.fwd(p.x, y)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[0, 7, 39]] = True
    assert bool(y[bad][:, :p.width].isnan().all()) and torch.equal(y[~bad][:, :p.width], good[~bad][:, :p.width])


def test_qk_norm_of_no_rows_and_of_zero_heads(B):
    p = Heads(B, 6, 2, 2, 64, True)
    p.x[2] = 0
    p.x[4, 64:128] = 0
    y, dx = torch.empty_like(p.x), torch.empty_like(p.x)
    dgq, dgk = (torch.empty(64, device="cuda") for _ in range(2))
    p.fwd(p.x, y)
    p.bwd(p.dy, p.x, dx, dgq, dgk)
    assert not bool(y[2, :p.width].any()) and not bool(y[4, 64:128].any())
    want, bound, sums, sizes = p.want_bwd()
    within(p.heads(dx), want, bound)
    within(dgq, sums[0], sizes[0])
    p.t = 0
    p.fwd(None, None)
    p.bwd(None, None, None, dgq, dgk, accumulate=1)
    within(dgq, sums[0], sizes[0])
    p.bwd(None, None, None, dgq, dgk)
    assert not bool(dgq.any()) and not bool(dgk.any())


def test_qk_norm_rope_gradients_with_more_scratch(B):
    """Scratch of a longer microbatch, and a microbatch long enough for lane groups that walk over several heads, repeated bit for bit."""
    p = Heads(B, 9000, 14, 2, 64, True)
    want, bound, sums, sizes = p.want_bwd()
    runs = []
    for floats in (B.mllm_op_qk_norm_rope_bwd_partial_bytes(p.t, p.hq, p.hkv, p.hd) // 4, B.mllm_op_qk_norm_rope_bwd_partial_bytes(100000, p.hq, p.hkv, p.hd) // 4):
        partial = torch.full((floats,), float("nan"), device="cuda")
        dx, dgq, dgk = torch.zeros_like(p.x), torch.empty(p.hd, device="cuda"), torch.empty(p.hd, device="cuda")
        B.mllm_op_qk_norm_rope_bwd(p.dy, p.x, p.gq, p.gk, dx, dgq, dgk, p.t, p.hq, p.hkv, p.hd, p.stride, p.stride, p.stride, p.eps, partial, **p.rope())
        runs.append((dx, dgq, dgk))
    within(p.heads(dx), want, bound)
    within(dgq, sums[0], sizes[0])
    within(dgk, sums[1], sizes[1])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


# ---------------------------------------------------------------------------------------------
# loss
# ---------------------------------------------------------------------------------------------
def want_loss(logits, targets, vocab, scale, dloss):
    """(loss, its bound, gradient, its bound) from the definition, logits [t, cols]."""
    x = logits[:, :vocab].double()
    t = x.shape[0]
    there, at = targets >= 0, targets.clamp(0, vocab - 1).long()[:, None]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    s = e.sum(1, keepdim=True)
    loss = (s.log() + (m - x.gather(1, at)))[:, 0]
    w = torch.full((t, 1), float(torch.tensor(scale, dtype=torch.float32)), dtype=torch.float64, device="cuda")
    if dloss is not None:
        w = w * dloss.double()[:, None]
    p = e / s
    grad = torch.zeros(logits.shape, dtype=torch.float64, device="cuda")
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    grad[:, :vocab] = (p - one) * w
    # exponents up to 128 in fp32 (2^-24 each of them and of a difference): a probability is off by 2^-16 of itself; below the
    # smallest normal number (2^-126, of it and of its product with the weight) it may be flushed
    slack = torch.zeros_like(grad)
    slack[:, :vocab] = w.abs() * (p * 2.0 ** -16 + 2.0 ** -126)
    bound = grad.abs() * BF16 + slack + 2.0 ** -126
    bad = targets >= vocab
    loss[bad], grad[bad, :vocab] = float("nan"), float("nan")
    loss[~there], grad[~there] = 0.0, 0.0
    # the sum (terms weighted by their size: exponents near zero count most), its logarithm, the difference to the target
    size = 2.0 ** -20 * (1 + s.log().abs() + (m - x.gather(1, at)).abs())[:, 0]
    size[~there], bound[~there] = 0.0, 0.0
    return loss, size, grad, bound


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("t,vocab,cols", [(1, 1, 8), (2, 2, 8), (5, 7, 8), (3, 8, 8), (4, 9, 16), (300, 61, 64), (67, 1000, 1000), (9, 2047, 2048), (6, 2050, 2176),
                                          (5, 8191, 8192), (3, 16384, 16384), (4, 16393, 16400), (3, 32768, 32768), (7, 50257, 50264), (3, 65536, 65536),
                                          (2, 65537, 65600), (2, 131071, 131072), (3, 131073, 131080), (2, 200000, 200000), (2, 262144, 262144),
                                          (2, 262145, 262152), (2, 600001, 600008)])
def test_loss_and_gradient(B, t, vocab, cols, fp32):
    g = gen(t + vocab)
    logits = randn(g, t, cols, scale=4.0, dtype=torch.float32 if fp32 else torch.bfloat16)
    logits[:, vocab:] = float("nan")                         # padding of the vocabulary is never used
    targets = torch.randint(0, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    targets[0] = vocab - 1
    if t > 2:
        targets[1] = -100
        logits[1] = float("nan")                             # nor is a row without a target
    dloss = torch.rand(t, generator=g, device="cuda") + 0.5
    for weights, scale in ((None, 1.0), (dloss, 0.37)):
        want, size, grad, bound = want_loss(logits, targets, vocab, scale, weights)
        loss = torch.full((t,), float("nan"), device="cuda")
        out = torch.full((t, cols), 7.0, dtype=torch.bfloat16, device="cuda")
        B.mllm_op_xent(logits, targets, loss, out, t, vocab, cols, dloss=weights, scale=scale, logits_fp32=fp32)
        within(loss, want, size, "loss")
        within(out, grad, bound, "gradient")
        alone = torch.full((t,), float("nan"), device="cuda")
        B.mllm_op_xent(logits, targets, alone, None, t, vocab, cols, logits_fp32=fp32)
        assert torch.equal(alone, loss)
    if not fp32:
        place, alone = logits.clone(), torch.empty(t, device="cuda")
        B.mllm_op_xent(place, targets, alone, place, t, vocab, cols, dloss=dloss, scale=0.37)
        assert torch.equal(place, out) and torch.equal(alone, loss)


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("t,vocab,cols", [(300, 2043, 2048), (257, 4099, 4104), (260, 8195, 8200), (257, 16401, 16408), (300, 32771, 32784),
                                          (140, 65537, 65544), (90, 98309, 98312), (100, 140001, 140008), (90, 200003, 200016)])
def test_loss_and_gradient_of_many_rows(B, t, vocab, cols, fp32):
    """More rows than the few that several workgroups share, one or two vectors beyond each form's step."""
    g = gen(t + vocab)
    logits = randn(g, t, cols, scale=4.0, dtype=torch.float32 if fp32 else torch.bfloat16)
    logits[:, vocab:] = float("nan")
    targets = torch.randint(0, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    targets[::5], targets[-1], logits[7] = -1, vocab - 1, -float("inf")
    logits[7, vocab - 1] = 1.0
    loss, out = torch.full((t,), float("nan"), device="cuda"), torch.full((t, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, vocab, cols, scale=-0.6, logits_fp32=fp32)
    for rows in torch.arange(t, device="cuda").split(50):
        want, size, grad, bound = want_loss(logits[rows], targets[rows], vocab, -0.6, None)
        within(loss[rows], want, size, "loss")
        within(out[rows], grad, bound, "gradient")
    if not fp32:
        B.mllm_op_xent(logits, targets, loss, logits, t, vocab, cols, scale=-0.6)
        assert torch.equal(logits, out)


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("vocab,cols", [(50, 56), (3000, 3008), (50257, 50264), (140000, 140000), (300000, 300000)])
def test_loss_of_masked_and_broken_rows(B, vocab, cols, fp32):
    inf, nan = float("inf"), float("nan")
    t, g = 12, gen(vocab)
    kind = torch.float32 if fp32 else torch.bfloat16
    logits = randn(g, t, cols, dtype=kind)
    targets = torch.randint(0, 40, (t,), generator=g, device="cuda", dtype=torch.int32)
    low = torch.finfo(kind).min
    logits[0, 45:] = -inf                                    # masked with -inf
    logits[1, 45:] = low                                     # masked with the type's lowest value
    logits[2, int(targets[2])] = -inf                        # the target itself masked: loss +inf
    logits[3] = -inf                                         # nothing left
    logits[4, 41] = inf
    logits[5, 41] = nan
    targets[6] = vocab                                       # beyond the vocabulary
    targets[7] = INT32_MAX
    targets[8] = -INT32_MAX - 1                              # no target
    logits[9] = low                                          # all equal: log(vocab)
    logits[10], logits[10, int(targets[10])] = -inf, 3.0     # one left: probability 1, loss 0
    logits[11] = 100.0 * logits[11]
    want, size, grad, bound = want_loss(logits, targets, vocab, 1.0, None)
    assert want[2] == inf and bool(want[3:8].isnan().all()) and want[8] == 0 and abs(float(want[9]) - math.log(vocab)) < 1e-9 and want[10] == 0
    loss, out = torch.empty(t, device="cuda"), torch.empty(t, cols, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, vocab, cols, logits_fp32=fp32)
    within(loss, want, size)
    for row in range(t):
        within(out[row], grad[row], bound[row], row)


def test_loss_of_strided_rows_and_of_no_rows(B):
    g = gen(9)
    t, vocab, cols, stride, dstride = 31, 333, 336, 400, 352
    logits, targets = randn(g, t, stride, scale=2.0), torch.randint(0, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    loss, out = torch.empty(t, device="cuda"), torch.full((t, dstride), 7.0, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, vocab, cols, logits_stride=stride, dlogits_stride=dstride)
    want, size, grad, bound = want_loss(logits[:, :cols].contiguous(), targets, vocab, 1.0, None)
    within(loss, want, size)
    within(out[:, :cols], grad, bound)
    assert bool((out[:, cols:] == 7.0).all())
    B.mllm_op_xent(None, None, None, None, 0, vocab, cols)


def test_loss_gradient_against_differences(B):
    g = gen(11)
    t, vocab = 6, 96
    logits, targets = randn(g, t, vocab, scale=2.0, dtype=torch.float32), torch.randint(0, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.rand(t, generator=g, device="cuda") + 0.5
    loss, out = torch.empty(t, device="cuda"), torch.empty(t, vocab, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, vocab, vocab, dloss=weights, logits_fp32=1)
    h, x0 = 1e-4, logits.double()
    value = lambda x: float((weights.double() * (x.logsumexp(1) - x.gather(1, targets.long()[:, None])[:, 0])).sum())
    for _ in range(4):
        v = torch.randn(t, vocab, generator=g, device="cuda", dtype=torch.float64)
        slope, part = (value(x0 + h * v) - value(x0 - h * v)) / (2 * h), out.double() * v
        assert abs(float(part.sum()) - slope) <= (BF16 + 1e-5) * float(part.abs().sum())


def test_loss_beyond_32_bit_offsets(B):
    t, vocab = 33000, 131072                                 # 4.3e9 elements, 8.6 GB, the gradient in place
    logits = torch.zeros(t, vocab, dtype=torch.bfloat16, device="cuda")
    rows = [0, 1, 16383, 16384, 32767, 32768, t - 1]
    targets = torch.full((t,), -1, dtype=torch.int32, device="cuda")
    for i, r in enumerate(rows):
        logits[r], targets[r] = randn(gen(i), vocab, scale=3.0), 7 + i
    kept = logits[rows].clone()
    loss = torch.empty(t, device="cuda")
    B.mllm_op_xent(logits, targets, loss, logits, t, vocab, vocab)
    want, size, grad, bound = want_loss(kept, targets[rows], vocab, 1.0, None)
    within(loss[rows], want, size)
    within(logits[rows], grad, bound)
    logits[rows], loss[rows] = 0, 0
    assert not bool(loss.any())
    for part in logits.split(4096):
        assert not bool(part.any())


def test_more_rows_than_a_dimension_of_a_grid_holds(B):
    """Launches that go on in a second dimension, or walk on: 2^20 workgroups along the first."""
    g = gen(23)
    t = 4 * (1 << 20) + 4099                                 # four rows a workgroup
    logits = randn(g, t, 8, scale=2.0)
    targets = torch.randint(-1, 5, (t,), generator=g, device="cuda", dtype=torch.int32)
    loss, out = torch.full((t,), float("nan"), device="cuda"), torch.full_like(logits, 7.0)
    B.mllm_op_xent(logits, targets, loss, out, t, 5, 8)
    want, size, grad, bound = want_loss(logits, targets, 5, 1.0, None)
    within(loss, want, size)
    within(out, grad, bound)
    t = 2 * (1 << 20) + 77                                   # one row a workgroup
    logits, targets = logits[:t].expand(t, 8).repeat(1, 257), targets[:t].contiguous()       # 2056 columns
    loss, out = torch.full((t,), float("nan"), device="cuda"), torch.empty(t, 2056, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, 2050, 2056)
    rows = torch.cat([torch.arange(3), torch.arange((1 << 20) - 2, (1 << 20) + 3), torch.arange((1 << 21) - 2, t)]).cuda()
    want, size, grad, bound = want_loss(logits[rows], targets[rows], 2050, 1.0, None)
    within(loss[rows], want, size)
    within(out[rows], grad, bound)
    assert not bool(loss.isnan().any())
    del logits, out
    t = 32 * (1 << 20) + 1003                                # 32 rows of 64 columns or fewer a workgroup
    table = randn(g, 11, 8)
    ids = torch.randint(-1, 11, (t,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.full((t, 8), 7.0, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_embed_fwd(table, ids, y, t, 11, 8)
    assert torch.equal(y, torch.cat([table, torch.zeros_like(table[:1])])[ids.long()])


@pytest.mark.parametrize("t", [30, 100, 5000])
def test_a_table_of_more_than_a_dimension_of_a_grid_is_cleared_but_for_the_ids(B, t):
    """Where a table is overwritten a workgroup takes 4 KB of it: 2^18 rows of 4096 columns fill the first dimension."""
    g = gen(31 + t)
    vocab, d = (1 << 18) + 1500, 4096
    ids = torch.cat([torch.randint(0, vocab, (t - 12,), generator=g, device="cuda", dtype=torch.int32),
                     torch.tensor([0, vocab - 1, (1 << 18) - 1, 1 << 18, vocab, -1] * 2, dtype=torch.int32, device="cuda")])
    dy = torch.randint(-4, 5, (t, d), generator=g, device="cuda").bfloat16()    # whose sums have no roundings
    want = torch.zeros(vocab, d, device="cuda")
    held = (ids >= 0) & (ids < vocab)
    want.index_add_(0, ids[held], dy[held].float())
    got = torch.full((vocab, d), float("nan"), device="cuda")
    B.mllm_op_embed_bwd(dy, ids, got, t, vocab, d, garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d)))
    assert torch.equal(got, want)


# ---------------------------------------------------------------------------------------------
# streams and graphs
# ---------------------------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph(B):
    """Every call captured into one graph and replayed on new inputs, with eager work in between, equals eager calls; and so do calls
    on a stream of their own."""
    g = gen(13)
    t, vocab, d = 700, 3001, 264
    table = randn(g, vocab, d)
    ids, ids2 = (draw_ids("zipf", t, vocab, g) for _ in range(2))
    dy = randn(g, t, d)
    cols = 3008
    logits, targets = randn(g, t, cols, scale=3.0), draw_ids("uniform", t, vocab, g)
    heads = Heads(B, t, 6, 2, 64, True)
    partial = torch.empty(B.mllm_op_qk_norm_rope_bwd_partial_bytes(t, 6, 2, 64) // 4, device="cuda")
    ws = garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d))

    def outputs():
        return [torch.zeros(t, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(vocab, d, device="cuda"), torch.zeros_like(heads.x),
                torch.zeros_like(heads.x), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(t, device="cuda"),
                torch.zeros(t, cols, dtype=torch.bfloat16, device="cuda")]

    def calls(o, stream=None):
        B.mllm_op_embed_fwd(table, ids, o[0], t, vocab, d, stream=stream)
        B.mllm_op_embed_bwd(dy, ids, o[1], t, vocab, d, ws, stream=stream)
        rope, dims = heads.rope(), (t, 6, 2, 64)
        B.mllm_op_qk_norm_rope_fwd(heads.x, heads.gq, heads.gk, o[2], *dims, heads.stride, heads.stride, 1e-5, stream=stream, **rope)
        B.mllm_op_qk_norm_rope_bwd(heads.dy, heads.x, heads.gq, heads.gk, o[3], o[4], o[5], *dims, heads.stride, heads.stride, heads.stride, 1e-5,
                                   partial, stream=stream, **rope)
        B.mllm_op_xent(logits, targets, o[6], o[7], t, vocab, cols, stream=stream)

    side = torch.cuda.Stream()
    own = outputs()
    torch.cuda.synchronize()
    calls(own, stream=side)
    torch.cuda.synchronize()
    eager = outputs()
    calls(eager)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(own, eager))
    replayed = outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(replayed)
    for turn in range(4):
        ids.copy_(ids2 if turn % 2 else ids.flip(0))
        logits.mul_(0.9)
        heads.x.mul_(-1.1)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in replayed]
        eager = outputs()
        calls(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), turn
