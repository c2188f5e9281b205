"""Calls at the edge of what the token side's entry points document, each against its definition in float64."""
import math

import pytest

import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.gpu_util import GpuStage  # noqa: E402
from tests.test_gpu_token_ops import BF16, FP32, SHAPES, Heads, draw_ids, garbage, gen, randn, want_loss, within  # noqa: E402


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


# ---------------------------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("scale", [0.0, -2.0, float("inf"), float("nan")])
@pytest.mark.parametrize("fp32", [0, 1])
def test_rows_without_a_token_are_zero_whatever_the_scale(B, fp32, scale):
    g = gen(3)
    t, vocab, d = 70, 50, 264
    table, ids = randn(g, vocab, d, dtype=torch.float32 if fp32 else torch.bfloat16), draw_ids("mixed", t, vocab, g)
    y = torch.full((t, d), 7.0, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_embed_fwd(table, ids, y, t, vocab, d, scale=scale, table_fp32=fp32)
    want = table.double()[ids.clamp(0, vocab - 1).long()] * scale
    want[ids < 0], want[ids >= vocab] = 0.0, float("nan")
    assert bool((ids < 0).any()) and bool((ids >= vocab).any())
    within(y, want, want.abs() * (BF16 + FP32))
    assert not bool(y[ids < 0].view(torch.int16).any())      # +0


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("t,vocab,d,how", [(30000, 500, 136, "one"), (30000, 500, 136, "two"), (100000, 3000, 72, "zipf"), (65, 3, 8, "two"),
                                           (20000, 700, 4096, "one"), (20000, 700, 4096, "two"), (20000, 700, 4096, "zipf"), (16385, 5000, 4096, "uniform"),
                                           (40000, 700, 4096, "one"), (40000, 700, 4096, "two"), (40000, 700, 4096, "zipf"), (33000, 5000, 4104, "mixed"),
                                           (64, 7, 520, "one"), (64, 7, 520, "two"), (2999, 50257, 264, "zipf")])
def test_sums_of_whole_numbers_are_exact(B, t, vocab, d, how, accumulate):
    """No rounding in any order, so that one row too many or too few shows: chunks of 8, 16 and 32 tokens, ids of a whole microbatch."""
    g = gen(t + d)
    ids = draw_ids(how, t, vocab, g)
    dy = (torch.randint(1, 5, (t, d), generator=g, device="cuda") * (2 * torch.randint(0, 2, (t, d), generator=g, device="cuda") - 1)).bfloat16()
    before = torch.randint(-9, 10, (vocab, d), generator=g, device="cuda").float()
    got = before.clone() if accumulate else torch.full_like(before, float("nan"))
    B.mllm_op_embed_bwd(dy, ids, got, t, vocab, d, garbage(B.mllm_op_embed_bwd_workspace_bytes(t, vocab, d)), scale=-2.0, accumulate=accumulate)
    held = (ids >= 0) & (ids < vocab)
    want = torch.zeros(vocab, d, dtype=torch.float64, device="cuda").index_add_(0, ids[held].long(), dy[held].double()) * -2.0
    assert torch.equal(got.double(), want + before.double() if accumulate else want)


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


def quarter_turns(n_pos, hd, g):
    """A table of rotations by 0, 90, 180 and 270 degrees, an angle of its own for every pair."""
    turn = torch.randint(0, 4, (n_pos, hd // 2), generator=g, device="cuda")
    return torch.cat([torch.tensor([1.0, 0.0, -1.0, 0.0], device="cuda")[turn], torch.tensor([0.0, 1.0, 0.0, -1.0], device="cuda")[turn]], 1).contiguous()


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("t,hq,hkv,hd", [(1, 1, 1, 16), (9000, 14, 2, 64), (1500, 28, 4, 128), (33000, 32, 8, 128), (8000, 12, 3, 256), (4097, 7, 1, 32),
                                         (70001, 4, 4, 16), (777, 32, 8, 128), (20000, 1, 3, 64)])
def test_gains_gradients_of_whole_numbers_are_exact(B, t, hq, hkv, hd, rotate):
    """Heads of +1 and -1 keep their values in the norm (eps 0), and whole numbers in dy make whole terms: one head too many or too few
    shows, in lane groups that walk over many heads as well."""
    p = Heads(B, t, hq, hkv, hd, rotate)
    g, p.eps = gen(hd), 0.0
    p.x = (2 * torch.randint(0, 2, p.x.shape, generator=g, device="cuda") - 1).bfloat16()
    p.dy = (torch.randint(1, 5, p.dy.shape, generator=g, device="cuda") * (2 * torch.randint(0, 2, p.dy.shape, generator=g, device="cuda") - 1)).bfloat16()
    if rotate:
        p.table = quarter_turns(p.n_pos, hd, g)
    _, _, sums, _ = p.want_bwd()
    dx, q, k = torch.empty_like(p.x), *(torch.full((hd,), float("nan"), device="cuda") for _ in range(2))
    p.bwd(p.dy, p.x, dx, q, k)
    assert torch.equal(q.double(), sums[0]) and torch.equal(k.double(), sums[1])
    p.bwd(p.dy, p.x, dx, q, k, accumulate=1)
    assert torch.equal(q.double(), 2 * sums[0]) and torch.equal(k.double(), 2 * sums[1])


def test_positions_outside_the_table_make_their_gradients_nan(B):
    """dx of those rows, and the gains' gradients, which take terms of every row; the other rows of dx as they were."""
    p = Heads(B, 40, 3, 1, 64, True)
    good, dx, gq, gk = torch.empty_like(p.x), torch.empty_like(p.x), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    p.bwd(p.dy, p.x, good, gq, gk)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    for row, v in ((0, -1), (7, p.n_pos), (39, (1 << 31) - 1)):
        p.pos[row], bad[row] = v, True
    p.bwd(p.dy, p.x, dx, gq, gk)
    assert bool(dx[bad][:, :p.width].isnan().all()) and torch.equal(dx[~bad][:, :p.width], good[~bad][:, :p.width])
    assert bool(gq.isnan().all()) and bool(gk.isnan().all())


# ---------------------------------------------------------------------------------------------
# loss
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("t,vocab", [(600, 61), (600, 1000), (600, 2048), (300, 4096), (300, 16000), (300, 32771), (130, 65544), (2, 131072), (130, 131072)])
def test_target_s_gradient_of_confident_rows(B, t, vocab, fp32):
    """Probabilities of the target from 1 - 1e-2 to 1 - 1e-5: its gradient is weight * (p - 1), off by what the sum of the row's exponentials
    is off and by half a step of bf16.  Where the target is the row's maximum its term is 1, the additions that meet it have a half step of 2^-24
    each, the others count by their share 1 - p."""
    g, cols, weight = gen(vocab), vocab + -vocab % 8, 1.0 / 5087
    x = randn(g, t, cols, scale=2.0, dtype=torch.float32)
    targets = torch.randint(0, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    at = targets.long()[:, None]
    x.scatter_(1, at, -float("inf"))
    rest = x[:, :vocab].double().logsumexp(1)
    x.scatter_(1, at, (rest + math.log(10) * (2 + 3 * torch.rand(t, generator=g, device="cuda"))).float()[:, None])
    logits = x if fp32 else x.bfloat16()
    z = logits[:, :vocab].double()
    assert bool((z.argmax(1) == at[:, 0]).all())
    short = ((z - z.amax(1, keepdim=True)).exp().scatter(1, at, 0.0)).sum(1)
    short = short / (1 + short)                              # 1 - p, without a difference
    loss, out = torch.empty(t, device="cuda"), torch.empty(t, cols, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, vocab, cols, scale=weight, logits_fp32=fp32)
    w = float(torch.tensor(weight, dtype=torch.float32))
    # in a vector 3 and to the sum 1; vectors a thread at most 20, and 2 sums of earlier ones behind each rescaling; 6 among lanes, 16 among wavefronts; 1 / s, p - 1, w
    threads = 64 if vocab <= 2048 else 256
    vectors = min(20, -(-vocab // (8 * threads)))
    depth = 3 + vectors + 2 + 6 + (16 if vocab > 2048 else 0) + 3
    bound = w * (depth * FP32 + short * 2.0 ** -14) + w * short * BF16
    got = out.gather(1, at)[:, 0]
    within(got, -w * short, bound)
    within(loss, -torch.log1p(-short), depth * FP32 + short * 2.0 ** -14)


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("vocab,cols", [(1000, 1000), (32771, 32784), (50257, 50264), (65544, 65544), (98301, 98304), (98309, 98312), (131072, 131072),
                                        (163841, 163848), (200003, 200016), (262145, 262152)])
def test_a_row_s_loss_and_gradient_do_not_depend_on_the_rows_beside_it(B, vocab, cols, fp32):
    """Alone, among a few and among many, with the gradient, without it and in place: the same bits."""
    t, g = 300, gen(vocab)
    logits = randn(g, t, cols, scale=4.0, dtype=torch.float32 if fp32 else torch.bfloat16)
    targets = torch.randint(-1, vocab, (t,), generator=g, device="cuda", dtype=torch.int32)
    targets[:4] = vocab - 1 - torch.arange(4, device="cuda", dtype=torch.int32)
    weights = torch.rand(t, generator=g, device="cuda") + 0.5

    def call(rows, grad=True, place=False):
        x = logits[rows].clone()
        loss = torch.full((len(x),), float("nan"), device="cuda")
        out = None if not grad else x if place else torch.full((len(x), cols), 7.0, dtype=torch.bfloat16, device="cuda")
        B.mllm_op_xent(x, targets[rows], loss, out, len(x), vocab, cols, dloss=weights[rows], scale=0.37, logits_fp32=fp32)
        return loss, out

    loss, out = call(slice(0, t))
    for rows in (slice(0, 1), slice(3, 4), slice(0, 2), slice(0, 7), slice(0, 30), slice(0, 64), slice(0, 65), slice(0, 129), slice(200, 300)):
        few, part = call(rows)
        assert torch.equal(few, loss[rows]) and torch.equal(part, out[rows]), rows
        assert torch.equal(call(rows, grad=False)[0], loss[rows]), rows
        if not fp32:
            few, part = call(rows, place=True)
            assert torch.equal(few, loss[rows]) and torch.equal(part, out[rows]), rows


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("vocab,cols", [(50257, 50264), (70001, 70008), (131072, 131072), (200003, 200016)])
def test_masked_and_broken_rows_among_many(B, vocab, cols, fp32):
    """The forms for many long rows, on rows that hold no number or none but masked ones."""
    inf, nan, t, g = float("inf"), float("nan"), 300, gen(vocab)
    kind = torch.float32 if fp32 else torch.bfloat16
    logits, low = randn(g, t, cols, dtype=kind), torch.finfo(kind).min
    targets = torch.randint(0, 40, (t,), generator=g, device="cuda", dtype=torch.int32)
    for base in (0, 137, 290):
        logits[base, 45:], logits[base + 1, 45:], logits[base + 2, int(targets[base + 2])] = -inf, low, -inf
        logits[base + 3], logits[base + 4, 41], logits[base + 5, vocab - 1] = -inf, inf, nan
        targets[base + 6], targets[base + 7] = vocab, -1
        logits[base + 8], logits[base + 9] = low, -inf
        logits[base + 9, int(targets[base + 9])] = 3.0
    logits[:, vocab:] = nan
    loss, out = torch.empty(t, device="cuda"), torch.empty(t, cols, dtype=torch.bfloat16, device="cuda")
    B.mllm_op_xent(logits, targets, loss, out, t, vocab, cols, logits_fp32=fp32)
    for rows in torch.arange(t, device="cuda").split(50):
        want, size, grad, bound = want_loss(logits[rows], targets[rows], vocab, 1.0, None)
        within(loss[rows], want, size, "loss")
        within(out[rows], grad, bound, "gradient")
    alone = torch.empty(t, device="cuda")
    B.mllm_op_xent(logits, targets, alone, None, t, vocab, cols, logits_fp32=fp32)
    assert torch.equal(alone.view(torch.int32)[~loss.isnan()], loss.view(torch.int32)[~loss.isnan()]) and torch.equal(alone.isnan(), loss.isnan())


# ---------------------------------------------------------------------------------------------
# stages
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("seed", [5, 2, 3, 11])
def test_a_sample_of_a_headnorm_stage_does_not_depend_on_what_is_packed_with_it(B, seed):
    wl = W.workload_tiny_headnorm(seed)
    st = GpuStage(B, wl.layers)
    try:
        y, dx_img, dx_seq, _ = st.run(wl)
        cu = wl.batch.seq.cu_seqlens
        for s, sample in enumerate(wl.batch.samples):
            img, seq = slice(64 * s, 64 * (s + 1)), slice(cu[s], cu[s + 1])
            one = W.Workload("one", wl.layers, W.batch_from_samples([sample], img_tokens=64), wl.params, wl.x_img[img], wl.x_seq[seq], wl.dy[seq])
            y1, dx_img1, dx_seq1, _ = st.run(one)
            assert torch.equal(y1, y[seq]) and torch.equal(dx_img1, dx_img[img]) and torch.equal(dx_seq1, dx_seq[seq])
    finally:
        st.close()
