"""Sums of the residual norms over many rows and many workgroups: every workgroup's part has to be there.

The sums of random signs nearly cancel, so that a bound by the size of their terms takes little notice of a part that is missing.  Here all terms are positive, and
for gates as they are (without tanh or sigmoid) whole numbers whose sums stay below 2^24, which fp32 holds exactly in any order."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_residual_norm import FP32, HALF, ROW, B, backward, check, check_backward, check_forward, formulas, forward, gate_of, make

gpu = pytest.mark.gpu


def split(B, t, d):
    """(workgroups, rows that one takes at a time, rows that a lane adds up) of the backward pass."""
    workgroups = B.mllm_op_residual_norm_bwd_partial_bytes(t, d) // 4 // (4 * d + 1)
    rows = max(1, 8 // -(-d // 512))
    return workgroups, rows, -(-t // (workgroups * rows))


def depth(B, t, d):
    """Additions that a sum over the rows is deep at most: a lane's rows, eight wavefronts of a workgroup, 16 + 5 additions in the second launch, the sum that is there
    already; with 30 roundings of the terms themselves and of what the sums are multiplied by (a gate's exponential and quotient among them)."""
    return split(B, t, d)[2] + 8 + 21 + 1 + 30


# Forms: one workgroup alone, one wavefront a row (512 workgroups), several wavefronts on 512, 768 and 1024 threads, rows whose results go past the caches.
SIZES = [(1, 8), (1, 4104), (2, 8192), (16, 256), (300, 1024), (3000, 72), (20000, 136), (1100, 3584), (900, 5120), (1600, 6144), (1600, 6152), (1600, 8192)]
KINDS = [("layer", "layer"), ("rms", "layer"), ("layer", "none"), ("none", "rms"), ("rms", "rms"), ("none", "none")]
GATES = ["shared", "row", "shared tanh", "none", "shared sigmoid", "row tanh"]
CASES = [(t, d, *KINDS[(i + j) % 6], (i + j) % 2 == 0, GATES[(i // 2 + 2 * j) % 6]) for i, (t, d) in enumerate(SIZES) for j in range(3)]
CASES += [(t, d, "layer", "layer", True, gate) for t, d in ((20000, 136), (1100, 3584), (1600, 8192)) for gate in ("shared", "shared tanh")]
MANY = [((8 << 20) + 13, 8, "layer", "layer", True, "shared"), ((8 << 20) + 13, 8, "none", "rms", True, "shared sigmoid"),
        (8200, 8192, "layer", "layer", True, "shared"), (11000, 6144, "rms", "layer", True, "shared tanh")]


def positive(t, d, post, pre, scale, gate, device):
    """Inputs and statistics.  The pre norm's gain is zero, so that the stream's gradient is dy as it is and whole numbers go on."""
    g = torch.Generator(device=device).manual_seed(t + d)
    whole = lambda lo, hi, *shape: torch.randint(lo, hi + 1, shape, generator=g, device=device)
    some = lambda share, *shape: (torch.rand(*shape, generator=g, device=device) < share).bfloat16()
    p = dict(t=t, d=d, post=post, pre=pre, gate_kind=gate)
    p["o"], p["y"] = whole(2, 3, t, d).bfloat16(), whole(2, 3, t, d).bfloat16()
    p["dy"], p["dn"] = some(min(0.5, 2.0 ** 20 / (t * d)), t, d), some(min(0.5, 2.0 ** 21 / t), t, d)
    p["dy"][0, 0] = 1
    p["x"] = p["y"]
    for name in ("post_g", "post_b"):
        p[name] = whole(1, 2, d).bfloat16()
    p["scale"] = whole(1, 2, d).bfloat16() if scale else None
    p["pre_g"], p["pre_b"] = torch.zeros(d, device=device).bfloat16(), torch.ones(d, device=device).bfloat16()
    p["gate"] = None if gate == "none" else whole(1, 2, t if gate.startswith("row") else 1).float()
    # factors 1 or 2, means 0 or 1: of the rows, not of their values, which plays no part in the sums
    p["stats"] = torch.stack([whole(1, 2, t), whole(0, 1, t), whole(1, 2, t), whole(0, 1, t)]).float()
    return p


def sums(p):
    """{gradient: (terms of every row [t, columns], what their sum is multiplied by)}, float64; the scale's is made of two of them."""
    f2, m2, f1, m1 = p["stats"].double()[:, :, None]
    dY, o, y = p["dy"].double(), p["o"].double(), p["y"].double()
    gate, slope = (torch.ones(1, 1, dtype=torch.float64, device=dY.device), None) if p["gate"] is None else gate_of(p)
    z = o if p["post"] == "none" else (o - (m2 if p["post"] == "layer" else 0)) * f2
    post_g = p["post_g"].double() if p["post"] != "none" else torch.ones(p["d"], dtype=torch.float64, device=dY.device)
    post_b = p["post_b"].double() if p["post"] == "layer" else torch.zeros_like(post_g)
    scale = p["scale"].double() if p["scale"] is not None else torch.ones_like(post_g)
    out, v = {}, dY * gate
    if p["post"] != "none":
        out["post_g"] = v * z * scale
    if p["post"] == "layer":
        out["post_b"] = v * scale
    if p["scale"] is not None:
        out["scale"] = v * (z * post_g + post_b)
    if p["pre"] != "none":
        out["pre_g"] = p["dn"].double() * (y - (m1 if p["pre"] == "layer" else 0)) * f1
    if p["pre"] == "layer":
        out["pre_b"] = p["dn"].double()
    if slope is not None:
        out["gate"] = (dY * (z * post_g + post_b) * scale).sum(1, keepdim=True) * slope
    dz = dY * scale * post_g
    t0 = (dz * z).mean(1, keepdim=True) if p["post"] != "none" else torch.zeros_like(f2)
    t1 = dz.mean(1, keepdim=True) if p["post"] == "layer" else torch.zeros_like(f2)
    factor = f2 * gate if p["post"] != "none" else gate
    return out, ((dz - t1 - z * t0) * factor, (dz + t1 + z * t0) * factor)


def exact(p):
    return " " not in p["gate_kind"]


@gpu
@pytest.mark.parametrize("t,d,post,pre,scale,gate", CASES + MANY)
def test_positive_sums(B, t, d, post, pre, scale, gate):
    p = positive(t, d, post, pre, scale, gate, "cuda")
    accumulate, start = (t + d) // 8 % 2, 3.0
    dx, d_o, grads = backward(B, p, p["y"], p["stats"], accumulate=accumulate, start=start)
    want, (v, size) = sums(p)
    assert torch.equal(dx, p["dy"])
    check(d_o, v, HALF * v.abs() + ROW * size, "d_o")
    assert sorted(grads) == sorted(want)
    for name, got in grads.items():
        rows = name == "gate" and gate.startswith("row")
        w = want[name][:, 0] if rows else want[name].sum(0) + (start if accumulate else 0.0)
        assert w.abs().max() < 2 ** 24 and (w > 0).any()
        if exact(p) or name.startswith("pre"):
            assert torch.equal(got.double(), w), name
        else:
            check(got, w, depth(B, t, d) * FP32 * w, name)


@pytest.mark.parametrize("t,d,post,pre,scale,gate", CASES)
def test_a_missing_part_is_noticed(B, t, d, post, pre, scale, gate):
    """Of the oracle, on the CPU: leave out one workgroup, or any wavefront's rows of one, and a gradient is further off than test_positive_sums lets it be."""
    p = positive(t, d, post, pre, scale, gate, "cpu")
    want, _ = sums(p)
    workgroups, rows, _ = split(B, t, d)
    for name, terms in want.items():
        if name == "gate" and gate.startswith("row"):
            continue
        part = torch.zeros(workgroups * rows, terms.shape[1], dtype=torch.float64).index_add_(0, torch.arange(t) % (workgroups * rows), terms)
        total = part.sum(0)
        assert torch.equal(total, terms.sum(0)) or not exact(p)
        bound = 0.0 if exact(p) or name.startswith("pre") else depth(B, t, d) * FP32 * (total + 3)
        has_rows = torch.arange(workgroups * rows) < t
        assert (part > bound).any(1)[has_rows].all(), name


# ------------------------------------------------------------------------------------------------
# Rows of 9 to 16 wavefronts, a workgroup over three rows and more in either direction.
# ------------------------------------------------------------------------------------------------
def check_gradients(B, p, y, grads):
    """The bound of the sums by their depth, the gate's terms times its slope."""
    want = formulas(p, y)
    for name, got in grads.items():
        v, size = want[name]
        if name == "gate":
            size = size * gate_of(p)[1].abs()[:, 0]
        check(got, v, (4 * ROW + depth(B, p["t"], p["d"]) * FP32) * size, name)


def check_block(B, t, d, post, pre, scale, gate):
    p = make(t, d, post, pre, scale, gate, seed=d)
    y, n, stats = forward(B, p)
    check_forward(p, y, n, stats)
    dx, d_o, grads = backward(B, p, y, stats)
    check_backward(p, y, dx, d_o, {})
    check_gradients(B, p, y, grads)


@gpu
@pytest.mark.parametrize("d", (4104, 6144, 6152, 8192))
@pytest.mark.parametrize("post,pre,scale,gate", [("layer", "layer", True, "shared tanh"), ("rms", "layer", False, "row"), ("layer", "none", True, "row sigmoid"),
                                                 ("none", "rms", True, "shared"), ("rms", "rms", False, "shared sigmoid"), ("layer", "rms", False, "none")])
def test_wide_rows(B, d, post, pre, scale, gate):
    assert split(B, 1600, d)[2] >= 3
    check_block(B, 1600, d, post, pre, scale, gate)


@gpu
@pytest.mark.parametrize("t,d", [(17000, 4000), (11000, 6144), (8200, 8192), (270000, 256)])
@pytest.mark.parametrize("post,pre,gate", [("layer", "layer", "shared tanh"), ("rms", "rms", "row")])
def test_results_past_the_caches(B, t, d, post, pre, gate):
    assert 2 * t * d >= 128 << 20
    check_block(B, t, d, post, pre, True, gate)


@gpu
@pytest.mark.parametrize("post,pre", [("layer", "rms"), ("layer", "layer"), ("rms", "rms")])
def test_bad_rows_have_no_finite_norm(B, post, pre):
    """An infinity in a block's output or a NaN in the stream leaves nothing finite of the next norm in that row, and every other row as it is."""
    for d in (64, 1536, 4104):
        p = make(90, d, post, pre, True, "row tanh")
        p["gate"][3] = 0.7
        _, n, _ = forward(B, p)
        p["o"][3, 5], p["x"][50, 1], p["x"][60, d - 1] = float("inf"), float("nan"), -float("inf")
        _, bad, _ = forward(B, p)
        rows = torch.ones(90, dtype=torch.bool, device="cuda")
        rows[[3, 50, 60]] = False
        assert torch.equal(bad[rows], n[rows])
        assert torch.isnan(bad[[3, 50]].float()).all()
        if pre == "layer":                        # (RMSNorm of an infinity alone: zeros beside a NaN)
            assert torch.isnan(bad[60].float()).all()
