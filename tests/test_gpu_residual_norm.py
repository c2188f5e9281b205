"""The residual stream between two blocks, forward and backward, against the formulas in float64."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8          # one rounding to bf16, of the value
FP32 = 2.0 ** -24
# Sums over a row of at most 8192: 8 in a lane, 6 + 4 exchanges, so 18 additions deep; a square, a quotient and the square root's two ulps with it.
# Factors of a norm are therefore off by at most 24 FP32 of themselves, and what is made from a few of them and a few products by at most:
ROW = 64 * FP32
KINDS = ("none", "rms", "layer")


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


def make(t, d, post, pre, scale, gate, seed=0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    p = dict(post=post, pre=pre, gate_kind=gate, t=t, d=d)
    p["x"], p["o"] = rand(t, d).bfloat16(), (0.7 * rand(t, d) + mean).bfloat16()
    p["dn"], p["dy"] = (0.3 * rand(t, d)).bfloat16(), (0.3 * rand(t, d)).bfloat16()
    vector = lambda m, s: (m + s * rand(d)).bfloat16()
    p["post_g"], p["pre_g"], p["scale"] = vector(1, 0.3), vector(1, 0.3), vector(0.5, 0.3) if scale else None
    p["post_b"], p["pre_b"] = vector(0, 0.3), vector(0, 0.3)
    p["gate"] = None if gate == "none" else rand(t) if gate.startswith("row") else rand(1)
    if gate == "row":
        p["gate"][::3] = 0.0
    return p


def block(B, p, eps=1e-5):
    kinds = dict(none=B.NORM_NONE, rms=B.NORM_RMS, layer=B.NORM_LAYER)
    act = B.GATE_TANH if "tanh" in p["gate_kind"] else B.GATE_SIGMOID if "sigmoid" in p["gate_kind"] else B.GATE_LINEAR
    return B.ResidualNorm(post_kind=kinds[p["post"]], post_g=p["post_g"], post_b=p["post_b"], post_eps=eps, scale=p["scale"], gate=p["gate"],
                          gate_per_row=p["gate_kind"].startswith("row"), gate_act=act, pre_kind=kinds[p["pre"]], pre_g=p["pre_g"],
                          pre_b=p["pre_b"], pre_eps=eps)


def forward(B, p, **kw):
    y, n = torch.empty_like(p["x"]), torch.full_like(p["x"], 5.0)
    stats = torch.full((4, p["t"]), 7.0, device="cuda")
    B.mllm_op_residual_norm_fwd(block(B, p, **kw), p["x"], p["o"], y, n, stats, p["t"], p["d"])
    return y, n, stats


def norm(kind, v, g, b, eps):
    """(result, normalised values, factor, size of the result's terms)."""
    if kind == "none":
        one = torch.ones_like(v[:, :1])
        return v, v, one, torch.zeros_like(v)
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    f = ((v - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    h = (v - mean) * f
    size = (h.abs() + mean.abs() * f) * g.double().abs()
    if kind == "layer":
        return h * g.double() + b.double(), h, f, size + b.double().abs()
    return h * g.double(), h, f, size


def gate_of(p):
    """(gate, slope), [t or 1, 1]."""
    if p["gate"] is None:
        return torch.ones(1, 1, dtype=torch.float64, device="cuda"), None
    v = p["gate"].double()[:, None]
    if "tanh" in p["gate_kind"]:
        return v.tanh(), 1 - v.tanh() ** 2
    if "sigmoid" in p["gate_kind"]:
        return v.sigmoid(), v.sigmoid() * (1 - v.sigmoid())
    return v, torch.ones_like(v)


def check(got, want, bound, what):
    excess = ((got.double() - want).abs() - bound)
    assert torch.isfinite(want).all() and bool((excess <= 0).all()), (what, excess.max().item(), bound.max().item())


def check_forward(p, y, n, stats, eps=1e-5):
    u, _, f, size = norm(p["post"], p["o"].double(), p["post_g"], p["post_b"], eps)
    by = gate_of(p)[0] * (1.0 if p["scale"] is None else p["scale"].double())
    want = p["x"].double() + u * by
    check(y, want, HALF * want.abs() + ROW * (p["x"].double().abs() + (u.abs() + size) * by.abs()), "y")
    if p["post"] != "none":
        check(stats[0], f[:, 0], ROW * f[:, 0], "factor of post")
    if p["pre"] == "none":
        assert bool((n == 5.0).all()) and bool((stats[2:] == 7.0).all())
        return
    want, _, f, size = norm(p["pre"], y.double(), p["pre_g"], p["pre_b"], eps)
    check(n, want, HALF * want.abs() + ROW * size, "n")
    check(stats[2], f[:, 0], ROW * f[:, 0], "factor of pre")


GRADS = ("post_g", "post_b", "scale", "pre_g", "pre_b", "gate")


def backward(B, p, y, stats, accumulate=0, dy=True, only=GRADS, start=0.0, dx=None, d_o=None):
    there = dict(post_g=p["post"] != "none", post_b=p["post"] == "layer", scale=p["scale"] is not None, pre_g=p["pre"] != "none",
                 pre_b=p["pre"] == "layer", gate=p["gate"] is not None)
    grads = {k: torch.full((len(p["gate"]) if k == "gate" else p["d"],), start if accumulate else float("nan"), device="cuda")
             for k in GRADS if there[k] and k in only}
    dx, d_o = torch.empty_like(p["x"]) if dx is None else dx, torch.empty_like(p["x"]) if d_o is None else d_o
    partial = torch.full((B.mllm_op_residual_norm_bwd_partial_bytes(p["t"], p["d"]) // 4,), float("nan"), device="cuda")
    B.mllm_op_residual_norm_bwd(block(B, p), p["dn"], p["dy"] if dy else None, y, p["o"], stats, dx, d_o, B.ResidualNormGrads(**grads), partial,
                                p["t"], p["d"], accumulate=accumulate)
    return dx, d_o, grads


def formulas(p, y, dy=True, eps=1e-5):
    """{output: (value, size of the terms that it is the sum of)}."""
    out = {}
    dY = p["dy"].double() if dy else torch.zeros_like(p["x"], dtype=torch.float64)
    size_dY = dY.abs()

    def through(kind, dv, size_dv, v, g):
        """The gradient in front of a norm from that behind it."""
        _, h, f, _ = norm(kind, v, g, torch.zeros_like(g), eps)
        mean = v.mean(1, keepdim=True).abs() if kind == "layer" else 0.0
        dh, size = dv * g.double(), size_dv * g.double().abs()
        reach = h.abs() + mean * f                       # what a rounding of the mean or the value amounts to in h
        out_v = dh - h * (dh * h).mean(1, keepdim=True) - (dh.mean(1, keepdim=True) if kind == "layer" else 0.0)
        return out_v * f, (size + reach * (size * reach).mean(1, keepdim=True) + size.mean(1, keepdim=True)) * f, h, reach

    if p["pre"] != "none":
        dn = p["dn"].double()
        add, size, h, reach = through(p["pre"], dn, dn.abs(), y.double(), p["pre_g"])
        dY, size_dY = dY + add, size_dY + size
        out["pre_g"] = (dn * h).sum(0), (dn.abs() * reach).sum(0)
        out["pre_b"] = dn.sum(0), dn.abs().sum(0)
    out["dx"] = dY, size_dY
    gate, slope = gate_of(p)
    scale = torch.ones(p["d"], dtype=torch.float64, device="cuda") if p["scale"] is None else p["scale"].double()
    u, z, f, size_u = norm(p["post"], p["o"].double(), p["post_g"], p["post_b"], eps)
    size_u = size_u + u.abs()
    if slope is not None:
        rows, size = (dY * u * scale).sum(1, keepdim=True) * slope, (size_dY * size_u * scale.abs()).sum(1, keepdim=True)
        out["gate"] = (rows[:, 0], size[:, 0]) if p["gate_kind"].startswith("row") else (rows.sum()[None], size.sum()[None])
    v, size_v = dY * gate, size_dY * gate.abs()
    out["scale"] = (v * u).sum(0), (size_v * size_u).sum(0)
    v, size_v = v * scale, size_v * scale.abs()
    if p["post"] != "none":
        v, size_v_in, h, reach = through(p["post"], v, size_v, p["o"].double(), p["post_g"])
        out["post_g"] = (dY * gate * scale * h).sum(0), (size_v * reach).sum(0)
        out["post_b"] = (dY * gate * scale).sum(0), size_v.sum(0)
        size_v = size_v_in
    out["d_o"] = v, size_v
    return out


def check_backward(p, y, dx, d_o, grads, dy=True, times=1, start=0.0):
    want = formulas(p, y, dy)
    for name, got in (("dx", dx), ("d_o", d_o)):
        v, size = want[name]
        check(got, v, HALF * v.abs() + 4 * ROW * size, name)
    for name, got in grads.items():
        v, size = want[name]
        # a lane adds its rows one after the other (at most t of them), then the workgroups' sums: counted with the terms' own errors
        check(got, times * v + start, (4 * ROW + (p["t"] + 40) * FP32) * (times * size + abs(start)), name)


SHAPES = [(1, 8), (3, 8), (5, 64), (17, 504), (64, 512), (33, 520), (40, 1024), (9, 1032), (20, 1536), (7, 2056), (700, 256), (30, 4096), (11, 5120),
          (5, 8192), (2, 8184)]
BLOCKS = list(itertools.product(KINDS, KINDS, (False, True)))
GATES = ("none", "row", "shared", "shared tanh", "row sigmoid", "row tanh", "shared sigmoid")


@pytest.mark.parametrize("post,pre,scale", BLOCKS)
def test_every_kind(B, post, pre, scale):
    for i, (t, d) in enumerate(SHAPES):
        p = make(t, d, post, pre, scale, GATES[(i + 3 * scale) % len(GATES)], seed=i)
        y, n, stats = forward(B, p)
        check_forward(p, y, n, stats)
        dx, d_o, grads = backward(B, p, y, stats)
        check_backward(p, y, dx, d_o, grads)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("t,d", [(1, 16), (300, 1024), (3000, 72), (1100, 3584)])
def test_gates(B, gate, t, d):
    for post, scale in (("rms", True), ("layer", False), ("none", True)):
        p = make(t, d, post, "rms", scale, gate, seed=t)
        y, n, stats = forward(B, p)
        check_forward(p, y, n, stats)
        check_backward(p, y, *backward(B, p, y, stats))


def test_gates_far_out(B):
    """Where the gate's slope is small it is off by a few roundings of itself, not of 1: 20 FP32 and the exponential's argument of up to 40."""
    for gate in ("row tanh", "row sigmoid"):
        p = make(41, 64, "none", "none", False, gate)
        p["gate"] = torch.linspace(-20, 20, 41, device="cuda")
        y, n, stats = forward(B, p)
        check_forward(p, y, n, stats)
        dx, d_o, grads = backward(B, p, y, stats)
        v = p["gate"].double()
        slope = 1 / torch.cosh(v) ** 2 if "tanh" in gate else 1 / (2 + v.exp() + (-v).exp())
        dots = p["dy"].double() * p["o"].double()
        assert bool(((grads["gate"].double() - dots.sum(1) * slope).abs() <= 100 * FP32 * dots.abs().sum(1) * slope).all())


def test_many_rows(B):
    """Workgroups that go over many rows, and more rows than a dimension of a grid holds workgroups of eight."""
    p = make(20000, 136, "layer", "layer", True, "shared tanh", seed=1)
    y, n, stats = forward(B, p)
    check_forward(p, y, n, stats)
    check_backward(p, y, *backward(B, p, y, stats))
    t = (8 << 20) + 13
    p = make(t, 8, "none", "rms", False, "none", seed=2)
    y, n, stats = forward(B, p)
    check_forward(p, y, n, stats)
    dx, d_o, grads = backward(B, p, y, stats)
    want = formulas(p, y)
    for name, got in (("dx", dx), ("d_o", d_o)):
        v, size = want[name]
        check(got, v, HALF * v.abs() + 4 * ROW * size, name)


def test_rows_far_from_zero(B):
    """A mean of many times the deviation: LayerNorm subtracts it before it squares."""
    for post, pre in (("layer", "layer"), ("layer", "none")):
        p = make(50, 1000, post, pre, False, "none", mean=60.0)
        p["x"] += 40
        y, n, stats = forward(B, p)
        check_forward(p, y, n, stats)
        check_backward(p, y, *backward(B, p, y, stats))


def test_rows_of_zeros(B):
    """Dropped or padded rows: no block output and no stream; with eps the norms are finite, and zero."""
    p = make(6, 256, "rms", "layer", True, "row")
    p["x"][2:4], p["o"][2:4] = 0, 0
    y, n, stats = forward(B, p)
    check_forward(p, y, n, stats)
    assert bool((y[2:4] == 0).all()) and torch.equal(n[2:4], p["pre_b"].expand(2, -1))
    check_backward(p, y, *backward(B, p, y, stats))


@pytest.mark.parametrize("d", (8, 1000, 3200, 4104, 8184))
def test_rows_of_equal_values(B, d):
    """The mean of equal values is that value (their sum has no more than 24 digits), so that nothing is left of them, whatever eps."""
    p = make(40, d, "layer", "layer", False, "none")
    p["x"][:], p["o"][:] = torch.linspace(-300, 500, 40, device="cuda").bfloat16()[:, None], torch.linspace(90, -7, 40, device="cuda").bfloat16()[:, None]
    p["post_b"][:] = 0
    y, n, stats = forward(B, p, eps=1e-12)
    assert torch.equal(y, p["x"]) and torch.equal(n, p["pre_b"].expand(40, -1))
    assert torch.equal(stats[1], p["o"][:, 0].float()) and torch.equal(stats[3], p["x"][:, 0].float())


@pytest.mark.parametrize("scale,gate", [(False, "none"), (True, "row")])
def test_gradient_of_a_plain_residual(B, scale, gate):
    """Without a norm behind the block and without the scale's and the gate's gradients its output plays no part."""
    p = make(300, 1032, "none", "rms", scale, gate)
    y, _, stats = forward(B, p)
    want = backward(B, p, y, stats)
    p["o"] = torch.full_like(p["o"], float("nan"))
    dx, d_o, grads = backward(B, p, y, stats, only=("pre_g",))
    assert torch.equal(dx, want[0]) and torch.equal(d_o, want[1]) and torch.equal(grads["pre_g"], want[2]["pre_g"])
    assert scale or torch.equal(d_o, dx)


@pytest.mark.parametrize("t,d", [(77, 640), (5, 640), (1, 4104), (9, 136)])      # the last three by one workgroup alone
def test_accumulate_and_what_is_not_wanted(B, t, d):
    p = make(t, d, "layer", "layer", True, "shared tanh")
    y, _, stats = forward(B, p)
    dx, d_o, once = backward(B, p, y, stats)
    _, _, twice = backward(B, p, y, stats, accumulate=1, start=0.5)
    check_backward(p, y, dx, d_o, twice, start=0.5)
    for name in GRADS:                       # one of them at a time: the same bits
        dx1, d_o1, alone = backward(B, p, y, stats, only=(name,))
        assert list(alone) == [name] and torch.equal(alone[name], once[name]) and torch.equal(dx1, dx) and torch.equal(d_o1, d_o)
    dx1, d_o1, none = backward(B, p, y, stats, only=())
    assert not none and torch.equal(dx1, dx) and torch.equal(d_o1, d_o)
    p = make(t, d, "layer", "layer", True, "row tanh")      # a gate for every row is overwritten, never added to
    y, _, stats = forward(B, p)
    _, _, once = backward(B, p, y, stats)
    _, _, twice = backward(B, p, y, stats, accumulate=1, start=0.5)
    assert torch.equal(once["gate"], twice["gate"])


def test_without_the_streams_gradient(B):
    p = make(50, 264, "rms", "rms", True, "shared")
    y, _, stats = forward(B, p)
    dx, d_o, grads = backward(B, p, y, stats, dy=False)
    check_backward(p, y, dx, d_o, grads, dy=False)


@pytest.mark.parametrize("t,d", [(37, 96), (600, 4096)])
def test_in_place(B, t, d):
    p = make(t, d, "rms", "layer", True, "row")
    y, n, stats = forward(B, p)
    want = backward(B, p, y, stats)
    x = p["x"].clone()
    stats2, n2 = torch.empty_like(stats), torch.empty_like(n)
    B.mllm_op_residual_norm_fwd(block(B, p), x, p["o"], x, n2, stats2, t, d)
    assert torch.equal(x, y) and torch.equal(n2, n)
    for swap in (False, True):
        dn, dy = p["dn"].clone(), p["dy"].clone()
        q = dict(p, dn=dn, dy=dy)
        got = backward(B, q, y, stats, dx=dn if swap else dy, d_o=dy if swap else dn)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and all(torch.equal(got[2][k], want[2][k]) for k in want[2])


def test_rows_by_themselves(B):
    """A row's results have the same bits whatever rows are beside it, and bad rows stay among themselves."""
    p = make(90, 1536, "layer", "rms", True, "row tanh")
    y, n, stats = forward(B, p)
    dx, d_o, grads = backward(B, p, y, stats)
    few = {k: v[40:47].contiguous() if torch.is_tensor(v) and v.shape[0] == 90 else v for k, v in p.items()}
    few["t"] = 7
    y2, n2, stats2 = forward(B, few)
    assert torch.equal(y2, y[40:47]) and torch.equal(n2, n[40:47])
    dx2, d_o2, grads2 = backward(B, few, y2, stats2)
    assert torch.equal(dx2, dx[40:47]) and torch.equal(d_o2, d_o[40:47]) and torch.equal(grads2["gate"], grads["gate"][40:47])
    p["o"][3, 5], p["x"][50, 1], p["dn"][70, 9] = float("inf"), float("nan"), -float("inf")
    y3, n3, stats3 = forward(B, p)
    rows = torch.ones(90, dtype=torch.bool, device="cuda")
    rows[[3, 50]] = False
    assert torch.equal(y3[rows], y[rows]) and torch.equal(n3[rows], n[rows]) and not torch.isfinite(n3[~rows].float()).any(1).all()
    rows[70] = False
    dx3, d_o3, _ = backward(B, p, y3, stats3)
    assert torch.equal(dx3[rows], dx[rows]) and torch.equal(d_o3[rows], d_o[rows]) and not torch.isfinite(dx3[70].float()).any()


def test_no_rows(B):
    p = make(0, 64, "layer", "layer", True, "shared")
    forward(B, p)
    _, _, grads = backward(B, p, torch.empty_like(p["x"]), torch.empty(4, 0, device="cuda"))
    assert all(bool((v == 0).all()) for v in grads.values())
    _, _, grads = backward(B, p, torch.empty_like(p["x"]), torch.empty(4, 0, device="cuda"), accumulate=1, start=0.25)
    assert all(bool((v == 0.25).all()) for v in grads.values())


def test_gradients_by_differences(B):
    """The formulas above against central differences of their own forward pass, in float64."""
    torch.manual_seed(0)
    for post, pre, gate in (("rms", "layer", "shared tanh"), ("layer", "rms", "row sigmoid"), ("none", "rms", "row")):
        p = make(4, 16, post, pre, True, gate, seed=3)

        def loss(q):
            u = norm(post, q["o"].double(), q["post_g"], q["post_b"], 1e-5)[0]
            y = q["x"].double() + u * gate_of(q)[0] * q["scale"].double()
            return (norm(pre, y, q["pre_g"], q["pre_b"], 1e-5)[0] * p["dn"].double()).sum() + (y * p["dy"].double()).sum()

        wide = {k: v.double() if torch.is_tensor(v) else v for k, v in p.items()}
        u = norm(post, wide["o"], p["post_g"], p["post_b"], 1e-5)[0]
        want = formulas(wide, wide["x"] + u * gate_of(wide)[0] * wide["scale"])
        pairs = dict(dx="x", d_o="o", scale="scale", pre_g="pre_g", gate="gate")
        if post != "none":
            pairs["post_g"] = "post_g"
        if post == "layer":
            pairs["post_b"] = "post_b"
        if pre == "layer":
            pairs["pre_b"] = "pre_b"
        for name, leaf in pairs.items():
            direction, step = torch.randn_like(wide[leaf]), 1e-5
            ends = [loss(dict(wide, **{leaf: wide[leaf] + s * step * direction})) for s in (1, -1)]
            slope, formula = (ends[0] - ends[1]) / (2 * step), (want[name][0] * direction).sum()
            assert abs(slope - formula).item() <= 1e-6 * (1 + abs(formula).item()), (name, slope.item(), formula.item())
