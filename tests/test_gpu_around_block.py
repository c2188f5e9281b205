"""The operators around a layer's products as a layer uses them: a decoder layer with positions on three axes, norms on both sides of its blocks and
activations kept in 8 bits, forward and backward, against float64; the same calls captured into graphs and on other streams."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.gpu_util import TOL_GRAD, TOL_OUT, empty_bf16, host_f64, nmax_err, scratch  # noqa: E402

CU = [0, 90, 90, 91, 230]
GRIDS = [(10, 1, 5, 6, 1), (50, 3, 3, 4, 2), (100, 1, 8, 8, 1), (170, 2, 4, 5, 1)]
T, D, HQ, HKV, HD, F = 230, 256, 4, 2, 64, 512
AXES = [i % 3 for i in range(24)]                       # 48 of a head's 64 elements are rotated
FREQ = [10000.0 ** (-i / 24) for i in range(24)]
SHAPES = dict(rms=(D,), w_qkv=(D, (HQ + 2 * HKV) * HD), w_o=(HQ * HD, D), post1=(D,), pre2=(D,), gate=(1,), w_gu=(D, 2 * F), w_d=(F, D), post2=(D,),
              scale=(D,))
EPS = 1e-5


class Pack:
    cu_seqlens = np.array(CU, dtype=np.int32)
    mask_kind = np.ones(len(CU) - 1, dtype=np.uint8)


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


def parameters(seed):
    g = torch.Generator().manual_seed(seed)
    p = {}
    for name, shape in SHAPES.items():
        v = torch.randn(*shape, generator=g)
        v = v / shape[0] ** 0.5 if len(shape) == 2 else 0.7 + 0.2 * v
        p[name] = v if name == "gate" else v.bfloat16()
    return p, torch.randn(T, D, generator=g).bfloat16(), torch.randn(T, D, generator=g).bfloat16()


def layer(B, p, x, dy, format):
    """(y, gradients by name) through the entry points."""
    width = (HQ + 2 * HKV) * HD
    plan, axes = B.PositionGrids(CU, GRIDS), B.pair_axes(AXES)
    n_pos = B.mllm_grid_positions_count(plan)
    pos, table = torch.empty(3, T, dtype=torch.int32, device="cuda"), torch.empty(n_pos, 48, device="cuda")
    B.mllm_op_grid_positions(plan, pos)
    B.mllm_op_rope_freq_table(table, n_pos, FREQ)
    rope = lambda v, inverse: B.mllm_op_rope_axes(v, v, pos, axes, table, n_pos, T, HQ + HKV, HD, width, width, inverse=inverse)
    first = B.ResidualNorm(post_kind=B.NORM_RMS, post_g=p["post1"], post_eps=EPS, gate=p["gate"], gate_act=B.GATE_TANH, pre_kind=B.NORM_RMS,
                           pre_g=p["pre2"], pre_eps=EPS)
    second = B.ResidualNorm(post_kind=B.NORM_RMS, post_g=p["post2"], post_eps=EPS, scale=p["scale"])
    # forward
    n0, stats0 = empty_bf16(T, D), torch.empty(2, T, device="cuda")
    B.mllm_op_norm_fwd(1, x, p["rms"], None, n0, stats0, T, D, EPS)
    qkv = empty_bf16(T, width)
    B.mllm_op_gemm(n0, p["w_qkv"], qkv, T, width, D)
    rope(qkv, 0)
    q, k, v = qkv[:, :HQ * HD], qkv[:, HQ * HD:(HQ + HKV) * HD], qkv[:, (HQ + HKV) * HD:]
    o, lse = empty_bf16(T, HQ * HD), torch.empty(HQ, T, device="cuda")
    ws = scratch(B.mllm_op_attn_workspace_bytes(len(CU) - 1, T, HQ))
    B.mllm_op_attn_fwd(q, k, v, o, lse, Pack, HQ, HKV, HD, width, width, HQ * HD, ws)
    out1, y1, n1, stats1 = empty_bf16(T, D), empty_bf16(T, D), empty_bf16(T, D), torch.empty(4, T, device="cuda")
    B.mllm_op_gemm(o, p["w_o"], out1, T, D, HQ * HD)
    B.mllm_op_residual_norm_fwd(first, x, out1, y1, n1, stats1, T, D)
    gu, a = empty_bf16(T, 2 * F), empty_bf16(T, F)
    B.mllm_op_gemm(n1, p["w_gu"], gu, T, 2 * F, D)
    kept_n, kept_gu = (torch.empty(T, D, dtype=torch.uint8, device="cuda"), torch.empty(T, D // 32, dtype=torch.uint8, device="cuda")), (
        torch.empty(T, 2 * F, dtype=torch.uint8, device="cuda"), torch.empty(T, F // 16, dtype=torch.uint8, device="cuda"))
    B.mllm_op_act_fwd_keep8(2, gu, a, *kept_gu, T, F, format)
    B.mllm_op_keep8(n1, *kept_n, T, D, format)
    out2, y2, stats2 = empty_bf16(T, D), empty_bf16(T, D), torch.empty(4, T, device="cuda")
    B.mllm_op_gemm(a, p["w_d"], out2, T, D, F)
    B.mllm_op_residual_norm_fwd(second, y1, out2, y2, None, stats2, T, D)
    for gone in (n1, gu, a):
        gone.fill_(float("nan"))
    # backward
    grads = {name: torch.full(shape, float("nan"), device="cuda") for name, shape in SHAPES.items()}
    partial = scratch(B.mllm_op_residual_norm_bwd_partial_bytes(T, D))
    dy1, d_out2 = empty_bf16(T, D), empty_bf16(T, D)
    B.mllm_op_residual_norm_bwd(second, None, dy, y2, out2, stats2, dy1, d_out2, B.ResidualNormGrads(post_g=grads["post2"], scale=grads["scale"]), partial, T, D)
    da, dgu, dn1 = empty_bf16(T, F), empty_bf16(T, 2 * F), empty_bf16(T, D)
    B.mllm_op_act_bwd_keep8(2, None, *kept_gu, None, T, F, format, a=a)
    B.mllm_op_linear_bwd(d_out2, a, p["w_d"], da, grads["w_d"], T, F, D)
    B.mllm_op_act_bwd_keep8(2, da, *kept_gu, dgu, T, F, format)
    B.mllm_op_linear_bwd_keep8(dgu, *kept_n, p["w_gu"], dn1, grads["w_gu"], T, D, 2 * F, format, scratch(B.mllm_op_linear_bwd_keep8_workspace_bytes(T, D, 2 * F)))
    dx1, d_out1 = dy1, dn1                                             # in place
    B.mllm_op_residual_norm_bwd(first, dn1, dy1, y1, out1, stats1, dx1, d_out1,
                                B.ResidualNormGrads(post_g=grads["post1"], pre_g=grads["pre2"], gate=grads["gate"]), partial, T, D)
    d_o, dqkv, delta = empty_bf16(T, HQ * HD), empty_bf16(T, width), torch.empty(HQ, T, device="cuda")
    B.mllm_op_linear_bwd(d_out1, o, p["w_o"], d_o, grads["w_o"], T, HQ * HD, D)
    dq, dk, dv = dqkv[:, :HQ * HD], dqkv[:, HQ * HD:(HQ + HKV) * HD], dqkv[:, (HQ + HKV) * HD:]
    B.mllm_op_attn_bwd(q, k, v, o, lse, d_o, dq, dk, dv, delta, Pack, HQ, HKV, HD, width, width, HQ * HD, ws)
    rope(dqkv, 1)
    dn0, dx = empty_bf16(T, D), empty_bf16(T, D)
    B.mllm_op_linear_bwd(dqkv, n0, p["w_qkv"], dn0, grads["w_qkv"], T, D, width)
    B.mllm_op_norm_bwd(1, dn0, x, p["rms"], stats0, dx1, dx, grads["rms"], None, 0, scratch(B.mllm_op_norm_bwd_partial_bytes(T, D)), T, D)
    B.mllm_op_keep8_load(*kept_n, n1, T, D, format)
    B.mllm_op_keep8_load(*kept_gu, gu, T, 2 * F, format)      # halves of whole blocks: the matrix has the same
    return y2, dict(grads, x=dx), (n1, gu)


class Map(torch.autograd.Function):
    """v @ w whose weight gradient is taken from what was kept of v."""

    @staticmethod
    def forward(ctx, v, w, kept):
        ctx.save_for_backward(w, kept)
        return v @ w

    @staticmethod
    def backward(ctx, g):
        w, kept = ctx.saved_tensors
        return g @ w.T, kept.T @ g, None


class SwiGLU(torch.autograd.Function):
    """Its slopes are those at what was kept of its input."""

    @staticmethod
    def forward(ctx, v, kept):
        ctx.save_for_backward(kept)
        gate, up = v.chunk(2, 1)
        return gate * gate.sigmoid() * up

    @staticmethod
    def backward(ctx, g):
        gate, up = ctx.saved_tensors[0].chunk(2, 1)
        s = gate.sigmoid()
        return torch.cat([g * up * s * (1 + gate * (1 - s)), g * gate * s], 1), None


def positions():
    pos, at = np.zeros((3, T)), {g[0]: g[1:] for g in GRIDS}
    for first, end in zip(CU, CU[1:]):
        row, p = first, 0
        while row < end:
            if row in at:
                f, h, w, step = at[row]
                i = np.arange(f * h * w)
                pos[:, row:row + f * h * w] = np.stack([i // (h * w) * step, i // w % h, i % w]) + p
                row, p = row + f * h * w, p + max((f - 1) * step + 1, h, w)
            else:
                pos[:, row], row, p = p, row + 1, p + 1
    return torch.from_numpy(pos)


def definition(p, x, dy, kept_n, kept_gu):
    """The layer in float64 on the CPU, gradients by automatic differentiation, through what was kept where it is used."""
    a_kept = SwiGLU.apply(kept_gu, kept_gu)
    p = {k: v.double().requires_grad_() for k, v in p.items()}
    x = x.double().requires_grad_()
    rms = lambda v, g: v * (v.square().mean(1, keepdim=True) + EPS).rsqrt() * g
    angle = positions()[AXES].T * torch.tensor(FREQ, dtype=torch.float64)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    qkv = (rms(x, p["rms"]) @ p["w_qkv"]).view(T, -1, HD)
    head = qkv[:, :HQ + HKV]
    a, b = head[..., :24], head[..., 24:48]
    head = torch.cat([a * cos - b * sin, b * cos + a * sin, head[..., 48:]], -1)
    q, k, v = head[:, :HQ], head[:, HQ:].repeat_interleave(HQ // HKV, 1), qkv[:, HQ + HKV:].repeat_interleave(HQ // HKV, 1)
    parts = []
    for first, end in zip(CU, CU[1:]):
        s = torch.einsum("ihd,jhd->hij", q[first:end], k[first:end]) / HD ** 0.5
        s = s.masked_fill(torch.ones(end - first, end - first).triu(1).bool(), -float("inf"))
        parts.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), v[first:end]))
    o = torch.cat(parts).reshape(T, HQ * HD)
    y1 = x + rms(o @ p["w_o"], p["post1"]) * torch.tanh(p["gate"])
    gu = Map.apply(rms(y1, p["pre2"]), p["w_gu"], kept_n)
    y2 = y1 + rms(Map.apply(SwiGLU.apply(gu, kept_gu), p["w_d"], a_kept), p["post2"]) * p["scale"]
    y2.backward(dy.double())
    return y2.detach(), dict({k: v.grad for k, v in p.items()}, x=x.grad)


@pytest.mark.parametrize("format", ["KEEP_INT8", "KEEP_E4M3"])
def test_a_layer(B, format):
    """The stage tests' tolerances, against gradients taken through the values that were kept; those are the format's nearest to the layer's own."""
    p, x, dy = parameters(0)
    dev = {k: v.cuda() for k, v in p.items()}
    y, grads, kept = layer(B, dev, x.cuda(), dy.cuda(), getattr(B, format))
    kept_n, kept_gu = (v.double().cpu() for v in kept)
    want_y, want = definition(p, x, dy, kept_n, kept_gu)
    assert nmax_err(host_f64(y), want_y.numpy()) <= TOL_OUT
    errors = {k: nmax_err(host_f64(grads[k]), want[k].numpy()) for k in want}
    assert all(v <= TOL_GRAD for v in errors.values()), errors
    again = layer(B, dev, x.cuda(), dy.cuda(), getattr(B, format))
    assert torch.equal(y, again[0]) and all(torch.equal(grads[k], again[1][k]) for k in grads)


class Calls:
    """One of each call on buffers of its own, t rows of d columns; begin() refills the inputs."""

    def __init__(self, B, t=300, d=640, seed=0):
        self.B, self.t, self.d, self.seed = B, t, d, seed
        bf = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
        by = lambda *shape: torch.empty(*shape, dtype=torch.uint8, device="cuda")
        fp = lambda *shape: torch.empty(*shape, device="cuda")
        self.x, self.o, self.dn, self.dy, self.w = bf(t, d), bf(t, d), bf(t, d), bf(t, d), bf(d, 256)
        self.dz, self.gain, self.gate = bf(t, 256), bf(d), fp(1)
        self.plan, self.axes = B.PositionGrids([0, t // 2, t], [(3, 2, 2, 5, 1), (t // 2 + 7, 1, 3, 4, 1)]), B.section_axes([8, 12, 12])
        self.pos, self.table = torch.empty(3, t, dtype=torch.int32, device="cuda"), fp(400, 64)
        self.y, self.n, self.stats, self.turned = bf(t, d), bf(t, d), fp(4, t), bf(t, d)
        self.dx, self.d_o, self.g = bf(t, d), bf(t, d), {k: fp(d) for k in ("post_g", "pre_g")}
        self.g["gate"] = fp(1)
        self.partial = by(max(256, B.mllm_op_residual_norm_bwd_partial_bytes(t, d)))
        self.kept, self.loaded = (by(t, d), by(t, d // 32)), bf(t, d)
        self.a, self.kept_pre, self.dpre, self.again = bf(t, d // 2), (by(t, d), by(t, d // 32)), bf(t, d), bf(t, d // 2)
        self.dlin, self.dw, self.ws = bf(t, d), fp(d, 256), by(max(256, B.mllm_op_linear_bwd_keep8_workspace_bytes(t, d, 256)))
        self.block = B.ResidualNorm(post_kind=B.NORM_RMS, post_g=self.gain, post_eps=EPS, gate=self.gate, gate_act=B.GATE_TANH, pre_kind=B.NORM_RMS,
                                    pre_g=self.gain, pre_eps=EPS)
        self.grads = B.ResidualNormGrads(**self.g)

    def begin(self, n):
        g = torch.Generator(device="cuda").manual_seed(1000 * self.seed + n)
        for v in (self.x, self.o, self.dn, self.dy, self.w, self.dz, self.gain, self.gate):
            v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
        for v in self.outputs():
            v.view(torch.uint8).fill_(0xFF)

    def outputs(self):
        return [self.pos, self.table, self.y, self.n, self.stats, self.turned, self.dx, self.d_o, *self.g.values(), *self.kept, self.loaded, self.a,
                *self.kept_pre, self.dpre, self.again, self.dlin, self.dw]

    def run(self, stream=None):
        B, t, d = self.B, self.t, self.d
        B.mllm_op_grid_positions(self.plan, self.pos, stream=stream)
        B.mllm_op_rope_freq_table(self.table, 400, [100.0 ** (-i / 32) for i in range(32)], stream=stream)
        B.mllm_op_rope_axes(self.x, self.turned, self.pos, self.axes, self.table, 400, t, d // 64, 64, d, d, stream=stream)
        B.mllm_op_residual_norm_fwd(self.block, self.turned, self.o, self.y, self.n, self.stats, t, d, stream=stream)
        B.mllm_op_residual_norm_bwd(self.block, self.dn, self.dy, self.y, self.o, self.stats, self.dx, self.d_o, self.grads, self.partial, t, d, stream=stream)
        B.mllm_op_keep8(self.n, *self.kept, t, d, B.KEEP_INT8, stream=stream)
        B.mllm_op_keep8_load(*self.kept, self.loaded, t, d, B.KEEP_INT8, stream=stream)
        B.mllm_op_act_fwd_keep8(2, self.y, self.a, *self.kept_pre, t, d // 2, B.KEEP_E4M3, stream=stream)
        B.mllm_op_act_bwd_keep8(2, self.a, *self.kept_pre, self.dpre, t, d // 2, B.KEEP_E4M3, a=self.again, stream=stream)
        B.mllm_op_linear_bwd_keep8(self.dz, *self.kept, self.w, self.dlin, self.dw, t, d, 256, B.KEEP_INT8, self.ws, stream=stream)

    def eager(self, n):
        self.begin(n)
        self.run()
        torch.cuda.synchronize()
        return [v.clone() for v in self.outputs()]

    def same(self, want):
        return all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(self.outputs(), want))


def test_captured_and_replayed(B):
    """Two graphs of the same calls on buffers of their own, with eager calls between the replays."""
    calls = [Calls(B, seed=0), Calls(B, t=77, d=1280, seed=1)]
    want = [[c.eager(n) for n in range(3)] for c in calls]
    graphs = []
    for c in calls:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            c.run()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        graphs.append(graph)
    other = Calls(B, t=50, d=640, seed=2)
    for n in (0, 1, 2, 1, 0):
        for c, graph, w in zip(calls, graphs, want):
            c.begin(n)
            graph.replay()
            first = other.eager(n)
            graph.replay()
            torch.cuda.synchronize()
            assert c.same(w[n]) and other.same(first)


def test_two_streams(B):
    """The same calls at once on two streams, on buffers of their own."""
    calls = [Calls(B, seed=3), Calls(B, seed=4)]
    want = [c.eager(0) for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for c in calls:
        c.begin(0)
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            c.run(stream=s)
    torch.cuda.synchronize()
    assert all(c.same(w) for c, w in zip(calls, want))
    with torch.cuda.stream(streams[0]):           # the current stream is taken where none is named
        calls[0].begin(0)
        calls[0].run()
    torch.cuda.synchronize()
    assert calls[0].same(want[0])


def test_nothing_is_allocated(B):
    c = Calls(B)
    c.eager(0)
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    c.run()
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    torch.cuda.synchronize()
