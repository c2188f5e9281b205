"""Matrices whose elements or bytes pass 2^31 and 2^32: the last rows come out as they do by themselves (a row's bits do not depend on the rows beside it)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TAIL = 37


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    yield binding
    torch.cuda.empty_cache()


def rows(t, width, seed=0):
    """bf16 rows that differ, made by the block of a few million values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(t, width, dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 26) // width)
    for i in range(0, t, step):
        x[i:i + step].normal_(generator=g)
    return x


def same(got, want):
    assert torch.equal(got.contiguous().view(torch.uint8), want.contiguous().view(torch.uint8))


@pytest.mark.parametrize("t,width", [((1 << 29) + TAIL, 8), (70000, 65536)])      # more items than a launch takes, and rows behind 2^32 values
@pytest.mark.parametrize("format", [0, 1])
def test_keep8(B, t, width, format):
    x, blocks = rows(t, width), -(-width // 32)
    q, e = torch.empty(t, width, dtype=torch.uint8, device="cuda"), torch.empty(t, blocks, dtype=torch.uint8, device="cuda")
    B.mllm_op_keep8(x, q, e, t, width, format)
    parts = [slice(0, TAIL), slice(t - 3 * TAIL - 64, t)]                          # the last one across the second launch's first row
    for part in parts:
        n = part.stop - part.start
        q1, e1 = torch.empty_like(q[part]), torch.empty_like(e[part])
        B.mllm_op_keep8(x[part].clone(), q1, e1, n, width, format)
        same(q[part], q1), same(e[part], e1)
    y = x.fill_(7)
    B.mllm_op_keep8_load(q, e, y, t, width, format)
    for part in parts:
        n = part.stop - part.start
        y1 = torch.empty_like(y[part])
        B.mllm_op_keep8_load(q[part].clone(), e[part].clone(), y1, n, width, format)
        same(y[part], y1)


def test_activations(B):
    t, f = 70000, 32768
    pre, blocks = rows(t, 2 * f), f // 32
    a, q = torch.empty(t, f, dtype=torch.bfloat16, device="cuda"), torch.empty(t, 2 * f, dtype=torch.uint8, device="cuda")
    e = torch.empty(t, 2 * blocks, dtype=torch.uint8, device="cuda")
    B.mllm_op_act_fwd_keep8(2, pre, a, q, e, t, f, 0)
    last = slice(t - TAIL, t)
    a1, q1, e1 = torch.empty_like(a[last]), torch.empty_like(q[last]), torch.empty_like(e[last])
    B.mllm_op_act_fwd_keep8(2, pre[last].clone(), a1, q1, e1, TAIL, f, 0)
    same(a[last], a1), same(q[last], q1), same(e[last], e1)
    da, dpre, again = rows(t, f, 1), pre.fill_(7), a.fill_(7)
    B.mllm_op_act_bwd_keep8(2, da, q, e, dpre, t, f, 0, a=again)
    dpre1, again1 = torch.empty_like(dpre[last]), torch.empty_like(again[last])
    B.mllm_op_act_bwd_keep8(2, da[last].clone(), q1, e1, dpre1, TAIL, f, 0, a=again1)
    same(dpre[last], dpre1), same(again[last], again1)


@pytest.mark.parametrize("t,d", [(300000, 8192), (9000000, 256)])
def test_residual_norms(B, t, d):
    x, o = rows(t, d, 1), rows(t, d, 2)
    v = [rows(1, d, 10 + i)[0] for i in range(5)]
    gate = torch.linspace(-2, 2, t, device="cuda")

    def block(gate):
        return B.ResidualNorm(post_kind=0, post_g=v[0], post_b=v[1], post_eps=1e-5, scale=v[2], gate=gate, gate_per_row=True, gate_act=1, pre_kind=1,
                              pre_g=v[3], pre_eps=1e-5)

    n, stats = torch.empty_like(x), torch.empty(4, t, device="cuda")
    last = slice(t - TAIL, t)
    x1, o1, g1 = x[last].clone(), o[last].clone(), gate[last].clone()
    y1, n1, stats1 = torch.empty_like(x1), torch.empty_like(x1), torch.empty(4, TAIL, device="cuda")
    B.mllm_op_residual_norm_fwd(block(gate), x, o, x, n, stats, t, d)
    B.mllm_op_residual_norm_fwd(block(g1), x1, o1, y1, n1, stats1, TAIL, d)
    same(x[last], y1), same(n[last], n1), same(stats[:3, last], stats1[:3])
    dn1, dy = n1.clone(), rows(t, d, 3)
    dy1 = dy[last].clone()
    grads = [B.ResidualNormGrads(gate=torch.empty(m, device="cuda")) for m in (t, TAIL)]
    partial = torch.empty(B.mllm_op_residual_norm_bwd_partial_bytes(t, d) // 4, device="cuda")
    B.mllm_op_residual_norm_bwd(block(gate), n, dy, x, o, stats, n, dy, grads[0], partial, t, d)
    B.mllm_op_residual_norm_bwd(block(g1), dn1, dy1, y1, o1, stats1, dn1, dy1, grads[1], partial, TAIL, d)
    same(n[last], dn1), same(dy[last], dy1), same(grads[0].tensors[5][last], grads[1].tensors[5])


@pytest.mark.parametrize("t,heads,stride", [(600000, 32, 4096), ((1 << 20) + 5, 64, 8192)])      # the second a token a workgroup, and more of them than a dimension of the grid has
def test_rotation(B, t, heads, stride):
    x = rows(t, stride)
    pos = torch.randint(0, 1000, (3, t), device="cuda", dtype=torch.int32)
    table, axes = torch.empty(1000, 128, device="cuda"), B.section_axes([24, 20, 20], dealt=True)
    B.mllm_op_rope_freq_table(table, 1000, [10000.0 ** (-i / 64) for i in range(64)])
    last = slice(t - TAIL, t)
    x1, pos1 = x[last].clone(), pos[:, last].contiguous()
    B.mllm_op_rope_axes(x, x, pos, axes, table, 1000, t, heads, 128, stride, stride)
    B.mllm_op_rope_axes(x1, x1, pos1, axes, table, 1000, TAIL, heads, 128, stride, stride)
    same(x[last], x1)


def test_many_positions(B):
    """2^30 rows, values behind 2^31, in runs of two launches; what lies behind the rows stays."""
    t = 1 << 30
    cu = [0, 5, t - 3000] + [t - 3000 + 10 * i for i in range(1, 301)]
    grids = [(10, 1000, 100, 1000, 2), (t - 2995, 1, 2, 2, 1)]
    plan = B.PositionGrids(cu, grids)
    pos = torch.full((3, t + 64), -1, dtype=torch.int32, device="cuda")
    B.mllm_op_grid_positions(plan, pos, pos_stride=t + 64)
    assert bool((pos[:, t:] == -1).all())
    assert pos[:, :5].tolist() == [list(range(5))] * 3
    first, end = 10, 10 + 1000 * 100 * 1000
    assert pos[:, first - 1].tolist() == [4] * 3 and pos[:, first].tolist() == [5] * 3
    assert pos[:, end - 1].tolist() == [5 + 999 * 2, 5 + 99, 5 + 999] and pos[:, end].tolist() == [5 + 1999] * 3
    assert pos[:, t - 3001].tolist() == [5 + 1999 + t - 3001 - end] * 3
    assert pos[:, t - 3000:t - 2990].tolist() == [[0, 1, 2, 3, 4, 5, 5, 5, 5, 7], [0, 1, 2, 3, 4, 5, 5, 6, 6, 7], [0, 1, 2, 3, 4, 5, 6, 5, 6, 7]]
    assert bool((pos[:, t - 2990:t].view(3, 299, 10) == torch.arange(10, device="cuda", dtype=torch.int32)).all())
