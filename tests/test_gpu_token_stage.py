"""Stages with per-head QK normalisation, and a whole training step around one: token rows, stage, head, loss, and back to the gradient
of the token table, against the same chain in float64.  Tolerances are the stage's: normalised max error 2e-2 on outputs, 3e-2 on
gradients."""
import numpy as np
import pytest

import workloads as W
from oracle import stage_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.gpu_util import GpuStage, TOL_GRAD, TOL_OUT, compare, dev_bf16, host_f64, nmax_err, oracle_run, scratch  # noqa: E402


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_tiny_headnorm_stage_matches_oracle(B, seed):
    wl = W.workload_tiny_headnorm(seed)
    st = GpuStage(B, wl.layers)
    try:
        compare(st, wl, st.run(wl), oracle_run(wl))
    finally:
        st.close()


@pytest.mark.parametrize("case", ["vit", "vit_128", "dec_gqa_128", "dec_bias_two_layers", "dec_mqa_mixed"])
def test_head_norm_layer_shapes(B, case):
    n = W.QK_NORM_HEADS
    if case == "vit":
        layers, batch = [W.vit_layer(1280, 20, 64, 512, qk_norm=n)], W.Batch(W.make_pack([130, 0, 1, 77], W.MASK_BIDIR), None, None, [])
    elif case == "vit_128":
        layers, batch = [W.vit_layer(384, 3, 128, 256, qk_norm=n)] * 2, W.Batch(W.make_pack([300, 1, 5], W.MASK_BIDIR), None, None, [])
    elif case == "dec_gqa_128":
        layers, batch = [W.decoder_layer(2048, 16, 2, 128, 512, 500000.0, qk_norm=n)], W.Batch(None, W.make_pack([150, 1, 0, 93], W.MASK_CAUSAL), None, [])
    elif case == "dec_bias_two_layers":
        layers = [W.decoder_layer(512, 8, 1, 64, 256, 10000.0, qkv_bias=1, qk_norm=n), W.decoder_layer(512, 8, 8, 64, 320, 10000.0, qk_norm=n)]
        batch = W.Batch(None, W.make_pack([260, 3], W.MASK_CAUSAL), None, [])
    else:                                                    # every kind of layer in one stage
        layers = [W.decoder_layer(512, 8, 1, 64, 256, 10000.0, qk_norm=q) for q in (n, 0, 1, n)]
        batch = W.Batch(None, W.make_pack([5, 700], W.MASK_CAUSAL), None, [])
    wl = W.make_workload("layer", layers, batch, 43)
    st = GpuStage(B, layers)
    try:
        compare(st, wl, st.run(wl), oracle_run(wl))
    finally:
        st.close()


def test_head_norm_of_no_tokens(B):
    layers, batch = [W.decoder_layer(256, 4, 2, 64, 256, 10000.0, qk_norm=W.QK_NORM_HEADS)], W.Batch(None, W.make_pack([0, 0], W.MASK_CAUSAL), None, [])
    wl = W.make_workload("layer", layers, batch, 43)
    st = GpuStage(B, layers)
    try:
        params, row = [dev_bf16(p) for p in wl.params], torch.full((1, 256), 7.0, dtype=torch.bfloat16, device="cuda")
        dparams = [torch.full((r, c), float("nan"), device="cuda") for _, _, r, c in st.infos]
        sb, wb = B.mllm_stage_sizes(st.h, batch)
        saved, ws = scratch(sb), scratch(wb)
        B.mllm_stage_fwd(st.h, batch, params, None, row, row, saved, ws)
        B.mllm_stage_bwd(st.h, batch, params, row, saved, None, row, dparams, 0, ws)
        assert bool((row == 7.0).all()) and all(not bool(g.any()) for g in dparams)
    finally:
        st.close()


def test_head_norm_gradients_accumulate_and_packing_changes_nothing(B):
    wl = W.workload_tiny_headnorm(3)
    st = GpuStage(B, wl.layers)
    try:
        a = st.run(wl)
        acc = [torch.zeros_like(g) for g in a[3]]
        st.run(wl, accumulate=1, dparams=acc)
        st.run(wl, accumulate=1, dparams=acc)
        for g2, g1 in zip(acc, a[3]):
            assert nmax_err(host_f64(g2), 2 * host_f64(g1)) < 1e-5
        b = st.run(wl)                                       # the same bits again
        assert torch.equal(a[0], b[0]) and all(torch.equal(x, y) for x, y in zip(a[3], b[3]))
    finally:
        st.close()


def test_training_step_around_a_stage(B):
    """Two microbatches of one optimizer step, the second one accumulating every gradient."""
    layers = W.tiny_headnorm_layers()
    d, vocab, cols, emb_scale, eps = 256, 1003, 1008, 4.0, 1e-5
    rng = np.random.default_rng(5)
    table = W.bf16_round(rng.standard_normal((vocab, d)) * 0.1)
    gain = W.bf16_round(1 + 0.1 * rng.standard_normal((1, d)))
    head = np.zeros((d, cols), np.float32)                   # columns behind the vocabulary are padding
    head[:, :vocab] = W.bf16_round(rng.standard_normal((d, vocab)) * 0.05)
    dt_table, dt_gain, dt_head = dev_bf16(table), dev_bf16(gain), dev_bf16(head)
    st = GpuStage(B, layers)
    dparams = [torch.full((r, c), float("nan"), device="cuda") for _, _, r, c in st.infos]
    dtable, dgain, dhead = (torch.full(s, float("nan"), device="cuda") for s in ((vocab, d), (1, d), (d, cols)))
    want = None
    losses = []
    try:
        for mb, seed in enumerate((21, 22)):
            wl = W.workload_tiny_headnorm(seed)
            if mb == 0:
                params = wl.params
            T = wl.batch.seq.total_tokens
            ids = rng.integers(0, vocab, T).astype(np.int32)
            ids[::3] = ids[0]                                # a frequent token
            ids[wl.batch.img_to_seq_row] = -1
            targets = np.full(T, -100, np.int32)
            for a, b in zip(wl.batch.seq.cu_seqlens[:-1], wl.batch.seq.cu_seqlens[1:]):
                targets[a:b - 1] = ids[a + 1:b]              # the next token, where there is one
            weight = 1.0 / max(1, int((targets >= 0).sum()))

            # the library
            dev = lambda a: torch.from_numpy(a).cuda()
            t_ids, t_targets, t_params, x_img = dev(ids), dev(targets), [dev_bf16(p) for p in params], dev_bf16(wl.x_img)
            new = lambda *s, dtype=torch.bfloat16: torch.full(s, float("nan"), dtype=dtype, device="cuda")
            x, y, n, dn, dy, dx = (new(T, d) for _ in range(6))
            logits, stats, loss, dlogits = new(T, cols, dtype=torch.float32), new(2, T, dtype=torch.float32), new(T, dtype=torch.float32), new(T, cols)
            sb, wb = B.mllm_stage_sizes(st.h, wl.batch)
            saved, ws = scratch(sb), scratch(wb)
            B.mllm_op_embed_fwd(dt_table, t_ids, x, T, vocab, d, scale=emb_scale)
            B.mllm_stage_fwd(st.h, wl.batch, t_params, x_img, x, y, saved, ws)
            B.mllm_op_norm_fwd(1, y, dt_gain, None, n, stats, T, d, eps)
            B.mllm_op_gemm(n, dt_head, logits, T, cols, d, out_fp32=1)
            B.mllm_op_xent(logits, t_targets, loss, dlogits, T, vocab, cols, scale=weight, logits_fp32=1)
            acc = int(mb > 0)
            _, need = B.mllm_linear_bwd_form(T, d, cols)
            B.mllm_op_linear_bwd(dlogits, n, dt_head, dn, dhead, T, d, cols, accumulate=acc, workspace=scratch(need), scratch_bytes=need)
            B.mllm_op_norm_bwd(1, dn, y, dt_gain, stats, None, dy, dgain, None, acc, scratch(B.mllm_op_norm_bwd_partial_bytes(T, d)), T, d)
            B.mllm_stage_bwd(st.h, wl.batch, t_params, dy, saved, None, dx, dparams, acc, ws)
            B.mllm_op_embed_bwd(dx, t_ids, dtable, T, vocab, d, scratch(B.mllm_op_embed_bwd_workspace_bytes(T, vocab, d)), scale=emb_scale, accumulate=acc)
            torch.cuda.synchronize()

            # the definition in float64
            x64 = np.where(ids[:, None] >= 0, emb_scale * table[np.maximum(ids, 0)].astype(np.float64), 0.0)
            y64, caches = O.stage_fwd(layers, params, wl.batch, wl.x_img, x64)
            n64, c = O.rmsnorm_fwd(y64, gain.astype(np.float64), eps)
            z = n64 @ head.astype(np.float64)[:, :vocab]
            m = z.max(axis=1, keepdims=True)
            e = np.exp(z - m)
            s = e.sum(axis=1, keepdims=True)
            there, at = targets >= 0, np.maximum(targets, 0)
            loss64 = np.where(there, (np.log(s) + m)[:, 0] - z[np.arange(T), at], 0.0)
            g = e / s
            g[np.arange(T), at] -= 1.0
            g = np.where(there[:, None], g * weight, 0.0)
            dn64 = g @ head.astype(np.float64)[:, :vocab].T
            dy64, dgain64 = O.rmsnorm_bwd(dn64, c, gain.astype(np.float64))
            _, dx64, dp64 = O.stage_bwd(layers, params, wl.batch, caches, dy64)
            dtable64, dhead64 = np.zeros((vocab, d)), np.zeros((d, cols))
            np.add.at(dtable64, ids[ids >= 0], emb_scale * dx64[ids >= 0])
            dhead64[:, :vocab] = n64.T @ g
            losses.append((nmax_err(host_f64(y), y64), nmax_err(host_f64(loss), loss64)))
            now = [dtable64, dgain64, dhead64] + dp64
            want = now if want is None else [a + b for a, b in zip(want, now)]
    finally:
        st.close()
    assert max(max(v) for v in losses) <= TOL_OUT, losses
    errs = [nmax_err(host_f64(g), w) for g, w in zip([dtable, dgain, dhead] + dparams, want)]
    assert max(errs) <= TOL_GRAD, errs
    assert not bool(dhead[:, vocab:].any())
