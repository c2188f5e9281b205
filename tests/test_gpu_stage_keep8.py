"""Stages whose layers keep what the backward pass reads in 8 bits, against the fp64 oracle with the values that the stage kept.

The forward pass and what it keeps are checked by themselves: a kept value is the format's nearest to the oracle's activation, or beside it where the
library's bf16 roundings on the way carry it over a border.  The gradients are then held to the stages' tolerances against those of the oracle at the very
values that were kept, read from the saved buffer."""
import dataclasses

import numpy as np
import pytest

import workloads as W
from oracle import stage_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.gpu_util import GpuStage, compare, dev_bf16, scratch  # noqa: E402

NAMES = {1: "int8", 2: "e4m3"}


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    binding.lib()
    return binding


def keeping(layers, keep8):
    return [l if l.kind == W.LAYER_PROJECTOR else dataclasses.replace(l, keep8=keep8) for l in layers]


class Stage(GpuStage):
    """A run that hands out what was kept: per layer (n1, n2, pre) in float64, None where the layer keeps bf16."""

    def run(self, wl, accumulate=0, dparams=None):
        B = self.B
        params = [dev_bf16(p) for p in wl.params]
        x_img = dev_bf16(wl.x_img) if wl.x_img is not None else None
        x_seq = dev_bf16(wl.x_seq) if wl.x_seq is not None else None
        dy = dev_bf16(wl.dy)
        sb, wb = B.mllm_stage_sizes(self.h, wl.batch)
        saved, ws = scratch(sb), scratch(wb)
        saved.fill_(0xFF), ws.fill_(0xFF)
        y = torch.empty_like(dy)
        B.mllm_stage_fwd(self.h, wl.batch, params, x_img, x_seq, y, saved, ws)
        torch.cuda.synchronize()
        self.kept = self.decode(wl.batch, saved)
        if dparams is None:
            dparams = [torch.full((r, c), float("nan"), device="cuda") for _, _, r, c in self.infos]
        dx_img, dx_seq = torch.empty_like(x_img) if x_img is not None else None, torch.empty_like(x_seq) if x_seq is not None else None
        ws.fill_(0xFF)
        B.mllm_stage_bwd(self.h, wl.batch, params, dy, saved, dx_img, dx_seq, dparams, accumulate, ws)
        torch.cuda.synchronize()
        return y, dx_img, dx_seq, dparams

    def decode(self, batch, saved):
        """saved holds every layer's tensors one behind the other, each on 256 bytes."""
        at, out = 0, []

        def take(nbytes):
            nonlocal at
            part = saved[at:at + nbytes]
            at += -(-nbytes // 256) * 256
            return part

        for L in self.layers:
            if L.kind == W.LAYER_PROJECTOR:
                rows = len(batch.img_to_seq_row)
                take(batch.img.total_tokens * L.d_model * 2)
                if L.pool > 1:
                    take(rows * L.d_model * 2)
                if L.d_ff:
                    take(rows * L.d_ff * 2), take(rows * L.d_ff * 2)
                out.append(None)
                continue
            vit = L.kind == W.LAYER_VIT
            T, d, nq = (batch.img if vit else batch.seq).total_tokens, L.d_model, (L.n_q_heads + 2 * L.n_kv_heads) * L.head_dim
            fup, size = (1 if vit else 2) * L.d_ff, 1 if L.keep8 else 2
            take(T * d * 2), take(T * 8)
            n1 = take(T * d * size)
            take(T * nq * 2)
            if L.qk_norm:
                take(T * nq * 2)
                if L.qk_norm == 1:
                    take(T * 8), take(T * 8)
            take(T * d * 2), take(T * L.n_q_heads * 4), take(T * d * 2), take(T * 8)
            n2, pre = take(T * d * size), take(T * fup * size)
            if not L.keep8:
                take(T * L.d_ff * 2)
                out.append(None)
                continue
            exps = [take(T * width // 32) for width in (d, d, fup)]
            parts = []
            for q, e, width in zip((n1, n2, pre), exps, (d, d, fup)):
                v = torch.empty(T, width, dtype=torch.bfloat16, device="cuda")
                self.B.mllm_op_keep8_load(q, e, v, T, width, L.keep8 - 1)
                parts.append(v.double().cpu().numpy())
            out.append(parts)
        assert at <= saved.numel() < at + 256 or saved.numel() == at
        return out


def beside(got, exact, name):
    """Within the format's rounding of the block (int8: half of 1/64 of its largest value; e4m3: 1/16 of the value) and the activation's own error, 2e-2 of the largest."""
    t, width = exact.shape
    block = np.abs(exact).reshape(t, -1, 32).max(2).repeat(32, 1)
    slack = 2e-2 * np.abs(exact).max()
    bound = (block / 127 if name == "int8" else np.abs(exact) / 16 + block * 2.0 ** -17) + 1.1 * slack
    assert (np.abs(got - exact) <= bound).all()


def oracle(wl, layers, kept_by_layer):
    """Forward as ever; the backward pass reads the kept values, and the activation that they give."""
    y, caches = O.stage_fwd(layers, wl.params, wl.batch, wl.x_img, wl.x_seq)
    for L, c, k in zip(layers, caches, kept_by_layer):
        if k is None:
            assert not L.keep8
            continue
        pre = c["h"] if L.kind == W.LAYER_VIT else np.concatenate([c["gate"], c["up"]], 1)
        for got, exact in zip(k, (c["n1"], c["n2"], pre)):
            beside(got, exact, NAMES[L.keep8])
        c["n1"], c["n2"] = k[0], k[1]
        if L.kind == W.LAYER_VIT:
            c["h"] = k[2]
            c["a"] = O._act_fwd(L.act, c["h"])
        else:
            c["gate"], c["up"] = k[2][:, :L.d_ff], k[2][:, L.d_ff:]
            c["a"] = O.swiglu_fwd(c["gate"], c["up"])
    return (y, *O.stage_bwd(layers, wl.params, wl.batch, caches, wl.dy.astype(np.float64)))


CASES = {
    "tiny": lambda: W.workload_tiny(1),
    "variants": lambda: W.workload_tiny_variant(2),
    "qk_norm": lambda: W.workload_tiny_qknorm(3),
    "head_norm": lambda: W.workload_tiny_headnorm(4),
    "pooled": lambda: W.workload_tiny_pooled(5),
    "encoder": lambda: W.make_workload("encoder", [W.vit_layer(256, 4, 64, 448, act=W.ACT_GELU_TANH)] * 2,
                                       W.Batch(W.make_pack([130, 0, 1, 77], W.MASK_BIDIR), None, None, []), 6),
    "decoder_bias": lambda: W.make_workload("decoder_bias", [W.decoder_layer(512, 4, 2, 128, 320, 10000.0, qkv_bias=1)] * 2,
                                            W.Batch(None, W.make_pack([260, 1, 0, 3], W.MASK_CAUSAL), None, []), 7),
    # the products with the activation and its gradient in their epilogues: 200 tiles of 256 x 256
    "fused": lambda: W.make_workload("fused", [W.decoder_layer(128, 2, 1, 64, 4096, 10000.0)],
                                     W.Batch(None, W.make_pack([100] * 33 + [28], W.MASK_CAUSAL), None, []), 8),
}


@pytest.mark.parametrize("keep8", [1, 2])
@pytest.mark.parametrize("case", sorted(CASES))
def test_against_the_oracle(B, case, keep8):
    wl = CASES[case]()
    layers = keeping(wl.layers, keep8)
    stage = Stage(B, layers)
    try:
        got = stage.run(wl)
        compare(stage, wl, got, oracle(wl, layers, stage.kept))
    finally:
        stage.close()


@pytest.mark.parametrize("keep8", [1, 2])
def test_some_layers_and_accumulation(B, keep8):
    """One of two decoder layers, two microbatches added up, bit for bit the same a second time."""
    wl = W.workload_tiny_headnorm(9)
    layers = list(wl.layers)
    layers[2] = dataclasses.replace(layers[2], keep8=keep8)
    stage = Stage(B, layers)
    try:
        first = stage.run(wl)
        want = oracle(wl, layers, stage.kept)
        compare(stage, wl, first, want)
        again = stage.run(wl)
        assert all(torch.equal(a, b) for a, b in zip(first[3], again[3])) and torch.equal(first[0], again[0])
        y, dx_img, dx_seq, grads = stage.run(wl, accumulate=1, dparams=[g.clone() for g in first[3]])
        compare(stage, wl, (y, dx_img, dx_seq, grads), want[:3] + ([2 * g for g in want[3]],))
    finally:
        stage.close()


def test_forward_is_the_same(B):
    """The kept values are for the backward pass alone: where the activation is formed in the product's epilogue the output has the same bits."""
    wl = CASES["fused"]()
    outs = []
    for keep8 in (0, 1, 2):
        stage = Stage(B, keeping(wl.layers, keep8))
        outs.append(stage.run(wl)[0])
        stage.close()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_sizes(B):
    """A decoder layer of the 8B shape keeps 54 % of what it keeps otherwise."""
    batch = W.Batch(None, W.make_pack([1000, 24], W.MASK_CAUSAL), None, [])
    T, d, f = 1024, 4096, 14336
    sizes = []
    for keep8 in (0, 1, 2):
        h = B.mllm_stage_create([dataclasses.replace(W.dec8b_layer(), keep8=keep8)])
        sizes.append(B.mllm_stage_sizes(h, batch))
        B.mllm_stage_destroy(h)
    less = T * (2 * d + 2 * f) + T * f * 2 - T * (2 * d + 2 * f) // 32
    assert sizes[0][0] - sizes[1][0] == less and sizes[1] == sizes[2]
    assert sizes[1][0] <= 0.55 * sizes[0][0]
    # the workspace has one layer's activations in bf16
    assert 0 <= sizes[1][1] - sizes[0][1] - (T * d + T * 2 * f + T * f) * 2 <= 4096


def test_buffers_of_a_longer_microbatch(B):
    """saved and workspace sized for a longer one, and full of NaN, serve a shorter one with the same results."""
    wl = W.workload_tiny(11)
    layers = keeping(wl.layers, 1)
    long = W.batch_from_samples([(1, 300), (1, 200), (2, 10)], img_tokens=64)
    stage = Stage(B, layers)
    try:
        want = stage.run(wl)
        sb, wb = B.mllm_stage_sizes(stage.h, long)
        saved, ws = scratch(sb), scratch(wb)
        saved.fill_(0xFF), ws.fill_(0xFF)
        params = [dev_bf16(p) for p in wl.params]
        x_img, x_seq, dy = dev_bf16(wl.x_img), dev_bf16(wl.x_seq), dev_bf16(wl.dy)
        y, dx_img, dx_seq = torch.empty_like(dy), torch.empty_like(x_img), torch.empty_like(x_seq)
        grads = [torch.empty_like(g) for g in want[3]]
        B.mllm_stage_fwd(stage.h, wl.batch, params, x_img, x_seq, y, saved, ws)
        ws.fill_(0xFF)
        B.mllm_stage_bwd(stage.h, wl.batch, params, dy, saved, dx_img, dx_seq, grads, 0, ws)
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx_img, want[1]) and torch.equal(dx_seq, want[2]) and all(torch.equal(a, b) for a, b in zip(grads, want[3]))
    finally:
        stage.close()
