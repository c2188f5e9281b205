"""The oracle's per-head QK normalisation against PyTorch CPU autograd in float64, and its parameter table against the library's."""
import os

import numpy as np
import pytest

import workloads as W
from oracle import stage_oracle as O


@pytest.fixture(scope="module")
def B():
    from paper_2603_25120_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_25120_amd import build
        build.build()
    binding.lib()
    return binding


def test_gains_of_a_head(B):
    layers = W.tiny_headnorm_layers() + [W.decoder_layer(256, 4, 2, 64, 512, 1e4, qkv_bias=1, qk_norm=W.QK_NORM_HEADS)]
    h = B.mllm_stage_create(layers)
    got = [B.mllm_stage_param_info(h, i) for i in range(B.mllm_stage_param_count(h))]
    B.mllm_stage_destroy(h)
    assert got == [(n, li, r, c) for li, L in enumerate(layers) for n, r, c in W.param_specs(L)]
    assert [g[2:] for g in got if g[0].startswith("qkn_")] == [(1, 64)] * 8


@pytest.mark.parametrize("value", [2, 4, 5, 7, -1])
def test_other_flags_are_refused(B, value):
    for layer in (W.vit_layer(192, 3, 64, 768, qk_norm=value), W.decoder_layer(256, 4, 2, 64, 512, 1e4, qk_norm=value)):
        with pytest.raises(B.MllmError) as e:
            B.mllm_stage_create([layer])
        assert e.value.status == 2


def test_no_statistics_are_kept(B):
    """A second [T, nq] matrix in `saved` and one more in the workspace, nothing else."""
    import dataclasses
    base = W.decoder_layer(512, 8, 2, 64, 1024, 10000.0)
    batch = W.Batch(None, W.make_pack([300, 212], W.MASK_CAUSAL), None, [])
    sizes = []
    for layer in (base, dataclasses.replace(base, qk_norm=W.QK_NORM_HEADS)):
        h = B.mllm_stage_create([layer, layer])
        sizes.append(B.mllm_stage_sizes(h, batch))
        B.mllm_stage_destroy(h)
    nbytes = 512 * (8 + 2 * 2) * 64 * 2
    assert sizes[1][0] - sizes[0][0] == 2 * nbytes and sizes[1][1] - sizes[0][1] == nbytes


def test_stage_against_torch_cpu_autograd():
    torch = pytest.importorskip("torch")
    F = torch.nn.functional
    wl = W.workload_tiny_headnorm(7)
    t64 = lambda a: torch.tensor(np.asarray(a, dtype=np.float64), requires_grad=True)
    P = [t64(p) for p in wl.params]
    x_img, x_seq = t64(wl.x_img), t64(wl.x_seq)
    vit, _, dec, _ = wl.layers
    heads = lambda z, h: z.reshape(z.shape[0], h, 64).permute(1, 0, 2)
    outs, cu = [], wl.batch.seq.cu_seqlens
    for s, _ in enumerate(wl.batch.samples):
        xi = x_img[64 * s:64 * (s + 1)]
        g1, b1, wqkv, bqkv, wo, bo, g2, b2, w1, bb1, w2, bb2, gq, gk = P[:14]
        qkv = F.layer_norm(xi, (192,), g1[0], b1[0], vit.norm_eps) @ wqkv + bqkv
        q = F.rms_norm(heads(qkv[:, :192], 3), (64,), gq[0], vit.norm_eps)
        k = F.rms_norm(heads(qkv[:, 192:384], 3), (64,), gk[0], vit.norm_eps)
        o = F.scaled_dot_product_attention(q, k, heads(qkv[:, 384:], 3))
        x1 = xi + o.permute(1, 0, 2).reshape(64, 192) @ wo + bo
        yv = x1 + F.gelu(F.layer_norm(x1, (192,), g2[0], b2[0], vit.norm_eps) @ w1 + bb1) @ w2 + bb2
        x = torch.cat([yv @ P[14] + P[15], x_seq[cu[s] + 64:cu[s + 1]]], dim=0)
        L = x.shape[0]
        ang = torch.arange(L, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, 32, dtype=torch.float64) * 2 / 64)
        cos, sin = torch.cos(ang), torch.sin(ang)
        rot = lambda z: torch.cat([z[..., :32] * cos - z[..., 32:] * sin, z[..., 32:] * cos + z[..., :32] * sin], dim=-1)
        for first in (16, 24):
            r1, wqkv, wo, r2, wgu, wd, gq, gk = P[first:first + 8]
            qkv = F.rms_norm(x, (256,), r1[0], dec.norm_eps) @ wqkv
            q = rot(F.rms_norm(heads(qkv[:, :256], 4), (64,), gq[0], dec.norm_eps))
            k = rot(F.rms_norm(heads(qkv[:, 256:384], 2), (64,), gk[0], dec.norm_eps))
            o = F.scaled_dot_product_attention(q, k.repeat_interleave(2, dim=0), heads(qkv[:, 384:], 2).repeat_interleave(2, dim=0), is_causal=True)
            x1 = x + o.permute(1, 0, 2).reshape(L, 256) @ wo
            gu = F.rms_norm(x1, (256,), r2[0], dec.norm_eps) @ wgu
            x = x1 + (F.silu(gu[:, :1024]) * gu[:, 1024:]) @ wd
        outs.append(x)
    y_t = torch.cat(outs, dim=0)
    y_t.backward(torch.tensor(wl.dy.astype(np.float64)))
    y, caches = O.stage_fwd(wl.layers, wl.params, wl.batch, wl.x_img, wl.x_seq)
    dx_img, dx_seq, dparams = O.stage_bwd(wl.layers, wl.params, wl.batch, caches, wl.dy.astype(np.float64))
    rel = lambda a, b: np.max(np.abs(a - b)) / max(np.max(np.abs(b)), 1e-30)
    assert rel(y, y_t.detach().numpy()) < 1e-11
    assert rel(dx_img, x_img.grad.numpy()) < 1e-10 and rel(dx_seq, x_seq.grad.numpy()) < 1e-10
    assert len(dparams) == len(P)
    for g, p in zip(dparams, P):
        assert rel(g, p.grad.numpy()) < 1e-10
