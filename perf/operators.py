"""The token side of a language model around the pipeline stage: measured calls.

Four parts of a training step that lie outside a stage's layers or that its decoder layers take as a variant:
  embed_fwd   rows of the token table, scaled, into the packed sequence (rows of image tokens are left to the connector: zero)
  embed_bwd   the table's gradient, summed token by token over the microbatches of an optimizer step
  qk_fwd      RMS norm of every query and key head with the rotary positions in the same pass
  qk_bwd      its gradients
  xent        the loss over the vocabulary with the gradient of the logits, or the loss alone (evaluation)

A case is a dict of plain values.  `run` computes it with elementary torch operations in 32 bits, or, where `own` is true, with the
library's entry points; `exact` is the definition in float64.
"""
import math

import torch

own = False

DEVICE = "cuda"
IMAGE = 576            # tokens of a 336-pixel image in 14-pixel patches: their rows carry no token and no target
IGNORE = -100


def listed():
    return [
        # The toy stage of smoke runs and unit-sized models: two short samples.  Latency.
        dict(name="embed_toy", kind="embed_fwd", tokens=220, vocab=1000, d=256, scaled=False, fp32=False, pad=0),
        # The packed microbatch that a first decoder stage reads, 8B-shaped: half of the rows are images.
        dict(name="embed_32768", kind="embed_fwd", tokens=32768, vocab=131072, d=4096, scaled=False, fp32=False, pad=0),
        # A ragged small microbatch, a 7B-shaped width, a vocabulary that is a multiple of nothing: one microbatch, gradients overwritten.
        dict(name="embed_grad_2999", kind="embed_bwd", tokens=2999, vocab=50257, d=3584, scaled=True, microbatches=1, images=True),
        # Two large microbatches of one optimizer step, the second one adding to the first one's gradient.
        dict(name="embed_grad_2x32768", kind="embed_bwd", tokens=32768, vocab=131072, d=4096, scaled=False, microbatches=2, images=True),
        # The toy decoder layer's queries and keys.
        dict(name="qk_toy", kind="qk_fwd", tokens=220, hq=4, hkv=2, head_dim=64, rotate=True),
        # The 8B-shaped decoder layer on its large microbatch.
        dict(name="qk_32768", kind="qk_fwd", tokens=32768, hq=32, hkv=8, head_dim=128, rotate=True),
        # One short sample through the 8B-shaped layer, backward.
        dict(name="qk_grad_777", kind="qk_bwd", tokens=777, hq=32, hkv=8, head_dim=128, rotate=True),
        # An encoder layer on five tiles of a dynamic-resolution image: 25 heads, no rotation.
        dict(name="qk_grad_encoder_5125", kind="qk_bwd", tokens=5125, hq=25, hkv=25, head_dim=128, rotate=False),
        # The large microbatch, backward.
        dict(name="qk_grad_32768", kind="qk_bwd", tokens=32768, hq=32, hkv=8, head_dim=128, rotate=True),
        # Evaluation of a few answer tokens: the loss alone, logits kept in fp32.
        dict(name="loss_64", kind="xent", tokens=64, vocab=131072, pad=0, fp32=True, grad=False, images=False),
        # A ragged small microbatch, fp32 logits, a vocabulary of an odd size in a padded matrix.
        dict(name="loss_grad_2999", kind="xent", tokens=2999, vocab=50257, pad=7, fp32=True, grad=True, images=True),
        # The vocabulary loss of an ordinary microbatch: bf16 logits, half of the rows are images and ignored.
        dict(name="loss_grad_8192", kind="xent", tokens=8192, vocab=131072, pad=0, fp32=False, grad=True, images=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["embed_fwd", "embed_bwd", "qk_fwd", "qk_bwd", "xent"])
    if kind in ("embed_fwd", "embed_bwd"):
        d = 8 * _log_int(rng, 8, 512)
        tokens, vocab = _log_int(rng, 1, 30000), _log_int(rng, 500, 131000)
        if kind == "embed_fwd":
            return dict(kind=kind, tokens=tokens, vocab=vocab, d=d, scaled=rng.random() < 0.5, fp32=rng.random() < 0.3,
                        pad=rng.choice([0, 0, 8, 64]))
        return dict(kind=kind, tokens=tokens, vocab=vocab, d=d, scaled=rng.random() < 0.5, microbatches=rng.choice([1, 2]),
                    images=rng.random() < 0.5)
    if kind in ("qk_fwd", "qk_bwd"):
        head_dim = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
        hkv = rng.choice([1, 2, 3, 4, 5, 8])
        hq = hkv * rng.choice([1, 2, 4, 7])
        while hq * head_dim > 4096:
            hq -= hkv
        hq = max(hq, 1)
        return dict(kind=kind, tokens=_log_int(rng, 1, 30000), hq=hq, hkv=hkv, head_dim=head_dim, rotate=rng.random() < 0.8)
    vocab = _log_int(rng, 500, 260000)
    most = min(30000, 1000000000 // vocab)
    return dict(kind=kind, tokens=_log_int(rng, 1, most), vocab=vocab, pad=-vocab % rng.choice([8, 64, 128]), fp32=rng.random() < 0.4,
                grad=rng.random() < 0.75, images=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _text(tokens, images):
    """Truth for the rows of text: with images, every other run of IMAGE rows is one."""
    t = torch.arange(tokens, device=DEVICE)
    return (t // IMAGE) % 2 == 0 if images else t >= 0


def _texts(tokens, images):
    if not images:
        return tokens
    whole, rest = divmod(tokens, 2 * IMAGE)
    return whole * IMAGE + min(rest, IMAGE)


def _zipf(n, vocab, g):
    """Token ids with frequencies that fall as one over the rank."""
    u = torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1).int()


def _ids(tokens, vocab, images, g):
    ids = _zipf(tokens, vocab, g)
    return torch.where(_text(tokens, images), ids, torch.full_like(ids, -1))


def _gauss(g, scale, *shape, dtype=torch.bfloat16):
    out = torch.empty(shape, dtype=dtype, device=DEVICE)
    step = max(1, (1 << 28) // max(1, out[0].numel()))
    for r in range(0, shape[0], step):
        out[r:r + step] = torch.randn(out[r:r + step].shape, generator=g, device=DEVICE) * scale
    return out


def _scale(case):
    return math.sqrt(case["d"]) if case["scaled"] else 1.0


def _rope_table(n_pos, head_dim, base=500000.0):
    """[n_pos, head_dim] fp32: the cosines of every position's angles, then the sines."""
    inv = base ** (-2.0 * torch.arange(head_dim // 2, dtype=torch.float64, device=DEVICE) / head_dim)
    angle = torch.arange(n_pos, dtype=torch.float64, device=DEVICE)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    kind, t = case["kind"], case["tokens"]
    s = dict(case=case, keep={})
    if kind == "embed_fwd":
        s["table"] = _gauss(g, 0.02, case["vocab"], case["d"], dtype=torch.float32 if case["fp32"] else torch.bfloat16)
        s["ids"] = _ids(t, case["vocab"], True, g)
        s["y"] = torch.empty(t, case["d"] + case["pad"], dtype=torch.bfloat16, device=DEVICE)[:, :case["d"]]
    elif kind == "embed_bwd":
        s["ids"] = [_ids(t, case["vocab"], case["images"], g) for _ in range(case["microbatches"])]
        s["dy"] = [_gauss(g, 1e-3, t, case["d"]) for _ in range(case["microbatches"])]
        s["dtable"] = torch.empty(case["vocab"], case["d"], dtype=torch.float32, device=DEVICE)
    elif kind in ("qk_fwd", "qk_bwd"):
        h, hd = case["hq"] + case["hkv"], case["head_dim"]
        width = (h + case["hkv"]) * hd                  # [q | k | v] rows, as a projection leaves them
        s["x"] = _gauss(g, 1.5, t, width)
        s["gamma_q"], s["gamma_k"] = (1.0 + 0.1 * torch.randn(2, hd, generator=g, device=DEVICE)).bfloat16()
        n_pos = min(t, 4096)
        s["pos"] = (torch.arange(t, device=DEVICE, dtype=torch.int32) % n_pos) if case["rotate"] else None
        s["table"] = _rope_table(n_pos, hd) if case["rotate"] else None
        if kind == "qk_fwd":
            s["y"] = torch.zeros(t, width, dtype=torch.bfloat16, device=DEVICE)
        else:
            s["dy"] = _gauss(g, 0.05, t, width)
            s["dx"] = torch.zeros(t, width, dtype=torch.bfloat16, device=DEVICE)
            s["dgamma_q"], s["dgamma_k"] = (torch.empty(hd, device=DEVICE) for _ in range(2))
    else:
        vocab, cols = case["vocab"], case["vocab"] + case["pad"]
        s["logits"] = _gauss(g, 2.5, t, cols + -cols % 8, dtype=torch.float32 if case["fp32"] else torch.bfloat16)
        target = _zipf(t, vocab, g)
        s["logits"][torch.arange(t, device=DEVICE), target.long()] += 8.0
        s["targets"] = torch.where(_text(t, case["images"]), target, torch.full_like(target, IGNORE))
        s["weight"] = 1.0 / max(1, _texts(t, case["images"]))
        s["loss"] = torch.empty(t, device=DEVICE)
        s["dlogits"] = torch.empty(t, s["logits"].shape[1], dtype=torch.bfloat16, device=DEVICE) if case["grad"] else None
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind == "embed_fwd":
        return _plain_embed(s, torch.float32).bfloat16()
    if kind == "embed_bwd":
        return _plain_embed_grad(s, torch.float32)
    if kind == "qk_fwd":
        return [v.bfloat16() for v in _plain_qk(s)]
    if kind == "qk_bwd":
        dq, dk, gq, gk = _plain_qk_grad(s)
        return [dq.bfloat16(), dk.bfloat16(), gq, gk]
    loss, grad = _plain_loss(s)
    return [loss] if grad is None else [loss, grad.bfloat16()]


def _keep(s, nbytes):
    """The program's scratch buffer, allocated on its first call."""
    if s["keep"].get("bytes", -1) < nbytes:
        s["keep"].update(bytes=nbytes, buffer=torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEVICE))
    return s["keep"]["buffer"]


def _own(s):
    from paper_2603_25120_amd import binding as B
    c = s["case"]
    kind, t = c["kind"], c["tokens"]
    if kind == "embed_fwd":
        B.mllm_op_embed_fwd(s["table"], s["ids"], s["y"], t, c["vocab"], c["d"], y_stride=c["d"] + c["pad"], scale=_scale(c),
                            table_fp32=int(c["fp32"]))
        return s["y"]
    if kind == "embed_bwd":
        ws = _keep(s, B.mllm_op_embed_bwd_workspace_bytes(t, c["vocab"], c["d"]))
        for i, (dy, ids) in enumerate(zip(s["dy"], s["ids"])):
            B.mllm_op_embed_bwd(dy, ids, s["dtable"], t, c["vocab"], c["d"], ws, scale=_scale(c), accumulate=int(i > 0))
        return s["dtable"]
    if kind in ("qk_fwd", "qk_bwd"):
        hq, hkv, hd = c["hq"], c["hkv"], c["head_dim"]
        width = (hq + 2 * hkv) * hd
        n_pos = 0 if s["table"] is None else s["table"].shape[0]
        if kind == "qk_fwd":
            B.mllm_op_qk_norm_rope_fwd(s["x"], s["gamma_q"], s["gamma_k"], s["y"], t, hq, hkv, hd, width, width, 1e-6,
                                       pos=s["pos"], rope_table=s["table"], n_pos=n_pos)
            return [s["y"][:, :hq * hd], s["y"][:, hq * hd:(hq + hkv) * hd]]
        partial = _keep(s, B.mllm_op_qk_norm_rope_bwd_partial_bytes(t, hq, hkv, hd))
        B.mllm_op_qk_norm_rope_bwd(s["dy"], s["x"], s["gamma_q"], s["gamma_k"], s["dx"], s["dgamma_q"], s["dgamma_k"], t, hq, hkv, hd,
                                   width, width, width, 1e-6, partial, pos=s["pos"], rope_table=s["table"], n_pos=n_pos)
        return [s["dx"][:, :hq * hd], s["dx"][:, hq * hd:(hq + hkv) * hd], s["dgamma_q"], s["dgamma_k"]]
    B.mllm_op_xent(s["logits"], s["targets"], s["loss"], s["dlogits"], t, c["vocab"], s["logits"].shape[1],
                   logits_fp32=int(c["fp32"]), scale=s["weight"])
    return [s["loss"]] if s["dlogits"] is None else [s["loss"], s["dlogits"]]


def _plain_embed(s, kind):
    ids = s["ids"]
    rows = s["table"][ids.clamp(min=0).long()].to(kind) * _scale(s["case"])
    return torch.where((ids >= 0)[:, None], rows, torch.zeros((), dtype=kind, device=DEVICE))


def _plain_embed_grad(s, kind):
    c = s["case"]
    out = torch.zeros(c["vocab"], c["d"], dtype=kind, device=DEVICE)
    ids, dy = torch.cat(s["ids"]), torch.cat(s["dy"])
    there = ids >= 0
    out.index_add_(0, ids[there].long(), dy[there].to(kind) * _scale(c))
    return out


def _rotated(v, s, sign):
    """The half-split pairs (i, i + head_dim/2) turned by the angles of each row's position."""
    if s["table"] is None:
        return v
    half = s["case"]["head_dim"] // 2
    f = s["table"][s["pos"].long()][:, None]
    cos, sin = f[..., :half], sign * f[..., half:]
    a, b = v[..., :half], v[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _heads(v, s):
    c = s["case"]
    q, k = v[:, :c["hq"] * c["head_dim"]], v[:, c["hq"] * c["head_dim"]:(c["hq"] + c["hkv"]) * c["head_dim"]]
    return q.reshape(c["tokens"], c["hq"], -1).float(), k.reshape(c["tokens"], c["hkv"], -1).float()


def _plain_qk(s):
    out = []
    for x, gamma in zip(_heads(s["x"], s), (s["gamma_q"], s["gamma_k"])):
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        out.append(_rotated(x * r * gamma.float(), s, 1).reshape(x.shape[0], -1))
    return out


def _plain_qk_grad(s):
    dx, dgamma = [], []
    for x, dy, gamma in zip(_heads(s["x"], s), _heads(s["dy"], s), (s["gamma_q"], s["gamma_k"])):
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        n, d = x * r, _rotated(dy, s, -1)
        dgamma.append((d * n).sum(0).sum(0))
        d = d * gamma.float()
        dx.append((r * (d - n * (d * n).mean(-1, keepdim=True))).reshape(x.shape[0], -1))
    return dx + dgamma


def _plain_loss(s):
    c = s["case"]
    x = s["logits"][:, :c["vocab"]].float()
    target = s["targets"].long()
    there, at = target >= 0, target.clamp(min=0)[:, None]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    zero = torch.zeros((), device=DEVICE)
    loss = torch.where(there, (torch.log(total) + (m - x.gather(1, at)))[:, 0], zero)
    if not c["grad"]:
        return loss, None
    e = e / total
    e.scatter_add_(1, at, torch.full_like(total, -1.0))
    grad = torch.zeros(c["tokens"], s["logits"].shape[1], device=DEVICE)
    grad[:, :c["vocab"]] = torch.where(there[:, None], e * s["weight"], zero)
    return loss, grad


# ------------------------------------------------------------------------------------------------
# needs, and the definition in 64 bits
# ------------------------------------------------------------------------------------------------
def work(case):
    """Bytes and operations that a pass cannot do without: inputs read once, outputs written once."""
    kind, t = case["kind"], case["tokens"]
    if kind in ("embed_fwd", "embed_bwd"):
        vocab, d = case["vocab"], case["d"]
        n = _texts(t, kind == "embed_fwd" or case["images"])
        # expected number of distinct ids among n draws, rank r with probability log((r + 2) / (r + 1)) / log(vocab + 1)
        rank = torch.arange(vocab, dtype=torch.float64)
        p = torch.log((rank + 2) / (rank + 1)) / math.log(vocab + 1)
        distinct = float((-torch.expm1(n * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())
        if kind == "embed_fwd":
            return dict(bytes=4 * t + distinct * d * (4 if case["fp32"] else 2) + 2 * t * d, flops=n * d if case["scaled"] else 0)
        m = case["microbatches"]
        return dict(bytes=m * (4 * t + 2 * n * d) + 4 * vocab * d + (m - 1) * 8 * distinct * d, flops=m * n * d)
    if kind in ("qk_fwd", "qk_bwd"):
        values = t * (case["hq"] + case["hkv"]) * case["head_dim"]
        table = 4 * t + 4 * min(t, 4096) * case["head_dim"] if case["rotate"] else 0
        return dict(bytes=values * (4 if kind == "qk_fwd" else 6) + table, flops=values * (7 if kind == "qk_fwd" else 14))
    n, cols = _texts(t, case["images"]), case["vocab"] + case["pad"]
    cols += -cols % 8
    return dict(bytes=8 * t + n * case["vocab"] * (4 if case["fp32"] else 2) + (2 * t * cols if case["grad"] else 0),
                flops=n * case["vocab"] * (8 if case["grad"] else 4))


def exact(case, seed):
    """The definition in float64, element by element of what it sums over, laid out as `run` returns it."""
    s = prepare(case, seed)
    kind, t = case["kind"], case["tokens"]
    if kind == "embed_fwd":
        y = torch.zeros(t, case["d"], dtype=torch.float64, device=DEVICE)
        text = (s["ids"] >= 0).nonzero()[:, 0]
        y[text] = _scale(case) * s["table"].index_select(0, s["ids"][text]).double()
        return y
    if kind == "embed_bwd":
        out = torch.zeros(case["vocab"], case["d"], dtype=torch.float64, device=DEVICE)
        for ids, dy in zip(s["ids"], s["dy"]):
            order = torch.argsort(ids, stable=True)
            order = order[int((ids < 0).sum()):]
            names, counts = torch.unique_consecutive(ids[order], return_counts=True)
            ends = counts.cumsum(0)
            for c0 in range(0, case["d"], 512):           # sums of runs as differences of running sums, exact to 2^-53 of them
                runs = dy[order, c0:c0 + 512].double().cumsum(0)
                runs = torch.cat([torch.zeros_like(runs[:1]), runs])
                out[names.long(), c0:c0 + 512] += (runs[ends] - runs[ends - counts]) * _scale(case)
        return out
    if kind in ("qk_fwd", "qk_bwd"):
        hq, hkv, hd = case["hq"], case["hkv"], case["head_dim"]
        half = hd // 2
        ys, gammas = [], []
        for first, heads, gamma in ((0, hq, s["gamma_q"]), (hq, hkv, s["gamma_k"])):
            x = s["x"].double().view(t, -1, hd)[:, first:first + heads]
            gain = gamma.double()
            rms = ((x ** 2).sum(-1, keepdim=True) / hd + 1e-6) ** 0.5
            turn = torch.ones(t, 1, half, dtype=torch.complex128, device=DEVICE)
            if case["rotate"]:
                f = s["table"].double()[s["pos"].long()]
                turn = torch.complex(f[:, :half], f[:, half:])[:, None]
            if kind == "qk_fwd":
                n = x / rms * gain
                z = torch.complex(n[..., :half], n[..., half:]) * turn
                ys.append(torch.cat([z.real, z.imag], -1).reshape(t, -1))
                continue
            dy = s["dy"].double().view(t, -1, hd)[:, first:first + heads]
            z = torch.complex(dy[..., :half], dy[..., half:]) * turn.conj()
            d = torch.cat([z.real, z.imag], -1)
            gammas.append((d * x / rms).sum((0, 1)))
            d = d * gain
            ys.append((d / rms - x * (d * x).sum(-1, keepdim=True) / (hd * rms ** 3)).reshape(t, -1))
        return ys + gammas
    vocab, cols = case["vocab"], s["logits"].shape[1]
    loss = torch.zeros(t, dtype=torch.float64, device=DEVICE)
    grad = torch.zeros(t, cols, dtype=torch.float64, device=DEVICE) if case["grad"] else None
    rows = (s["targets"] >= 0).nonzero()[:, 0]
    for part in rows.split(max(1, (1 << 27) // vocab)):
        x = s["logits"][part, :vocab].double()
        target = s["targets"][part].long()
        lse = torch.logsumexp(x, 1)
        loss[part] = lse - x[torch.arange(len(part), device=DEVICE), target]
        if grad is not None:
            p = torch.exp(x - lse[:, None])
            p[torch.arange(len(part), device=DEVICE), target] -= 1.0
            grad[part, :vocab] = p * s["weight"]
    return [loss] if grad is None else [loss, grad]
