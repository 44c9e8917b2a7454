"""What runs around packed attention in a block's training step: rotary positions with several axes, layer norm, and
checkpoints of activations in 8 bits with the backward passes that read them.

A case names an operator and sizes; `prepare` makes the tensors a training program holds, `run` is one pass, through the
package's entry points where `own` is true, else in elementary torch operations; `exact` is the definition in 64 bits.
`step` in a case: forward and backward; otherwise the forward.

Keys
    op        positions | rotary | norm | act8 | attn
    recipe, n, lo, hi, lens_seed   the packed samples (see `segments`)
    hq, hkv, d                     heads and head dimension (rotary, act8, attn; norm over heads: hq rows of d a token)
    c                              row length of a norm over the model's width
    style     rotary: half | interleaved      axes: 2 (height, width) or 3 (time, height, width)
    far       rotary: positions start anywhere up to this
    grid      rotary: the positions are made in the pass, from the samples' grids
    residual, saved, weights       norm: sum of two streams; 8-bit checkpoint (int8 | e4m3 | ""); type of the weight
    fmt       act8, attn: int8 | e4m3
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128                          # channels that share a scale
MOST = {"int8": 127.0, "e4m3": 448.0}  # largest code
EPS = 1e-5


def _case(op, name=None, **kw):
    case = {"op": op, "recipe": "tokens", "n": 0, "lo": 0, "hi": 0, "lens_seed": 0, **kw}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # The positions of a packed batch of text and video, made once a step: bound by the launch and 12 bytes a token.
        _case("positions", "positions-video", recipe="video", n=200, lo=16, hi=600, lens_seed=7, merge=2),
        # The smallest calls: four samples of 246 tokens, positions included; latency is everything.
        _case("rotary", "rotary-tiny-step-d64", recipe="tiny", hq=2, hkv=2, d=64, axes=2, style="half", far=0, grid=True,
              merge=1, step=True),
        # The ViT encoder on dynamic-resolution images: q, k, v out of the fused projection and back, height and width.
        _case("rotary", "rotary-vit-step-d64", recipe="images", n=64, lens_seed=1002, hq=16, hkv=16, d=64, axes=2, style="half",
              far=0, grid=False, merge=2, step=True),
        # The LLM backbone's packed microbatch: time, height, width, grouped heads, far positions.
        _case("rotary", "rotary-llm-fwd-d128", n=32768, hq=32, hkv=8, d=128, axes=3, style="half", far=1 << 20, grid=False,
              merge=1, step=False),
        # A few rows (what one rank holds of a small batch): latency.
        _case("norm", "norm-tiny-fwd-1280", recipe="tiny", c=1280, residual=False, saved="", weights="bf16", step=False),
        # The encoder's width with the residual sum, training step, input kept as it is.
        _case("norm", "norm-vit-step-1024", recipe="images", n=64, lens_seed=1002, c=1024, residual=True, saved="", weights="bf16",
              step=True),
        # Wider rows, the input kept in 8 bits for the backward pass.
        _case("norm", "norm-act8-step-1280", n=65537, c=1280, residual=False, saved="int8", weights="f32", step=True),
        # The norm of q's heads, rows of one head's 128 channels out of the fused projection.
        _case("norm", "norm-heads-step-d128", n=32768, hq=32, hkv=8, d=128, c=0, residual=False, saved="", weights="bf16", step=True),
        # Checkpoint of what attention keeps (q, k, v, o), there and back: a handful of samples, and the encoder's batch.
        _case("act8", "act8-tiny-d64", recipe="tiny", hq=2, hkv=2, d=64, fmt="int8"),
        _case("act8", "act8-vit-d80-e4m3", recipe="images", n=64, lens_seed=1002, hq=16, hkv=16, d=80, fmt="e4m3"),
        # Attention's training step from its checkpoint: packed after the forward, gradients from the packed tensors.
        _case("attn", "attn-act8-tiny-d64", recipe="tiny", hq=2, hkv=2, d=64, causal=False, fmt="int8"),
        _case("attn", "attn-act8-llm-d128", recipe="pack", n=8192, lens_seed=4, hq=32, hkv=8, d=128, causal=True, fmt="int8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = [work(c) for c in listed()]
    most = {m: max(w[m] for w in top) for m in ("bytes", "flops")}
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def _draw(rng):
    op, seed, d = rng.choice(("positions", "rotary", "rotary", "norm", "norm", "norm", "act8", "act8", "attn")), rng.randrange(1 << 20), \
        rng.choice((64, 80, 96, 128))
    g, hkv = rng.choice((1, 1, 2, 4)), rng.choice((1, 2, 3, 8, 16))
    if op == "positions":
        return _case(op, recipe="video", n=_log(rng, 1, 300), lo=rng.randint(1, 40), hi=_log(rng, 60, 2000), lens_seed=seed,
                     merge=rng.choice((1, 2)))
    if op == "rotary":
        recipe = rng.choice(("tokens", "images", "video"))
        n = _log(rng, 1, 60000) if recipe == "tokens" else _log(rng, 1, 48)
        return _case(op, recipe=recipe, n=n, lo=8, hi=300, lens_seed=seed, hq=g * hkv, hkv=hkv, d=d, axes=rng.choice((2, 3)),
                     style=rng.choice(("half", "interleaved")), far=rng.choice((0, 1 << 14, 1 << 20)), grid=rng.random() < 0.3,
                     merge=rng.choice((1, 2)), step=rng.random() < 0.6)
    if op == "norm":
        n, common = _log(rng, 1, 100000), {"weights": rng.choice(("bf16", "f32")), "step": rng.random() < 0.7}
        if rng.random() < 0.3:
            return _case(op, n=n, hq=g * hkv, hkv=hkv, d=d, c=0, residual=False, saved="", **common)
        c = rng.choice((8 * _log(rng, 4, 1024), 64 * _log(rng, 4, 128), _log(rng, 33, 8000)))
        return _case(op, n=n, c=c, residual=rng.random() < 0.4, saved=rng.choice(("", "", "int8", "e4m3")), **common)
    fmt = rng.choice(("int8", "e4m3"))
    if op == "act8":
        return _case(op, n=_log(rng, 1, 100000), hq=g * hkv, hkv=hkv, d=d, fmt=fmt)
    return _case(op, recipe="pack", n=_log(rng, 130, 8192), lens_seed=seed, hq=g * hkv, hkv=hkv, d=d, causal=rng.random() < 0.5, fmt=fmt)


# ------------------------------------------------------------------------------------------------ sizes and inputs


def segments(case):
    """(lengths, grids) of the packed segments, from the case alone: grid (t, h, w) of an image or video, zeros for text."""
    rng, n = np.random.Generator(np.random.PCG64(case["lens_seed"])), case["n"]
    if case["recipe"] == "tiny":
        grids = np.array([[1, 4, 4], [0, 0, 0], [1, 8, 8], [0, 0, 0]])
        return np.array([16, 37, 64, 129]), grids
    if case["recipe"] == "tokens":  # one run of text
        return np.array([n]), np.zeros((1, 3), dtype=np.int64)
    if case["recipe"] == "pack":    # lognormal lengths, at least one token
        lens = np.maximum(1, np.round(np.exp(rng.normal(math.log(1 + n / 6), 1.0, size=64)))).astype(np.int64)
        ends = np.minimum(np.cumsum(lens), n)
        lens = np.diff(np.concatenate([[0], ends]))
        lens[-1] += n - ends[-1]
        return lens[lens > 0], np.zeros((int((lens > 0).sum()), 3), dtype=np.int64)
    kh, kw = rng.integers(8, 49, size=n), rng.integers(8, 49, size=n)
    grids = np.stack([np.ones_like(kh), 2 * kh, 2 * kw], axis=1)
    if case["recipe"] == "images":
        return grids.prod(axis=1), grids
    frames = np.stack([rng.integers(1, 17, size=n), 2 * rng.integers(2, 17, size=n), 2 * rng.integers(2, 17, size=n)], axis=1)
    text = rng.integers(case["lo"], case["hi"] + 1, size=n)  # video: each clip follows some text
    lens = np.stack([text, frames.prod(axis=1)], axis=1).reshape(-1)
    grids = np.stack([np.zeros_like(frames), frames], axis=1).reshape(-1, 3)
    return lens, grids


def _tokens(case):
    return int(segments(case)[0].sum())


def _rows(case):
    """(rows, channels) of a norm."""
    return (_tokens(case), case["c"]) if case["c"] else (_tokens(case) * case["hq"], case["d"])


def work(case):
    """Each input read once and each output written once; the formulas' operations."""
    op, t = case["op"], _tokens(case)
    if op == "positions":
        return {"bytes": 12 * t + 32 * len(segments(case)[0]), "flops": 20 * t}
    if op == "norm":
        rows, c = _rows(case)
        fwd = 4 + 4 * case["residual"] + (1 + 4 / BLOCK if case["saved"] else 0)
        bwd = 4 + 2 * case["residual"] + (1 + 4 / BLOCK if case["saved"] else 2)
        return {"bytes": rows * c * (fwd + bwd * case["step"]) + 8 * rows * (1 + case["step"]), "flops": rows * c * (8 + 14 * case["step"])}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if op == "rotary":
        passes = 1 + case["step"]
        made = 12 * t if case["grid"] else 0
        return {"bytes": passes * (4 * d * (hq + 2 * hkv) * t + 4 * case["axes"] * t) + made, "flops": passes * 3 * d * (hq + hkv) * t}
    kept = d * (2 * hq + 2 * hkv) * t
    if op == "act8":
        return {"bytes": kept * (6 + 8 / d), "flops": 4 * kept}
    lens = segments(case)[0].astype(np.float64)
    pairs = float(np.sum(lens * (lens + 1) / 2 if case["causal"] else lens * lens))
    return {"bytes": kept * (4 + 8 / d) + 2 * d * (2 * hq + 2 * hkv) * t + 4 * hq * t, "flops": 10.0 * d * hq * pairs + 4 * kept}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def activations(*shape):  # channels of different size, some of them off zero, as a trained model's are
        x = normal(*shape) * torch.exp(0.5 * normal(shape[-1])) + 0.3 * normal(shape[-1])
        return x.to(torch.bfloat16)

    op, s = case["op"], {"case": case}
    lens, grids = segments(case)
    t = int(lens.sum())
    if op in ("positions", "rotary"):
        cu = np.zeros(len(lens) + 1, dtype=np.int32)
        np.cumsum(lens, out=cu[1:])
        s["cu"] = torch.from_numpy(cu).cuda()
        s["grids"] = torch.from_numpy(grids.astype(np.int32)).cuda()
        top = case.get("far", 1000) or 1
        s["first"] = torch.randint(0, top, (len(lens),), generator=gen, device="cuda", dtype=torch.int32)
        s["tokens"] = t
    if op == "positions":
        return s
    if op == "rotary":
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        half = d // 2
        if case["axes"] == 2:   # height and width, each with frequencies of its own
            axis = np.repeat([1, 2], [half // 2, half - half // 2])
            at = np.concatenate([np.arange(half // 2) / (half // 2), np.arange(half - half // 2) / (half - half // 2)])
        else:                   # time, height, width take parts of one range of frequencies
            part = half // 4
            axis = np.repeat([0, 1, 2], [part, (half - part) // 2, half - part - (half - part) // 2])
            at = np.arange(half) / half
        s["axis"] = torch.from_numpy(axis.astype(np.int32)).cuda()
        s["inv_freq"] = torch.from_numpy((10000.0 ** -at).astype(np.float32)).cuda()
        if not case["grid"]:
            s["positions"] = _positions(s["cu"], s["grids"], s["first"], case["merge"], t)
        s["qkv"] = normal(t, hq + 2 * hkv, d).to(torch.bfloat16)
        if case["step"]:
            s["dq"], s["dk"], s["dv"] = (normal(t, h, d).to(torch.bfloat16) for h in (hq, hkv, hkv))
        return s
    if op == "norm":
        weights = torch.bfloat16 if case["weights"] == "bf16" else torch.float32
        if case["c"]:
            shape = (t, case["c"])
            s["x"] = activations(*shape)
        else:
            shape = (t, case["hq"], case["d"])
            s["x"] = activations(t, case["hq"] + 2 * case["hkv"], case["d"])[:, : case["hq"]]  # q in the fused projection
        if case["residual"]:
            s["residual"] = (0.5 * normal(*shape)).to(torch.bfloat16)
        s["w"], s["b"] = (1 + 0.2 * normal(shape[-1])).to(weights), (0.1 * normal(shape[-1])).to(weights)
        if case["step"]:
            s["dy"] = normal(*shape).to(torch.bfloat16)
            if case["residual"]:
                s["dsummed"] = normal(*shape).to(torch.bfloat16)
        return s
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    s["q"], s["k"], s["v"] = (normal(t, h, d).to(torch.bfloat16) for h in (hq, hkv, hkv))
    if op == "act8":
        s["o"] = (0.1 * normal(t, hq, d)).to(torch.bfloat16)
        return s
    cu = np.zeros(len(lens) + 1, dtype=np.int32)
    np.cumsum(lens, out=cu[1:])
    s["cu"], s["longest"], s["scale"] = torch.from_numpy(cu).cuda(), int(lens.max()), d ** -0.5
    s["dout"] = normal(t, hq, d).to(torch.bfloat16)
    scores = _scores(s["q"], s["k"], s["cu"], case["causal"], s["scale"])  # what the forward left behind
    s["lse"] = torch.logsumexp(scores, dim=-1)
    s["o"] = torch.matmul(torch.exp(scores - s["lse"][..., None]), _by_head(s["v"], hq)).transpose(0, 1).to(torch.bfloat16).contiguous()
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(s):
    case, op = s["case"], s["case"]["op"]
    if op == "positions":
        if own:
            from paper_2605_08962_amd import binding
            return binding.varlen_attn_rotary_positions(s["cu"], s["grids"], s["tokens"], first=s["first"], merge=case["merge"])
        return _positions(s["cu"], s["grids"], s["first"], case["merge"], s["tokens"])
    if op == "rotary":
        return _run_rotary_own(s) if own else _run_rotary_plain(s)
    if op == "norm":
        return _run_norm_own(s) if own else _run_norm_plain(s)
    if op == "act8":
        kept = [s[n] for n in ("q", "k", "v", "o")]
        if own:
            from paper_2605_08962_amd import binding
            packed = binding.varlen_attn_act8_pack(kept, case["fmt"])
            return {"values": binding.varlen_attn_act8_unpack(packed), "scales": [p.scales for p in packed]}
        packed = [_pack(x, case["fmt"]) for x in kept]
        return {"values": [_unpack(*p).to(torch.bfloat16) for p in packed], "scales": [p[1] for p in packed]}
    return _run_attn_own(s) if own else _run_attn_plain(s)


def _positions(cu, grids, first, merge, tokens):
    at = torch.arange(tokens, device=cu.device)
    seg = torch.searchsorted(cu.long(), at, right=True) - 1
    i = at - cu.long()[seg]
    h, w = grids[seg, 1].long(), grids[seg, 2].long()
    text = h == 0
    h, w = torch.where(text, merge, h), torch.where(text, merge, w)
    time, r = i // (h * w), i % (h * w)
    block, e = r // (merge * merge), r % (merge * merge)
    row = block // (w // merge) * merge + e // merge
    col = block % (w // merge) * merge + e % merge
    return (torch.where(text, i, torch.stack([time, row, col])) + first.long()[seg]).to(torch.int32)


def _angles(positions, inv_freq, axis):
    """cos and sin of position times frequency; in 64 bits up to there, since 32 lose the angle of a far position."""
    phi = positions[axis.long()].double().T * inv_freq.double()
    return torch.cos(phi).float()[:, None], torch.sin(phi).float()[:, None]


def _rotate(x, cos, sin, style):
    x = x.float()
    a, b = x.chunk(2, dim=-1) if style == "half" else (x[..., 0::2], x[..., 1::2])
    y = a * cos - b * sin, b * cos + a * sin
    return (torch.cat(y, dim=-1) if style == "half" else torch.stack(y, dim=-1).flatten(-2)).to(torch.bfloat16)


def _run_rotary_plain(s):
    case, style = s["case"], s["case"]["style"]
    hq, hkv = case["hq"], case["hkv"]
    positions = _positions(s["cu"], s["grids"], s["first"], case["merge"], s["tokens"]) if case["grid"] else s["positions"]
    cos, sin = _angles(positions, s["inv_freq"], s["axis"])
    out = {"q": _rotate(s["qkv"][:, :hq], cos, sin, style), "k": _rotate(s["qkv"][:, hq:hq + hkv], cos, sin, style),
           "v": s["qkv"][:, hq + hkv:].contiguous()}
    if case["step"]:
        out["dqkv"] = torch.cat([_rotate(s["dq"], cos, -sin, style), _rotate(s["dk"], cos, -sin, style), s["dv"]], dim=1)
    return out


def _run_rotary_own(s):
    from paper_2605_08962_amd import binding
    case = s["case"]
    hq, hkv = case["hq"], case["hkv"]
    positions = s["positions"] if not case["grid"] else \
        binding.varlen_attn_rotary_positions(s["cu"], s["grids"], s["tokens"], first=s["first"], merge=case["merge"])
    turn = (positions, s["inv_freq"], s["axis"])
    kind = {"interleaved": case["style"] == "interleaved"}
    qkv = s["qkv"]
    q, k, v = binding.varlen_attn_rotary_fwd(qkv[:, :hq], qkv[:, hq:hq + hkv], *turn, v=qkv[:, hq + hkv:], **kind)
    out = {"q": q, "k": k, "v": v}
    if case["step"]:
        out["dqkv"] = g = torch.empty_like(qkv)
        binding.varlen_attn_rotary_bwd(s["dq"], s["dk"], *turn, dv=s["dv"], dq_out=g[:, :hq], dk_out=g[:, hq:hq + hkv],
                                       dv_out=g[:, hq + hkv:], **kind)
    return out


def _pack(x, fmt):
    """(codes, scales): blocks of up to 128 channels of a row, the largest at the format's largest code."""
    c = x.shape[-1]
    blocks = torch.nn.functional.pad(x.float(), (0, -c % BLOCK)).unflatten(-1, (-1, BLOCK)) if c > BLOCK else x.float()[..., None, :]
    scales = (blocks.abs().amax(dim=-1) * (1.0 / MOST[fmt])).clamp_min(2.0 ** -126)
    codes = blocks * torch.reciprocal(scales)[..., None]
    codes = codes.round().to(torch.int8) if fmt == "int8" else codes.to(torch.float8_e4m3fn)
    return codes.flatten(-2)[..., :c], scales


def _unpack(codes, scales):
    c = codes.shape[-1]
    return codes.float() * scales.repeat_interleave(min(c, BLOCK), dim=-1)[..., :c]


def _run_norm_plain(s):
    case, x = s["case"], s["x"]
    out = {}
    if case["residual"]:
        x = out["summed"] = (x.float() + s["residual"].float()).to(torch.bfloat16)
    w, b, h = s["w"].float(), s["b"].float(), x.float()
    mean = h.mean(dim=-1)
    centred = h - mean[..., None]
    rstd = torch.rsqrt((centred * centred).mean(dim=-1) + EPS)
    out |= {"y": (centred * rstd[..., None] * w + b).to(torch.bfloat16), "mean": mean, "rstd": rstd}
    if not case["step"]:
        return out
    if case["saved"]:
        h = _unpack(*_pack(x, case["saved"]))
    dy, xhat = s["dy"].float(), (h - mean[..., None]) * rstd[..., None]
    g = dy * w
    dx = rstd[..., None] * (g - g.mean(dim=-1, keepdim=True) - xhat * (g * xhat).mean(dim=-1, keepdim=True))
    if case["residual"]:
        dx = dx + s["dsummed"].float()
    return out | {"dx": dx.to(torch.bfloat16), "dw": (dy * xhat).flatten(0, -2).sum(dim=0), "db": dy.flatten(0, -2).sum(dim=0)}


def _run_norm_own(s):
    from paper_2605_08962_amd import binding
    case = s["case"]
    f = binding.varlen_attn_norm_fwd(s["x"], s["w"], s["b"], eps=EPS, residual=s.get("residual"), save=case["saved"] or None)
    out = {"y": f.out, "mean": f.mean, "rstd": f.rstd}
    if case["residual"]:
        out["summed"] = f.summed
    if case["step"]:
        x = f.saved if case["saved"] else f.summed if case["residual"] else s["x"]
        out["dx"], out["dw"], out["db"] = binding.varlen_attn_norm_bwd(s["dy"], x, f.mean, f.rstd, s["w"], dsummed=s.get("dsummed"))
    return out


def _by_head(x, heads):
    """[T, H, D] as float32 [heads, T, D], each kv head as often as query heads share it."""
    return x.float().transpose(0, 1).repeat_interleave(heads // x.shape[1], dim=0).contiguous()


def _scores(q, k, cu, causal, scale):
    """Scaled scores [Hq, T, T], -inf where the mask leaves nothing."""
    at = torch.arange(q.shape[0], device=q.device)
    sample = torch.searchsorted(cu.long(), at, right=True)
    seen = sample[:, None] == sample
    if causal:
        seen = seen & (at[:, None] >= at)
    s = torch.matmul(_by_head(q, q.shape[1]), _by_head(k, q.shape[1]).transpose(1, 2).contiguous()) * scale
    return s.masked_fill_(~seen, float("-inf"))


def _run_attn_plain(s):
    case, hq = s["case"], s["case"]["hq"]
    q, k, v, o = (_unpack(*_pack(s[n], case["fmt"])).to(torch.bfloat16) for n in ("q", "k", "v", "o"))
    p = torch.exp(_scores(q, k, s["cu"], case["causal"], s["scale"]) - s["lse"][..., None])
    do = _by_head(s["dout"], hq)
    delta = (do * _by_head(o, hq)).sum(dim=-1, keepdim=True)
    ds = p * (torch.matmul(do, _by_head(v, hq).transpose(1, 2).contiguous()) - delta) * s["scale"]
    dq, dk = torch.matmul(ds, _by_head(k, hq)), torch.matmul(ds.transpose(1, 2).contiguous(), _by_head(q, hq))
    dv = torch.matmul(p.transpose(1, 2).contiguous(), do)
    dk, dv = (g.unflatten(0, (case["hkv"], -1)).sum(dim=1) for g in (dk, dv))  # query heads that share a kv head
    return {n: g.transpose(0, 1).to(torch.bfloat16).contiguous() for n, g in (("dq", dq), ("dk", dk), ("dv", dv))}


def _run_attn_own(s):
    from paper_2605_08962_amd import binding
    case = s["case"]
    kept = binding.varlen_attn_act8_pack([s[n] for n in ("q", "k", "v", "o")], case["fmt"])
    dq, dk, dv = binding.varlen_attn_bwd_act8(s["dout"], *kept, s["lse"], s["cu"], case["causal"], s["scale"], max_seqlen=s["longest"])
    return {"dq": dq, "dk": dk, "dv": dv}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"positions": _exact_positions, "rotary": _exact_rotary, "norm": _exact_norm, "act8": _exact_act8, "attn": _exact_attn}[case["op"]](s)


def _exact_positions(s):
    return _grid_walk(s)


def _grid_walk(s):
    """Segment by segment: the tokens in the order in which blocks of merge x merge patches are laid out."""
    m, parts = s["case"]["merge"], []
    lens = torch.diff(s["cu"]).tolist()
    for n, (t, h, w), first in zip(lens, s["grids"].tolist(), s["first"].tolist()):
        if h == 0:
            parts.append(torch.arange(first, first + n).expand(3, n))
            continue
        g = torch.stack(torch.meshgrid(torch.arange(t), torch.arange(h), torch.arange(w), indexing="ij"))
        g = g.view(3, t, h // m, m, w // m, m).permute(0, 1, 2, 4, 3, 5).reshape(3, -1)
        parts.append(g + first)
    return torch.cat(parts, dim=1).to(torch.int32).cuda()


def _exact_rotary(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pos = _grid_walk(s) if case["grid"] else s["positions"]
    freq, turn = s["inv_freq"].double(), torch.empty((pos.shape[1], d // 2), dtype=torch.complex128, device="cuda")
    for a in range(3):
        mine = s["axis"] == a
        phi = pos[a].double()[:, None] * freq[mine]
        turn[:, mine] = torch.polar(torch.ones_like(phi), phi)

    def spin(x, factor):
        x = x.double()
        z = torch.complex(x[..., : d // 2], x[..., d // 2:]) if case["style"] == "half" else torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous())
        z = z * factor[:, None]
        return torch.cat([z.real, z.imag], dim=-1) if case["style"] == "half" else torch.view_as_real(z).flatten(-2)

    x = s["qkv"]
    out = {"q": spin(x[:, :hq], turn), "k": spin(x[:, hq:hq + hkv], turn), "v": x[:, hq + hkv:].double()}
    if case["step"]:
        out["dqkv"] = torch.cat([spin(s["dq"], turn.conj()), spin(s["dk"], turn.conj()), s["dv"].double()], dim=1)
    return out


def _stored(x, fmt):
    """The values (64 bits) and scales that a packed tensor stands for; scale, its inverse and their product with x are 32-bit
    numbers by definition of the format."""
    x, c = x.double(), x.shape[-1]
    values, scales = torch.empty_like(x), []
    for at in range(0, c, BLOCK):
        b = x[..., at:at + BLOCK]
        most = torch.maximum(b.max(dim=-1, keepdim=True).values, -b.min(dim=-1, keepdim=True).values)
        share = float(np.float32(1.0 / MOST[fmt]))
        scale = torch.maximum((most * share).float(), torch.tensor(2.0 ** -126, device=x.device)).double()
        u = (b * (1 / scale).float().double()).float().double()
        if fmt == "int8":
            code = torch.round(u)
        else:  # 3 bits behind the leading one, steps of 2^-9 at least
            _, e = torch.frexp(u)
            step = torch.ldexp(torch.ones_like(u), torch.clamp(e - 4, min=-9))
            code = torch.clamp(torch.round(u / step) * step, -448, 448)
        values[..., at:at + BLOCK] = code * scale
        scales.append(scale)
    return values, torch.cat(scales, dim=-1)


def _exact_act8(s):
    kept = [_stored(s[n], s["case"]["fmt"]) for n in ("q", "k", "v", "o")]
    return {"values": [v for v, _ in kept], "scales": [a for _, a in kept]}


def _exact_norm(s):
    case, x, out = s["case"], s["x"], {}
    if case["residual"]:
        out["summed"] = x.double() + s["residual"].double()
        x = out["summed"].to(torch.bfloat16)  # the stream is kept in this type, and the norm is of what is kept
    h, w, b, c = x.double(), s["w"].double(), s["b"].double(), x.shape[-1]
    mean = h.sum(-1, keepdim=True) / c
    rstd = ((h * h).sum(-1, keepdim=True) / c - mean * mean + EPS) ** -0.5
    out |= {"y": (h - mean) * rstd * w + b, "mean": mean[..., 0], "rstd": rstd[..., 0]}
    if case["step"]:
        if case["saved"]:
            h = _stored(x, case["saved"])[0]
        n, dy = (h - mean) * rstd, s["dy"].double()
        out["dw"], out["db"] = (dy * n).reshape(-1, c).sum(0), dy.reshape(-1, c).sum(0)
        a = dy * w * rstd
        out["dx"] = a - a.sum(-1, keepdim=True) / c - n * ((a * n).sum(-1, keepdim=True) / c)
        if case["residual"]:
            out["dx"] += s["dsummed"].double()
    return out


def _exact_attn(s):
    """Sample by sample and kv head by kv head."""
    case = s["case"]
    # (the kept tensors are used as bf16, as they were before they were packed)
    q, k, v, o = (_stored(s[n], case["fmt"])[0].to(torch.bfloat16).double() for n in ("q", "k", "v", "o"))
    do, group, f = s["dout"].double(), case["hq"] // case["hkv"], s["scale"]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    cu = s["cu"].tolist()
    for lo, hi in zip(cu[:-1], cu[1:]):
        for h in range(case["hq"]):
            c = h // group
            a, b, val, g = q[lo:hi, h], k[lo:hi, c], v[lo:hi, c], do[lo:hi, h]
            p = torch.exp(f * (a @ b.T) - s["lse"][h, lo:hi].double()[:, None])
            if case["causal"]:
                p = p.tril()
            ds = f * p * (g @ val.T - (g * o[lo:hi, h]).sum(-1, keepdim=True))
            dq[lo:hi, h] = ds @ b
            dk[lo:hi, c] += ds.T @ a
            dv[lo:hi, c] += p.T @ g
    return {"dq": dq, "dk": dk, "dv": dv}
