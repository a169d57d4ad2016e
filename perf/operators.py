"""Attention and group normalisation, the operators that stand between a diffusion transformer's (or a U-Net's) quantized
linears, as timed cases: from one query to packed batches of images, from an 8 x 8 feature map to whole high-resolution ones.

Kinds
  attn   dp_attention on bf16 projections: columns of one buffer (self-attention on the output of a qkv linear) or buffers of
         their own (cross-attention). Sequences of equal length, or ("lq", "lk": one length per sequence) packed one behind
         the other, which keeps documents apart. "mask": "" or "causal", the latter with the first "prefix" keys of a sequence
         visible to all of its queries; "cap" > 0: scores capped by a tanh; "bias": one slope per head times the distance.
  norm   dp_group_norm (bf16 out) on channels-last feature maps, or with "codes" dp_group_norm_daq (int8 codes and a scale per
         row, returned as the values that they stand for).

run() computes the plain form where `own` is false.
"""
import math

import torch

own = False


# ---- the cases ------------------------------------------------------------------------------------

def listed():
    return [
        # one image of 256 tokens through a 1152-wide block: the smallest self-attention, latency
        _attn("attn_l256_b1", 16, 72, "256"),
        # the batch that samplers run (8 images of 256 tokens)
        _attn("attn_l256_b8", 16, 72, "256*8"),
        # 512-pixel images, batch 32: throughput
        _attn("attn_l1024_b32", 16, 72, "1024*32"),
        # images of many sizes packed into one batch, kept apart by their offsets; a few tokens long the smallest, and some
        # rows of the buffer unused
        _attn("attn_packed_d64", 12, 64, "1024,77,256,1,640,333,1024,16,900,256,50,1500,129,700,256,64", pad=37),
        # text in front of image tokens that are generated one after the other: the text sees itself whole, capped scores
        _attn("attn_prefix_cap", 16, 64, "1101,1353,1024,1280", mask="causal", prefix="77,300,0,256", cap=30.0),
        # a long sequence, four query heads to a key head, decaying with the distance
        _attn("attn_long_bias", 16, 128, "8192", kv=4, mask="causal", bias=True),
        # one query per sequence over a long context (pooling a video's or a document's tokens)
        _attn("attn_q1_k4096", 16, 72, "1*8", "4096*8"),
        # the next tokens of a batch of sequences behind their own, ragged caches
        _attn("attn_few_gqa", 16, 128, "1,4,1,2,7,1,3,1", "1500,333,4096,77,2048,900,5000,1", kv=4, mask="causal"),
        # the innermost map of a U-Net, two images: latency
        _norm("norm_64x1280_b2", 2, 64, 1280),
        # outer maps of a batch: throughput, the larger one beyond the L2
        _norm("norm_4096x320_b8", 8, 4096, 320),
        _norm("norm_16384x320_b16", 16, 16384, 320),
        # in front of a transformer's input projection: codes for the quantized linear, no activation, a ragged map
        _norm("norm_codes_1023x640_b8", 8, 1023, 640, act="", codes=True),
    ]


def draw(rng):
    if rng.random() < 0.3:
        C = rng.choice((64, 128, 256, 320, 384, 512, 640, 768, 960, 1152, 1280, 1920, 2560))
        B = rng.choice((1, 2, 3, 4, 8))
        return _norm(None, B, _spread(rng, 16, 32 * 1024 * 1024 // (C * B)), C, act=rng.choice(("silu", "silu", "")),
                     codes=rng.random() < 0.4)
    H, D = rng.choice(((6, 64), (12, 64), (16, 64), (16, 72), (8, 40), (8, 80), (12, 96), (8, 128), (16, 128)))
    kw = dict(kv=rng.choice((H, H, H // 2, 1, 2)), cap=rng.choice((0.0, 0.0, 0.0, 30.0, 50.0)), bias=rng.random() < 0.25)
    if rng.random() < 0.4:
        kw["mask"] = "causal"
    kind = rng.choice(("equal", "equal", "packed", "packed", "cross", "few"))
    if kind == "equal":
        n = _spread(rng, 32, 6000)
        B = _spread(rng, 1, max(1, min(32, 60_000_000 // (n * n))))
        lq = lk = "%d*%d" % (n, B)
    elif kind == "packed":
        B = rng.randint(2, 24)
        lq = lk = _text([_spread(rng, 1, 6000 // B * 2) for _ in range(B)])
        kw["pad"] = rng.choice((0, 5, 64))
    elif kind == "cross":
        B = rng.randint(1, 6)
        lq, lk = _text([_spread(rng, 16, 1500) for _ in range(B)]), _text([_spread(rng, 1, 1200) for _ in range(B)])
    else:
        B = rng.randint(1, 12)
        lq, lk = _text([_spread(rng, 1, 16) for _ in range(B)]), _text([_spread(rng, 1, 8000) for _ in range(B)])
    if "mask" in kw and kind != "cross" and rng.random() < 0.5:
        kw["prefix"] = _text([rng.randint(0, n) for n in _lens(lk)])
    return _attn(None, H, D, lq, lk, **kw)


def _attn(name, H, D, lq, lk=None, kv=None, mask="", prefix="", cap=0.0, bias=False, pad=0):
    return _named(name, dict(kind="attn", heads=H, kv_heads=kv or H, dim=D, lq=lq, lk=lk or lq, same=lk is None or lk == lq,
                             mask=mask, prefix=prefix, cap=cap, bias=bias, pad=pad))


def _norm(name, samples, rows, C, act="silu", codes=False):
    return _named(name, dict(kind="norm", samples=samples, rows=rows, C=C, groups=32, act=act, codes=codes))


def _named(name, case):
    return dict(name=name, **case) if name else case


def _spread(rng, lo, hi):
    """A size spread over its logarithm, odd as often as not."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def _text(lens):
    return ",".join(str(n) for n in lens)


def _lens(text):
    """One length per sequence: "a,b,c", or "a*n" for n equal ones."""
    if "," not in text:
        n, _, b = text.partition("*")
        return [int(n)] * int(b or 1)
    return [int(n) for n in text.split(",")]


def _equal(case):
    return "," not in case["lq"] and "," not in case["lk"]


EPS = 1e-5


# ---- inputs -----------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "norm":
        B, R, C = case["samples"], case["rows"], case["C"]
        # channels of their own level and spread, as a convolution leaves them
        level, spread = torch.randn(C, generator=gen, device="cuda"), 0.5 + torch.rand(C, generator=gen, device="cuda")
        s["x"] = (torch.randn(B * R, C, generator=gen, device="cuda") * spread + level).to(torch.bfloat16)
        s["gamma"] = (1 + 0.2 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
        s["beta"] = (0.2 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
        s["y"] = torch.empty(B * R, C, dtype=torch.bfloat16, device="cuda")
        if case["codes"]:
            s["q"] = torch.empty(B * R, C, dtype=torch.int8, device="cuda")
            s["s_a"] = torch.empty(B * R, 1, device="cuda")
        return s
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    lq, lk = _lens(case["lq"]), _lens(case["lk"])
    Mq, Mk = sum(lq) + case["pad"], sum(lk) + case["pad"]
    if case["same"]:  # the output of a qkv linear
        qkv = torch.randn(Mq, (H + 2 * KV) * D, generator=gen, device="cuda")
        qkv[:, :H * D] *= 1.5
        s["qkv"] = qkv.to(torch.bfloat16)
        s["q"], s["k"], s["v"] = s["qkv"].split((H * D, KV * D, KV * D), dim=1)
    else:  # queries of their own, keys and values side by side
        s["q"] = (1.5 * torch.randn(Mq, H * D, generator=gen, device="cuda")).to(torch.bfloat16)
        s["kv"] = torch.randn(Mk, 2 * KV * D, generator=gen, device="cuda").to(torch.bfloat16)
        s["k"], s["v"] = s["kv"].split(KV * D, dim=1)
    # rows behind the last sequence keep what they hold
    s["y"] = torch.randn(Mq, H * D, generator=gen, device="cuda").to(torch.bfloat16)
    starts = lambda lens: torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")  # noqa: E731
    s["q_start"], s["k_start"] = (None, None) if _equal(case) else (starts(lq), starts(lk))
    s["prefix"] = torch.tensor(_lens(case["prefix"]), dtype=torch.int32, device="cuda") if case["prefix"] else None
    # slopes from 1/2 down to 1/256, as distance-biased models take them
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H) if case["bias"] else None
    s["n_seq"], s["max_q"], s["max_k"] = len(lq), max(lq), max(lk)
    return s


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _own_norm(state) if case["kind"] == "norm" else _own_attention(state)
    return _plain_norm(state) if case["kind"] == "norm" else _plain_attention(state)


def _own_attention(s):
    from paper_2511_11446_b200 import binding as B
    case = s["case"]
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    if "attn" not in s:  # the call's description, which a program keeps beside its buffers
        s["attn"] = B.make_attn(H, KV, D, s["n_seq"], s["max_q"], s["max_k"], 1 / math.sqrt(D), q_start=s["q_start"],
                                k_start=s["k_start"], mask=B.DP_MASK_CAUSAL if case["mask"] else B.DP_MASK_NONE,
                                prefix=s["prefix"], cap=case["cap"], slopes=s["slopes"])
    q, k, v, y = s["q"], s["k"], s["v"], s["y"]
    B.dp_attention(s["attn"], q, q.stride(0), q.shape[0], k, k.stride(0), v, v.stride(0), k.shape[0], y, y.stride(0))
    return y


def _own_norm(s):
    from paper_2511_11446_b200 import binding as B
    case = s["case"]
    n, R, C, G = case["samples"], case["rows"], case["C"], case["groups"]
    if "ws" not in s:
        s["ws"] = torch.empty(B.dp_group_norm_workspace(n, R, C, G), dtype=torch.uint8, device="cuda")
    act = B.DP_ACT_SILU if case["act"] == "silu" else B.DP_ACT_NONE
    if case["codes"]:
        B.dp_group_norm_daq(s["x"], n, R, C, C, G, s["gamma"], s["beta"], EPS, act, s["q"], C, s["s_a"], s["ws"])
        return torch.mul(s["q"], s["s_a"], out=s["y"])
    B.dp_group_norm(s["x"], n, R, C, C, G, s["gamma"], s["beta"], EPS, act, s["y"], C, s["ws"])
    return s["y"]


def _positions(start, rows, n_seq, length):
    """Sequence and place in it of every row (sequence n_seq: behind the last one)."""
    row = torch.arange(rows, device="cuda", dtype=torch.int32)
    if start is None:
        return row // length, row % length
    seq = torch.searchsorted(start[1:], row, right=True)
    return seq, row - start[seq.clamp(max=n_seq)]


def _plain_attention(s):
    case = s["case"]
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    n, Mq, Mk = s["n_seq"], s["q"].shape[0], s["k"].shape[0]
    B = n if _equal(case) and not case["pad"] else 1  # packed sequences: all against all, other sequences masked
    q = s["q"].float().view(B, Mq // B, H, D).transpose(1, 2)
    k, v = (t.float().view(B, Mk // B, KV, D).transpose(1, 2).repeat_interleave(H // KV, dim=1) for t in (s["k"], s["v"]))
    qs, qp = _positions(s["q_start"], Mq, n, s["max_q"])
    ks, kp = _positions(s["k_start"], Mk, n, s["max_k"])
    if s["q_start"] is None:
        behind = torch.full((n + 1,), s["max_k"] - s["max_q"], dtype=torch.int32, device="cuda")
    else:
        behind = torch.nn.functional.pad(s["k_start"].diff() - s["q_start"].diff(), (0, 1))
    qp = qp + behind[qs.clamp(max=n)]
    qs, qp, ks, kp = qs.view(B, -1, 1), qp.view(B, -1, 1), ks.view(B, 1, -1), kp.view(B, 1, -1)
    t = (q @ k.transpose(2, 3)) * (1 / math.sqrt(D))
    if case["cap"]:
        t = case["cap"] * torch.tanh(t / case["cap"])
    if s["slopes"] is not None:
        t = t - s["slopes"].view(H, 1, 1) * (qp - kp).abs().unsqueeze(1)
    seen = (qs == ks) & (qs < n)
    if case["mask"]:
        ahead = torch.zeros_like(seen) if s["prefix"] is None else kp < torch.nn.functional.pad(s["prefix"], (0, 1))[qs.clamp(max=n)]
        seen = seen & ((kp <= qp) | ahead)
    t = t.masked_fill(~seen.unsqueeze(1), -math.inf)
    p = torch.exp(t - t.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    total = p.sum(-1, keepdim=True)
    o = ((p @ v) / total.masked_fill(total == 0, 1.0)).transpose(1, 2).reshape(Mq, H * D).to(torch.bfloat16)
    return torch.where((qs < n).view(Mq, 1), o, s["y"])


def _plain_norm(s):
    case = s["case"]
    n, R, C, G = case["samples"], case["rows"], case["C"], case["groups"]
    x = s["x"].float().view(n, R, G, C // G)
    d = x - x.mean((1, 3), keepdim=True)
    h = d * torch.rsqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    h = h.view(n * R, C) * s["gamma"].float() + s["beta"].float()
    if case["act"] == "silu":
        h = h / (1 + torch.exp(-h))
    if case["codes"]:
        scale = h.abs().amax(1, keepdim=True) / 127
        h = torch.round(h / scale.masked_fill(scale == 0, 1.0)) * scale
    return h.to(torch.bfloat16)


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        n, R, C, G = case["samples"], case["rows"], case["C"], case["groups"]
        out = torch.empty(n * R, C, dtype=torch.float64, device="cuda")
        for b in range(n):  # a sample at a time: 64 bits of the largest maps take memory
            x = s["x"][b * R:(b + 1) * R].double().view(R, G, C // G)
            var, mean = torch.var_mean(x, dim=(0, 2), correction=0, keepdim=True)
            h = ((x - mean) / torch.sqrt(var + EPS)).view(R, C) * s["gamma"].double() + s["beta"].double()
            if case["act"] == "silu":
                h = h * torch.sigmoid(h)
            if case["codes"]:  # (a code next to a border may go either way: one value in very many)
                scale = (h.abs().amax(1, keepdim=True) / 127).clamp(min=1e-300)
                h = torch.round(h / scale) * scale
            out[b * R:(b + 1) * R] = h
        return out
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    lq, lk = _lens(case["lq"]), _lens(case["lk"])
    prefix = _lens(case["prefix"]) if case["prefix"] else [0] * len(lq)
    out = s["y"].double()
    q0 = k0 = 0
    for b in range(len(lq)):
        nq, nk = lq[b], lk[b]
        place = torch.arange(nq, device="cuda").view(-1, 1) + (nk - nq)
        key = torch.arange(nk, device="cuda").view(1, -1)
        hidden = (key > place) & (key >= prefix[b]) if case["mask"] else torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
        for h in range(H):
            g = h * KV // H
            q = s["q"][q0:q0 + nq, h * D:(h + 1) * D].double()
            k, v = (s[t][k0:k0 + nk, g * D:(g + 1) * D].double() for t in ("k", "v"))
            score = q @ k.T / math.sqrt(D)
            if case["cap"]:
                score = torch.tanh(score / case["cap"]) * case["cap"]
            if case["bias"]:
                score = score - s["slopes"][h].double() * (place - key).abs()
            weight = torch.softmax(score.masked_fill(hidden, -math.inf), dim=1)
            out[q0:q0 + nq, h * D:(h + 1) * D] = torch.nan_to_num(weight) @ v  # (no key in sight: 0)
        q0, k0 = q0 + nq, k0 + nk
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    if case["kind"] == "norm":
        n = case["samples"] * case["rows"] * case["C"]
        # (codes: they and the scales out, and read back to be returned as values of 16 bits)
        extra = 2 * (n + 4 * case["samples"] * case["rows"]) if case["codes"] else 0
        return {"bytes": 4 * n + 4 * case["C"] + extra, "flops": 8 * n}
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    lq, lk = _lens(case["lq"]), _lens(case["lk"])
    prefix = _lens(case["prefix"]) if case["prefix"] else [0] * len(lq)
    pairs = sum(_pairs(a, b, p, case["mask"]) for a, b, p in zip(lq, lk, prefix))
    return {"bytes": 2 * D * (2 * H * sum(lq) + 2 * KV * sum(lk)), "flops": 4 * D * H * pairs}


def _pairs(nq, nk, prefix, mask):
    """Visible pairs of a sequence."""
    if not mask:
        return nq * nk
    return sum(max(0, min(nk, max(i + nk - nq + 1, prefix))) for i in range(nq))
