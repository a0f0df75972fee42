"""Operators on packed batches: requests of different lengths, one after the other along one token axis, without padding.

Kinds of a case:
  layout     offsets, request index and (time, height, width) position of every packed token from the requests' sizes (hyb_packed_layout)
  rotary     rotary positions with several axes on queries and keys (hyb_rotary)
  attention  attention of every request's queries over its own keys, grouped heads, causal or full (hyb_packed_attention)

run() computes a case in its plain form, elementary torch operations, or with the framework's calls where `own` is true."""
import math
import random

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LOG2E = math.log2(math.e)


def listed():
    return [
        # A step's worth of images of 512 x 512 to 1024 x 1024 with their prompts, laid out when the batch is put together: all latency.
        {"name": "layout_eight_images", "kind": "layout", "requests": 8, "frames": 1, "side_lo": 32, "side_hi": 64, "txt": 333, "text_after": False, "mix": 1},
        # A large queue of images and short videos, text positions behind the image's: bandwidth.
        {"name": "layout_videos", "kind": "layout", "requests": 256, "frames": 16, "side_lo": 16, "side_hi": 45, "txt": 154, "text_after": True, "mix": 2},
        # One new token per sequence of a text model, positions far into long contexts: the smallest call.
        {"name": "rotary_single_tokens", "kind": "rotary", "tokens": 16, "q_heads": 32, "k_heads": 8, "head_dim": 128, "axes": 1, "rest": 0, "pairs": "halves",
         "far": 1000000, "q_scaled": False, "inverse": False, "dtype": "bf16"},
        # Queries and keys of one 1024 x 1024 image and its prompt inside a joint block; the queries leave with the softmax scale in them.
        {"name": "rotary_1024_image", "kind": "rotary", "tokens": 4429, "q_heads": 24, "k_heads": 24, "head_dim": 64, "axes": 3, "rest": 0, "pairs": "neighbours",
         "far": 64, "q_scaled": True, "inverse": False, "dtype": "bf16"},
        # A small model at reference precision, two axes over part of the head, the gradient's direction.
        {"name": "rotary_f32_inverse", "kind": "rotary", "tokens": 2102, "q_heads": 12, "k_heads": 12, "head_dim": 64, "axes": 2, "rest": 16, "pairs": "neighbours",
         "far": 45, "q_scaled": False, "inverse": True, "dtype": "f32"},
        # A long video with grouped keys: bandwidth.
        {"name": "rotary_video", "kind": "rotary", "tokens": 65537, "q_heads": 24, "k_heads": 8, "head_dim": 128, "axes": 3, "rest": 0, "pairs": "halves",
         "far": 4096, "q_scaled": True, "inverse": False, "dtype": "bf16"},
        # Two short prompts through a small text encoder: the smallest attention, launch latency.
        {"name": "attention_two_prompts", "kind": "attention", "sequences": 2, "lo": 40, "hi": 77, "new": 0, "q_heads": 12, "k_heads": 12, "head_dim": 64,
         "causal": True, "prescaled": False, "dtype": "bf16", "mix": 3},
        # Six images between 512 x 512 and 1024 x 1024 with their text, one launch for all of them.
        {"name": "attention_images", "kind": "attention", "sequences": 6, "lo": 1101, "hi": 4429, "new": 0, "q_heads": 24, "k_heads": 24, "head_dim": 64,
         "causal": False, "prescaled": True, "dtype": "bf16", "mix": 4},
        # One 2048 x 2048 image: the longest full attention.
        {"name": "attention_2048_image", "kind": "attention", "sequences": 1, "lo": 16717, "hi": 16717, "new": 0, "q_heads": 24, "k_heads": 24, "head_dim": 64,
         "causal": False, "prescaled": True, "dtype": "bf16", "mix": 5},
        # Whole prompts of a text model with grouped heads, 33 to 4000 tokens: causal.
        {"name": "attention_prompts", "kind": "attention", "sequences": 24, "lo": 33, "hi": 4000, "new": 0, "q_heads": 32, "k_heads": 8, "head_dim": 128,
         "causal": True, "prescaled": False, "dtype": "bf16", "mix": 6},
        # One new token per sequence over caches of 100 to 8000: the memory's bandwidth.
        {"name": "attention_single_tokens", "kind": "attention", "sequences": 64, "lo": 100, "hi": 8000, "new": 1, "q_heads": 32, "k_heads": 8, "head_dim": 128,
         "causal": True, "prescaled": False, "dtype": "bf16", "mix": 7},
        # A small model at reference precision with grouped heads: fp32 matrix cores.
        {"name": "attention_f32", "kind": "attention", "sequences": 3, "lo": 203, "hi": 1400, "new": 0, "q_heads": 12, "k_heads": 4, "head_dim": 64,
         "causal": False, "prescaled": False, "dtype": "f32", "mix": 8},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("layout", "rotary", "rotary", "attention", "attention", "attention"))
    mix = rng.randrange(1 << 20)
    if kind == "layout":
        lo = rng.randint(4, 32)
        return {"kind": kind, "requests": _log_int(rng, 2, 256), "frames": rng.choice((1, 1, 5, 16)), "side_lo": lo, "side_hi": lo + rng.randint(1, 13),
                "txt": rng.choice((0, 77, 154, 333)), "text_after": rng.random() < 0.5, "mix": mix}
    if kind == "rotary":
        k_heads = rng.choice((1, 2, 4, 5, 8, 10, 12))
        q_heads = k_heads * rng.choice((1, 1, 2, 3, 4))
        head_dim = rng.choice((64, 64, 128))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        tokens = min(_log_int(rng, 1, 65536), 600000000 // (4 * (q_heads + k_heads) * head_dim * (2 if dtype == "bf16" else 4)))
        return {"kind": kind, "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "head_dim": head_dim, "axes": rng.randint(1, 4),
                "rest": rng.choice((0, 0, 16, 32)), "pairs": rng.choice(("neighbours", "halves")), "far": _log_int(rng, 64, 1000000),
                "q_scaled": rng.random() < 0.5, "inverse": rng.random() < 0.3, "dtype": dtype}
    dtype = rng.choice(("bf16", "bf16", "bf16", "bf16", "f32"))
    head_dim = rng.choice((64, 64, 128))
    k_heads = rng.choice((1, 2, 4, 5, 8, 10, 12))
    q_heads = k_heads * rng.choice((1, 1, 2, 3, 4))
    form = rng.choice(("self", "self", "new"))
    sequences = _log_int(rng, 1, 64) if form == "new" else _log_int(rng, 1, 24)
    hi = _log_int(rng, 64, 8192 if form == "new" else 4096 if dtype == "bf16" else 1400)
    new = 0 if form == "self" else rng.choice((1, 1, 2, 5, 17, 100))
    while sequences > 1 and sequences * q_heads * hi * (min(new, hi) or hi) > 2000000000:      # (padded scores of the plain form)
        sequences //= 2
    return {"kind": "attention", "sequences": sequences, "lo": max(1, hi // rng.choice((1, 2, 8, 64))), "hi": hi, "new": new, "q_heads": q_heads, "k_heads": k_heads,
            "head_dim": head_dim, "causal": rng.random() < 0.5, "prescaled": rng.random() < 0.5, "dtype": dtype, "mix": mix}


# ---- sizes that a case stands for (the same for every seed; a seed decides their order) -------------------------------------------------

def _shapes(case):
    """(frames, height, width, text tokens) of every request: half of them single images."""
    r = random.Random(case["mix"])
    return [(r.choice((1, r.randint(1, case["frames"]))), r.randint(case["side_lo"], case["side_hi"]), r.randint(case["side_lo"], case["side_hi"]),
             r.randint(0, case["txt"])) for _ in range(case["requests"])]


def _lengths(case):
    """(queries, keys) of every sequence; lengths over the logarithm of the range."""
    r = random.Random(case["mix"])
    keys = [_log_int(r, case["lo"], case["hi"]) for _ in range(case["sequences"])]
    return [(min(n, case["new"]) if case["new"] else n, n) for n in keys]


def _axis_dims(case):
    """Widths of the axes' sections: even numbers whose sum is the rotated width, the first axis' the smallest."""
    pairs = (case["head_dim"] - case["rest"]) // 2
    each = pairs // case["axes"]
    return [2 * each] * (case["axes"] - 1) + [2 * (pairs - each * (case["axes"] - 1))]


def _pairs_seen(case):
    """Query-key pairs of all sequences that count."""
    return sum(nq * nk - (nq * (nq - 1) // 2 if case["causal"] else 0) for nq, nk in _lengths(case))


def work(case):
    if case["kind"] == "layout":
        rows = sum(f * h * w + t for f, h, w, t in _shapes(case))
        return {"bytes": 20 * case["requests"] + 4 + 16 * rows, "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rotary":
        values = case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        return {"bytes": 2 * size * values + 4 * case["tokens"] * case["axes"], "flops": 3 * values}
    q, k = (sum(n[i] for n in _lengths(case)) for i in (0, 1))
    return {"bytes": 2 * size * case["head_dim"] * (q * case["q_heads"] + k * case["k_heads"]), "flops": 4 * case["head_dim"] * case["q_heads"] * _pairs_seen(case)}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    order = random.Random(seed)
    s = {"case": case}
    if case["kind"] == "layout":
        shapes = [(f, *order.sample((h, w), 2), t) for f, h, w, t in _shapes(case)]
        order.shuffle(shapes)
        rows = sum(f * h * w + t for f, h, w, t in shapes)
        s["shapes"] = torch.tensor(shapes, dtype=torch.int32).cuda()
        s["offsets"] = torch.empty(len(shapes) + 1, dtype=torch.int32, device="cuda")
        s["request"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        s["positions"] = torch.empty(rows, 3, dtype=torch.int32, device="cuda")
        return s
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, hq, hk, d = DT[case["dtype"]], case["q_heads"], case["k_heads"], case["head_dim"]
    if case["kind"] == "rotary":
        # queries and keys lie in the projection's output, beside the values
        n = case["tokens"]
        s["qkv"] = torch.randn(n, hq + 2 * hk, d, generator=gen, device="cuda").to(dt)
        s["q"], s["k"] = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hk]
        s["positions"] = torch.randint(0, case["far"], (n, case["axes"]), generator=gen, device="cuda", dtype=torch.int32)
        s["q_out"], s["k_out"] = torch.empty(n, hq, d, device="cuda", dtype=dt), torch.empty(n, hk, d, device="cuda", dtype=dt)
        return s
    lengths = _lengths(case)
    order.shuffle(lengths)
    nq, nk = ([n[i] for n in lengths] for i in (0, 1))
    s["max_q"], s["max_k"] = max(nq), max(nk)
    s["cu_q"], s["cu_k"] = (torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32).cuda() for n in (nq, nk))
    # scores of standard deviation 1.5 before the softmax
    q_std = 1.5 * (LOG2E / math.sqrt(d) if case["prescaled"] else 1.0)
    if case["new"]:
        s["q"] = (q_std * torch.randn(sum(nq), hq, d, generator=gen, device="cuda")).to(dt)
        kv = torch.randn(sum(nk), 2 * hk, d, generator=gen, device="cuda").to(dt)
        s["k"], s["v"] = kv[:, :hk], kv[:, hk:]
    else:
        qkv = torch.randn(sum(nq), hq + 2 * hk, d, generator=gen, device="cuda")
        qkv[:, :hq] *= q_std
        qkv = qkv.to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    s["o"] = torch.empty(sum(nq), hq, d, device="cuda", dtype=dt)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"layout": _own_layout, "rotary": _own_rotary, "attention": _own_attention}[kind](s)
    return {"layout": _plain_layout, "rotary": _plain_rotary, "attention": _plain_attention}[kind](s)


def _own_layout(s):
    hb = s.get("hb")
    if hb is None:
        from paper_2602_21760_amd import binding as hb
        s["hb"] = hb
    hb.hyb_packed_layout(s["shapes"], s["offsets"], s["request"], s["positions"], s["case"]["text_after"])
    return s["offsets"], s["request"], s["positions"]


def _own_rotary(s):
    desc = s.get("desc")
    if desc is None:
        from paper_2602_21760_amd import binding as hb
        c = s["case"]
        s["hb"] = hb
        desc = s["desc"] = hb.rotary_desc(s["q"], s["k"], _axis_dims(c), theta=10000.0, pairs=hb.HYB_ROTARY_HALVES if c["pairs"] == "halves" else hb.HYB_ROTARY_NEIGHBOURS,
                                          q_scale=LOG2E / math.sqrt(c["head_dim"]) if c["q_scaled"] else 1.0, inverse=c["inverse"], q_out=s["q_out"], k_out=s["k_out"])
    s["hb"].hyb_rotary(desc, s["positions"], s["q"], s["k"], s["q_out"], s["k_out"])
    return s["q_out"], s["k_out"]


def _own_attention(s):
    desc = s.get("desc")
    if desc is None:
        from paper_2602_21760_amd import binding as hb
        s["hb"] = hb
        desc = s["desc"] = hb.packed_attention_desc(s["q"], s["k"], s["v"], s["o"], s["cu_q"], s["max_q"], s["max_k"], causal=s["case"]["causal"],
                                                    prescaled=s["case"]["prescaled"])
        s["ws"] = torch.empty(hb.hyb_packed_attention_workspace_bytes(desc), device="cuda", dtype=torch.uint8)
    s["hb"].hyb_packed_attention(desc, s["q"], s["k"], s["v"], s["o"], s["cu_q"], s["cu_k"], s["ws"])
    return s["o"]


def _plain_layout(s):
    shapes = s["shapes"].long()
    f, h, w, t = shapes.unbind(1)
    images = f * h * w
    offsets = torch.zeros(len(shapes) + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum(images + t, 0)
    row = torch.arange(s["request"].shape[0], device="cuda")
    req = torch.searchsorted(offsets[1:].contiguous(), row, right=True)
    i = row - offsets[req]
    hw = h * w
    image = torch.stack((i // hw[req], i % hw[req] // w[req], i % w[req]), 1)
    text = i - images[req]
    text = (text + torch.maximum(f, torch.maximum(h, w))[req] if s["case"]["text_after"] else torch.zeros_like(text))[:, None].expand(-1, 3)
    return offsets.int(), req.int(), torch.where((i < images[req])[:, None], image, text).int()


def _plain_rotary(s):
    c = s["case"]
    dims = _axis_dims(c)
    # angle of every pair of every token, in 64 bits
    freq = torch.cat([10000.0 ** (-torch.arange(0, n, 2, dtype=torch.float64, device="cuda") / n) for n in dims])
    axis = torch.cat([torch.full((n // 2,), a, dtype=torch.int64, device="cuda") for a, n in enumerate(dims)])
    angle = s["positions"].double()[:, axis] * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin
    width = sum(dims)

    def rotate(x, scale):
        x = x.float() * scale
        turned = x.clone()
        if c["pairs"] == "halves":
            a, b = x[..., :width // 2], x[..., width // 2:width]
            turned[..., :width // 2], turned[..., width // 2:width] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = x[..., 0:width:2], x[..., 1:width:2]
            turned[..., 0:width:2], turned[..., 1:width:2] = a * cos - b * sin, a * sin + b * cos
        return turned.to(s["q"].dtype)
    return rotate(s["q"], LOG2E / math.sqrt(c["head_dim"]) if c["q_scaled"] else 1.0), rotate(s["k"], 1.0)


def _plain_attention(s):
    c = s["case"]
    hq, hk, d = c["q_heads"], c["k_heads"], c["head_dim"]
    nq, nk = s["cu_q"].diff(), s["cu_k"].diff()
    # every sequence padded to the longest: [sequence, head, row, feature] in 32 bits
    iq, ik = torch.arange(s["max_q"], device="cuda"), torch.arange(s["max_k"], device="cuda")

    def padded(x, cu, i):
        at = (cu[:-1, None] + i).clamp(max=x.shape[0] - 1)
        return x[at].float().permute(0, 2, 1, 3).repeat_interleave(hq // x.shape[1], 1).contiguous()
    q, k, v = padded(s["q"], s["cu_q"], iq), padded(s["k"], s["cu_k"], ik), padded(s["v"], s["cu_k"], ik)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous())
    scores *= math.log(2.0) if c["prescaled"] else 1.0 / math.sqrt(d)
    last = (nk - nq)[:, None] + iq if c["causal"] else (nk - 1)[:, None].expand(-1, len(iq))     # the last key that a query sees
    seen = ik <= torch.minimum(last, (nk - 1)[:, None])[:, :, None]
    scores.masked_fill_(~seen[:, None], -math.inf)
    top = scores.amax(3, keepdim=True)
    scores -= torch.where(top == -math.inf, 0.0, top)
    scores.exp_()
    total = scores.sum(3, keepdim=True)
    o = torch.matmul(scores, v) / torch.where(total == 0.0, 1.0, total)
    row = torch.arange(s["q"].shape[0], device="cuda")
    of = torch.searchsorted(s["cu_q"][1:].contiguous(), row.int(), right=True)
    return o.permute(0, 2, 1, 3)[of, row - s["cu_q"][of]].to(s["q"].dtype)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "layout":
        return None
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(s)
    return _exact_attention(s)


def _exact_rotary(s):
    """Pairs as complex numbers times e^(i angle)."""
    c = s["case"]
    turns = []
    for a, n in enumerate(_axis_dims(c)):
        for j in range(n // 2):
            turns.append(s["positions"][:, a].double() * math.exp(-2.0 * j / n * math.log(10000.0)))
    angle = torch.stack(turns, 1) * (-1.0 if c["inverse"] else 1.0)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    half = angle.shape[1]

    def rotate(x, scale):
        out = x.double() * scale
        z = torch.complex(out[..., :half], out[..., half:2 * half]) if c["pairs"] == "halves" else torch.view_as_complex(out[..., :2 * half].unflatten(-1, (half, 2)).contiguous())
        z = z * turn
        out[..., :2 * half] = torch.cat((z.real, z.imag), -1) if c["pairs"] == "halves" else torch.view_as_real(z).flatten(-2)
        return out
    return rotate(s["q"], LOG2E / math.sqrt(c["head_dim"]) if c["q_scaled"] else 1.0), rotate(s["k"], 1.0)


def _exact_attention(s):
    """Sequence by sequence and head by head."""
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    cu_q, cu_k = s["cu_q"].tolist(), s["cu_k"].tolist()
    group = c["q_heads"] // c["k_heads"]
    for n in range(len(cu_q) - 1):
        nq, nk = cu_q[n + 1] - cu_q[n], cu_k[n + 1] - cu_k[n]
        k, v = s["k"][cu_k[n]:cu_k[n + 1]].double(), s["v"][cu_k[n]:cu_k[n + 1]].double()
        hidden = torch.ones(nq, nk, dtype=torch.bool, device="cuda").triu(nk - nq + 1) if c["causal"] else None
        for h in range(c["q_heads"]):
            z = s["q"][cu_q[n]:cu_q[n + 1], h].double() @ k[:, h // group].t() * (math.log(2.0) if c["prescaled"] else c["head_dim"] ** -0.5)
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            out[cu_q[n]:cu_q[n + 1], h] = torch.softmax(z, 1) @ v[:, h // group]
    return out
