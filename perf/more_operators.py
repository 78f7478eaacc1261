"""Timed cases of attention between packed sequences and of rotary positions.

A case is one call, or the calls of one training step, on packed tokens.
``op`` is
  "attend"  cross_attention: each image's queries attend to its keys;
  "learn"   cross_attention and cross_attention_backward, with all gradients;
  "rotate"  rotary, and rotary_backward of another gradient where ``train``;
  "encode"  rotary of queries and keys, cross_attention of the two, and the
            gradients of all of it back to the unrotated inputs.
``q`` and ``k`` list the images' lengths ("64x1024" is 64 images of 1024).
``heads`` query heads share ``kv_heads`` heads of keys and values, ``dim`` is the
width of a head.  ``mask`` is the share of keys that a key mask leaves (1: no mask);
masked keys hold what a padded batch's buffer happened to hold.

Rotary positions: pair p of a head's features turns by positions[t, axis(p)] *
frequencies[p] radians.  ``sections`` counts the pairs of each axis; features
after them are left.  Layout "halves" pairs feature p with p + pairs,
"interleaved" 2 p with 2 p + 1.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
# Largest drawn cases: flops, scores of the padded batch, values of one rotated tensor.
MAX_FLOPS = 6e11
MAX_SCORES = 1 << 31
MAX_ELEMS = 1 << 27


def _attend(name, op, q, k, heads, kv_heads, dim, dtype, mask=1.0, sections="", layout="halves", far=0.0):
    return {"name": name, "op": op, "q": q, "k": k, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "mask": mask, "sections": sections, "layout": layout, "far": far}


def _rotate(name, rows, heads, dim, dtype, sections, layout, far, train):
    return {"name": name, "op": "rotate", "rows": rows, "heads": heads, "dim": dim, "dtype": dtype, "sections": sections,
            "layout": layout, "far": far, "train": train}


def listed():
    # Images of a base encoder after one merge: 820 to 877 of 1024 tokens.
    merged = ",".join(str(820 + (37 * b) % 58) for b in range(64))
    # Mixed resolutions, 32 x 32 to 64 x 64 patches.
    mixed = "1600,4096,2x1600,1024,1600,1024,2304,2x4096,1024,3x1600,3x4096,5x1024,2x2304"
    # Captions of a batch.
    captions = "77,12,33,1,60,77,41,18,77,25,9,64,77,50,30,7"
    return [
        # A pooling token over one image, at the end of an encoder: launch and host time.
        _attend("attend_token", "attend", "1", "1024", 12, 12, 64, "bf16"),
        # One decoding step of 16 requests over long encoded videos, shared kv heads: bytes of the keys.
        _attend("attend_token_video", "attend", "16x1", "15x16384,12345", 32, 8, 128, "bf16"),
        # A mask decoder's queries over images of mixed resolution in a masked batch.
        _attend("attend_queries", "attend", "24x100", mixed, 8, 8, 32, "bf16", 0.8),
        # fp32 features, odd sizes on all sides, an image without queries and one without keys.
        _attend("attend_odd_f32", "attend", "197,1,0,577,33", "300,129,50,0,1023", 6, 3, 40, "f32"),
        # A base encoder's own tokens behind a merge.
        _attend("attend_vit_b", "attend", merged, merged, 12, 12, 64, "bf16"),
        # Wide heads, long queries over longer states, shared kv heads.
        _attend("attend_wide", "attend", "4x4096", "3x8192,7777", 16, 4, 128, "bf16"),
        # Tuning a small fp32 head.
        _attend("learn_odd_f32", "learn", "100,17,1,64", "785,197,1,0", 6, 6, 64, "f32", 0.9),
        # Image tokens that learn from captions: many queries, few keys, heads of 80.
        _attend("learn_captions", "learn", "16x4096", captions, 8, 8, 80, "bf16"),
        # Tuning a base encoder behind a merge.
        _attend("learn_vit_b", "learn", merged, merged, 12, 12, 64, "bf16"),
        # One new token of a stream: time, height and width; launch and host time.
        _rotate("rotate_token", 1, 40, 128, "bf16", "16,24,24", "halves", 1e5, False),
        # Queries and keys of a merged base batch, two axes, both directions.
        _rotate("rotate_vit_b", 54208, 24, 64, "bf16", "16,16", "interleaved", 0.0, True),
        # A step of video clips through one attention: positions, attention, all gradients.
        _attend("encode_video", "encode", "2x5000,1999", "2x5000,1999", 8, 2, 128, "bf16", 1.0, "16,24,24", "halves", 2e4),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(low * (high / low) ** rng.random())))


def _sections(rng, dim):
    axes = rng.choice([1, 2, 3])
    pairs = max(axes, dim // 2 if rng.random() < 0.7 else dim // 4)
    cut = [pairs // axes] * axes
    cut[-1] += pairs - sum(cut)
    return ",".join(map(str, cut))


def draw(rng):
    op = rng.choices(["attend", "learn", "rotate", "encode"], [5, 4, 3, 1])[0]
    dtype = rng.choices(["bf16", "f32"], [5, 2])[0]
    dim = rng.choices([64, 128, 8 * rng.randint(1, 16), rng.randint(6, 128)], [5, 4, 3, 1])[0]
    layout = rng.choice(["halves", "interleaved"])
    far = rng.choice([0.0, _log(rng, 10, 1000000) * 1.0])
    if op == "rotate":
        heads = _log(rng, 1, 64)
        rows = _log(rng, 1, max(1, min(100000, MAX_ELEMS // (heads * dim))))
        case = _rotate("", rows, heads, dim, dtype, _sections(rng, dim), layout, far, rng.random() < 0.6)
        del case["name"]
        return case
    kv_heads = rng.choice([1, 2, 3, 4, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    batch = _log(rng, 1, 64)
    top_q, top_k = _log(rng, 1, 8192), _log(rng, 1, 32768)
    if op == "encode" or rng.random() < 0.3:
        top_k = top_q
    if rng.random() < 0.25:
        top_q = rng.choice([1, 1, 2, 8])
    q = [max(0, round(top_q * rng.uniform(0.3, 1.0))) if top_q > 8 else top_q for _ in range(batch)]
    k = [max(0, round(top_k * rng.uniform(0.3, 1.0))) for _ in range(batch)]
    most = MAX_FLOPS * (1 if dtype == "bf16" else 0.1) * (1 if dim % 8 == 0 else 0.1) / {"attend": 4, "learn": 14, "encode": 14}[op]
    while len(q) > 1 and (sum(a * b for a, b in zip(q, k)) * heads * dim > most or
                          len(q) * max(q) * max(k) * heads > MAX_SCORES or
                          max(sum(k) * kv_heads, sum(q) * heads) * dim > MAX_ELEMS):
        q.pop()
        k.pop()
    while q[0] * k[0] * heads * max(dim, 64) > min(most, 64 * MAX_SCORES):
        q[0], k[0] = max(1, q[0] // 2), max(1, k[0] // 2)
    if sum(q) == 0 or op == "encode":
        q = [max(1, n) for n in q]
    if op == "encode":
        k = q
    if sum(k) == 0:
        k[0] = 1
    case = _attend("", op, ",".join(map(str, q)), ",".join(map(str, k)), heads, kv_heads, dim, dtype,
                   rng.choice([1.0, 1.0, 0.9, 0.5]), _sections(rng, dim) if op == "encode" else "", layout,
                   far if op == "encode" else 0.0)
    del case["name"]
    return case


def _counts(text):
    got = []
    for part in text.split(","):
        k, _, n = part.rpartition("x")
        got += [int(n)] * int(k or 1)
    return got


def work(case):
    e, d = BYTES[case["dtype"]], case["dim"]
    if case["op"] == "rotate":
        n = case["rows"] * case["heads"] * d * (2 if case["train"] else 1)
        return {"bytes": 2.0 * n * e, "flops": 3.0 * n}
    q, k = _counts(case["q"]), _counts(case["k"])
    nq, nk = sum(q) * case["heads"] * d, sum(k) * case["kv_heads"] * d
    products = 2.0 * sum(a * b for a, b in zip(q, k)) * case["mask"] * case["heads"] * d
    if case["op"] == "attend":  # q, k, v in, the output out
        return {"bytes": (2.0 * nq + 2 * nk) * e, "flops": 2 * products}
    # q, k, v and the output's gradient in, the output and three gradients out; scores, output, and five products back.
    return {"bytes": (4.0 * nq + 4 * nk) * e, "flops": 7 * products}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _positions(gen, rows, axes, far):
    """Time steps up to `far`, and centres of merged patches on a grid of 64: halves, quarters and so on."""
    at = torch.rand(rows, axes, generator=gen, device="cuda") * 64
    at = torch.round(at * 8) / 8
    if far > 0:
        at[:, 0] = torch.floor(torch.rand(rows, generator=gen, device="cuda") * far)
    return at


def _frequencies(sections, base=10000.0):
    """Axis by axis, pair i of n turns by base^(-i / n) radians a position."""
    return torch.tensor([base ** (-i / n) for n in sections for i in range(n)], dtype=torch.float64, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, d = DTYPES[case["dtype"]], case["dim"]

    def tokens(rows, heads, size=1.0):
        """Heads' features: of unequal size, around a mean of their own."""
        x = torch.randn(rows, heads, d, generator=gen, device="cuda")
        x *= torch.exp(0.3 * torch.randn(heads, d, generator=gen, device="cuda"))
        return (size * (x + 0.3 * torch.randn(heads, d, generator=gen, device="cuda"))).to(dtype)

    s = {"case": case, "scale": d ** -0.5}
    if case["sections"]:
        s["sections"] = tuple(int(n) for n in case["sections"].split(","))
        s["frequencies"] = _frequencies(s["sections"])
    if case["op"] == "rotate":
        s["x"] = tokens(case["rows"], case["heads"])
        s["positions"] = _positions(gen, case["rows"], len(s["sections"]), case["far"])
        if case["train"]:
            s["d_y"] = tokens(case["rows"], case["heads"])
        return s
    q, k = _counts(case["q"]), _counts(case["k"])
    s["q"], s["k"], s["v"] = tokens(sum(q), case["heads"]), tokens(sum(k), case["kv_heads"]), tokens(sum(k), case["kv_heads"])
    s["q_offsets"] = torch.tensor([0] + q, device="cuda").cumsum(0)
    s["k_offsets"] = torch.tensor([0] + k, device="cuda").cumsum(0)
    s["longest"] = (max(q), max(k))
    s["mask"] = None
    if case["mask"] < 1:
        s["mask"] = (torch.rand(sum(k), generator=gen, device="cuda") < case["mask"]).to(torch.uint8)
    if case["op"] != "attend":
        s["d_out"] = tokens(sum(q), case["heads"])
    if case["op"] == "encode":
        s["q_positions"] = _positions(gen, sum(q), len(s["sections"]), case["far"])
        s["k_positions"] = s["q_positions"]
    return s


# ---------------------------------------------------------------------------
# Plain form: elementary operations in fp32 on padded batches
# ---------------------------------------------------------------------------
def _pad(x, offsets, longest):
    """Packed [T, H, D] -> fp32 [B, H, longest, D] with zeros, and where a row is one [B, longest]."""
    at = torch.arange(longest, device=x.device)
    valid = at < (offsets[1:] - offsets[:-1])[:, None]
    row = torch.where(valid, offsets[:-1, None] + at, 0)
    full = torch.where(valid[:, :, None, None], x[row].float(), 0.0)
    return full.transpose(1, 2), valid


def _unpad(x, valid):
    return x.transpose(1, 2)[valid]


def _rotated(x, positions, frequencies, sections, layout, sign=1.0):
    """fp32 values of x [T, H, D] turned by the positions' angles; angles in 64 bits."""
    pairs = sum(sections)
    axis = torch.repeat_interleave(torch.arange(len(sections), device=x.device), torch.tensor(sections, device=x.device))
    angle = positions.double()[:, axis] * frequencies
    c, s = angle.cos().float()[:, None, :], sign * angle.sin().float()[:, None, :]
    v = x.float()
    out = v.clone()
    first = slice(0, pairs) if layout == "halves" else slice(0, 2 * pairs, 2)
    second = slice(pairs, 2 * pairs) if layout == "halves" else slice(1, 2 * pairs, 2)
    out[..., first] = v[..., first] * c - v[..., second] * s
    out[..., second] = v[..., first] * s + v[..., second] * c
    return out


def _probabilities(s, q, k):
    """Softmax over the keys that are there, [B, H, Lq, Lk] in fp32, and its padded operands; zeros where there is none."""
    group = s["q"].shape[1] // s["k"].shape[1]
    qp, q_valid = _pad(q, s["q_offsets"], s["longest"][0])
    kp, k_valid = _pad(k, s["k_offsets"], s["longest"][1])
    vp, _ = _pad(s["v"], s["k_offsets"], s["longest"][1])
    seen = k_valid
    if s["mask"] is not None:
        seen = k_valid.masked_scatter(k_valid, s["mask"].bool())
    kp, vp = kp.repeat_interleave(group, 1), vp.repeat_interleave(group, 1)
    score = torch.matmul(qp, kp.transpose(2, 3)) * s["scale"]
    score = torch.where(seen[:, None, None, :], score, -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(3, keepdim=True)
    return p / torch.where(total > 0, total, 1.0), qp, kp, vp, q_valid, k_valid


def _of_kv_heads(x, kv_heads):
    """Sums the query heads of each kv head."""
    b, h, n, d = x.shape
    return x.view(b, kv_heads, h // kv_heads, n, d).sum(2)


def _plain_attention(s, q, k, learn):
    """fp32 (out, d_q, d_k, d_v), packed."""
    p, qp, kp, vp, q_valid, k_valid = _probabilities(s, q, k)
    out = torch.matmul(p, vp)
    if not learn:
        return _unpad(out, q_valid), None, None, None
    g, _ = _pad(s["d_out"], s["q_offsets"], s["longest"][0])
    kv_heads = s["k"].shape[1]
    d_v = _of_kv_heads(torch.matmul(p.transpose(2, 3), g), kv_heads)
    d_score = p * (torch.matmul(g, vp.transpose(2, 3)) - (g * out).sum(3, keepdim=True)) * s["scale"]
    d_q = torch.matmul(d_score, kp)
    d_k = _of_kv_heads(torch.matmul(d_score.transpose(2, 3), qp), kv_heads)
    return _unpad(out, q_valid), _unpad(d_q, q_valid), _unpad(d_k, k_valid), _unpad(d_v, k_valid)


def _plain(s):
    case = s["case"]
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "rotate":
        how = (s["positions"], s["frequencies"], s["sections"], case["layout"])
        y = _rotated(s["x"], *how).to(dtype)
        return {"y": y, "d_x": _rotated(s["d_y"], *how, sign=-1.0).to(dtype)} if case["train"] else {"y": y}
    if case["op"] == "encode":
        how = (s["frequencies"], s["sections"], case["layout"])
        # The rotated queries and keys are tensors of the tokens' type.
        q = _rotated(s["q"], s["q_positions"], *how).to(dtype)
        k = _rotated(s["k"], s["k_positions"], *how).to(dtype)
        out, d_q, d_k, d_v = _plain_attention(s, q, k, True)
        return {"out": out.to(dtype), "d_q": _rotated(d_q, s["q_positions"], *how, sign=-1.0).to(dtype),
                "d_k": _rotated(d_k, s["k_positions"], *how, sign=-1.0).to(dtype), "d_v": d_v.to(dtype)}
    out, d_q, d_k, d_v = _plain_attention(s, s["q"], s["k"], case["op"] == "learn")
    if case["op"] == "attend":
        return {"out": out.to(dtype)}
    return {"out": out.to(dtype), "d_q": d_q.to(dtype), "d_k": d_k.to(dtype), "d_v": d_v.to(dtype)}


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _own(s):
    import paper_2604_05718_gb300 as mpm

    case = s["case"]
    if case["op"] == "rotate":
        how = dict(frequencies=s["frequencies"], sections=s["sections"], layout=case["layout"])
        y = mpm.rotary(s["x"], s["positions"], **how)
        return {"y": y, "d_x": mpm.rotary_backward(s["d_y"], s["positions"], **how)} if case["train"] else {"y": y}
    args = dict(q_offsets=s["q_offsets"], k_offsets=s["k_offsets"], key_mask=s["mask"], scale=s["scale"])
    if case["op"] == "attend":
        return {"out": mpm.cross_attention(s["q"], s["k"], s["v"], **args)[0]}
    q, k = s["q"], s["k"]
    if case["op"] == "encode":
        how = dict(frequencies=s["frequencies"], sections=s["sections"], layout=case["layout"])
        q, k = mpm.rotary(q, s["q_positions"], **how), mpm.rotary(k, s["k_positions"], **how)
    out, lse = mpm.cross_attention(q, k, s["v"], with_lse=True, **args)
    grads = mpm.cross_attention_backward(s["d_out"], q, k, s["v"], out, lse, **args)
    d_q, d_k = grads.d_q, grads.d_k
    if case["op"] == "encode":
        d_q = mpm.rotary_backward(d_q, s["q_positions"], **how, out=d_q)
        d_k = mpm.rotary_backward(d_k, s["k_positions"], **how, out=d_k)
    return {"out": out, "d_q": d_q, "d_k": d_k, "d_v": grads.d_v}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# From the definitions, in 64 bits, image by image
# ---------------------------------------------------------------------------
def _turn(x, positions, frequencies, sections, layout, back=False):
    """x as complex numbers times e^(i angle)."""
    pairs = sum(sections)
    place = positions.double().repeat_interleave(torch.tensor(sections, device=x.device), dim=1)
    angle = place * frequencies * (-1 if back else 1)
    unit = torch.complex(torch.cos(angle), torch.sin(angle))[:, None, :]
    head, tail = x[..., :2 * pairs].double(), x[..., 2 * pairs:].double()
    if layout == "halves":
        z = torch.complex(head[..., :pairs].contiguous(), head[..., pairs:].contiguous()) * unit
        return torch.cat([z.real, z.imag, tail], dim=-1)
    z = torch.view_as_complex(head.reshape(*head.shape[:-1], pairs, 2).contiguous()) * unit
    return torch.cat([torch.view_as_real(z).flatten(-2), tail], dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        how = (s["positions"], s["frequencies"], s["sections"], case["layout"])
        y = _turn(s["x"], *how)
        return {"y": y, "d_x": _turn(s["d_y"], *how, back=True)} if case["train"] else {"y": y}
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    if case["op"] == "encode":
        how = (s["frequencies"], s["sections"], case["layout"])
        # What attends are the rotated tensors in the tokens' type.
        q = _turn(s["q"], s["q_positions"], *how).to(DTYPES[case["dtype"]]).double()
        k = _turn(s["k"], s["k_positions"], *how).to(DTYPES[case["dtype"]]).double()
    learn = case["op"] != "attend"
    out, d_q, d_k, d_v = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    group = q.shape[1] // k.shape[1]
    q0 = k0 = 0
    for nq, nk in zip(_counts(case["q"]), _counts(case["k"])):
        rows, cols = slice(q0, q0 + nq), torch.arange(k0, k0 + nk, device="cuda")
        q0, k0 = q0 + nq, k0 + nk
        if s["mask"] is not None:
            cols = cols[s["mask"][cols] != 0]
        if nq == 0 or cols.numel() == 0:
            continue
        for h in range(q.shape[1]):
            qh, kh, vh = q[rows, h], k[cols, h // group], v[cols, h // group]
            p = torch.softmax(qh @ kh.t() * s["scale"], dim=1)
            out[rows, h] = p @ vh
            if learn:
                g = s["d_out"][rows, h].double()
                d_v[cols, h // group] += p.t() @ g
                t = g @ vh.t()
                t = p * (t - (p * t).sum(1, keepdim=True)) * s["scale"]
                d_q[rows, h] = t @ kh
                d_k[cols, h // group] += t.t() @ qh
    if not learn:
        return {"out": out}
    if case["op"] == "encode":
        d_q = _turn(d_q, s["q_positions"], *how, back=True)
        d_k = _turn(d_k, s["k_positions"], *how, back=True)
    return {"out": out, "d_q": d_q, "d_k": d_k, "d_v": d_v}
