"""What the operators around the cache are measured on: the preparation of a layer's queries and keys
(norm of every head, rotation by positions) with its gradient, and attention of sequences that
continue shared prompts.

A case describes one attention layer (heads, head_dim, window, tau) and the call:

  rotate    qk_norm_rope: queries, keys and values out of one projection's rows, normed, rotated by
            1 to 3 position axes, laid out as the cache's calls take them
  gradient  qk_norm_rope_backward: the gradients of those into the projection's, and of the weights
  decode    decode_attention_shared: the newest token of every sequence over its own cache and over
            the prompt that it continues
  question  prefix_attention: many tokens of every sequence (its own prompt) over the shared one,
            joined with their attention over the sequence itself

With `own` false, `run` computes the plain form of the same, in 32 bits with one rounding at the end.
"""

from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


def _rope(name, kind, **kw):
    c = {"name": name, "kind": kind, "tokens": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "rot_dim": 128, "adjacent": False, "axes": 1, "theta": 1e6, "start": 0, "norm": True,
         "dtype": "bf16"}
    c.update(kw)
    return c


def _shared(name, kind, **kw):
    c = {"name": name, "kind": kind, "batch": 16, "prefixes": 1, "prefix_min": 32768,
         "prefix_max": 32768, "own_min": 1, "own_max": 300, "tokens": 1, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "keep_min": 0.10, "keep_max": 0.33, "window": 128,
         "tau": 0.5}
    c.update(kw)
    return c


def listed():
    return [
        # one conversation, one token: the layer's first launch in every decoding step
        _rope("rotate_b1", "rotate", start=40000),
        # a decoding step of 64 sequences at far positions
        _rope("rotate_b64_far", "rotate", tokens=64, start=1000000),
        # prompts in pieces, an 8B-shaped layer (the most bytes)
        _rope("rotate_32k", "rotate", tokens=32768, start=0),
        # images and video between text: three axes, small heads, an odd number of tokens
        _rope("rotate_images_d64", "rotate", tokens=10007, q_heads=24, kv_heads=3, head_dim=64, rot_dim=64,
              axes=3, theta=1e4),
        # one training sequence
        _rope("gradient_16k", "gradient", tokens=16384),
        # a short odd one in 32 bits, half of every head rotated in neighbouring pairs
        _rope("gradient_half_fp32", "gradient", tokens=777, q_heads=8, kv_heads=2, head_dim=64, rot_dim=32,
              adjacent=True, theta=1e4, dtype="fp32"),
        # one short conversation on a small model: launches and host work
        _shared("decode_b1_2k_d64", "decode", batch=1, prefix_min=2048, prefix_max=2048, q_heads=8,
                kv_heads=2, head_dim=64, own_min=64, own_max=64),
        # the usual serving step behind one long system prompt
        _shared("decode_b16_32k", "decode"),
        # many sessions over one long document
        _shared("decode_b64_128k", "decode", batch=64, prefix_min=131072, prefix_max=131072, own_max=2000,
                keep_min=0.02, keep_max=0.15),
        # three prompts of different lengths among seven sequences; odd sizes, one head group of eight
        _shared("decode_b7_odd_d64", "decode", batch=7, prefixes=3, prefix_min=901, prefix_max=9973,
                q_heads=24, kv_heads=3, head_dim=64, own_max=77, window=100, tau=0.3),
        # four questions of up to 512 tokens about one document
        _shared("question_b4_32k", "question", batch=4, tokens=512, own_min=301, own_max=512),
        # a few drafts or words each about three prompts; odd sizes
        _shared("question_b7_odd_d64", "question", batch=7, prefixes=3, prefix_min=901, prefix_max=9973,
                q_heads=24, kv_heads=3, head_dim=64, tokens=37, own_min=3, own_max=37, window=100, tau=0.3),
    ]


SHAPES = [(32, 8, 128), (32, 8, 128), (8, 2, 64), (16, 2, 128), (24, 3, 64), (16, 1, 128), (8, 8, 128)]


def draw(rng):
    """One more case: sizes over the whole range of the listed ones, odd ones among them."""
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "rotate", "gradient", "gradient", "decode", "decode", "decode", "question"])
    hq, hk, d = rng.choice(SHAPES)
    if kind in ("rotate", "gradient"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        adjacent = rng.random() < 0.3
        c = _rope("", kind, q_heads=hq, kv_heads=hk, head_dim=d, adjacent=adjacent, dtype=dtype,
                  rot_dim=rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)]),
                  axes=rng.choice([1, 1, 1, 2, 3]), theta=rng.choice([1e4, 5e5, 1e6]),
                  start=rng.choice([0, 0, span(1, 2000000)]), norm=rng.random() < 0.8)
        most = 8192 if dtype == "fp32" else 16384
        c["tokens"] = span(1, most if kind == "rotate" else most // 2)
    else:
        c = _shared("", kind, q_heads=hq, kv_heads=hk, head_dim=d, tau=rng.choice([0.5, 0.5, 0.3, 0.7]),
                    window=rng.choice([128, 128, 64, span(16, 512)]))
        c["keep_min"] = round(rng.uniform(0.02, 0.15), 3)
        c["keep_max"] = round(c["keep_min"] + rng.uniform(0.0, 0.25), 3)
        if kind == "question":
            c["batch"] = rng.randint(1, 4)
            c["tokens"] = span(2, 500)
            c["own_min"], c["own_max"] = max(1, c["tokens"] * 2 // 3), c["tokens"]
            c["prefix_max"] = span(256, 16384)
        else:
            c["batch"] = span(1, 64)
            c["own_max"] = span(1, 1500)
            c["own_min"] = rng.randint(1, c["own_max"])
            c["prefix_max"] = span(64, 100000)
        c["prefixes"] = rng.choice([1, 1, 2, 3]) if c["batch"] > 2 else 1
        c["prefix_min"] = c["prefix_max"] if rng.random() < 0.5 else max(1, c["prefix_max"] // rng.randint(2, 20))
    del c["name"]
    return c


# ------------------------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _frac(i):
    return (0.6180339887498949 * (i + 1)) % 1.0


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, the ends among them."""
    if n == 1:
        return [hi]
    inner = [lo + int((hi - lo) * _frac(i)) for i in range(n - 2)]
    return [lo] + inner + [hi]


def _keep(case):
    """Keep rate of every KV head."""
    return [case["keep_min"] + (case["keep_max"] - case["keep_min"]) * _frac(h) for h in range(case["kv_heads"])]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _sections(case):
    """Rotated pairs of every axis: time, height, width."""
    n = case["rot_dim"] // 2
    if case["axes"] == 1:
        return [n]
    if case["axes"] == 2:
        return [n // 2, n - n // 2]
    return [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2]


def _rope_inputs(case, seed):
    g = _generator(seed)
    t, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    dt = _TYPES[case["dtype"]]
    x = {"qkv": (_randn(g, t, hq + 2 * hk, d) * (0.25 + 2.0 * torch.rand(t, 1, 1, generator=g, device="cuda"))).to(dt)}
    x["q_weight"] = 1.0 + 0.2 * _randn(g, d)
    x["k_weight"] = 1.0 + 0.2 * _randn(g, d)
    pos = torch.arange(t, device="cuda", dtype=torch.int32) + case["start"]
    if t <= 64:                                   # decoding: every row is another sequence
        pos = pos + torch.randint(0, 1000, (t,), generator=g, device="cuda", dtype=torch.int32)
    if case["axes"] > 1:
        # rows of patches: time moves slowly, height and width within a picture
        side = 32
        more = [case["start"] + (pos - case["start"]) % side] if case["axes"] == 2 else \
            [case["start"] + ((pos - case["start"]) // side) % side, case["start"] + (pos - case["start"]) % side]
        pos = torch.stack([case["start"] + (pos - case["start"]) // side] + more).to(torch.int32)
    x["positions"] = pos.contiguous()
    if case["kind"] == "gradient":
        x["dq"] = _randn(g, t, hq, d).to(dt)
        x["dk"] = _randn(g, t, hk, d).to(dt)
        x["dv"] = _randn(g, t, hk, d).to(dt)
    return x


def _split(case, qkv):
    hq, hk = case["q_heads"], case["kv_heads"]
    return qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]


def _sequences(case):
    """Lengths of the prompts, and for every sequence its prompt, its own tokens and the rows it asks for."""
    lengths = _spread(case["prefix_min"], case["prefix_max"], case["prefixes"])
    member = [int(_frac(7 * b + 3) * case["prefixes"]) % case["prefixes"] for b in range(case["batch"])]
    tokens = _spread(case["own_min"], case["own_max"], case["batch"])
    rows = list(tokens) if case["kind"] == "question" else [1] * case["batch"]
    return lengths, member, tokens, rows


def _theta(case):
    return math.log(case["tau"] / (1.0 - case["tau"]))


def _shared_inputs(case, seed):
    g = _generator(seed)
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    lengths, member, tokens, rows = _sequences(case)
    theta = _theta(case)
    # logits of unit variance around the mean that lets `keep` of them reach the threshold
    mu = torch.special.ndtri(torch.tensor(_keep(case), dtype=torch.float64)).float().cuda() + theta

    def some(n):
        return (_randn(g, n, hk, d).bfloat16(), _randn(g, n, hk, d).bfloat16(), (_randn(g, n, hk) + mu).contiguous())

    x = {"prefix": some(sum(lengths)), "own": some(sum(tokens)),
         "q": _randn(g, sum(rows), hq, d).bfloat16()}
    if case["kind"] == "question":
        # what attention over the sequences' own tokens leaves: averages of values, and their weights' logarithm
        x["own_out"] = (0.3 * _randn(g, sum(rows), hq, d)).bfloat16()
        x["own_lse"] = 4.0 + _randn(g, sum(rows), hq)
    return x


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    if case["kind"] in ("rotate", "gradient"):
        state = {"case": case, **_rope_inputs(case, seed)}
        if own:
            import paper_2605_14037_amd as spkv
            state["rope"] = spkv.Rope(case["head_dim"], rot_dim=case["rot_dim"], theta=case["theta"],
                                      sections=_sections(case), adjacent=case["adjacent"])
        return state
    x = _shared_inputs(case, seed)
    lengths, member, tokens, rows = _sequences(case)
    state = {"case": case, "q": x["q"]}
    if case["kind"] == "question":
        state["own_out"], state["own_lse"] = x["own_out"], x["own_lse"]
    if not own:
        state.update(x)
        return state
    import paper_2605_14037_amd as spkv
    w = case["window"]

    def filled(kvf, counts, n_seq):
        ev = sum(max(0, n - w) for n in counts) * case["kv_heads"]
        cache = spkv.SPKVCache(n_seq, case["q_heads"], case["kv_heads"], case["head_dim"],
                               max_context=max(counts) + 64, max_total_kept_tokens=ev + 64 * n_seq * case["kv_heads"],
                               window=w, tau=case["tau"])
        at, done, piece = _starts(counts), [0] * n_seq, 4096
        while any(a < n for a, n in zip(done, counts)):
            take = [min(piece, n - a) for a, n in zip(done, counts)]
            parts = [torch.cat([t[at[b] + done[b]:at[b] + done[b] + take[b]] for b in range(n_seq)]).contiguous()
                     for t in kvf]
            cache.append(*parts, _starts(take))
            done = [a + n for a, n in zip(done, take)]
        cache.stats()
        return cache

    state["prefix_cache"] = filled(x["prefix"], lengths, len(lengths))
    state["cache"] = filled(x["own"], tokens, len(tokens))
    state["sharing"] = spkv.PrefixSharing(state["prefix_cache"], member)
    state["cu"] = state["cache"].make_cu(_starts(rows))
    return state


# -------------------------------------------------------------------------- plain forms
def _angles(case, positions):
    """cos and sin [tokens, 1, pairs] of every rotated pair, angles in 64 bits."""
    n = case["rot_dim"] // 2
    inv = case["theta"] ** (-torch.arange(n, device="cuda", dtype=torch.float64) * 2.0 / case["rot_dim"])
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"),
                                   torch.tensor(_sections(case), device="cuda"))
    pos = positions.reshape(case["axes"], -1).double()
    angle = pos[axis].transpose(0, 1) * inv
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _pairs(case, x):
    """First and second elements of the rotated pairs, and what is not rotated."""
    r = case["rot_dim"]
    if case["adjacent"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def _joined(case, a, b, rest):
    if case["adjacent"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _rotated(case, x, cos, sin):
    a, b, rest = _pairs(case, x)
    return _joined(case, a * cos - b * sin, a * sin + b * cos, rest)


def _plain_rotate(s):
    c = s["case"]
    q, k, v = _split(c, s["qkv"])
    cos, sin = _angles(c, s["positions"])
    out = []
    for x, w in ((q, s["q_weight"]), (k, s["k_weight"])):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        out.append(_rotated(c, x, cos, sin).to(s["qkv"].dtype))
    return out[0], out[1], v.contiguous()


def _plain_gradient(s):
    c = s["case"]
    q, k, _ = _split(c, s["qkv"])
    cos, sin = _angles(c, s["positions"])
    dx, dw = [], []
    for x, w, dy in ((q, s["q_weight"], s["dq"]), (k, s["k_weight"], s["dk"])):
        g = _rotated(c, dy.float(), cos, -sin)
        if c["norm"]:
            x = x.float()
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            dw.append((g * x * r).sum(0).sum(0))
            u = g * w
            g = r * (u - x * (r * r * (u * x).mean(-1, keepdim=True)))
        dx.append(g.to(s["qkv"].dtype))
    return [torch.cat(dx + [s["dv"]], 1)] + dw


def _plain_shared(s):
    """Row by row of the definition: a key is seen inside the window or where its gate is on."""
    c = s["case"]
    hq, hk, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    group, w, theta = hq // hk, c["window"], _theta(c)
    lengths, member, tokens, rows = _sequences(c)
    at_p, at_o, at_r = _starts(lengths), _starts(tokens), _starts(rows)
    out = torch.empty(sum(rows), hq, d, device="cuda")
    lse = torch.empty(sum(rows), hq, device="cuda")
    dev = "cuda"
    # own tokens of every sequence side by side, padded to the longest
    most, whole = max(tokens), c["kind"] == "decode"
    for p, n_p in enumerate(lengths):
        seqs = [b for b in range(c["batch"]) if member[b] == p]
        if not seqs:
            continue
        row = torch.cat([torch.arange(at_r[b], at_r[b + 1], device=dev) for b in seqs])
        last = torch.cat([torch.arange(tokens[b] - rows[b], tokens[b], device=dev) for b in seqs])   # own position
        q = s["q"][row].float().reshape(len(row), hk, group, d) / math.sqrt(d)
        distance = n_p + last[:, None] - torch.arange(n_p, device=dev)[None]
        if whole:
            index = torch.tensor([[at_o[b] + min(j, tokens[b] - 1) for j in range(most)] for b in seqs], device=dev)
            back = last[:, None] - torch.arange(most, device=dev)[None]
        for h in range(hk):
            qh = q[:, h].reshape(-1, d).contiguous()
            k, v, f = (t[at_p[p]:at_p[p + 1], h] for t in s["prefix"])
            seen = (distance < w) | (f >= theta)[None]
            x = (qh @ k.float().t().contiguous()).reshape(len(row), group, n_p)
            x = x.masked_fill(~seen[:, None], -math.inf)
            if whole:
                ko, vo, fo = (t[:, h][index] for t in s["own"])
                seen = (back >= 0) & ((back < w) | (fo >= theta))
                y = torch.bmm(qh.reshape(len(row), group, d), ko.float().transpose(1, 2).contiguous())
                y = y.masked_fill(~seen[:, None], -math.inf)
                top = torch.maximum(x.amax(-1), y.amax(-1))[..., None]
                x, y = torch.exp(x - top), torch.exp(y - top)
                total = x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
                o = (x.reshape(-1, n_p) @ v.float().contiguous()).reshape(len(row), group, d) + torch.bmm(y, vo.float())
            else:
                own_lse = s["own_lse"][row][:, h * group:(h + 1) * group, None]
                top = torch.maximum(x.amax(-1, keepdim=True), own_lse)
                x, y = torch.exp(x - top), torch.exp(own_lse - top)
                total = x.sum(-1, keepdim=True) + y
                o = (x.reshape(-1, n_p) @ v.float().contiguous()).reshape(len(row), group, d)
                o = o + y * s["own_out"][row][:, h * group:(h + 1) * group].float()
            out[row, h * group:(h + 1) * group] = o / total
            lse[row, h * group:(h + 1) * group] = (top + torch.log(total))[..., 0]
    return out.bfloat16(), lse


def run(state):
    c = state["case"]
    if not own:
        if c["kind"] == "rotate":
            return _plain_rotate(state)
        if c["kind"] == "gradient":
            return _plain_gradient(state)
        return _plain_shared(state)
    import paper_2605_14037_amd as spkv
    if c["kind"] in ("decode", "question"):
        if c["kind"] == "decode":
            return state["cache"].decode_attention_shared(state["sharing"], state["q"], want_lse=True)
        return state["cache"].prefix_attention(state["sharing"], state["q"], state["cu"], state["own_out"],
                                               state["own_lse"])
    q, k, v = _split(c, state["qkv"])
    norm = {"q_weight": state["q_weight"], "k_weight": state["k_weight"], "eps": EPS} if c["norm"] else {}
    if c["kind"] == "rotate":
        return spkv.qk_norm_rope(q, k, state["positions"], state["rope"], v=v, **norm)
    grad = torch.empty(state["qkv"].shape, dtype=state["qkv"].dtype, device="cuda")
    dw = spkv.qk_norm_rope_backward(state["dq"], state["dk"], state["positions"], state["rope"], q=q, k=k,
                                    dv=state["dv"], out=_split(c, grad), **norm)
    return [grad] + list(dw)


# ------------------------------------------------------------------------------- work
def work(case):
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] in ("rotate", "gradient"):
        size = 2 if case["dtype"] == "bf16" else 4
        rows = case["tokens"] * (hq + 2 * hk)
        normed = case["tokens"] * (hq + hk)
        weights = 2 * d * 4 if case["norm"] else 0
        if case["kind"] == "rotate":
            return {"bytes": 2 * rows * d * size + case["tokens"] * case["axes"] * 4 + weights,
                    "flops": normed * d * (7 if case["norm"] else 3)}
        again = normed * d * size if case["norm"] else 0         # the forward's inputs
        return {"bytes": 2 * rows * d * size + again + case["tokens"] * case["axes"] * 4 + 2 * weights,
                "flops": normed * d * (14 if case["norm"] else 3)}
    lengths, member, tokens, rows = _sequences(case)
    w, keep, group = case["window"], _keep(case), hq // hk
    n_bytes = sum(rows) * hq * (2 * d * 2 + 4)                    # queries, outputs, their weights' logarithm
    flops = 0.0
    for k in keep:
        for p, n in enumerate(lengths):
            cols = sum(rows[b] for b in range(case["batch"]) if member[b] == p) * group
            if cols:
                n_bytes += (max(0, n - w) * k + min(n, w)) * 2 * d * 2
                flops += 4.0 * d * cols * (max(0, n - w) * k + min(n, w) * k)
        if case["kind"] == "decode":
            for n in tokens:
                kept = max(0, n - w) * k + min(n, w)
                n_bytes += kept * 2 * d * 2
                flops += 4.0 * d * group * kept
    if case["kind"] == "question":
        n_bytes += sum(rows) * hq * (2 * d + 4)
    return {"bytes": int(n_bytes), "flops": int(flops)}


# ------------------------------------------------------------------------------- exact
def _exact_rotate(case, x, positions, q_weight, k_weight):
    """Rotation as a product of complex numbers; differentiable in x and the weights."""
    hq, hk = case["q_heads"], case["kv_heads"]
    r, axis, inv = case["rot_dim"], [], []
    for a, n in enumerate(_sections(case)):
        axis += [a] * n
    for i in range(r // 2):
        inv.append(math.exp(-2.0 * i / r * math.log(case["theta"])))
    pos = positions.reshape(case["axes"], -1).to(torch.float64)
    phase = torch.stack([pos[a] * f for a, f in zip(axis, inv)], dim=1)
    turn = torch.polar(torch.ones_like(phase), phase)[:, None]
    if case["adjacent"]:
        first, second = torch.arange(0, r, 2, device="cuda"), torch.arange(1, r, 2, device="cuda")
    else:
        first = torch.arange(0, r // 2, device="cuda")
        second = first + r // 2
    out = []
    for rows, weight in ((x[:, :hq], q_weight), (x[:, hq:hq + hk], k_weight)):
        if case["norm"]:
            rows = rows / torch.sqrt(rows.pow(2).sum(-1, keepdim=True) / case["head_dim"] + EPS) * weight
        z = torch.complex(rows[..., first], rows[..., second]) * turn
        y = rows.clone()
        y[..., first] = z.real
        y[..., second] = z.imag
        out.append(y)
    return out[0], out[1], x[:, hq + hk:]


def _exact_shared(case, x):
    """Every row for itself: the keys it sees gathered, one softmax over them."""
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    group, w = hq // hk, case["window"]
    theta = torch.tensor(_theta(case), dtype=torch.float64).float().item()
    lengths, member, tokens, rows = _sequences(case)
    at_p, at_o, at_r = _starts(lengths), _starts(tokens), _starts(rows)
    out = torch.zeros(sum(rows), hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(sum(rows), hq, dtype=torch.float64, device="cuda")
    q = x["q"].double() * d ** -0.5
    for h in range(hk):
        on = [(x["prefix"][2][:, h] >= theta), (x["own"][2][:, h] >= theta)]
        heads = slice(h * group, (h + 1) * group)
        for p, n_p in enumerate(lengths):
            # long lists once for all rows: keys that some row can see, those with their gate on first
            mine = slice(at_p[p], at_p[p + 1])
            gate = on[0][mine]
            near = torch.zeros_like(gate)
            near[max(0, n_p - w):] = True
            kept = torch.nonzero(gate | near).flatten()
            k, v = x["prefix"][0][mine, h][kept].double(), x["prefix"][1][mine, h][kept].double()
            for b in range(case["batch"]):
                if member[b] != p:
                    continue
                first = tokens[b] - rows[b]
                for r0 in range(0, rows[b], 128):
                    n = min(128, rows[b] - r0)
                    here = slice(at_r[b] + r0, at_r[b] + r0 + n)
                    qq = q[here, heads].reshape(n * group, d)
                    own_pos = torch.arange(first + r0, first + r0 + n, device="cuda")
                    allowed = gate[kept][None] | (n_p + own_pos[:, None] - kept[None] < w)
                    score = (qq @ k.t()).reshape(n, group, -1)
                    score = torch.where(allowed[:, None], score, torch.full_like(score, -math.inf))
                    if case["kind"] == "decode":
                        t = tokens[b]
                        sl = slice(at_o[b], at_o[b] + t)
                        j = torch.arange(t, device="cuda")
                        ok = (j[None] <= own_pos[:, None]) & ((own_pos[:, None] - j[None] < w) | on[1][sl][None])
                        more = (qq @ x["own"][0][sl, h].double().t()).reshape(n, group, -1)
                        more = torch.where(ok[:, None], more, torch.full_like(more, -math.inf))
                        value = x["own"][1][sl, h].double()
                        both = torch.cat([score, more], -1)
                        z = torch.logsumexp(both, -1)
                        weight = torch.exp(both - z[..., None]).reshape(n * group, -1)
                        o = weight @ torch.cat([v, value])
                    else:
                        mine_lse = x["own_lse"][here, heads].double()
                        z = torch.logaddexp(torch.logsumexp(score, -1), mine_lse)
                        o = torch.exp(score - z[..., None]).reshape(n * group, -1) @ v
                        o = o + (torch.exp(mine_lse - z)[..., None] * x["own_out"][here, heads].double()).reshape(-1, d)
                    out[here, heads] = o.reshape(n, group, d)
                    lse[here, heads] = z
    return out, lse


def exact(case, seed):
    if case["kind"] in ("decode", "question"):
        return _exact_shared(case, _shared_inputs(case, seed))
    x = _rope_inputs(case, seed)
    rows = x["qkv"].double()
    wq, wk = x["q_weight"].double(), x["k_weight"].double()
    if case["kind"] == "rotate":
        return _exact_rotate(case, rows, x["positions"], wq, wk)
    # the gradient by reversing the definition itself
    rows.requires_grad_(True)
    wq.requires_grad_(True)
    wk.requires_grad_(True)
    y = _exact_rotate(case, rows, x["positions"], wq, wk)
    wanted = [rows, wq, wk] if case["norm"] else [rows]
    return list(torch.autograd.grad(y, wanted, [x["dq"].double(), x["dk"].double(), x["dv"].double()]))
