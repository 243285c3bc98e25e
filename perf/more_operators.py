"""The operators of batches over a paged cache, as calls whose speed this repository is measured by, with plain forms of them.

A server decodes several sequences at once.  Their keys and values lie in pages of one cache: position p of sequence s is
row p % page of page table[s][p // page].  The rows of a call are packed: those of sequence s are starts[s] ..
starts[s + 1] - 1, the last positions of its lengths[s].

  append  norms of the queries' and keys' heads, rotary embedding, and keys and values into the pages
  attend  attention of the new rows over the pages: one token a sequence, chains of drafts, or a prompt's next chunk
  prompt  causal attention of whole packed prompts over keys and values that are packed like their queries

A case is a dict: "op", the shape ("heads", "kv_heads", "head_dim", "dtype" of the cache, "x" the type of queries and outputs),
"seqs" sequences of "rows_lo" to "rows_hi" new rows after "past_lo" to "past_hi" cached positions, "page" positions of a page,
and "mix" (a number that gives the sizes within those ranges).  Heads and widths are those of the 7B, 13B and 70B shapes and
of the tiny float32 model.
"""

import math
import random

import torch

own = False

SHAPES = {
    # query heads, kv heads, head_dim, cache type
    "tiny": (4, 4, 64, "f32"),
    "7b": (32, 32, 128, "bf16"),
    "13b": (40, 40, 128, "bf16"),
    "70b": (64, 8, 128, "bf16"),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _case(name, op, model, x, seqs, rows, past=(0, 0), page=16, mix=0, **more):
    heads, kv_heads, head_dim, dtype = SHAPES[model]
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "x": x, "seqs": seqs,
         "rows_lo": rows[0], "rows_hi": rows[1], "past_lo": past[0], "past_hi": past[1], "page": page, "mix": mix}
    c.update(more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # A decode step of a small batch, as every layer rotates and stores its tokens; latency only.
        _case("append 70b 16 tokens", "append", "70b", "f32", 16, (1, 1), (3, 2000), 16, 1),
        # Packed prompts with normed heads, far past the trained context.
        _case("append 70b prompts, norms", "append", "70b", "bf16", 5, (90, 700), (0, 1000), 64, 2, norm=True, far=40000,
              scaling="yarn", factor=16.0),
        # The smallest call: tokens of the tiny float32 model; latency only.
        _case("token tiny 3 sequences", "attend", "tiny", "f32", 3, (1, 1), (0, 60), 16, 3),
        # A decode step with as many kv heads as query heads, ragged contexts.
        _case("token 13b 8 sequences", "attend", "13b", "f32", 8, (1, 1), (100, 1500), 16, 4),
        # A busy server: bound by the read of the pages.
        _case("token 70b 64 sequences", "attend", "70b", "bf16", 64, (1, 1), (500, 8000), 64, 5),
        # One long document: the context is split over the chip.
        _case("token 70b 60k", "attend", "70b", "f32", 1, (1, 1), (60001, 60001), 128, 6),
        # Verification of chains of drafts.
        _case("chains 70b 12 sequences", "attend", "70b", "f32", 12, (2, 13), (300, 4000), 32, 7),
        # A prompt's chunk behind what is cached of it.
        _case("chunk 70b after 15k", "attend", "70b", "bf16", 1, (1000, 1000), (15111, 15111), 64, 8),
        # Short prompts of the tiny float32 model.
        _case("prompt tiny 5 packed", "prompt", "tiny", "f32", 5, (1, 60), mix=9),
        # The prompt of a 1024 + 512 token decode, all but its last token, in the framework's float32 activations.
        _case("prompt 13b 1023 rows", "prompt", "13b", "f32", 1, (1023, 1023), mix=10),
        # Ragged prompts with grouped heads.
        _case("prompt 70b 16 packed", "prompt", "70b", "bf16", 16, (30, 1500), mix=11),
        # A long document.
        _case("prompt 7b 8000 rows", "prompt", "7b", "bf16", 1, (8000, 8000), mix=12),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend", "prompt", "prompt"])
    model = rng.choice(["tiny", "7b", "13b", "70b", "70b"])
    mix, page, x = rng.randint(13, 10**6), rng.choice([16, 32, 64, 128, 256]), rng.choice(["f32", "bf16"])
    heads, _, head_dim, _ = SHAPES[model]
    more = {"dtype": "f32"} if rng.random() < 0.15 else {}
    if op == "append":
        hi = log_int(1, 700)
        past = log_int(1, 1500)
        if rng.random() < 0.4:
            more["norm"] = True
        if rng.random() < 0.4:
            more["layout"] = "interleaved"
        if rng.random() < 0.4:
            more["rotary_dim"] = rng.choice([head_dim // 4, head_dim // 2, 3 * head_dim // 4])
        more.update(rng.choice([{}, {"far": 40000, "scaling": "yarn", "factor": 8.0}, {"scaling": "linear", "factor": 2.0}]))
        return _case(None, op, model, x, log_int(1, max(1, 1500 // hi)), (max(1, hi // 4), hi), (0, past), page, mix, **more)
    if op == "attend":
        hi = rng.choice([1, 1, 1, rng.randint(2, 16), log_int(17, 500)])
        past = log_int(1, 60000 if hi == 1 and model == "70b" else 8000 if model == "70b" else 4000)
        if "dtype" in more or model == "tiny":
            past = min(past, 4000)
        # keys and scores of at most the listed cases'
        most = min(64, (500000 if model == "70b" else 100000) // (past + hi), 2 * 10**8 // (hi * heads * (past + hi)))
        return _case(None, op, model, x, log_int(1, max(1, most)), (rng.choice([1, hi]), hi), (rng.randint(0, past), past), page, mix,
                     **more)
    hi = log_int(1, 700 if "dtype" in more else 4000)
    most = min(24, 10**9 // (heads * hi * hi))
    return _case(None, op, model, x, log_int(1, max(1, most)), (max(1, hi // rng.choice([1, 8, 100])), hi), mix=mix, **more)


# ----------------------------------------------------------------------------
# inputs


def _sizes(case):
    """New rows and cached positions of each sequence; the largest of each range are there."""
    rng = random.Random(case["mix"])
    rows = [case["rows_hi"]] + [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["seqs"] - 1)]
    past = [rng.randint(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"] - 1)] + [case["past_hi"]]
    return rows, past


def prepare(case, seed):
    H, KVH, D, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    dt, xt = TYPES[case["dtype"]], TYPES[case["x"]]
    rows, past = _sizes(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + case["mix"] + 17)

    def normal(*shape, dtype=torch.float32, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    n = sum(rows)
    starts = [0]
    for m in rows:
        starts.append(starts[-1] + m)
    s = {"op": case["op"], "heads": H, "starts": ints(starts), "max_rows": max(rows)}
    if case["op"] == "prompt":
        s["q"] = normal(n, H, D, dtype=xt)
        kv = normal(2, n, KVH, D, dtype=dt)  # packed like the queries
        s["k"], s["v"] = kv[0].transpose(0, 1), kv[1].transpose(0, 1)
        return s
    lengths = [p + m for p, m in zip(past, rows)]
    pages = [-(-length // page) for length in lengths]
    order = list(range(sum(pages)))
    random.Random(int(seed) * 31 + case["mix"]).shuffle(order)
    table, at = [], 0
    for c in pages:  # what a sequence does not have yet has no page
        table.append(order[at:at + c] + [-1] * (max(pages) - c))
        at += c
    s["table"], s["lengths"], s["max_length"] = ints(table), ints(lengths), max(lengths)
    s["k"], s["v"] = normal(at, KVH, page, D, dtype=dt), normal(at, KVH, page, D, dtype=dt)
    if case["op"] == "attend":
        s["q"] = normal(n, H, D, dtype=xt)
        return s
    s["qkv"] = normal(n, (H + 2 * KVH) * D, dtype=xt)
    R = case.get("rotary_dim", D)
    s["rope"] = {"base": 10000.0, "rotary_dim": R, "layout": case.get("layout", "half"), "scaling": case.get("scaling", "none"),
                 "factor": case.get("factor", 1.0), "original_context": 4096, "beta_fast": 32.0, "beta_slow": 1.0}
    s["positions"] = None
    if "far" in case:  # the cache holds the end of a longer text
        s["positions"] = ints([case["far"] + length - m + i for length, m in zip(lengths, rows) for i in range(m)])
    s["q_norm"] = normal(D, dtype=dt, std=0.2, mean=1.0) if case.get("norm") else None
    s["k_norm"] = normal(D, dtype=dt, std=0.2, mean=1.0) if case.get("norm") else None
    return s


# ----------------------------------------------------------------------------
# the operators


def run(s):
    return {"append": _append, "attend": _attend, "prompt": _prompt}[s["op"]](s)


def _rows_of(s, n):
    """Of each row: its sequence, and its number there; of each sequence: its rows."""
    row = torch.arange(n, device="cuda")
    starts = s["starts"].long()
    seq = (row[:, None] >= starts[None, 1:]).sum(dim=1)
    return seq, row - starts[seq], starts[1:] - starts[:-1]


def _append(s):
    qkv, k, v, H = s["qkv"], s["k"], s["v"], s["heads"]
    if own:
        from paper_2309_08168_amd import binding

        batch = binding.batch(s["table"], s["lengths"], s["starts"], s["max_rows"], s["max_length"])
        q = binding.paged_append(binding.rope(**s["rope"]), qkv, k, v, batch, H, positions=s["positions"], q_norm=s["q_norm"],
                                 k_norm=s["k_norm"], eps=EPS)
        return {"q": q, "k": k, "v": v}
    r = s["rope"]
    KVH, page, D = k.shape[1:]
    R, n = r["rotary_dim"], qkv.shape[0]
    seq, i, m = _rows_of(s, n)
    slot = s["lengths"].long()[seq] - m[seq] + i
    positions = slot if s["positions"] is None else s["positions"]
    freq = torch.pow(r["base"], -2.0 * torch.arange(R // 2, dtype=torch.float64, device="cuda") / R)
    gain = 1.0
    if r["scaling"] == "linear":
        freq = freq / r["factor"]
    elif r["scaling"] == "yarn":
        turns = freq * (r["original_context"] / (2 * math.pi))
        part = ((turns - r["beta_slow"]) / (r["beta_fast"] - r["beta_slow"])).clamp(0.0, 1.0)
        freq = freq * (part + (1.0 - part) / r["factor"])
        gain = 0.1 * math.log(r["factor"]) + 1.0
    angle = positions.double()[:, None, None] * freq
    cos, sin = (angle.cos() * gain).float(), (angle.sin() * gain).float()
    x = qkv.float().view(n, H + 2 * KVH, D)
    qk = x[:, :H + KVH]
    if s["q_norm"] is not None:
        weight = torch.cat([s["q_norm"].float().expand(H, D), s["k_norm"].float().expand(KVH, D)])
        qk = qk * torch.rsqrt((qk * qk).mean(dim=-1, keepdim=True) + EPS) * weight
    if r["layout"] == "half":
        a, b = qk[..., :R // 2], qk[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = qk[..., 0:R:2], qk[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    out = torch.cat([turned, qk[..., R:]], dim=-1)
    to = s["table"].long()[seq, slot // page]
    k[to, :, slot % page] = out[:, H:].to(k.dtype)
    v[to, :, slot % page] = x[:, H + KVH:].to(v.dtype)
    return {"q": out[:, :H].to(qkv.dtype), "k": k, "v": v}


def _softmax(q, keys, values, visible):
    """q [seqs, kv heads, rows, D], keys and values [seqs, kv heads, positions, D], visible [seqs, 1, rows, positions]; float32."""
    scores = torch.matmul(q, keys.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(q.shape[3]))
    scores = scores.masked_fill(~visible, float("-inf"))
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, values) / torch.where(total == 0, torch.ones_like(total), total)


def _padded(s, q, KVH):
    """The packed queries as [seqs, kv heads, most rows * heads of a kv head, D], float32; the packed row of each padded one."""
    n, H, D = q.shape
    M, G = s["max_rows"], H // KVH
    row = (s["starts"][:-1, None].long() + torch.arange(M, device="cuda")).clamp(max=n - 1)
    return q[row].float().view(-1, M, KVH, G, D).permute(0, 2, 1, 3, 4).reshape(-1, KVH, M * G, D), row


def _packed(s, o, seq, i, H):
    """The rows that there are, of the padded form."""
    S, KVH, _, D = o.shape
    M, G = s["max_rows"], H // KVH
    return o.view(S, KVH, M, G, D).permute(0, 2, 1, 3, 4).reshape(S, M, H, D)[seq, i]


def _attend(s):
    q, k, v = s["q"], s["k"], s["v"]
    if own:
        from paper_2309_08168_amd import binding

        batch = binding.batch(s["table"], s["lengths"], s["starts"], s["max_rows"], s["max_length"])
        return binding.paged_attention(q, k, v, batch)
    n, H, D = q.shape
    KVH, G, M = k.shape[1], H // k.shape[1], s["max_rows"]
    seq, i, m = _rows_of(s, n)
    pages = s["table"].long().clamp(min=0)
    keys = k[pages].permute(0, 2, 1, 3, 4).flatten(2, 3).float()
    values = v[pages].permute(0, 2, 1, 3, 4).flatten(2, 3).float()
    rows, _ = _padded(s, q, KVH)
    last = s["lengths"].long()[:, None] - m[:, None] + torch.arange(M, device="cuda")  # the position of each padded row
    seen = torch.arange(keys.shape[2], device="cuda") <= last[:, :, None]
    o = _softmax(rows, keys, values, seen.repeat_interleave(G, dim=1)[:, None])
    return _packed(s, o, seq, i, H).to(q.dtype)


def _prompt(s):
    q, k, v = s["q"], s["k"], s["v"]
    if own:
        from paper_2309_08168_amd import binding

        return binding.prompt_attention(q, k, v, s["starts"])
    n, H, D = q.shape
    KVH, G, M = k.shape[0], H // k.shape[0], s["max_rows"]
    seq, i, _ = _rows_of(s, n)
    rows, at = _padded(s, q, KVH)
    keys, values = (t[:, at].transpose(0, 1).float() for t in (k, v))
    seen = torch.ones(M, M, dtype=torch.bool, device="cuda").tril().repeat_interleave(G, dim=0)
    o = _softmax(rows, keys, values, seen[None, None])
    return _packed(s, o, seq, i, H).to(q.dtype)


# ----------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    H, KVH, D = case["heads"], case["kv_heads"], case["head_dim"]
    c, x = (2 if case[t] == "bf16" else 4 for t in ("dtype", "x"))
    rows, past = _sizes(case)
    n, S = sum(rows), case["seqs"]
    if case["op"] == "append":
        return {"bytes": x * n * (2 * H + 2 * KVH) * D + 2 * c * n * KVH * D + 8 * S,
                "flops": n * (H + KVH) * (3 * case.get("rotary_dim", D) + (4 * D if case.get("norm") else 0))}
    pairs = sum(m * p + m * (m + 1) // 2 for m, p in zip(rows, past))
    return {"bytes": 2 * x * n * H * D + 2 * c * (n + sum(past)) * KVH * D + 8 * S, "flops": 4 * pairs * H * D}


# ----------------------------------------------------------------------------
# the definitions in 64 bits, sequence by sequence


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "prompt": _exact_prompt}[case["op"]](s, *_sizes(case))


def _exact_append(s, rows, past):
    r, H = s["rope"], s["heads"]
    KVH, page, D = s["k"].shape[1:]
    n, R = s["qkv"].shape[0], r["rotary_dim"]
    x = s["qkv"].double().view(n, H + 2 * KVH, D)
    slots = [p + i for m, p in zip(rows, past) for i in range(m)]
    where = torch.tensor(slots, device="cuda") if s["positions"] is None else s["positions"]
    y = x.clone()
    if s["q_norm"] is not None:
        y = y / (y.square().sum(dim=-1, keepdim=True) / D + EPS).sqrt()
        y[:, :H] *= s["q_norm"].double()
        y[:, H:] *= s["k_norm"].double()
    out = y.clone()
    for i in range(R // 2):
        f, gain = r["base"] ** (-2.0 * i / R), 1.0
        if r["scaling"] == "linear":
            f /= r["factor"]
        elif r["scaling"] == "yarn":
            t = f * r["original_context"] / (2 * math.pi)
            w = min(1.0, max(0.0, (t - r["beta_slow"]) / (r["beta_fast"] - r["beta_slow"])))
            f = w * f + (1.0 - w) * f / r["factor"]
            gain = 1.0 + 0.1 * math.log(r["factor"])
        e = (i, i + R // 2) if r["layout"] == "half" else (2 * i, 2 * i + 1)
        turn = torch.polar(torch.full((n, 1), gain, dtype=torch.float64, device="cuda"), where.double()[:, None] * f)
        z = torch.complex(y[:, :, e[0]].contiguous(), y[:, :, e[1]].contiguous()) * turn
        out[:, :, e[0]], out[:, :, e[1]] = z.real, z.imag
    k, v, table = s["k"].double(), s["v"].double(), s["table"].tolist()
    row = 0
    for seq, m in enumerate(rows):
        for _ in range(m):
            b, o = table[seq][slots[row] // page], slots[row] % page
            k[b, :, o], v[b, :, o] = out[row, H:H + KVH], x[row, H + KVH:]
            row += 1
    return {"q": out[:, :H].contiguous(), "k": k, "v": v}


def _exact_rows(q, keys, values, past):
    """q [m, G, D], keys and values [past + m, D] of one kv head."""
    m, G, D = q.shape
    scores = (q.double().reshape(m * G, D) @ keys.t().contiguous() / math.sqrt(D)).view(m, G, -1)
    later = torch.arange(past + m, device="cuda")[None, :] > past + torch.arange(m, device="cuda")[:, None]
    p = torch.softmax(scores.masked_fill(later[:, None], -math.inf), dim=-1)
    return (p.view(m * G, -1) @ values).view(m, G, D)


def _exact_attend(s, rows, past):
    q, k, v = s["q"], s["k"], s["v"]
    KVH = k.shape[1]
    n, H, D = q.shape
    out, at = torch.zeros(n, H, D, dtype=torch.float64, device="cuda"), 0
    G = H // KVH
    for seq, (m, p) in enumerate(zip(rows, past)):
        length = p + m
        pages = s["table"][seq, :-(-length // k.shape[2])].long()
        for g in range(KVH):
            keys, values = (t[pages, g].reshape(-1, D)[:length].double() for t in (k, v))
            out[at:at + m, g * G:(g + 1) * G] = _exact_rows(q[at:at + m, g * G:(g + 1) * G], keys, values, p)
        at += m
    return out


def _exact_prompt(s, rows, past):
    q, k, v = s["q"], s["k"], s["v"]
    KVH = k.shape[0]
    n, H, D = q.shape
    out, at, G = torch.zeros(n, H, D, dtype=torch.float64, device="cuda"), 0, H // KVH
    for m in rows:
        for g in range(KVH):
            keys, values = (t[g, at:at + m].double() for t in (k, v))
            out[at:at + m, g * G:(g + 1) * G] = _exact_rows(q[at:at + m, g * G:(g + 1) * G], keys, values, 0)
        at += m
    return out
