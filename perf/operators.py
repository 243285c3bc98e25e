"""The operators of tree drafts, as calls whose speed this repository is measured by, with plain forms of them.

A verification of a token tree scores several continuations of one prefix in a single forward: node 0 is the last
committed token, every other node a drafted token after its parent (parents come first), and the nodes' keys and values
stand behind the prefix in the cache.  Four operators make one up:

  rope    rotary embedding of a QKV product at given positions (a node's position is the prefix plus its depth; pairing in
          halves or interleaved, part of the head, frequencies scaled for long contexts), keys and values into the cache
  attend  attention of the nodes over the prefix and their own ancestors (one bit per pair of nodes)
  accept  the greedy walk: each node's best token, and the path of nodes that the model itself would have emitted
  keep    the cache rows of that path moved together, in every layer and head

A case is a dict: "op", the shape ("heads", "kv_heads", "head_dim", "dtype" of the cache), "n" nodes or rows, "prefix"
cached positions, "cap" the cache's capacity, "tree" (a number that gives the shape of the tree) and what one operator
needs besides.  Heads, widths and vocabularies are those of the 7B, 13B and 70B shapes and of the tiny float32 model.
"""

import math
import random

import torch

own = False

SHAPES = {
    # query heads, kv heads, head_dim, vocabulary, cache type, layers
    "tiny": (4, 4, 64, 1024, "f32", 4),
    "7b": (32, 32, 128, 32000, "bf16", 32),
    "13b": (40, 40, 128, 32000, "bf16", 40),
    "70b": (64, 8, 128, 32000, "bf16", 80),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ORIGINAL = 4096  # the context that the scaled frequencies start from


def _case(name, op, model, n, prefix, cap, tree=0, **more):
    heads, kv_heads, head_dim, vocab, dtype, layers = SHAPES[model]
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "n": n, "prefix": prefix,
         "cap": cap, "tree": tree}
    if op == "accept":
        c["vocab"] = vocab
    if op == "keep":
        c["layers"] = layers
    c.update(more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The nodes of a small tree, as every layer of a verification rotates and stores them; latency only.
        _case("rope 13b 13 nodes", "rope", "13b", 13, 1200, 1550, 1),
        # A long document's chunk with grouped-query heads, positions far past the trained context, frequencies by parts.
        _case("rope 70b 1000 rows far", "rope", "70b", 1000, 50000, 52000, 0, scaling="yarn", factor=16.0),
        # A float32 cache, half of the head rotated in interleaved pairs, an odd number of rows.
        _case("rope f32 interleaved part", "rope", "13b", 257, 700, 1024, 2, dtype="f32", layout="interleaved",
              rotary_dim=64, scaling="linear", factor=2.0),
        # The smallest call: a tree of the tiny float32 model; latency only.
        _case("attend tiny 5 nodes", "attend", "tiny", 5, 30, 64, 3),
        # A small tree in the middle of a 1024 + 512 token decode.
        _case("attend 13b 13 nodes", "attend", "13b", 13, 1200, 1550, 4),
        # A wide tree over a long chat, ragged sizes.
        _case("attend 7b 61 nodes", "attend", "7b", 61, 3001, 4096, 5),
        # Grouped-query heads share the cache among many rows: bound by the products.
        _case("attend 70b 64 nodes, 16k", "attend", "70b", 64, 16000, 16384, 6),
        # A long document and few nodes: bound by the read of the cache.
        _case("attend 70b 9 nodes, 60k", "attend", "70b", 9, 60000, 61000, 7),
        # The walk over the logits of a small tree.
        _case("accept 13 nodes", "accept", "13b", 13, 0, 0, 8, follow=0.6),
        # And of the largest trees.
        _case("accept 700 nodes", "accept", "13b", 700, 0, 0, 9, follow=0.4),
        # A path of a few nodes moved together in every layer of the 70B cache.
        _case("keep 70b 4 rows", "keep", "70b", 33, 300, 350, 10, count=4),
        # A long accepted path in the 13B cache, which has as many kv heads as query heads.
        _case("keep 13b 17 rows", "keep", "13b", 64, 80, 160, 11, count=17),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rope", "attend", "attend", "accept", "keep"])
    model = rng.choice(["tiny", "7b", "13b", "70b", "70b"])
    tree = rng.randint(12, 10**6)
    if op == "rope":
        n, prefix = log_int(1, 1000), log_int(1, 60000 if model == "70b" else 8000)
        dim = SHAPES[model][2]
        more = rng.choice([{}, {"scaling": "yarn", "factor": rng.choice([4.0, 16.0])}, {"scaling": "linear", "factor": 2.0},
                           {"scaling": "ntk", "factor": 4.0}])
        if rng.random() < 0.4:
            more = dict(more, layout="interleaved")
        if rng.random() < 0.4:
            more = dict(more, rotary_dim=rng.choice([dim // 4, dim // 2, 3 * dim // 4]))
        return _case(None, op, model, n, prefix, prefix + n + log_int(1, 1000), tree, **more)
    if op == "attend":
        n = log_int(1, 64 if model == "70b" else 128)
        prefix = log_int(1, {"tiny": 4000, "7b": 4000, "13b": 4000, "70b": 16000 if n > 9 else 60000}[model])
        more = {"dtype": "f32"} if model != "tiny" and n * prefix < 20000 and rng.random() < 0.3 else {}
        return _case(None, op, model, n, prefix, prefix + n + log_int(1, 1000), tree, **more)
    if op == "accept":
        return _case(None, op, model, log_int(1, 600), 0, 0, tree, follow=rng.choice([0.0, 0.4, 0.7, 1.0]))
    count = log_int(1, 16)
    n, prefix = 2 * count + log_int(1, 30), log_int(1, 80)
    return _case(None, op, model, n, prefix, prefix + n + rng.randint(0, 16), tree, count=count)


# ----------------------------------------------------------------------------
# inputs


def _parents(n, tree):
    """Node 0 is the root; a node hangs below one of the last few before it, more often the last."""
    rng = random.Random(tree * 31 + n)
    back = rng.choice([1, 3, 8, 20])
    return [-1] + [max(0, i - 1 - rng.randrange(back)) for i in range(1, n)]


def _ancestors(parents):
    """Depths, and per node the set of nodes on its path as bits, itself among them."""
    depth, seen = [], []
    for i, p in enumerate(parents):
        depth.append(0 if p < 0 else depth[p] + 1)
        seen.append((1 << i) | (0 if p < 0 else seen[p]))
    return depth, seen


def _mask(seen, n):
    """[n][words] int64, bit j of row i: node i sees node j."""
    words = (n + 63) // 64
    rows = [[(s >> (64 * w)) & (2**64 - 1) for w in range(words)] for s in seen]
    return torch.tensor([[w - 2**64 if w >= 2**63 else w for w in r] for r in rows], dtype=torch.int64, device="cuda")


def _keep_path(case):
    """Nodes of an accepted path of case["count"] nodes: the root, then nodes past the ones that stay in place."""
    n, count = case["n"], case["count"]
    return [0] + sorted(random.Random(case["tree"]).sample(range(count, n), count - 1))


def prepare(case, seed):
    n, P, cap = case["n"], case["prefix"], case["cap"]
    H, KVH, D = case["heads"], case["kv_heads"], case["head_dim"]
    dt = TYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + case["tree"] + 17)

    def normal(*shape, dtype=torch.float32, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    parents = _parents(n, case["tree"])
    depth, seen = _ancestors(parents)
    s = {"op": case["op"], "prefix": P}
    if case["op"] == "rope":
        s["qkv"] = normal(n, (H + 2 * KVH) * D)
        s["k"], s["v"] = normal(KVH, cap, D, dtype=dt), normal(KVH, cap, D, dtype=dt)
        s["positions"] = torch.tensor([P + d for d in depth], dtype=torch.int32, device="cuda")
        s["heads"] = H
        s["rope"] = {"base": 10000.0, "rotary_dim": case.get("rotary_dim", D), "layout": case.get("layout", "half"),
                     "scaling": case.get("scaling", "none"), "factor": case.get("factor", 1.0),
                     "original_context": ORIGINAL, "beta_fast": 32.0, "beta_slow": 1.0}
    elif case["op"] == "attend":
        s["q"] = normal(n, H, D)
        s["k"], s["v"] = normal(KVH, cap, D, dtype=dt), normal(KVH, cap, D, dtype=dt)
        s["mask"] = _mask(seen, n)
    elif case["op"] == "accept":
        s["logits"] = normal(n, case["vocab"], std=2.0)
        rng = random.Random(int(seed) * 7919 + case["tree"])
        best = s["logits"].argmax(dim=1).tolist()
        tokens = [rng.randrange(case["vocab"])]
        tokens += [best[p] if rng.random() < case["follow"] else rng.randrange(case["vocab"]) for p in parents[1:]]
        s["tokens"] = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        s["parents"] = torch.tensor(parents, dtype=torch.int32, device="cuda")
        s["mask"] = _mask(seen, n)
    else:
        s["kv"] = normal(case["layers"], 2, KVH, cap, D, dtype=dt)
        path = _keep_path(case)
        # what the walk leaves: the number of nodes, the next token, the path, each node's best token
        s["walk"] = torch.tensor([len(path), 7] + path + [-1] * (n - len(path)) + [7] * n, dtype=torch.int32, device="cuda")
    return s


# ----------------------------------------------------------------------------
# the operators


def run(s):
    return {"rope": _rope, "attend": _attend, "accept": _accept, "keep": _keep}[s["op"]](s)


def _rope(s):
    qkv, k, v, H = s["qkv"], s["k"], s["v"], s["heads"]
    if own:
        from paper_2309_08168_amd import binding

        q = binding.rope_append(binding.rope(**s["rope"]), qkv, k, v, s["prefix"], H, positions=s["positions"])
        return {"q": q, "k": k, "v": v}
    r = s["rope"]
    KVH, D, R, n = k.shape[0], k.shape[2], r["rotary_dim"], qkv.shape[0]
    half = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    base = r["base"] * (r["factor"] ** (R / (R - 2)) if r["scaling"] == "ntk" else 1.0)
    freq = torch.pow(base, -2.0 * half / R)
    gain = 1.0
    if r["scaling"] == "linear":
        freq = freq / r["factor"]
    elif r["scaling"] == "yarn":
        turns = freq * (r["original_context"] / (2 * math.pi))
        part = ((turns - r["beta_slow"]) / (r["beta_fast"] - r["beta_slow"])).clamp(0.0, 1.0)
        freq = freq * (part + (1.0 - part) / r["factor"])
        gain = 0.1 * math.log(r["factor"]) + 1.0
    angle = s["positions"].double()[:, None, None] * freq
    cos, sin = (angle.cos() * gain).float(), (angle.sin() * gain).float()
    x = qkv.view(n, H + 2 * KVH, D)
    qk = x[:, :H + KVH]
    if r["layout"] == "half":
        a, b = qk[..., :R // 2], qk[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = qk[..., 0:R:2], qk[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    out = torch.cat([turned, qk[..., R:]], dim=-1)
    P = s["prefix"]
    k[:, P:P + n] = out[:, H:].transpose(0, 1).to(k.dtype)
    v[:, P:P + n] = x[:, H + KVH:].transpose(0, 1).to(v.dtype)
    return {"q": out[:, :H].contiguous(), "k": k, "v": v}


def _visible(mask, prefix, n):
    """[n][prefix + n] truth values."""
    bits = (mask[:, :, None] >> torch.arange(64, device="cuda")) & 1
    nodes = bits.flatten(1)[:, :n].bool()
    return torch.cat([torch.ones(n, prefix, dtype=torch.bool, device="cuda"), nodes], dim=1)


def _attend(s):
    q, k, v, P = s["q"], s["k"], s["v"], s["prefix"]
    if own:
        from paper_2309_08168_amd import binding

        return binding.tree_attention(q, k, v, P, mask=s["mask"])
    n, H, D = q.shape
    KVH = k.shape[0]
    G = H // KVH
    keys, values = k[:, :P + n].float(), v[:, :P + n].float()
    rows = q.view(n, KVH, G, D).permute(1, 0, 2, 3).reshape(KVH, n * G, D)
    scores = torch.matmul(rows, keys.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
    hidden = ~_visible(s["mask"], P, n).repeat_interleave(G, dim=0)
    scores = scores.masked_fill(hidden, float("-inf"))
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, values) / torch.where(total == 0, torch.ones_like(total), total)
    return o.view(KVH, n, G, D).permute(1, 0, 2, 3).reshape(n, H, D)


def _accept(s):
    logits, tokens, parents = s["logits"], s["tokens"], s["parents"]
    if own:
        from paper_2309_08168_amd import binding

        return binding.tree_accept(logits, tokens, parents)
    n, V = logits.shape
    node = torch.arange(n, device="cuda")
    top = logits.amax(dim=1, keepdim=True)
    best = torch.where(logits == top, torch.arange(V, device="cuda"), V).amin(dim=1)
    up = parents.clamp(min=0).long()
    match = (tokens == best[up]) & (node > 0)
    # the lowest matching child of each parent
    rivals = match[None, :] & (parents[None, :] == parents[:, None]) & (node[None, :] < node[:, None])
    chosen = (match & ~rivals.any(dim=1)) | (node == 0)
    # on the path: every ancestor chosen
    path = ((_visible(s["mask"], 0, n) & ~chosen[None, :]).sum(dim=1) == 0)
    order = torch.sort(torch.where(path, node, n)).values
    count = path.sum(dim=0, keepdim=True)
    last = torch.where(path, node, 0).amax(dim=0, keepdim=True)
    return torch.cat([count, best[last], torch.where(order == n, -1, order), best]).to(torch.int32)


def _keep(s):
    kv, walk, P = s["kv"], s["walk"], s["prefix"]
    n = (walk.shape[0] - 2) // 2
    if own:
        from paper_2309_08168_amd import binding

        return binding.kv_keep(kv, P, walk)
    row = torch.arange(n, device="cuda")
    source = torch.where(row < walk[0], walk[2:2 + n], row)
    kv[..., P:P + n, :] = kv[..., P:P + n, :].index_select(3, source.long())
    return kv


# ----------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    n, P, H, KVH, D = case["n"], case["prefix"], case["heads"], case["kv_heads"], case["head_dim"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        return {"bytes": 4 * n * (H + 2 * KVH) * D + 4 * n * H * D + 2 * n * KVH * D * size + 4 * n,
                "flops": 3 * n * (H + KVH) * case.get("rotary_dim", D)}
    if case["op"] == "attend":
        pairs = n * P + sum(d + 1 for d in _ancestors(_parents(n, case["tree"]))[0])
        return {"bytes": 2 * 4 * n * H * D + 2 * (P + n) * KVH * D * size + 8 * n * ((n + 63) // 64),
                "flops": 4 * pairs * H * D}
    if case["op"] == "accept":
        return {"bytes": 4 * n * case["vocab"] + 4 * (4 * n + 2), "flops": n * case["vocab"]}
    planes = case["layers"] * 2 * KVH
    moved = sum(p != i for i, p in enumerate(_keep_path(case)))
    return {"bytes": 2 * moved * planes * D * size + 4 * (case["count"] + 1), "flops": 0}


# ----------------------------------------------------------------------------
# the definitions in 64 bits, row by row


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "accept": _exact_accept, "keep": _exact_keep}[case["op"]](s)


def _exact_rope(s):
    r, H, P = s["rope"], s["heads"], s["prefix"]
    KVH, _, D = s["k"].shape
    n, R = s["qkv"].shape[0], r["rotary_dim"]
    x = s["qkv"].double().view(n, H + 2 * KVH, D)
    out = x.clone()
    for i in range(R // 2):
        f = r["base"] ** (-2.0 * i / R)
        m = 1.0
        if r["scaling"] == "linear":
            f /= r["factor"]
        elif r["scaling"] == "ntk":
            f *= r["factor"] ** (-2.0 * i / (R - 2))
        elif r["scaling"] == "yarn":
            t = f * r["original_context"] / (2 * math.pi)
            w = min(1.0, max(0.0, (t - r["beta_slow"]) / (r["beta_fast"] - r["beta_slow"])))
            f = w * f + (1.0 - w) * f / r["factor"]
            m = 1.0 + 0.1 * math.log(r["factor"])
        e = (i, i + R // 2) if r["layout"] == "half" else (2 * i, 2 * i + 1)
        turn = torch.polar(torch.full((n, 1), m, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * f)
        z = torch.complex(x[:, :H + KVH, e[0]].contiguous(), x[:, :H + KVH, e[1]].contiguous()) * turn
        out[:, :H + KVH, e[0]], out[:, :H + KVH, e[1]] = z.real, z.imag
    k, v = s["k"].double(), s["v"].double()
    k[:, P:P + n] = out[:, H:H + KVH].transpose(0, 1)
    v[:, P:P + n] = x[:, H + KVH:].transpose(0, 1)
    return {"q": out[:, :H].contiguous(), "k": k, "v": v}


def _exact_attend(s):
    q, k, v, P = s["q"].double(), s["k"], s["v"], s["prefix"]
    n, H, D = q.shape
    G = H // k.shape[0]
    words = [[w & (2**64 - 1) for w in row] for row in s["mask"].tolist()]
    out = torch.zeros(n, H, D, dtype=torch.float64, device="cuda")
    cols = [torch.tensor(list(range(P)) + [P + j for j in range(n) if (words[i][j // 64] >> (j % 64)) & 1], device="cuda")
            for i in range(n)]
    for h in range(H):
        kh, vh = k[h // G].double(), v[h // G].double()
        for i in range(n):
            if len(cols[i]):
                p = torch.softmax(kh[cols[i]] @ q[i, h] / math.sqrt(D), dim=0)
                out[i, h] = p @ vh[cols[i]]
    return out


def _exact_accept(s):
    return None  # whole numbers


def _exact_keep(s):
    kv, P = s["kv"].double(), s["prefix"]
    walk = s["walk"].tolist()
    rows = [kv[..., P + p, :].clone() for p in walk[2:2 + walk[0]]]
    for i, row in enumerate(rows):
        kv[..., P + i, :] = row
    return kv
