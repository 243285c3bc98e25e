"""Tree forwards and verifications of a model against the oracle, which scores
every node's own chain of tokens: a node of a tree is the last token of the
prompt followed by its path.

Tolerances are those of the other model tests (gpu_util): float32 models 1e-4,
bfloat16 models 3e-2 standard deviations of the oracle's logits.
"""

import numpy as np
import pytest

import sd_synth as S
from tests import gpu_util as U
from tests import tree_ref as T

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MODELS = {
    "tiny": S.MODELS["tiny"],                                                   # float32, head_dim 64
    "micro": U.MICRO_GQA,                                                       # float32, head_dim 16, grouped heads
    "mini": U.MINI_BF16,                                                        # bfloat16, head_dim 64, grouped heads
    "wide": S.ModelConfig("wide", 2, 256, 8, 2, 128, 512, 700, "bf16"),         # head_dim 128
    "narrow": S.ModelConfig("narrow", 2, 128, 8, 4, 16, 256, 500, "bf16"),      # no matrix-core prefill
}
_built = {}


def built(name):
    """(config, GPU model, oracle model), built once."""
    import oracle

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if name not in _built:
        cfg = MODELS[name]
        w = S.make_weights(cfg, 4)
        _built[name] = cfg, U.device_model(cfg, w), oracle.Model(cfg, w)
    return _built[name]


def nan_logits(cfg, n):
    return torch.full((n, cfg.vocab), float("nan"), dtype=torch.float32, device="cuda")


def path_of(parents, i):
    path = []
    while i >= 0:
        path.append(i)
        i = int(parents[i])
    return path[::-1]


def oracle_nodes(omodel, prompt, tokens, parents, nodes):
    """Logits of the given nodes, each from its own chain."""
    rows = []
    for i in nodes:
        chain = [int(tokens[j]) for j in path_of(parents, i)]
        rows.append(omodel.score(np.concatenate([prompt, chain]).astype(np.int32))["logits"][-1])
    return np.stack(rows)


@pytest.mark.parametrize("name", sorted(MODELS))
@pytest.mark.parametrize("n,prefix", [(1, 0), (1, 9), (2, 5), (9, 0), (16, 30), (17, 31), (45, 7), (70, 12), (140, 3)])
def test_tree_forward(name, n, prefix):
    cfg, model, om = built(name)
    rng = np.random.default_rng(n + prefix)
    prompt = S.prompt(cfg, prefix + 1, seed=3)[:prefix]
    tokens = rng.integers(0, cfg.vocab, n).astype(np.int32)
    parents = T.random_parents(n, rng, 5)
    c = model.cache(prefix + n + 8)
    if prefix:
        model.forward(prompt, c)
    lg = model.forward_tree(tokens, parents, c, logits=nan_logits(cfg, n))
    assert c.length == prefix
    nodes = sorted(set(rng.integers(0, n, 6).tolist()) | {0, n - 1})
    ref = oracle_nodes(om, prompt, tokens, parents, nodes)
    U.check_logits(cfg, lg.cpu().numpy()[nodes], ref, f"{name}: nodes {nodes} of {n}")
    # a path taken over: the next tokens see it and nothing else of the tree
    path = path_of(parents, n - 1)
    c.keep(path)
    assert c.length == prefix + len(path)
    more = rng.integers(0, cfg.vocab, 3).astype(np.int32)
    got = model.forward(more, c, logits=nan_logits(cfg, 3)).cpu().numpy()
    seq = np.concatenate([prompt, tokens[path], more]).astype(np.int32)
    U.check_logits(cfg, got, om.score(seq)["logits"][-3:], f"{name}: after a path of {len(path)}")


@pytest.mark.parametrize("name", ["tiny", "mini", "wide"])
def test_the_largest_tree(name):
    """1024 nodes, some 20 deep; one more is refused."""
    from paper_2309_08168_amd import binding as B

    cfg, model, om = built(name)
    n, prefix = B.SD_TREE_MAX, 5
    rng = np.random.default_rng(1)
    prompt = S.prompt(cfg, prefix, seed=3)
    tokens = rng.integers(0, cfg.vocab, n).astype(np.int32)
    parents = T.random_parents(n, rng, 100)
    c = model.cache(prefix + n + 1)
    model.forward(prompt, c)
    lg = model.forward_tree(tokens, parents, c, logits=nan_logits(cfg, n)).cpu().numpy()
    nodes = [0, 1, 500, 1000, n - 1]
    U.check_logits(cfg, lg[nodes], oracle_nodes(om, prompt, tokens, parents, nodes), f"{name}: nodes {nodes}")
    with pytest.raises(B.SDError) as e:
        model.forward_tree([0] * (n + 1), [-1] + [0] * n, c)
    assert e.value.status == B.SD_ERR_INVALID_ARG
    path = path_of(parents, n - 1)
    c.keep(path)
    more = rng.integers(0, cfg.vocab, 2).astype(np.int32)
    got = model.forward(more, c, logits=nan_logits(cfg, 2)).cpu().numpy()
    seq = np.concatenate([prompt, tokens[path], more]).astype(np.int32)
    U.check_logits(cfg, got, om.score(seq)["logits"][-2:], f"{name}: after a path of {len(path)}")


@pytest.mark.parametrize("name", ["tiny", "mini"])
@pytest.mark.parametrize("n", [6, 40])
def test_tree_forward_with_a_skip_mask(name, n):
    """A chain as a tree against sd_forward, with sublayers skipped."""
    cfg, model, _ = built(name)
    z = S.skip_mask(cfg, "random2" if cfg.n_layers == 2 else "tiny", 0)
    toks = S.prompt(cfg, n + 10, seed=5)
    a, b = model.cache(60), model.cache(60)
    model.forward(toks[:10], a)
    model.forward(toks[:10], b)
    ref = model.forward(toks[10:], a, skip=z, logits=nan_logits(cfg, n)).cpu().numpy().astype(np.float64)
    got = model.forward_tree(toks[10:], np.arange(-1, n - 1), b, skip=z, logits=nan_logits(cfg, n)).cpu().numpy()
    U.check_logits(cfg, got, ref, name)


@pytest.mark.parametrize("name", sorted(MODELS))
def test_verification_emits_the_greedy_tokens(name):
    """Trees around the greedy continuation, some with it and some without: the
    tokens of the accepted paths are those of greedy decoding."""
    cfg, model, om = built(name)
    rng = np.random.default_rng(11)
    prompt = S.prompt(cfg, 12, seed=8)
    max_new = 30
    ref, _ = model.generate_ar(prompt, max_new + 20)
    c = model.cache(200)
    model.forward(prompt[:-1], c)
    out, last, accepted = [], int(prompt[-1]), []
    while len(out) < max_new:
        depth, width = int(rng.integers(1, 7)), int(rng.integers(1, 5))
        tokens, parents, spine = [last], [-1], 0
        for d in range(depth):
            # a level: wrong siblings, and the right token in a random place among them
            right = rng.random() < 0.85
            place = int(rng.integers(0, width))
            nxt = spine
            for k in range(width):
                good = right and k == place and spine >= 0
                tok = int(ref[len(out) + d]) if good else int(rng.integers(0, cfg.vocab))
                tokens.append(tok)
                parents.append(max(spine, 0))
                if good:
                    nxt = len(tokens) - 1
            if not right:
                break
            spine = nxt
        before = c.length
        path, nxt_tok = model.verify_tree(tokens, parents, c)
        assert path[0] == 0 and c.length == before + len(path)
        assert all(parents[path[i + 1]] == path[i] for i in range(len(path) - 1))
        out += [tokens[i] for i in path[1:]] + [nxt_tok]
        last = nxt_tok
        accepted.append(len(path) - 1)
    assert max(accepted) >= 2
    U.check_tokens_teacher_forced(cfg, om, prompt, np.array(out, np.int32), name)
    if cfg.dtype == "f32":
        assert out[:max_new] == ref[:max_new].tolist()


def test_tree_forward_refuses():
    from paper_2309_08168_amd import binding as B

    cfg, model, _ = built("mini")
    c = model.cache(20)
    model.forward([1, 2, 3], c)

    def status(fn, *args, **kw):
        with pytest.raises(B.SDError) as e:
            fn(*args, **kw)
        return e.value.status

    assert status(model.forward_tree, [], [], c) == B.SD_ERR_INVALID_ARG
    assert status(model.forward_tree, [1, 2], [-1], c) == B.SD_ERR_INVALID_ARG
    assert status(model.forward_tree, [1, 2], [0, 0], c) == B.SD_ERR_INVALID_ARG
    assert status(model.forward_tree, [1, 2], [-1, 1], c) == B.SD_ERR_INVALID_ARG
    assert status(model.forward_tree, [1, cfg.vocab], [-1, 0], c) == B.SD_ERR_INVALID_ARG
    assert status(model.forward_tree, [1] * 1025, [-1] + [0] * 1024, c) == B.SD_ERR_INVALID_ARG
    assert status(model.forward_tree, [1] * 18, [-1] + [0] * 17, c) == B.SD_ERR_CAPACITY
    assert status(model.verify_tree, [1] * 18, [-1] + [0] * 17, c) == B.SD_ERR_CAPACITY
    assert status(c.keep, [0]) == B.SD_ERR_INVALID_ARG  # no tree forward yet
    model.forward_tree([4, 5, 6], [-1, 0, 0], c)
    for path in ([], [3], [-1], [0, 0], [1, 0], [0, 1, 2, 2]):
        assert status(c.keep, path) == B.SD_ERR_INVALID_ARG
    c.truncate(2)
    assert status(c.keep, [0]) == B.SD_ERR_INVALID_ARG  # the nodes went with it
    model.forward_tree([4, 5, 6], [-1, 0, 0], c)
    model.forward([7], c)
    assert status(c.keep, [0]) == B.SD_ERR_INVALID_ARG
    z = S.skip_mask(cfg, "random2", 0)
    model.quantize_draft(z)
    try:
        assert status(model.forward_tree, [4, 5], [-1, 0], c, skip=z) == B.SD_ERR_INVALID_ARG
    finally:
        model.quantize_draft(None)
    assert c.length == 3


def keys_of(buf, cfg):
    """The first layer's keys of 60 positions, float64 [60, n_kv_heads, head_dim]."""
    t = buf.view(torch.bfloat16 if cfg.dtype == "bf16" else torch.float32)
    return t.view(cfg.n_layers, 2, cfg.n_kv_heads, 80, cfg.head_dim)[0, 0, :, :60].double().cpu().numpy().transpose(1, 0, 2)


def check_keys(cfg, got, plain, form):
    """The first layer's keys do not depend on the form but for their rotation:
    plain turned back, and turned by the form.  Each side was rounded once
    (bfloat16: half a step, 2^-8 of an element; float32: eight roundings of 2^-24)."""
    pos = np.arange(60)
    raw = T.rope(plain, -pos, {"rotary_dim": cfg.head_dim, "base": cfg.rope_base})
    want = T.rope(raw, pos, form)
    half = cfg.head_dim // 2
    pair = np.abs(plain[:, :, :half]) + np.abs(plain[:, :, half:])
    pair = np.concatenate([pair, pair], axis=2)
    step = 2.0 ** -8 if cfg.dtype == "bf16" else 8 * 2.0 ** -24
    # the plain side's rounding, carried through two rotations of at most
    # sqrt(2) each and the gain, and the other side's own
    gain = np.abs(want).max() / np.abs(plain).max() + 1.0
    assert (np.abs(got - want) <= step * (2 * gain * pair + np.abs(want))).all()
    assert np.abs(got - plain).max() > 0.3 * np.abs(plain).max()


@pytest.mark.parametrize("name", ["tiny", "wide"])
@pytest.mark.parametrize("form", [dict(scaling="linear", factor=2.0), dict(scaling="yarn", factor=4.0, original_context=16),
                                  dict(scaling="ntk", factor=3.0), dict(base=500.0, gain=1.1)], ids=str)
def test_scaled_rotary_form(name, form):
    """The forwards' own rotary table against the operator of the tree forward,
    whose formula the operator's tests check; NTK also against a model of the
    larger base."""
    from paper_2309_08168_amd import binding as B

    cfg, _, _ = built(name)
    w = S.make_weights(cfg, 4)
    model = U.device_model(cfg, w)
    toks = S.prompt(cfg, 60, seed=6)
    plain_buf, a_buf = (torch.zeros(model.kv_cache_bytes(80), dtype=torch.uint8, device="cuda") for _ in range(2))
    plain_cache = model.cache(80, device_buf=plain_buf)
    plain = model.forward(toks, plain_cache, logits=nan_logits(cfg, 60)).cpu().numpy()
    plain_cache.truncate(0)
    model.set_rope(B.rope(rotary_dim=cfg.head_dim, **form))
    a, b = model.cache(80, device_buf=a_buf), model.cache(120)
    got = model.forward(toks, a, logits=nan_logits(cfg, 60)).cpu().numpy()
    model.forward(toks[:20], b)
    chain = model.forward_tree(toks[20:], np.arange(-1, 39), b, logits=nan_logits(cfg, 40)).cpu().numpy()
    U.check_logits(cfg, chain, got[20:].astype(np.float64), name)
    check_keys(cfg, keys_of(a_buf, cfg), keys_of(plain_buf, cfg), {"rotary_dim": cfg.head_dim, **form})
    if form.get("scaling") == "ntk":
        d = cfg.head_dim
        other = S.ModelConfig(**{**cfg.__dict__, "rope_base": cfg.rope_base * 3.0 ** (d / (d - 2))})
        big = U.device_model(other, w)
        ref = big.forward(toks, big.cache(80), logits=nan_logits(cfg, 60)).cpu().numpy()
        U.check_logits(cfg, got, ref.astype(np.float64), name)
        big.close()
    for c in (a, b):
        c.truncate(0)
    model.set_rope(None)
    back = model.forward(toks, a, logits=nan_logits(cfg, 60)).cpu().numpy()
    assert np.array_equal(back, plain)
    with pytest.raises(B.SDError) as e:
        model.set_rope(None)  # a holds keys
    assert e.value.status == B.SD_ERR_INVALID_ARG
    a.truncate(0)
    for bad in (dict(layout="interleaved"), dict(rotary_dim=cfg.head_dim // 2)):
        with pytest.raises(B.SDError) as e:
            model.set_rope(B.rope(**{"rotary_dim": cfg.head_dim, **bad}))
        assert e.value.status == B.SD_ERR_UNIMPLEMENTED
    model.close()
