"""The tree operators on the GPU against their plain float64 forms.

Tolerances: float32 results count the roundings on the way (2^-24 each, see
the helpers); what is stored as bfloat16 adds half a step, 2^-8 of the value;
whole numbers are equal.
"""

import math

import numpy as np
import pytest

from tests import tree_ref as T

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2309_08168_amd import binding

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def layers(rng, kvh, cap, d, dtype, order="heads"):
    """k and v [kvh, cap, d] on the GPU; order "positions": a [cap][kvh][d]
    buffer, "padded": rows with a gap."""
    def one():
        x = torch.tensor(rng.standard_normal((kvh, cap, d)), dtype=TYPES[dtype], device="cuda")
        if order == "positions":
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        if order == "padded":
            return torch.nn.functional.pad(x, (0, 16))[:, :, :d]
        return x

    return one(), one()


def f64(t):
    return t.detach().double().cpu().numpy()


# ----------------------------------------------------------------------------
# rope_append

FORMS = [
    dict(rotary_dim=64), dict(rotary_dim=64, layout="interleaved"), dict(rotary_dim=32, scaling="linear", factor=4.0),
    dict(rotary_dim=48, layout="interleaved", scaling="ntk", factor=2.5), dict(rotary_dim=64, scaling="yarn", factor=16.0),
    dict(rotary_dim=20, scaling="yarn", factor=4.0, original_context=512, beta_fast=20.0, beta_slow=2.0, gain=1.25),
    dict(rotary_dim=6, layout="interleaved", base=500.0), dict(rotary_dim=2), dict(rotary_dim=4, scaling="ntk", factor=3.0),
]


def check_rope(n, heads, kvh, d, dtype, form, positions, order="heads", slot=3, strided=False, seed=0):
    rng = np.random.default_rng(seed + n)
    k, v = layers(rng, kvh, slot + n + 2, d, dtype, order)
    k0, v0 = f64(k), f64(v)
    width = (heads + 2 * kvh) * d
    buf = torch.tensor(rng.standard_normal((n, width + (8 if strided else 0))), dtype=torch.float32, device="cuda")
    qkv = buf[:, :width]
    explicit = positions is not None
    pos = np.asarray(positions if explicit else 11 + np.arange(n))
    q_out = torch.full((n, heads + (1 if strided else 0), d), 7.0, device="cuda")[:, :heads] if strided else None
    q = binding.rope_append(binding.rope(**form), qkv, k, v, slot, heads, pos0=11, q_out=q_out,
                            positions=torch.tensor(pos, dtype=torch.int32, device="cuda") if explicit else None)
    x = f64(qkv).reshape(n, heads + 2 * kvh, d)
    want = T.rope(x[:, :heads + kvh], pos, form)
    # angle, cosine and sine, gain, two products and a sum: eight roundings of |a| + |b|
    gain = form.get("gain") or (0.1 * math.log(form["factor"]) + 1.0 if form.get("scaling") == "yarn" else 1.0)
    tol = 8 * 2.0 ** -24 * gain * 2 * np.abs(x).max()
    assert np.abs(f64(q) - want[:, :heads]).max() <= tol
    wk, wv = k0.copy(), v0.copy()
    wk[:, slot:slot + n] = want[:, heads:].transpose(1, 0, 2)
    wv[:, slot:slot + n] = x[:, heads + kvh:].transpose(1, 0, 2)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    new = slice(slot, slot + n)
    assert (np.abs(f64(k) - wk)[:, new] <= half * np.abs(wk[:, new]) + tol * (1 + half)).all()
    exact_v = torch.tensor(wv[:, new]).to(TYPES[dtype]).double().numpy()
    assert np.array_equal(f64(v)[:, new], exact_v)
    rest = np.r_[0:slot, slot + n:slot + n + 2]
    assert np.array_equal(f64(k)[:, rest], k0[:, rest]) and np.array_equal(f64(v)[:, rest], v0[:, rest])
    if strided:
        assert (q_out._base[:, heads:] == 7.0).all()


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rope_forms(form, dtype):
    check_rope(5, 6, 2, 64, dtype, form, [0, 1, 4095, 100000, 3])


@pytest.mark.parametrize("n,heads,kvh,d", [(1, 40, 40, 128), (13, 64, 8, 128), (300, 4, 4, 16), (2100, 2, 1, 32), (7, 3, 3, 16)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rope_sizes(n, heads, kvh, d, dtype):
    check_rope(n, heads, kvh, d, dtype, dict(rotary_dim=d), None)


@pytest.mark.parametrize("order", ["positions", "padded"])
@pytest.mark.parametrize("rotary_dim", [64, 10])
def test_rope_strides(order, rotary_dim):
    check_rope(9, 4, 2, 64, "bf16", dict(rotary_dim=rotary_dim), list(range(50, 59)), order=order, strided=True)


def test_rope_far_and_negative_positions():
    check_rope(4, 2, 2, 128, "f32", dict(rotary_dim=128), [2**31 - 1, 2**30, -1, -70000])


@pytest.mark.parametrize("form", [
    dict(scaling="ntk", factor=1e150, rotary_dim=4), dict(gain=3e37), dict(base=1e308, rotary_dim=32),
    dict(scaling="linear", factor=1e308), dict(scaling="yarn", factor=1e308, gain=1.0)], ids=str)
def test_rope_forms_at_the_limits(form):
    check_rope(3, 2, 1, 64, "f32", {"rotary_dim": 64, **form}, [0, 1, 2**31 - 1])


# ----------------------------------------------------------------------------
# tree_attention


def check_attention(n, heads, kvh, d, dtype, prefix, see=None, order="heads", scale=0.0, spoil=None, seed=0, strided=False,
                    peak=1.0):
    """see: None for the causal form, else a truth table.  spoil(k, v): changes
    the cache in places that the reference must not read."""
    rng = np.random.default_rng(seed + 31 * n + prefix)
    k, v = layers(rng, kvh, prefix + n + 3, d, dtype, order)
    wide = torch.tensor(peak * rng.standard_normal((n, heads + (2 if strided else 0), d)), dtype=torch.float32, device="cuda")
    q = wide[:, :heads]
    k64, v64 = f64(k), f64(v)
    if spoil is not None:
        spoil(k, v)
    mask = None if see is None else torch.tensor(T.pack(see).astype(np.int64), device="cuda")
    out = torch.full((n, heads + 1, d), 5.0, device="cuda")[:, :heads] if strided else None
    got = binding.tree_attention(q, k, v, prefix, mask=mask, scale=scale, out=out)
    table = np.tril(np.ones((n, n), bool)) if see is None else see
    sc = scale if scale else 1.0 / math.sqrt(d)
    want, size = T.attention(f64(q), k64, v64, prefix, table, sc)
    tol = T.attention_tol(d, prefix + n, size, np.abs(v64).max())
    err = np.abs(f64(got) - want).max()
    assert err <= tol, (err, tol)
    if strided:
        assert (out._base[:, heads:] == 5.0).all()
    again = binding.tree_attention(q, k, v, prefix, mask=mask, scale=scale)
    assert torch.equal(again, got.contiguous())
    return got


def tree(n, seed=0, back=4):
    return T.layout(T.random_parents(n, np.random.default_rng(seed + n), back))[1]


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,prefix", [(1, 0), (1, 1), (5, 0), (13, 63), (33, 64), (65, 129), (130, 1000)])
def test_attention_sizes(d, dtype, n, prefix):
    check_attention(n, 4, 2, d, dtype, prefix, tree(n))


@pytest.mark.parametrize("heads,kvh", [(1, 1), (5, 5), (8, 1), (24, 2), (64, 8), (7, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 17])
def test_attention_heads(heads, kvh, dtype, n):
    check_attention(n, heads, kvh, 128, dtype, 200, tree(n))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,prefix", [(1, 0), (16, 100), (64, 64), (100, 1), (257, 30)])
def test_attention_causal(dtype, n, prefix):
    chain = check_attention(n, 4, 4, 64, dtype, prefix)
    same = check_attention(n, 4, 4, 64, dtype, prefix, np.tril(np.ones((n, n), bool)))
    assert torch.equal(chain, same)


@pytest.mark.parametrize("d,n,kvh,prefix", [(128, 80, 32, 1500), (16, 130, 20, 2500), (64, 260, 10, 2000), (32, 30, 140, 1300)])
def test_float32_tiles_for_more_than_half_the_cus(d, n, kvh, prefix):
    """160 to 280 tiles of 16 rows over a long context."""
    check_attention(n, kvh, kvh, d, "f32", prefix, tree(n))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40, 1024])
def test_attention_long(dtype, n):
    check_attention(n, 2, 1, 128, dtype, 5000 if n < 1024 else 50, tree(n, back=30))


@pytest.mark.parametrize("d,dtype,n", [(16, "f32", 1), (128, "f32", 3), (32, "bf16", 2), (128, "bf16", 1), (128, "bf16", 40)])
def test_attention_many_shares(d, dtype, n):
    """More shares than the join takes at once: hundreds for one kv head."""
    prefix = 35001
    k = torch.empty(1, prefix + n, d, dtype=TYPES[dtype], device="cuda")
    assert binding.tree_attention_workspace(k, k, 1, n, prefix) > 100 * n * 4 * (d + 2)
    check_attention(n, 1, 1, d, dtype, prefix, tree(n))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,heads", [(5, 4), (40, 4)])
@pytest.mark.parametrize("gap", [2**24 - 8, 2**24 + 8])
def test_a_layer_past_32_bits(dtype, n, heads, gap):
    """Rows so far apart that offsets pass 2^31 elements and 2^32 bytes, with
    row strides on both sides of where a block's offsets fit 32 bits."""
    kvh, d, cap = 2, 128, 132
    size = (cap - 1) * gap + 2 * kvh * d
    assert size > 2**31
    # k and v interleaved in one buffer: heads of k, then of v, in each row
    buf = torch.empty(size, dtype=TYPES[dtype], device="cuda")
    k, v = (torch.as_strided(buf, (kvh, cap, d), (d, gap, 1), i * kvh * d) for i in range(2))
    rng = np.random.default_rng(n)
    near_k, near_v = layers(rng, kvh, cap, d, dtype)
    k.copy_(near_k)
    v.copy_(near_v)
    prefix = cap - n
    qkv = torch.tensor(rng.standard_normal((n, (heads + 2 * kvh) * d)), dtype=torch.float32, device="cuda")
    form = binding.rope(rotary_dim=d)
    q = binding.rope_append(form, qkv, k, v, prefix, heads, pos0=prefix)
    near_q = binding.rope_append(form, qkv, near_k, near_v, prefix, heads, pos0=prefix)
    assert torch.equal(q, near_q) and torch.equal(k, near_k) and torch.equal(v, near_v)
    mask = torch.tensor(T.pack(tree(n)).astype(np.int64), device="cuda")
    assert torch.equal(binding.tree_attention(q, k, v, prefix, mask=mask),
                       binding.tree_attention(q, near_k, near_v, prefix, mask=mask))


def test_walk_and_move_past_32_bits():
    n, ld, vocab = 600, 2**21, 500
    rng = np.random.default_rng(1)
    parents = T.random_parents(n, rng)
    logits = rng.standard_normal((n, vocab)).astype(np.float32)
    best = logits.argmax(axis=1)
    tokens = [0] + [int(best[p]) for p in parents[1:]]
    x = torch.empty(n, ld, device="cuda")[:, :vocab]
    x.copy_(torch.tensor(logits))
    walk = binding.tree_accept(x, torch.tensor(tokens, dtype=torch.int32, device="cuda"), torch.tensor(parents, device="cuda"))
    del x
    w = walk.cpu().numpy()
    assert np.array_equal(w, T.walk(logits, tokens, parents))
    planes, d, cap = 2, 128, 9_000_000  # a plane of 2.3 GB
    base = cap - n
    kv = torch.empty(planes, cap, d, dtype=torch.bfloat16, device="cuda")
    kv[:, base:] = torch.randn(planes, n, d, device="cuda")
    kv[:, :n] = 1.0
    want = T.keep(f64(kv[:, base:]), 0, w[2:2 + w[0]])
    binding.kv_keep(kv, base, walk)
    assert np.array_equal(f64(kv[:, base:]), want) and (kv[:, :n] == 1.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("prefix", [0, 70])
def test_attention_any_mask(dtype, prefix):
    """Bits before and behind the diagonal, rows without any, bits past n."""
    n = 70
    see = np.random.default_rng(3).random((n, n)) < 0.3
    see[5] = see[66] = False
    got = check_attention(n, 6, 3, 64, dtype, prefix, see)
    if prefix == 0:
        assert (got[5] == 0).all() and (got[66] == 0).all()
    past = np.concatenate([see, np.ones((n, 58), bool)], axis=1)
    rng = np.random.default_rng(1)
    k, v = layers(rng, 3, prefix + n + 60, 64, dtype)
    q = torch.tensor(rng.standard_normal((n, 6, 64)), dtype=torch.float32, device="cuda")
    a, b = (binding.tree_attention(q, k, v, prefix, mask=torch.tensor(T.pack(m).astype(np.int64), device="cuda"))
            for m in (see, past))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("heads,n,prefix", [(4, 12, 70), (2, 70, 0), (32, 40, 130)])
def test_attention_ignores_what_is_hidden(dtype, bad, heads, n, prefix):
    """NaN and infinities in keys and values that no row, or not every row, sees."""
    see = tree(n, back=6)
    see[:, 3] = False  # no row sees node 3, every row its own path otherwise
    one = n - 1        # only the last node sees this one

    def spoil(k, v):
        k[:, prefix + 3] = v[:, prefix + 3] = bad
        k[:, prefix + n:] = v[:, prefix + n:] = bad

    check_attention(n, heads, 2, 128, dtype, prefix, see, spoil=spoil)
    see[:, one] = False
    see[one, one] = True
    rng = np.random.default_rng(9)
    k, v = layers(rng, 2, prefix + n, 128, dtype)
    q = torch.tensor(rng.standard_normal((n, heads, 128)), dtype=torch.float32, device="cuda")
    mask = torch.tensor(T.pack(see).astype(np.int64), device="cuda")
    clean = binding.tree_attention(q, k, v, prefix, mask=mask)
    v[:, prefix + one, 7] = bad
    got = binding.tree_attention(q, k, v, prefix, mask=mask)
    # float32 sums in another order where a value is not finite
    size = float((q.abs().max() * k.float().abs().max() * math.sqrt(128)).item())
    tol = T.attention_tol(128, prefix + n, size, float(clean.abs().max()))
    assert (got[:one] - clean[:one]).abs().max() <= tol
    assert not torch.isfinite(got[one, :, 7]).any() and torch.isfinite(got[one, :, :7]).all()


# rows of a kv head: up to 16, 17 to 32, 33 to 64, more
ROWS = [(12, 1), (12, 2), (20, 2), (40, 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("n,group", ROWS)
def test_rows_keep_their_bits_whatever_they_do_not_see(dtype, d, n, group):
    """A node's key and value, and its rows' queries, changed: the rows that do
    not see it keep every bit, next to rows of their tile that do.  (64 kv heads,
    so that the nodes' block is not the first that a wave takes.)"""
    prefix, kvh = 1000, 64
    see = tree(n)
    node = max(range(1, n), key=lambda j: min(see[:, j].sum(), n - see[:, j].sum()))
    sees = torch.tensor(see[:, node], device="cuda")
    assert 0 < int(sees.sum()) < n
    g = torch.Generator(device="cuda").manual_seed(n + d)
    k, v = (torch.randn(kvh, prefix + n, d, device="cuda", generator=g).to(TYPES[dtype]) for _ in range(2))
    q = torch.randn(n, kvh * group, d, device="cuda", generator=g)
    mask = torch.tensor(T.pack(see).astype(np.int64), device="cuda")
    before = binding.tree_attention(q, k, v, prefix, mask=mask)
    k0, v0, q0 = k[:, prefix + node].clone(), v[:, prefix + node].clone(), q[sees].clone()

    def same():
        return torch.equal(binding.tree_attention(q, k, v, prefix, mask=mask)[~sees], before[~sees])

    k[:, prefix + node] *= 60  # scores of some hundred, far above the others
    assert same()
    k[:, prefix + node] = k0
    q[sees] *= 60
    assert same()
    q[sees] = q0
    for bad in (float("nan"), float("inf"), float("-inf")):
        v[:, prefix + node, ::5] = bad
        assert same()
        k[:, prefix + node, ::7] = bad
        assert same()
        k[:, prefix + node], v[:, prefix + node] = k0, v0
    assert torch.equal(binding.tree_attention(q, k, v, prefix, mask=mask), before)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("n,group", ROWS)
@pytest.mark.parametrize("prefix", [0, 70])
def test_attention_any_mask_in_every_tile(dtype, d, n, group, prefix):
    """Bits before and behind the diagonal, and rows without any, which see the
    prefix or nothing."""
    see = np.random.default_rng(n + d).random((n, n)) < 0.3
    see[2] = see[n - 1] = False
    got = check_attention(n, 2 * group, 2, d, dtype, prefix, see)
    if prefix == 0:
        assert (got[2] == 0).all() and (got[n - 1] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("n,group", ROWS)
@pytest.mark.parametrize("prefix", [0, 1100])
def test_attention_with_hidden_nan_in_every_tile(dtype, d, n, group, prefix):
    """A node that no row sees, and the cache behind the tree, hold NaN and
    infinities; then a value that is seen by some rows is infinite: those rows
    receive it, and only there."""
    see = tree(n)
    see[:, 3] = False

    def spoil(k, v):
        k[:, prefix + 3] = v[:, prefix + 3, ::2] = float("nan")
        v[:, prefix + 3, 1::2] = float("-inf")
        k[:, prefix + n:] = v[:, prefix + n:] = float("inf")

    clean = check_attention(n, 2 * group, 2, d, dtype, prefix, see, spoil=spoil)
    seen = torch.tensor(see[:, 5], device="cuda")
    assert 0 < int(seen.sum()) < n

    def infinite(k, v):
        v[:, prefix + 5, 3] = v[:, prefix + 5, d - 2] = float("inf")

    rng = np.random.default_rng(31 * n + prefix)  # (the inputs of check_attention)
    k, v = layers(rng, 2, prefix + n + 3, d, dtype)
    q = torch.tensor(rng.standard_normal((n, 2 * group, d)), dtype=torch.float32, device="cuda")
    spoil(k, v)
    infinite(k, v)
    got = binding.tree_attention(q, k, v, prefix, mask=torch.tensor(T.pack(see).astype(np.int64), device="cuda"))
    there = torch.zeros_like(got, dtype=torch.bool)
    there[seen, :, 3] = there[seen, :, d - 2] = True
    assert (got[there] == float("inf")).all() and torch.equal(got[~there], clean[~there])


@pytest.mark.parametrize("dtype,n,kvh,group,d", [
    ("f32", 512, 1, 1, 128), ("f32", 1000, 2, 1, 32), ("bf16", 500, 1, 1, 128), ("bf16", 500, 1, 1, 16), ("bf16", 1024, 1, 2, 64)])
def test_rows_that_see_nothing_in_several_shares(dtype, n, kvh, group, d):
    """No prefix, and nodes enough that their keys are split: rows that see
    nothing in one share, and in none."""
    k = torch.empty(kvh, n + 3, d, dtype=TYPES[dtype], device="cuda")
    assert binding.tree_attention_workspace(k, k, kvh * group, n, 0) > 0
    see = tree(n, back=2)
    see[7] = see[n - 1] = see[n // 2] = False
    see[n - 2] = False
    see[n - 2, n - 2] = True  # only the last share has a key of it
    got = check_attention(n, kvh * group, kvh, d, dtype, 0, see)
    assert (got[[7, n // 2, n - 1]] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["positions", "padded"])
def test_attention_strides(dtype, order):
    check_attention(21, 6, 3, 64, dtype, 150, tree(21), order=order, strided=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,peak", [(0.5, 1.0), (-0.1, 1.0), (0.0, 30.0), (1e-6, 1.0)])
def test_attention_scales(dtype, scale, peak):
    check_attention(9, 4, 4, 128, dtype, 300, tree(9), scale=scale, peak=peak)


def test_attention_offsets_past_32_bits():
    """The last head of a layer whose elements pass 2^31, and a position past 2^31 bytes of a head."""
    kvh, cap, d = 3, 6_000_000, 128
    buf = torch.zeros(kvh, cap, d, dtype=torch.bfloat16, device="cuda")
    n, prefix = 3, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    small = torch.randn(kvh, prefix + n, d, device="cuda", generator=g).to(torch.bfloat16)
    q = torch.randn(n, kvh, d, device="cuda", generator=g)
    buf[:, :prefix + n] = small
    want = binding.tree_attention(q, small, small, prefix)
    assert torch.equal(binding.tree_attention(q, buf, buf, prefix), want)
    rows = buf.view(kvh, cap // 1_000_000, 1_000_000 * d)[:, :, :d]  # a row every 256 MB: 6 positions
    rows[:] = small[:, :6]
    want = binding.tree_attention(q, small[:, :6].contiguous(), small[:, :6].contiguous(), 3)
    assert torch.equal(binding.tree_attention(q, rows, rows, 3), want)


def test_attention_workspace_and_graph_replay():
    """Two captured graphs with workspaces of their own, replayed with new
    inputs in the same buffers, eager calls between."""
    rng = np.random.default_rng(0)
    n, prefix = 11, 1500
    k, v = layers(rng, 4, prefix + n, 128, "bf16")
    mask = torch.tensor(T.pack(tree(n)).astype(np.int64), device="cuda")
    graphs = []
    for _ in range(2):
        q = torch.zeros(n, 8, 128, device="cuda")
        ws = torch.empty(binding.tree_attention_workspace(k, v, 8, n, prefix), dtype=torch.uint8, device="cuda")
        binding.tree_attention(q, k, v, prefix, mask=mask, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = binding.tree_attention(q, k, v, prefix, mask=mask, workspace=ws)
        graphs.append((g, q, out, ws))
    for i in range(4):
        new = [torch.randn(n, 8, 128, device="cuda") for _ in graphs]
        for (g, q, _, _), x in zip(graphs, new):
            q.copy_(x)
            g.replay()
        eager = [binding.tree_attention(x, k, v, prefix, mask=mask) for x in new]
        torch.cuda.synchronize()
        for (_, _, out, _), e in zip(graphs, eager):
            assert torch.equal(out, e)


def test_attention_on_another_stream():
    rng = np.random.default_rng(0)
    k, v = layers(rng, 2, 3000, 64, "bf16")
    q = torch.randn(7, 4, 64, device="cuda")
    want = binding.tree_attention(q, k, v, 2900)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = binding.tree_attention(q, k, v, 2900)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


# ----------------------------------------------------------------------------
# tree_accept and kv_keep


def check_accept(logits, tokens, parents, strided=0):
    n, vocab = logits.shape
    buf = torch.full((n, vocab + strided), 1e30, device="cuda")
    x = buf[:, :vocab]
    x.copy_(torch.tensor(logits))
    got = binding.tree_accept(x, torch.tensor(tokens, dtype=torch.int32, device="cuda"),
                              torch.tensor(parents, dtype=torch.int32, device="cuda")).cpu().numpy()
    want = T.walk(logits, tokens, parents)
    assert np.array_equal(got, want)
    return got


@pytest.mark.parametrize("n", [1, 2, 13, 64, 65, 1024])
@pytest.mark.parametrize("vocab,strided", [(1, 0), (3, 1), (97, 3), (4096, 0), (32000, 5), (131072, 0)])
def test_accept(n, vocab, strided):
    if n * vocab > 40_000_000:
        vocab = 32001
    rng = np.random.default_rng(n + vocab)
    parents = T.random_parents(n, rng)
    # few different values, so that rows have ties
    logits = rng.integers(-6, 6 if vocab < 5000 else 40000, (n, vocab)).astype(np.float32)
    best = logits.argmax(axis=1)
    tokens = [0] + [int(best[p]) if rng.random() < 0.8 else int(rng.integers(vocab)) for p in parents[1:]]
    check_accept(logits, tokens, parents, strided)


def test_accept_the_largest_vocabulary():
    """Slices that would end past 2^31 - 1, with larger values right behind the row."""
    vocab = 2**31 - 4097
    buf = torch.zeros(vocab + 4096, device="cuda")
    buf[vocab:] = 2.0
    root = torch.zeros(1, dtype=torch.int32, device="cuda")
    for last in (vocab - 1, vocab - 4096, 0):
        buf[last] = 1.0
        walk = binding.tree_accept(buf[None, :vocab], root, root - 1)
        assert walk.tolist() == [1, last, 0, last]
        buf[last] = 0.0


def test_accept_not_a_number_and_infinities():
    nan, inf = float("nan"), float("inf")
    logits = np.array([[nan, 1, 2, nan, 2], [nan] * 5, [-inf] * 5, [inf, nan, inf, 0, 0], [-0.0, 0.0, -1, nan, -0.0],
                       [nan, -inf, -inf, nan, -inf]], np.float32)
    # 0 -> token 2 -> all NaN: token 0 -> all -inf: token 0 -> inf: token 0 -> zeros: token 0 -> token 1
    check_accept(logits, [3, 2, 0, 0, 0, 0], [-1, 0, 1, 2, 3, 4])


def test_accept_takes_the_lowest_child_and_bad_parents_nothing():
    logits = np.zeros((8, 10), np.float32)
    logits[np.arange(8), [4, 1, 2, 3, 5, 6, 7, 8]] = 1.0
    walk = check_accept(logits, [0, 9, 4, 4, 2, 2, 3, 3], [-1, 0, 0, 0, 2, 2, 3, 3])
    assert walk[:5].tolist() == [3, 5, 0, 2, 4]
    # parents out of range, the node itself, a later node: never reached
    got = binding.tree_accept(torch.tensor(logits, device="cuda"),
                              torch.tensor([4, 4, 4, 4, 4, 4, 4, 4], dtype=torch.int32, device="cuda"),
                              torch.tensor([-1, 1, 5, -7, 99, 2**31 - 1, 7, -1], dtype=torch.int32, device="cuda"))
    assert got[:3].tolist() == [1, 4, 0] and (got[3:10] == -1).all()


def test_accept_chain_of_every_node():
    n = 1024
    logits = np.zeros((n, 7), np.float32)
    logits[:, 3] = 1.0
    walk = check_accept(logits, [3] * n, np.arange(-1, n - 1).astype(np.int32))
    assert walk[0] == n


@pytest.mark.parametrize("d,dtype", [(8, "bf16"), (16, "f32"), (64, "bf16"), (128, "bf16"), (128, "f32"), (24, "bf16")])
@pytest.mark.parametrize("planes,n,count", [(1, 1, 1), (3, 5, 5), (6, 40, 9), (5, 1024, 700), (641, 30, 4)])
def test_keep(d, dtype, planes, n, count):
    rng = np.random.default_rng(planes + n + count)
    base, cap = 17, 17 + n + 4
    path = np.sort(rng.choice(n, count, replace=False)) if count < n else np.arange(n)
    kv = torch.tensor(rng.standard_normal((planes, cap, d)), dtype=TYPES[dtype], device="cuda")
    before = f64(kv)
    walk = np.concatenate([[count, 3], path, np.full(n - count, -1), np.zeros(n)]).astype(np.int32)
    assert binding.kv_keep(kv, base, torch.tensor(walk, device="cuda")) is kv
    assert np.array_equal(f64(kv), T.keep(before, base, path))


def test_keep_refuses_bad_walks_on_the_device():
    kv = torch.randn(4, 30, 64, device="cuda")
    before = kv.clone()
    for count, path in ((0, [0, 1, 2, 3]), (5, [0, 1, 2, 3]), (-1, [0, 1, 2, 3]), (3, [0, 2, 2, 3]), (3, [0, 3, 1, 2]),
                        (3, [0, 2, 4, 5]), (2, [-1, 2, 3, 3]), (2**31 - 1, [0, 1, 2, 3])):
        walk = torch.tensor([count, 1] + path + [0] * 4, dtype=torch.int32, device="cuda")
        assert torch.equal(binding.kv_keep(kv, 2, walk), before), (count, path)


# ----------------------------------------------------------------------------
# together, as a verification uses them


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_of_a_verification(dtype):
    """Rotate and store the nodes, attend, walk, keep: the cache then equals
    the one that the accepted chain alone would have left, and the chain's
    next row sees the same keys."""
    rng = np.random.default_rng(5)
    heads, kvh, d, prefix, n, vocab = 8, 2, 64, 90, 25, 300
    parents = T.random_parents(n, rng, 3)
    depth, see = T.layout(parents)
    k, v = layers(rng, kvh, prefix + n, d, dtype)
    kv = torch.stack([k, v])
    qkv = torch.tensor(rng.standard_normal((n, (heads + 2 * kvh) * d)), dtype=torch.float32, device="cuda")
    form = dict(rotary_dim=d, scaling="yarn", factor=4.0)
    pos = torch.tensor(prefix + depth, dtype=torch.int32, device="cuda")
    q = binding.rope_append(binding.rope(**form), qkv, kv[0], kv[1], prefix, heads, positions=pos)
    out = binding.tree_attention(q, kv[0], kv[1], prefix, mask=torch.tensor(T.pack(see).astype(np.int64), device="cuda"))
    logits = rng.standard_normal((n, vocab)).astype(np.float32)
    best = logits.argmax(axis=1)
    tokens = [0] + [int(best[p]) for p in parents[1:]]
    walk = binding.tree_accept(torch.tensor(logits, device="cuda"), torch.tensor(tokens, dtype=torch.int32, device="cuda"),
                               torch.tensor(parents, device="cuda"))
    binding.kv_keep(kv, prefix, walk)
    w = walk.cpu().numpy()
    path = w[2:2 + w[0]]
    assert len(path) >= 3 and np.array_equal(w, T.walk(logits, tokens, parents))
    # the chain alone: its rows at consecutive positions
    ck, cv = k.clone(), v.clone()
    rows = torch.tensor(path.astype(np.int64), device="cuda")
    cq = binding.rope_append(binding.rope(**form), qkv[rows].contiguous(), ck, cv, prefix, heads, pos0=prefix)
    m = len(path)
    assert torch.equal(kv[0][:, :prefix + m], ck[:, :prefix + m]) and torch.equal(kv[1][:, :prefix + m], cv[:, :prefix + m])
    assert torch.equal(cq, q[rows])
    chain = binding.tree_attention(cq, ck, cv, prefix)
    k64, v64 = f64(ck), f64(cv)
    want, size = T.attention(f64(cq), k64, v64, prefix, np.tril(np.ones((m, m), bool)), 1 / math.sqrt(d))
    tol = T.attention_tol(d, prefix + m, size, np.abs(v64).max())
    assert np.abs(f64(chain) - want).max() <= tol and np.abs(f64(out[rows]) - want).max() <= tol


def test_a_layer_captured_and_replayed():
    """The four operators in one graph, replayed with new inputs in the same
    buffers; every replay against the eager calls, on a cache of its own, with
    eager work between the replays."""
    rng = np.random.default_rng(8)
    heads, kvh, d, prefix, n, vocab = 8, 4, 128, 700, 19, 1000
    parents = T.random_parents(n, rng, 3)
    depth, see = T.layout(parents)
    form = binding.rope(rotary_dim=d)
    pos = torch.tensor(prefix + depth, dtype=torch.int32, device="cuda")
    mask = torch.tensor(T.pack(see).astype(np.int64), device="cuda")
    par = torch.tensor(parents, device="cuda")
    start = torch.randn(2, kvh, prefix + n, d, device="cuda").to(torch.bfloat16)

    def layer(qkv, kv, logits, tokens):
        q = binding.rope_append(form, qkv, kv[0], kv[1], prefix, heads, positions=pos)
        out = binding.tree_attention(q, kv[0], kv[1], prefix, mask=mask)
        walk = binding.tree_accept(logits, tokens, par)
        binding.kv_keep(kv, prefix, walk)
        return q, out, walk

    def inputs(i):
        r = np.random.default_rng(100 + i)
        logits = r.standard_normal((n, vocab)).astype(np.float32)
        best = logits.argmax(axis=1)
        tokens = [0] + [int(best[p]) if r.random() < 0.7 else 5 for p in parents[1:]]
        qkv = r.standard_normal((n, (heads + 2 * kvh) * d))
        return (torch.tensor(qkv, dtype=torch.float32, device="cuda"), torch.tensor(logits, device="cuda"),
                torch.tensor(tokens, dtype=torch.int32, device="cuda"))

    qkv, logits, tokens = inputs(0)
    kv = start.clone()
    layer(qkv, kv, logits, tokens)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = layer(qkv, kv, logits, tokens)
    for i in range(5):
        new = inputs(i)
        for to, x in zip((qkv, logits, tokens), new):
            to.copy_(x)
        kv.copy_(start)
        g.replay()
        mine = start.clone()
        want = layer(new[0], mine, new[1], new[2])
        torch.cuda.synchronize()
        assert torch.equal(kv, mine) and all(torch.equal(a, b) for a, b in zip(outs, want))


def test_calls_on_two_streams_at_once():
    rng = np.random.default_rng(2)
    work = []
    for i in range(2):
        k, v = layers(rng, 4, 2100, 128, "bf16")
        q = torch.randn(9 + 20 * i, 8, 128, device="cuda")
        logits = torch.randn(64, 32000, device="cuda")
        par = torch.tensor(T.random_parents(64, rng), device="cuda")
        tok = torch.zeros(64, dtype=torch.int32, device="cuda")
        want = binding.tree_attention(q, k, v, 2000), binding.tree_accept(logits, tok, par)
        work.append((torch.cuda.Stream(), q, k, v, logits, tok, par, want, []))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, q, k, v, logits, tok, par, _, got in work:
            with torch.cuda.stream(s):
                got.append((binding.tree_attention(q, k, v, 2000), binding.tree_accept(logits, tok, par)))
    torch.cuda.synchronize()
    for *_, want, got in work:
        assert all(torch.equal(a, b) for pair in got for a, b in zip(pair, want))
