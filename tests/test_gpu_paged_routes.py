"""paged_attention by every way a call is shared out, against float64: streams of many
spans, tiles over pages with and without shares, many sequences.

Tolerances count roundings: see the helpers.  What a row must not see holds NaN throughout.
"""

import numpy as np
import pytest

from tests import paged_routes as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_paged import TYPES, Cache, _gpu, check_append, f64, gpu, starts_of  # noqa: E402,F401

if torch.cuda.is_available():
    from paper_2309_08168_amd import binding


def apart(t, row_stride):
    """A copy of pages whose rows lie row_stride elements apart, all first rows beside each other."""
    pages, kvh, page, d = t.shape
    flat = torch.empty((page - 1) * row_stride + pages * kvh * d, dtype=t.dtype, device=t.device)
    far = flat.as_strided(t.shape, (kvh * d, d, row_stride, 1))
    return far.copy_(t)


def check(call, d, x, dtype, want_plan=None, max_length=0, gap=0, heads_of=None, spoil=None, seed=0, row_stride=0):
    """One call, on some kv heads (all of a few) against float64.  want_plan: what its plan has to hold."""
    rng = np.random.default_rng(seed + 31 * sum(call.rows) + sum(call.lengths) + d)
    rows, lengths, kvh, heads = call.rows, call.lengths, call.kvh, call.heads
    c = Cache(rng, lengths, kvh, call.page, d, dtype)
    if spoil is not None:
        spoil(c)
    k, v = (apart(t, row_stride) for t in (c.k, c.v)) if row_stride else (c.k, c.v)
    starts, G = starts_of(rows, gap), heads // kvh
    n = int(starts[-1]) + gap
    q = torch.tensor(rng.standard_normal((n, heads, d)), dtype=TYPES[x], device="cuda")
    out = torch.full((n, heads, d), 5.0, dtype=TYPES[x], device="cuda")
    batch = binding.batch(gpu(c.table), gpu(lengths), gpu(starts), call.max_rows, max_length)
    p = R.plan(binding.kv_pages(k, v), batch, x, heads, n)
    for name, value in (want_plan or {}).items():
        assert getattr(p, name) == value, (name, p)
    got, q64 = f64(binding.paged_attention(q, k, v, batch, out=out)), f64(q)
    limit = max_length or c.table.shape[1] * call.page
    of_heads = range(kvh) if kvh <= 4 else sorted({0, 1, kvh // 2, kvh - 1}) if heads_of is None else heads_of
    vmax = max(np.abs(v).max() for v in c.v64 if v.size)
    live = np.zeros(n, bool)
    for s, (m, length) in enumerate(zip(rows, lengths)):
        at, take = starts[s], min(m, call.max_rows)
        live[at:at + take] = True
        pages = c.table[s, np.arange(length) // call.page]
        there = (pages >= 0) & (pages < c.n_pages)
        for g in of_heads if m else ():
            hs = slice(g * G, (g + 1) * G)
            want, size, spread = R.attention(q64[at:at + m, hs], c.k64[s][:, g], c.v64[s][:, g], length, take, limit,
                                             R.scale_of(d), there)
            tol = R.tolerance(x, R.weight_of(p, dtype), d, max(length, 1), size, vmax, want, spread)
            off = np.abs(got[at:at + take, hs] - want)
            assert (off <= tol).all(), (s, g, float(np.nanmax(off / tol)))
    assert np.isfinite(got).all() and (got[~live] == 5.0).all()
    return p


# ----------------------------------------------------------------------------
# streams


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("kind", R.STREAMS, ids=str)
def test_chunks_of_several_spans(kind, d, x):
    """Chunks that hold several sequences, parts of them, and one whose middle is all of it."""
    p = check(R.STREAMS[kind], d, x, "bf16", dict(tile=kind[0], waves=kind[1]))
    assert p.chunks and R.layout(R.STREAMS[kind], p)[1] > 1


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("kind", R.MANY_PARTS, ids=str)
def test_sequences_of_many_parts(kind, d, x):
    """More parts than a wave has lanes, joined by one wave and by four."""
    p = check(R.MANY_PARTS[kind], d, x, "bf16", dict(tile=kind[0]))
    assert p.chunks and R.parts(R.MANY_PARTS[kind], p) > 64


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("n,tile", R.MANY)
def test_streams_of_a_thousand_sequences(n, tile, x):
    """As many as a work-group adds up the spans of, and one more, which takes them whole."""
    p = check(R.many_sequences(n, tile), 32, x, "bf16", dict(tile=tile))
    assert (p.chunks > 0) == (n <= 1024)


# ----------------------------------------------------------------------------
# tiles


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", R.TILES, ids=str)
def test_tiles_over_pages(kind, d):
    """Sequences of several tiles, some of them short, rows of no sequence around them and pages that are not there."""
    def spoil(c):
        c.table[0, 1], c.table[3, 0], c.table[2, 1 if c.table.shape[1] > 2 else 0] = -1, c.n_pages, -2**31

    call, tile, shares, wide = R.TILES[kind]
    p = check(call, d, kind[1], "bf16", dict(tile=tile, chunks=0, wide=wide), gap=3)
    assert p.splits == shares if shares else p.splits > 1
    if len(call.rows) > 1:
        check(call, d, kind[1], "bf16", dict(tile=tile, chunks=0, wide=wide), spoil=spoil, seed=1)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("name", ["five chunks, 64-row tiles", "one chunk", "70 sequences, shares"])
def test_tiles_over_float32_pages(name, d, x):
    call = R.TILES[name, x][0]
    check(call._replace(heads=call.heads // (call.kvh // 2), kvh=2), d, x, "f32", dict(tile=16, chunks=0), gap=1)


# ----------------------------------------------------------------------------
# few rows


@pytest.mark.parametrize("x,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", R.FEW, ids=str)
def test_few_rows_hold_their_weights(kind, d, x, dtype):
    """Two bfloat16 terms of a softmax weight, and all of it over float32 pages: the tolerance has no room for one term."""
    check(R.FEW[kind], d, x, dtype, dict(tile=kind[0], waves=kind[1], chunks=0) if dtype == "bf16" else dict(tile=16), gap=1)


# ----------------------------------------------------------------------------
# rows far apart, large pages

FAR = [("few", (16, 4), "bf16"), ("few", (32, 4), "f32"), ("few", (32, 1), "bf16"), ("streams", (16, 8), "bf16"),
       ("streams", (64, 4), "f32"), ("streams", (128, 4), "bf16"), ("five chunks, 64-row tiles", "bf16"),
       ("five chunks, tiles for every CU", "bf16"), ("five chunks, small pages", "bf16"), ("one chunk", "bf16"), ("one chunk", "f32")]


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("row_stride", [2**24 - 8, 2**24], ids=["near", "far"])
@pytest.mark.parametrize("kind", FAR, ids=str)
def test_rows_far_apart(kind, row_stride, d):
    """The last stride at which a lane's offsets within a block are 32 bits, and the first at which they are not."""
    if kind[0] in ("few", "streams"):
        call, tile = (R.FEW if kind[0] == "few" else R.STREAMS)[kind[1]], kind[1][0]
    else:
        call, tile = R.TILES[kind][:2]
    check(call, d, kind[-1], "bf16", dict(tile=tile), row_stride=row_stride)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("kind", [(16, 4), (32, 4)], ids=str)
def test_rows_of_float32_pages_far_apart(kind, x):
    check(R.FEW[kind], 64, x, "f32", dict(tile=16), row_stride=2**24)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 64])
@pytest.mark.parametrize("row_stride", [2**24 - 8, 2**24], ids=["near", "far"])
@pytest.mark.parametrize("heads,kvh", [(4, 2), (832, 13)])
def test_prompt_rows_far_apart(heads, kvh, row_stride, d, x):
    """Tiles of 64 rows, and of 128 (more than 450 of them)."""
    rng = np.random.default_rng(kvh + d)
    n, G = 70, heads // kvh
    kv = torch.tensor(rng.standard_normal((2, 1, kvh, n, d)), dtype=torch.bfloat16, device="cuda")
    k, v = (apart(t, row_stride)[0] for t in kv)
    q = torch.tensor(rng.standard_normal((n, heads, d)), dtype=TYPES[x], device="cuda")
    got, q64, k64, v64 = (f64(t) for t in (binding.prompt_attention(q, k, v), q, kv[0, 0], kv[1, 0]))
    for g in range(kvh):
        hs = slice(g * G, (g + 1) * G)
        want, size, spread = R.attention(q64[:, hs], k64[g], v64[g], n, n, n, R.scale_of(d))
        tol = R.tolerance(x, "one", d, n, size, np.abs(v64).max(), want, spread)
        assert (np.abs(got[:, hs] - want) <= tol).all(), g


@pytest.mark.parametrize("page", [1024, 65536])
@pytest.mark.parametrize("x,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("rows,heads", [([1, 2, 1], 8), ([4, 3, 1], 16), ([16, 1, 9], 16), ([130, 60, 1], 8)])
def test_large_pages(rows, heads, x, dtype, page):
    """Sequences that end within a page, at its end and behind it."""
    call = R.Call(rows, [page + 1000, page, 200], heads, 2, page, max(rows))
    check(call, 64, x, dtype)
    check(call._replace(lengths=[1500, 1024, 200]), 64, x, dtype, max_length=1500)


@pytest.mark.parametrize("x,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
def test_append_to_large_pages(x, dtype):
    assert check_append([5, 3, 1], [65538, 65536, 7], 2, 1, 16, x, dtype, dict(rotary_dim=16), 65536) == 9


# ----------------------------------------------------------------------------
# batches of some of the sequences


@pytest.mark.parametrize("x,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("cut", [0, 1, 5, 8])
def test_a_step_as_two_batches(cut, x, dtype):
    """Tokens and a chunk: one call and two over slices of the same tensors, appends too; each writes its own rows."""
    rng = np.random.default_rng(cut)
    rows, past, heads, kvh, d, page = [1] * 5 + [3, 1, 1, 130], [700, 0, 1500, 40, 63, 10, 2000, 1, 300], 8, 2, 64, 32
    lengths, starts, n = [m + p for m, p in zip(rows, past)], starts_of(rows), sum(rows)
    c = Cache(rng, lengths, kvh, page, d, dtype)
    table, at, begin = gpu(c.table), gpu(lengths), gpu(starts)
    qkv = torch.tensor(rng.standard_normal((n, (heads + 2 * kvh) * d)), dtype=TYPES[x], device="cuda")
    form = binding.rope(rotary_dim=d)
    halves = [slice(0, cut), slice(cut, len(rows))]
    batches = [binding.batch(table[h], at[h], begin[h.start:h.stop + 1], max(rows[h]), max(lengths[h])) for h in halves if rows[h]]
    k, v = c.k.clone(), c.v.clone()
    whole = binding.batch(table, at, begin, max(rows))
    q = binding.paged_append(form, qkv, c.k, c.v, whole, heads)
    q2 = torch.full_like(q, 3.0)
    for b in batches:
        binding.paged_append(form, qkv, k, v, b, heads, q_out=q2)
    assert torch.equal(q, q2) and torch.equal(k.nan_to_num(7.0), c.k.nan_to_num(7.0)) and torch.equal(v.nan_to_num(7.0), c.v.nan_to_num(7.0))
    out = torch.full_like(q, 3.0)
    for b in batches:
        binding.paged_attention(q, k, v, b, out=out)
    one = binding.paged_attention(q, k, v, whole)
    q64, k64, v64 = f64(q), f64(k), f64(v)
    for s, (m, length) in enumerate(zip(rows, lengths)):
        pos = np.arange(length)
        pages, place = c.table[s, pos // page], pos % page
        for g in range(kvh):
            a, hs = slice(starts[s], starts[s] + m), slice(g * heads // kvh, (g + 1) * heads // kvh)
            kk, vv = k64[pages, g, place], v64[pages, g, place]
            want, size, spread = R.attention(q64[a, hs], kk, vv, length, m, length, R.scale_of(d))
            tol = R.tolerance(x, "float32" if dtype == "f32" else "one", d, length, size, np.abs(vv).max(), want, spread)
            assert (np.abs(f64(out[a, hs]) - want) <= tol).all() and (np.abs(f64(one[a, hs]) - want) <= tol).all(), (s, g)
