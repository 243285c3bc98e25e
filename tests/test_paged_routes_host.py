"""That the calls of the GPU tests are shared out as those say (no GPU is needed)."""

import numpy as np
import pytest

from paper_2309_08168_amd import binding
from tests import paged_routes as R


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("kind", R.STREAMS, ids=str)
def test_chunks_of_several_spans(kind, d, x):
    """Every way in which a sequence can lie in a chunk."""
    c = R.STREAMS[kind]
    p = R.plan_of(c, d, x, "bf16")
    chunks, step = R.layout(c, p)
    assert (p.tile, p.waves) == kind and 1 < p.chunks < sum(k[-1][-1] for k in chunks if k) and step > 1
    ends = [[(first == 0, end == spans) for _, first, end, spans in k] for k in chunks]
    assert any(len(k) > 2 for k in ends)
    assert any((True, True) in k and len(k) > 1 for k in ends)  # a sequence whole beside another
    assert any((False, True) in k and (True, False) in k for k in ends)  # the end of one and the beginning of another
    assert any(k == [(False, False)] for k in ends)  # nothing but the middle of one
    assert any(first == 0 and 1 < end == spans for k in chunks for _, first, end, spans in k)  # whole, of several spans


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("kind", R.MANY_PARTS, ids=str)
def test_sequences_of_many_parts(kind, d, x):
    c = R.MANY_PARTS[kind]
    p = R.plan_of(c, d, x, "bf16")
    assert p.tile == kind[0] and R.parts(c, p) > 64
    assert (p.chunks <= 8 * len(c.rows)) == (kind[1] == 64)


@pytest.mark.parametrize("n,tile", R.MANY)
def test_streams_of_a_thousand_sequences(n, tile):
    """Streams up to 1024 sequences, whole ones past that."""
    c = R.many_sequences(n, tile)
    for x in ("f32", "bf16"):
        p = R.plan_of(c, 32, x, "bf16")
        assert (p.tile, p.chunks > 0) == (tile, n <= 1024)
        if p.chunks:
            assert R.layout(c, p)[1] > 1 and sum(k > p.span for k in c.lengths) > 200


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", R.TILES, ids=str)
def test_tiles_over_pages(kind, d):
    """Sequences of several tiles each."""
    c, tile, shares, wide = R.TILES[kind]
    p = R.plan_of(c, d, kind[1], "bf16")
    assert (p.tile, p.chunks, p.wide) == (tile, 0, wide) and (p.splits == shares if shares else p.splits > 1)
    assert c.max_rows * c.heads // c.kvh > tile


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("kind", R.FEW, ids=str)
def test_few_rows(kind, x):
    p = R.plan_of(R.FEW[kind], 64, x, "bf16")
    assert (p.tile, p.waves) == kind and p.chunks == 0


@pytest.mark.parametrize("d", [16, 64, 128])
def test_tolerance_of_two_terms_does_not_take_one(d):
    """Weights rounded to one bfloat16 term, in the oracle, are outside the tolerance of two: what calls of few
    rows promise would not be lost unseen.  Two terms are within it."""
    torch = pytest.importorskip("torch")

    def rounded(t):
        return torch.tensor(t, dtype=torch.float64).to(torch.bfloat16).double().numpy()

    rng = np.random.default_rng(d)
    rows, length = 32, 60
    q, k, v = (rounded(rng.standard_normal(s)) for s in ((rows, 1, d), (length, d), (length, d)))
    want, size, spread = R.attention(q, k, v, length, rows, length, R.scale_of(d))
    tol = R.tolerance("bf16", "two", d, length, size, np.abs(v).max(), want, spread)
    off = {"one": np.zeros(want.shape), "two": np.zeros(want.shape)}
    for i in range(rows):
        z = k[:length - rows + i + 1] @ q[i, 0] * R.scale_of(d)
        w = np.exp(z - z.max())
        one = rounded(w)
        for name, terms in (("one", one), ("two", one + rounded(w - one))):
            off[name][i, 0] = np.abs(rounded(terms @ v[:len(z)] / w.sum()) - want[i, 0])
    assert (off["two"] <= tol).all() and (off["one"] > tol).mean() > 0.01
    assert (off["one"] <= R.tolerance("bf16", "one", d, length, size, np.abs(v).max(), want, spread)).all()


# ----------------------------------------------------------------------------
# the bounds of a call

AT = 1 << 20  # an aligned address that nothing reads


def refusal(n, heads, seqs, kvh, prompt):
    """What sd_last_error() says of a call of these sizes without queries."""
    lib, kv = binding.load(), binding.sd_kv_pages(AT, AT, kvh * 256, 256, 16, kvh, 4, 16, 16, 1)
    batch = binding.sd_batch(AT, AT, AT, 4, seqs, 4, n, 0)
    ld = heads * 16
    if prompt:
        layer = binding.sd_kv_layer(AT, AT, 16, kvh * 16, kvh, 1 << 20, 16, 1)
        status = lib.sd_prompt_attention(layer, AT, seqs, None, ld, 0, heads, n, 0.0, AT, ld, None)
    else:
        status = lib.sd_paged_attention(kv, batch, None, ld, 0, heads, n, 0.0, AT, ld, AT, 1 << 40, None)
    assert status == binding.SD_ERR_INVALID_ARG
    said = lib.sd_last_error()
    if not prompt and b"q and out" not in said:
        assert lib.sd_paged_attention_workspace(kv, batch, 0, heads, n) == 0 and lib.sd_last_error() == said
    return said


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("n,heads,seqs,kvh,fits", [
    (1 << 20, 64, 3, 8, True), (1 << 20, 65, 3, 5, False), (1 << 20, 128, 3, 8, False), (1 << 14, 4096, 3, 8, True),
    ((1 << 14) + 1, 4096, 3, 8, False), (1 << 16, 64, 1 << 16, 64, True), (1 << 16, 65, 1 << 16, 65, False),
    (1 << 16, 128, 1 << 15, 128, True), (1 << 16, 128, (1 << 15) + 1, 128, False)])
def test_rows_times_heads_and_sequences_times_kv_heads(n, heads, seqs, kvh, fits, prompt):
    """2^26 and 2^22 are taken (refused only further on: without queries), one more of either is not."""
    said = refusal(n, heads, seqs, kvh, prompt)
    assert (b"q and out" in said) == fits and (b"2^26" in said and b"2^22" in said) != fits


def test_pages_that_reach_past_64_bits():
    """Refused for that, and not for a stride that is no multiple of 16 bytes."""
    lib, far = binding.load(), dict(page_stride=1 << 40, head_stride=0, row_stride=128, n_kv_heads=1, page_size=16, head_dim=128)
    batch = binding.sd_batch(AT, AT, AT, 4, 1, 4, 1, 0)
    for n_pages, fits in ((1 << 22, True), ((1 << 22) + 2, False), (2**31 - 1, False)):
        kv = binding.sd_kv_pages(k=AT, v=AT, n_pages=n_pages, dtype=0, **far)
        assert lib.sd_paged_attention(kv, batch, None, 128, 0, 1, 1, 0.0, AT, 128, AT, 1 << 40, None) == binding.SD_ERR_INVALID_ARG
        assert (b"past 64 bits" in lib.sd_last_error()) != fits
