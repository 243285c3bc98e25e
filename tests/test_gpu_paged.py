"""The operators of batches on the GPU against their plain float64 forms.

Tolerances count roundings: float32 results those on the way (2^-24 each, see the
helpers); what is stored as bfloat16 adds half a step, 2^-8 of the value.
What a row must not see (unused rows of pages, pages of no sequence, later positions)
holds NaN throughout.
"""

import math

import numpy as np
import pytest

from tests import paged_ref as P
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


def f64(t):
    return t.detach().double().cpu().numpy()


def gpu(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def page_tensors(kvh, pages, page, d, dtype, order="heads"):
    """k and v [pages, kvh, page, d] of NaN; order: which dimension lies where."""
    def new(*shape):
        return torch.full(shape, float("nan"), dtype=TYPES[dtype], device="cuda")

    if order == "rows":  # [pages][page][kvh][d]
        return new(pages, page, kvh, d).transpose(1, 2), new(pages, page, kvh, d).transpose(1, 2)
    if order == "outer":  # [kvh][pages][page][d]
        return new(kvh, pages, page, d).transpose(0, 1), new(kvh, pages, page, d).transpose(0, 1)
    if order == "joined":  # k and v of a page beside each other, rows with a gap
        kv = new(pages, 2, kvh, page, d + 16)
        return kv[:, 0, ..., :d], kv[:, 1, ..., :d]
    return new(pages, kvh, page, d), new(pages, kvh, page, d)


class Cache:
    """Pages of a batch whose sequences hold `lengths` positions; every other row of them is NaN."""

    def __init__(self, rng, lengths, kvh, page, d, dtype, order="heads", spare=2, fill=True, peak=1.0):
        self.page, self.lengths = page, lengths
        need = [-(-n // page) for n in lengths]
        self.n_pages = sum(need) + spare
        free = list(rng.permutation(self.n_pages))
        width = max(need + [1]) + 1
        self.table = np.full((len(lengths), width), -1, np.int64)
        for s, c in enumerate(need):
            self.table[s, :c] = [free.pop() for _ in range(c)]
            self.table[s, c:] = rng.choice([-1, self.n_pages, 2**31 - 1, -2**31], width - c)
        self.k, self.v = page_tensors(kvh, self.n_pages, page, d, dtype, order)
        self.k64, self.v64 = [], []
        for s, n in enumerate(lengths):
            a, b = (torch.tensor(peak * rng.standard_normal((n, kvh, d)), dtype=TYPES[dtype], device="cuda") for _ in "kv")
            if fill:
                pos = np.arange(n)
                at, row = gpu(self.table[s, pos // page], torch.int64), gpu(pos % page, torch.int64)
                self.k[at, :, row], self.v[at, :, row] = a, b
            self.k64.append(f64(a))
            self.v64.append(f64(b))


def starts_of(rows, gap=0):
    return np.concatenate([[gap], gap + np.cumsum(rows)]).astype(int)


# ----------------------------------------------------------------------------
# paged_append

FORMS = [dict(rotary_dim=64), dict(rotary_dim=64, layout="interleaved"), dict(rotary_dim=32, scaling="linear", factor=4.0),
         dict(rotary_dim=48, layout="interleaved", scaling="ntk", factor=2.5), dict(rotary_dim=64, scaling="yarn", factor=16.0),
         dict(rotary_dim=20, scaling="yarn", factor=4.0, original_context=512, beta_fast=20.0, beta_slow=2.0, gain=1.25),
         dict(rotary_dim=6, layout="interleaved", base=500.0), dict(rotary_dim=2)]


def check_append(rows, lengths, heads, kvh, d, x, dtype, form, page=16, norm=False, order="heads", far=None, gap=0,
                 uniform=False, max_rows=None, max_length=0, strided=False, seed=0, eps=1e-5, spoil=None):
    rng = np.random.default_rng(seed + 7 * sum(rows) + len(rows))
    starts = starts_of(rows, gap)
    n = int(starts[-1]) + gap
    c = Cache(rng, lengths, kvh, page, d, dtype, order, fill=False)
    if spoil is not None:
        spoil(c)
    c.k.normal_(), c.v.normal_()
    k0, v0 = f64(c.k), f64(c.v)
    width = (heads + 2 * kvh) * d
    buf = torch.tensor(rng.standard_normal((n, width + (16 if strided else 0))), dtype=TYPES[x], device="cuda")
    qkv = buf[:, :width]
    wq, wk = (torch.tensor(1 + 0.3 * rng.standard_normal(d), dtype=TYPES[dtype], device="cuda") for _ in "qk")
    bound = max_rows or max(max(rows), 1)
    batch = binding.batch(gpu(c.table), gpu(lengths), None if uniform else gpu(starts), bound, max_length)
    q_out = torch.full((n, heads + (1 if strided else 0), d), 7.0, dtype=TYPES[x], device="cuda")
    places = P.row_places(starts, lengths, n, bound)
    pos = np.array([0 if t is None else t[1] for t in places])
    positions = None if far is None else gpu(far + 3 * np.arange(n))
    if far is not None:
        pos = far + 3 * np.arange(n)
    got = binding.paged_append(binding.rope(**form), qkv, c.k, c.v, batch, heads, positions=positions, eps=eps,
                               q_norm=wq if norm else None, k_norm=wk if norm else None, q_out=q_out[:, :heads])
    x64 = f64(qkv).reshape(n, heads + 2 * kvh, d)
    qk, raw = x64[:, :heads + kvh].copy(), np.abs(x64).max()
    if norm:
        qk[:, :heads] = P.normed(qk[:, :heads], f64(wq), eps)
        qk[:, heads:] = P.normed(qk[:, heads:], f64(wk), eps)
    want = T.rope(qk, pos, form)
    # angle, cosine and sine, gain, two products and a sum: eight roundings of |a| + |b|; a
    # norm's squares, their sum, mean, eps, root, quotient and two products: d / 8 + 16 more
    gain = form.get("gain") or (0.1 * math.log(form["factor"]) + 1.0 if form.get("scaling") == "yarn" else 1.0)
    tol = (8 + (d / 8 + 16 if norm else 0)) * 2.0 ** -24 * gain * 2 * max(raw, np.abs(qk).max())
    hx, hc = (P.HALF[t] if t == "bf16" else 0.0 for t in (x, dtype))
    live = np.array([t is not None for t in places])
    q64 = f64(got)
    assert (np.abs(q64 - want[:, :heads])[live] <= (hx * np.abs(want[:, :heads]) + tol * (1 + hx))[live]).all()
    assert (q64[~live] == 7.0).all()
    if strided:
        assert (q_out[:, heads:] == 7.0).all()
    limit = max_length or c.table.shape[1] * page
    wk64, wv64, new = k0.copy(), v0.copy(), np.zeros(k0.shape, bool)
    for r, t in enumerate(places):
        at = None if t is None else P.page_row(c.table, t[0], t[1], page, c.n_pages, limit)
        if at is not None:
            b, o = at
            new[b, :, o] = True
            wk64[b, :, o], wv64[b, :, o] = want[r, heads:], x64[r, heads + kvh:]
    k64, v64 = f64(c.k), f64(c.v)
    assert np.array_equal(k64[~new], k0[~new]) and np.array_equal(v64[~new], v0[~new])
    assert (np.abs(k64 - wk64) <= hc * np.abs(wk64) + tol * (1 + hc))[new].all()
    assert np.array_equal(v64[new], torch.tensor(wv64[new]).to(TYPES[dtype]).double().numpy())
    return new.any(axis=(1, 3)).sum()


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("x,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_append_forms(form, norm, x, dtype):
    assert check_append([3, 1, 2], [40, 1, 17], 6, 2, 64, x, dtype, form, norm=norm) == 6


@pytest.mark.parametrize("rows,lengths,heads,kvh,d,page", [
    ([1], [1], 1, 1, 16, 16), ([1] * 70, list(range(1, 71)), 8, 8, 128, 16), ([33, 0, 1, 0, 90], [33, 5, 200, 0, 91], 64, 8, 128, 32),
    ([300], [1000], 4, 4, 32, 256), ([0, 0, 2], [0, 9, 2], 5, 5, 16, 64), ([5, 1] * 40, [7, 400] * 40, 2, 1, 64, 128)])
@pytest.mark.parametrize("norm", [False, True])
def test_append_sizes(rows, lengths, heads, kvh, d, page, norm):
    assert check_append(rows, lengths, heads, kvh, d, "f32", "bf16", dict(rotary_dim=d), page, norm) == sum(rows)


@pytest.mark.parametrize("order", ["rows", "outer", "joined"])
@pytest.mark.parametrize("rotary_dim", [64, 10])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_append_strides(order, rotary_dim, x):
    check_append([4, 5], [30, 5], 4, 2, 64, x, "bf16", dict(rotary_dim=rotary_dim), order=order, strided=True, norm=True)


def test_append_uniform_rows():
    assert check_append([3, 3, 3], [3, 50, 20], 4, 2, 64, "f32", "bf16", dict(rotary_dim=64), uniform=True) == 9


@pytest.mark.parametrize("far", [0, 2**31 - 40, -100])
def test_append_positions_of_their_own(far):
    check_append([4, 9], [30, 9], 4, 2, 64, "f32", "f32", dict(rotary_dim=64), far=far)


def test_append_rows_outside_sequences_are_left():
    """A padded batch: rows before the first sequence and behind the last."""
    assert check_append([4, 9], [30, 9], 4, 2, 64, "bf16", "bf16", dict(rotary_dim=64), gap=5) == 13


def test_append_rows_past_max_rows_are_left():
    assert check_append([4, 9, 1], [30, 9, 3], 4, 2, 64, "f32", "bf16", dict(rotary_dim=64), max_rows=3) == 7


def test_append_negative_and_late_positions_are_not_stored():
    """Positions -2 .. 1, -3 .. -1, 29 .. 30 and 62 .. 63 of max_length 30; q comes all the same."""
    assert check_append([4, 3, 2, 2], [2, 0, 31, 64], 4, 2, 64, "f32", "bf16", dict(rotary_dim=64), max_length=30) == 3


def test_append_bad_pages_are_not_stored():
    def spoil(c):
        c.table[0, 1], c.table[1, 0], c.table[2, 0] = -1, c.n_pages, -2**31

    assert check_append([20, 4, 3], [40, 4, 3], 4, 2, 64, "f32", "bf16", dict(rotary_dim=64), spoil=spoil) == 8


def test_append_many_sequences():
    """More than the 64 that a wave looks at together, and than 64 times 64."""
    rng = np.random.default_rng(3)
    rows = [int(m) for m in rng.integers(0, 3, 4200)]
    assert check_append(rows, [m + 1 for m in rows], 1, 1, 16, "f32", "f32", dict(rotary_dim=16)) == sum(rows)


# ----------------------------------------------------------------------------
# paged_attention


def check_paged(rows, lengths, heads, kvh, d, x, dtype, page=16, order="heads", scale=0.0, gap=0, uniform=False,
                max_rows=None, max_length=0, seed=0, spoil=None, peak=1.0, strided=False, odd_q=None, value_of=None):
    rng = np.random.default_rng(seed + 7 * sum(rows) + sum(lengths))
    starts = starts_of(rows, gap)
    n = int(starts[-1]) + gap
    c = Cache(rng, lengths, kvh, page, d, dtype, order)
    if spoil is not None:
        spoil(c)
    bound = max_rows or max(max(rows), 1)
    wide = torch.tensor(peak * rng.standard_normal((n, heads + (2 if strided else 0), d)), dtype=TYPES[x], device="cuda")
    q = wide[:, :heads]
    if odd_q is not None:
        q[odd_q] = float("nan")
    batch = binding.batch(gpu(c.table), gpu(lengths), None if uniform else gpu(starts), bound, max_length)
    out = torch.full((n, heads + (1 if strided else 0), d), 5.0, dtype=TYPES[x], device="cuda")
    got = binding.paged_attention(q, c.k, c.v, batch, scale=scale, out=out[:, :heads])
    G, sc, limit = heads // kvh, scale if scale else 1.0 / math.sqrt(d), max_length or c.table.shape[1] * page
    places = P.row_places(starts, lengths, n, bound)

    def seen(side):
        def of(r, h):
            s, p = places[r]
            pos = [j for j in range(max(0, min(p + 1, limit))) if P.page_row(c.table, s, j, page, c.n_pages, limit)]
            return side[s][pos, h // G]
        return of

    want, size, spread = P.attention(f64(q), seen(c.k64), seen(c.v64), lambda r: places[r] is not None, sc)
    tol = P.attention_tol(x, d, max(lengths + [1]), size, max([1e-30] + [np.abs(v).max() for v in c.v64 if v.size]), want, spread)
    live = np.array([t is not None for t in places])
    if odd_q is not None:
        live[odd_q] = False
    g64 = f64(got)
    assert (np.abs(g64 - want)[live] <= np.broadcast_to(tol, want.shape)[live]).all(), \
        np.nanmax(np.abs(g64 - want)[live] / np.broadcast_to(tol, want.shape)[live])
    gone = np.array([t is None for t in places])
    assert (g64[gone] == 5.0).all()
    if strided:
        assert (out[:, heads:] == 5.0).all()
    return got


KINDS = [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")]


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,kvh", [(2, 2), (8, 1), (6, 2)])
def test_paged_tokens(x, dtype, d, heads, kvh):
    check_paged([1] * 7, [1, 2, 16, 17, 63, 130, 300], heads, kvh, d, x, dtype)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("page", [16, 32, 64, 512])
@pytest.mark.parametrize("rows,lengths", [([5, 1, 0, 13], [5, 200, 4, 77]), ([40, 3], [141, 3]), ([130], [150])])
def test_paged_rows(x, dtype, page, rows, lengths):
    check_paged(rows, lengths, 4, 2, 64, x, dtype, page)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("d,heads,kvh", [(16, 16, 1), (32, 4, 4), (128, 16, 2), (128, 3, 3)])
@pytest.mark.parametrize("m", [2, 9, 33])
def test_paged_chains(x, dtype, d, heads, kvh, m):
    check_paged([m, 1, m // 2], [m + 41, 90, m // 2], heads, kvh, d, x, dtype, 32)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("order", ["rows", "outer", "joined"])
@pytest.mark.parametrize("d", [32, 128])
def test_paged_strides(x, dtype, order, d):
    check_paged([1, 6, 2], [70, 40, 2], 4, 2, d, x, dtype, order=order, strided=True)
    check_paged([45, 6], [170, 40], 4, 2, d, x, dtype, 64, order=order, strided=True)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("rows,lengths", [([1, 1, 1], [5000, 1, 777]), ([4], [6001]), ([60, 2], [3100, 900])])
def test_paged_long(x, dtype, rows, lengths):
    """Contexts in several shares."""
    check_paged(rows, lengths, 4, 1, 64, x, dtype, 128)


@pytest.mark.parametrize("x,dtype", KINDS)
def test_paged_empty_rows(x, dtype):
    """Lengths of zero, and below the rows: rows that see nothing give zeros."""
    got = check_paged([3, 1, 4, 2], [0, 0, 2, 50], 4, 2, 64, x, dtype)
    assert (got[:6] == 0).all() and (got[6:] != 0).any()


@pytest.mark.parametrize("x,dtype", KINDS)
def test_paged_gaps_and_bounds(x, dtype):
    check_paged([3, 1, 9], [30, 70, 9], 4, 2, 64, x, dtype, gap=4)
    check_paged([3, 1, 9], [30, 70, 9], 4, 2, 64, x, dtype, max_rows=2)
    check_paged([3, 1, 40], [30, 70, 99], 4, 2, 64, x, dtype, max_rows=20)
    check_paged([3, 1, 9, 1], [30, 70, 9, 33], 4, 2, 64, x, dtype, max_length=32)
    check_paged([2, 2, 2], [30, 70, 2], 4, 2, 64, x, dtype, uniform=True)
    check_paged([50, 50], [300, 70], 4, 2, 64, x, dtype, uniform=True)
    check_paged([1] * 5, [30, 70, 2, 0, 1], 4, 2, 64, x, dtype, uniform=True)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("m", [1, 20])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_paged_bad_pages_hold_nothing(x, dtype, m, page):
    def spoil(c):
        c.table[0, 1], c.table[1, 0] = -1, c.n_pages
        c.table[2, -3:] = 2**31 - 1

    check_paged([m, 1, m], [4 * page + 5, page + 9, 300], 4, 2, 64, x, dtype, page, spoil=spoil)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("m", [5, 40])
def test_paged_later_rows_change_no_bit(x, dtype, m):
    """Infinities and NaN at later rows' positions, and in other rows' queries."""
    rng = np.random.default_rng(11)
    c = Cache(rng, [m + 30], 2, 16, 64, dtype)
    q = torch.tensor(rng.standard_normal((m, 8, 64)), dtype=TYPES[x], device="cuda")
    batch = binding.batch(gpu(c.table), gpu([m + 30]), None, m)
    want = binding.paged_attention(q, c.k, c.v, batch).clone()
    for bad in (float("nan"), float("inf"), -float("inf")):
        k, v, q2 = c.k.clone(), c.v.clone(), q.clone()
        for p in range(30 + m // 2 + 1, 30 + m):
            b = int(c.table[0, p // 16])
            k[b, :, p % 16], v[b, :, p % 16, ::3] = bad, bad
        q2[m // 2 + 1:] = bad
        got = binding.paged_attention(q2, k, v, batch)
        assert torch.equal(got[:m // 2 + 1], want[:m // 2 + 1]), bad


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("m", [3, 40])
def test_paged_seen_infinities_arrive(x, dtype, m):
    """An infinite value that a row sees is its result's, and no earlier row's."""
    rng = np.random.default_rng(12)
    c = Cache(rng, [m + 20], 1, 16, 64, dtype)
    q = torch.tensor(rng.standard_normal((m, 2, 64)), dtype=TYPES[x], device="cuda")
    batch = binding.batch(gpu(c.table), gpu([m + 20]), None, m)
    want = binding.paged_attention(q, c.k, c.v, batch).clone()
    p = 20 + m // 2
    c.v[int(c.table[0, p // 16]), :, p % 16, 5] = float("inf")
    got = binding.paged_attention(q, c.k, c.v, batch)
    rest = [e for e in range(64) if e != 5]
    assert torch.equal(got[..., rest], want[..., rest]) and torch.equal(got[:m // 2], want[:m // 2])
    assert (got[m // 2:, :, 5] == float("inf")).all()


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("m", [1, 30])
def test_paged_peaks_and_scales(x, dtype, m):
    """Scores of hundreds, where one key takes all the weight; a negative scale."""
    check_paged([m, m], [90, 250], 4, 2, 64, x, dtype, peak=8.0)
    check_paged([m, m], [90, 250], 4, 2, 64, x, dtype, scale=-0.3)
    check_paged([m, m], [90, 250], 4, 2, 64, x, dtype, scale=1e-30)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("m", [1, 17])
def test_paged_scores_that_grow(x, dtype, m):
    """Keys in ascending order of their score: every block raises the maximum."""
    rng = np.random.default_rng(5)
    c = Cache(rng, [600], 1, 16, 32, dtype)
    q = torch.zeros(m, 1, 32, dtype=TYPES[x], device="cuda")
    q[:, :, 0] = 1.0
    for p in range(600):
        c.k64[0][p] = 0.0
        c.k64[0][p, 0, 0] = float(torch.tensor(p / 8.0).to(TYPES[dtype]))
        c.k[int(c.table[0, p // 16]), :, p % 16] = torch.tensor(c.k64[0][p], device="cuda").to(TYPES[dtype])
    batch = binding.batch(gpu(c.table), gpu([600]), None, m)
    got = f64(binding.paged_attention(q, c.k, c.v, batch, scale=1.0))
    for i in range(m):
        p = 600 - m + i
        want, size, spread = P.attention(f64(q[i:i + 1]), lambda r, h: c.k64[0][:p + 1, h], lambda r, h: c.v64[0][:p + 1, h],
                                         lambda r: True, 1.0)
        tol = P.attention_tol(x, 32, 600, size, np.abs(c.v64[0]).max(), want, spread)
        assert (np.abs(got[i:i + 1] - want) <= tol).all()


def test_paged_offsets_past_32_bits():
    """A row of a page 5 GB from its start: pages of a wide stride."""
    rng = np.random.default_rng(8)
    page, d, far = 16, 64, 1_300_000_000
    flat = torch.zeros(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    k = flat.as_strided((3, 1, page, d), (far, 2 * page * d, d, 1))
    v = flat.as_strided((3, 1, page, d), (far, 2 * page * d, d, 1), page * d)
    for t in (k, v):
        t.copy_(torch.tensor(rng.standard_normal((3, 1, page, d)), dtype=torch.bfloat16))
    for m in (1, 40):
        q = torch.tensor(rng.standard_normal((m, 2, d)), dtype=torch.float32, device="cuda")
        got = f64(binding.paged_attention(q, k, v, binding.batch(gpu([[2, 0, 1]]), gpu([45]), None, m)))
        near = binding.paged_attention(q, k.contiguous(), v.contiguous(), binding.batch(gpu([[2, 0, 1]]), gpu([45]), None, m))
        assert np.array_equal(got, f64(near)) and np.isfinite(got).all() and (got[-1] != 0).any()
    qkv = torch.tensor(rng.standard_normal((2, 3 * d)), dtype=torch.float32, device="cuda")
    binding.paged_append(binding.rope(rotary_dim=d), qkv, k, v, binding.batch(gpu([[2, 0, 1]]), gpu([45]), None, 2), 1)
    assert torch.equal(v[1, 0, 11:13].float(), qkv[:, 2 * d:].bfloat16().float())


# ----------------------------------------------------------------------------
# prompt_attention


def check_prompt(rows, heads, kvh, d, x, dtype, order="rows", gap=0, scale=0.0, whole=False, seed=0, peak=1.0):
    rng = np.random.default_rng(seed + 3 * sum(rows) + heads)
    starts = starts_of(rows, gap)
    n = int(starts[-1]) + gap
    pad = {"rows": 0, "heads": 3}[order]
    kv = torch.tensor(rng.standard_normal((2, n + pad, kvh, d)), dtype=TYPES[dtype], device="cuda")
    k64, v64 = f64(kv[0]), f64(kv[1])
    for r in list(range(gap)) + list(range(n - gap, n + pad)):
        kv[:, r] = float("nan")
    k, v = (t.transpose(0, 1) if order == "rows" else t.transpose(0, 1).contiguous() for t in kv)
    q = torch.tensor(peak * rng.standard_normal((n, heads, d)), dtype=TYPES[x], device="cuda")
    out = torch.full((n, heads, d), 5.0, dtype=TYPES[x], device="cuda")
    got = f64(binding.prompt_attention(q, k, v, None if whole else gpu(starts), scale=scale, out=out))
    where = {}
    for s, m in enumerate(rows):
        for i in range(m):
            where[starts[s] + i] = starts[s]
    G, sc = heads // kvh, scale if scale else 1.0 / math.sqrt(d)
    want, size, spread = P.attention(f64(q), lambda r, h: k64[where[r]:r + 1, h // G], lambda r, h: v64[where[r]:r + 1, h // G],
                                     lambda r: r in where, sc)
    tol = np.broadcast_to(P.attention_tol(x, d, max(rows + [1]), size, np.abs(v64).max(), want, spread), want.shape)
    live = np.array([r in where for r in range(n)])
    assert (np.abs(got - want)[live] <= tol[live]).all(), np.nanmax(np.abs(got - want)[live] / tol[live])
    assert (got[~live] == 5.0).all()


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,kvh", [(2, 2), (8, 1), (6, 2)])
def test_prompt_packed(x, dtype, d, heads, kvh):
    check_prompt([1, 70, 0, 2, 33, 129], heads, kvh, d, x, dtype)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 257])
def test_prompt_lengths(x, dtype, n):
    check_prompt([n], 2, 1, 64, x, dtype, whole=True)


@pytest.mark.parametrize("x,dtype", KINDS)
def test_prompt_orders_gaps_scales(x, dtype):
    check_prompt([40, 1, 90], 4, 2, 64, x, dtype, order="heads")
    check_prompt([40, 1, 90], 4, 2, 128, x, dtype, gap=7)
    check_prompt([40, 150], 4, 4, 32, x, dtype, scale=-0.2)
    check_prompt([40, 150], 3, 1, 32, x, dtype, peak=8.0)
    check_prompt([0, 0, 5, 0], 3, 1, 32, x, dtype)


@pytest.mark.parametrize("x,dtype", KINDS)
def test_prompt_many_sequences(x, dtype):
    rng = np.random.default_rng(2)
    check_prompt([int(m) for m in rng.integers(0, 4, 300)], 2, 1, 16, x, dtype)


@pytest.mark.parametrize("x,dtype", KINDS)
def test_prompt_longer(x, dtype):
    check_prompt([700, 30], 2, 1, 128, x, dtype)


@pytest.mark.parametrize("x,dtype", KINDS)
def test_prompt_later_rows_change_no_bit(x, dtype):
    rng = np.random.default_rng(4)
    n, at = 150, 70
    kv = torch.tensor(rng.standard_normal((2, n, 2, 64)), dtype=TYPES[dtype], device="cuda")
    q = torch.tensor(rng.standard_normal((n, 4, 64)), dtype=TYPES[x], device="cuda")
    want = binding.prompt_attention(q, kv[0].transpose(0, 1), kv[1].transpose(0, 1)).clone()
    for bad in (float("nan"), float("inf"), -float("inf")):
        kv2, q2 = kv.clone(), q.clone()
        kv2[:, at:, :, ::5], q2[at:] = bad, bad
        got = binding.prompt_attention(q2, kv2[0].transpose(0, 1), kv2[1].transpose(0, 1))
        assert torch.equal(got[:at], want[:at]), bad


# ----------------------------------------------------------------------------
# together


def serve(rng, x, dtype, heads, kvh, d, page, capacity, seqs):
    """A cache and an object that runs steps of appends and attention over it."""
    pages = -(-capacity // page)
    k, v = page_tensors(kvh, pages * seqs, page, d, dtype)
    table = gpu(rng.permutation(pages * seqs).reshape(seqs, pages))
    return k, v, table


@pytest.mark.parametrize("x,dtype", KINDS)
def test_prompt_then_chunk_then_chains_then_tokens(x, dtype):
    """A run as a server makes it: prompts appended and attended whole (also from the pages), a chunk
    more, chains of drafts, tokens; each against float64 over what the pages hold."""
    rng = np.random.default_rng(21)
    heads, kvh, d, page, seqs = 8, 2, 64, 16, 3
    form = dict(rotary_dim=d)
    k, v, table = serve(rng, x, dtype, heads, kvh, d, page, 200, seqs)
    tab = table.cpu().numpy()
    length = np.zeros(seqs, int)
    for rows in ([40, 7, 65], [33, 1, 0], [5, 6, 2], [1, 1, 1]):
        n, starts = sum(rows), starts_of(rows)
        length = length + rows
        qkv = torch.tensor(rng.standard_normal((n, (heads + 2 * kvh) * d)), dtype=TYPES[x], device="cuda")
        batch = binding.batch(table, gpu(length), gpu(starts), max(rows), int(max(length)))
        q = binding.paged_append(binding.rope(**form), qkv, k, v, batch, heads)
        got = f64(binding.paged_attention(q, k, v, batch))
        places = P.row_places(starts, length, n, max(rows))
        k64, v64 = f64(k), f64(v)

        def seen(t):
            def of(r, h):
                s, p = places[r]
                return np.array([t[tab[s, j // page], h // (heads // kvh), j % page] for j in range(p + 1)])
            return of

        want, size, spread = P.attention(f64(q), seen(k64), seen(v64), lambda r: True, 1 / math.sqrt(d))
        tol = P.attention_tol(x, d, max(length), size, np.nanmax(np.abs(v64)), want, spread)
        assert (np.abs(got - want) <= tol).all()
        if rows[0] == 40:
            # the same prompts from packed keys and values
            at = [(tab[s, p // page], p % page) for s, p in places]
            pk, pv = (torch.stack([t[b, :, o] for b, o in at]).transpose(0, 1) for t in (k, v))
            again = f64(binding.prompt_attention(q, pk, pv, gpu(starts)))
            assert (np.abs(again - want) <= tol).all()


@pytest.mark.parametrize("x,dtype", KINDS)
def test_captured_steps_follow_the_lengths(x, dtype):
    """One step in a graph, replayed while lengths and rows change in device memory, with eager work between."""
    rng = np.random.default_rng(31)
    heads, kvh, d, page, seqs = 4, 2, 64, 16, 3
    k, v, table = serve(rng, x, dtype, heads, kvh, d, page, 2100, seqs)
    k.normal_(), v.normal_()
    form = binding.rope(rotary_dim=d)
    lengths = gpu([5, 900, 33])
    batch = binding.batch(table, lengths, None, 2)
    qkv = torch.zeros(2 * seqs, (heads + 2 * kvh) * d, dtype=TYPES[x], device="cuda")
    q, out = (torch.zeros(2 * seqs, heads, d, dtype=TYPES[x], device="cuda") for _ in "qo")
    ws = torch.zeros(max(16, binding.paged_attention_workspace(k, v, batch, heads, 2 * seqs, x == "bf16")), dtype=torch.uint8, device="cuda")

    def step():
        binding.paged_append(form, qkv, k, v, batch, heads, q_out=q)
        binding.paged_attention(q, k, v, batch, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, now in enumerate(([7, 902, 35], [2, 2000, 0], [64, 1, 1025], [7, 902, 35])):
        lengths.copy_(gpu(now))
        qkv.copy_(torch.tensor(rng.standard_normal(qkv.shape), dtype=TYPES[x], device="cuda"))
        k0, v0 = k.clone(), v.clone()
        graph.replay()
        torch.cuda.synchronize()
        replayed, rk, rv = out.clone(), k.clone(), v.clone()
        k.copy_(k0), v.copy_(v0)
        out.fill_(9.0)
        step()
        assert torch.equal(replayed, out) and torch.equal(rk, k) and torch.equal(rv, v), i


@pytest.mark.parametrize("x,dtype", KINDS)
def test_two_streams_at_once(x, dtype):
    rng = np.random.default_rng(41)
    c = Cache(rng, [3000, 40, 700], 2, 32, 128, dtype)
    batch = binding.batch(gpu(c.table), gpu([3000, 40, 700]), None, 2)
    qs = [torch.tensor(rng.standard_normal((6, 8, 128)), dtype=TYPES[x], device="cuda") for _ in range(2)]
    want = [binding.paged_attention(q, c.k, c.v, batch).clone() for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (q, st) in enumerate(zip(qs, streams)):
            with torch.cuda.stream(st):
                got[i].append(binding.paged_attention(q, c.k, c.v, batch))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_a_batch_does_not_change_its_neighbours_result():
    """A sequence alone, and among others, under the same bounds."""
    rng = np.random.default_rng(51)
    c = Cache(rng, [300, 40, 77], 2, 16, 64, "bf16")
    q = torch.tensor(rng.standard_normal((3, 8, 64)), dtype=torch.float32, device="cuda")
    every = binding.paged_attention(q, c.k, c.v, binding.batch(gpu(c.table), gpu([300, 40, 77]), None, 1, 304))
    again = binding.paged_attention(q, c.k, c.v, binding.batch(gpu(c.table[[0, 2, 1]]), gpu([300, 0, 40]), None, 1, 304))
    assert torch.equal(every[0], again[0])


# ----------------------------------------------------------------------------
# tiles of 128 rows and streams: blocks in the middle of long contexts


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_paged_chunks_of_many_rows(x, d, page):
    """Several tiles a sequence behind cached positions, ragged ends."""
    check_paged([150, 1, 67], [700, 333, 67 + 590], 4, 2, d, x, "bf16", page)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_paged_bad_pages_inside_long_contexts(x, page):
    """Pages missing in the middle and at the ends: of blocks that would be whole."""
    def spoil(c):
        for p in (0, 3, 5, 8):
            if p < c.table.shape[1] - 2:
                c.table[0, p] = (-1, c.n_pages, -2**31, 2**31 - 1)[p % 4]
        c.table[1, 2] = c.n_pages

    check_paged([140, 20, 1], [900, 620, 640], 4, 2, 64, x, "bf16", page, spoil=spoil)
    check_paged([20, 20, 1], [900, 620, 640], 4, 2, 128, x, "bf16", page, spoil=spoil)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 20, 150])
@pytest.mark.parametrize("at", [5, 200, 431])
def test_paged_infinities_inside_long_contexts(x, rows, at):
    """A value in a block that every row sees whole: infinite or NaN in its column for all of them, and nowhere else."""
    rng = np.random.default_rng(77)
    c = Cache(rng, [rows + 450], 1, 32, 64, "bf16")
    q = torch.tensor(rng.standard_normal((rows, 2, 64)), dtype=TYPES[x], device="cuda")
    batch = binding.batch(gpu(c.table), gpu([rows + 450]), None, rows)
    want = binding.paged_attention(q, c.k, c.v, batch).clone()
    c.v[int(c.table[0, at // 32]), :, at % 32, 9] = float("-inf")
    got = binding.paged_attention(q, c.k, c.v, batch)
    rest = [e for e in range(64) if e != 9]
    assert torch.equal(got[..., rest], want[..., rest]) and not got[..., 9].isfinite().any()


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_prompt_steps_at_every_end(x, d):
    """Tiles whose last block ends within the call's rows, and at them."""
    for rows in ([161], [130, 31], [30, 192], [97, 95, 1]):
        check_prompt(rows, 4, 1, d, x, "bf16")
    check_prompt([400], 1, 1, d, x, "bf16", order="heads")


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_prompt_large_enough_for_wide_tiles(x):
    """More than 450 tiles of 128 rows, so that they are not cut to 64."""
    rng = np.random.default_rng(6)
    rows, heads, kvh, d = [370, 1, 130, 64, 300, 33], 64, 32, 64
    starts, n = starts_of(rows), sum(rows)
    kv = torch.tensor(rng.standard_normal((2, n, kvh, d)), dtype=torch.bfloat16, device="cuda")
    q = torch.tensor(rng.standard_normal((n, heads, d)), dtype=TYPES[x], device="cuda")
    got = binding.prompt_attention(q, kv[0].transpose(0, 1), kv[1].transpose(0, 1), gpu(starts))
    q64, k64, v64 = (f64(t) for t in (q, kv[0], kv[1]))
    for s, m in enumerate(rows):
        for h in range(0, heads, 7):
            a = slice(starts[s], starts[s] + m)
            kk, vv, qq = k64[a, h // 2], v64[a, h // 2], q64[a, h]
            z = np.where(np.tril(np.ones((m, m), bool)), qq @ kk.T / math.sqrt(d), -np.inf)
            p = np.exp(z - z.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            want, spread = p @ vv, p @ np.abs(vv)
            size = float((np.abs(qq) @ np.abs(kk).T).max() / math.sqrt(d))
            tol = P.attention_tol(x, d, m, size, np.abs(vv).max(), want, spread)
            assert (np.abs(f64(got[a, h]) - want) <= tol).all(), (s, h)


@pytest.mark.parametrize("x,dtype", KINDS)
@pytest.mark.parametrize("heads,kvh,rows", [(4, 1, 1), (8, 1, 4), (16, 2, 8), (16, 1, 8)])
def test_streams_of_uneven_sequences(x, dtype, heads, kvh, rows):
    """Chunks that hold several sequences, parts of one, and none: empty ones between, one much longer than the rest."""
    rng = np.random.default_rng(14)
    lengths = [0, 40, 3000, 0, 1, 130, 2047, 0, 64, 700, 129, 0]
    m = [int(t) for t in rng.integers(0, rows + 1, len(lengths))]
    m[2], m[5] = rows, 0
    check_paged(m, lengths, heads, kvh, 32, x, dtype, 64)


@pytest.mark.parametrize("n_seqs", [63, 64, 65, 257, 1024, 1025])
def test_streams_of_many_sequences(n_seqs):
    """As many as a work-group adds up the spans of, and more."""
    rng = np.random.default_rng(n_seqs)
    lengths = [int(t) for t in rng.integers(0, 40, n_seqs)]
    lengths[n_seqs // 2] = 1500
    check_paged([1] * n_seqs, lengths, 2, 1, 16, "f32", "bf16", 16)


def test_streams_are_the_same_in_any_order():
    """The whole result does not follow from where chunks are cut, but for the order of float32 sums."""
    rng = np.random.default_rng(9)
    lengths = [2500, 10, 900, 1700]
    c = Cache(rng, lengths, 2, 16, 64, "bf16")
    q = torch.tensor(rng.standard_normal((4, 8, 64)), dtype=torch.float32, device="cuda")
    one = binding.paged_attention(q, c.k, c.v, binding.batch(gpu(c.table), gpu(lengths)))
    back = binding.paged_attention(q.flip(0), c.k, c.v, binding.batch(gpu(c.table[::-1].copy()), gpu(lengths[::-1]))).flip(0)
    assert (one - back).abs().max() <= 2.0 ** -20


# ----------------------------------------------------------------------------
# many short sequences: a wave each


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("rows,heads", [(1, 86), (3, 129), (18, 43)])
def test_many_short_sequences(x, d, rows, heads):
    """More than 512 work-groups of at most 32 rows, contexts of zero to several blocks, pages that are not there."""
    def spoil(c):
        c.table[0, 0] = -1
        c.table[4, 1], c.table[5, 2] = c.n_pages, -2**31

    lengths = [100, rows, 33, 0, 64, 250, 31, 32, 20, 129, 16, 65]
    m = [min(rows, n) for n in lengths]
    m[8] = 0
    check_paged(m, lengths, heads, 43, d, x, "bf16", 16, spoil=spoil, gap=1)
    check_paged(m, lengths, heads, 43, d, x, "bf16", 64, order="rows")


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [2, 20])
def test_many_short_sequences_and_values_that_are_infinite(x, rows):
    """What a row sees arrives in its column; what it does not, changes no bit of it."""
    rng = np.random.default_rng(78)
    lengths, kvh = [40 + 5 * s for s in range(40)], 16
    c = Cache(rng, lengths, kvh, 16, 32, "bf16")
    q = torch.tensor(rng.standard_normal((40 * rows, kvh, 32)), dtype=TYPES[x], device="cuda")
    batch = binding.batch(gpu(c.table), gpu(lengths), None, rows, max(lengths))
    want = binding.paged_attention(q, c.k, c.v, batch).clone()
    s, at = 11, lengths[11] - 1  # of its rows only the last sees it
    c.v[int(c.table[s, at // 16]), :, at % 16, 9] = float("inf")
    got = binding.paged_attention(q, c.k, c.v, batch)
    last = (s + 1) * rows - 1
    others = [r for r in range(40 * rows) if r != last]
    rest = [e for e in range(32) if e != 9]
    assert torch.equal(got[others], want[others]) and torch.equal(got[last][:, rest], want[last][:, rest])
    assert not got[last, :, 9].isfinite().any()


# ----------------------------------------------------------------------------
# prompts of many tiles a sequence


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("rows,heads,kvh", [([150, 129, 161, 1, 200], 120, 3), ([577], 128, 16), ([300, 90, 511], 128, 16),
                                            ([40] * 12, 64, 64)])
def test_prompts_of_many_tiles(x, d, rows, heads, kvh):
    """More than 450 tiles of 128 rows, of sequences of many tiles and of one each."""
    rng = np.random.default_rng(60 + d)
    starts, n, G = starts_of(rows), sum(rows), heads // kvh
    kv = torch.tensor(rng.standard_normal((2, n + 3, kvh, d)), dtype=torch.bfloat16, device="cuda")
    kv[:, n:] = float("nan")
    q = torch.tensor(rng.standard_normal((n, heads, d)), dtype=TYPES[x], device="cuda")
    got = binding.prompt_attention(q, kv[0].transpose(0, 1), kv[1].transpose(0, 1), gpu(starts))
    q64, k64, v64 = (f64(t) for t in (q, kv[0], kv[1]))
    for s, m in enumerate(rows):
        for h in range(s % 3, heads, 11):
            a = slice(starts[s], starts[s] + m)
            kk, vv, qq = k64[a, h // G], v64[a, h // G], q64[a, h]
            z = np.where(np.tril(np.ones((m, m), bool)), qq @ kk.T / math.sqrt(d), -np.inf)
            p = np.exp(z - z.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            want, spread = p @ vv, p @ np.abs(vv)
            size = float((np.abs(qq) @ np.abs(kk).T).max() / math.sqrt(d))
            tol = P.attention_tol(x, d, m, size, np.abs(vv).max(), want, spread)
            assert (np.abs(f64(got[a, h]) - want) <= tol).all(), (s, h)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_paged_chunks_of_short_and_long_contexts(x, d, page):
    """Tiles of 128 rows over at most 512 positions and over more."""
    check_paged([150, 0, 67, 129], [500, 333, 67, 129], 4, 2, d, x, "bf16", page, max_length=512)
    check_paged([150, 0, 67, 129], [500, 333, 67, 129], 4, 2, d, x, "bf16", page, max_length=513, max_rows=151, gap=2)
