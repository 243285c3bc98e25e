"""Host side of the operators of batches: where rows stand whatever the arrays in
device memory hold, and every refusal that is made before anything reaches the
GPU (no GPU is needed)."""

import ctypes

import pytest

from paper_2309_08168_amd import binding

BAD, FULL = binding.SD_ERR_INVALID_ARG, binding.SD_ERR_CAPACITY
P = 1 << 20  # an aligned address that nothing reads


def pages(**change):
    kv = dict(k=P, v=P, page_stride=2 * 16 * 128, head_stride=16 * 128, row_stride=128, n_kv_heads=2, n_pages=10, page_size=16,
              head_dim=128, dtype=binding.SD_BF16)
    kv.update(change)
    return binding.sd_kv_pages(**kv)


def batch(**change):
    b = dict(table=P, lengths=P, starts=P, ld_table=5, n_seqs=3, table_pages=5, max_rows=2, max_length=80)
    b.update(change)
    return binding.sd_batch(**b)


def append_call(kv=None, b=None, form=None, **change):
    a = dict(qkv=P, ld_qkv=1024, x=0, n=6, n_heads=4, positions=P, wq=None, wk=None, eps=1e-6, q=P, ld_q=512)
    a.update(change)
    form = binding.rope() if form is None else form
    return binding.load().sd_paged_append(form, a["qkv"], a["ld_qkv"], a["x"], a["n"], a["n_heads"], a["positions"], a["wq"],
                                          a["wk"], a["eps"], a["q"], a["ld_q"], kv or pages(), b or batch(), None)


def paged_call(kv=None, b=None, **change):
    a = dict(q=P, ld_q=512, x=0, n_heads=4, n=6, scale=0.0, out=P, ld_out=512, ws=P, nbytes=1 << 40)
    a.update(change)
    return binding.load().sd_paged_attention(kv or pages(), b or batch(), a["q"], a["ld_q"], a["x"], a["n_heads"], a["n"],
                                             a["scale"], a["out"], a["ld_out"], a["ws"], a["nbytes"], None)


def prompt_call(**change):
    a = dict(starts=P, n_seqs=3, q=P, ld_q=512, x=0, n_heads=4, n=6, scale=0.0, out=P, ld_out=512)
    a.update(change)
    kv = dict(k=P, v=P, head_stride=128, row_stride=256, n_kv_heads=2, capacity=64, head_dim=128, dtype=binding.SD_BF16)
    kv.update({k: a.pop(k) for k in list(a) if k in kv})
    return binding.load().sd_prompt_attention(binding.sd_kv_layer(**kv), a["starts"], a["n_seqs"], a["q"], a["ld_q"], a["x"],
                                              a["n_heads"], a["n"], a["scale"], a["out"], a["ld_out"], None)


def workspace(kv=None, b=None, x=0, n_heads=4, n=6):
    return binding.load().sd_paged_attention_workspace(kv or pages(), b or batch(), x, n_heads, n)


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(dtype=2), dict(dtype=-1), dict(head_dim=96),
             dict(head_dim=8), dict(head_dim=256), dict(n_kv_heads=0), dict(n_kv_heads=4097), dict(n_pages=0), dict(page_size=8),
             dict(page_size=24), dict(page_size=1 << 17), dict(page_size=0), dict(row_stride=64), dict(row_stride=132),
             dict(row_stride=-128), dict(head_stride=-128), dict(head_stride=0), dict(head_stride=12), dict(page_stride=0),
             dict(page_stride=12), dict(page_stride=-4096), dict(head_stride=15 * 128), dict(page_stride=31 * 128),
             dict(row_stride=256), dict(page_stride=(1 << 40) + 8), dict(head_stride=1 << 41),
             dict(page_stride=1 << 40, n_pages=2**31 - 1, n_kv_heads=1, head_stride=0, dtype=0) | dict(row_stride=127)]


@pytest.mark.parametrize("change", BAD_PAGES, ids=str)
def test_bad_pages(change):
    kv = pages(**change)
    assert append_call(kv) == BAD and paged_call(kv) == BAD and workspace(kv) == 0


@pytest.mark.parametrize("change", [
    dict(), dict(page_stride=256, row_stride=2560, head_stride=128), dict(page_stride=2048, head_stride=20480),
    dict(n_kv_heads=1, head_stride=0), dict(n_pages=1, page_stride=0), dict(row_stride=144, head_stride=16 * 144, page_stride=1 << 20)],
    ids=str)
def test_orders_of_pages_are_taken(change):
    """(refused only further on: without their queries)"""
    kv = pages(**change)
    heads = 4 // (2 // kv.n_kv_heads)
    assert paged_call(kv, q=None, n_heads=heads) == BAD
    assert b"q and out" in binding.load().sd_last_error()


BAD_BATCHES = [dict(n_seqs=0), dict(n_seqs=65537), dict(table_pages=0), dict(ld_table=4), dict(ld_table=-5),
               dict(table_pages=(1 << 26) + 1, ld_table=1 << 27), dict(max_rows=0), dict(max_rows=-1), dict(max_length=-1),
               dict(max_length=81), dict(starts=None, max_rows=3), dict(starts=None, n_seqs=2)]
BAD_ADDRESSES = [dict(table=None), dict(lengths=None), dict(table=P + 2), dict(lengths=P + 1), dict(starts=P + 2)]


@pytest.mark.parametrize("change", BAD_BATCHES, ids=str)
def test_bad_batches(change):
    b = batch(**change)
    assert append_call(b=b) == BAD and paged_call(b=b) == BAD and workspace(b=b) == 0


@pytest.mark.parametrize("change", BAD_ADDRESSES, ids=str)
def test_bad_addresses_of_batches(change):
    b = batch(**change)
    assert append_call(b=b) == BAD and paged_call(b=b) == BAD


def test_null_structures():
    lib = binding.load()
    assert lib.sd_paged_append(None, P, 1024, 0, 6, 4, None, None, None, 0.0, P, 512, pages(), batch(), None) == BAD
    assert lib.sd_paged_append(binding.rope(), P, 1024, 0, 6, 4, None, None, None, 0.0, P, 512, None, batch(), None) == BAD
    assert lib.sd_paged_append(binding.rope(), P, 1024, 0, 6, 4, None, None, None, 0.0, P, 512, pages(), None, None) == BAD
    assert lib.sd_paged_attention(None, batch(), P, 512, 0, 4, 6, 0.0, P, 512, P, 1 << 30, None) == BAD
    assert lib.sd_paged_attention(pages(), None, P, 512, 0, 4, 6, 0.0, P, 512, P, 1 << 30, None) == BAD
    assert lib.sd_paged_attention_workspace(None, batch(), 0, 4, 6) == 0
    assert lib.sd_prompt_attention(None, P, 3, P, 512, 0, 4, 6, 0.0, P, 512, None) == BAD


@pytest.mark.parametrize("change", [
    dict(qkv=None), dict(qkv=P + 4), dict(q=None), dict(q=P + 8), dict(positions=P + 2), dict(x=2), dict(x=-1), dict(n=0),
    dict(n=(1 << 20) + 1), dict(n_heads=3), dict(n_heads=0), dict(n_heads=4098, ld_qkv=1 << 22, ld_q=1 << 22),
    dict(ld_qkv=1020), dict(ld_qkv=1026), dict(x=1, ld_qkv=1028), dict(ld_q=508), dict(ld_q=514), dict(x=1, ld_q=516),
    dict(wq=P), dict(wk=P), dict(wq=P + 4, wk=P), dict(wq=P, wk=P + 8), dict(eps=-1e-6), dict(eps=float("nan")),
    dict(eps=float("inf"))], ids=str)
def test_append_refuses(change):
    assert append_call(**change) == BAD


@pytest.mark.parametrize("form", [dict(rotary_dim=0), dict(rotary_dim=130), dict(base=float("nan")), dict(scaling="linear", factor=0.5)],
                         ids=str)
def test_append_refuses_rotary_forms(form):
    assert append_call(form=binding.rope(**form)) == BAD


ROWS = [dict(q=None), dict(q=P + 4), dict(out=None), dict(out=P + 8), dict(x=2), dict(n=0), dict(n=(1 << 20) + 1), dict(n_heads=3),
        dict(n_heads=0), dict(n_heads=4098, ld_q=1 << 22, ld_out=1 << 22), dict(ld_q=508), dict(ld_q=514), dict(x=1, ld_q=516),
        dict(ld_out=508), dict(ld_out=514), dict(x=1, ld_out=516), dict(scale=float("nan")), dict(scale=float("inf")),
        dict(scale=3e38), dict(n=1 << 20, n_heads=128, ld_q=1 << 20, ld_out=1 << 20)]


@pytest.mark.parametrize("change", ROWS, ids=str)
def test_attention_refuses(change):
    assert paged_call(b=batch(max_rows=1 << 20), **change) == BAD
    assert prompt_call(**change) == BAD


@pytest.mark.parametrize("change,status", [
    (dict(starts=P + 2), BAD), (dict(starts=None), BAD), (dict(n_seqs=0), BAD), (dict(n_seqs=65537), BAD), (dict(n=65), FULL),
    (dict(k=P + 8), BAD), (dict(head_dim=96), BAD), (dict(row_stride=128), BAD), (dict(dtype=3), BAD)], ids=str)
def test_prompt_refuses(change, status):
    assert prompt_call(**change) == status


def test_too_many_sequences_times_heads_are_refused():
    kv = pages(n_kv_heads=128, head_stride=16 * 128, page_stride=1 << 20)
    assert paged_call(kv, batch(n_seqs=65536), n_heads=128, ld_q=1 << 20, ld_out=1 << 20) == BAD
    assert workspace(kv, batch(n_seqs=65536), n_heads=128) == 0


def test_joins_stay_within_a_launch_and_a_workspace():
    """A launch has at most 2^32 threads, and the join 256 a row and head: no parts
    for more rows than that, also where most rows are of no sequence."""
    kv = pages(n_kv_heads=128, page_stride=128 * 16 * 128)
    chains = batch(n_seqs=1024, max_rows=128, max_length=0, table_pages=320, ld_table=320)
    assert workspace(kv, chains, n_heads=128, n=131072) == 0
    kv = pages(n_kv_heads=64, page_stride=64 * 16 * 128)
    assert workspace(kv, chains, n_heads=64, n=131072) > 0  # 2^23 of them
    one = batch(n_seqs=1, max_length=0, table_pages=4000, ld_table=4000)
    for n, shares in ((6, None), (1 << 18, 4), (1 << 20, 1)):
        need = workspace(pages(dtype=binding.SD_F32), one, n_heads=4, n=n)
        assert need <= (1 << 22) * (128 * 4 + 8)
        if shares:
            assert need == (0 if shares == 1 else shares * n * 4 * (128 * 4 + 8))


def test_workspace_is_asked_for():
    b = batch(n_seqs=1, table_pages=1000, ld_table=1000, max_length=16000, max_rows=1)
    for x in (0, 1):
        need = workspace(b=b, x=x, n=1)
        assert need > 0
        assert paged_call(b=b, x=x, n=1, nbytes=need - 1) == BAD
        assert paged_call(b=b, x=x, n=1, ws=None, nbytes=0) == BAD
        assert paged_call(b=b, x=x, n=1, ws=P + 8, nbytes=need) == BAD


@pytest.mark.parametrize("start,end,length,n,most,want", [
    (0, 1, 1, 1, 1, (0, 1, 0)), (3, 8, 20, 10, 9, (3, 5, 15)), (3, 8, 20, 10, 2, (3, 2, 15)), (3, 8, 2, 10, 9, (3, 5, -3)),
    (3, 3, 7, 10, 9, (3, 0, 7)), (8, 3, 7, 10, 9, (8, 0, 7)), (-5, 3, 7, 10, 9, (0, 3, 4)), (8, 2**31 - 1, 7, 10, 9, (8, 2, 5)),
    (2**31 - 1, -2**31, 7, 10, 9, (10, 0, 7)), (-2**31, 2**31 - 1, 2**31 - 1, 10, 9, (0, 9, 2**30 - 10)),
    (0, 4, -2**31, 10, 9, (0, 4, -4)), (0, 4, -1, 10, 9, (0, 4, -4))])
def test_rows_stay_within_the_call(start, end, length, n, most, want):
    out = [ctypes.c_int32() for _ in range(3)]
    binding.load().sdk_seq_rows(start, end, length, n, most, *(ctypes.byref(x) for x in out))
    assert tuple(x.value for x in out) == want


def test_positions_seen():
    seen = binding.load().sdk_seen_from
    assert [seen(p, 5) for p in (-2**31, -1, 0, 3, 4, 5, 2**31 - 1)] == [0, 0, 1, 4, 5, 5, 5]


def test_tensors_on_the_cpu_are_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(binding.SDError, match="GPU"):
        binding.batch(torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    k = torch.zeros(16, 2, 64).transpose(0, 1)
    with pytest.raises(binding.SDError, match="GPU"):
        binding.prompt_attention(torch.zeros(16, 4, 64), k, k)


def test_tensor_shapes_types_and_strides_are_refused():
    torch = pytest.importorskip("torch")
    i32 = torch.int32
    table, lengths, starts = torch.zeros(3, 4, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(4, dtype=i32)
    k, layer, q = torch.zeros(5, 2, 16, 64), torch.zeros(2, 16, 64), torch.zeros(6, 4, 64)
    for bad in (lambda: binding.batch(table.long(), lengths), lambda: binding.batch(table[0], lengths),
                lambda: binding.batch(table.t(), lengths), lambda: binding.batch(table, lengths[:2]),
                lambda: binding.batch(table, lengths.float()), lambda: binding.batch(table, lengths, starts[:3]),
                lambda: binding.batch(table, lengths, max_rows=1 << 32), lambda: binding.batch(table, lengths, max_length=1 << 32),
                lambda: binding.kv_pages(k, k[:, :1]), lambda: binding.kv_pages(k, k.double()),
                lambda: binding.kv_pages(k.half(), k.half()), lambda: binding.kv_pages(k[0], k[0]),
                lambda: binding.kv_pages(k[..., ::2], k[..., ::2]), lambda: binding.kv_pages(k, k.transpose(1, 2).contiguous().transpose(1, 2)),
                lambda: binding.paged_attention(q.half(), k, k, None), lambda: binding.paged_attention(q[0], k, k, None),
                lambda: binding.paged_attention(q[..., :32], k, k, None), lambda: binding.paged_attention(q.transpose(0, 1), k, k, None),
                lambda: binding.paged_append(binding.rope(rotary_dim=64), torch.zeros(6, 7 * 64), k, k, None, 4),
                lambda: binding.paged_append(binding.rope(rotary_dim=64), torch.zeros(6 * 8 * 64), k, k, None, 4),
                lambda: binding.paged_append(binding.rope(rotary_dim=64), torch.zeros(6, 8 * 64).half(), k, k, None, 4),
                lambda: binding.prompt_attention(q.half(), layer, layer), lambda: binding.prompt_attention(q[0], layer, layer),
                lambda: binding.prompt_attention(q, layer, layer, starts.long()),
                lambda: binding.prompt_attention(q, layer, layer[:, :8])):
        with pytest.raises(binding.SDError) as e:
            bad()
        assert e.value.status == BAD


def test_sizes_past_32_bits_are_refused_and_not_cut():
    """(a meta tensor has a shape and no memory)"""
    torch = pytest.importorskip("torch")
    far, i32 = 2**32, torch.int32

    def meta(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    k, layer = meta(5, 2, 16, 64), meta(2, 64, 64)
    for bad in (lambda: binding.kv_pages(meta(far + 5, 2, 16, 64), meta(far + 5, 2, 16, 64)),
                lambda: binding.kv_pages(meta(5, far + 2, 16, 64), meta(5, far + 2, 16, 64)),
                lambda: binding.kv_pages(meta(5, 2, far + 16, 64), meta(5, 2, far + 16, 64)),
                lambda: binding.batch(meta(far + 3, 4, dtype=i32), meta(far + 3, dtype=i32)),
                lambda: binding.batch(meta(3, far + 4, dtype=i32), meta(3, dtype=i32)),
                lambda: binding.paged_attention(meta(far + 6, 4, 64), k, k, None),
                lambda: binding.paged_attention(meta(6, far + 4, 64), k, k, None),
                lambda: binding.paged_append(binding.rope(rotary_dim=64), meta(far + 6, 8 * 64), k, k, None, 4),
                lambda: binding.paged_append(binding.rope(rotary_dim=64), meta(6, (far + 8) * 64), k, k, None, far + 4),
                lambda: binding.paged_attention_workspace(k, k, None, far + 4, 6),
                lambda: binding.paged_attention_workspace(k, k, None, 4, far + 6),
                lambda: binding.prompt_attention(meta(far + 6, 4, 64), layer, layer),
                lambda: binding.prompt_attention(meta(6, 4, 64), meta(2, far + 64, 64), meta(2, far + 64, 64))):
        with pytest.raises(binding.SDError, match="32-bit") as e:
            bad()
        assert e.value.status == BAD
