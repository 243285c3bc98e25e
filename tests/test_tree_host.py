"""Host side of the tree operators: the layout of a tree, and every refusal
that is made before anything reaches the GPU (no GPU is needed)."""

import ctypes

import numpy as np
import pytest

from paper_2309_08168_amd import binding
from tests import tree_ref as T

BAD, FULL = binding.SD_ERR_INVALID_ARG, binding.SD_ERR_CAPACITY
P = 1 << 20  # an aligned address that nothing reads


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 200, 1024])
@pytest.mark.parametrize("back", [1, 5])
def test_layout(n, back):
    parents = T.random_parents(n, np.random.default_rng(n + back), back)
    depth, see = T.layout(parents)
    got_depth, got_mask = binding.tree_layout(parents)
    assert np.array_equal(got_depth, depth)
    assert np.array_equal(got_mask, T.pack(see))


@pytest.mark.parametrize("parents", [[], [0], [-2], [-1, -1], [-1, 1], [-1, 0, 2], [-1, 0, 5], [-1] + [0] * 1024])
def test_layout_refuses(parents):
    with pytest.raises(binding.SDError) as e:
        binding.tree_layout(parents)
    assert e.value.status == BAD


def layer(**change):
    kv = dict(k=P, v=P, head_stride=64 * 128, row_stride=128, n_kv_heads=2, capacity=64, head_dim=128,
              dtype=binding.SD_BF16)
    kv.update(change)
    return binding.sd_kv_layer(**kv)


BAD_LAYERS = [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(dtype=2), dict(head_dim=96),
              dict(head_dim=8), dict(head_dim=256), dict(n_kv_heads=0), dict(capacity=0), dict(capacity=(1 << 30) + 1, head_stride=1 << 39), dict(row_stride=64),
              dict(row_stride=132), dict(head_stride=-128), dict(head_stride=12), dict(head_stride=0), dict(head_stride=128),
              dict(head_stride=63 * 128), dict(head_stride=128, row_stride=128 + 64)]


def rope_call(form=None, kv=None, **change):
    a = dict(qkv=P, ld_qkv=1024, n=4, n_heads=4, positions=P, pos0=0, q=P, ld_q=512, slot=0)
    a.update(change)
    form = binding.rope() if form is None else form
    return binding.load().sd_rope_append(ctypes.byref(form), a["qkv"], a["ld_qkv"], a["n"], a["n_heads"],
                                         a["positions"], a["pos0"], a["q"], a["ld_q"],
                                         ctypes.byref(layer() if kv is None else kv), a["slot"], None)


def attn_call(kv=None, **change):
    a = dict(q=P, ld_q=512, n_heads=4, n=4, prefix=10, mask=P, scale=0.0, out=P, ld_out=512, ws=P, nbytes=1 << 40)
    a.update(change)
    return binding.load().sd_tree_attention(ctypes.byref(layer() if kv is None else kv), a["q"], a["ld_q"], a["n_heads"],
                                            a["n"], a["prefix"], a["mask"], a["scale"], a["out"], a["ld_out"], a["ws"],
                                            a["nbytes"], None)


@pytest.mark.parametrize("change", BAD_LAYERS, ids=str)
def test_bad_layers(change):
    assert rope_call(kv=layer(**change)) == BAD
    assert attn_call(kv=layer(**change)) == BAD
    assert binding.load().sd_tree_attention_workspace(ctypes.byref(layer(**change)), 4, 4, 10) == 0


@pytest.mark.parametrize("change,status", [
    (dict(qkv=None), BAD), (dict(qkv=P + 4), BAD), (dict(q=None), BAD), (dict(q=P + 8), BAD), (dict(positions=P + 2), BAD),
    (dict(n=0), BAD), (dict(n=(1 << 20) + 1), BAD), (dict(n_heads=3), BAD), (dict(n_heads=0), BAD), (dict(n_heads=4098, ld_qkv=1 << 22, ld_q=1 << 22), BAD), (dict(ld_qkv=1020), BAD),
    (dict(ld_qkv=1026), BAD), (dict(ld_q=508), BAD), (dict(ld_q=514), BAD), (dict(slot=-1), FULL), (dict(slot=61), FULL),
    (dict(n=65), FULL), (dict(positions=None, pos0=2**31 - 3), BAD)], ids=str)
def test_rope_append_refuses(change, status):
    assert rope_call(**change) == status


@pytest.mark.parametrize("form", [
    dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=130), dict(base=0.0), dict(base=float("nan")),
    dict(base=float("inf")), dict(scaling="linear", factor=0.5), dict(scaling="yarn", factor=float("inf")),
    dict(scaling="ntk", rotary_dim=2, factor=2.0), dict(scaling="yarn", factor=2.0, beta_fast=1.0),
    dict(scaling="yarn", factor=2.0, original_context=0), dict(gain=float("nan")),
    dict(scaling="yarn", factor=2.0, beta_slow=-1.0)], ids=str)
def test_rope_forms_refused(form):
    assert rope_call(form=binding.rope(**form)) == BAD


@pytest.mark.parametrize("form", [
    dict(scaling="ntk", factor=1e300, base=1e10), dict(scaling="ntk", factor=1e160, rotary_dim=4), dict(gain=1e39),
    dict(gain=-1e39), dict(base=9e-10), dict(base=5e-324)], ids=str)
def test_rope_forms_whose_numbers_overflow_are_refused(form):
    """(slot 61 is refused too, but only further on)"""
    assert rope_call(form=binding.rope(**form), slot=61) == BAD


@pytest.mark.parametrize("form", [
    dict(scaling="ntk", factor=1e150, rotary_dim=4), dict(gain=3e38), dict(base=1e-9), dict(base=1e308),
    dict(scaling="linear", factor=1e308), dict(scaling="yarn", factor=1e308)], ids=str)
def test_rope_forms_at_the_limits_are_taken(form):
    assert rope_call(form=binding.rope(**form), slot=61) == FULL


def test_position_major_layers_are_taken():
    """[capacity][n_kv_heads][head_dim]: refused only further on."""
    assert rope_call(kv=layer(head_stride=128, row_stride=256), slot=61) == FULL


def test_unknown_rope_kinds():
    for field in ("layout", "scaling"):
        for value in (-1, 4):
            form = binding.rope()
            setattr(form, field, value)
            assert rope_call(form=form) == BAD


@pytest.mark.parametrize("change,status", [
    (dict(q=None), BAD), (dict(q=P + 4), BAD), (dict(out=None), BAD), (dict(out=P + 4), BAD), (dict(mask=P + 4), BAD),
    (dict(n=0), BAD), (dict(n=1025), BAD), (dict(n_heads=3), BAD), (dict(n_heads=0), BAD), (dict(n_heads=4098), BAD),
    (dict(ld_q=508), BAD), (dict(ld_q=514), BAD), (dict(ld_out=508), BAD), (dict(ld_out=514), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(prefix=-1), FULL), (dict(prefix=61), FULL),
    (dict(n=65, prefix=0), FULL)], ids=str)
def test_attention_refuses(change, status):
    assert attn_call(**change) == status


def test_attention_workspace_refused():
    kv = layer(capacity=60000, head_stride=60000 * 128)
    need = binding.load().sd_tree_attention_workspace(ctypes.byref(kv), 4, 4, 50000)
    assert need > 0
    assert attn_call(kv=kv, prefix=50000, nbytes=need - 1) == BAD
    assert attn_call(kv=kv, prefix=50000, ws=None, nbytes=0) == BAD
    assert attn_call(kv=kv, prefix=50000, ws=P + 8, nbytes=need) == BAD


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(logits=P + 2), dict(tokens=None), dict(parents=None), dict(walk=None), dict(walk=P + 1),
    dict(n=0), dict(n=1025), dict(vocab=0), dict(ld=99), dict(ws=None), dict(ws=P + 4), dict(nbytes=8)], ids=str)
def test_accept_refuses(change):
    a = dict(logits=P, ld=100, vocab=100, tokens=P, parents=P, n=5, walk=P, ws=P, nbytes=1 << 20)
    a.update(change)
    assert binding.load().sd_tree_accept(a["logits"], a["ld"], a["vocab"], a["tokens"], a["parents"], a["n"], a["walk"],
                                         a["ws"], a["nbytes"], None) == BAD


@pytest.mark.parametrize("change,status", [
    (dict(kv=None), BAD), (dict(kv=P + 8), BAD), (dict(walk=None), BAD), (dict(planes=0), BAD), (dict(planes=1 << 25), BAD),
    (dict(row=0), BAD), (dict(row=24), BAD), (dict(row=1 << 17), BAD), (dict(stride=1000 * 256 - 16), BAD),
    (dict(stride=1000 * 256 + 8), BAD), (dict(n=0), BAD), (dict(n=1025, cap=4000), BAD), (dict(base=-1), FULL),
    (dict(base=996), FULL), (dict(cap=0), BAD)], ids=str)
def test_keep_refuses(change, status):
    a = dict(kv=P, planes=4, stride=1000 * 256, row=256, cap=1000, base=0, walk=P, n=5)
    a.update(change)
    assert binding.load().sd_kv_keep(a["kv"], a["planes"], a["stride"], a["row"], a["cap"], a["base"], a["walk"], a["n"],
                                     None) == status


def test_tensors_on_the_cpu_are_refused():
    torch = pytest.importorskip("torch")
    k = torch.zeros(2, 16, 64)
    with pytest.raises(binding.SDError):
        binding.tree_attention(torch.zeros(3, 4, 64), k, k.clone(), 0)
    with pytest.raises(binding.SDError):
        binding.tree_accept(torch.zeros(3, 10), torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(binding.SDError):
        binding.kv_keep(k, 0, torch.zeros(8, dtype=torch.int32))
    with pytest.raises(binding.SDError):
        binding.rope_append(binding.rope(rotary_dim=64), torch.zeros(3, 8 * 64), k, k.clone(), 0, 4)


def test_tensor_shapes_types_and_strides_are_refused():
    torch = pytest.importorskip("torch")
    k = torch.zeros(2, 16, 64)
    q = torch.zeros(3, 4, 64)
    for bad in (lambda: binding.kv_layer(k, k[:, :8]), lambda: binding.kv_layer(k, k.double()),
                lambda: binding.kv_layer(k.half(), k.half()), lambda: binding.kv_layer(k[:, :, ::2], k[:, :, ::2]),
                lambda: binding.tree_attention(q.half(), k, k, 0), lambda: binding.tree_attention(q[:, :, :32], k, k, 0),
                lambda: binding.tree_attention(q, k, k, 0, mask=torch.zeros(3, 2, dtype=torch.int64)),
                lambda: binding.tree_attention(q, k, k, 0, mask=torch.zeros(3, 1)),
                lambda: binding.tree_attention(q, k, k, 0, mask=torch.zeros(3, 1, dtype=torch.complex64)),
                lambda: binding.tree_attention(q, k, k, 1 << 32),
                lambda: binding.tree_attention(q[0], k, k, 0),
                lambda: binding.rope_append(binding.rope(rotary_dim=64), torch.zeros(3, 8 * 64), k, k, 1 << 32, 4),
                lambda: binding.rope_append(binding.rope(rotary_dim=64), torch.zeros(3, 8, 64), k, k, 0, 4),
                lambda: binding.kv_keep(k, 1 << 32, torch.zeros(8, dtype=torch.int32)),
                lambda: binding.kv_keep(k, 0, torch.zeros(9, dtype=torch.int32)),
                lambda: binding.tree_attention(q.transpose(0, 1), k, k, 0),
                lambda: binding.tree_accept(torch.zeros(3, 10), torch.zeros(3), torch.zeros(3)),
                lambda: binding.kv_keep(k.transpose(0, 1), 0, torch.zeros(8, dtype=torch.int32)),
                lambda: binding.kv_keep(k, 0, torch.zeros(8)),
                lambda: binding.rope_append(binding.rope(rotary_dim=64), torch.zeros(3, 7 * 64), k, k, 0, 4)):
        with pytest.raises(binding.SDError) as e:
            bad()
        assert e.value.status == BAD


def test_null_models_and_caches_are_refused():
    lib, out = binding.load(), ctypes.c_int32()
    assert lib.sd_forward_tree(None, P, P, 3, None, P, None) == BAD
    assert lib.sd_verify_tree(None, P, P, 3, P, P, ctypes.byref(out), ctypes.byref(out)) == BAD
    assert lib.sd_kv_cache_keep(None, P, 1) == BAD
    assert lib.sd_model_set_rope(None, None) == BAD
    assert b"model" in lib.sd_last_error()


LARGEST = 2**31 - 4097  # of the vocabularies


@pytest.mark.parametrize("n", [1, 2, 3, 600, 1024])
@pytest.mark.parametrize("vocab", [1, 2047, 2049, 32000, 2146435074, 2147475456, 2147475457, LARGEST])
def test_slices_of_a_row_cover_the_vocabulary(n, vocab):
    """Each id is in one slice, also where a slice would end past 2^31 - 1."""
    lib, first, end = binding.load(), ctypes.c_int32(), ctypes.c_int32()
    slices = lib.sdk_accept_slice(n, vocab, 0, ctypes.byref(first), ctypes.byref(end))
    assert 1 <= slices <= 2048 and lib.sd_tree_accept_workspace(n, vocab) == 8 * n * slices
    at = 0
    for s in range(slices):
        lib.sdk_accept_slice(n, vocab, s, ctypes.byref(first), ctypes.byref(end))
        assert first.value == at and at < end.value <= vocab
        at = end.value
    assert at == vocab


def test_the_walk_needs_no_workspace_for_a_vocabulary_that_it_refuses():
    for vocab in (0, -1, LARGEST + 1, 2**31 - 1):
        assert binding.load().sd_tree_accept_workspace(1, vocab) == 0
        assert binding.load().sd_tree_accept(P, 1 << 40, vocab, P, P, 1, P, P, 1 << 20, None) == BAD


def test_sizes_past_32_bits_are_refused_and_not_cut():
    """(a meta tensor has a shape and no memory)"""
    torch = pytest.importorskip("torch")
    far = 2**32

    def meta(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    k, long, many = meta(2, 64, 64), meta(2, far + 64, 64), meta(far + 2, 64, 64)
    i32, form = torch.int32, binding.rope(rotary_dim=64)
    for bad in (lambda: binding.kv_layer(long, long), lambda: binding.kv_layer(many, many),
                lambda: binding.tree_attention_workspace(long, long, 4, 4, 10),
                lambda: binding.tree_attention_workspace(k, k, far + 4, 4, 10),
                lambda: binding.tree_attention_workspace(k, k, 4, far + 4, 10),
                lambda: binding.tree_attention_workspace(k, k, 4, 4, far + 10),
                lambda: binding.tree_attention(meta(far + 3, 4, 64), k, k, 0),
                lambda: binding.tree_attention(meta(3, far + 4, 64), k, k, 0),
                lambda: binding.rope_append(form, meta(far + 3, 8 * 64), k, k, 0, 4),
                lambda: binding.rope_append(form, meta(3, (far + 8) * 64), k, k, 0, far + 4),
                lambda: binding.tree_accept(meta(3, far + 5), meta(3, dtype=i32), meta(3, dtype=i32)),
                lambda: binding.tree_accept(meta(far + 3, 5), meta(far + 3, dtype=i32), meta(far + 3, dtype=i32)),
                lambda: binding.tree_accept_workspace(far + 3, 5), lambda: binding.tree_accept_workspace(3, far + 5),
                lambda: binding.kv_keep(long, 0, meta(8, dtype=i32)),
                lambda: binding.kv_keep(meta(2, 16, far + 16), 0, meta(8, dtype=i32)),
                lambda: binding.kv_keep(k, 0, meta(2 * far + 8, dtype=i32)),
                lambda: binding.rope(rotary_dim=far + 64), lambda: binding.rope(original_context=far + 4096)):
        with pytest.raises(binding.SDError, match="32-bit") as e:
            bad()
        assert e.value.status == BAD


def f32_shares(rows, kvh, d, prefix):
    """Shares of the keys that a float32 layer's attention takes, by its workspace:
    an output, a maximum and a sum per share, row and head."""
    cap = prefix + rows
    kv = layer(head_stride=cap * d, row_stride=d, n_kv_heads=kvh, capacity=cap, head_dim=d, dtype=binding.SD_F32)
    nbytes = binding.load().sd_tree_attention_workspace(ctypes.byref(kv), kvh, rows, prefix)
    assert nbytes % (4 * rows * kvh * (d + 2)) == 0
    return nbytes // (4 * rows * kvh * (d + 2)) or 1


@pytest.mark.parametrize("rows,kvh,d,prefix,least,most", [
    # more tiles than half the CUs, long contexts: split, so that no CU idles over the whole of it
    (61, 34, 128, 4000, 3, 8), (64, 40, 128, 4000, 3, 8), (80, 32, 128, 4000, 3, 8), (112, 40, 128, 4000, 2, 8),
    (80, 32, 64, 4000, 3, 8), (80, 32, 32, 4000, 3, 12), (80, 32, 16, 4000, 3, 12), (80, 32, 16, 1400, 3, 12),
    # small heads: a long context is not short because its rows are
    (13, 2, 16, 1400, 6, 24), (13, 8, 16, 1400, 6, 24), (13, 8, 32, 1400, 6, 24),
    # tiles for every CU, or short contexts: whole
    (96, 40, 128, 4000, 1, 1), (64, 40, 128, 1000, 1, 1), (60, 40, 128, 300, 1, 1), (5, 4, 64, 30, 1, 1), (5, 40, 128, 100, 1, 1),
    # few tiles: one work-group per CU
    (4, 40, 128, 4000, 5, 6), (19, 32, 128, 1000, 4, 5)])
def test_float32_shares(rows, kvh, d, prefix, least, most):
    assert least <= f32_shares(rows, kvh, d, prefix) <= most


@pytest.mark.parametrize("scale", [3e38, -3e38, 2.4e38])
def test_attention_refuses_a_scale_that_overflows_in_log2(scale):
    assert attn_call(scale=scale) == BAD


def test_attention_takes_the_largest_scale():
    """(without its workspace: refused only further on, and by another message)"""
    kv = layer(capacity=60000, head_stride=60000 * 128)
    assert attn_call(kv=kv, prefix=50000, scale=2.3e38, ws=None, nbytes=0) == BAD
    assert b"workspace" in binding.load().sd_last_error()
