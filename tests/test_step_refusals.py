"""What the calls around a step refuse, and what they take as nothing to do: decided on the host before
anything is enqueued, so these run without a GPU; the pointers are numbers that nothing follows."""
import ctypes as C
import math

import pytest
import torch

from paper_2504_03648_b200 import binding as aibx
from test_paged_refusals import BAD_BATCH, BAD_CACHE, FAKE, batch, cache, lib, params  # noqa: F401 (lib is a fixture)


def at(x):
    return None if x is None else C.addressof(x)


# ------------------------------------------------------------------------------------------
# block tables


def tables(lib, R=2, **kw):  # noqa: F811
    d = dict(d_held=FAKE, d_new=FAKE + 64, d_free_ids=FAKE + 128, free_capacity=9, d_free_head=FAKE + 192,
             d_free_tail=FAKE + 200, d_free_head_out=FAKE + 208, d_block_table=FAKE + 256, d_blk_off=0, table_stride=4,
             d_match_ids=0, d_match_off=0, d_tok_off=FAKE + 512, d_kv_len=FAKE + 640, d_pos=FAKE + 700,
             d_slots=FAKE + 800, n_tokens=5, block_tokens=16, num_blocks=9)
    assert set(kw) <= set(d)
    d.update(kw)
    return lib.aibx_kv_tables(aibx._TABLES_BYTES.pack(*d.values()), R, None)


@pytest.mark.parametrize("kw", [
    dict(R=-1), dict(block_tokens=0), dict(block_tokens=-16), dict(table_stride=-1), dict(free_capacity=-1), dict(free_capacity=0),
    dict(n_tokens=-1), dict(d_held=0), dict(d_new=0), dict(d_free_ids=0), dict(d_free_head=0), dict(d_free_tail=0),
    dict(d_free_head_out=0), dict(d_block_table=0), dict(d_tok_off=0), dict(d_kv_len=0), dict(d_match_ids=FAKE + 900),
    dict(d_match_off=FAKE + 904), dict(d_held=FAKE + 2), dict(d_pos=FAKE + 701), dict(d_slots=FAKE + 804), dict(d_tok_off=FAKE + 516),
    dict(d_blk_off=FAKE + 4), dict(d_free_head=FAKE + 196), dict(d_kv_len=FAKE + 64), dict(d_pos=FAKE), dict(d_pos=FAKE + 64),
    dict(d_match_ids=FAKE + 256, d_match_off=FAKE + 904), dict(d_block_table=FAKE + 128), dict(d_free_head_out=FAKE + 200)])
def test_bad_tables(lib, kw):  # noqa: F811
    assert tables(lib, **kw) == aibx.ERR_INVALID


def test_tables_of_nothing(lib):  # noqa: F811
    assert lib.aibx_kv_tables(None, 2, None) == aibx.ERR_INVALID
    assert tables(lib, block_tokens=65537) == aibx.ERR_UNSUPPORTED
    assert tables(lib, R=0, d_held=0, d_tok_off=0, free_capacity=0) == aibx.OK


# ------------------------------------------------------------------------------------------
# trees


def masks(lib, parent=FAKE, off=FAKE + 64, kv=FAKE + 128, R=2, n=5, words=1, mask=FAKE + 256, pos=FAKE + 512):  # noqa: F811
    return lib.aibx_tree_masks(parent, off, kv, R, n, words, mask, pos, None)


@pytest.mark.parametrize("kw", [dict(parent=None), dict(off=None), dict(mask=None), dict(kv=None), dict(R=-1), dict(n=-1), dict(words=0),
                                dict(words=-2), dict(parent=FAKE + 2), dict(off=FAKE + 68), dict(mask=FAKE + 260), dict(pos=FAKE + 513),
                                dict(pos=FAKE), dict(pos=FAKE + 128)])
def test_bad_masks(lib, kw):  # noqa: F811
    assert masks(lib, **kw) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", [dict(mask=FAKE), dict(mask=FAKE + 64), dict(mask=FAKE + 128), dict(pos=FAKE + 64)])
def test_masks_in_the_place_of_inputs(lib, kw):  # noqa: F811
    assert masks(lib, **kw) == aibx.ERR_INVALID


def test_masks_of_nothing(lib):  # noqa: F811
    assert masks(lib, words=9) == aibx.ERR_UNSUPPORTED
    assert masks(lib, R=0, parent=None) == aibx.OK and masks(lib, n=0, mask=None) == aibx.OK


def test_tree_workspace(lib):  # noqa: F811
    def size(c, b, p):
        return lib.aibx_attn_tree_workspace_bytes(at(c), at(b), at(p))

    few = size(cache(), batch(max_new=1), params())
    assert 0 < few == size(cache(num_blocks=500, layout=2), batch(max_new=1, n_tokens=900, R=900), params())
    assert few < size(cache(), batch(max_new=20), params()) < size(cache(), batch(max_new=100), params())
    assert size(cache(), batch(max_new=0, R=7), params()) == size(cache(), batch(max_new=100), params())
    assert size(cache(), batch(), params(scale=0.0)) == 0
    assert tree(lib, cache(), batch(max_new=20), params(), size=size(cache(), batch(max_new=20), params()) - 1) == aibx.ERR_INVALID


def tree(lib, c, b, p, mask=FAKE + 8192, words=1, q=FAKE, out=FAKE + 4096, lse=None, ws=FAKE, size=1 << 40):  # noqa: F811
    return lib.aibx_attn_tree(at(c), at(b), at(p), mask, words, q, out, lse, ws, size, None)


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_tree_bad_cache(lib, kw):  # noqa: F811
    assert tree(lib, cache(**kw), batch(), params()) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", BAD_BATCH)
def test_tree_bad_batch(lib, kw):  # noqa: F811
    assert tree(lib, cache(), batch(**kw), params()) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", [dict(q_type=aibx.TYPE_FP32), dict(num_q_heads=0), dict(num_q_heads=6), dict(window=-1), dict(scale=0.0),
                                dict(scale=math.nan), dict(scale=3.4e38), dict(q_token_stride=1028), dict(out_head_stride=129)])
def test_tree_bad_params(lib, kw):  # noqa: F811
    assert tree(lib, cache(), batch(), params(**kw)) == aibx.ERR_INVALID


def test_tree_masks_shapes_and_pointers(lib):  # noqa: F811
    for kw in (dict(mask=None), dict(mask=FAKE + 4), dict(words=0), dict(words=-1), dict(q=None), dict(out=FAKE), dict(ws=None), dict(size=1000),
               dict(lse=FAKE + 2), dict(q=FAKE + 8)):
        assert tree(lib, cache(), batch(), params(), **kw) == aibx.ERR_INVALID, kw
    assert tree(lib, cache(), batch(), None) == aibx.ERR_INVALID
    assert tree(lib, cache(), batch(), params(), words=9) == aibx.ERR_UNSUPPORTED
    for kw in (dict(head_dim=96), dict(block_tokens=12), dict(num_blocks=0x80000000)):
        assert tree(lib, cache(**kw), batch(), params()) == aibx.ERR_UNSUPPORTED, kw
    assert tree(lib, cache(), batch(n_tokens=1 << 24), params()) == aibx.ERR_UNSUPPORTED
    for kw in (dict(R=0), dict(n_tokens=0)):
        assert tree(lib, cache(d_pool=None), batch(**kw), params(), mask=None, q=None, out=None, ws=None) == aibx.OK


# ------------------------------------------------------------------------------------------
# rotary positions


def rope_bytes(freq=FAKE, pos=FAKE + 64, dim=64, style=0, factor=1.0):
    return aibx._ROPE_BYTES.pack(freq, pos, dim, style, factor)


def rope(lib, n=5, heads=2, dim=128, x=FAKE, xs=(256, 128), y=FAKE + 4096, ys=(256, 128), type=aibx.TYPE_BF16, **kw):  # noqa: F811
    return lib.aibx_rope(rope_bytes(**kw), n, heads, dim, x, xs[0], xs[1], y, ys[0], ys[1], type, None)


BAD_ROPE = [dict(freq=0), dict(freq=FAKE + 4), dict(pos=FAKE + 2), dict(dim=0), dict(dim=-16), dict(dim=17), dict(dim=144), dict(style=2), dict(style=-1)]


@pytest.mark.parametrize("kw", BAD_ROPE + [dict(pos=0), dict(x=None), dict(y=None), dict(n=-1), dict(heads=-1), dict(xs=(-1, 128)),
                                           dict(ys=(256, -2)), dict(x=FAKE + 1), dict(type=aibx.TYPE_E4M3), dict(type=8),
                                           dict(y=FAKE, ys=(512, 128)), dict(y=FAKE, ys=(256, 64)), dict(x=FAKE + 2, type=aibx.TYPE_FP32)])
def test_bad_rope(lib, kw):  # noqa: F811
    kw = dict(kw)
    if "dim" in kw:
        rd = kw.pop("dim")
        assert lib.aibx_rope(rope_bytes(dim=rd), 5, 2, 128, FAKE, 256, 128, FAKE + 4096, 256, 128, 0, None) == aibx.ERR_INVALID
        return
    assert rope(lib, **kw) == aibx.ERR_INVALID


def test_rope_shapes(lib):  # noqa: F811
    assert lib.aibx_rope(None, 5, 2, 128, FAKE, 256, 128, FAKE + 4096, 256, 128, 0, None) == aibx.ERR_INVALID
    for rd, dim in ((20, 128), (64, 520), (64, 132)):
        assert lib.aibx_rope(rope_bytes(dim=rd), 5, 2, dim, FAKE, 2048, 1024, FAKE + 8, 2048, 1024, 0, None) == aibx.ERR_UNSUPPORTED
    assert rope(lib, heads=65537) == aibx.ERR_UNSUPPORTED
    assert rope(lib, n=0, x=None, y=None, pos=0, freq=0) == aibx.OK and rope(lib, heads=0, x=None) == aibx.OK


def rope_append(lib, c, b, heads=4, q=FAKE, q_out=FAKE + 4096, k=FAKE, v=FAKE, strides=(512, 128) * 4, type=aibx.TYPE_BF16, **kw):  # noqa: F811
    rows = aibx._ROPE_ROWS_BYTES.pack(q, q_out, k, v, *strides, heads, type)
    return lib.aibx_rope_append(at(c), at(b), rope_bytes(**kw), rows, None)


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_rope_append_bad_cache(lib, kw):  # noqa: F811
    assert rope_append(lib, cache(**kw), batch()) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", BAD_BATCH)
def test_rope_append_bad_batch(lib, kw):  # noqa: F811
    assert rope_append(lib, cache(), batch(**kw)) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", BAD_ROPE + [dict(heads=-1), dict(q=0), dict(q_out=0), dict(k=0), dict(v=0), dict(k=FAKE + 1), dict(type=aibx.TYPE_E4M3),
                                           dict(strides=(512, 128, 512, 128, -8, 128, 512, 128)), dict(strides=(512, 128, 512, 128, 512, 128, 512, -1)),
                                           dict(q_out=FAKE, strides=(512, 128, 640, 128) + (512, 128) * 2)])
def test_rope_append_bad_rows(lib, kw):  # noqa: F811
    assert rope_append(lib, cache(), batch(), **kw) == aibx.ERR_INVALID


def test_rope_append_shapes(lib):  # noqa: F811
    assert lib.aibx_rope_append(at(cache()), at(batch()), rope_bytes(), None, None) == aibx.ERR_INVALID
    assert lib.aibx_rope_append(at(cache()), at(batch()), None, aibx._ROPE_ROWS_BYTES.pack(*[FAKE] * 4, *(512, 128) * 4, 4, 0), None) == aibx.ERR_INVALID
    assert rope_append(lib, cache(head_dim=520), batch()) == aibx.ERR_UNSUPPORTED
    assert rope_append(lib, cache(), batch(), dim=24) == aibx.ERR_UNSUPPORTED
    assert rope_append(lib, cache(), batch(), heads=65537) == aibx.ERR_UNSUPPORTED
    assert rope_append(lib, cache(d_pool=None), batch(R=0), k=0, v=0, q=0) == aibx.OK


def test_structures_are_packed_as_c_lays_them_out():
    assert aibx._TABLES_BYTES.size == 17 * 8 + 2 * 4
    assert aibx._ROPE_ROWS_BYTES.size == 4 * 8 + 8 * 8 + 8 and aibx._ROPE_BYTES.size == 28


# ------------------------------------------------------------------------------------------
# frequencies


def test_frequencies():
    f, m = aibx.rope_frequencies(64)
    assert m == 1.0 and f.dtype == torch.float64
    for i in (0, 1, 17, 31):
        assert math.isclose(f[i], 10000.0 ** (-2 * i / 64), rel_tol=1e-15)
    g, m = aibx.rope_frequencies(64, scaling="linear", scale=4.0)
    assert m == 1.0 and torch.equal(g, f / 4)
    g, _ = aibx.rope_frequencies(64, scaling="base", scale=4.0)
    assert g[0] == f[0] and math.isclose(g[31], f[31] / 4, rel_tol=1e-14)
    g, m = aibx.rope_frequencies(128, 1e6, scaling="parts", scale=8.0, trained=4096)
    f, _ = aibx.rope_frequencies(128, 1e6)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32])
    assert torch.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert bool(mid.any()) and bool((g[mid] < f[mid]).all()) and bool((g[mid] > f[mid] / 8).all())
    assert math.isclose(m, 0.1 * math.log(8.0) + 1)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=64, scaling="other"), dict(rotary_dim=64, scaling="parts"),
                dict(rotary_dim=2, scaling="base"), dict(rotary_dim=64, base=0.0), dict(rotary_dim=64, scale=0.0)):
        with pytest.raises(ValueError):
            aibx.rope_frequencies(**bad)


def test_binding_refuses_tensors_of_the_wrong_kind():
    """Shapes, types and devices, before anything is called (all on the host here)."""
    i32, u64 = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 1, dtype=torch.int64).view(torch.uint64)
    with pytest.raises(ValueError):
        aibx._vector(i32, "x", torch.int64, 4, -1)
    with pytest.raises(ValueError):
        aibx._vector(i32, "x", torch.int32, 5, -1)
    with pytest.raises(ValueError):
        aibx._vector(torch.zeros(4, 2, dtype=torch.int32)[:, 0], "x", torch.int32, 4, -1)
    with pytest.raises(ValueError):
        aibx._vector(i32, "x", torch.int32, 4, 0)             # on another device
    assert aibx._vector(i32, "x", torch.int32, 4, -1) == i32.data_ptr()
    assert u64.dtype == torch.uint64
