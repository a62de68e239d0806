"""What the token-wise calls on a paged pool refuse, and what they take as nothing to do.  All of it is
decided on the host before anything is enqueued, so these run without a GPU: the pointers are
numbers that nothing follows."""
import ctypes as C
import math

import pytest

from paper_2504_03648_b200 import binding as aibx
from paper_2504_03648_b200 import build as aibx_build

FAKE = 0x10000


def cache(**kw):
    lay = dict(layout=0, num_layers=2, num_kv_heads=4, block_tokens=16, head_dim=128, elem_bytes=2, num_blocks=9)
    top = dict(d_pool=FAKE, d_scales=None, type=aibx.TYPE_BF16, inner=0, layer=1)
    for k, v in kw.items():
        (lay if k in lay else top)[k] = v
    l = aibx.KVLayout(*[lay[k] for k in ("layout", "num_layers", "num_kv_heads", "block_tokens", "head_dim",
                                         "elem_bytes", "num_blocks")])
    return aibx._CacheC(top["d_pool"], top["d_scales"], l, top["type"], top["inner"], top["layer"])


def batch(**kw):
    d = dict(d_block_table=FAKE, d_blk_off=None, table_stride=4, d_tok_off=FAKE, d_kv_len=FAKE, n_tokens=5, R=2,
             max_new=3)
    d.update(kw)
    return aibx._BatchC(*[d[k] for k in ("d_block_table", "d_blk_off", "table_stride", "d_tok_off", "d_kv_len",
                                         "n_tokens", "R", "max_new")])


def params(**kw):
    d = dict(q_type=aibx.TYPE_BF16, num_q_heads=8, q_token_stride=1024, q_head_stride=128, out_token_stride=1024,
             out_head_stride=128, scale=0.1, causal=1, window=0)
    d.update(kw)
    return aibx._AttnC(*[d[k] for k in ("q_type", "num_q_heads", "q_token_stride", "q_head_stride",
                                        "out_token_stride", "out_head_stride", "scale", "causal", "window")])


@pytest.fixture(scope="module")
def lib():
    aibx_build.build()
    return aibx.lib()


def tokens(lib, name, c, b, k=FAKE, v=FAKE, strides=(512, 128, 512, 128), type=aibx.TYPE_BF16):
    return getattr(lib, name)(C.addressof(c) if c is not None else None, C.addressof(b) if b is not None else None, k,
                              strides[0], strides[1], v, strides[2], strides[3], type, None)


def attn(lib, c, b, p, q=FAKE, out=FAKE + 4096, lse=None, ws=FAKE, size=1 << 40):
    return lib.aibx_attn_paged(C.addressof(c) if c is not None else None, C.addressof(b) if b is not None else None,
                               C.addressof(p) if p is not None else None, q, out, lse, ws, size, None)


BAD_CACHE = [dict(layout=3), dict(layout=-1), dict(num_layers=0), dict(num_kv_heads=0), dict(block_tokens=0),
             dict(head_dim=0), dict(layer=2), dict(layer=-1), dict(inner=2), dict(type=aibx.TYPE_FP32), dict(type=9),
             dict(elem_bytes=1), dict(elem_bytes=4), dict(d_pool=None), dict(d_pool=FAKE + 8),
             dict(type=aibx.TYPE_E4M3, elem_bytes=1), dict(type=aibx.TYPE_E4M3, d_scales=FAKE)]
BAD_BATCH = [dict(R=-1), dict(n_tokens=-1), dict(max_new=-1), dict(table_stride=-1), dict(d_block_table=None),
             dict(d_tok_off=None), dict(d_kv_len=None), dict(d_tok_off=FAKE + 4), dict(d_kv_len=FAKE + 2),
             dict(d_block_table=FAKE + 1), dict(d_blk_off=FAKE + 4)]


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_bad_cache(lib, kw):
    for name in ("aibx_kv_append", "aibx_kv_read"):
        assert tokens(lib, name, cache(**kw), batch()) == aibx.ERR_INVALID
    assert attn(lib, cache(**kw), batch(), params()) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", BAD_BATCH)
def test_bad_batch(lib, kw):
    for name in ("aibx_kv_append", "aibx_kv_read"):
        assert tokens(lib, name, cache(), batch(**kw)) == aibx.ERR_INVALID
    assert attn(lib, cache(), batch(**kw), params()) == aibx.ERR_INVALID


@pytest.mark.parametrize("kw", [dict(head_dim=1032), dict(head_dim=12), dict(num_kv_heads=5000),
                                dict(block_tokens=70000), dict(head_dim=8, elem_bytes=1, type=aibx.TYPE_E4M3,
                                                               d_scales=FAKE)])
def test_unsupported_rows(lib, kw):
    for name in ("aibx_kv_append", "aibx_kv_read"):
        assert tokens(lib, name, cache(**kw), batch()) == aibx.ERR_UNSUPPORTED
    assert attn(lib, cache(**kw), batch(), params()) == aibx.ERR_UNSUPPORTED


def test_bad_tokens(lib):
    for name in ("aibx_kv_append", "aibx_kv_read"):
        for kw in (dict(k=None), dict(v=None), dict(k=FAKE + 1), dict(v=FAKE + 1), dict(type=aibx.TYPE_E4M3),
                   dict(type=7), dict(strides=(-1, 128, 512, 128)), dict(strides=(512, 128, 512, -8))):
            assert tokens(lib, name, cache(), batch(), **kw) == aibx.ERR_INVALID, kw
        assert tokens(lib, name, cache(), batch(), k=FAKE + 2, type=aibx.TYPE_FP32) == aibx.ERR_INVALID
        assert tokens(lib, name, None, batch()) == aibx.ERR_INVALID
        assert tokens(lib, name, cache(), None) == aibx.ERR_INVALID


def test_nothing_to_do(lib):
    for kw in (dict(R=0), dict(n_tokens=0), dict(R=0, d_block_table=None, d_tok_off=None, d_kv_len=None)):
        for name in ("aibx_kv_append", "aibx_kv_read"):
            assert tokens(lib, name, cache(d_pool=None), batch(**kw), k=None, v=None) == aibx.OK
        assert attn(lib, cache(d_pool=None), batch(**kw), params(), q=None, out=None, ws=None) == aibx.OK


@pytest.mark.parametrize("kw", [dict(q_type=aibx.TYPE_FP32), dict(q_type=aibx.TYPE_E4M3), dict(num_q_heads=0),
                                dict(num_q_heads=6), dict(window=-1), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=math.inf), dict(scale=math.nan), dict(q_token_stride=1028),
                                dict(q_head_stride=-128), dict(out_token_stride=4), dict(out_head_stride=129)])
def test_bad_attention(lib, kw):
    assert attn(lib, cache(), batch(), params(**kw)) == aibx.ERR_INVALID
    assert lib.aibx_attn_workspace_bytes(*[C.addressof(x) for x in (cache(), batch(), params(**kw))]) == 0


def test_attention_shapes_and_pointers(lib):
    for kw in (dict(head_dim=96), dict(head_dim=256), dict(block_tokens=12), dict(num_blocks=0x80000000)):
        assert attn(lib, cache(**kw), batch(), params()) == aibx.ERR_UNSUPPORTED, kw
    assert attn(lib, cache(num_kv_heads=1), batch(), params(num_q_heads=129)) == aibx.ERR_UNSUPPORTED
    assert attn(lib, cache(), batch(), params(q_type=aibx.TYPE_FP16)) == aibx.ERR_UNSUPPORTED
    assert attn(lib, cache(), batch(n_tokens=1 << 24), params()) == aibx.ERR_UNSUPPORTED
    for kw in (dict(q=None), dict(out=None), dict(ws=None), dict(q=FAKE + 8), dict(out=FAKE + 2), dict(ws=FAKE + 4),
               dict(lse=FAKE + 2), dict(size=1000)):
        assert attn(lib, cache(), batch(), params(), **kw) == aibx.ERR_INVALID, kw
    assert attn(lib, cache(), batch(), None) == aibx.ERR_INVALID


def test_workspace_depends_on_the_shape_of_the_work_alone(lib):
    def size(c, b, p):
        return lib.aibx_attn_workspace_bytes(C.addressof(c), C.addressof(b), C.addressof(p))

    few = size(cache(), batch(max_new=1), params())
    assert 0 < few == size(cache(num_blocks=500, layout=2), batch(max_new=1, n_tokens=900, R=900), params())
    assert few < size(cache(), batch(max_new=100), params()) == size(cache(), batch(max_new=0, R=7), params())


def test_output_in_place_of_queries(lib):
    assert attn(lib, cache(), batch(), params(), q=FAKE, out=FAKE) == aibx.ERR_INVALID
