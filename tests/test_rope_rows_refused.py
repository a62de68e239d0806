"""Rotations whose output rows lie upon one another: refused on the host, so this runs without a GPU; the pointers
are numbers that nothing follows."""
import pytest
import torch

from paper_2504_03648_b200 import binding as aibx
from test_paged_refusals import FAKE, batch, cache, lib  # noqa: F401 (lib is a fixture)
from test_step_refusals import rope, rope_append


@pytest.mark.parametrize("ys", [(0, 128), (256, 0), (0, 0), (120, 128), (256, 64), (64, 640)])
def test_output_rows_upon_one_another(lib, ys):  # noqa: F811
    """Strides below a row's length, of an expanded tensor or otherwise, where there is more than one such row."""
    assert rope(lib, ys=ys) == aibx.ERR_INVALID
    assert rope(lib, x=FAKE, xs=ys, y=FAKE, ys=ys) == aibx.ERR_INVALID              # in place, too
    assert rope_append(lib, cache(), batch(), strides=(512, 128) + ys + (512, 128) * 2) == aibx.ERR_INVALID
    assert rope_append(lib, cache(), batch(), q_out=FAKE, strides=ys * 2 + (512, 128) * 2) == aibx.ERR_INVALID


@pytest.mark.parametrize("ys", [(128, 128), (640, 576), (128, 256), (384, 256), (300, 200)])
def test_rows_of_two_tokens_and_heads_upon_one_another(lib, ys):  # noqa: F811
    """Neighbours are apart, but a token's next heads meet the next tokens (5 tokens, 4 heads)."""
    tok, head = ys
    assert any(abs(t * tok - h * head) < 128 for t in range(1, 5) for h in range(1, 4))
    assert rope(lib, heads=4, ys=ys) == aibx.ERR_INVALID
    assert rope_append(lib, cache(), batch(), strides=(512, 128) + ys + (512, 128) * 2) == aibx.ERR_INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("n,heads,tok,head", [(1, 1, 0, 0), (1, 3, 0, 64), (4, 1, 64, 0), (3, 4, 64, 192), (2, 3, 64, 128),
                                              (3, 2, 128, 64), (2, 5, 64, 192)])
def test_output_rows_in_any_places_that_differ(n, heads, tok, head):
    """Strides of single rows do not count; heads before tokens; rows of both in turn.  A broadcast input is turned."""
    x = torch.randn(64, device="cuda").expand(n, heads, 64)
    rope = aibx.Rope(aibx.rope_frequencies(64)[0].cuda())
    pos = torch.arange(n, dtype=torch.int32, device="cuda") + 5
    y = torch.zeros(4096, device="cuda").as_strided((n, heads, 64), (tok, head, 1))
    want = torch.empty(n, heads, 64, device="cuda")
    aibx.rope(rope, pos, x, y)
    aibx.rope(rope, pos, x, want)
    assert torch.equal(y, want) and bool((want != 0).all())
    if n > 1:
        with pytest.raises(aibx.AibxError):
            aibx.rope(rope, pos, x, x)
