"""The range of scales that attention takes, decided on the host (no GPU needed)."""
import ctypes as C

import pytest

from paper_2504_03648_b200 import binding as aibx
from test_paged_refusals import attn, batch, cache, lib, params  # noqa: F401 (lib is a fixture)


@pytest.mark.parametrize("scale,taken", [(2.0 ** -149, False), (2.0 ** -127, False), (2.0 ** -126, True), (1e-3, True), (1e30, True),
                                         (2.0 ** 127, True), (2.5e38, False), (3.4e38, False)])
def test_scales(lib, scale, taken):  # noqa: F811
    objs = cache(), batch(), params(scale=scale)
    size = lib.aibx_attn_workspace_bytes(*[C.addressof(x) for x in objs])
    assert (size > 0) == taken
    if not taken:
        assert attn(lib, *objs) == aibx.ERR_INVALID
