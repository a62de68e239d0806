"""GPU tests of block tables for requests without new tokens whose rows are too short for what they hold."""
import numpy as np
import pytest
import torch

from paged_ref import NO_BLOCK
from paper_2504_03648_b200 import binding as aibx
from test_gpu_tables import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("match", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("held,said", [(64, 0), (65, 1), (200, 1)])
def test_a_row_too_short_for_a_request_without_new_tokens(held, said, ragged, match):
    """Rows of four entries of 16 slots; the middle request gets no new tokens.  Its later blocks are left out, and
    that is said."""
    aibx.status_fetch()
    had = -(-held // 16)
    table = torch.full((3, 4), -1, dtype=torch.int32, device="cuda").view(torch.uint32)
    kv, off = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    ids = np.concatenate([[50], np.arange(20, 20 + had), [60]]).astype(np.uint32)
    more = dict(match_ids=dev(ids), match_off=dev(np.array([0, 1, 1 + had, 2 + had]))) if match else {}
    if ragged:
        more["blk_off"] = dev(np.array([0, 4, 8, 12]))
    head = torch.zeros(1, dtype=torch.int64, device="cuda")
    aibx.kv_tables(dev(np.array([16, held, 16], dtype=np.int32)), dev(np.array([1, 0, 20], dtype=np.int32)), 16, 100,
                   dev(np.arange(9, dtype=np.uint32)), head, torch.full_like(head, 9), table.view(-1) if ragged else table,
                   off, kv, 21, **more)
    assert aibx.status_fetch() == ((aibx.ERR_RANGE, 1) if said else (0, 0))
    want = np.full((3, 4), NO_BLOCK, dtype=np.uint32)
    if match:
        want[0, 0], want[2, 0] = 50, 60
        want[1] = np.arange(20, 24)
    want[0, 1], want[2, 1:3] = 0, [1, 2]
    assert np.array_equal(table.cpu().numpy(), want)
    assert kv.tolist() == [17, held, 36] and off.tolist() == [0, 1, 1, 21] and int(head) == 3
