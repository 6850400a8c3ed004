"""Host side of the paged calls, on the CPU: the sizes that the binding hands over.  No call
here reaches a kernel."""
import os

import pytest
import torch

import paper_2608_15522_amd as sa
from paper_2608_15522_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH),
                                reason="libsa.so not built")


@pytest.mark.parametrize("pools,page_bytes", [
    (torch.zeros(3, 5, 2, 16, 64), 2 * 16 * 64 * 4),
    (torch.zeros(3, 5, 32, dtype=torch.bfloat16), 64),
    # a dimension of one may have any stride: a tensor seen from its other side is contiguous,
    # and its pages lie a page apart all the same
    (torch.zeros(1, 7, 2, 16, 64).transpose(0, 1), 2 * 16 * 64 * 4),
    (torch.zeros(4, 16, dtype=torch.uint8).as_strided((1, 1, 16), (16, 1 << 20, 1)), 16)])
def test_bytes_of_a_page(monkeypatch, pools, page_bytes):
    seen = []

    class Library:
        def sa_pages_copy(self, *args):
            seen.append(args)
            return sa.SA_OK

    assert pools.is_contiguous()
    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(binding, "_ptr", lambda t: t.data_ptr())
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    pairs = torch.zeros(1, dtype=torch.int32)
    sa.sa_pages_copy(pools, pairs, pairs)
    (args,) = seen
    assert args[1:4] == (pools.shape[0], pools.shape[1], page_bytes)
