"""Host side of the paged calls, on the CPU: the sizes that the binding hands over, and
numbers of pages near the end of their type.  No call here reaches a kernel."""
import os

import pytest
import torch

import paper_2608_15522_amd as sa
from paper_2608_15522_amd import binding
from test_host_pages import _compact, _fork, _free, _reserve

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


@pytest.mark.parametrize("call", [_reserve, _fork, _free, _compact], ids=lambda c: c.name)
@pytest.mark.parametrize("n_pages", [2 ** 30 + 1, 2 ** 31 - 16384, 2 ** 31 - 1])
def test_more_pages_than_can_be_counted_are_refused(call, n_pages):
    """The kernels take 16384 page numbers a step, in 32 bits: the number behind the last step
    has to fit."""
    assert call(n_pages=n_pages) == sa.SA_ERR_UNSUPPORTED
    assert call.name in sa.sa_last_error() and f"n_pages={n_pages}" in sa.sa_last_error()
