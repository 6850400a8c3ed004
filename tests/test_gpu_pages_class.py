"""KVPages: what its calls take by default.  Every copied value is compared bit for bit."""
import pytest
import torch

import paper_2608_15522_amd as sa

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def ints(v):
    return torch.tensor(v, **I32)


def tokens(cache, layer, b):
    """What sequence b holds in a layer: [2,Hkv,n,d]."""
    n = int(cache.seq_len[b])
    ids = cache.page_table[b, :-(-n // cache.page)].long()
    return cache.kv[layer][:, ids].transpose(1, 2).flatten(2, 3)[:, :, :n].clone()


def test_rows_of_a_ragged_reservation_by_default():
    """Samples forked from one prompt, each grown by another number of tokens: rows behind them
    are not written, so neither older tokens nor pages that others own change."""
    B, Hkv, d, S, layers = 4, 2, 64, 9, 2
    cache = sa.KVPages(B, 200, 60, Hkv, d, page=16, layers=layers)
    cache.kv.zero_()
    g = torch.Generator(device="cuda").manual_seed(1)
    for first in ([48, 0, 0, 0], None):  # whole pages, then a partial last one
        if first is not None:
            assert cache.reserve(ints(first)).item() == 0
            for layer in range(layers):
                cache.write(layer, *(torch.randn(B, Hkv, 48, d, device="cuda", generator=g)
                                     .bfloat16() for _ in range(2)))
            assert cache.fork(ints([0, 0, 0]), ints([1, 2, 3])).item() == 0
        for new in ([0, 1, 9, 4], [3, 0, -2, 9], [0, 0, 0, 0]):
            old = [[tokens(cache, layer, b) for b in range(B)] for layer in range(layers)]
            n_new = ints(new)
            assert cache.reserve(n_new).item() == 0
            n_new.fill_(S)  # the caller's own again
            k, v = (torch.randn(B, Hkv, S, d, device="cuda", generator=g).bfloat16()
                    for _ in range(2))
            for layer in range(layers):
                cache.write(layer, k, v)
                for b, c in enumerate(new):
                    rows = torch.stack([k[b, :, :max(c, 0)], v[b, :, :max(c, 0)]])
                    assert torch.equal(tokens(cache, layer, b), torch.cat([old[layer][b], rows], 2))
        cache.free(ints([1, 2]))
        assert cache.fork(ints([0, 0]), ints([1, 2])).item() == 0
        assert torch.equal(tokens(cache, 1, 2), tokens(cache, 1, 0))
