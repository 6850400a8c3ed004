"""KVPages: what its calls take by default, and what they do behind a reservation that
failed.  Every copied value is compared bit for bit."""
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


def test_nothing_is_answered_behind_a_reservation_that_failed():
    B, Hkv, d = 2, 1, 64
    cache = sa.KVPages(B, 64, 4, Hkv, d, page=16, dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(2)

    def step(new, S):
        k, v, q = (torch.randn(B, Hkv, S, d, device="cuda", generator=g) for _ in range(3))
        missing = cache.reserve(ints(new)).item()
        cache.write(0, k, v)
        return missing, *cache.attend(0, q, 0.125, causal=True, q_len=cache.new, want_lse=True)

    missing, o, lse = step([20, 7], 20)
    assert missing == 0 and cache.new.tolist() == [20, 7]
    assert (o[0] != 0).any(-1).all() and (o[1, :, 7:] == 0).all()
    old = [tokens(cache, 0, b) for b in range(B)]
    missing, o, lse = step([3, 30], 30)  # two pages more than there are
    assert missing == 1 and cache.new.tolist() == [0, 0] and cache.seq_len.tolist() == [20, 7]
    assert (o == 0).all() and (lse == 0).all()  # made by the call, and left as they were
    assert all(torch.equal(tokens(cache, 0, b), x) for b, x in enumerate(old))
    missing, o, lse = step([3, 9], 9)
    assert missing == 0 and cache.new.tolist() == [3, 9]
    assert (o[0, :, :3] != 0).any(-1).all() and (o[1] != 0).any(-1).all()


def test_captured_steps_of_unequal_numbers_of_tokens():
    """reserve, write and attend in one graph, replayed until a reservation fails and once
    more after it: each replay gives what eager calls give."""
    B, Hkv, d, S = 3, 2, 64, 5

    def new_cache():
        c = sa.KVPages(B, 64, 8, Hkv, d, page=16, dtype=torch.float32)
        c.kv.zero_()
        return c

    n_new = ints([0] * B)
    k, v, q = (torch.zeros(B, Hkv, S, d, device="cuda") for _ in range(3))
    o, lse = torch.zeros_like(q), torch.zeros(B, Hkv, S, device="cuda")
    ws = torch.empty(sa.sa_prefix_attention_workspace(B, Hkv, Hkv, S, d, torch.float32),
                     dtype=torch.uint8, device="cuda")

    def calls(c):
        c.reserve(n_new)
        c.write(0, k, v)
        c.attend(0, q, 0.125, causal=True, q_len=c.new, o=o, lse=lse, ws=ws)

    captured, eager = new_cache(), new_cache()
    calls(captured)  # nothing new
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(captured)
    g = torch.Generator(device="cuda").manual_seed(3)
    failed = []
    for new in ([5, 5, 5], [5, 1, 0], [5, 5, 4], [2, 2, 5], [5, 5, 5], [0, 3, 5], [1, 1, 1],
                [5, 5, 5], [5, 5, 5], [5, 5, 5], [5, 5, 5], [5, 5, 5], [1, 0, 1]):
        n_new.copy_(ints(new))
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        seen = []
        for run, c in ((graph.replay, captured), (lambda: calls(eager), eager)):
            o.fill_(7.0)
            lse.fill_(7.0)
            run()
            torch.cuda.synchronize()
            seen.append([x.clone() for x in (o, lse, c.new, c.missing, c.seq_len, c.page_table,
                                             c.page_ref, c.kv)])
        assert all(torch.equal(x, y) for x, y in zip(*seen)), new
        failed.append(seen[0][3].item() > 0)
        if failed[-1]:
            assert (seen[0][0] == 7).all() and (seen[0][1] == 7).all()
    assert any(failed) and not failed[0] and not failed[-1]
