"""The page oracle on the CPU: hand-made lists, invariants of random ones, and its
attention against a library routine in fp64."""
import random

import numpy as np
import pytest
import torch

from oracle import pages


def test_reserve_by_hand():
    # page of 4: sequence 0 has room for one more token, 1 is empty
    table, lens, ref = [[2, -1, -1], [-1, -1, -1]], [3, 0], [0, 0, 1, 0]
    t, n, r, lack = pages.reserve(table, lens, ref, [2, 5], 4)
    assert (t, n, r, lack) == ([[2, 0, -1], [1, 3, -1]], [5, 5], [1, 1, 1, 1], 0)
    t, n, r, lack = pages.reserve(table, lens, ref, [6, 5], 4)  # four of three pages
    assert (t, n, r, lack) == (table, lens, ref, 1)
    t, n, r, lack = pages.reserve(table, lens, ref, [0, 13], 4)  # a row of three entries
    assert (t, n, r, lack) == (table, lens, ref, 2)


def test_fork_by_hand():
    table, lens, ref = [[3, 1, -1], [-1] * 3, [-1] * 3], [6, 0, 0], [0, 1, 0, 1]
    t, n, r, a, b, lack = pages.fork(table, lens, ref, [0, 0, 0, 1], [1, 2, 1, 2], 4)
    assert t == [[3, 1, -1], [3, 0, -1], [3, 2, -1]] and n == [6, 6, 6]
    assert r == [1, 1, 1, 3] and (a, b, lack) == ([1, 1, -1, -1], [0, 2, -1, -1], 0)
    t, n, r, a, b, lack = pages.fork(table, lens, [1, 1, 1, 1], [0], [1], 4)
    assert (t, n, a, b, lack) == (table, lens, [-1], [-1], 1)


def test_free_and_compact_by_hand():
    table, lens, ref = [[5, 1], [5, 4], [-1, -1]], [8, 6, 0], [0, 1, 0, 0, 1, 2]
    t, n, r = pages.free(table, lens, ref, [0, 0, 7, -1], 4)
    assert (t, n, r) == ([[-1, -1], [5, 4], [-1, -1]], [0, 6, 0], [0, 0, 0, 0, 1, 1])
    t, r, a, b, c = pages.compact(t, r)
    assert t == [[-1, -1], [1, 0], [-1, -1]] and r == [1, 1, 0, 0, 0, 0]
    assert (a, b, c) == ([4, 5, -1], [0, 1, -1], [2, 2])


@pytest.mark.parametrize("seed", range(20))
def test_random_histories_keep_the_owners(seed):
    """After any history an owner count is the number of table entries of the page."""
    rng = random.Random(seed)
    page, B, n_pages, width = rng.choice([4, 16]), 6, 40, 9
    table, lens, ref = [[-1] * width for _ in range(B)], [0] * B, [0] * n_pages
    for _ in range(40):
        what = rng.randrange(4)
        if what == 0:
            table, lens, ref, _ = pages.reserve(table, lens, ref,
                                                [rng.randrange(-1, 9) for _ in range(B)], page)
        elif what == 1:
            k = rng.randrange(1, B)
            table, lens, ref, *_ = pages.fork(table, lens, ref,
                                              [rng.randrange(-1, B + 1) for _ in range(k)],
                                              [rng.randrange(-1, B + 1) for _ in range(k)], page)
        elif what == 2:
            table, lens, ref = pages.free(table, lens, ref,
                                          [rng.randrange(-1, B + 1) for _ in range(2)], page)
        else:
            table, ref, src, dst, (used, moves) = pages.compact(table, ref)
            assert all(r > 0 for r in ref[:used]) and not any(ref[used:])
            assert len([p for p in src if p >= 0]) == moves
        count = [0] * n_pages
        for b, row in enumerate(table):
            held = -(-lens[b] // page)
            assert all(0 <= p < n_pages for p in row[:held]) and set(row[held:]) <= {-1}
            for p in row[:held]:
                count[p] += 1
        assert count == ref


@pytest.mark.parametrize("causal", [False, True])
def test_attention_against_a_library_routine(causal):
    rng = np.random.default_rng(3)
    B, Hq, Hkv, S, d, page, n_pages = 3, 4, 2, 5, 8, 16, 12
    lens = [37, 16, 9]
    perm = rng.permutation(n_pages).tolist()
    table = [[perm.pop() for _ in range(3)] for _ in range(B)]
    q = rng.standard_normal((B, Hq, S, d))
    k, v = rng.standard_normal((2, n_pages, Hkv, page, d))
    o, lse, size = pages.paged_attention(q, k, v, table, lens, 0.3, causal=causal)
    for b in range(B):
        kk, vv = (torch.from_numpy(x[table[b]].transpose(1, 0, 2, 3).reshape(Hkv, -1, d)
                                   [:, :lens[b]].copy()).repeat_interleave(2, 0) for x in (k, v))
        mask = torch.ones(S, lens[b], dtype=torch.bool)
        if causal:
            mask = torch.tril(mask, lens[b] - S)
        want = torch.nn.functional.scaled_dot_product_attention(
            torch.from_numpy(q[b]), kk, vv, attn_mask=mask, scale=0.3)
        np.testing.assert_allclose(o[b], want.numpy(), atol=1e-12)
        x = (torch.from_numpy(q[b]) @ kk.transpose(1, 2) * 0.3).masked_fill(~mask, -np.inf)
        np.testing.assert_allclose(lse[b], torch.logsumexp(x, -1).numpy(), atol=1e-12)
    assert (size >= np.abs(o) - 1e-12).all()


def test_attention_leaves_out_what_is_no_page_and_empty_rows():
    rng = np.random.default_rng(4)
    q = rng.standard_normal((2, 1, 2, 4))
    k, v = rng.standard_normal((2, 3, 1, 16, 4))
    o, lse, _ = pages.paged_attention(q, k, v, [[1, 7, 2], [-1, -1, -1]], [40, 0], 1.0,
                                      q_len=[2, 1])
    keys = np.concatenate([k[1, 0], k[2, 0, :8]])
    vals = np.concatenate([v[1, 0], v[2, 0, :8]])
    w = np.exp(keys @ q[0, 0, 1])
    np.testing.assert_allclose(o[0, 0, 1], w @ vals / w.sum(), atol=1e-12)
    assert (o[1, 0, 0] == 0).all() and lse[1, 0, 0] == -np.inf and np.isnan(lse[1, 0, 1])
