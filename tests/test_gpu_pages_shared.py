"""Pages with several owners, on the GPU against the plain lists of oracle.pages: every call
on lists in which sequences share pages, through each of its kernels."""
import random

import pytest
import torch

import paper_2608_15522_amd as sa
from oracle import pages
from test_gpu_pages import SIZES, ints, on_gpu, same

pytestmark = pytest.mark.gpu


def shared_lists(seed, B, n_pages, width, page, longest, used):
    """Lists of a cache in which three of four sequences have leading full pages of an earlier
    one, of a family of up to eight, and about `used` of the pages are taken."""
    rng = random.Random(seed)
    table, lens, ref = [[-1] * width for _ in range(B)], [0] * B, [0] * n_pages
    order = list(range(n_pages))
    rng.shuffle(order)
    left = int(used * n_pages)
    for b in range(B):
        held, n = [], rng.randrange(0, min(longest, width * page) + 1)
        if b % 8:
            a = rng.randrange(b // 8 * 8, b)
            held = table[a][:rng.randrange(0, lens[a] // page + 1)]
        n = max(n, len(held) * page)
        more = min(-(-n // page) - len(held), left)
        n = min(n, (len(held) + more) * page)
        left -= more
        row = held + [order.pop() for _ in range(more)]
        table[b][:len(row)] = row
        for p in row:
            ref[p] += 1
        lens[b] = n
    if B > 8:
        assert max(ref) > 2
    return table, lens, ref


MANY = [c for c in SIZES if c[0] > 1]
# the sizes of tables on either side of what one kernel rewrites by itself (8192 entries)
assert {B * width > 8192 for B, _, width, _, _ in MANY} == {False, True}


@pytest.mark.parametrize("B,n_pages,width,page,longest", MANY)
def test_reserve_and_fork_beside_shared_pages(B, n_pages, width, page, longest):
    print(f"case shared reserve, fork B={B} n_pages={n_pages}", flush=True)
    for seed in range(2):
        lists = shared_lists(seed, B, n_pages, width, page, longest, 0.5)
        rng = random.Random(seed)
        n_new = [min(rng.randrange(0, page + 2), width * page - n) for n in lists[1]]
        t, n, r = on_gpu(lists)
        missing = sa.sa_pages_reserve(t, n, r, ints(n_new), page)
        want = pages.reserve(*lists, n_new, page)
        same((t, n, r, missing), want)
        gone = rng.sample(range(B), B // 2)
        lists = pages.free(*want[:3], gone, page)
        stay = [b for b in range(B) if b not in set(gone)]
        src = [rng.choice(stay[:3]) for _ in gone]  # many owners more for few pages
        t, n, r = on_gpu(lists)
        a, b, missing = sa.sa_pages_fork(t, n, r, ints(src), ints(gone), page)
        same((t, n, r, a, b, missing), pages.fork(*lists, src, gone, page))


@pytest.mark.parametrize("B,n_pages,width,page,longest", MANY)
@pytest.mark.parametrize("share", [0.3, 1.0])
def test_several_owners_freed_at_once(B, n_pages, width, page, longest, share):
    print(f"case shared free B={B} n_pages={n_pages} share={share}", flush=True)
    lists = shared_lists(3, B, n_pages, width, page, longest, 0.6)
    rng = random.Random(4)
    seqs = rng.sample(range(B), max(1, int(share * B)))
    seqs = (seqs + seqs[:5])[:16384]  # some named twice
    t, n, r = on_gpu(lists)
    sa.sa_pages_free(t, n, r, ints(seqs), page)
    want = pages.free(*lists, seqs, page)
    same((t, n, r), want)
    if share == 1.0:
        assert not r.any() and not n.any()


@pytest.mark.parametrize("B,n_pages,width,page,longest", MANY)
@pytest.mark.parametrize("used", [0.1, 0.5, 0.9])
def test_compaction_moves_pages_of_several_owners(B, n_pages, width, page, longest, used):
    print(f"case shared compact B={B} n_pages={n_pages} used={used}", flush=True)
    table, lens, ref = shared_lists(5, B, n_pages, width, page, longest, used)
    want = pages.compact(table, ref)
    t, r = on_gpu((table, ref))
    a, b, c = sa.sa_pages_compact(t, r)
    same((t, r, a, b, c), want)
    if B > 8:  # pages of several owners are among those that moved
        assert max([ref[p] for p in want[2] if p >= 0]) > 1


def test_pools_of_one_page_seen_from_their_other_side():
    pools = torch.arange(6 * 2 * 16 * 64, device="cuda", dtype=torch.float32).view(
        1, 6, 2, 16, 64).transpose(0, 1)  # six pools of one page
    assert pools.is_contiguous() and pools.stride(1) != 2 * 16 * 64
    want = pools.clone()
    sa.sa_pages_copy(pools, ints([0, 0, -1]), ints([0, 1, 0]))  # onto itself; no such pages
    assert torch.equal(pools, want)
