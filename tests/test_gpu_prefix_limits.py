"""sa_prefix_attention at the ends of its lengths, against the fp64 oracle and against
sums that are exact."""
import math
import random

import pytest
import torch

import paper_2608_15522_amd as sa
from oracle import pages
from test_gpu_prefix import I32, check_one, f64, make

pytestmark = pytest.mark.gpu

# few rows, many rows and fp32, by themselves and in groups
FORMS = [("bf16", 4, 2, 2, 5, 64, None), ("bf16", 3, 4, 2, 40, 64, None),
         ("bf16", 5, 2, 1, 150, 128, None), ("f32", 4, 4, 2, 7, 64, None),
         ("f32", 3, 2, 2, 40, 128, None), ("bf16", 6, 2, 2, 3, 128, [64]),
         ("bf16", 20, 4, 1, 2, 64, [48, 96]), ("f32", 6, 4, 2, 3, 64, [64])]


def beyond(form, room):
    """A call of `form` whose sequences fill their rows of the table, with entries that are no
    page for `room` tokens before the last two pages; and the tokens of a row."""
    dtype, B, Hq, Hkv, S, d, shared = form
    page, held = 16, 208
    q, kp, vp, table = make(S + B, [held] * B, Hq, Hkv, S, d, page, dtype, shared or ())
    n = held // page
    table = [r[:n - 2] + [-1] * (room // page) + r[n - 2:n] for r in table]
    return (q, kp, vp, table), held + room // page * page


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("room", [0, 4800])
def test_queries_of_lengths_beyond_the_row_stay_where_they_are(form, room):
    """Query s is token seq_len - q_len + s, also where the table row ends before it: it sees
    every token up to its own that has a page."""
    dtype, B, Hq, Hkv, S, d, shared = form
    (q, kp, vp, table), cap = beyond(form, room)
    rng = random.Random(S)
    for most in (1, S - 1, S, S + 30):
        lens = [cap + (most if b == 0 else rng.randint(0, most)) for b in range(B)]
        for q_len in (None, [S] + [rng.randint(0, S) for _ in range(B - 1)]):
            print(f"case beyond {form} room={room} most={most} q_len={q_len}", flush=True)
            want = pages.paged_attention(f64(q), f64(kp), f64(vp), table, lens, d ** -0.5, q_len,
                                         True)
            check_one(q, kp, vp, table, lens, d ** -0.5, shared, q_len, True, want)


@pytest.mark.parametrize("form", FORMS)
def test_longest_length_that_a_number_holds(form):
    """Every query of a sequence of 2^31 - 1 tokens stands behind the whole row."""
    dtype, B, Hq, Hkv, S, d, shared = form
    print(f"case longest {form}", flush=True)
    (q, kp, vp, table), cap = beyond(form, 0)
    t = torch.tensor(table, **I32)
    sh = None if shared is None else torch.tensor(shared, **I32)
    q_len = torch.tensor([S - b % 2 if b != 1 else 0 for b in range(B)], **I32)
    for n in (None, q_len):
        got = sa.sa_prefix_attention(q, kp, vp, t, torch.full((B,), 2 ** 31 - 1, **I32), d ** -0.5,
                                     shared_len=sh, q_len=n, causal=True, want_lse=True)
        want = sa.sa_prefix_attention(q, kp, vp, t, torch.full((B,), cap, **I32), d ** -0.5,
                                      shared_len=sh, q_len=n, want_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,S,n_pages", [("bf16", 384, (1 << 23) - 1), ("f32", 48, (1 << 23) - 2),
                                             ("bf16", 1, 1 << 23)])
def test_nearly_as_many_tokens_as_there_may_be(dtype, S, n_pages):
    """2^30 tokens, all in one page but for the last 128; with more queries than one, three row
    tiles of 2^24 + 2 units of work each, a number whose threefold no float holds.  The keys
    of the first page are 0, so that every weight before the last page is the same and every
    sum exact; those of the last one outweigh them all."""
    page, d, t = 128, 64, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    print(f"case {n_pages} pages {dtype} S={S}", flush=True)
    kp, vp = torch.zeros(2, 1, page, d, dtype=t, device="cuda"), torch.ones(2, 1, page, d, dtype=t,
                                                                          device="cuda")
    q = torch.zeros(1, 1, S, d, dtype=t, device="cuda")
    q[..., 0], kp[1, ..., 0], vp[1] = 1.0, 240.0, 2.0
    table = torch.zeros(1, 1 << 23, **I32)
    table[0, n_pages - 1] = 1
    o, lse = sa.sa_prefix_attention(q, kp, vp, table, torch.tensor([n_pages * page], **I32), 0.125,
                                    want_lse=True)
    # scores of 0 and 30: the others weigh n_pages / e^30 < 1e-6 of the last page, and O differs
    # from 2 by as much (bf16: 2); 30 log2(e) is off by 4 * 2^-24 of itself at most
    assert (o.float() - 2).abs().max() <= 2e-6
    assert (lse - (30 + math.log(128))).abs().max() <= 2e-5
