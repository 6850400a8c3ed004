"""sa_prefix_attention: every tile of values counts, once, and at its place.

A bound on each element of O that allows for the rounding of every weight does not shrink
with the number of keys, though O does, so it would let a wrong tile of V in a long sequence
pass.  Two checks that would not:

* Keys of 0 give every visible key the same weight.  All sums are then exact (integers below
  2^24 times a power of two), and O, the mean of the visible values, is off by its division
  (2^-22 of itself) and its own rounding (bf16: half a step, 2^-8 of itself).  The values of
  64-key tile t are 0 but for channel t mod d, so a tile that is left out, taken twice or taken
  for another one changes a channel by far more than that.
* Random keys: an error of a weight is at most half a step of bf16, 2^-8 of it, and that of
  its score, (d + 4) 2^-24 of sum |q_i k_i| * scale.  Errors of different keys have no common
  sign, so the root mean square of O's error over all rows and channels is at most so many
  times that of sqrt(sum (w v)^2), besides the share of O's own root mean square that its
  rounding and those of the row sum take, 2^-8 and (64 + keys) 2^-24.
"""
import random

import pytest
import torch

import paper_2608_15522_amd as sa
from test_gpu_prefix import I32, TYPES, make

pytestmark = pytest.mark.gpu

# dtype, sequences, query heads, key heads, queries, d, page, shared tokens, own tokens
CALLS = [
    ("bf16", 5, 4, 2, 1, 64, 16, 0, 1, 700),
    ("bf16", 2, 2, 1, 1, 64, 16, 40000, 1, 9),          # a row tile in every slot
    ("bf16", 3, 2, 2, 1, 128, 64, 0, 20000, 33000),
    ("bf16", 64, 8, 2, 1, 128, 64, 2048, 1, 700),       # shared keys in tiles of 128 rows
    ("bf16", 12, 4, 2, 6, 64, 32, 1024, 6, 900),
    ("bf16", 3, 4, 4, 200, 128, 128, 1024, 200, 900),
    ("bf16", 1, 2, 2, 1000, 64, 32, 0, 1000, 3000),
    ("bf16", 1, 1, 1, 300, 128, 16, 0, 30000, 30001),
    ("bf16", 1, 16, 16, 4224, 64, 128, 0, 4224, 4300),  # rounds, then the rest cut
    ("bf16", 130, 4, 4, 1, 128, 64, 0, 2480, 2500),
    ("bf16", 512, 8, 8, 1, 64, 16, 0, 1, 60),
    ("f32", 5, 4, 2, 1, 128, 32, 0, 1, 700),
    ("f32", 2, 2, 1, 1, 64, 16, 40000, 1, 9),
    ("f32", 16, 4, 1, 3, 64, 32, 1024, 3, 400),
    ("f32", 2, 2, 2, 100, 128, 64, 512, 100, 700),
    ("f32", 70, 8, 8, 2, 64, 64, 0, 1500, 1510),
]
# as many queries as there may be
LONGEST = [("bf16", 1, 1, 1, 262144, 64, 128, 0, 262144, 262144),
           ("f32", 1, 1, 1, 40000, 64, 32, 0, 40000, 40100)]


def lengths(call):
    _, B, _, _, _, _, _, shared, lo, hi = call
    return [shared + lo + (hi - lo) * b // max(B - 1, 1) for b in range(B - 1)] + [shared + hi]


def rows(call, seed, causal):
    """q_len: all queries, or an unequal number of each sequence."""
    B, S = call[1], call[4]
    rng = random.Random(seed)
    return (None if not causal or S == 1 else
            [S] + [rng.choice([0, 1, S // 2, S - 1, S]) for _ in range(B - 1)])


def attend(q, kp, vp, table, lens, shared, q_len, causal, room):
    table = [r + [-1] * (room // kp.shape[2]) for r in table]
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device="cuda")
    return sa.sa_prefix_attention(
        q, kp, vp, torch.tensor(table, **I32), torch.tensor(lens, **I32), q.shape[3] ** -0.5,
        shared_len=torch.tensor([shared], **I32) if shared else None, causal=causal,
        q_len=None if q_len is None else torch.tensor(q_len, **I32), o=o, lse=lse)


def tile_values(at, tokens, heads, d, off):
    """[tokens,heads,d]: position p holds 1 to 4, by p // (64 d), in channel
    p // 64 + 3 head + off, else 0."""
    p = torch.arange(at, at + tokens, device="cuda")
    h = torch.arange(heads, device="cuda")
    c = (p[:, None] // 64 + 3 * h + off) % d
    amp = (1 + p // (64 * d) % 4).double()
    v = torch.zeros(tokens, heads, d, dtype=torch.float64, device="cuda")
    return v.scatter_(2, c[..., None], amp[:, None, None].expand(tokens, heads, 1))


@pytest.mark.parametrize("call", CALLS + LONGEST, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("causal", [False, True])
def test_every_tile_counts_once(call, causal):
    print(f"case tiles {call} causal={causal}", flush=True)
    dtype, B, Hq, Hkv, S, d, page, shared, _, _ = call
    shared = shared // page * page
    lens, q_len = lengths(call), rows(call, 1, causal)
    q, kp, vp, table = make(S, lens, Hq, Hkv, S, d, page, dtype, [shared] if shared else ())
    kp.zero_()
    flat = vp.transpose(1, 2).reshape(-1, Hkv, d)  # a copy, token by token
    want, seen = [], []
    for b, n in enumerate(lens):
        v = torch.cat([tile_values(0, shared, Hkv, d, 0),
                       tile_values(shared, n - shared, Hkv, d, 5 * b)])
        at = torch.tensor(table[b], device="cuda").clamp(min=0)[:, None] * page + torch.arange(
            page, device="cuda")
        flat[at.flatten()[:n]] = v.to(vp.dtype)
        new = S if q_len is None else q_len[b]
        s = torch.arange(new, device="cuda")
        see = n - new + 1 + s if causal else torch.full_like(s, n)
        see = see.clamp(min=0)
        sums = torch.cat([torch.zeros(1, Hkv, d, device="cuda"), v]).cumsum(0)[see]
        mean = sums / see.clamp(min=1)[:, None, None]
        want.append(mean.transpose(0, 1).repeat_interleave(Hq // Hkv, 0))  # [Hq,new,d]
        seen.append(see)
    vp = flat.view(-1, page, Hkv, d).transpose(1, 2).contiguous()
    for room in (0, 10000):
        o, lse = attend(q, kp, vp, table, lens, shared, q_len, causal, room)
        for b in range(B):
            new = len(seen[b])
            off = (o[b, :, :new].double() - want[b]).abs()
            tol = (2.0 ** -22 + (2.0 ** -8 if dtype == "bf16" else 0)) * want[b]
            assert (off <= tol).all(), (room, b, (off - tol).max())
            z = seen[b].double().log()
            # a logarithm below 8 in magnitude (fp32 sums are taken down by 2^-8), twice its last
            # place, and the rounding of lse
            assert ((lse[b, :, :new] - z).abs() <= 2.0 ** -20 + 2.0 ** -22 * z).logical_or(
                seen[b] == 0).all()
            assert (o[b, :, new:] == 7).all() and (lse[b, :, new:] == 7).all()


@pytest.mark.parametrize("call", [c for c in CALLS if c[0] == "bf16"],
                         ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("causal", [False, True])
def test_mean_square_of_the_error(call, causal):
    print(f"case mean square {call} causal={causal}", flush=True)
    dtype, B, Hq, Hkv, S, d, page, shared, _, _ = call
    shared = shared // page * page
    lens, q_len = lengths(call), rows(call, 2, causal)
    q, kp, vp, table = make(S + 1, lens, Hq, Hkv, S, d, page, dtype, [shared] if shared else ())
    calls = [attend(q, kp, vp, table, lens, shared, q_len, causal, room)[0] for room in (0, 10000)]
    # per call: sums of squares of the error; of the bound on the weights' part; of O
    err, spread, size, number = [0.0, 0.0], 0.0, 0.0, 0
    X = 0.0  # largest sum of a score's products in magnitude
    for b, n in enumerate(lens):
        new = S if q_len is None else q_len[b]
        ids = torch.tensor(table[b][:-(-n // page)], dtype=torch.long, device="cuda")
        for h in range(Hkv):
            k, v = (p[ids, h].reshape(-1, d)[:n].double() for p in (kp, vp))
            at = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv)
            x = torch.matmul(q[b, at, :new].double().reshape(-1, d),
                             k.t().contiguous()).view(Hq // Hkv, new, n) * d ** -0.5
            if new > 0:
                X = max(X, torch.matmul(q[b, at, :new].double().abs().reshape(-1, d),
                                        k.t().abs().contiguous()).max().item() * d ** -0.5)
            if causal:
                see = (torch.arange(n, device="cuda") <=
                       n - new + torch.arange(new, device="cuda")[:, None])
                x.masked_fill_(~see, -float("inf"))
            w = x.softmax(-1).nan_to_num_(0.0)  # a row without a key
            o = torch.matmul(w, v)
            spread += torch.matmul(w.square_(), v.square()).sum().item()
            size += o.square().sum().item()
            number += o.numel()
            for i, got in enumerate(calls):
                err[i] += (got[b, at, :new].double() - o).square().sum().item()
    u = 2.0 ** -24
    bound = ((2.0 ** -8 + (d + 4) * X * u) * (spread / number) ** 0.5 +
             (2.0 ** -8 + (64 + max(lens)) * u) * (size / number) ** 0.5)
    for e in err:
        assert (e / number) ** 0.5 <= bound, ((e / number) ** 0.5, bound)
