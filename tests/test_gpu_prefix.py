"""sa_prefix_attention through the binding against the fp64 oracle.

Bounds.  With u = 2^-24 (fp32) and X = scale * sum |q_i k_i| of a row, a score is off by
at most (d + 4) u X (products and sums in fp32, the scale and the subtraction of the
reference), so a weight by that, relatively, and lse by that.  A sum over n keys in fp32 is
off by less than n u, relatively, and the exp2 of the weights and of the joined parts by
64 u in all.  O is a weighted mean of v: errors e in the weights
change it by at most 2 e * size, size the weighted mean of |v|.  In bf16 the weights are
rounded (half a step: 2^-8) and so is O (2^-8 of its value); the row sum is not, so an
error of the weights counts once.
"""
import random

import numpy as np
import pytest
import torch

import paper_2608_15522_amd as sa
from oracle import pages

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(seed, lens, Hq, Hkv, S, d, page, dtype, shared=(), spare=2, gain=1.0):
    """Inputs with the groups' first shared[g] tokens (whole pages) in the same pages."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    per = B // len(shared) if shared else B
    width = max(1, -(-max(max(lens), 1) // page)) + 1
    need = sum(-(-max(n, 0) // page) for n in lens) + spare
    order = torch.randperm(need, generator=g).tolist()
    table = []
    common = []
    for b, n in enumerate(lens):
        if shared and b % per == 0:
            common = []
        n_sh = shared[b // per] // page if shared else 0
        row = []
        for j in range(-(-max(n, 0) // page)):
            if j < n_sh:
                if j == len(common):
                    common.append(order.pop())
                row.append(common[j])
            else:
                row.append(order.pop())
        table.append(row + [-1] * (width - len(row)))
    t = TYPES[dtype]
    q = (torch.randn(B, Hq, S, d, generator=g) * gain).to(t).cuda()
    kp, vp = (torch.randn(need, Hkv, page, d, generator=g).to(t).cuda() for _ in range(2))
    return q, kp, vp, table


def f64(x):
    return x.double().cpu().numpy()


def check(q, kp, vp, table, lens, scale, shared=None, q_len=None, causal=False, want=None):
    """Runs the call on poisoned outputs and compares it, with the table as given and with
    rows that have room for 10000 tokens more (the length of the rows decides how the work is
    cut up); returns (o, lse) of the first."""
    if want is None:
        want = pages.paged_attention(f64(q), f64(kp), f64(vp), table, lens, scale, q_len, causal)
    wide = [list(r) + [-1] * (10000 // kp.shape[2]) for r in table]
    check_one(q, kp, vp, wide, [min(n, len(table[0]) * kp.shape[2]) for n in lens], scale, shared,
              q_len, causal, want)
    return check_one(q, kp, vp, table, lens, scale, shared, q_len, causal, want)


def check_one(q, kp, vp, table, lens, scale, shared, q_len, causal, want):
    B, Hq, S, d = q.shape
    bf = q.dtype == torch.bfloat16
    o = torch.full_like(q, 7.0)
    lse = torch.full((B, Hq, S), 7.0, device="cuda")
    sa.sa_prefix_attention(
        q, kp, vp, torch.tensor(table, **I32), torch.tensor(lens, **I32), scale,
        shared_len=None if shared is None else torch.tensor(shared, **I32),
        q_len=None if q_len is None else torch.tensor(q_len, **I32), causal=causal, o=o, lse=lse)
    torch.cuda.synchronize()
    ro, rl, size = want
    got_o, got_l = f64(o), f64(lse)
    real = ~np.isnan(rl)
    if q_len is not None:
        assert (~real).sum() == Hq * sum(S - n for n in q_len)
    assert (got_o[~real] == 7.0).all() and (got_l[~real] == 7.0).all(), "rows behind q_len written"
    none = real & (rl == -np.inf)
    assert (got_o[none] == 0.0).all() and (got_l[none] == -np.inf).all(), "rows without a key"
    some = real & ~none
    big = max(float(np.nanmax(np.abs(f64(kp)))), 1e-30)
    X = scale * np.abs(f64(q)).sum(-1) * big
    e = ((d + 4) * X + max(lens) + 64) * 2.0 ** -24
    assert np.isfinite(got_o[some]).all()
    # lse: the same relative error, and its own rounding
    off = np.abs(got_l[some] - rl[some]) - (e[some] + 2.0 ** -22 * np.abs(rl[some]))
    assert off.max(initial=-1) <= 0, f"lse off by {np.abs(got_l[some] - rl[some]).max()}"
    tol = 2 * e[..., None] * size + (2.0 ** -8 * (size * 1.02 + np.abs(ro)) if bf else
                                     2.0 ** -23 * np.abs(ro)) + 1e-37
    off = (np.abs(got_o - ro) - tol)[some]
    assert off.max(initial=-1) <= 0, f"o off by {np.abs(got_o - ro)[some].max()}"
    return o, lse


LENS = [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 257]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_one_token_of_unequal_lengths(dtype, page, d):
    print(f"case one token {dtype} page={page} d={d}", flush=True)
    q, kp, vp, table = make(page + d, LENS + [0], 4, 2, 1, d, page, dtype)
    check(q, kp, vp, table, LENS + [0], d ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hkv,S,page", [(1, 1, 2, 16), (6, 2, 5, 32), (8, 1, 17, 16),
                                           (3, 3, 33, 64), (4, 2, 70, 16), (2, 1, 129, 128),
                                           (1, 1, 300, 32), (16, 2, 40, 16)])
def test_several_queries(dtype, causal, Hq, Hkv, S, page):
    print(f"case {dtype} causal={causal} Hq={Hq} Hkv={Hkv} S={S} page={page}", flush=True)
    lens = [S, S + 64, S + 1, max(S - 3, 0), 2 * S + 129]
    q, kp, vp, table = make(S, lens, Hq, Hkv, S, 64, page, dtype)
    check(q, kp, vp, table, lens, 0.125, causal=causal)
    q_len = [S, 0, S // 2, min(2, S), S - 1]
    check(q, kp, vp, table, lens, 0.125, q_len=q_len, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups,per,Hq,Hkv,S,page,shared", [
    (1, 2, 2, 2, 1, 16, [16]), (1, 5, 4, 2, 1, 16, [80]), (2, 3, 4, 1, 1, 32, [32, 96]),
    (1, 40, 2, 1, 1, 64, [320]), (2, 4, 6, 2, 7, 16, [48, 0]), (1, 3, 2, 2, 33, 128, [256]),
    (3, 2, 1, 1, 20, 16, [112, 64, 16]), (1, 9, 8, 1, 5, 16, [144]), (2, 20, 2, 2, 4, 16, [64, 208])])
@pytest.mark.parametrize("causal", [False, True])
def test_shared_tokens(dtype, groups, per, Hq, Hkv, S, page, shared, causal):
    print(f"case shared {dtype} {groups}x{per} Hq={Hq} Hkv={Hkv} S={S} page={page} {shared} "
          f"causal={causal}", flush=True)
    rng = random.Random(S + per)
    lens = [shared[b // per] + S + rng.randrange(0, 150) for b in range(groups * per)]
    for d in (64, 128):
        q, kp, vp, table = make(per + d, lens, Hq, Hkv, S, d, page, dtype, shared)
        o, lse = check(q, kp, vp, table, lens, d ** -0.5, shared=shared, causal=causal)
        # a statement that holds for fewer tokens, or is no whole number of pages
        check(q, kp, vp, table, lens, d ** -0.5, shared=[max(n - 5, 0) for n in shared],
              causal=causal)


def test_shared_tokens_are_what_every_sequence_has():
    """Claims beyond a sequence's tokens, sequences without tokens, padded queries."""
    page, S, shared = 16, 3, [96, 64]
    lens = [130, 0, 100, 20, 0, 0, 0, 0]
    for dtype in ("bf16", "f32"):
        q, kp, vp, table = make(3, lens, 4, 2, S, 64, page, dtype, [96, 0])
        for claim in (shared, [2 ** 31 - 1, 5], [-3, -1]):
            check(q, kp, vp, table, lens, 0.125, shared=claim)
            check(q, kp, vp, table, lens, 0.125, shared=claim, q_len=[3, 2, 0, 1, 3, 0, 1, 2],
                  causal=True)
        # causal, and the newest queries lie among the shared tokens
        lens2 = [97, 96, 99, 98]
        q, kp, vp, table = make(4, lens2, 4, 2, S, 64, page, dtype, [96])
        check(q, kp, vp, table, lens2, 0.125, shared=[96], causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_whatever_lies_behind_a_sequence_is_not_used(dtype):
    """NaN and infinities in every free slot of the pages and in unused pages, entries
    that are no page, lengths beyond the table."""
    lens, page = [5, 70, 0, 130, 33], 16
    q, kp, vp, table = make(9, lens, 2, 1, 2, 64, page, dtype)
    used = torch.zeros(kp.shape[0], page, dtype=torch.bool)
    for row, n in zip(table, lens):
        for t in range(n):
            used[row[t // page], t % page] = True
    gone = (~used).cuda()[:, None, :, None].expand_as(kp)
    clean = check(q, kp, vp, table, lens, 0.2)
    want = pages.paged_attention(f64(q), f64(kp), f64(vp), table, lens, 0.2)
    for bad in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = kp.masked_fill(gone, bad), vp.masked_fill(gone, bad)
        o, lse = check(q, k2, v2, table, lens, 0.2, want=want)
        assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    # entries that are no page: their keys are left out
    holes = [list(r) for r in table]
    holes[1][1], holes[1][3], holes[3][0], holes[4][2], holes[0][0] = -1, 999999, -7, 2 ** 30, -1
    check(q, kp, vp, holes, lens, 0.2)
    check(q, kp, vp, holes, lens, 0.2, causal=True)
    # longer than the row of the table
    width = len(table[0])
    check(q, kp, vp, table, [5, 70, -4, 130, 33], 0.2,
          want=pages.paged_attention(f64(q), f64(kp), f64(vp), table, [5, 70, 0, 130, 33], 0.2))
    full = [list(range(6))[:width] + [-1] * (width - 6) for _ in lens]
    got = sa.sa_prefix_attention(q, kp, vp, torch.tensor([r[:3] for r in full], **I32),
                                 torch.tensor([10 ** 9] * 5, **I32), 0.2, want_lse=True)
    ref = sa.sa_prefix_attention(q, kp, vp, torch.tensor([r[:3] for r in full], **I32),
                                 torch.tensor([48] * 5, **I32), 0.2, want_lse=True)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_every_size(dtype):
    """Logits that rise or fall by a hundred units along the keys, that are -inf, and a
    row of -inf only; infinite and NaN keys that the row sees give what they give in fp64."""
    lens, page, d = [300, 300, 150], 32, 64
    q, kp, vp, table = make(21, lens, 2, 2, 3, d, page, dtype)
    u = torch.zeros(d)
    u[0] = 1.0
    q = (q * 0.25 + 8 * u.cuda().to(q.dtype))
    for rise in (0.35, -0.35):
        k2 = kp.clone()
        for row, n in zip(table, lens):
            for t in range(n):
                k2[row[t // page], :, t % page, 0] = rise * t
        check(q, k2, vp, table, lens, 0.125)
    # the first component of q is positive: -inf keys give -inf logits, others stay
    k2 = kp.clone()
    for t in list(range(0, 64)) + list(range(100, 150)):
        for row in table:
            k2[row[t // page], :, t % page, 0] = -float("inf")
    o, lse = sa.sa_prefix_attention(q, k2, vp, torch.tensor(table, **I32),
                                    torch.tensor(lens, **I32), 0.125, want_lse=True)
    keep = [[t for t in range(n) if not (t < 64 or 100 <= t < 150)] for n in lens]
    for b, at in enumerate(keep):
        ids = torch.tensor([table[b][t // page] for t in at], device="cuda")
        pos = torch.tensor([t % page for t in at], device="cuda")
        x = torch.einsum("hsd,khd->hsk", q[b].double(), k2[ids, :, pos].double()) * 0.125
        ref = torch.einsum("hsk,khd->hsd", x.softmax(-1), vp[ids, :, pos].double())
        # size <= max |v| < 5; weights and O rounded as above
        assert (o[b].double() - ref).abs().max() <= (0.05 if dtype == "bf16" else 1e-4)
        assert (lse[b].double() - x.logsumexp(-1)).abs().max() <= 1e-4
    k2 = kp.clone()
    k2[..., 0] = -float("inf")
    o, lse = sa.sa_prefix_attention(q, k2, vp, torch.tensor(table, **I32),
                                    torch.tensor(lens, **I32), 0.125, want_lse=True)
    assert (o == 0).all() and (lse == -float("inf")).all()
    k2 = kp.clone()
    k2[table[1][3], :, 5] = float("nan")
    o, lse = sa.sa_prefix_attention(q, k2, vp, torch.tensor(table, **I32),
                                    torch.tensor(lens, **I32), 0.125, want_lse=True)
    assert o[1].isnan().all() and lse[1].isnan().all()
    assert o[0].isfinite().all() and o[2].isfinite().all()


@pytest.mark.parametrize("dtype,B,Hq,Hkv,S,d,shared,lo,hi,page", [
    ("bf16", 64, 8, 2, 1, 128, 2048, 1, 700, 64),      # prefix rows of two wide tiles
    ("bf16", 2, 2, 1, 1, 64, 40000, 1, 9, 16),         # one row tile in every slot
    ("bf16", 3, 4, 4, 200, 128, 1024, 200, 900, 128),  # each sequence by itself, rows cut
    ("bf16", 1, 2, 2, 1000, 64, 0, 1000, 3000, 32),
    ("f32", 16, 4, 1, 3, 64, 1024, 3, 400, 32),
    ("f32", 2, 2, 2, 100, 128, 512, 100, 700, 64),
    ("bf16", 512, 1, 1, 1, 64, 256, 0, 200, 16),       # as many segments as there may be
    # more row tiles than slots of nearly the same length: whole ones first, the rest cut
    ("bf16", 1, 16, 16, 4224, 64, 0, 4224, 4300, 128),
    ("bf16", 130, 4, 4, 1, 128, 0, 2480, 2500, 64),
    ("f32", 70, 8, 8, 2, 64, 0, 1500, 1510, 64),
    ("bf16", 512, 8, 8, 1, 64, 0, 1, 60, 16),          # eight row tiles a slot
])
@pytest.mark.parametrize("causal", [False, True])
def test_larger_calls(dtype, B, Hq, Hkv, S, d, shared, lo, hi, page, causal):
    print(f"case large {dtype} B={B} Hq={Hq} S={S} shared={shared} causal={causal}", flush=True)
    lens = [shared + lo + (hi - lo) * b // max(B - 1, 1) for b in range(B)]
    lens[-1] = shared + hi
    q, kp, vp, table = make(B + S, lens, Hq, Hkv, S, d, page, dtype, [shared])
    want = reference(q, kp, vp, table, lens, d ** -0.5, causal)
    for claim in ([shared], None) if B < 512 or Hkv > 1 else ([shared] * 512, [shared]):
        o, lse = check(q, kp, vp, table, lens, d ** -0.5, shared=claim, causal=causal, want=want)
        again = check(q, kp, vp, table, lens, d ** -0.5, shared=claim, causal=causal, want=want)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1]), "run to run"


@pytest.mark.parametrize("dtype,B,Hq,Hkv,S,d,lo,hi", [
    ("bf16", 7, 16, 4, 410, 64, 0, 500),      # two XCDs to a head, an odd number of row tiles
    ("bf16", 5, 3, 3, 2600, 128, 0, 400),     # three
    ("bf16", 6, 5, 1, 700, 64, 1, 300),       # eight
    ("bf16", 2, 1, 1, 200, 64, 0, 90),        # fewer row tiles than XCDs
    ("bf16", 24, 8, 8, 70, 64, 0, 1200),
    ("f32", 9, 4, 4, 130, 64, 0, 200),
    ("f32", 30, 10, 5, 9, 128, 0, 150),
    ("bf16", 40, 8, 8, 1, 128, 0, 700),       # one token or none
    ("bf16", 11, 24, 3, 33, 128, 0, 260),
    ("bf16", 140, 4, 4, 1, 64, 0, 2000)])
@pytest.mark.parametrize("causal", [False, True])
def test_sequences_with_unequal_numbers_of_queries(dtype, B, Hq, Hkv, S, d, lo, hi, causal):
    """From none to S queries a sequence, behind lo to hi older tokens: row tiles without a
    query, their order among XCDs and workgroups, runs and rounds without them."""
    print(f"case queries {dtype} B={B} Hq={Hq}/{Hkv} S={S} d={d} causal={causal}", flush=True)
    rng = random.Random(B * S)
    q_len = [rng.choice([0, 1, S // 3, S // 2, S - 1, S, S]) for _ in range(B)]
    q_len[-1] = S
    lens = [n + rng.randint(lo, hi) for n in q_len]
    q, kp, vp, table = make(B, lens, Hq, Hkv, S, d, 32, dtype)
    want = reference(q, kp, vp, table, lens, d ** -0.5, causal, q_len)
    check(q, kp, vp, table, lens, d ** -0.5, q_len=q_len, causal=causal, want=want)
    q_len = [S - n % 2 for n in range(B)]  # nearly all of them
    lens = [max(n, S) for n in lens]
    q, kp, vp, table = make(B, lens, Hq, Hkv, S, d, 64, dtype)
    want = reference(q, kp, vp, table, lens, d ** -0.5, causal, q_len)
    check(q, kp, vp, table, lens, d ** -0.5, q_len=q_len, causal=causal, want=want)


def reference(q, kp, vp, table, lens, scale, causal, q_len=None):
    """pages.paged_attention on the GPU, a sequence at a time (fp64)."""
    B, Hq, S, d = q.shape
    Hkv, page = kp.shape[1:3]
    out = [torch.full((B, Hq, S, d), float("nan"), dtype=torch.float64),
           torch.full((B, Hq, S), float("nan"), dtype=torch.float64),
           torch.full((B, Hq, S, d), float("nan"), dtype=torch.float64)]
    for b, n in enumerate(lens):
        new = S if q_len is None else q_len[b]
        ids = torch.tensor(table[b][:-(-n // page)], dtype=torch.long, device="cuda")
        k, v = (p[ids].transpose(0, 1).reshape(Hkv, -1, d)[:, :n].double().repeat_interleave(
            Hq // Hkv, 0).contiguous() for p in (kp, vp))
        x = torch.matmul(q[b, :, :new].double(), k.transpose(1, 2).contiguous()) * scale
        if causal:
            see = (torch.arange(n, device="cuda") <=
                   n - new + torch.arange(new, device="cuda")[:, None])
            x = x.masked_fill(~see, -float("inf"))
        z = x.logsumexp(-1)
        w = torch.where(z[..., None] == -float("inf"), torch.zeros_like(x), (x - z[..., None]).exp())
        out[0][b, :, :new], out[1][b, :, :new] = torch.matmul(w, v), z
        out[2][b, :, :new] = torch.matmul(w, v.abs())
    return [t.cpu().numpy() for t in out]


def test_oracles_agree():
    lens = [70, 33]
    q, kp, vp, table = make(2, lens, 4, 2, 5, 64, 16, "f32")
    for causal in (False, True):
        a = pages.paged_attention(f64(q), f64(kp), f64(vp), table, lens, 0.1, causal=causal)
        for x, y in zip(a, reference(q, kp, vp, table, lens, 0.1, causal)):
            np.testing.assert_allclose(x, y, rtol=1e-9, atol=1e-12)


def test_captured_call_follows_the_lengths():
    """A captured call replayed over grown lengths, tables and shared tokens, with eager
    calls between the replays, on two workspaces and streams."""
    B, Hq, Hkv, S, d, page = 6, 4, 2, 2, 64, 16
    lens = [100 + 7 * b for b in range(B)]
    q, kp, vp, table = make(5, [n + 60 for n in lens], Hq, Hkv, S, d, page, "bf16", [64, 32])
    t, n = torch.tensor(table, **I32), torch.tensor(lens, **I32)
    sh = torch.tensor([64, 32], **I32)
    need = sa.sa_prefix_attention_workspace(B, Hq, Hkv, S, d, torch.bfloat16, 2)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(B, Hq, S, device="cuda")

    def call(o, lse, ws):
        sa.sa_prefix_attention(q, kp, vp, t, n, 0.125, shared_len=sh, causal=True, o=o, lse=lse,
                               ws=ws)

    call(o, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, lse, ws)
    side = torch.cuda.Stream()
    for step in range(4):
        o.zero_()
        graph.replay()
        o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(o2, lse2, torch.empty(need, dtype=torch.uint8, device="cuda"))
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2), step
        check(q, kp, vp, table, n.tolist(), 0.125, shared=sh.tolist(), causal=True)
        n += 13
        sh.copy_(torch.tensor([64 - 16 * (step % 2), 32 * (step % 2)], **I32))


def test_pool_past_32_bits():
    Hkv, page, d, n_pages = 16, 128, 128, 9000  # 4.7 GB a matrix
    g = torch.Generator(device="cuda").manual_seed(3)
    kp = torch.empty(n_pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty_like(kp)
    row = [n_pages - 1, 0, n_pages - 2, 4500, n_pages - 3]
    for p in row:
        for pool in (kp, vp):
            pool[p] = torch.randn(Hkv, page, d, device="cuda", generator=g).bfloat16()
    q = torch.randn(2, Hkv, 1, d, device="cuda", generator=g).bfloat16()
    lens, table = [600, 530], [row, row]
    want = reference(q, kp, vp, table, lens, d ** -0.5, False)
    for claim in (None, [512]):
        o, lse = sa.sa_prefix_attention(
            q, kp, vp, torch.tensor(table, **I32), torch.tensor(lens, **I32), d ** -0.5,
            shared_len=None if claim is None else torch.tensor(claim, **I32), want_lse=True)
        # as in check(): |v| < 6, weights and O rounded to bf16
        assert np.abs(f64(o) - want[0]).max() <= 2.0 ** -8 * 2.02 * np.abs(want[2]).max() + 1e-4
        assert np.abs(f64(lse) - want[1]).max() <= 1e-4


def test_a_generation_chunk_by_chunk():
    """The calls together, as a program makes them: a clip read in, forked into samples,
    each grown chunk by chunk, one dropped, the cache compacted; after each step the
    attention is that over all tokens a sample has been given."""
    B, Hq, Hkv, d, page, width, n_pages, S = 5, 4, 2, 64, 16, 20, 60, 24
    g = torch.Generator(device="cuda").manual_seed(4)
    kp, vp = (torch.full((n_pages, Hkv, page, d), float("nan"), dtype=torch.bfloat16,
                         device="cuda") for _ in range(2))
    t = torch.full((B, width), -1, **I32)
    n, r = torch.zeros(B, **I32), torch.zeros(n_pages, **I32)
    have = [[torch.empty(Hkv, 0, d, device="cuda") for _ in range(2)] for _ in range(B)]

    def grow(new):
        k, v = (torch.randn(B, Hkv, S, d, device="cuda", generator=g).bfloat16() for _ in range(2))
        m = torch.tensor(new, **I32)
        assert sa.sa_pages_reserve(t, n, r, m, page).item() == 0
        sa.sa_pages_write(k, v, kp, vp, t, n, n_new=m)
        for b, c in enumerate(new):
            have[b] = [torch.cat([x, y[b, :, :c].float()], 1) for x, y in zip(have[b], (k, v))]

    def look(new, shared, causal):
        q = torch.randn(B, Hq, S, d, device="cuda", generator=g).bfloat16()
        m = torch.tensor(new, **I32)
        o, lse = sa.sa_prefix_attention(q, kp, vp, t, n, d ** -0.5, q_len=m, causal=causal,
                                        shared_len=torch.tensor([shared], **I32), want_lse=True)
        for b, c in enumerate(new):
            L = have[b][0].shape[1]
            assert n[b].item() == L
            x = torch.matmul(q[b, :, :c].double(), have[b][0].double().repeat_interleave(
                Hq // Hkv, 0).transpose(1, 2).contiguous()) * d ** -0.5
            if causal:
                see = torch.arange(L, device="cuda") <= L - c + torch.arange(
                    c, device="cuda")[:, None]
                x = x.masked_fill(~see, -float("inf"))
            v = have[b][1].double().repeat_interleave(Hq // Hkv, 0)
            w = x.softmax(-1).nan_to_num(0.0)  # a sequence without tokens
            off = (o[b, :, :c].double() - torch.matmul(w, v)).abs()
            tol = 2.0 ** -8 * 2.02 * torch.matmul(w, v.abs()) + 1e-4
            assert (off <= tol).all(), (b, off.max())
            assert (o[b, :, c:] == 0).all()

    grow([24, 0, 0, 0, 0])
    grow([17, 0, 0, 0, 0])
    look([17, 1, 0, 2, 3], 0, True)
    src, dst, _ = sa.sa_pages_fork(t, n, r, torch.tensor([0, 0, 0, 0], **I32),
                                   torch.tensor([1, 2, 3, 4], **I32), page)
    for p in (kp, vp):
        sa.sa_pages_copy(p.unsqueeze(0), src, dst)
    for b in range(1, B):
        have[b] = [x.clone() for x in have[0]]
    shared = 41 // page * page
    for new in ([24, 24, 24, 24, 24], [1, 3, 24, 7, 0], [5, 5, 5, 5, 5]):
        grow(new)
        look(new, shared, False)
        look(new, shared, True)
    sa.sa_pages_free(t, n, r, torch.tensor([2], **I32), page)
    have[2] = [x[:, :0] for x in have[2]]
    src, dst, counts = sa.sa_pages_compact(t, r)
    for p in (kp, vp):
        sa.sa_pages_copy(p.unsqueeze(0), src, dst)
    assert counts[0].item() == (r > 0).sum().item()
    for new in ([1, 1, 0, 1, 1], [24, 2, 20, 24, 1]):
        grow(new)
        look(new, shared, True)


@pytest.mark.parametrize("seed", range(48))
def test_random_calls(seed):
    """Sizes, types, groups, masks, lengths and table widths drawn together, so that every
    way of cutting a call up is met."""
    rng = random.Random(1000 + seed)
    dtype = "f32" if seed % 4 == 3 else "bf16"
    page, d = rng.choice([16, 32, 64, 128]), rng.choice([64, 128])
    Hkv, R = rng.choice([1, 2, 3, 8]), rng.choice([1, 1, 2, 5, 8])
    groups, per = rng.choice([1, 1, 2, 3]), rng.choice([1, 2, 5, 12, 33])
    S = rng.choice([1, 1, 1, 2, 4, 9, 31, 64, 150, 333])
    while groups * per * Hkv * R * S > 20000 and per > 1:
        per //= 2
    shared = [rng.choice([0, 16, 100, 512, 1500, 4200]) // page * page for _ in range(groups)]
    causal = rng.random() < 0.5
    least = S if causal and rng.random() < 0.7 else 0
    lens = [shared[b // per] + least + rng.choice([0, 1, 17, 64, 130, 700, 2100])
            for b in range(groups * per)]
    q_len = [rng.randrange(0, S + 1) for _ in lens] if rng.random() < 0.4 else None
    print(f"case random {seed}: {dtype} page={page} d={d} Hkv={Hkv} R={R} {groups}x{per} S={S} "
          f"shared={shared} causal={causal} q_len={q_len is not None}", flush=True)
    q, kp, vp, table = make(seed, lens, Hkv * R, Hkv, S, d, page, dtype, shared)
    full = reference(q, kp, vp, table, lens, d ** -0.5, causal, q_len)
    claim = rng.choice([shared, shared, [n // 2 for n in shared], None])
    o, lse = check(q, kp, vp, table, lens, d ** -0.5, shared=claim, q_len=q_len, causal=causal,
                   want=full)
    again = check(q, kp, vp, table, lens, d ** -0.5, shared=claim, q_len=q_len, causal=causal,
                  want=full)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1]), "run to run"


# row tiles whole, in runs, in rounds and runs, of groups; both forms and types
SPLITS = [("bf16", 3, 2, 1, 5, 64, None, 300, 0), ("bf16", 3, 2, 1, 5, 64, None, 300, 9000),
          ("bf16", 4, 8, 4, 60, 128, None, 700, 0), ("bf16", 4, 8, 4, 60, 128, None, 700, 9000),
          ("f32", 70, 8, 8, 2, 64, None, 150, 9000), ("bf16", 6, 4, 2, 3, 128, [128, 256], 400, 9000),
          ("bf16", 40, 4, 2, 3, 64, [512], 100, 9000), ("f32", 6, 4, 2, 3, 64, [128, 64], 400, 9000)]


def case(split, seed=0):
    """A call of SPLITS: its arguments, without outputs and workspace, and those of make."""
    dtype, B, Hq, Hkv, S, d, shared, hi, room = split
    rng = random.Random(seed)
    lens = [(shared[b * len(shared) // B] if shared else 0) + rng.randint(0, hi) for b in range(B)]
    q, kp, vp, table = make(seed, lens, Hq, Hkv, S, d, 64, dtype, shared or ())
    table = [list(r) + [-1] * (room // 64) for r in table]
    args = [q, kp, vp, torch.tensor(table, **I32), torch.tensor(lens, **I32), d ** -0.5]
    return args, dict(shared_len=None if shared is None else torch.tensor(shared, **I32)), lens, table


@pytest.mark.parametrize("split", range(len(SPLITS)))
def test_workspaces_of_any_content(split):
    """The bits that a workspace is left with, those of NaN and of large numbers too, change
    nothing; queries that are not there may be NaN."""
    print(f"case workspace {SPLITS[split]}", flush=True)
    args, kw, lens, _ = case(SPLITS[split], split)
    q = args[0]
    B, Hq, S, d = q.shape
    rng = random.Random(split)
    q_len = [rng.randint(0, S) for _ in range(B)]
    for b, n in enumerate(q_len):
        q[b, :, n:] = float("nan")
    for causal in (False, True):
        need = sa.sa_prefix_attention_workspace(B, Hq, args[1].shape[1], S, d, q.dtype,
                                                0 if kw["shared_len"] is None else
                                                kw["shared_len"].numel())
        seen = []
        for fill in (0, 0xff, 0x7f, 1):
            ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
            o, lse = torch.full_like(q, 7.0), torch.full((B, Hq, S), 7.0, device="cuda")
            sa.sa_prefix_attention(*args, **kw, q_len=torch.tensor(q_len, **I32), causal=causal,
                                   o=o, lse=lse, ws=ws)
            torch.cuda.synchronize()
            seen.append((o, lse))
        assert all(torch.isfinite(seen[0][0][b, :, :n]).all() for b, n in enumerate(q_len))
        assert all((seen[0][0][b, :, n:] == 7).all() for b, n in enumerate(q_len))
        for o, lse in seen[1:]:
            assert torch.equal(o, seen[0][0]) and torch.equal(lse, seen[0][1])


def test_calls_on_two_streams_at_once():
    """Every kind of call beside every other, each with a workspace of its own."""
    calls = [case(s, 50 + i) for i, s in enumerate(SPLITS)]
    alone = []
    for args, kw, _, _ in calls:
        alone.append(sa.sa_prefix_attention(*args, **kw, want_lse=True))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        got = [None] * len(calls)
        for i in range(len(calls)):
            k = (i * 3 + turn) % len(calls)
            with torch.cuda.stream(streams[i % 2]):
                got[k] = sa.sa_prefix_attention(*calls[k][0], **calls[k][1], want_lse=True)
        torch.cuda.synchronize()
        for (o, lse), (p, m) in zip(alone, got):
            assert torch.equal(o, p) and torch.equal(lse, m)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_of_queries_outside_their_range(dtype):
    """q_len counts as 0 below and as S above."""
    lens = [40, 41, 130, 7, 64]
    q, kp, vp, table = make(9, lens, 4, 2, 6, 64, 16, dtype)
    want = pages.paged_attention(f64(q), f64(kp), f64(vp), table, lens, 0.125, [0, 6, 3, 6, 0], True)
    o, lse = torch.full_like(q, 7.0), torch.full((5, 4, 6), 7.0, device="cuda")
    sa.sa_prefix_attention(q, kp, vp, torch.tensor(table, **I32), torch.tensor(lens, **I32), 0.125,
                           q_len=torch.tensor([-5, 13, 3, 2 ** 31 - 1, -2 ** 31], **I32),
                           causal=True, o=o, lse=lse)
    a, m = check(q, kp, vp, table, lens, 0.125, q_len=[0, 6, 3, 6, 0], causal=True, want=want)
    assert torch.equal(o, a) and torch.equal(lse, m)


@pytest.mark.parametrize("Hkv", [1, 63])
def test_as_many_sequences_and_heads_as_there_may_be(Hkv):
    B = 1024
    print(f"case most sequences Hkv={Hkv}", flush=True)
    lens = [b % 35 for b in range(B)]
    q, kp, vp, table = make(3, lens, 2 * Hkv, Hkv, 1, 64, 16, "bf16")
    want = reference(q, kp, vp, table, [max(n, 1) for n in lens], 0.125, False)
    for b, n in enumerate(lens):
        if n == 0:
            want[0][b], want[1][b], want[2][b] = 0.0, -np.inf, 0.0
    check(q, kp, vp, table, lens, 0.125, want=want)
