"""Keys and values kept in pages, and the attention that reads them, as cases that can be timed.

A case is a dict of plain values.  ``prepare`` makes what a program holds before
the call, ``run`` makes one pass, in plain torch (``own`` false) or through the
library (``own`` true), ``exact`` gives the outputs in 64 bits.

Kinds of work:

* ``attend``: attention of a batch over its pages, the sequences of a group
  sharing their first pages;
* ``append``: pages reserved for the new tokens of every sequence, and the
  tokens' keys and values written into them;
* ``branch``: finished sequences freed, then others forked into their places
  (full pages shared, a partial last page copied in every pool);
* ``compact``: the pages in use moved to the front of every pool.

The pools are [n_pages, Hkv, page, d] per matrix; a page table [B, max_pages]
(int32, -1 = none), the sequences' lengths [B] and the owners of each page
[n_pages] describe them.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# What the largest listed case holds at most, in numbers: the plain form's scores
# (4 samples, 24 heads, 1560 queries, 21248 keys) and its gathered keys (those of the
# step of 64 samples).
MOST_SCORES = 3.2e9
MOST_KEYS = 1.3e9
MOST_POOL = 1.1e9


def listed():
    return [
        # The smallest step: a few samples of a short prompt, one token each; launches
        # and latency.
        {"name": "step_small", "kind": "attend", "groups": 1, "per": 4, "Hq": 8, "Hkv": 8,
         "d": 64, "page": 16, "S": 1, "shared": 256, "lo": 1, "hi": 60, "causal": False,
         "ragged": False, "dtype": "bf16"},
        # One token for each of 64 samples that continue one long prompt, four query
        # heads to a key head; the samples have come unequally far.
        {"name": "step_gqa_long", "kind": "attend", "groups": 1, "per": 64, "Hq": 32, "Hkv": 8,
         "d": 128, "page": 64, "S": 1, "shared": 16384, "lo": 1, "hi": 2000, "causal": False,
         "ragged": False, "dtype": "bf16"},
        # A guidance pair of prompts, eight samples each, up to six drafted tokens a
        # sample checked at once under the causal mask.
        {"name": "draft_pair", "kind": "attend", "groups": 2, "per": 8, "Hq": 24, "Hkv": 24,
         "d": 128, "page": 128, "S": 6, "shared": 4992, "lo": 9, "hi": 700, "causal": True,
         "ragged": True, "dtype": "bf16"},
        # The largest call: four samples of one clip, each generating a frame of the
        # 30x52 latent (1560 tokens, seen by each other) behind ten shared frames and up
        # to three of its own.
        {"name": "chunk_frame", "kind": "attend", "groups": 1, "per": 4, "Hq": 24, "Hkv": 24,
         "d": 128, "page": 128, "S": 1560, "shared": 15488, "lo": 1672, "hi": 4792,
         "causal": False, "ragged": False, "dtype": "bf16"},
        # Prompts of unequal lengths read in under the causal mask, behind a short
        # common beginning, small heads and pages.
        {"name": "prompt_causal", "kind": "attend", "groups": 2, "per": 3, "Hq": 16, "Hkv": 4,
         "d": 64, "page": 32, "S": 701, "shared": 512, "lo": 701, "hi": 1203, "causal": True,
         "ragged": True, "dtype": "bf16"},
        # fp32, the type in which a model is compared with its reference: an audio
        # chunk behind the tiny workload's 1024 tokens.
        {"name": "chunk_f32", "kind": "attend", "groups": 1, "per": 3, "Hq": 4, "Hkv": 2,
         "d": 64, "page": 64, "S": 128, "shared": 1024, "lo": 131, "hi": 517, "causal": False,
         "ragged": False, "dtype": "f32"},
        # One token more for each of 64 samples.
        {"name": "append_step", "kind": "append", "B": 64, "Hkv": 8, "d": 128, "page": 64, "S": 1,
         "lo": 100, "hi": 2500, "n_pages": 4096, "ragged": False, "dtype": "bf16"},
        # A frame's tokens for each of four samples.
        {"name": "append_frame", "kind": "append", "B": 4, "Hkv": 24, "d": 128, "page": 128,
         "S": 1560, "lo": 1672, "hi": 19000, "n_pages": 700, "ragged": False, "dtype": "bf16"},
        # Four samples of a short prompt started in the places of four finished ones.
        {"name": "branch_small", "kind": "branch", "B": 16, "n": 4, "parents": 1, "Hkv": 8,
         "d": 64, "page": 16, "pools": 4, "lo": 90, "hi": 301, "n_pages": 512, "dtype": "bf16"},
        # 48 samples of two longer prompts, the pools of three layers.
        {"name": "branch_long", "kind": "branch", "B": 50, "n": 48, "parents": 2, "Hkv": 8,
         "d": 128, "page": 64, "pools": 6, "lo": 90, "hi": 2501, "n_pages": 1200,
         "dtype": "bf16"},
        # A small cache of one layer.
        {"name": "compact_small", "kind": "compact", "B": 16, "Hkv": 8, "d": 64, "page": 16,
         "pools": 2, "lo": 1, "hi": 300, "n_pages": 600, "dtype": "bf16"},
        # Two layers' pools of a larger one, in use to half of their pages.
        {"name": "compact_large", "kind": "compact", "B": 48, "Hkv": 8, "d": 128, "page": 64,
         "pools": 4, "lo": 100, "hi": 5000, "n_pages": 4000, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "branch", "compact"])
    page = rng.choice([16, 32, 64, 128])
    d = rng.choice([64, 128])
    dtype = "bf16" if rng.random() < 0.85 else "f32"
    if kind == "attend":
        Hkv = rng.choice([1, 2, 3, 4, 8, 12, 24])
        Gq = rng.choice([1, 1, 2, 4, 8]) if Hkv <= 8 else 1
        groups, per = rng.choice([1, 1, 2, 3]), _log(rng, 1, 64)
        u = rng.random()
        S = 1 if u < 0.45 else _log(rng, 2, 16) if u < 0.7 else _log(rng, 17, 1600)
        shared = _log(rng, 1, 16384) // page * page if rng.random() < 0.9 else 0
        causal = rng.random() < 0.5
        lo = _log(rng, 1, 300)
        hi = lo + _log(rng, 1, 4000)
        if causal:  # queries are the last of a sequence's own tokens
            lo, hi = lo + S, hi + S
        elif rng.random() < 0.1:
            lo = 0  # with no prefix, a sequence without a key
        f32_cost = 8 if dtype == "f32" else 1
        while groups * per > 1 and (
                groups * per * Hkv * Gq * S * (shared + hi) * f32_cost > MOST_SCORES or
                groups * per * Hkv * (shared + hi) * d > MOST_KEYS):
            groups, per = (groups, per // 2) if per > 1 else (1, 1)
        return {"kind": kind, "groups": groups, "per": per, "Hq": Hkv * Gq, "Hkv": Hkv, "d": d,
                "page": page, "S": S, "shared": shared, "lo": lo, "hi": hi, "causal": causal,
                "ragged": S > 1 and rng.random() < 0.5, "dtype": dtype}
    Hkv = rng.choice([1, 2, 4, 8, 16, 24])
    lo = _log(rng, 1, 400)
    hi = lo + _log(rng, 1, 6000)
    row = Hkv * page * d
    B = _log(rng, 2, 64)
    if kind == "append":
        S = 1 if rng.random() < 0.5 else _log(rng, 2, 1600)
        while B > 1 and B * (-(-(hi + S) // page) + 1) * row > MOST_POOL:
            B //= 2
        n_pages = B * (-(-(hi + S) // page) + 1) + rng.randrange(1, 300)
        return {"kind": kind, "B": B, "Hkv": Hkv, "d": d, "page": page, "S": S, "lo": lo, "hi": hi,
                "n_pages": n_pages, "ragged": S > 1 and rng.random() < 0.5, "dtype": dtype}
    pools = rng.choice([1, 2, 4, 8])
    while B > 2 and B * (-(-hi // page) + 1) * row * pools > MOST_POOL:
        B //= 2
    while pools > 1 and B * (-(-hi // page) + 1) * row * pools > MOST_POOL:
        pools //= 2
    n_pages = B * (-(-hi // page) + 1) + rng.randrange(1, 300)
    case = {"kind": kind, "B": B, "Hkv": Hkv, "d": d, "page": page, "pools": pools, "lo": lo,
            "hi": hi, "n_pages": n_pages, "dtype": dtype}
    if kind == "branch":
        n = rng.randrange(1, B)
        case.update(n=n, parents=rng.randrange(1, B - n + 1))
    return case


def _spread(lo, hi, n):
    """n lengths from lo to hi, the same for every seed."""
    return [lo + (hi - lo) * i // max(n - 1, 1) for i in range(n)] if n > 1 else [hi]


def _lengths(case):
    """Tokens of each sequence before a pass (attend: with the shared ones)."""
    if case["kind"] == "attend":
        B = case["groups"] * case["per"]
        return [case["shared"] + n for n in _spread(case["lo"], case["hi"], B)]
    return _spread(case["lo"], case["hi"], case["B"])


def _new(case):
    """Tokens that each sequence brings."""
    B = case["groups"] * case["per"] if case["kind"] == "attend" else case["B"]
    return _spread(1, case["S"], B) if case["ragged"] else [case["S"]] * B


def _normal(g, dtype, *shape):
    """Standard normal values, some 2^28 of them at a time."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device=DEV))
    return out


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    order = torch.Generator().manual_seed(seed)
    dt, page, d, Hkv = DT[case["dtype"]], case["page"], case["d"], case["Hkv"]
    if case["kind"] == "attend":
        B, per, Hq, S = case["groups"] * case["per"], case["per"], case["Hq"], case["S"]
        mix = torch.randperm(B, generator=order).tolist()
        lens = [_lengths(case)[i] for i in mix]
        n_sh = case["shared"] // page
        max_pages = max(1, -(-max(lens) // page))
        n_pages = case["groups"] * n_sh + sum(-(-n // page) - n_sh for n in lens) + 1
        free = torch.randperm(n_pages, generator=order).tolist()
        table, common = [], None
        for b, n in enumerate(lens):
            if b % per == 0:
                common = [free.pop() for _ in range(n_sh)]
            row = common + [free.pop() for _ in range(-(-n // page) - n_sh)]
            table.append(row + [-1] * (max_pages - len(row)))
        return SimpleNamespace(
            kind="attend", case=case, q=_normal(g, dt, B, Hq, S, d),
            k_pages=_normal(g, dt, n_pages, Hkv, page, d),
            v_pages=_normal(g, dt, n_pages, Hkv, page, d), table=_ints(table), lens=_ints(lens),
            shared=_ints([case["shared"]] * case["groups"]),
            q_len=_ints([_new(case)[i] for i in mix]) if case["ragged"] else None,
            o=torch.zeros(B, Hq, S, d, dtype=dt, device=DEV),
            lse=torch.zeros(B, Hq, S, device=DEV), scale=d ** -0.5)
    B, n_pages = case["B"], case["n_pages"]
    mix = torch.randperm(B, generator=order).tolist()
    lens = [_lengths(case)[i] for i in mix]
    st = SimpleNamespace(kind=case["kind"], case=case)
    free = torch.randperm(n_pages, generator=order).tolist()
    more = case.get("S", 0)
    max_pages = -(-(max(lens) + more) // page) + 1
    table = []
    for n in lens:
        row = [free.pop() for _ in range(-(-n // page))]
        table.append(row + [-1] * (max_pages - len(row)))
    ref = [0] * n_pages
    for p in sum(table, []):
        if p >= 0:
            ref[p] += 1
    # table, lengths and owners lie one behind the other, so that a pass begins with one copy
    st.ints = _ints(sum(table, []) + lens + ref)
    st.sizes = (B, max_pages, n_pages)
    if case["kind"] == "append":
        st.n_new = _ints([_new(case)[i] for i in mix])
        st.k, st.v = (_normal(g, dt, B, Hkv, more, d) for _ in range(2))
        st.k_pages, st.v_pages = (_normal(g, dt, n_pages, Hkv, page, d) for _ in range(2))
        return st
    st.pools = _normal(g, dt, case["pools"], n_pages, Hkv, page, d)
    if case["kind"] == "branch":
        slots = torch.randperm(B, generator=order).tolist()
        parents = slots[case["n"]:case["n"] + case["parents"]]
        st.dst = _ints(slots[:case["n"]])
        st.src = _ints([parents[i % len(parents)] for i in range(case["n"])])
    return st


def _views(st, ints):
    B, max_pages, n_pages = st.sizes
    return (ints[:B * max_pages].view(B, max_pages), ints[B * max_pages:B * max_pages + B],
            ints[B * max_pages + B:])


# ---- the plain forms -------------------------------------------------------------------
def _plain_attend(st):
    case = st.case
    B, Hq, S, d = st.q.shape
    Hkv, page = case["Hkv"], case["page"]
    L = st.table.shape[1] * page

    def gathered(pages):
        return (pages[st.table.clamp(min=0)].transpose(1, 2).reshape(B, Hkv, L, d).float())

    j = torch.arange(L, device=DEV)
    seen = (j < st.lens[:, None])[:, None]  # [B,1,L]
    new = st.q_len if st.q_len is not None else torch.full_like(st.lens, S)
    s = torch.arange(S, device=DEV)
    if case["causal"]:
        seen = seen & (j <= ((st.lens - new)[:, None] + s)[:, :, None])
    x = st.q.float().view(B, Hkv, Hq // Hkv * S, d) @ gathered(st.k_pages).transpose(2, 3)
    x = x.view(B, Hkv, Hq // Hkv, S, L).mul_(st.scale)
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    den = p.sum(-1, keepdim=True)
    v = gathered(st.v_pages)
    v = torch.where((j < st.lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = (p.view(B, Hkv, Hq // Hkv * S, L) @ v).view(B, Hkv, Hq // Hkv, S, d)
    o = torch.where(den > 0, o / den, torch.zeros_like(o)).view(B, Hq, S, d)
    lse = (m + den.log())[..., 0].view(B, Hq, S)
    real = (s < new[:, None])[:, None]  # [B,1,S]
    return {"o": torch.where(real[..., None], o.to(st.q.dtype), st.o),
            "lse": torch.where(real, lse, st.lse)}


def _free_first(ref):
    """Page numbers, the free ones first, ascending, and how many are free."""
    return torch.argsort((ref > 0).to(torch.int8), stable=True).int(), (ref == 0).sum()


def _one_more(t):
    """t with a place behind it for what is not to be written."""
    return torch.cat([t.reshape(-1), t.new_zeros(1)])


def _plain_reserve(table, lens, ref, n_new, page, most):
    B, max_pages = table.shape
    have, want = (lens + page - 1) // page, (lens + n_new + page - 1) // page
    need = want - have
    ends = need.cumsum(0).int()
    order, n_free = _free_first(ref)
    missing = (ends[-1] - n_free).clamp(min=0) + (want - max_pages).clamp(min=0).sum()
    r = torch.arange(B * (most // page + 1), device=DEV, dtype=torch.int32)
    b = torch.searchsorted(ends, r, right=True).clamp(max=B - 1)
    go = (r < ends[-1]) & (missing == 0)
    got = order[r.clamp(max=ref.numel() - 1)]
    flat, owners = _one_more(table), _one_more(ref)
    at = b * max_pages + have[b] + r - (ends[b] - need[b])
    flat[torch.where(go, at, B * max_pages)] = got
    owners[torch.where(go, got, ref.numel()).long()] = 1
    lens = torch.where(missing == 0, lens + n_new, lens)
    return flat[:-1].view(B, max_pages), lens, owners[:-1], missing.int().view(1)


def _plain_append(st):
    page = st.case["page"]
    table, lens, ref = _views(st, st.ints)
    table, lens, ref, missing = _plain_reserve(table, lens, ref, st.n_new, page, st.case["S"])
    s = torch.arange(st.k.shape[2], device=DEV)
    bi, si = (s < st.n_new[:, None]).nonzero(as_tuple=True)
    pos = (lens - st.n_new)[bi] + si
    at = table[bi, pos // page].long()
    st.k_pages[at, :, pos % page] = st.k[bi, :, si]
    st.v_pages[at, :, pos % page] = st.v[bi, :, si]
    return {"table": table, "lens": lens, "ref": ref, "missing": missing,
            "k_pages": st.k_pages, "v_pages": st.v_pages}


def _plain_free(table, lens, ref, seqs, page):
    B, max_pages = table.shape
    gone = torch.zeros(B, dtype=torch.bool, device=DEV)
    gone[seqs.long()] = True
    j = torch.arange(max_pages, device=DEV)
    held = gone[:, None] & (j < ((lens + page - 1) // page)[:, None])
    owners = _one_more(ref)
    ids = torch.where(held, table, ref.numel()).view(-1).long()
    owners.index_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
    return (torch.where(gone[:, None], torch.full_like(table, -1), table),
            torch.where(gone, torch.zeros_like(lens), lens), owners[:-1])


def _plain_fork(table, lens, ref, src, dst, page):
    B, max_pages = table.shape
    n, n_pages = src.numel(), ref.numel()
    src, dst = src.long(), dst.long()
    able = (lens[src] > 0) & (lens[dst] == 0)
    full, part = lens[src] // page, able & (lens[src] % page > 0)
    rank = part.cumsum(0) - part.long()
    order, n_free = _free_first(ref)
    missing = (part.sum() - n_free).clamp(min=0)
    act = able & (missing == 0)
    part = part & act
    fresh = order[rank.clamp(max=n_pages - 1)]
    j = torch.arange(max_pages, device=DEV)
    whole = act[:, None] & (j < full[:, None])
    rows = torch.where(whole, table[src], torch.full_like(table[src], -1))
    rows = torch.where(part[:, None] & (j == full[:, None]), fresh[:, None], rows)
    last = table[src].gather(1, full.clamp(max=max_pages - 1).long()[:, None])[:, 0]
    none = torch.full_like(fresh, -1)
    out = torch.cat([table, table[:1]])
    out[torch.where(act, dst, B)] = rows
    lens2, owners = _one_more(lens), _one_more(ref)
    lens2[torch.where(act, dst, B)] = lens[src]
    ids = torch.where(whole, table[src], n_pages).view(-1).long()
    owners.index_add_(0, ids, torch.ones_like(ids, dtype=torch.int32))
    owners[torch.where(part, fresh, n_pages).long()] = 1
    return (out[:-1], lens2[:-1], owners[:-1], torch.where(part, last, none),
            torch.where(part, fresh, none), missing.int().view(1))


def _plain_copy(pools, src, dst):
    some = src >= 0
    pools[:, dst[some].long()] = pools[:, src[some].long()]


def _plain_branch(st):
    page = st.case["page"]
    table, lens, ref = _views(st, st.ints)
    table, lens, ref = _plain_free(table, lens, ref, st.dst, page)
    table, lens, ref, src, dst, missing = _plain_fork(table, lens, ref, st.src, st.dst, page)
    _plain_copy(st.pools, src, dst)
    return {"table": table, "lens": lens, "ref": ref, "copy_src": src, "copy_dst": dst,
            "missing": missing, "pools": st.pools}


def _plain_compact(st):
    table, lens, ref = _views(st, st.ints)
    n = ref.numel()
    p = torch.arange(n, device=DEV, dtype=torch.int32)
    used = ref > 0
    count = used.sum()
    high, hole = used & (p >= count), ~used & (p < count)
    moves = high.sum()
    k = torch.arange(n // 2, device=DEV)
    none = torch.full((n // 2,), -1, dtype=torch.int32, device=DEV)
    src = torch.where(k < moves, torch.argsort((~high).to(torch.int8), stable=True)[:n // 2].int(),
                      none)
    dst = torch.where(k < moves, torch.argsort((~hole).to(torch.int8), stable=True)[:n // 2].int(),
                      none)
    to = torch.arange(n + 1, device=DEV, dtype=torch.int32)
    to[torch.where(src >= 0, src, n).long()] = dst
    table = torch.where(table >= 0, to[table.clamp(min=0).long()], table)
    owners = _one_more(ref)
    owners[torch.where(src >= 0, dst, n).long()] = ref[src.clamp(min=0).long()]
    owners[torch.where(src >= 0, src, n).long()] = 0
    _plain_copy(st.pools, src, dst)
    return {"table": table, "ref": owners[:-1], "move_src": src, "move_dst": dst,
            "counts": torch.stack([count, moves]).int(), "pools": st.pools}


# ---- one pass --------------------------------------------------------------------------
def run(st):
    case = st.case
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "branch": _plain_branch,
                "compact": _plain_compact}[st.kind](st)
    import paper_2608_15522_amd as sa
    if st.kind == "attend":
        o, lse = sa.sa_prefix_attention(st.q, st.k_pages, st.v_pages, st.table, st.lens, st.scale,
                                        shared_len=st.shared, q_len=st.q_len,
                                        causal=case["causal"], o=st.o, lse=st.lse)
        return {"o": o, "lse": lse}
    table, lens, ref = _views(st, st.ints.clone())
    if st.kind == "append":
        missing = sa.sa_pages_reserve(table, lens, ref, st.n_new, case["page"])
        sa.sa_pages_write(st.k, st.v, st.k_pages, st.v_pages, table, lens, n_new=st.n_new)
        return {"table": table, "lens": lens, "ref": ref, "missing": missing,
                "k_pages": st.k_pages, "v_pages": st.v_pages}
    if st.kind == "branch":
        sa.sa_pages_free(table, lens, ref, st.dst, case["page"])
        src, dst, missing = sa.sa_pages_fork(table, lens, ref, st.src, st.dst, case["page"])
        sa.sa_pages_copy(st.pools, src, dst)
        return {"table": table, "lens": lens, "ref": ref, "copy_src": src, "copy_dst": dst,
                "missing": missing, "pools": st.pools}
    src, dst, counts = sa.sa_pages_compact(table, ref)
    sa.sa_pages_copy(st.pools, src, dst)
    return {"table": table, "ref": ref, "move_src": src, "move_dst": dst, "counts": counts,
            "pools": st.pools}


# ---- what a pass cannot do without -----------------------------------------------------
def work(case):
    e, page, d, Hkv = DT[case["dtype"]].itemsize, case["page"], case["d"], case["Hkv"]
    lens = _lengths(case)
    if case["kind"] == "attend":
        new, Hq = _new(case), case["Hq"]
        keys = case["groups"] * case["shared"] + sum(n - case["shared"] for n in lens)
        pairs = 0
        for n, s in zip(lens, new):
            # causal: query i of s sees n - s + i + 1 keys
            pairs += s * n - s * (s - 1) // 2 if case["causal"] else s * n
        rows = Hq * sum(new)
        return {"bytes": 2 * keys * Hkv * d * e + 2 * rows * d * e + 4 * rows,
                "flops": 4 * Hq * d * pairs}
    ints = 4 * (len(lens) + case["n_pages"])
    if case["kind"] == "append":
        return {"bytes": 4 * Hkv * sum(_new(case)) * d * e + ints, "flops": 0}
    if case["kind"] == "branch":
        # a fork of the mean length: its table row, and a partial page in every pool
        held = sum(-(-n // page) for n in lens) / len(lens)
        part = sum(n % page > 0 for n in lens) / len(lens)
        return {"bytes": case["n"] * (4 * held + 2 * part * case["pools"] * Hkv * page * d * e) +
                ints, "flops": 0}
    used = sum(-(-n // page) for n in lens)
    moves = used * (case["n_pages"] - used) / case["n_pages"]  # on the mean
    return {"bytes": 2 * moves * case["pools"] * Hkv * page * d * e + ints, "flops": 0}


# ---- the definition, in 64 bits --------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    page = case["page"]
    if case["kind"] == "attend":
        B, Hq, S, d = st.q.shape
        ratio = Hq // case["Hkv"]
        o, lse = st.o.double(), st.lse.double()
        for b in range(B):
            n = int(st.lens[b])
            new = S if st.q_len is None else int(st.q_len[b])
            if n == 0:
                o[b, :, :new], lse[b, :, :new] = 0, -math.inf
                continue
            ids = st.table[b, :-(-n // page)].long()
            at = torch.arange(n, device=DEV)
            for h in range(case["Hkv"]):
                k = st.k_pages[ids, h].reshape(-1, d)[:n].double()
                v = st.v_pages[ids, h].reshape(-1, d)[:n].double()
                q = st.q[b, h * ratio:(h + 1) * ratio, :new].double()
                x = torch.matmul(q.reshape(-1, d), k.t()).view(ratio, new, n) * st.scale
                if case["causal"]:
                    last = n - new + torch.arange(new, device=DEV)
                    x[:, at[None] > last[:, None]] = -math.inf
                z = torch.logsumexp(x, -1)
                w = torch.where(torch.isinf(z)[..., None], torch.zeros_like(x),
                                torch.exp(x - z[..., None]))
                o[b, h * ratio:(h + 1) * ratio, :new] = torch.matmul(
                    w.view(-1, n), v).view(ratio, new, d)
                lse[b, h * ratio:(h + 1) * ratio, :new] = z
        return {"o": o, "lse": lse}
    B, max_pages, n_pages = st.sizes
    ints = st.ints.tolist()
    table = [ints[b * max_pages:(b + 1) * max_pages] for b in range(B)]
    lens, ref = ints[B * max_pages:B * max_pages + B], ints[B * max_pages + B:]
    if case["kind"] == "append":
        n_new, k_pages, v_pages = st.n_new.tolist(), st.k_pages.double(), st.v_pages.double()
        p = 0
        for b in range(B):
            for i in range(-(-lens[b] // page), -(-(lens[b] + n_new[b]) // page)):
                while ref[p]:
                    p += 1
                table[b][i], ref[p] = p, 1
            s = 0
            while s < n_new[b]:
                i, r = divmod(lens[b] + s, page)
                n = min(page - r, n_new[b] - s)
                k_pages[table[b][i], :, r:r + n] = st.k[b, :, s:s + n].double()
                v_pages[table[b][i], :, r:r + n] = st.v[b, :, s:s + n].double()
                s += n
            lens[b] += n_new[b]
        return {"table": None, "lens": None, "ref": None, "missing": None, "k_pages": k_pages,
                "v_pages": v_pages}
    pools = st.pools.double()
    if case["kind"] == "branch":
        for b in st.dst.tolist():
            for p in table[b]:
                if p >= 0:
                    ref[p] -= 1
        for a in st.src.tolist():
            if lens[a] % page:
                p = ref.index(0)
                ref[p] = 1
                pools[:, p] = pools[:, table[a][lens[a] // page]]
        return {"table": None, "lens": None, "ref": None, "copy_src": None, "copy_dst": None,
                "missing": None, "pools": pools}
    used = [p for p in range(n_pages) if ref[p]]
    holes = [p for p in range(len(used)) if not ref[p]]
    for p in used:
        if p >= len(used):
            pools[:, holes.pop(0)] = pools[:, p]
    return {"table": None, "ref": None, "move_src": None, "move_dst": None, "counts": None,
            "pools": pools}
