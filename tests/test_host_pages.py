"""Host side of the paged calls, on the CPU: what the C entry points and the binding
refuse, before any launch.  No call here reaches a kernel."""
import os

import pytest
import torch

import paper_2608_15522_amd as sa
from paper_2608_15522_amd import binding

FAKE = 0x10000           # aligned stand-in pointers, never dereferenced
FAR = 0x100000000000     # behind anything that starts at FAKE
FARTHER = 0x200000000000
FARTHEST = 0x300000000000

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH),
                                reason="libsa.so not built")


class Call:
    def __init__(self, name, **defaults):
        self.name, self.defaults = name, defaults

    def __call__(self, **kw):
        assert set(kw) <= set(self.defaults), kw
        args = {**self.defaults, **kw}
        return getattr(sa.lib(), self.name)(*args.values())


_cache = dict(B=4, max_pages=8, n_pages=32, page=16)
_reserve = Call("sa_pages_reserve", page_table=FAKE, seq_len=FAKE, page_ref=FAKE, n_new=FAKE,
                **_cache, missing=FAKE, stream=None)
_write = Call("sa_pages_write", k=FAR, v=FAR, k_pages=FAKE, v_pages=FARTHER, page_table=FAKE,
              seq_len=FAKE, n_new=None, missing=None, B=4, Hkv=2, S=3, d=64, dtype=0, n_pages=32,
              page=16, max_pages=8, stream=None)
_fork = Call("sa_pages_fork", page_table=FAKE, seq_len=FAKE, page_ref=FAKE, src=FAKE, dst=FAKE,
             n=2, **_cache, copy_src=FAKE, copy_dst=FAKE, missing=FAKE, stream=None)
_free = Call("sa_pages_free", page_table=FAKE, seq_len=FAKE, page_ref=FAKE, seqs=FAKE, n=2,
             **_cache, stream=None)
_compact = Call("sa_pages_compact", page_table=FAKE, page_ref=FAKE, B=4, max_pages=8, n_pages=32,
                move_src=FAKE, move_dst=FAKE, counts=FAKE, stream=None)
_copy = Call("sa_pages_copy", pools=FAKE, n_pools=2, n_pages=32, page_bytes=4096, src=FAKE,
             dst=FAKE, n=3, stream=None)
_attend = Call("sa_prefix_attention", q=FAR, k_pages=FAKE, v_pages=FARTHER, o=FARTHEST, lse=None,
               page_table=FAKE, seq_len=FAKE, shared_len=FAKE, q_len=None, B=4, Hq=4, Hkv=2, S=3,
               d=64, dtype=0, scale=0.125, causal=0, n_groups=2, n_pages=32, page=16, max_pages=8,
               ws=FAKE, ws_bytes=1 << 40, stream=None)

ARG, UNS, WS = sa.SA_ERR_INVALID_ARG, sa.SA_ERR_UNSUPPORTED, sa.SA_ERR_WORKSPACE
INVALID = []
for call in (_reserve, _fork, _free, _write, _attend):
    INVALID += [(call, dict(B=0), ARG, "B=0"), (call, dict(max_pages=0), ARG, "max_pages=0"),
                (call, dict(n_pages=0), ARG, "n_pages=0"), (call, dict(B=-1), ARG, "B=-1"),
                (call, dict(page=0), UNS, "page=0"), (call, dict(page=48), UNS, "page=48"),
                (call, dict(page=256), UNS, "page=256"), (call, dict(page=-16), UNS, "page=-16"),
                (call, dict(max_pages=(1 << 26) + 1), UNS, "exceed"),
                (call, dict(page_table=None), ARG, "page_table is NULL"),
                (call, dict(page_table=FAKE + 2), ARG, "page_table is not 4-byte"),
                (call, dict(seq_len=None), ARG, "seq_len is NULL")]
for call in (_reserve, _fork, _free, _write):
    INVALID += [(call, dict(B=16385), UNS, "B=16385")]
for call in (_reserve, _fork, _free, _compact):
    INVALID += [(call, dict(page_ref=None), ARG, "page_ref is NULL")]
for call in (_write, _attend):
    INVALID += [(call, dict(Hkv=0), ARG, "H=0"), (call, dict(S=0), ARG, "S=0"),
                (call, dict(S=262145), UNS, "S=262145"), (call, dict(d=96), UNS, "d=96"),
                (call, dict(dtype=2), UNS, "dtype 2"),
                (call, dict(k_pages=FAKE + 8), ARG, "k_pages is not 16-byte"),
                (call, dict(v_pages=None), ARG, "v_pages is NULL")]
INVALID += [
    (_reserve, dict(n_new=None), ARG, "n_new is NULL"),
    (_reserve, dict(missing=None), ARG, "missing is NULL"),
    (_write, dict(k=None), ARG, "k is NULL"), (_write, dict(v=FAR + 4), ARG, "v is not 16"),
    (_write, dict(v_pages=FAKE + 4096), ARG, "k_pages and v_pages overlap"),
    (_write, dict(k=FAKE + 4096), ARG, "overlaps the pages"),
    (_write, dict(missing=FAKE + 2), ARG, "missing is not 4"),
    (_write, dict(B=1, S=1, n_pages=2 ** 31 - 1, Hkv=2 ** 29, d=128, dtype=1, page=128), UNS,
     "heads are too large"),
    (_write, dict(B=16384, Hkv=4096, S=64), UNS, "too large"),
    (_fork, dict(n=0), ARG, "n=0"), (_fork, dict(n=5), ARG, "n=5"),
    (_fork, dict(src=None), ARG, "src is NULL"), (_fork, dict(dst=None), ARG, "dst is NULL"),
    (_fork, dict(copy_src=None), ARG, "copy_src"), (_fork, dict(copy_dst=FAKE + 1), ARG, "copy_dst"),
    (_fork, dict(missing=None), ARG, "missing is NULL"),
    (_free, dict(n=0), ARG, "n=0"), (_free, dict(n=16385), ARG, "n=16385"),
    (_free, dict(seqs=None), ARG, "seqs is NULL"),
    (_compact, dict(B=0), ARG, "B=0"), (_compact, dict(counts=None), ARG, "counts is NULL"),
    (_compact, dict(move_src=None), ARG, "move_src is NULL"),
    (_compact, dict(move_dst=None), ARG, "move_dst is NULL"),
    (_copy, dict(n_pools=0), ARG, "n_pools=0"), (_copy, dict(n_pages=0), ARG, "n_pages=0"),
    (_copy, dict(page_bytes=8), ARG, "page_bytes=8"), (_copy, dict(page_bytes=24), ARG, "24"),
    (_copy, dict(page_bytes=(1 << 31) + 16), ARG, "page_bytes"),
    (_copy, dict(n=-1), ARG, "n=-1"), (_copy, dict(pools=FAKE + 8), ARG, "pools is not 16"),
    (_copy, dict(src=None), ARG, "src is NULL"), (_copy, dict(dst=None), ARG, "dst is NULL"),
    (_attend, dict(Hq=3), ARG, "Hq=3"), (_attend, dict(Hq=1), ARG, "Hq=1"),
    (_attend, dict(n_groups=3), ARG, "n_groups=3"), (_attend, dict(n_groups=-1), ARG, "n_groups=-1"),
    (_attend, dict(n_groups=8), ARG, "n_groups=8"),
    (_attend, dict(n_groups=0), ARG, "shared_len"),
    (_attend, dict(shared_len=None), ARG, "shared_len"),
    (_attend, dict(B=1025), UNS, "B=1025"),
    (_attend, dict(B=1000, n_groups=100), UNS, "B + n_groups = 1100"),
    (_attend, dict(B=1000, Hq=1 << 16, S=1 << 10), UNS, "too large"),
    (_attend, dict(B=64, Hq=1024, Hkv=1024), UNS, "B*Hkv=65536"),
    (_attend, dict(B=512, Hq=64, Hkv=64, S=64, max_pages=1 << 26), UNS, "too large for one call"),
    (_attend, dict(causal=2), ARG, "causal=2"), (_attend, dict(scale=0.0), ARG, "scale"),
    (_attend, dict(scale=float("nan")), ARG, "scale"), (_attend, dict(scale=-1.0), ARG, "scale"),
    (_attend, dict(q=None), ARG, "q is NULL"), (_attend, dict(o=FARTHEST + 8), ARG, "o is not 16"),
    (_attend, dict(lse=FAKE + 2), ARG, "lse is not 4"),
    (_attend, dict(o=FAR), ARG, "o overlaps"), (_attend, dict(o=FARTHER), ARG, "o overlaps"),
    (_attend, dict(ws=None), ARG, "ws is NULL"), (_attend, dict(ws=FAKE + 8), ARG, "ws is not 16"),
    (_attend, dict(ws_bytes=0), WS, "workspace"),
    (_attend, dict(ws_bytes=-1 + 2 ** 20), WS, "workspace"),
]


@pytest.mark.parametrize("call,kw,code,needle", INVALID,
                         ids=[f"{c.name}-{'-'.join(k)}-{i}" for i, (c, k, _, _) in
                              enumerate(INVALID)])
def test_invalid_arguments_are_refused(call, kw, code, needle):
    assert call(**kw) == code
    assert call.name in sa.sa_last_error() and needle in sa.sa_last_error(), sa.sa_last_error()


def test_copy_of_nothing_launches_nothing():
    assert _copy(n=0, src=None, dst=None) == sa.SA_OK


def test_attention_workspace():
    ws = sa.sa_prefix_attention_workspace
    bf, f32 = torch.bfloat16, torch.float32
    assert ws(4, 8, 8, 1, 128, bf) > 0
    # with groups there is room for both parts' rows: d floats and (m, l) each
    more = ws(64, 32, 8, 1, 128, bf, 1) - ws(64, 32, 8, 1, 128, bf)
    assert more >= 2 * 64 * 32 * (128 * 4 + 8)
    # one sequence a group, or many queries a sequence: nothing is taken for several
    assert ws(3, 8, 8, 1, 128, bf, 3) == ws(3, 8, 8, 1, 128, bf)
    assert ws(4, 8, 8, 1560, 128, bf, 1) == ws(4, 8, 8, 1560, 128, bf)
    for bad in ((0, 8, 8, 1, 128, bf), (4, 8, 3, 1, 128, bf), (4, 8, 8, 0, 128, bf),
                (4, 8, 8, 1, 96, bf), (4, 8, 8, 1, 128, torch.float16), (4, 8, 8, 1, 128, f32, 3),
                (1025, 8, 8, 1, 128, bf), (1024, 1 << 16, 1, 1 << 10, 64, bf),
                (4, 8, 8, 1, 128, bf, -1), (4, 8, 8, 262145, 128, bf)):
        assert ws(*bad) == 0, bad


def test_binding_refuses_mismatched_tensors():
    """Shapes, types and places are checked before any pointer is taken."""
    i32 = dict(dtype=torch.int32)
    t, n, r = torch.zeros(4, 8, **i32), torch.zeros(4, **i32), torch.zeros(32, **i32)
    two = torch.zeros(2, **i32)
    kp = torch.zeros(32, 2, 16, 64, dtype=torch.bfloat16)
    kv = torch.zeros(4, 2, 3, 64, dtype=torch.bfloat16)
    q = torch.zeros(4, 4, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        sa.sa_pages_reserve(t, n, r, n, 16)
    with pytest.raises(ValueError, match="n_new"):
        sa.sa_pages_reserve(t, n, r, two, 16)
    with pytest.raises(TypeError, match="seq_len"):
        sa.sa_pages_reserve(t, n.long(), r, n, 16)
    with pytest.raises(TypeError, match="page_table"):
        sa.sa_pages_free(t.long(), n, r, two, 16)
    with pytest.raises(ValueError, match="page_table"):
        sa.sa_pages_free(t.view(-1), n, r, two, 16)
    with pytest.raises(ValueError, match="dst"):
        sa.sa_pages_fork(t, n, r, two, n, 16)
    with pytest.raises(ValueError, match="move_src"):
        sa.sa_pages_compact(t, r, move_src=two)
    with pytest.raises(ValueError, match="pools"):
        sa.sa_pages_copy(r, two, two)
    with pytest.raises(ValueError, match="v_pages"):
        sa.sa_pages_write(kv, kv, kp, kp[1:], t, n)
    with pytest.raises(TypeError, match="v"):
        sa.sa_pages_write(kv, kv.float(), kp, kp, t, n)
    with pytest.raises(ValueError, match="seq_len"):
        sa.sa_pages_write(kv[:2], kv[:2], kp, kp, t, n)
    with pytest.raises(ValueError, match="missing"):
        sa.sa_pages_write(kv, kv, kp, kp, t, n, missing=two)
    with pytest.raises(TypeError, match="k_pages"):
        sa.sa_prefix_attention(q, kp.float(), kp, t, n, 1.0)
    with pytest.raises(ValueError, match="page_table"):
        sa.sa_prefix_attention(q[:2], kp, kp, t, n, 1.0)
    with pytest.raises(ValueError, match="q_len"):
        sa.sa_prefix_attention(q, kp, kp, t, n, 1.0, q_len=two)
    with pytest.raises(TypeError, match="shared_len"):
        sa.sa_prefix_attention(q, kp, kp, t, n, 1.0, shared_len=two.float())
    with pytest.raises(ValueError, match="k_pages"):
        sa.sa_prefix_attention(q, kp.view(32, 2, 8, 128), kp, t, n, 1.0)
