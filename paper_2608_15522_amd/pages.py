"""Keys and values of several sequences in pages, over the C-ABI calls.

``KVPages`` allocates the pages of every layer and the lists that describe them once
(with torch), as ``LayerPlan`` does for one layer of the sparse path; its methods enqueue
the library's kernels on the current stream and never wait for the GPU.  What may fail
for want of pages (``reserve``, ``fork``) returns how many lack, a device tensor that the
caller reads when it likes: until then a reservation that failed has changed nothing,
``write`` writes nothing, and ``new``, the tokens that the reservation brought, is 0.
"""
from __future__ import annotations

import torch

from . import binding as sa


class KVPages:
    """Pages for up to B sequences of at most max_tokens tokens, in ``layers`` layers.

    kv         [layers,2,n_pages,Hkv,page,d]: keys and values of every layer
    page_table, seq_len, page_ref: as the C calls document them
    missing, fork_missing: [1] i32, of the last reserve and of the last fork
    new        [B] i32: tokens of each sequence that the last reserve made room for (0 for
               all if it failed), to be passed on as q_len of their queries
    """

    def __init__(self, B, max_tokens, n_pages, Hkv, d, page=64, layers=1,
                 dtype=torch.bfloat16, device="cuda"):
        self.B, self.page, self.layers = B, page, layers
        e = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)
        self.kv = torch.empty(layers, 2, n_pages, Hkv, page, d, dtype=dtype, device=device)
        self.page_table = e(B, -(-max_tokens // page)).fill_(-1)
        self.seq_len, self.page_ref = e(B), e(n_pages)
        self.missing, self.fork_missing, self.new = e(1), e(1), e(B)
        self._done = torch.zeros(1, dtype=torch.bool, device=device)
        self._pools = self.kv.view(2 * layers, n_pages, Hkv, page, d)

    def reserve(self, n_new):
        """Room for n_new[b] more tokens of every sequence (all or nothing)."""
        sa.sa_pages_reserve(self.page_table, self.seq_len, self.page_ref, n_new, self.page,
                            missing=self.missing)
        torch.eq(self.missing, 0, out=self._done)
        torch.mul(n_new, self._done, out=self.new)
        return self.missing

    def write(self, layer, k, v, n_new=None):
        """Keys and values [B,Hkv,S,d] of the tokens reserved last, if they were: the first
        new[b] rows of each sequence (or n_new[b], what reserve was given).  Every layer's
        before the next fork or free."""
        sa.sa_pages_write(k, v, self.kv[layer, 0], self.kv[layer, 1], self.page_table,
                          self.seq_len, n_new=self.new if n_new is None else n_new,
                          missing=self.missing)

    def attend(self, layer, q, scale, **options):
        """sa_prefix_attention of q [B,Hq,S,d] over the layer's pages; returns (o, lse).
        q_len: new, or another number of each sequence's last tokens; ws: a workspace that
        calls one behind the other may share (sa_prefix_attention_workspace bytes, tens of
        MB; else made for each call).  The groups of shared_len are equal numbers of
        neighbouring sequences."""
        return sa.sa_prefix_attention(q, self.kv[layer, 0], self.kv[layer, 1], self.page_table,
                                      self.seq_len, scale, **options)

    def fork(self, src, dst):
        """Sequences dst (without tokens) become copies of sequences src; the pages that
        both would write are copied in every layer."""
        pairs = sa.sa_pages_fork(self.page_table, self.seq_len, self.page_ref, src, dst,
                                 self.page, missing=self.fork_missing)
        sa.sa_pages_copy(self._pools, pairs[0], pairs[1])
        return self.fork_missing

    def free(self, seqs):
        """The sequences of seqs give up their pages."""
        sa.sa_pages_free(self.page_table, self.seq_len, self.page_ref, seqs, self.page)

    def compact(self):
        """The pages in use move to the front; returns counts [2]: pages in use, moves."""
        src, dst, counts = sa.sa_pages_compact(self.page_table, self.page_ref)
        sa.sa_pages_copy(self._pools, src, dst)
        return counts
