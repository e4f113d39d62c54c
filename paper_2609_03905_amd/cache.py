"""A paged cache of keys and values on one GPU: a relation with one block a page
of a plane (a layer's keys, then its values), and the page table's state.  This
module only holds tensors and sequences calls of ea.pages_*."""
from __future__ import annotations

import torch

from . import ea


class KVCache:
    """``pages`` pages of ``page_size`` keys of ``heads_kv`` heads in each of
    ``layers`` layers, for ``sequences`` sequences of at most ``max_pages``
    pages.  k[layer] and v[layer] are what ea.heads writes to and
    ea.attention_paged reads; table, lengths and refs are the state's device
    arrays, replaced by every select (captured calls keep the arrays they were
    given).  The first element of ``status`` says what became of the last call
    (ea.PAGES_OK, or why nothing was done), the second how many pages are free;
    it is on the device, so that asking is the caller's choice."""

    def __init__(self, layers: int, pages: int, heads_kv: int, page_size: int, d_head: int, sequences: int,
                 max_pages: int, dtype: str = "bf16", device="cuda"):
        self.page_size = page_size
        shape = (2 * layers, pages, heads_kv, page_size, d_head)
        one = [[0, heads_kv], [0, page_size], [0, d_head]]
        self.data = ea.Relation(shape, dtype, [range(2 * layers + 1), range(pages + 1)] + one, device=device)
        plane = self.data.block(pages)[2] if layers else 0  # bytes from plane to plane
        views = [self.data.view(i * plane, shape[1:], dtype, [range(pages + 1)] + one) for i in range(2 * layers)]
        self.k, self.v = views[0::2], views[1::2]
        zeros = lambda *n: torch.zeros(n, dtype=torch.int32, device=device)
        self.table, self.lengths, self.refs = zeros(sequences, max_pages), zeros(sequences), zeros(pages)
        self._other = (zeros(sequences, max_pages), zeros(sequences), zeros(pages))
        self.status = zeros(2)
        # of its own: captured calls share no workspace with another cache's
        self._workspace = ea.new_workspace(ea.pages_workspace(sequences, pages), device=device)

    def extend(self, add: torch.Tensor, tokens: int):
        """add[s] more keys for every sequence; the new tokens' slots and
        positions, sequence by sequence (``tokens`` of them)."""
        slots = torch.empty(tokens, dtype=torch.int32, device=self.table.device)
        positions = torch.empty_like(slots)
        ea.pages_extend(self.table, self.lengths, self.refs, add, page_size=self.page_size, status=self.status,
                        slots=slots, positions=positions, workspace=self._workspace)
        return slots, positions

    def select(self, parent: torch.Tensor):
        """Sequence i becomes a copy of sequence parent[i] (-1: empty)."""
        table, lengths, refs = self._other
        ea.pages_select([self.data], parent, self.table, self.lengths, self.refs, out_table=table, out_lengths=lengths,
                        out_refs=refs, status=self.status, workspace=self._workspace)
        self._other = (self.table, self.lengths, self.refs)
        self.table, self.lengths, self.refs = table, lengths, refs

    def compact(self):
        """Move the used pages to the first places."""
        ea.pages_compact([self.data], self.table, self.lengths, self.refs, status=self.status,
                         workspace=self._workspace)
