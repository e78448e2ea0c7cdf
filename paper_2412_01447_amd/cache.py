"""A layer's paged key-value cache: the buffers of the model-side calls of a verification pass.

A convenience over pld_cache_write, pld_cache_attn and pld_cache_attn_rows: it owns the
pages, the block table, the scales of a quantised cache and the attention's workspace of one
layer and batch shape.  Beside DraftStep it closes the generation loop for attention-ranked
drafting (arXiv 2412.01447, Eq. 3): the target model's layers write and attend, and after
verification `weights` renews the attention rows that the next step ranks by.
"""
import torch

from . import (PLD_ERR_INVALID, PLD_ROPE_HALVES, PageLayers, PageTable, PLDError, pld_cache_attn,
               pld_cache_attn_rows, pld_cache_attn_workspace_bytes, pld_cache_write, pld_cache_write_packed,
               pld_pages_compact, pld_pages_copy, pld_pages_fork, pld_pages_free, pld_pages_take,
               pld_pages_workspace_bytes)


def _under(stream, device):
    """torch.cuda.stream of a stream, its handle, or None (the current one)."""
    if stream is not None and not hasattr(stream, "cuda_stream"):
        # a handle; 0, the default stream's, makes ExternalStream a new stream
        stream = (torch.cuda.ExternalStream(int(stream), device=device)
                  if int(stream) else torch.cuda.default_stream(device))
    return torch.cuda.stream(stream)


class PagedCache:
    """Pages for B sequences of up to max_len positions each (committed tokens plus draft).
    dtype: torch.bfloat16, or torch.float8_e4m3fn with one fp32 scale per slot and head.
    `table` [B][pages] starts as sequence b's own run of pages; a caller that shares, moves or
    grows sequences writes its entries (num_pages: the pages to allocate, default B's own).
    There is one workspace: attend() calls on several streams at once need a PagedCache each,
    or pld_cache_attn with workspaces of their own."""

    def __init__(self, B, max_len, heads, head_dim, page_size=64, dtype=torch.bfloat16,
                 device="cuda", num_pages=None):
        if dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise TypeError("dtype must be bfloat16 or float8_e4m3fn")
        per = -(-max_len // page_size)
        num_pages = B * per if num_pages is None else num_pages
        self.B, self.heads, self.head_dim, self.page_size = B, heads, head_dim, page_size
        self.k, self.v = (self._pages(num_pages, dtype, device) for _ in range(2))
        self.k_scale = self.v_scale = None
        if dtype == torch.float8_e4m3fn:
            self.k_scale = torch.zeros((num_pages, heads, page_size), device=device)
            self.v_scale = torch.zeros((num_pages, heads, page_size), device=device)
        self.table = torch.arange(B * per, dtype=torch.int32, device=device).view(B, per)
        self.workspace = None
        self.grown = []                  # workspaces that a larger one has replaced

    def _pages(self, num_pages, dtype, device):
        """[pages][slots][heads][head_dim].  Rows of less than 128 bytes lie slot by slot within a
        head: a line would hold two heads' rows, and be read by two blocks (64 sequences of 16384
        tokens, 8 heads of 64 in e4m3: an attention of 337 us, 202 this way)."""
        if self.head_dim * dtype.itemsize < 128:
            return torch.zeros((num_pages, self.heads, self.page_size, self.head_dim), dtype=dtype,
                               device=device).transpose(1, 2)
        return torch.zeros((num_pages, self.page_size, self.heads, self.head_dim), dtype=dtype,
                           device=device)

    def reserve(self, n, Hq, stream=None):
        """The attention's workspace for up to n rows a sequence (grown by attend() as needed: a
        caller that captures a graph reserves before the capture).  One that is replaced is
        kept: captured graphs and prepared calls go on using it.  `stream`: the one that first
        uses it, default the current one; memory that another stream's work may still be using
        is not taken."""
        need = pld_cache_attn_workspace_bytes(self.B, n, Hq, self.heads, self.head_dim)
        if self.workspace is None or self.workspace.numel() < need:
            if self.workspace is not None:
                self.grown.append(self.workspace)
            with _under(stream, self.k.device):
                self.workspace = torch.empty(need, dtype=torch.uint8, device=self.k.device)

    def write(self, q, k, v, lens, q_out, draft_len=None, q_norm=None, k_norm=None, eps=1e-6,
              rope=None, rope_pairs=PLD_ROPE_HALVES, stream=None, prepare=False):
        """The rows' keys and values into their slots, the finished queries into q_out."""
        return pld_cache_write(q, k, v, self.k, self.v, self.table, lens, q_out,
                               draft_len=draft_len, k_scale=self.k_scale, v_scale=self.v_scale,
                               q_norm=q_norm, k_norm=k_norm, eps=eps, rope=rope,
                               rope_pairs=rope_pairs, stream=stream, prepare=prepare)

    def write_packed(self, q, k, v, starts, first, q_out, k_out=None, q_norm=None, k_norm=None, eps=1e-6,
                     rope=None, rope_pairs=PLD_ROPE_HALVES, positions=None, pair_axis=None,
                     stream=None, prepare=False):
        """The packed rows' keys and values into their slots, the finished queries (and keys, for
        pld_prompt_attn) into q_out and k_out."""
        return pld_cache_write_packed(q, k, v, self.k, self.v, self.table, starts, first, q_out,
                                      k_out=k_out, k_scale=self.k_scale, v_scale=self.v_scale,
                                      q_norm=q_norm, k_norm=k_norm, eps=eps, rope=rope,
                                      rope_pairs=rope_pairs, positions=positions,
                                      pair_axis=pair_axis, stream=stream, prepare=prepare)

    def attend(self, q, lens, out, draft_len=None, lse=None, scale=None, softcap=0.0, window=0,
               stream=None, prepare=False):
        """The rows' attention over the cache."""
        self.reserve(q.shape[1], q.shape[2], stream)
        return pld_cache_attn(q, self.k, self.v, self.table, lens, out, self.workspace,
                              draft_len=draft_len, k_scale=self.k_scale, v_scale=self.v_scale,
                              lse=lse, scale=scale, softcap=softcap, window=window, stream=stream,
                              prepare=prepare)

    def weights(self, q, lens, row, heads, lse, attn, scale=None, softcap=0.0, window=0,
                stream=None, prepare=False):
        """The chosen heads' attention weights at row row[b] (a verification's accept_len gives
        the next step's artifact) into attn [B][R][n_keys]."""
        return pld_cache_attn_rows(q, self.k, self.table, lens, row, heads, lse, attn,
                                   k_scale=self.k_scale, scale=scale, softcap=softcap,
                                   window=window, stream=stream, prepare=prepare)


class PagePool:
    """The pages of several layers' caches, shared by sequences that go on from the same prompt.

    Lists of [pages][slots][heads][D] tensors for keys and values, and of [pages][heads][slots]
    scales, one a layer (of_caches: PagedCache objects, which get the pool's table); table int32
    [seqs][pages], with -1 for entries that name no page, and refs int32 [pages], how many entries
    name a page.  Left out, both are absent: such a pool only copies.  A call has at least one entry.
    Calls on one pool follow each other (one stream, or events between): there is one workspace."""

    def __init__(self, k_caches, v_caches, k_scales=None, v_scales=None, table=None, refs=None):
        if not k_caches or (table is None) != (refs is None):
            raise TypeError("a pool has caches, and a table and references or neither")
        self.layers = PageLayers(k_caches, v_caches, k_scales, v_scales)
        self.table, self.refs = table, refs
        self.pages = None if table is None else PageTable(table, refs, k_caches[0].shape[1])
        self.workspace, self.most = None, 0
        self.grown = []                  # workspaces that a larger one has replaced

    @classmethod
    def of_caches(cls, caches, seqs=None, max_len=None):
        """A pool over PagedCache objects of the same shape, all pages free: seqs sequences of up to
        max_len positions (default: as the first cache has them)."""
        c = caches[0]
        seqs = c.table.shape[0] if seqs is None else seqs
        per = c.table.shape[1] if max_len is None else -(-max_len // c.page_size)
        table = torch.full((seqs, per), -1, dtype=torch.int32, device=c.k.device)
        refs = torch.zeros(c.k.shape[0], dtype=torch.int32, device=c.k.device)
        scales = (None, None) if c.k_scale is None else ([x.k_scale for x in caches], [x.v_scale for x in caches])
        pool = cls([x.k for x in caches], [x.v for x in caches], *scales, table=table, refs=refs)
        for x in caches:                 # (not before the pool has found them alike)
            x.table = table
        return pool

    def _paged(self):
        if self.pages is None:
            raise TypeError("the pool has no table and references: it only copies")
        return self.pages

    def reserve(self, count, stream=None):
        """The workspace for calls of up to `count` sequences or forks (grown as needed: a caller that
        captures a graph reserves before the capture).  One that is replaced is kept."""
        count = max(1, count)
        if count <= self.most:
            return
        need = pld_pages_workspace_bytes(self._paged(), count)
        if need == 0:                    # (no call takes so many)
            raise PLDError("pld_pages_workspace_bytes", PLD_ERR_INVALID)
        with _under(stream, self.refs.device):
            workspace = torch.empty(need, dtype=torch.uint8, device=self.refs.device)
        if self.workspace is not None:
            self.grown.append(self.workspace)
        self.workspace, self.most = workspace, count

    def take(self, seq, need, status, stream=None, prepare=False):
        """Pages for the positions below need[i] of sequences seq[i]."""
        self.reserve(seq.numel(), stream)
        return pld_pages_take(self._paged(), seq, need, status, self.workspace, stream=stream,
                              prepare=prepare)

    def free(self, seq, keep=None, stream=None, prepare=False):
        """Sequences seq[i] give back what lies behind their first keep[i] positions (all)."""
        return pld_pages_free(self._paged(), seq, keep, stream=stream, prepare=prepare)

    def fork(self, src, dst, lens, status, stream=None, prepare=False):
        """Sequences dst[i] go on from the first lens[i] tokens of src[i]."""
        self.reserve(src.numel(), stream)
        return pld_pages_fork(self._paged(), self.layers, src, dst, lens, status, self.workspace,
                              stream=stream, prepare=prepare)

    def compact(self, page_map, used, table_out=None, refs_out=None, stream=None, prepare=False):
        """Pages in use move to the lowest indices; page_map and used say where and how many."""
        self.reserve(1, stream)
        return pld_pages_compact(self._paged(), self.layers, page_map, used, self.workspace,
                                 table_out=table_out, refs_out=refs_out, stream=stream, prepare=prepare)

    def copy_from(self, other, src, dst, slots=None, stream=None, prepare=False):
        """Page src[i] of another pool (its first slots[i] slots) to page dst[i] of this one."""
        return pld_pages_copy(other.layers, self.layers, src, dst, slots, stream=stream, prepare=prepare)
