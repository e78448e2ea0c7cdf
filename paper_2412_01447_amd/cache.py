"""A layer's paged key-value cache: the buffers of the model-side calls of a verification pass.

A convenience over pld_cache_write, pld_cache_attn and pld_cache_attn_rows: it owns the
pages, the block table, the scales of a quantised cache and the attention's workspace of one
layer and batch shape.  Beside DraftStep it closes the generation loop for attention-ranked
drafting (arXiv 2412.01447, Eq. 3): the target model's layers write and attend, and after
verification `weights` renews the attention rows that the next step ranks by.
"""
import torch

from . import (PLD_ROPE_HALVES, pld_cache_attn, pld_cache_attn_rows,
               pld_cache_attn_workspace_bytes, pld_cache_write)


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
            if stream is not None and not hasattr(stream, "cuda_stream"):
                # a handle; 0, the default stream's, makes ExternalStream a new stream
                stream = (torch.cuda.ExternalStream(int(stream), device=self.k.device)
                          if int(stream) else torch.cuda.default_stream(self.k.device))
            with torch.cuda.stream(stream):      # (None: the current one)
                self.workspace = torch.empty(need, dtype=torch.uint8, device=self.k.device)

    def write(self, q, k, v, lens, q_out, draft_len=None, q_norm=None, k_norm=None, eps=1e-6,
              rope=None, rope_pairs=PLD_ROPE_HALVES, stream=None, prepare=False):
        """The rows' keys and values into their slots, the finished queries into q_out."""
        return pld_cache_write(q, k, v, self.k, self.v, self.table, lens, q_out,
                               draft_len=draft_len, k_scale=self.k_scale, v_scale=self.v_scale,
                               q_norm=q_norm, k_norm=k_norm, eps=eps, rope=rope,
                               rope_pairs=rope_pairs, stream=stream, prepare=prepare)

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
