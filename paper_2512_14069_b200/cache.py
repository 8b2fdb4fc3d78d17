"""Paged KV caches for the requests of a batch, in 4 bits (`FourBitCache`) and in whole bf16 or fp32 numbers (`PagedCache`): the pool of all layers,
block tables, lengths and the stack of free pages.

They own the device buffers and issue the library's calls on the current stream; nothing returns to the host, so that a
decoding loop over them can be captured in a CUDA graph.  They contain no arithmetic but that of positions.  A request is a row of the block table:

    cache.admit(new_len, K, V)          # prompts (0 for the other requests) and their rows of all layers
    step.attention_cached(cache, layer, Q, Kt, Vt)      # or cache.attention for other rows than a step's tree
    cache.append(step, K, V)            # behind step.accept: the root and the accepted nodes, from the tree's rows
    cache.release(finished)             # their pages go back onto the stack

and, with a `PagedCache`, whose prompts attend over it chunk by chunk and layer by layer:

    cache.begin(new_len, n)             # room for a chunk of each request's prompt, or for a token: n rows
    cache.store(layer, K, V, Q=Q, Q_out=Q, inv_freq=f)  # the layer's rows, turned by their positions on the way
    cache.attention(layer, Q, O)        # each row over what its request has stored up to it
    step.attention_paged(cache, layer, Q, Kt, Vt)       # a step's tree, its Q and Kt turned by `radar_rotate`
    cache.append(step, K, V); cache.release(finished)

`live` says which rows hold a request: from an admission that was granted until its release.  Only those take what a step accepted.
"""
from __future__ import annotations

import torch

from . import binding as rb


class _Requests:
    """Block tables, lengths and the stack of free pages."""

    def __init__(self, ctx: rb.Context, n_layers, B, Hq, Hkv, d, page_size, n_pages, max_len, max_new, device):
        self.ctx = ctx
        self.n_layers, self.B, self.Hq, self.Hkv, self.d, self.page_size = n_layers, B, Hq, Hkv, d, page_size
        self.max_len = -(-max_len // page_size) * page_size              # what the table has room for, which is what is granted
        dev, i32 = torch.device(device), torch.int32
        self.block_table = torch.full((B, self.max_len // page_size), -1, dtype=i32, device=dev)
        self.cache_len, self.start = torch.zeros(B, dtype=i32, device=dev), torch.zeros(B + 1, dtype=i32, device=dev)
        self.granted, self.live = torch.zeros(B, dtype=torch.uint8, device=dev), torch.zeros(B, dtype=torch.bool, device=dev)
        self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=i32, device=dev)           # taken from the top: page 0 first
        self.free_count = torch.full((1,), n_pages, dtype=i32, device=dev)
        self.slots, self.src_row = torch.full((max_new,), -1, dtype=torch.int64, device=dev), torch.zeros(max_new, dtype=i32, device=dev)

    def _workspace(self, n):
        ws = torch.zeros(n + 255, dtype=torch.uint8, device=self.slots.device)
        off = (-ws.data_ptr()) % 256
        self.workspace = ws[off:off + n]

    def _extend(self, new_len, extra=0, n=None, path_nodes=None, rows=0):
        """Slots of the added tokens: n of them, or (n None) the whole buffer; those that no token takes are -1."""
        slots, src_row = self.slots[:n], self.src_row[:n]
        rb.radar_cache_extend(self.ctx, page_size=self.page_size, cache_len=self.cache_len, new_len=new_len, extra=extra, block_table=self.block_table,
                              free_pages=self.free_pages, free_count=self.free_count, slots=slots, start=self.start, granted=self.granted,
                              path_nodes=path_nodes, rows=rows, src_row=None if path_nodes is None else src_row)
        return slots, None if path_nodes is None else src_row

    def _added(self, new_len, n, requests):
        """Slots of n new rows, and the requests that hold them marked as live."""
        if n > self.slots.numel():
            raise ValueError(f"{n} tokens, the cache was made for {self.slots.numel()} in a call")
        slots, _ = self._extend(new_len, n=n)
        self.live |= ((new_len > 0) if requests is None else (requests != 0)) & (self.granted != 0)
        return slots

    def _accepted(self, step, rows):
        """Slots and rows of what a step accepted."""
        n = step.path_nodes.numel()
        if n > self.slots.numel():
            raise ValueError(f"a step may accept {n} tokens, the cache was made for {self.slots.numel()} in a call")
        return self._extend(torch.where(self.live, step.accept_len, -1), extra=1, n=n, path_nodes=step.path_nodes, rows=rows)

    def release(self, finished):
        """Gives up the tokens of the requests with finished[b] != 0 ([B] on the GPU)."""
        self._extend(torch.where(finished != 0, -self.cache_len, 0).to(torch.int32))
        self.live &= finished == 0


class FourBitCache(_Requests):
    def __init__(self, ctx: rb.Context, *, n_layers, B, Hq, Hkv, d, page_size, n_pages, max_len, max_new, rows=rb.RADAR_MAX_NODES, device="cuda:0"):
        """Pool of n_pages pages of page_size tokens in each layer; requests of up to max_len tokens (and to the end of their last
        page); max_new: added tokens of all requests in one call (B * (t_max + 1) for a step's); rows: query rows of a sequence, at
        most."""
        super().__init__(ctx, n_layers, B, Hq, Hkv, d, page_size, n_pages, max_len, max_new, device)
        self.pages = torch.zeros((n_layers, n_pages, rb.radar_cache_page_bytes(Hkv, d, page_size)), dtype=torch.uint8, device=torch.device(device))
        self._workspace(rb.radar_cache_attn_workspace_bytes(ctx, B, Hq, Hkv, d, rows, self.max_len))

    def admit(self, new_len, K, V, requests=None):
        """New tokens of the requests: new_len [B] int32 on the GPU, K and V [layers, sum of new_len, Hkv, d], the requests' rows one
        behind the other; more rows than that are left out.  Requests that the pool had no pages for, or the table no room, are left as
        they are; `granted` says which.  requests [B] on the GPU names those that are admitted (not 0) where one of them has no
        tokens to cache yet; without it they are those with new_len > 0."""
        slots = self._added(new_len, K.shape[1], requests)
        rb.radar_cache_store(self.ctx, K=K, V=V, slots=slots, pages=self.pages, page_size=self.page_size)

    def append(self, step, K, V):
        """What a step accepted: the root and step.path_nodes, from the tree's rows of all layers, [layers, B, rows, Hkv, d].  Rows that
        hold no request take nothing; a request that the pool had no pages for keeps its length (`granted`), and takes the step again
        when there are some."""
        slots, src_row = self._accepted(step, K.shape[2])
        rb.radar_cache_store(self.ctx, K=K.flatten(1, 2), V=V.flatten(1, 2), slots=slots, src_row=src_row, pages=self.pages, page_size=self.page_size)

    def attention(self, layer, Q, Kt, Vt, O, lse=None, mask=None, n_nodes=None, scale=0.0, max_cache_len=None):
        """radar_cache_attention over one layer's pool: Q [B, rows, Hq, d], Kt and Vt [B, rows, Hkv, d], the rows' own keys and values.
        max_cache_len: a bound of the lengths, if the caller has a nearer one than the cache's capacity; the form that takes the
        call goes by it (one request of 2048 tokens in a cache for 32768, 32 / 8 heads of 128, one row: 14.4 us, with its length as the
        bound 6.8; 64 rows over 300 tokens 22 and 10)."""
        rb.radar_cache_attention(self.ctx, Q=Q, Kt=Kt, Vt=Vt, pages=self.pages[layer], page_size=self.page_size, block_table=self.block_table,
                                 cache_len=self.cache_len, max_cache_len=self.max_len if max_cache_len is None else max_cache_len, O=O, lse=lse, mask=mask, n_nodes=n_nodes,
                                 workspace=self.workspace, scale=scale)

    def load(self, first, start, K, V):
        """Tokens first[b] .. of each request as rows start[b] .. start[b + 1] - 1 of K and V, [layers, rows, Hkv, d]; those below
        cache_len[b] are the request's."""
        rb.radar_cache_load(self.ctx, pages=self.pages, page_size=self.page_size, block_table=self.block_table, first=first, start=start, K=K, V=V)


class PagedCache(_Requests):
    def __init__(self, ctx: rb.Context, *, n_layers, B, Hq, Hkv, d, page_size, n_pages, max_len, max_new, dtype=torch.bfloat16, device="cuda:0"):
        """Kc and Vc [layers, n_pages * page_size, Hkv, d] of bfloat16 or float32; the other arguments as for `FourBitCache`, max_new being
        also the rows of all requests in a chunk."""
        super().__init__(ctx, n_layers, B, Hq, Hkv, d, page_size, n_pages, max_len, max_new, device)
        self.Kc, self.Vc = (torch.zeros((n_layers, n_pages * page_size, Hkv, d), dtype=dtype, device=torch.device(device)) for _ in range(2))
        self.pos, self.n = torch.zeros(max_new, dtype=torch.int32, device=self.slots.device), None        # (n None: there is no chunk)
        self._row = torch.arange(max_new, dtype=torch.int32, device=self.slots.device)
        self._workspace(rb.radar_chunk_attn_workspace_bytes(ctx, B, Hq, Hkv, d, rb.dtype_code(self.Kc), max_new, self.max_len))

    def begin(self, new_len, n, requests=None):
        """Room for a chunk: new_len [B] int32 on the GPU, new tokens of each request, n their sum (or more: rows behind the last one are
        left out).  Behind it `slots`, `pos` (the rows' positions) and `start` (the requests' first rows) are the chunk's.  Requests that
        the pool had no pages for, or the table no room, are left as they are, as `granted` says; their rows reach no cache and their
        attention's output says nothing.  requests as in `FourBitCache.admit`.

        `append` and `release` share out slots and pages anew, and with them the chunk is over: `store` and `attention` refuse to run
        until the next `begin`.  (Parts of a round that are captured as graphs of their own have to be captured, and replayed, in such an order.)"""
        self._added(new_len, n, requests)
        self.n = n
        b = torch.searchsorted(self.start[1:], self._row[:n], right=True).clamp_(max=self.B - 1)
        torch.add(self.cache_len[b] - self.start[1:][b], self._row[:n], out=self.pos[:n])

    def _chunk(self):
        if self.n is None:
            raise ValueError("there is no chunk: begin makes room for one, and append and release end it")

    def store(self, layer, K, V, *, Q=None, Q_out=None, pos=None, **rotation):
        """The chunk's rows of a layer, K and V [n, Hkv, d], into their slots.  With inv_freq (and pair_axis, neighbours, as in
        `radar_rotate`) keys and queries are turned by their positions, `pos` or those given [axes, n]; Q [n, Hq, d] into Q_out."""
        self._chunk()
        if rotation.get("inv_freq") is not None:
            rotation["pos"] = self.pos[:self.n] if pos is None else pos
        elif pos is not None or rotation.get("pair_axis") is not None or rotation.get("neighbours"):
            raise ValueError("pos, pair_axis and neighbours: expected inv_freq beside them")
        rb.radar_paged_store(self.ctx, K=K, V=V, slots=self.slots[:self.n], Kc=self.Kc[layer], Vc=self.Vc[layer], Q=Q, Q_out=Q_out, **rotation)

    def attention(self, layer, Q, O, lse=None, *, max_new=None, max_cache_len=None, scale=0.0):
        """radar_chunk_attention of the chunk's rows, Q [n, Hq, d], over one layer's pool, where `store` has put their keys and values.  max_new,
        max_cache_len: bounds of a request's rows and tokens, if the caller has nearer ones than the chunk's and the cache's: the
        form that takes the call goes by them (single tokens want max_new = 1)."""
        self._chunk()
        rb.radar_chunk_attention(self.ctx, Q=Q, q_start=self.start, Kc=self.Kc[layer], Vc=self.Vc[layer], page_size=self.page_size, block_table=self.block_table,
                                 cache_len=self.cache_len, max_new=self.n if max_new is None else max_new,
                                 max_cache_len=self.max_len if max_cache_len is None else max_cache_len, O=O, lse=lse, workspace=self.workspace, scale=scale)

    def append(self, step, K, V):
        """What a step accepted, as `FourBitCache.append`; the keys as they were verified, turned already."""
        slots, src_row = self._accepted(step, K.shape[2])
        self.n = None
        rb.radar_paged_store(self.ctx, K=K.flatten(1, 2), V=V.flatten(1, 2), slots=slots, src_row=src_row, Kc=self.Kc, Vc=self.Vc)

    def release(self, finished):
        super().release(finished)
        self.n = None
