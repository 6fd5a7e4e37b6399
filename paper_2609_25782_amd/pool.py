"""A pool object over the C ABI: torch supplies device memory and streams,
every operation is a call into the HIP library."""

from __future__ import annotations

import contextlib
from typing import Optional, Sequence

import torch

from . import hotcold_kv as kv

_DTYPES = {"bf16": (kv.KV_DTYPE_BF16, torch.bfloat16), "f32": (kv.KV_DTYPE_F32, torch.float32)}


_HERE = contextlib.nullcontext()


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    # the current stream's handle without building a Stream object (2.7 us, of a
    # decode call's 15 us on the host)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


class HotColdPool:
    """Hot and cold page pools plus the pool's page table, all caller-owned torch
    tensors, bound to one library pool handle."""

    def __init__(self, num_layers: int, num_kv_heads: int, head_dim: int, dtype: str,
                 num_hot_pages: int, num_cold_pages: int, max_sessions: int,
                 max_pages_per_session: int, device: int = 0, cold_location: str = "device",
                 stream: Optional[torch.cuda.Stream] = None):
        kdtype, self.torch_dtype = _DTYPES[dtype]
        self.dtype = dtype
        self.device = torch.device("cuda", device)
        self.desc = kv.kv_pool_desc(num_layers, num_kv_heads, head_dim, kv.KV_PAGE_TOKENS, kdtype,
                                    num_hot_pages, num_cold_pages,
                                    kv.KV_COLD_PINNED_HOST if cold_location == "host" else kv.KV_COLD_DEVICE,
                                    max_sessions, max_pages_per_session, device, 0)
        self.page_bytes = kv.kv_page_bytes(self.desc)
        if self.page_bytes == 0:
            raise ValueError("invalid pool shape")
        self.num_layers, self.num_kv_heads, self.head_dim = num_layers, num_kv_heads, head_dim
        self.num_hot_pages, self.num_cold_pages = num_hot_pages, num_cold_pages
        self.max_sessions, self.stride = max_sessions, max_pages_per_session
        self.hot = torch.empty(max(num_hot_pages, 1) * self.page_bytes, dtype=torch.uint8,
                               device=self.device)
        if cold_location == "host":
            self.cold = torch.empty(max(num_cold_pages, 1) * self.page_bytes, dtype=torch.uint8,
                                    pin_memory=True)
        else:
            self.cold = torch.empty(max(num_cold_pages, 1) * self.page_bytes, dtype=torch.uint8,
                                    device=self.device)
        self.page_table = torch.empty((max_sessions, max_pages_per_session), dtype=torch.int32,
                                      device=self.device)
        self.handle = kv.kv_pool_create(self.desc, self.hot.data_ptr(), self.hot.numel(),
                                        self.cold.data_ptr(), self.cold.numel(),
                                        self.page_table.data_ptr(), _stream(stream))
        self._ws = {}   # decode workspace per stream: decodes on different streams may overlap
        self.bounds = None   # key bounds of the pages (set_bounds)

    # -- layout ------------------------------------------------------------
    @property
    def slice_bytes(self) -> int:
        """Bytes of one layer of one page: [kv_head][K tile, V tile]."""
        return self.page_bytes // self.num_layers

    def hot_pages(self) -> torch.Tensor:
        """The hot pool as [num_hot_pages][num_layers][slice_bytes], a view in page
        order.  The hot pool is layer-major: the slice of page p for layer l sits at
        byte (l * num_hot_pages + p) * slice_bytes."""
        return self.hot.view(self.num_layers, max(self.num_hot_pages, 1), self.slice_bytes).transpose(0, 1)

    def hot_page_bytes(self, ids=None) -> torch.Tensor:
        """Hot pages (all, or the ids given) as [n][page_bytes] in the cold pool's
        page-major order (a copy): what the same pages hold, byte for byte, once
        copied to the cold tier."""
        v = self.hot_pages()
        if ids is not None:
            v = v[torch.as_tensor(ids, dtype=torch.long, device=self.device).reshape(-1)]
        return v.reshape(v.shape[0], self.page_bytes)

    # -- lifetime ----------------------------------------------------------
    def close(self) -> None:
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            kv.kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- sessions ----------------------------------------------------------
    def create_session(self, seq_len: int, hot_pages: Optional[Sequence[int]] = None, stream=None) -> int:
        return kv.kv_session_create(self.handle, int(seq_len), hot_pages, _stream(stream))

    def import_cold(self, seq_len: int, cold_pages: Sequence[int]) -> int:
        return kv.kv_session_import_cold(self.handle, int(seq_len), cold_pages)

    def extend(self, sid: int, new_seq_len: int, stream=None) -> None:
        kv.kv_session_extend(self.handle, sid, int(new_seq_len), _stream(stream))

    def reserve(self, sid: int, kept: int, new_seq_len: int, stream=None) -> None:
        """Tokens [kept, new_seq_len) become the session's last ones, to be written by accept_drafts or
        append_tokens_table; `kept` is how many it really holds (rejected drafts forgotten), or fewer."""
        kv.kv_session_reserve(self.handle, sid, int(kept), int(new_seq_len), _stream(stream))

    def pause(self, sid: int) -> None:
        kv.kv_session_pause(self.handle, sid)

    def evict_pages(self, n: int, stream=None) -> int:
        return kv.kv_evict_pages(self.handle, int(n), _stream(stream))

    def fork(self, sids, kept=None, stream=None):
        """Branches: the id of a new session with the first kept[i] tokens of session sids[i] (the same
        may stand several times) for each i, or of one for plain numbers; `kept` None: their lengths, which
        after `reserve` count room as well: give the number of tokens then, or `reserve` the branch from it."""
        one = isinstance(sids, int)
        sids = [sids] if one else [int(x) for x in sids]
        if kept is None:
            kept = [kv.kv_session_info(self.handle, sid)[1] for sid in sids]
        kept = [int(kept)] * len(sids) if isinstance(kept, int) else [int(x) for x in kept]
        made = kv.kv_fork_sessions(self.handle, sids, kept, self._raw(stream))
        return made[0] if one else made

    def destroy_session(self, sid: int, stream=None) -> None:
        kv.kv_session_destroy(self.handle, sid, _stream(stream))

    def info(self, sid: int):
        return kv.kv_session_info(self.handle, sid)

    def write_tokens(self, sid: int, layer: int, tok_begin: int, k: torch.Tensor, v: torch.Tensor,
                     stream=None) -> None:
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape
        assert k.dtype == self.torch_dtype and k.device == self.device
        kv.kv_write_tokens(self.handle, sid, layer, tok_begin, k.shape[0], k.data_ptr(), v.data_ptr(),
                           _stream(stream))

    def append_tokens(self, layer: int, sids, positions, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """One token per row: row i of k and v is token positions[i] of session sids[i]."""
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape and k.shape[0] == len(sids)
        assert k.dtype == self.torch_dtype and k.device == self.device
        kv.kv_append_tokens(self.handle, layer, sids, positions, k.data_ptr(), v.data_ptr(), _stream(stream))

    def write_tokens_layers(self, sid: int, layer_begin: int, tok_begin: int, k: torch.Tensor, v: torch.Tensor,
                            stream=None) -> None:
        """k and v [num_layers][n_tok][kv_heads][head_dim]: tokens of layers layer_begin.. in one launch."""
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape and k.dim() == 4
        assert k.dtype == self.torch_dtype and k.device == self.device
        kv.kv_write_tokens_layers(self.handle, sid, layer_begin, k.shape[0], tok_begin, k.shape[1], k.data_ptr(),
                                  v.data_ptr(), _stream(stream))

    def append_tokens_table(self, layer_begin: int, table: torch.Tensor, rows: torch.Tensor, positions: torch.Tensor,
                            k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """Device-resolved append: entry i is token positions[i] of table row rows[i]; k and v
        [num_layers][n][kv_heads][head_dim].  Capturable in a HIP graph."""
        assert table.dtype == torch.int32 and table.is_contiguous() and table.dim() == 2
        assert rows.dtype == positions.dtype == torch.int32 and rows.shape == positions.shape
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape and k.dim() == 4
        assert k.shape[1] == rows.shape[0] and k.dtype == self.torch_dtype
        kv.kv_append_tokens_table(self.handle, layer_begin, k.shape[0], table.data_ptr(), table.shape[1],
                                  table.shape[0], rows.data_ptr(), positions.data_ptr(), rows.shape[0],
                                  k.data_ptr(), v.data_ptr(), _stream(stream))

    def fill_synthetic(self, sid: int, gen_sid: int, seed: int, value_mult: float, stream=None) -> None:
        kv.kv_fill_synthetic(self.handle, sid, gen_sid, seed, float(value_mult), _stream(stream))

    def fill_synthetic_pages(self, sid: int, gen_sid: int, seed: int, value_mult: float,
                             first_page: int, num_pages: int, stream=None) -> None:
        kv.kv_fill_synthetic_pages(self.handle, sid, gen_sid, seed, float(value_mult), int(first_page),
                                   int(num_pages), _stream(stream))

    def evict(self, sids, stream=None) -> None:
        if isinstance(sids, int):
            kv.kv_evict_session(self.handle, sids, _stream(stream))
        else:
            kv.kv_evict_sessions(self.handle, list(sids), _stream(stream))

    def resume(self, sids, stream=None) -> None:
        if isinstance(sids, int):
            kv.kv_resume_session(self.handle, sids, _stream(stream))
        else:
            kv.kv_resume_sessions(self.handle, list(sids), _stream(stream))

    def resume_lazy(self, sids, stream=None) -> None:
        kv.kv_resume_sessions_lazy(self.handle, [sids] if isinstance(sids, int) else list(sids),
                                   _stream(stream))

    def set_spill(self, enable: bool) -> None:
        kv.kv_pool_set_spill(self.handle, enable)

    def promote(self, n: int, stream=None) -> int:
        return kv.kv_promote_pages(self.handle, int(n), _stream(stream))

    def set_copy_blocks(self, blocks: int) -> None:
        kv.kv_pool_set_copy_blocks(self.handle, int(blocks))

    def stats(self) -> dict:
        return kv.kv_pool_stats(self.handle)

    # -- decode ------------------------------------------------------------
    def workspace(self, batch: int, num_q_heads: int, stream=None) -> torch.Tensor:
        """The decode workspace of `stream` (one per stream: separate-merge decodes
        on different streams run concurrently and must not share partials)."""
        return self._workspace(batch, num_q_heads, _stream(stream), stream)

    def _workspace(self, batch: int, num_q_heads: int, key: int, stream) -> torch.Tensor:
        need = kv.paged_decode_workspace_bytes(self.handle, batch, num_q_heads)
        ws = self._ws.get(key)
        if ws is None or ws.numel() < need:
            # allocated on that stream, so torch reuses a dropped buffer only in its order
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
                ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            self._ws[key] = ws
        return ws

    def decode(self, layer: int, q: torch.Tensor, seq_lens: torch.Tensor,
               page_table: Optional[torch.Tensor] = None, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, stream=None, k_new: Optional[torch.Tensor] = None,
               v_new: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Decode attention of one layer; with k_new / v_new ([B][kv_heads][head_dim]) each
        row's token seq_lens[b] - 1 is appended first, in the same launch."""
        pt = self.page_table if page_table is None else page_table
        assert q.is_contiguous() and q.dtype == self.torch_dtype and q.dim() == 3
        assert pt.dtype == torch.int32 and pt.is_contiguous() and seq_lens.dtype == torch.int32
        B, Hq, D = q.shape
        if out is None:
            out = torch.empty_like(q)
        st = _stream(stream)
        ws = self._workspace(B, Hq, st, stream)
        s = float(scale if scale is not None else D ** -0.5)
        if k_new is None:
            kv.paged_decode_attention(self.handle, layer, q.data_ptr(), pt.data_ptr(), pt.shape[1],
                                      seq_lens.data_ptr(), B, Hq, s, out.data_ptr(), ws.data_ptr(), ws.numel(), st)
        else:
            assert k_new.is_contiguous() and v_new.is_contiguous() and k_new.shape == v_new.shape
            assert k_new.shape == (B, self.num_kv_heads, D) and k_new.dtype == self.torch_dtype
            kv.paged_decode_attention_append(self.handle, layer, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
                                             pt.data_ptr(), pt.shape[1], seq_lens.data_ptr(), B, Hq, s,
                                             out.data_ptr(), ws.data_ptr(), ws.numel(), st)
        return out

    # -- several new tokens per session --------------------------------------
    def _raw(self, stream) -> int:
        """Raw handle of `stream`, or of the pool device's current stream."""
        if stream is not None:
            return int(stream.cuda_stream)
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    def _capturing(self, stream) -> bool:
        """Whether the call's stream, which need not be the current one, is being captured."""
        if stream is None and torch.cuda.current_device() == self.device.index:
            return torch.cuda.is_current_stream_capturing()
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
            return torch.cuda.is_current_stream_capturing()

    def _on(self, stream):
        """The stream whose memory the call takes, as a context.  Entering one costs 6 us on the host, so a
        call on the current stream of the current device enters none."""
        if stream is None and torch.cuda.current_device() == self.device.index:
            return _HERE
        return torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device))

    def _memory(self, need, like: Optional[torch.Tensor], stream):
        """An output like `like` and, where `need` is not 0, bytes of workspace, both of the call's
        stream: torch hands out memory that another stream may still be using otherwise."""
        with self._on(stream):
            return (None if like is None else torch.empty_like(like),
                    torch.empty(need, dtype=torch.uint8, device=self.device) if need else None)

    def _chunk_buffers(self, need: int, q: torch.Tensor, out: Optional[torch.Tensor], st: int, stream):
        """(out, workspace) of a prompt or tree call.  A captured call's workspace is memory of its
        graph's own pool, so that no two graphs share one; other calls keep one per stream."""
        if out is not None:
            assert out.is_contiguous() and out.shape == q.shape and out.dtype == q.dtype and out.device == q.device
        if self._capturing(stream):
            new, ws = self._memory(need, q if out is None else None, stream)
            return (new if out is None else out), ws
        ws = self._ws.get(("chunk", st))
        if out is None or ws is None or ws.numel() < need:
            new, more = self._memory(0 if ws is not None and ws.numel() >= need else need,
                                     q if out is None else None, stream)
            if out is None:
                out = new
            if more is not None:
                ws = self._ws[("chunk", st)] = more
        return out, ws

    def _table(self, page_table, batch: int) -> torch.Tensor:
        if page_table is None:
            page_table = self.page_table
        assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.dim() == 2
        assert page_table.device == self.device
        assert page_table.shape[0] >= batch, "the page table has fewer rows than the batch"
        return page_table

    def _ints(self, t: torch.Tensor, *shape) -> int:
        assert t.dtype == torch.int32 and t.is_contiguous() and t.device == self.device
        assert t.shape == shape, "int32 %s expected, got %s" % (shape, tuple(t.shape))
        return t.data_ptr()

    def prefill(self, layer: int, q: torch.Tensor, q_starts: torch.Tensor, seq_lens: torch.Tensor,
                page_table: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Causal attention of packed prompt chunks: queries q_starts[b] .. q_starts[b + 1] of q
        ([total][Hq][head_dim]) are the last tokens of row b's seq_lens[b], whose K and V are in
        its pages.  Queries of no row keep what `out` holds (without `out`: anything)."""
        assert q.is_contiguous() and q.dtype == self.torch_dtype and q.dim() == 3 and q.device == self.device
        B, (total, Hq, D) = seq_lens.shape[0], q.shape
        assert D == self.head_dim
        pt = self._table(page_table, B)
        lens, starts = self._ints(seq_lens, B), self._ints(q_starts, B + 1)
        st = self._raw(stream)
        out, ws = self._chunk_buffers(kv.paged_prefill_workspace_bytes(self.handle, B, total, Hq), q, out, st, stream)
        kv.paged_prefill_attention(self.handle, layer, q.data_ptr(), starts, total, pt.data_ptr(), pt.shape[1],
                                   lens, B, Hq, float(scale if scale is not None else D ** -0.5), out.data_ptr(),
                                   ws.data_ptr() if ws is not None else 0, ws.numel() if ws is not None else 0, st)
        return out

    def tree_decode(self, layer: int, q: torch.Tensor, k_draft: torch.Tensor, v_draft: torch.Tensor,
                    masks: torch.Tensor, seq_lens: torch.Tensor, draft_lens: Optional[torch.Tensor] = None,
                    page_table: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                    out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of drafted tokens: q [B][width][Hq][head_dim], k_draft and v_draft
        [B][width][kv_heads][head_dim]; draft i of row b sees the row's seq_lens[b] cached tokens
        and the drafts whose bits are set in masks[b][i] (int64 or uint64).  Drafts at or past
        draft_lens[b] keep what `out` holds (without `out`: anything)."""
        assert q.is_contiguous() and q.dtype == self.torch_dtype and q.dim() == 4 and q.device == self.device
        B, T, Hq, D = q.shape
        assert D == self.head_dim
        for t in (k_draft, v_draft):
            assert t.is_contiguous() and t.shape == (B, T, self.num_kv_heads, D) and t.dtype == q.dtype
            assert t.device == self.device
        assert masks.dtype in (torch.int64, torch.uint64) and masks.is_contiguous() and masks.shape == (B, T)
        assert masks.device == self.device
        pt = self._table(page_table, B)
        lens = self._ints(seq_lens, B)
        drafts = 0 if draft_lens is None else self._ints(draft_lens, B)
        st = self._raw(stream)
        out, ws = self._chunk_buffers(kv.paged_tree_workspace_bytes(self.handle, B, T, Hq), q, out, st, stream)
        kv.paged_tree_attention(self.handle, layer, q.data_ptr(), k_draft.data_ptr(), v_draft.data_ptr(),
                                masks.data_ptr(), drafts, T, pt.data_ptr(), pt.shape[1], lens, B, Hq,
                                float(scale if scale is not None else D ** -0.5), out.data_ptr(),
                                ws.data_ptr() if ws is not None else 0, ws.numel() if ws is not None else 0, st)
        return out

    def accept_drafts(self, layer_begin: int, table: torch.Tensor, seq_lens: torch.Tensor, path: torch.Tensor,
                      counts: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """Token seq_lens[b] + j of table row b gets draft path[b][j], j < counts[b], of k and v
        ([num_layers][B][width][kv_heads][head_dim]).  Capturable in a HIP graph."""
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape and k.dim() == 5
        assert k.dtype == v.dtype == self.torch_dtype and k.device == v.device == self.device
        L, B, T, heads, D = k.shape
        assert heads == self.num_kv_heads and D == self.head_dim
        pt = self._table(table, B)
        kv.kv_accept_drafts(self.handle, layer_begin, L, pt.data_ptr(), pt.shape[1], self._ints(seq_lens, B),
                            self._ints(path, B, T), self._ints(counts, B), B, T, k.data_ptr(), v.data_ptr(),
                            self._raw(stream))

    # -- decode over picked pages ---------------------------------------------
    def set_bounds(self, enable: bool) -> None:
        """Keep key bounds of every page (kv_bounds_bytes of device memory, zeros at first), or none.  A graph
        that holds calls captured before is not to be replayed after it: the memory it names is released."""
        torch.cuda.synchronize(self.device)
        bounds = None
        if enable:
            bounds = torch.zeros(kv.kv_bounds_bytes(self.desc), dtype=torch.uint8, device=self.device)
            torch.cuda.synchronize(self.device)
        kv.kv_pool_set_bounds(self.handle, bounds.data_ptr() if enable else 0, bounds.numel() if enable else 0)
        self.bounds = bounds

    def update_bounds(self, layer_begin: int, num_layers: int, seq_lens: torch.Tensor,
                      starts: Optional[torch.Tensor] = None, page_table: Optional[torch.Tensor] = None,
                      stream=None) -> None:
        """Bounds of the pages that hold tokens starts[b] (default 0) .. seq_lens[b] of table row b: after
        writing those tokens, before picking pages.  Capturable in a HIP graph."""
        B = seq_lens.shape[0]
        pt = self._table(page_table, B)
        kv.kv_update_bounds(self.handle, layer_begin, num_layers, pt.data_ptr(), pt.shape[1],
                            0 if starts is None else self._ints(starts, B), self._ints(seq_lens, B), B,
                            self._raw(stream))

    def key_bounds(self, layer_begin: int, num_layers: int, pages: torch.Tensor, stream=None) -> torch.Tensor:
        """Bounds of the pages (int32 page-table entries [n]) as float32 [num_layers][n][kv_heads][2][head_dim]:
        the lowest and the highest value of each dim, rounded outwards to 8 bits."""
        n = pages.shape[0]
        with self._on(stream):
            out = torch.empty((num_layers, n, self.num_kv_heads, 2, self.head_dim), dtype=torch.float32,
                              device=self.device)
        kv.kv_read_bounds(self.handle, layer_begin, num_layers, self._ints(pages, n), n, out.data_ptr(),
                          self._raw(stream))
        return out

    def _scratch(self, kind: str, need: int, st: int, stream) -> torch.Tensor:
        """Workspace of a call: its graph's own memory under capture, else one per kind and stream."""
        if self._capturing(stream):
            return self._memory(need, None, stream)[1]
        ws = self._ws.get((kind, st))
        if ws is None or ws.numel() < need:
            ws = self._ws[(kind, st)] = self._memory(need, None, stream)[1]
        return ws

    def select_pages(self, layer: int, q: torch.Tensor, seq_lens: torch.Tensor, width: int, first: int = 1,
                     recent: int = 2, page_table: Optional[torch.Tensor] = None, stream=None):
        """(picks int32 [B][kv_heads][width], counts int32 [B][kv_heads]): for each row and KV head its first
        and last pages and those whose bounds allow the largest scores with q [B][Hq][head_dim]."""
        assert q.is_contiguous() and q.dtype == self.torch_dtype and q.dim() == 3 and q.device == self.device
        B, Hq, D = q.shape
        assert D == self.head_dim
        pt = self._table(page_table, B)
        lens = self._ints(seq_lens, B)
        st = self._raw(stream)
        ws = self._scratch("select", kv.paged_select_workspace_bytes(self.handle, B, pt.shape[1], width), st, stream)
        with self._on(stream):
            picks = torch.empty((B, self.num_kv_heads, width), dtype=torch.int32, device=self.device)
            counts = torch.empty((B, self.num_kv_heads), dtype=torch.int32, device=self.device)
        kv.paged_select_pages(self.handle, layer, q.data_ptr(), pt.data_ptr(), pt.shape[1], lens, B, Hq, width, first,
                              recent, picks.data_ptr(), counts.data_ptr(), ws.data_ptr() if ws is not None else 0,
                              ws.numel() if ws is not None else 0, st)
        return picks, counts

    def sparse_decode(self, layer: int, q: torch.Tensor, seq_lens: torch.Tensor, picks: torch.Tensor,
                      counts: Optional[torch.Tensor] = None, page_table: Optional[torch.Tensor] = None,
                      scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Decode attention of one layer over the listed pages of every row and KV head alone (picks
        [B][kv_heads][width] of select_pages or of any other rule, counts None: width each)."""
        assert q.is_contiguous() and q.dtype == self.torch_dtype and q.dim() == 3 and q.device == self.device
        B, Hq, D = q.shape
        assert D == self.head_dim and picks.dim() == 3
        width = picks.shape[2]
        listed = self._ints(picks, B, self.num_kv_heads, width)
        pt = self._table(page_table, B)
        lens = self._ints(seq_lens, B)
        st = self._raw(stream)
        if out is None:
            out = self._memory(0, q, stream)[0]
        assert out.is_contiguous() and out.shape == q.shape and out.dtype == q.dtype and out.device == q.device
        ws = self._scratch("sparse", kv.paged_sparse_workspace_bytes(self.handle, B, Hq, width), st, stream)
        kv.paged_sparse_attention(self.handle, layer, q.data_ptr(), pt.data_ptr(), pt.shape[1], lens, listed,
                                  0 if counts is None else self._ints(counts, B, self.num_kv_heads), width, B, Hq,
                                  float(scale if scale is not None else D ** -0.5), out.data_ptr(),
                                  ws.data_ptr() if ws is not None else 0, ws.numel() if ws is not None else 0, st)
        return out

    def gather_table(self, sids: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Page-table rows of the given sessions (device int32 ids), for decoding them as a batch."""
        assert sids.dtype == torch.int32 and sids.is_contiguous() and sids.device == self.device
        n = sids.shape[0]
        if out is None:
            out = torch.empty((n, self.stride), dtype=torch.int32, device=self.device)
        assert out.shape[0] >= n and out.shape[1] == self.stride and out.is_contiguous()
        kv.paged_decode_gather_table(self.handle, sids.data_ptr(), n, out.data_ptr(), _stream(stream))
        return out

    def partition(self, seq_lens: torch.Tensor, waves: int, stream=None) -> torch.Tensor:
        B = seq_lens.shape[0]
        slots = torch.empty((waves + B * self.num_kv_heads, 4), dtype=torch.int32, device=self.device)
        kv.paged_decode_partition(self.handle, seq_lens.data_ptr(), B, waves, slots.data_ptr(),
                                  _stream(stream))
        return slots

    def waves(self) -> int:
        return kv.paged_decode_waves(self.handle)

    def set_waves(self, waves: int) -> None:
        kv.kv_pool_set_decode_waves(self.handle, waves)

    def set_combine(self, fused: bool) -> None:
        kv.kv_pool_set_decode_combine(self.handle, kv.KV_COMBINE_FUSED if fused else kv.KV_COMBINE_SEPARATE)

    def set_host_copy(self, kernel: bool) -> None:
        kv.kv_pool_set_host_copy(self.handle, kv.KV_HOST_COPY_KERNEL if kernel else kv.KV_HOST_COPY_DMA)

    def set_compute(self, vector: bool) -> None:
        kv.kv_pool_set_decode_compute(self.handle, kv.KV_DECODE_VECTOR if vector else kv.KV_DECODE_MATRIX)


class CUStream:
    """A torch stream whose kernels run only on CU slots [begin, end) of every
    XCD (one slot = one CU per XCD).  The library creates the HIP stream; close()
    waits for the device and destroys it."""

    def __init__(self, begin: int, end: int, device: int = 0):
        xcds, _ = kv.kv_device_cu_slots(device)
        self.device = torch.device("cuda", device)
        self.handle = kv.kv_stream_create_cu_slots(device, begin, end)
        self.stream = torch.cuda.ExternalStream(self.handle, device=self.device)
        self.cus = xcds * (end - begin)

    def close(self) -> None:
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            kv.kv_stream_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def split_streams(copy_slots: int, device: int = 0):
    """A decode stream and a copy stream on disjoint CUs: the copy stream gets
    `copy_slots` CUs of every XCD, the decode stream the rest."""
    _, slots = kv.kv_device_cu_slots(device)
    if not 0 < copy_slots < slots:
        raise ValueError("copy_slots must be in [1, %d)" % slots)
    return CUStream(copy_slots, slots, device), CUStream(0, copy_slots, device)
