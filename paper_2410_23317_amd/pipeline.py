"""Sequencing of the hot path over the C-ABI calls: buffers and call order only, no arithmetic.

After prefill:  vlc_score -> vlc_sparsity (finalise) -> vlc_allocate -> vlc_topk_compact; compress() takes the two
in the middle in one launch (vlc_sparsity_allocate).
Fused route for the scores: vlc_window_attn (attention of the window rows + row statistics) ->
vlc_score_from_stats (column sweep only).
Every decode step: vlc_decode_attn over a layer range of the compressed cache.
Prompts that arrive in chunks (PagedPrompt): vlc_pages_attn per chunk and layer range; after the last chunk, the window,
vlc_pages_read -> vlc_score_from_stats -> vlc_sparsity_allocate -> vlc_topk_compact.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as V


def k_min_tokens(m: int) -> int:
    """Token form of the lower clip 0.01 of the layer budget (Alg. 1)."""
    return max(1, -(-m // 100))


class VLCachePath:
    """Holds the output buffers of the compression stages and the compressed cache of one batch."""

    def __init__(self, shape: V.vlc_shape, alpha: Tuple[int, int] = (1, 10), p: float = 0.01,
                 T_max: int = 128, n_recent: int = 0, device: str = "cuda", want_idx: bool = False,
                 recent_frac: Optional[Tuple[int, int]] = None, lens: Optional[torch.Tensor] = None,
                 kv_fp8: bool = False, options: Optional[V.vlc_cache_options] = None):
        s = shape
        self.lens = lens                      # the [B, 2] tensor behind shape.lens (ragged batches), kept alive here
        self.shape, self.alpha, self.p, self.T_max, self.n_recent = s, alpha, float(p), int(T_max), int(n_recent)
        self.recent_frac = recent_frac        # (num, den): recent window = floor(k_l * num / den) per layer
        dev = torch.device(device)
        f32, i32 = torch.float32, torch.int32
        self.scores = torch.empty((s.B, s.L, s.Hkv, s.m), dtype=f32, device=dev)
        self.row_max = torch.empty((s.B, s.L, s.Hq, s.tau), dtype=f32, device=dev)
        self.row_sum = torch.empty_like(self.row_max)
        self.nnz = torch.empty((s.B, s.L, s.Hq), dtype=torch.int64, device=dev)   # uint64 counts, < 2^63
        self.gamma = torch.empty((s.B, s.L, s.Hq), dtype=f32, device=dev)
        self.k = torch.empty((s.B, s.L), dtype=i32, device=dev)
        self.beta = torch.empty((s.B, s.L), dtype=f32, device=dev)
        self.workspace = torch.empty(V.vlc_workspace_bytes(s), dtype=torch.uint8, device=dev)
        self.idx_out = torch.full((s.B, s.L, s.Hkv, s.m), -1, dtype=i32, device=dev) if want_idx else None
        b_tot = (alpha[0] * s.L * s.m) // alpha[1]
        self.sum_k_max = min(s.L * s.m, b_tot + s.L * k_min_tokens(s.m))
        if options is not None:
            options.kv_fp8 = int(bool(kv_fp8)) or options.kv_fp8
            self.cache = V.vlc_cache_create_opt(s, self.T_max, self.sum_k_max, options, device)
        else:
            self.cache = (V.vlc_cache_create_fp8 if kv_fp8 else V.vlc_cache_create)(s, self.T_max, self.sum_k_max, device)

    # -- after prefill ---------------------------------------------------------------------
    def score(self, q_win, k, sm_scale) -> None:
        V.vlc_score(self.shape, q_win, k, sm_scale, self.p, self.scores, self.row_max, self.row_sum, self.nnz,
                    self.workspace)

    def window_attn(self, q_win, k, v, sm_scale, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the window rows that also fills row_max / row_sum: with it the scores come from
        score_from_stats and the row-statistics sweep of score() is not run."""
        if out is None:
            out = torch.empty_like(q_win)
        if getattr(self, "win_workspace", None) is None:
            self.win_workspace = torch.empty(V.vlc_window_attn_workspace_bytes(self.shape), dtype=torch.uint8,
                                             device=q_win.device)
        V.vlc_window_attn(self.shape, q_win, k, v, sm_scale, out, self.row_max, self.row_sum, self.win_workspace)
        return out

    def score_from_stats(self, q_win, k, sm_scale) -> None:
        V.vlc_score_from_stats(self.shape, q_win, k, sm_scale, self.p, self.row_max, self.row_sum, self.scores, self.nnz)

    def sparsity(self) -> None:
        V.vlc_sparsity(self.shape, None, None, None, None, self.p, self.nnz, self.gamma, None)

    def allocate(self) -> None:
        V.vlc_allocate(self.shape, self.nnz, self.alpha[0], self.alpha[1], self.k, self.beta)

    def topk_compact(self, k_full, v_full, k: Optional[torch.Tensor] = None) -> None:
        kk = self.k if k is None else k
        if self.recent_frac is not None:
            V.vlc_topk_compact_recent_frac(self.cache, self.scores, kk, self.recent_frac[0], self.recent_frac[1],
                                           k_full, v_full, self.idx_out)
        else:
            V.vlc_topk_compact(self.cache, self.scores, kk, self.n_recent, k_full, v_full, self.idx_out)

    def compress(self, q_win, k, v, sm_scale) -> None:
        self.score(q_win, k, sm_scale)
        V.vlc_sparsity_allocate(self.shape, self.nnz, self.gamma, self.alpha[0], self.alpha[1], self.k, self.beta)
        self.topk_compact(k, v)

    # -- every decode step -----------------------------------------------------------------
    def decode(self, layer_begin, layer_end, q, k_new, v_new, sm_scale, out) -> None:
        V.vlc_decode_attn(self.cache, layer_begin, layer_end, q, k_new, v_new, sm_scale, out)

    def decode_steps(self, layer_begin, layer_end, n_steps, q, k_new, v_new, sm_scale, out) -> None:
        V.vlc_decode_attn_steps(self.cache, layer_begin, layer_end, n_steps, q, k_new, v_new, sm_scale, out)

    def status(self) -> None:
        V.vlc_cache_status(self.cache)

    # -- diagnostic (Def. 3.1) ----------------------------------------------------------------
    def hit_rate(self, q_next, k, sm_scale):
        """CacheHitRate of the cache against the first decode query q_next [B, L, Hq, d]:
        returns (hits [B,L,Hkv] int32, rate [B,L,Hkv] float32, scores_star [B,L,Hkv,m])."""
        s = self.shape
        if not hasattr(self, "_star"):
            lens1 = None
            if self.lens is not None:             # same prompt lengths, a one-row window for every request
                lens1 = self.lens.clone()
                lens1[:, 1] = 1
            one = V.make_shape(s.B, s.L, s.Hq, s.Hkv, s.d, s.m, 1, "f32" if s.dtype == V.VLC_F32 else "bf16", lens=lens1,
                               flags=s.flags)
            dev = self.scores.device
            self._star = dict(
                shape=one, lens=lens1, scores=torch.empty_like(self.scores),
                row_max=torch.empty((s.B, s.L, s.Hq, 1), dtype=torch.float32, device=dev),
                row_sum=torch.empty((s.B, s.L, s.Hq, 1), dtype=torch.float32, device=dev),
                workspace=torch.empty(V.vlc_workspace_bytes(one), dtype=torch.uint8, device=dev),
                hits=torch.empty((s.B, s.L, s.Hkv), dtype=torch.int32, device=dev),
                rate=torch.empty((s.B, s.L, s.Hkv), dtype=torch.float32, device=dev))
        t = self._star
        V.vlc_score(t["shape"], q_next, k, sm_scale, self.p, t["scores"], t["row_max"], t["row_sum"], None, t["workspace"])
        V.vlc_cache_hit_rate(self.cache, t["scores"], t["hits"], t["rate"])
        return t["hits"], t["rate"], t["scores"]


class PagedPrompt:
    """A batch of prompts that arrive in chunks, kept in pages until they are compressed.

    page_table [B, max_pages] names the pages of each request (int32, on the device); by default request b owns pages
    b * max_pages .. of a pool with room for max_len tokens each.  The host keeps how many tokens each request holds.
    The constructor clears the pages on the stream that is current there; a call on another stream must wait for it.  Dropping the
    object while such a stream still works on it is safe: its own tensors stay allocated until that work is done."""

    def __init__(self, L: int, Hq: int, Hkv: int, d: int, dtype, B: int, max_len: int, page_slots: int = 64, format="plain",
                 n_pages: Optional[int] = None, page_table: Optional[torch.Tensor] = None, device: str = "cuda"):
        max_pages = -(-max_len // page_slots)
        self.max_len = int(max_len)
        if page_table is None:
            if n_pages is not None and n_pages < B * max_pages:
                raise ValueError(f"{n_pages} pages are fewer than {max_pages} for each of {B} requests; name shared ones in page_table")
            page_table = torch.arange(B * max_pages, dtype=torch.int32, device=device).view(B, max_pages)
        self.table = page_table
        self.pages = V.vlc_pages_create(V.make_pages_shape(L, Hq, Hkv, d, page_slots, n_pages or B * max_pages, dtype, format), device)
        self.tokens = [0] * B
        self.device = self.pages.arena.device
        self.workspace = None
        self.chunk = None
        self.before = None                    # (tokens, chunk) that drop_chunk() goes back to

    def begin_chunk(self, new_tokens) -> V.vlc_chunk:
        """The next chunk brings new_tokens[b] tokens to request b (0: none): the lengths that extend() and the calls on
        self.chunk take from here on, and what self.tokens counts.  An extend() that is refused may be repeated; a chunk whose rows
        will not come is taken back by drop_chunk().  Copies the lengths to the device, which waits for the current stream."""
        new = [int(c) for c in new_tokens]
        if len(new) != len(self.tokens) or min(new) < 0 or max(new) < 1:
            raise ValueError("new_tokens: a count for each request, none negative and not all zero")
        total = [n + c for n, c in zip(self.tokens, new)]
        if max(total) > self.max_len:
            raise ValueError(f"a request would hold {max(total)} tokens, {self.max_len} were provided for")
        lens = torch.tensor(list(zip(total, new)), dtype=torch.int32).to(self.device)
        chunk = V.make_chunk(self.table, max(new), max(total), lens)
        chunk.new_tokens = new
        self.before = (self.tokens, self.chunk)
        self.tokens, self.chunk = total, chunk
        return self.chunk

    def drop_chunk(self) -> None:
        """Takes the last begin_chunk() back, so that the next chunk starts where that one did: positions that were counted but
        never written would be attended as if they had been.  Once for each begin_chunk()."""
        if self.before is None:
            raise ValueError("no chunk to take back")
        self.tokens, self.chunk = self.before
        self.before = None

    def _used(self, *tensors) -> None:
        """The pages, the table and these own tensors are used on the current stream, which may be another than the one they were
        made on.  Not while it is captured: the next chunk replaces lengths and workspace, and a graph would go on using the old
        ones (vlc_pages_attn takes a caller's own)."""
        if torch.cuda.is_current_stream_capturing():
            raise ValueError("PagedPrompt replaces its lengths and workspace from chunk to chunk and is not captured")
        stream = torch.cuda.current_stream(self.device)
        for t in (self.pages.arena, self.table, *tensors):
            if t is not None:
                t.record_stream(stream)

    def extend(self, layer_begin, layer_end, q, k_new, v_new, sm_scale, out, row_max=None, row_sum=None) -> None:
        """The chunk's rows of layers [layer_begin, layer_end) into the pages, and their attention."""
        if self.chunk is None:
            raise ValueError("begin_chunk() comes first")
        self._used(self.chunk.tensors[1])
        need = V.vlc_pages_attn_workspace_bytes(self.pages, self.chunk, layer_end - layer_begin)
        if need and (self.workspace is None or self.workspace.numel() < need):
            self.workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        self._used(self.workspace)
        V.vlc_pages_attn(self.pages, self.chunk, layer_begin, layer_end, q, k_new, v_new, sm_scale, out, row_max, row_sum, self.workspace)

    def read(self, k_out, v_out) -> None:
        """Every request's K and V so far, into tensors [B, L, Hkv, m, d]; rows beyond a request's are left as they are."""
        if self.chunk is None:
            raise ValueError("begin_chunk() comes first")
        if k_out.shape[3] < max(self.tokens):
            raise ValueError(f"k_out and v_out have {k_out.shape[3]} rows, a request holds {max(self.tokens)} tokens")
        self._used(self.chunk.tensors[1])
        V.vlc_pages_read(self.pages, self.chunk, 0, self.pages.shape.L, 0, k_out.transpose(0, 1), v_out.transpose(0, 1))

    def compress(self, path: VLCachePath, q_win, sm_scale, k_out, v_out) -> None:
        """Compression of the prompts whose last chunk was the window and left its statistics in path.row_max and
        path.row_sum (extend(.., row_max=path.row_max.transpose(0, 1), row_sum=..)); path.shape.lens, if the batch is
        ragged, holds what self.chunk.lens holds.  Scores of quantised pages are formed with K as the read rounds it to the storage
        type, under statistics of the codes' own values."""
        if self.chunk is None:
            raise ValueError("begin_chunk() comes first")
        s = path.shape
        for name, t, dims in (("q_win", q_win, (s.B, s.L, s.Hq, s.tau, s.d)), ("k_out", k_out, (s.B, s.L, s.Hkv, s.m, s.d)),
                              ("v_out", v_out, (s.B, s.L, s.Hkv, s.m, s.d))):
            if tuple(t.shape) != dims:
                raise ValueError(f"{name} must have the path's shape {dims}, not {tuple(t.shape)}")
        if self.chunk.max_new > s.tau:
            raise ValueError(f"the last chunk, of up to {self.chunk.max_new} tokens, is longer than the path's window of {s.tau}")
        if not s.lens and (min(self.tokens) != s.m or min(self.chunk.new_tokens) != s.tau):
            raise ValueError("requests of different lengths or windows need their pairs in path.shape.lens")
        self.read(k_out, v_out)
        path.score_from_stats(q_win, k_out, sm_scale)
        V.vlc_sparsity_allocate(path.shape, path.nnz, path.gamma, path.alpha[0], path.alpha[1], path.k, path.beta)
        path.topk_compact(k_out, v_out)

    def status(self) -> None:
        V.vlc_pages_status(self.pages)


def pages_layer_view(pages: V.Pages, l: int):
    """(K, V) of a layer as tensors [n_pages, Hkv, page_slots, d] aliasing the arena; of quantised pages the codes (uint8 for
    FP8, int8), followed by the scales [n_pages, Hkv, page_slots] of both."""
    s, lay, arena = pages.shape, pages.layout, pages.arena
    dims = (s.n_pages, s.Hkv, s.page_slots)
    rows = s.n_pages * s.Hkv * s.page_slots
    dt = {V.VLC_PAGES_PLAIN: torch.float32 if s.dtype == V.VLC_F32 else torch.bfloat16, V.VLC_PAGES_FP8: torch.uint8,
          V.VLC_PAGES_INT8: torch.int8}[s.format]
    nb = rows * s.d * dt.itemsize
    view = [arena[off + l * nb: off + (l + 1) * nb].view(dt).view(*dims, s.d) for off in (lay.k_off, lay.v_off)]
    if s.format != V.VLC_PAGES_PLAIN:
        view += [arena[off + l * rows * 4: off + (l + 1) * rows * 4].view(torch.float32).view(dims)
                 for off in (lay.k_scale_off, lay.v_scale_off)]
    return tuple(view)


def cache_layer_view(cache: V.Cache, b: int, l: int, appended: int = 0):
    """(Kc, Vc, idx) of request b, layer l as tensors [Hkv, n, d] / [Hkv, n] aliasing the arena,
    n = kept + appended.  Pure address arithmetic over the layout the library reports.  For an FP8
    cache Kc and Vc are pairs (codes uint8 [Hkv, n, d], scales float32 [Hkv, n])."""
    s, lay, arena = cache.shape, cache.layout, cache.arena
    BL = s.B * s.L
    slot_off = arena[lay.slot_off_off: lay.slot_off_off + 8 * BL].view(torch.int64)
    kept = arena[lay.kept_off: lay.kept_off + 4 * BL].view(torch.int32)
    so, kk = int(slot_off[b * s.L + l]), int(kept[b * s.L + l])
    cap, n = kk + cache.T_max, kk + appended
    ib = lay.idx_off + so * s.Hkv * 4
    idx = arena[ib: ib + s.Hkv * cap * 4].view(torch.int32).view(s.Hkv, cap)[:, :n]
    if lay.kv_fp8:
        slab = s.Hkv * cap * s.d
        kb = lay.kv_off + so * 2 * s.Hkv * s.d
        kcodes = arena[kb: kb + slab].view(s.Hkv, cap, s.d)[:, :n]
        vcodes = arena[kb + slab: kb + 2 * slab].view(s.Hkv, cap, s.d)[:, :n]
        sb = lay.scale_off + so * 2 * s.Hkv * 4
        ksc = arena[sb: sb + s.Hkv * cap * 4].view(torch.float32).view(s.Hkv, cap)[:, :n]
        vsc = arena[sb + s.Hkv * cap * 4: sb + 2 * s.Hkv * cap * 4].view(torch.float32).view(s.Hkv, cap)[:, :n]
        return (kcodes, ksc), (vcodes, vsc), idx
    dt = torch.float32 if s.dtype == V.VLC_F32 else torch.bfloat16
    es = 4 if s.dtype == V.VLC_F32 else 2
    slab = s.Hkv * cap * s.d * es
    kb = lay.kv_off + so * 2 * s.Hkv * s.d * es
    kc = arena[kb: kb + slab].view(dt).view(s.Hkv, cap, s.d)[:, :n]
    vc = arena[kb + slab: kb + 2 * slab].view(dt).view(s.Hkv, cap, s.d)[:, :n]
    return kc, vc, idx
