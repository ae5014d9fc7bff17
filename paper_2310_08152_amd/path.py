"""Host-side orchestration of the hot path: buffer allocation (torch, device
memory only) and the order of C-ABI calls.  No arithmetic of the method is
done here; every step runs in libsckv.so kernels.

Typical use (one batch of sequences):
    meta  = SpanMeta(spans, L_meta, device)          # span metadata, tied positions
    cache = KVCache(M, b, H, L_cap, d, dtype, device)
    prefill_plan(...)                                 # the mask's visibility plan, once
    for m in layers: prefill_layer(..., planned=True) # rotary + masked attention
    cache.compact(meta, next_tok)                     # free closed spans in place
    for step: for m: decode_layer(...); commit(...)   # generate

A prompt too long for the cache is processed block by block instead
(prefill_progressive): each block is appended to the compacted cache,
attends to it, and the spans it closes are freed before the next block.

Beside that path:
  * models that normalise q and k by the head: a QKNorm, norm_rope_rows in the
    place of rope_rows for a prompt, norm= of prefill_progressive and
    decode_layer;
  * eviction by accumulated attention weight: cache.track_weights(), then
    prompt_weights / decode_weights_layer add to cache.w, and
    cache.evict(heavy, recent) keeps the rows that drew most of it;
  * sequences that continue a shared prefix: the prefix in a KVCache of its
    own, cache.start_behind(L) and shared_decode_layer.
"""
from __future__ import annotations

import math
from typing import List, Sequence, Tuple

import torch

from . import binding as B
from .workload import spans_to_arrays


class SpanMeta:
    """Device span metadata (vu) and tied position ids for a batch."""

    def __init__(self, spans: Sequence[Sequence[Tuple[int, int]]], L_meta: int, device,
                 stream=None):
        cl, cr, n = spans_to_arrays(list(spans))
        b, s_max = cl.shape
        self.b, self.L_meta, self.device = b, L_meta, torch.device(device)
        self.spans_dev = torch.empty(2 * b * s_max + b, dtype=torch.int32, device=device)
        self.vu = torch.empty(b, L_meta, dtype=torch.int32, device=device)
        self.pos = torch.empty(b, L_meta, dtype=torch.int32, device=device)
        B.sckv_span_meta(cl, cr, n, L_meta, self.spans_dev, self.vu, self.pos, stream=stream)


class KVCache:
    """(M, 2, b, H, L_cap, d) cache with per-sequence row bookkeeping (kv: an
    existing contiguous tensor of that shape to hold the rows)."""

    def __init__(self, M: int, b: int, H: int, L_cap: int, d: int, dtype, device, kv=None):
        self.M, self.b, self.H, self.L_cap, self.d = M, b, H, L_cap, d
        if kv is None:
            kv = torch.empty(M, 2, b, H, L_cap, d, dtype=dtype, device=device)
        elif tuple(kv.shape) != (M, 2, b, H, L_cap, d) or kv.dtype != dtype \
                or not kv.is_contiguous():
            raise ValueError(f"kv must be a contiguous {dtype} tensor of shape "
                             f"{(M, 2, b, H, L_cap, d)}")
        self.kv = kv
        self.w = self.total = None  # accumulated weights (track_weights)
        self.kv_len = torch.zeros(b, dtype=torch.int32, device=device)
        self.tok_idx = torch.zeros(b, L_cap, dtype=torch.int32, device=device)
        self.pos_ids = torch.zeros(b, L_cap, dtype=torch.int32, device=device)
        self.kept_src = torch.empty(b, L_cap, dtype=torch.int32, device=device)
        self.cur_tok = torch.zeros(b, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        # per-layer views, made once: indexing a tensor costs microseconds of
        # host time, and decode issues one call per layer per token
        self._k = [self.kv[m, 0] for m in range(M)]
        self._v = [self.kv[m, 1] for m in range(M)]

    def track_weights(self, w=None):
        """Accumulated attention weights beside the rows: w (M, b, H, L_cap)
        fp32, zeros unless given.  They then follow the rows through compact
        and evict; another prompt in the same cache starts with w.zero_()."""
        shape = (self.M, self.b, self.H, self.L_cap)
        if w is None:
            w = torch.zeros(shape, dtype=torch.float32, device=self.kv.device)
        elif tuple(w.shape) != shape or w.dtype != torch.float32 or not w.is_contiguous():
            raise ValueError(f"w must be a contiguous float32 tensor of shape {shape}")
        self.w = w
        self._w = [w[m] for m in range(self.M)]
        self.total = torch.zeros(self.b, self.L_cap, dtype=torch.float32, device=self.kv.device)

    def k(self, m: int):
        return self._k[m]

    def v(self, m: int):
        return self._v[m]

    def start_prompt(self, L: int, meta: SpanMeta):
        """Rows [0, L) hold prompt tokens 0..L-1; the next token is L."""
        pos = meta.pos
        if (pos.is_cuda and pos.device == self.kv_len.device and pos.dtype == torch.int32
                and pos.dim() == 2 and pos.is_contiguous() and pos.shape[0] == self.b
                and 0 < L <= min(self.L_cap, pos.shape[1])
                and pos.device.index == torch.cuda.current_device()):
            B.kv_start(self.kv_len, self.tok_idx, self.pos_ids, self.cur_tok, pos, pos.shape[1], L,
                       self.b, self.L_cap)
            return
        # an empty prompt, one sequence's positions for all, positions of another
        # type, layout or device, a cache on the host or on a GPU that is not the
        # current one (which a launch goes to), or sizes torch refuses
        self.tok_idx[:, :L] = torch.arange(L, dtype=torch.int32, device=self.kv.device)
        self.pos_ids[:, :L] = meta.pos[:, :L]
        self.kv_len.fill_(L)
        self.cur_tok.fill_(L)

    def compact(self, meta: SpanMeta, next_tok=None, kv_out=None, stream=None):
        nt = self.cur_tok if next_tok is None else next_tok
        B.kv_compact(self.kv, kv_out, self.M, self.b, self.H, self.L_cap, self.d, self.kv_len,
                     self.tok_idx, self.pos_ids, nt, meta.vu, meta.L_meta, self.kept_src,
                     stream=stream)
        if self.w is not None:
            B.kv_compact_weights(self.w, None, self.M, self.b, self.H, self.L_cap, self.kv_len,
                                 self.kept_src, stream=stream)

    def evict(self, heavy: int, recent: int, kv_out=None, w_out=None, stream=None):
        """Keep each sequence's `recent` last rows and, of those before them,
        the `heavy` with the largest accumulated weight (track_weights).  The
        totals that decided are left in self.total, at the old rows."""
        if self.w is None:
            raise ValueError("evict needs accumulated weights: call track_weights first")
        B.kv_evict(self.kv, kv_out, self.w, w_out, self.M, self.b, self.H, self.L_cap, self.d,
                   self.kv_len, self.tok_idx, self.pos_ids, heavy, recent, self.total,
                   self.kept_src, stream=stream)

    def start_behind(self, L: int):
        """No rows yet; every sequence's next token is L, the first behind a
        shared prefix of L tokens (which lies in a cache of its own)."""
        self.kv_len.zero_()
        self.cur_tok.fill_(L)

    def extend(self, meta: SpanMeta, tok0: int, n: int, row0, stream=None):
        """Rows for prompt tokens tok0 .. tok0+n-1 after the current rows;
        row0 (device int32 [b]) receives each sequence's first new row."""
        B.kv_extend(self.kv_len, self.tok_idx, self.pos_ids, row0, meta.pos, meta.L_meta, tok0, n,
                    self.b, self.L_cap, self.status, stream=stream)

    def commit(self, meta: SpanMeta, stream=None):
        B.kv_commit(self.kv_len, self.tok_idx, self.pos_ids, self.cur_tok, meta.vu, meta.pos,
                    meta.L_meta, self.b, self.L_cap, self.status, stream=stream)


DECODE_PARTIALS = 512  # chunk partials a decode workspace holds at least


class Workspace:
    """Device workspaces sized for a batch shape (block: the block size of
    block-wise prompt processing, if used; weights: the most queries of one
    prompt_weights call, at least 1 for decode_weights_layer, if used;
    prefixes, prefix_rows: the shared prefixes and their row capacity, if
    used)."""

    def __init__(self, b: int, H: int, L: int, L_cap: int, d: int, device, block: int = 0,
                 weights: int = 0, prefixes: int = 0, prefix_rows: int = 0):
        self.prefill = torch.empty(max(1, B.sckv_prefill_workspace_bytes(b, max(L, 1))),
                                   dtype=torch.uint8, device=device)
        # room for as many partials as a launch of few slices splits into (512
        # workgroups), which is more than the least the library accepts where
        # the cache is short
        self.decode = torch.empty(max(1, B.sckv_decode_workspace_bytes(b, H, L_cap, d),
                                      DECODE_PARTIALS * (d + 2) * 4),
                                  dtype=torch.uint8, device=device)
        self.prefill_cached = None
        if block > 0:
            self.prefill_cached = torch.empty(
                max(1, B.sckv_prefill_cached_workspace_bytes(b, block, L_cap)),
                dtype=torch.uint8, device=device)
        self.weights = self.shared = None
        if weights > 0:
            self.weights = torch.empty(
                max(B.sckv_attn_weights_workspace_bytes(b, H, weights, L_cap),
                    B.sckv_decode_weights_workspace_bytes(b, H, L_cap, d)),
                dtype=torch.uint8, device=device)
        if prefixes > 0:
            self.shared = torch.empty(
                max(1, B.sckv_shared_decode_workspace_bytes(b, H, prefixes, prefix_rows, L_cap,
                                                            d)),
                dtype=torch.uint8, device=device)


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)


def rope_rows(x, y, meta: SpanMeta, n: int, tok0: int, theta: float, stream=None):
    """Rotate rows [0, n) of every (b, h) slice of x (b, H, >=n, d) into y."""
    b, H, _, d = x.shape
    B.rope_apply(x, y, b, H, n, x.stride(1), y.stride(1), d, meta.pos, meta.L_meta, tok0, theta,
                 stream=stream)


def prefill_layer(q, k, v, o, meta: SpanMeta, ws: Workspace, L: int, scale=None, stream=None,
                  planned: bool = False):
    """Masked attention of q (b,H,L,d) over key/value slices k, v (b,H,>=L,d).
    With planned=True the visibility plan already in ws (prefill_plan) is
    used instead of being rebuilt: it is the same for every layer."""
    b, H, _, d = q.shape
    f = B.span_masked_prefill_attn_planned if planned else B.span_masked_prefill_attn
    f(q, k, v, o, b, H, L, d, q.stride(1), k.stride(1), o.stride(1),
      default_scale(d) if scale is None else scale, meta.vu, meta.L_meta, ws.prefill,
      stream=stream)


def prefill_plan(meta: SpanMeta, ws: Workspace, b: int, L: int, stream=None):
    """Visibility plan of the prompt's first L tokens, shared by all layers."""
    B.sckv_prefill_plan(meta.vu, meta.L_meta, b, L, ws.prefill, stream=stream)


class QKNorm:
    """RMS norm of each head's queries and keys: weights [d] of the cache's
    type (None: ones) and eps.  The normalised q and k of a decode step go to
    buffers kept here, made at the first step of a shape; steps that share
    this object must be ordered, as with a workspace."""

    def __init__(self, q_weight, k_weight, eps: float = 1e-6):
        self.q_weight, self.k_weight, self.eps = q_weight, k_weight, eps
        self._step = None

    def step_buffers(self, q):
        s = self._step
        if s is None or s[0].shape != q.shape or s[0].dtype != q.dtype or s[0].device != q.device:
            s = self._step = tuple(torch.empty(q.shape, dtype=q.dtype, device=q.device)
                                   for _ in range(2))
        return s


def norm_rope_rows(q, k, v, qr, k_out, v_out, norm: QKNorm, meta: SpanMeta, n: int, tok0: int,
                   theta: float, row0=None, status=None, stream=None):
    """Normalise and rotate rows [0, n) of q and k (tokens tok0..) into qr and
    k_out, and copy v into v_out; k_out and v_out are cache slices, written
    from row row0[s] on (row 0 without row0).  q, k, v: (b, H, n, d) views of
    any strides, for instance of a projection's token-major output; those of
    one stride pattern share a launch."""
    b, H, _, d = q.shape
    if not q.shape[2] == k.shape[2] == v.shape[2] == n:
        q, k, v = (t[:, :, :n] for t in (q, k, v))
    x = q.stride()
    sets = ([(q, k, v, qr, k_out, v_out)] if k.stride() == x and v.stride() == x else
            [(q, None, None, qr, None, None), (None, k, None, None, k_out, None),
             (None, None, v, None, None, v_out)])
    for xs in sets:
        x = next(t for t in xs[:3] if t is not None).stride()
        B.qk_norm_rope(*xs, norm.q_weight, norm.k_weight, norm.eps, b, H, n, x[0], x[1], x[2],
                       qr.stride(1), k_out.stride(1), k_out.shape[2], d, meta.pos, meta.L_meta,
                       tok0, None, row0, theta, status=status, stream=stream)


def norm_rope_step(q, k, q_out, k_out, norm: QKNorm, cache: KVCache, meta: SpanMeta,
                   theta: float, stream=None):
    """Normalise and rotate one token's q and k (b, H, d) a sequence, at the
    cache's current tokens."""
    b, H, d = q.shape
    B.qk_norm_rope(q, k, None, q_out, k_out, None, norm.q_weight, norm.k_weight, norm.eps, b, H, 1,
                   H * d, d, d, d, d, 1, d, meta.pos, meta.L_meta, 0, cache.cur_tok, None, theta,
                   status=cache.status, stream=stream)


def _normed(norm, q, k_new, cache, meta, theta, stream):
    """The q, k and rotary base that a decode call gets: with a norm, q and k
    are normalised and rotated ahead of it."""
    if norm is None:
        return q, k_new, theta
    qs, ks = norm.step_buffers(q)
    norm_rope_step(q, k_new, qs, ks, norm, cache, meta, theta, stream=stream)
    return qs, ks, 0.0


def decode_layer(q, k_new, v_new, cache: KVCache, m: int, meta: SpanMeta, ws: Workspace, o,
                 scale=None, theta: float = 0.0, stream=None, norm: QKNorm = None):
    d = q.shape[-1]
    if norm is not None:
        q, k_new, theta = _normed(norm, q, k_new, cache, meta, theta, stream)
    B.compacted_decode_attn(q, k_new, v_new, cache.k(m), cache.v(m), cache.kv_len, cache.cur_tok,
                            meta.vu, meta.pos, meta.L_meta, o, cache.b, cache.H, cache.L_cap, d,
                            default_scale(d) if scale is None else scale, theta, ws.decode,
                            cache.status, stream=stream)


def _sums_of(cache: KVCache, m: int):
    if cache.w is None:
        raise ValueError("no accumulated weights: call the cache's track_weights, or pass w_out")
    return cache._w[m]


def decode_weights_layer(q, k_new, v_new, cache: KVCache, m: int, meta: SpanMeta, ws: Workspace,
                         o, w_in=None, w_out=None, scale=None, theta: float = 0.0, stream=None,
                         norm: QKNorm = None):
    """decode_layer that adds the weight the step gives each row: w_out = w_in
    + weights, (b, H, L_cap) fp32, by default in place on the cache's own
    sums (track_weights)."""
    d = q.shape[-1]
    if w_out is None:
        w_in = w_out = _sums_of(cache, m)
    q, k_new, theta = _normed(norm, q, k_new, cache, meta, theta, stream)
    B.compacted_decode_attn_weights(q, k_new, v_new, cache.k(m), cache.v(m), cache.kv_len,
                                    cache.cur_tok, meta.vu, meta.pos, meta.L_meta, o, w_in, w_out,
                                    cache.b, cache.H, cache.L_cap, d,
                                    default_scale(d) if scale is None else scale, theta,
                                    ws.weights, cache.status, stream=stream)


def prompt_weights(q, cache: KVCache, m: int, meta: SpanMeta, ws: Workspace, tok0: int, w_in=None,
                   w_out=None, scale=None, stream=None):
    """Adds the weight that queries q (b, H, nq, d), tokens tok0.., give each
    row of layer m that the cache holds: w_out = w_in + weights, by default in
    place on the cache's own sums (track_weights).  q is rotated as the keys
    are; its last queries alone make a vote of recent tokens."""
    b, H, nq, d = q.shape
    if w_out is None:
        w_in = w_out = _sums_of(cache, m)
    B.cached_attn_weights(q, cache.k(m), w_in, w_out, b, H, nq, d, q.stride(1),
                          cache.k(m).stride(1), default_scale(d) if scale is None else scale,
                          meta.vu, meta.L_meta, tok0, cache.kv_len, cache.tok_idx, cache.L_cap,
                          ws.weights, stream=stream)


def shared_decode_layer(q, k_new, v_new, prefix: KVCache, cache: KVCache, m: int, meta: SpanMeta,
                        ws: Workspace, o, scale=None, theta: float = 0.0, stream=None,
                        norm: QKNorm = None):
    """decode_layer for sequences that continue shared prefixes: sequence s
    attends over the rows of prefix s // (cache.b / prefix.b), read once for
    all its sequences, and over its own rows."""
    d = q.shape[-1]
    q, k_new, theta = _normed(norm, q, k_new, cache, meta, theta, stream)
    B.shared_prefix_decode_attn(q, k_new, v_new, prefix.k(m), prefix.v(m), prefix.kv_len,
                                prefix.b, prefix.L_cap, cache.k(m), cache.v(m), cache.kv_len,
                                cache.cur_tok, meta.vu, meta.pos, meta.L_meta, o, cache.b,
                                cache.H, cache.L_cap, d,
                                default_scale(d) if scale is None else scale, theta, ws.shared,
                                cache.status, stream=stream)


def prefill_block(q, cache: KVCache, m: int, o, meta: SpanMeta, ws: Workspace, tok0: int, row0,
                  scale=None, stream=None, planned: bool = False):
    """Masked attention of a block's queries q (b,H,nq,d), tokens tok0.., over
    layer m of the cache, whose rows row0.. hold the block itself.  With
    planned=True the plan already in ws (prefill_block_plan) is used."""
    b, H, nq, d = q.shape
    f = B.span_masked_prefill_attn_cached_planned if planned else B.span_masked_prefill_attn_cached
    f(q, cache.k(m), cache.v(m), o, b, H, nq, d, q.stride(1), cache.k(m).stride(1), o.stride(1),
      default_scale(d) if scale is None else scale, meta.vu, meta.L_meta, tok0, row0,
      cache.tok_idx, cache.L_cap, ws.prefill_cached, status=cache.status, stream=stream)


def prefill_block_plan(cache: KVCache, meta: SpanMeta, ws: Workspace, tok0: int, nq: int, row0,
                       stream=None):
    """Plan of a block's masked attention over the cache, shared by all layers."""
    B.sckv_prefill_cached_plan(meta.vu, meta.L_meta, tok0, row0, cache.tok_idx, cache.L_cap,
                               cache.b, nq, ws.prefill_cached, stream=stream)


def prefill_progressive(q, k, v, o, cache: KVCache, meta: SpanMeta, ws: Workspace, L: int,
                        block: int, theta: float = 0.0, scale=None, stream=None,
                        on_block=None, norm: QKNorm = None, evict=None):
    """Process the prompt (tokens 0..L-1) in blocks of `block` tokens:
    for each block, append its rows to the compacted cache (keys rotated),
    run the masked attention of its queries over the cache for every layer,
    then free the spans closed within it (compaction at the block's end).

    q, k, v, o: (M, b, H, >= L, d) per-layer prompt tensors (o receives the
    outputs).  The cache starts empty; at the end it holds the rows a token
    after the prompt may see, exactly as a one-shot prefill + compaction
    leaves it.  on_block(B1), if given, is called after each block.

    norm: normalises q and k by the head before they are rotated.  evict =
    (heavy, recent): each block's queries add to the rows' accumulated weights
    (cache.track_weights, a workspace with weights >= block) and the rows
    beyond that budget leave after the block, so the cache needs room for
    heavy + recent + block rows and later blocks attend over what is left."""
    M, b, H, _, d = q.shape
    if evict is not None:
        if cache.w is None or ws.weights is None:
            raise ValueError("evict needs cache.track_weights() and a workspace with weights=block")
        cache.w.zero_()
    cache.kv_len.zero_()
    row0 = torch.empty(b, dtype=torch.int32, device=q.device)
    nxt = torch.empty(b, dtype=torch.int32, device=q.device)
    qr = torch.empty(b, H, block, d, dtype=q.dtype, device=q.device)
    for B0 in range(0, L, block):
        n = min(block, L - B0)
        cache.extend(meta, B0, n, row0, stream=stream)
        prefill_block_plan(cache, meta, ws, B0, n, row0, stream=stream)
        for m in range(M):
            qb, kb, vb = (x[m, :, :, B0:B0 + n] for x in (q, k, v))
            dst = cache.k(m)
            if norm is not None:
                norm_rope_rows(qb, kb, vb, qr[:, :, :n], dst, cache.v(m), norm, meta, n, B0, theta,
                               row0=row0, status=cache.status, stream=stream)
            else:
                B.rope_block(qb, kb, vb, qr, dst, cache.v(m), row0, cache.L_cap, b, H, n,
                             qb.stride(1), kb.stride(1), vb.stride(1), qr.stride(1), dst.stride(1),
                             d, meta.pos, meta.L_meta, B0, theta, status=cache.status,
                             stream=stream)
            prefill_block(qr[:, :, :n], cache, m, o[m, :, :, B0:B0 + n], meta, ws, B0, row0,
                          scale=scale, stream=stream, planned=True)
            if evict is not None:
                prompt_weights(qr[:, :, :n], cache, m, meta, ws, B0, scale=scale, stream=stream)
        nxt.fill_(B0 + n)
        cache.compact(meta, next_tok=nxt, stream=stream)
        if evict is not None:
            cache.evict(*evict, stream=stream)
        if on_block is not None:
            on_block(B0 + n)
    cache.cur_tok.fill_(L)


# ---------------------------------------------------------------------------
# local-attention comparator: a ring of the W most recent tokens
# ---------------------------------------------------------------------------

def ring_fill(x, y, W: int, L: int, meta: SpanMeta, theta: float, L_cap: int, stream=None):
    """Rotate tokens [L-W, L) of x (b, H, >=L, d) into the ring slices y
    (b, H, L_cap, d), token t at row t mod W."""
    b, H, _, d = x.shape
    t0 = L - W
    a = t0 % W
    pieces = ((t0, t0 + (W - a), a), (t0 + (W - a), L, 0))  # (first token, end, first row)
    for ts, te, r in pieces:
        if te <= ts:
            continue
        row0 = torch.full((b,), r, dtype=torch.int32, device=x.device)
        xs = x[:, :, ts:te]
        B.rope_apply_at(xs, y, row0, L_cap, b, H, te - ts, xs.stride(1), y.stride(1), d, meta.pos,
                        meta.L_meta, ts, theta, stream=stream)


def local_decode_layer(q, k_new, v_new, cache: KVCache, m: int, W: int, meta: SpanMeta,
                       ws: Workspace, o, scale=None, theta: float = 0.0, stream=None):
    """Attention of the current token over the W most recent tokens held in
    the ring rows of layer m; the new token replaces the oldest."""
    d = q.shape[-1]
    B.local_decode_attn(q, k_new, v_new, cache.k(m), cache.v(m), W, cache.cur_tok, meta.vu,
                        meta.pos, meta.L_meta, o, cache.b, cache.H, cache.L_cap, d,
                        default_scale(d) if scale is None else scale, theta, ws.decode,
                        cache.status, stream=stream)
