"""A compressed KV cache for one attention layer: buffers plus the two calls.

torch allocates the device buffers; encoding and attention are the library's
kernels.  Records are stored [batch][kv_heads][t_cap][C] so that the address of
a token's record follows from its index (App. A).
"""

from __future__ import annotations

import torch

from . import _lib


class KVCache:
    def __init__(self, batch: int, kv_heads: int, q_heads: int, t_cap: int, k_tables, v_tables,
                 device="cuda"):
        if t_cap % _lib.DQ_MEAN_WINDOW:
            raise ValueError("t_cap must be a multiple of 128")
        d = k_tables.head_dim
        self.batch, self.kv_heads, self.q_heads, self.t_cap, self.head_dim = batch, kv_heads, q_heads, t_cap, d
        self.k_tables, self.v_tables = k_tables, v_tables
        nw = t_cap // _lib.DQ_MEAN_WINDOW
        self.k_records = torch.zeros((batch, kv_heads, t_cap, k_tables.record_bytes), dtype=torch.uint8, device=device)
        self.v_records = torch.zeros((batch, kv_heads, t_cap, v_tables.record_bytes), dtype=torch.uint8, device=device)
        self.k_mean_q = torch.zeros((batch, kv_heads, nw, d), dtype=torch.int8, device=device)
        self.k_mean_scale = torch.zeros((batch, kv_heads, nw), dtype=torch.int16, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.workspace = torch.empty(
            _lib.dq_decode_workspace_bytes(batch, q_heads, kv_heads, t_cap, d), dtype=torch.uint8, device=device)

    def append(self, k, v, t0: int):
        """Encode bf16 k, v [B, T_new, H, d] as cache tokens [t0, t0 + T_new)."""
        _lib.dq_encode_kv(self.k_tables, k, t0, self.t_cap, self.k_records, self.k_mean_q,
                          self.k_mean_scale, self.status)
        _lib.dq_encode_kv(self.v_tables, v, t0, self.t_cap, self.v_records, None, None, self.status)

    def attend(self, q, seq_lens, out=None, softmax_scale=None):
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        _lib.dq_decode_attention(self.k_tables, self.v_tables, q, self.k_records, self.k_mean_q,
                                 self.k_mean_scale, self.v_records, seq_lens, out, self.workspace,
                                 softmax_scale=softmax_scale, status=self.status)
        return out

    def partial(self, q, seq_lens, softmax_scale=None):
        """Split-K partials of one decode step into the workspace (finish with merge)."""
        _lib.dq_decode_attention_partial(self.k_tables, self.v_tables, q, self.k_records, self.k_mean_q,
                                         self.k_mean_scale, self.v_records, seq_lens, self.workspace,
                                         softmax_scale=softmax_scale, status=self.status)

    def merge(self, seq_lens, out):
        _lib.dq_decode_attention_merge(self.batch, self.q_heads, self.kv_heads, seq_lens, self.t_cap,
                                       self.workspace, out)

    def compressed_bytes(self, tokens: int) -> int:
        """Bytes of records and key means that cover `tokens` tokens of every sequence."""
        per_tok = self.k_tables.record_bytes + self.v_tables.record_bytes
        mean = (self.head_dim + 2) * ((tokens + _lib.DQ_MEAN_WINDOW - 1) // _lib.DQ_MEAN_WINDOW)
        return self.batch * self.kv_heads * (per_tok * tokens + mean)


class TokenKVCache:
    """Compressed cache with one stream per token over all KV heads (tables
    built with head_dim 128 kv_heads): records of token_records_shape per
    tensor (64-token tiles, 8-byte chunks outermost), key means per head as in
    KVCache."""

    def __init__(self, batch: int, kv_heads: int, q_heads: int, t_cap: int, k_tables, v_tables,
                 device="cuda"):
        if t_cap % _lib.DQ_MEAN_WINDOW:
            raise ValueError("t_cap must be a multiple of 128")
        if k_tables.head_dim != 128 * kv_heads or v_tables.head_dim != 128 * kv_heads:
            raise ValueError("per-token tables need head_dim = 128 kv_heads")
        d = 128
        self.batch, self.kv_heads, self.q_heads, self.t_cap, self.head_dim = batch, kv_heads, q_heads, t_cap, d
        self.k_tables, self.v_tables = k_tables, v_tables
        nw = t_cap // _lib.DQ_MEAN_WINDOW
        self.k_records = torch.zeros(_lib.token_records_shape(k_tables, batch, t_cap), dtype=torch.uint8,
                                     device=device)
        self.v_records = torch.zeros(_lib.token_records_shape(v_tables, batch, t_cap), dtype=torch.uint8,
                                     device=device)
        self.k_mean_q = torch.zeros((batch, kv_heads, nw, d), dtype=torch.int8, device=device)
        self.k_mean_scale = torch.zeros((batch, kv_heads, nw), dtype=torch.int16, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.workspace = torch.empty(
            _lib.dq_decode_workspace_bytes(batch, q_heads, kv_heads, t_cap, d), dtype=torch.uint8, device=device)

    def append(self, k, v, t0: int):
        """Encode bf16 k, v [B, T_new, H, 128] as cache tokens [t0, t0 + T_new)."""
        _lib.dq_encode_kv_token(self.k_tables, k, t0, self.t_cap, self.k_records, self.k_mean_q,
                                self.k_mean_scale, self.status)
        _lib.dq_encode_kv_token(self.v_tables, v, t0, self.t_cap, self.v_records, None, None, self.status)

    def partial(self, q, seq_lens, softmax_scale=None):
        _lib.dq_decode_attention_token_partial(self.k_tables, self.v_tables, q, self.k_records, self.k_mean_q,
                                               self.k_mean_scale, self.v_records, seq_lens, self.workspace,
                                               softmax_scale=softmax_scale, status=self.status)

    def merge(self, seq_lens, out):
        _lib.dq_decode_attention_merge(self.batch, self.q_heads, self.kv_heads, seq_lens, self.t_cap,
                                       self.workspace, out)

    def attend(self, q, seq_lens, out=None, softmax_scale=None):
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        self.partial(q, seq_lens, softmax_scale)
        self.merge(seq_lens, out)
        return out


class Q8KVCache:
    """Cache of 8-bit codes ("int8" or "e4m3") with one fp32 scale per block of
    32 tokens, KV head and tensor (head_dim 128).

    scores=True also keeps every block's accumulated attention weight
    (``scores`` fp32 [B, H, t_cap/32]), which ``attend`` adds to and ``evict``
    goes by.  It is the weight since the block was encoded: a prompt's attention
    and the steps in which its tokens were raw do not count, and before the
    first step all scores are 0, of which ``evict`` keeps the oldest."""

    BLOCK = _lib.DQ_Q8_BLOCK

    def __init__(self, batch: int, kv_heads: int, q_heads: int, t_cap: int, fmt: str = "int8", scores: bool = False,
                 device="cuda"):
        if t_cap <= 0 or t_cap % _lib.DQ_MEAN_WINDOW:
            raise ValueError("t_cap must be a positive multiple of 128")
        if fmt not in _lib.Q8_FORMATS:
            raise ValueError("fmt must be 'int8' or 'e4m3'")
        self.batch, self.kv_heads, self.q_heads, self.t_cap, self.head_dim = batch, kv_heads, q_heads, t_cap, 128
        self.fmt = fmt
        self._format = _lib.Q8_FORMATS[fmt]
        nb = t_cap // self.BLOCK
        self._arrays = tuple(torch.zeros((batch, kv_heads, nb, *rest), dtype=dtype, device=device)
                             for rest, dtype in 2 * [((self.BLOCK * 128,), torch.uint8), ((), torch.float32)])
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.workspace = torch.empty(
            _lib.dq_decode_workspace_bytes(batch, q_heads, kv_heads, t_cap), dtype=torch.uint8, device=device)
        self._scores = self._block_lse = None
        if scores:
            self._scores = torch.zeros_like(self.k_scales)
            self._block_lse = torch.empty((batch, kv_heads, nb, q_heads // kv_heads), dtype=torch.float32,
                                          device=device)
        self._checked = None

    def __getstate__(self):
        return {**self.__dict__, "_checked": None}      # a copy's arrays lie elsewhere

    def _where(self):
        """Sizes, GPU and addresses of the arrays as _lib._q8_cache_args gives
        them, and the addresses of the two score arrays (0: none).  A tensor can
        be given other memory (set_, .data), so every call asks where they lie
        and how long they are; what has moved is checked anew."""
        k, ks, v, vs = self._arrays
        now = (k.data_ptr(), ks.data_ptr(), v.data_ptr(), vs.data_ptr(), k.nbytes, ks.nbytes, v.nbytes, vs.nbytes)
        if self._scores is not None:
            s, lse = self._scores, self._block_lse
            now += (s.data_ptr(), lse.data_ptr(), s.nbytes, lse.nbytes)
        checked = self._checked
        if checked is None or checked[0] != now:
            at = _lib._q8_cache_args(*self._arrays)
            if at[:3] != (self.batch, self.kv_heads, self.t_cap // self.BLOCK):
                raise ValueError("the cache's arrays must keep their shapes")
            score_at, lse_at = _lib._q8_scores(self._scores, self._block_lse, *at[:3],
                                               self.q_heads // self.kv_heads, at[3])
            self._checked = checked = now, (at, score_at, lse_at)
        return checked[1]

    @property
    def arrays(self):
        """(k_data, k_scales, v_data, v_scales)"""
        return self._arrays

    @property
    def k_data(self):
        return self._arrays[0]

    @property
    def k_scales(self):
        return self._arrays[1]

    @property
    def v_data(self):
        return self._arrays[2]

    @property
    def v_scales(self):
        return self._arrays[3]

    @property
    def scores(self):
        """fp32 [B, H, t_cap/32], or None"""
        return self._scores

    @property
    def block_lse(self):
        """the steps' scratch for the scores, fp32 [B, H, t_cap/32, Hq/H], or None"""
        return self._block_lse

    def append(self, k, v, t0: int):
        """Encode bf16 k, v [B, T_new, H, 128] as cache tokens [t0, t0 + T_new)
        (t0 a multiple of 32; a last block that is not full is completed with
        zeros).  The blocks' scores begin at 0."""
        _lib._q8_encode(self._format, self._where()[0], k, v, t0, self.status, None)
        if self.scores is not None:
            self.scores[:, :, t0 // self.BLOCK:(t0 + k.shape[1] + self.BLOCK - 1) // self.BLOCK].zero_()

    def read(self, t0: int, n: int):
        """bf16 k, v [B, n, H, 128]: the values of tokens [t0, t0 + n)."""
        return _lib._q8_read(self._format, self._where()[0], t0, n, None, None, None)

    def attend(self, q, seq_lens, out=None, softmax_scale=None, window: int = 0, sinks: int = 0, scores=None):
        """q bf16 [B, Hq, 128] -> out fp32 over the first seq_lens[b] tokens or,
        with a window, the first `sinks` and the newest `window` of them.  The
        cache's own scores grow by the blocks' weights, or the given ones."""
        at, score_at, lse_at = self._where()
        if score_at and (q.dim() != 3 or q.shape[1] != self.q_heads):
            raise ValueError("q must be [B, q_heads, 128]")
        if scores is not None:
            if self._scores is None:
                raise ValueError("the cache was made without scores")
            score_at, _ = _lib._q8_scores(scores, None, *at[:3], 1, at[3])
        return _lib._q8_attention(self._format, at, q, seq_lens, out, self.workspace, window, sinks, softmax_scale,
                                  lse_at, score_at, None)

    def partial(self, q, seq_lens, softmax_scale=None, window: int = 0, sinks: int = 0, extra_lens=None):
        """Split-K partials of one decode step over q bf16 [B, q_heads, 128] into
        the workspace (finish with merge; the scores' part of it with
        add_scores)."""
        if q.dim() != 3 or q.shape[1] != self.q_heads:
            raise ValueError("q must be [B, q_heads, 128]")      # merge takes the cache's head count
        self._partial(q, seq_lens, softmax_scale, window, sinks, extra_lens)

    def _partial(self, q, seq_lens, softmax_scale, window, sinks, extra_lens):
        _lib._q8_partial(self._format, self._where()[0], q, seq_lens, self.workspace, window, sinks, extra_lens,
                         softmax_scale, self.block_lse, None)

    def merge(self, seq_lens, out):
        _lib.dq_decode_attention_merge(self.batch, self.q_heads, self.kv_heads, seq_lens, self.t_cap,
                                       self.workspace, out)

    def add_scores(self, seq_lens, window: int = 0, sinks: int = 0, extra_lens=None):
        _lib.dq_q8_add_scores(self.q_heads, seq_lens, self.block_lse, self.workspace, self.scores, window, sinks,
                              extra_lens)

    def merge_scores(self, seq_lens, out, window: int = 0, sinks: int = 0, extra_lens=None):
        """merge and add_scores in one launch."""
        _lib.dq_q8_merge_scores(self.q_heads, seq_lens, self.block_lse, self.workspace, out, self.scores, window,
                                sinks, extra_lens)

    def evict(self, seq_lens, keep: int, sinks: int = 0, recent: int = 32, into=None, new_lens=None):
        """Cut every sequence to at most `keep` / 32 blocks (`keep` a multiple of
        32): its first `sinks` / 32 and newest `recent` / 32 blocks (both rounded
        up, and one at least of the newest) and those of the largest scores, in
        their order; in place, or into another Q8KVCache with scores.  The newest
        block counts as one however few tokens it holds: recent = n + 31 keeps
        the newest n tokens at every length.  Returns the kept blocks' old
        indexes int32 [B, H, keep/32] (-1: none) and the new lengths (new_lens
        if given, which may be seq_lens)."""
        to = self if into is None else into
        if self.scores is None or to.scores is None or to.fmt != self.fmt:
            raise ValueError("eviction needs scores, and caches of one format")
        if keep <= 0 or keep % self.BLOCK:
            raise ValueError("keep must be a positive multiple of 32")
        if sinks < 0 or recent < 0:
            raise ValueError("sinks and recent must not be negative")
        kept = self.status.new_empty((self.batch, self.kv_heads, keep // self.BLOCK))
        if new_lens is None:
            new_lens = torch.empty_like(seq_lens)
        up = -self.BLOCK
        at, score_at, _ = self._where()
        to_at, to_score_at, _ = to._where()
        _lib._q8_evict(seq_lens, new_lens, keep, sinks // up * up, max(recent // up * up, self.BLOCK), at, score_at,
                       to_at, to_score_at, kept, None)
        return kept, new_lens

    def cache_bytes(self, tokens: int) -> int:
        """Bytes of codes and scales that cover `tokens` tokens of every sequence."""
        blocks = (tokens + self.BLOCK - 1) // self.BLOCK
        return self.batch * self.kv_heads * blocks * 2 * (self.BLOCK * 128 + 4)


class StreamingKVCache:
    """A compressed cache plus the BF16 residual window of the newest tokens.

    Sec. 5.1 keeps the most recent tokens in BF16.  Here the newest tokens of
    every sequence sit raw in a ring of 2 x 128 slots (the library's residual
    window); when the ring is full its oldest 128 tokens are encoded as one
    key-mean window and leave it, so at least the 128 most recent tokens are
    always raw.  Decode attention runs over both parts in one step.  All
    sequences of the batch advance together (same length).

    streams="head" keeps one stream per (token, KV head) (a KVCache);
    streams="token" the paper's default grouping, one stream per token over
    all KV heads (a TokenKVCache, tables built with head_dim 128 kv_heads);
    streams="int8" or "e4m3" 8-bit codes (a Q8KVCache, no tables), which also
    give attention behind a window and, with scores=True, eviction.
    The ring, its append and commit, and the residual attention are the same
    for all.
    """

    WINDOW = _lib.DQ_MEAN_WINDOW

    def __init__(self, batch: int, kv_heads: int, q_heads: int, t_cap: int, k_tables, v_tables,
                 device="cuda", r_cap: int = 256, streams: str = "head", scores: bool = False):
        if r_cap % self.WINDOW or not (2 * self.WINDOW <= r_cap <= 256):
            raise ValueError("r_cap must be 256 (two mean windows)")
        if streams == "head":
            self.cache = KVCache(batch, kv_heads, q_heads, t_cap, k_tables, v_tables, device=device)
        elif streams == "token":
            self.cache = TokenKVCache(batch, kv_heads, q_heads, t_cap, k_tables, v_tables, device=device)
        elif streams in _lib.Q8_FORMATS:
            if k_tables is not None or v_tables is not None:
                raise ValueError("8-bit streams take no tables")
            self.cache = Q8KVCache(batch, kv_heads, q_heads, t_cap, streams, scores=scores, device=device)
        else:
            raise ValueError("streams must be 'head', 'token', 'int8' or 'e4m3'")
        if scores and streams not in _lib.Q8_FORMATS:
            raise ValueError("scores need 8-bit streams")
        self.streams = streams
        d = self.cache.head_dim
        self.r_cap = r_cap
        self.res_k = torch.zeros((batch, kv_heads, r_cap, d), dtype=torch.bfloat16, device=device)
        self.res_v = torch.zeros_like(self.res_k)
        self.seq_lens = torch.zeros(batch, dtype=torch.int32, device=device)   # compressed tokens
        self.res_lens = torch.zeros(batch, dtype=torch.int32, device=device)   # residual tokens
        self.n_comp = 0
        self.n_res = 0

    @property
    def status(self):
        return self.cache.status

    def __len__(self) -> int:
        return self.n_comp + self.n_res

    def prefill(self, k, v):
        """k, v bf16 [B, T, H, d] into an empty cache: whole windows are encoded,
        the last 128..255 tokens (all of them if T < 128) stay raw."""
        if len(self):
            raise RuntimeError("prefill needs an empty cache")
        T = k.shape[1]
        n_enc = max(0, (T - self.WINDOW) // self.WINDOW * self.WINDOW)
        if n_enc:
            self.cache.append(k[:, :n_enc], v[:, :n_enc], 0)
            self.seq_lens += n_enc
            self.n_comp = n_enc
        for t in range(n_enc, T):
            self.append(k[:, t].contiguous(), v[:, t].contiguous())

    def append(self, k1, v1):
        """One decode token per sequence: k1, v1 bf16 [B, H, d]."""
        if self.n_res == self.r_cap:
            self._flush()
        _lib.dq_residual_append(k1, v1, self.res_k, self.res_v, self.seq_lens, self.res_lens, self.status)
        self.n_res += 1
        if self.n_res == self.r_cap:
            self._flush()

    def _flush(self):
        W = self.WINDOW
        if self.n_comp + W > self.cache.t_cap:
            raise RuntimeError("compressed cache is full")
        s = self.n_comp % self.r_cap
        k = self.res_k[:, :, s:s + W].permute(0, 2, 1, 3)     # [B, W, H, d] view of the ring
        v = self.res_v[:, :, s:s + W].permute(0, 2, 1, 3)
        self.cache.append(k, v, self.n_comp)
        _lib.dq_residual_commit(self.seq_lens, self.res_lens, W, self.status)
        self.n_comp += W
        self.n_res -= W

    def attend(self, q, out=None, softmax_scale=None, window: int = 0, sinks: int = 0):
        """q bf16 [B, Hq, d] -> out fp32 [B, Hq, d] over every token so far, or
        (8-bit streams; window >= r_cap) over the first `sinks` and the newest
        `window` of them."""
        c = self.cache
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        if self.streams not in _lib.Q8_FORMATS:
            if window or sinks:
                raise ValueError("a window needs 8-bit streams")
            c.partial(q, self.seq_lens, softmax_scale)
        else:
            if window and window < self.r_cap:
                raise ValueError("window must be 0 or at least r_cap")
            c._partial(q, self.seq_lens, softmax_scale, window, sinks, self.res_lens)
            if c.scores is not None:
                # the scores' weights need the raw tokens' partials in the workspace
                _lib.dq_decode_attention_residual(q, self.res_k, self.res_v, self.seq_lens, self.res_lens, c.t_cap,
                                                  c.workspace, softmax_scale=softmax_scale)
                c.merge_scores(self.seq_lens, out, window, sinks, self.res_lens)
                return out
        _lib.dq_decode_attention_merge_residual(q, self.res_k, self.res_v, self.seq_lens, self.res_lens, c.t_cap,
                                                c.workspace, out, softmax_scale=softmax_scale)
        return out

    def evict(self, keep: int, sinks: int = 0, recent: int = 32):
        """Cut the compressed side to `keep` tokens and up to r_cap - 1 more (the
        ring's slots go by its length, so whole rings of tokens leave): of every
        sequence and KV head the blocks with the least attention weight since
        they left the ring, the first `sinks` and newest `recent` compressed
        tokens apart.  Returns the kept blocks' old indexes, or None if nothing
        had to go."""
        if self.streams not in _lib.Q8_FORMATS:
            raise ValueError("eviction needs 8-bit streams")
        gone = (self.n_comp - keep) // self.r_cap * self.r_cap
        if gone <= 0:
            return None
        kept, _ = self.cache.evict(self.seq_lens, self.n_comp - gone, sinks, recent, new_lens=self.seq_lens)
        self.n_comp -= gone
        return kept
