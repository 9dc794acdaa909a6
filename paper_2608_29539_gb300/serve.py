"""Serving the global branch for a batch that shares a long prefix: drafted
tokens, verified in one call, over caches that stay bounded.

A step of a sequence brings n_new tokens: the last accepted one and n_new - 1
drafts.  ``ServeBatch`` holds the shared prefix and every sequence's own cache
and chains the entry points as a serving loop does:

    batch.step(q, k_new, v_new, gate_p)   the new tokens' K and V join the caches;
                                          gate and packing (Eq. 7); attention of the
                                          selected rows over prefix and own cache
                                          (Eq. 8), adding up each cache row's weight
    batch.verify(draft, q_draft, p_target, u, noise)
                                          accepts or rejects the drafts, draws the
                                          next token, drops the rejected tokens' rows
    batch.evict()                         cuts the caches back to the budget by the
                                          accumulated weights

Nothing here waits for the GPU, and all lengths stay on the device.  Rejected
drafts have added to the weights by then; their own rows are gone.  The rest of
the layer (projections, the local branch, ContextNorm and fusion) is the
caller's, by logo_decode_local_attn and logo_combine where n_new is 1.

``ServeBatch4`` is the same loop for sequences whose own caches are kept whole, in
4 bits a value: prompts are filled in, nothing is evicted, and verification starts
from the target's logits and what each request asks of its sampling.
"""
from __future__ import annotations

import dataclasses

import torch

from . import logo as L


@dataclasses.dataclass
class ServeConfig:
    B: int             # sequences
    n_new: int         # tokens a step brings per sequence (drafts + 1)
    Hq: int
    Hkv: int
    D: int
    budget: int        # cache rows per sequence and KV head after an eviction
    recent: int        # latest positions that are never evicted
    slack: int = 0     # cache rows beyond budget + n_new (steps between evictions)
    mode: int = L.LOGO_SELECT_THRESHOLD
    b_th: float = 0.5
    ratio: float = 1.0
    scale: float = 0.0


class ServeBatch:
    """Own caches, weights and positions of a batch over one shared prefix.

    k_prefix / v_prefix [P, Hkv, D] bf16, or None.  Positions count from the
    prefix's first token.  At most slack / n_new + 1 steps may pass without an
    eviction: a cache holds budget + n_new + slack rows.  A step that might not fit
    is refused, counting rejected drafts too, as their number stays on the device.
    Replays of a captured CUDA graph are not seen here: once a call was captured
    nothing is refused, and a step that finds no room overwrites the latest rows."""

    def __init__(self, cfg: ServeConfig, k_prefix=None, v_prefix=None, device="cuda"):
        if cfg.budget < 1 or cfg.n_new < 1 or cfg.slack < 0 or not 0 <= cfg.recent <= cfg.budget:
            raise ValueError("need budget >= 1, n_new >= 1, slack >= 0 and 0 <= recent <= budget")
        self.cfg = c = cfg
        dev = torch.device(device)
        self.rows = c.budget + c.n_new + c.slack
        self.k_prefix, self.v_prefix = k_prefix, v_prefix
        P = 0 if k_prefix is None else k_prefix.shape[0]
        z = lambda shape, dt: torch.zeros(shape, dtype=dt, device=dev)  # noqa: E731
        self.k = z((c.B, self.rows, c.Hkv, c.D), torch.bfloat16)
        self.v = torch.zeros_like(self.k)
        self.mass = z((c.B, c.Hkv, self.rows), torch.float32)
        self.slot_pos = z((c.B, c.Hkv, self.rows), torch.int32)
        self.seq_len = z((c.B,), torch.int32)
        self.n_seen = torch.full((c.B,), P, dtype=torch.int32, device=dev)
        cap = c.B * c.n_new
        self.z = z((c.B, c.n_new), torch.uint8)
        self.pos = z((cap,), torch.int32)
        self.cu_q = z((c.B + 1,), torch.int32)
        self.row_of = z((c.B, c.n_new), torch.int32)
        self.n_sel = z((1,), torch.int32)
        self.o_c = z((cap, c.Hq, c.D), torch.bfloat16)
        self.lse_c = z((c.Hq, cap), torch.float32)
        self.new_len = z((c.B,), torch.int32)
        self._b = torch.arange(c.B, device=dev)[:, None]
        self._i = torch.arange(c.n_new, device=dev, dtype=torch.int32)
        self._rows_used = 0     # at most this many rows of any cache hold a token
        self._latest_last = True  # the latest step's rows are the caches' last ones, and all there
        self._captured = False  # whether a graph holds some of the calls
        dims = L.Dims(c.B, self.rows, c.Hq, c.Hkv, c.D)
        lib = L.lib()
        nbytes = max(int(lib.logo_decode_prefix_workspace_size(dims, c.n_new, P, 1)),
                     int(lib.logo_cache_evict_workspace_size(dims)),
                     int(lib.logo_select_workspace_size(L.Dims(c.B, c.n_new, 1, 1, 64))))
        self.ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=dev)  # the calls are stream-ordered

    def _counts(self):
        """Are all calls seen here?"""
        self._captured |= self.k.is_cuda and torch.cuda.is_current_stream_capturing()
        return not self._captured

    def append(self, k_new, v_new):
        """K and V [B, n_new, Hkv, D] of the new tokens into the caches' next rows."""
        n = self.cfg.n_new
        if self._counts() and self._rows_used + n > self.rows:
            raise ValueError(f"{n} more rows may not fit, {self._rows_used} of {self.rows} may be in use: evict first")
        self.seq_len.clamp_(max=self.rows - n)  # (a replay may come here with full caches)
        slots = (self.seq_len[:, None] + self._i).long()
        self.k[self._b, slots] = k_new
        self.v[self._b, slots] = v_new
        at = (self.n_seen[:, None] + self._i)[:, None].expand(-1, self.cfg.Hkv, -1)
        self.slot_pos.scatter_(2, slots[:, None].expand(-1, self.cfg.Hkv, -1), at)
        self.seq_len += n
        self.n_seen += n
        self._rows_used += n
        self._latest_last = True

    def step(self, q, k_new, v_new, gate_p):
        """q [B, n_new, Hq, D], k_new / v_new [B, n_new, Hkv, D] bf16, gate_p
        [B, n_new] float32.  Returns (o_c [B*n_new, Hq, D] packed, z, row_of):
        what logo_combine takes on (B, n_new); the next step writes to the same
        buffers."""
        c = self.cfg
        # what is refused is refused before the caches change
        L._need(q, torch.bfloat16, "q", (c.B, c.n_new, c.Hq, c.D))
        L._need(gate_p, torch.float32, "gate_p", (c.B, c.n_new))
        self.append(k_new, v_new)
        L.logo_select(gate_p, c.mode, c.b_th, c.ratio, self.z, self.pos, self.cu_q, self.row_of, self.n_sel,
                      workspace=self.ws)
        L.logo_decode_prefix_attn(q, self.k_prefix, self.v_prefix, self.k, self.v, self.seq_len, self.pos, self.cu_q,
                                  self.n_sel, c.scale, mass_in=self.mass, o_c=self.o_c, lse_c=self.lse_c,
                                  workspace=self.ws)
        return self.o_c, self.z, self.row_of

    def verify(self, draft, q_draft, p_target, u, noise, draft_len=None):
        """The step's drafts (n_new - 1 per sequence, of which the first draft_len [B]
        int32 count where it is given: a rejection past them would draw the next
        token from the wrong distribution) against the target's probabilities
        [B, n_new, V]; the tokens that are not accepted leave the caches.
        Returns (tokens [B, n_new], n_accept [B]).  Once a step and before evict,
        which moves the rows that are dropped from the end here."""
        if self._counts() and self.cfg.n_new > 1 and not self._latest_last:
            raise ValueError("the drafts were verified, or the caches cut, since the last step")
        if p_target.shape[0] != self.cfg.B or p_target.shape[1] > self.cfg.n_new:
            want = f"({self.cfg.B}, {self.cfg.n_new}, V)"
            raise ValueError(f"p_target has shape {tuple(p_target.shape)}, expected {want}")
        tokens, n_accept = L.logo_verify_draft(draft, q_draft, p_target, u, noise, draft_len=draft_len,
                                                workspace=self.ws)
        self._latest_last = False
        dropped = self.cfg.n_new - 1 - n_accept
        self.seq_len -= dropped
        self.n_seen -= dropped
        return tokens, n_accept

    def evict(self):
        """Every cache back to at most `budget` rows.  Lengths keep their place in
        memory, so that the call can be part of a captured graph."""
        c = self.cfg
        L.logo_cache_evict(self.k, self.v, self.mass, self.slot_pos, self.seq_len, self.n_seen, c.budget, c.recent,
                           new_len=self.new_len, workspace=self.ws)
        self.seq_len.copy_(self.new_len)
        self._counts()
        self._latest_last = False
        self._rows_used = min(self._rows_used, c.budget)


@dataclasses.dataclass
class Serve4Config:
    B: int             # sequences
    n_new: int         # tokens a step brings per sequence (drafts + 1)
    Hq: int
    Hkv: int
    D: int
    rows: int          # cache rows per sequence
    mode: int = L.LOGO_SELECT_THRESHOLD
    b_th: float = 0.5
    ratio: float = 1.0
    scale: float = 0.0


class ServeBatch4:
    """A batch over caches of its own that are held in 4 bits.

        batch.fill(k, v, n_valid)             prompts, or the next chunk of them
        batch.context(m)                      the rows held so far, for a chunk's dense attention
        batch.step(q, k_new, v_new, gate_p)   the new tokens join; gate, packing, attention
        batch.verify(draft, q_draft, logits, u, noise, ...)
                                              logits to probabilities, verdict, rejected rows dropped

    What might not fit the caches is refused, counting rejected drafts too, as their
    number stays on the device (recount() reads it back).  Replays of a captured graph are
    not seen here: once a call was captured nothing is refused, and where a sequence
    has no room for all that it brings, its latest rows are overwritten."""

    def __init__(self, cfg: Serve4Config, device="cuda"):
        if cfg.B < 1 or cfg.n_new < 1 or cfg.rows < cfg.n_new:
            raise ValueError("need B >= 1, n_new >= 1 and rows >= n_new")
        self.cfg = c = cfg
        lib = L.lib()
        attn_bytes = int(lib.logo_decode_cache4_workspace_size(L.Dims(c.B, c.rows, c.Hq, c.Hkv, c.D), c.n_new))
        # what the calls of a step would refuse each time (a size of 0: these sizes)
        if not attn_bytes:
            raise ValueError(f"logo_decode_cache4_attn does not take these sizes: {c}")
        if c.mode not in (L.LOGO_SELECT_THRESHOLD, L.LOGO_SELECT_RATIO) or \
                (c.mode == L.LOGO_SELECT_RATIO and not 0.0 <= c.ratio <= 1.0):
            raise ValueError("mode has to be a LOGO_SELECT_* and a ratio in [0, 1]")
        if not 0.0 <= c.scale <= 3.4e38:
            raise ValueError("scale has to be 0 or more, and finite in float32")
        dev = torch.device(device)
        z = lambda shape, dt: torch.zeros(shape, dtype=dt, device=dev)  # noqa: E731
        self.cache = L.logo_cache4_empty(c.B, c.rows, c.Hkv, c.D, dev)
        self.seq_len = z((c.B,), torch.int32)
        cap = c.B * c.n_new
        self.z = z((c.B, c.n_new), torch.uint8)
        self.pos = z((cap,), torch.int32)
        self.cu_q = z((c.B + 1,), torch.int32)
        self.row_of = z((c.B, c.n_new), torch.int32)
        self.n_sel = z((1,), torch.int32)
        self.o_c = z((cap, c.Hq, c.D), torch.bfloat16)
        self.lse_c = z((c.Hq, cap), torch.float32)
        nbytes = max(attn_bytes, int(lib.logo_select_workspace_size(L.Dims(c.B, c.n_new, 1, 1, 64))))
        self.ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=dev)  # the calls are stream-ordered
        self._rows_used = 0       # at most this many rows of any cache hold a token
        self._latest_step = False  # the caches' last rows are the latest step's, and all there
        self._captured = False    # whether a graph holds some of the calls

    _counts = ServeBatch._counts

    @property
    def k(self):  # (what _counts looks at)
        return self.cache.k

    def _room(self, n):
        if self._counts() and self._rows_used + n > self.cfg.rows:
            raise ValueError(f"{n} more rows may not fit, {self._rows_used} of {self.cfg.rows} may be in use")

    def recount(self):
        """Counts the rows in use, which waits for the GPU; returns the largest count."""
        self._rows_used = int(self.seq_len.max())
        return self._rows_used

    def fill(self, k, v, n_valid=None):
        """K and V [B, n, Hkv, D] bf16 behind what the caches hold; of sequence b the first
        n_valid[b] (int32; None: all n)."""
        n = k.shape[1]
        if n > self.cfg.rows:
            raise ValueError(f"{n} rows do not fit caches of {self.cfg.rows}")
        self._room(n)
        if n_valid is not None:
            L._need(n_valid, torch.int32, "n_valid", (self.cfg.B,))
            n_valid = n_valid.clamp(0, n)
        # (a replay may come here with full caches: room is made for what a sequence brings, no more)
        if n_valid is None:
            seq_len = self.seq_len.clamp(max=self.cfg.rows - n) + n
        else:
            seq_len = torch.minimum(self.seq_len, self.cfg.rows - n_valid) + n_valid
        L.logo_cache4_append(self.cache, k, v, seq_len, n_valid)
        self.seq_len.copy_(seq_len)
        self._rows_used += n
        self._latest_step = False

    def context(self, m=None):
        """The first m rows (None: all) of every cache as bf16 (k, v) [B, m, Hkv, D], zeros
        past a sequence's tokens."""
        return L.logo_cache4_read(self.cache, self.seq_len, m=m)

    def step(self, q, k_new, v_new, gate_p):
        """q [B, n_new, Hq, D], k_new / v_new [B, n_new, Hkv, D] bf16, gate_p [B, n_new]
        float32.  Returns (o_c [B*n_new, Hq, D] packed, z, row_of): what logo_combine takes
        on (B, n_new); the next step writes to the same buffers."""
        c = self.cfg
        # what one of the calls would refuse is refused before the caches change
        dev = self.cache.k.get_device()
        L._on(gate_p, dev, torch.float32, "gate_p", (c.B, c.n_new))
        for name, t, heads in (("q", q, c.Hq), ("k_new", k_new, c.Hkv), ("v_new", v_new, c.Hkv)):
            L._on(t, dev, torch.bfloat16, name, (c.B, c.n_new, heads, c.D))
            if t.data_ptr() % 16:
                raise ValueError(f"{name} does not begin at a multiple of 16 bytes")
        if dev >= 0:
            L._here(dev)
        self._room(c.n_new)
        self.seq_len.clamp_(max=c.rows - c.n_new)  # (a replay may come here with full caches)
        self.seq_len += c.n_new
        L.logo_cache4_append(self.cache, k_new, v_new, self.seq_len)
        self._rows_used += c.n_new
        self._latest_step = True
        L.logo_select(gate_p, c.mode, c.b_th, c.ratio, self.z, self.pos, self.cu_q, self.row_of, self.n_sel,
                      workspace=self.ws)
        L.logo_decode_cache4_attn(q, self.cache, self.seq_len, self.pos, self.cu_q, self.n_sel, c.scale, o_c=self.o_c,
                                  lse_c=self.lse_c, workspace=self.ws)
        return self.o_c, self.z, self.row_of

    def verify(self, draft, q_draft, logits, u, noise, draft_len=None, **sampling):
        """The step's drafts (n_new - 1 per sequence, of which the first draft_len [B] int32
        count where it is given) against the target's logits [B, n_new, V]; sampling: what
        logo_target_probs takes beside them (its draft is given here where there is a
        penalty).  The tokens that are not accepted leave the caches.  Returns (tokens [B,
        n_new], n_accept [B]).  Once a step."""
        c = self.cfg
        if self._counts() and c.n_new > 1 and not self._latest_step:
            raise ValueError("the drafts were verified, or rows filled in, since the last step")
        if logits.dim() != 3 or logits.shape[0] != c.B or logits.shape[1] != c.n_new:
            raise ValueError(f"logits has shape {tuple(logits.shape)}, expected ({c.B}, {c.n_new}, V)")
        if sampling.get("penalty") is not None and c.n_new > 1:
            sampling.setdefault("draft", draft)
        p = L.logo_target_probs(logits, **sampling)
        tokens, n_accept = L.logo_verify_draft(draft, q_draft, p, u, noise, draft_len=draft_len)
        self._latest_step = False
        self.seq_len -= c.n_new - 1 - n_accept
        return tokens, n_accept
