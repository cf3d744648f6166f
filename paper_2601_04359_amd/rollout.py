"""Rolling PackCache for one attention layer: the cache stays packed across frame steps.

Host-side bookkeeping only (buffers, the segment table, which C-ABI call comes next); every
step of the path runs in libpackcache kernels.  Per frame step (Sec. 3.4, Fig. 5(b)):

    reserve()/commit()  the frame generated last is appended whole (keys rotated on insert)
    pc_score            importance of every cached key under the step's queries
    pc_budget           per-distance token budgets (config rule or the paper's Eq. 6 / Eq. 7)
    pc_compact          in place: anchors stay, each past frame keeps its top-budget keys
    pc_frame_attn       the step's queries over the packed cache

The frame being generated may sit in the cache too (attention inside a frame is
bidirectional, Eq. 2): commit it with kind PC_SEG_SELF before step(); it takes part in the
softmax of scoring and attention, is never pruned at its own step, and promote_self() turns
it into the newest past frame when the next step begins, without moving a row.

A model that makes several attention passes per frame (iterative decoding) calls attend()
on the un-packed cache first, hands its log-sum-exp to refresh() and makes the remaining
passes on the packed cache: the compaction is paid once per frame.

EvictingStack is the cache of a stack of layers for generation in small steps (text, or video token
by token), held in 4 bits and kept within a budget by what attention itself looks at instead of by
the frames' age: pc_q4_store, pc_q4_attn (which adds up every key's attention weight) and one
pc_q4_evict for all layers when a step ends.

PagedStack holds the caches of several sequences at once in pages of one pool: prompts of any lengths go in together
(pc_prompt_attn), a sequence can be continued several ways at once without a copy of what is common, and a step's rows of all
sequences are stored (pc_page_store, with the rotation on the way) and attended to (pc_page_attn, the common rows once for all).

With slide_t_scale set the window slides (Sec. 3.4, Slide-Cache): when a step begins, the
oldest frames that the step before evicted completely leave the segment table and
pc_rebase lowers the temporal coordinate of every retained frame row by slide_t_scale per
dropped frame; `shift` is the total so far, and the caller places the frame it appends and
its queries at their coordinates minus `shift`.

Eviction is irreversible: a frame's candidates at one step are its survivors of the step
before.  With mode "dense" nothing is evicted (the full-cache baseline); with mode "slide"
only the newest frame survives (the sliding-window baseline of Sec. 3.3).
"""
from __future__ import annotations

from . import binding as pk

MODES = {"pow": pk.PC_BUDGET_POW, "norm": pk.PC_BUDGET_NORM, "half": pk.PC_BUDGET_HALF,
         "slide": pk.PC_BUDGET_SLIDE, "dense": None}


class RollingLayer:
    """The packed K/V cache of one layer in HBM and its host-side segment table."""

    def __init__(self, Hq: int, Hkv: int, D: int, capacity: int, n_frame: int, scale: float,
                 mode: str = "pow", gamma: float = 0.85, b_min: int = 512, budget_tokens: int | None = None,
                 n_score: int = 512, sections=(32, 48, 48), base: float = 10000.0, dtype=None, device="cuda:0",
                 slide_t_scale: int | None = None, share_heads: bool = False, fold_scale: bool = False):
        import torch
        if mode not in MODES:
            raise ValueError(f"mode {mode!r} not in {sorted(MODES)}")
        self.Hq, self.Hkv, self.D, self.capacity, self.n_frame = Hq, Hkv, D, capacity, n_frame
        self.scale, self.mode, self.gamma, self.b_min = scale, mode, gamma, b_min
        # fold_scale: the queries carry scale * log2(e) (step() multiplies it in while rotating; a
        # caller that rotates them itself passes them that way) and the scoring and attention calls
        # get ln 2 as their scale: the same softmax on the kernels' shorter loops
        self.fold_scale = fold_scale
        self.q_out_scale = pk.folded_q_scale(scale) if fold_scale else 1.0
        self.call_scale = pk.PC_SCALE_FOLDED if fold_scale else scale
        # POW floors gamma^d of a whole frame; NORM / HALF / SLIDE split a fixed token budget
        self.budget_tokens = n_frame if budget_tokens is None else budget_tokens
        self.sections, self.base = tuple(sections), base
        dtype = torch.bfloat16 if dtype is None else dtype
        # share_heads: one selection for all KV heads (the paper's per-token cache mask) instead
        # of one per KV head; positions and scores then have a single head
        self.share_heads = share_heads
        hsel = 1 if share_heads else Hkv
        self.K = torch.empty((Hkv, capacity, D), dtype=dtype, device=device)
        self.V = torch.empty_like(self.K)
        self.pos = torch.empty((hsel, capacity, 3), dtype=torch.int32, device=device)
        self.segments: list[tuple[int, int, int, int]] = []
        self.nk = 0
        self.slide_t_scale, self.shift = slide_t_scale, 0
        n_rows = min(n_score, n_frame)
        self.q_rows = ((torch.arange(n_rows, dtype=torch.int64) * n_frame) // n_rows).to(torch.int32).to(device)
        if mode != "dense":   # the full-cache baseline neither scores nor compacts
            self.score = torch.empty((hsel, capacity), dtype=torch.float32, device=device)
            self._ws_score = torch.empty(pk.pc_score_workspace_bytes(Hq, Hkv, n_rows, capacity, share_heads),
                                         dtype=torch.uint8, device=device)
            self._ws_compact = torch.empty(pk.pc_compact_workspace_bytes(Hkv, capacity, share_heads),
                                           dtype=torch.uint8, device=device)

    # ---- insertion: the producer writes straight into the cache, no copy ----------------------
    def reserve(self, n: int):
        """Views of the next n free rows: (K rows, V rows, pos rows [Hsel][n][3])."""
        if self.nk + n > self.capacity:
            raise ValueError(f"cache capacity {self.capacity} < {self.nk} + {n}")
        return pk._rows(self.K, self.V, self.pos, 1, self.nk, n)

    def commit(self, n: int, kind: int, frame: int, rotate_with=None, valid=None) -> None:
        """Make the n reserved rows part of the cache.  rotate_with: int32 [n][3] device
        positions; when given the new keys are rotated in place (a1) on insertion.
        valid (host array of n flags, the cache mask of Sec. 3.1 for this frame): only the
        unmasked tokens enter the cache.  The masked rows are removed on insertion by the
        compaction call itself (mask as the score, budget = unmasked count; the rest of the
        cache keeps every row), so no later scoring or attention ever sees them: masked
        entries are ignored in attention (Sec. 3.1), and removed rather than stored (Sec. 3.4)."""
        a = self.nk
        if rotate_with is not None:
            pk.pc_rope3d(self.K[:, a:a + n], rotate_with, self.sections, self.base)
        if valid is not None:
            import numpy as np
            import torch
            if kind != pk.PC_SEG_FRAME:
                raise ValueError("a cache mask applies to a generated frame entering the cache (PC_SEG_FRAME)")
            v = np.ascontiguousarray(np.asarray(valid) != 0, dtype=np.uint8)
            if v.shape != (n,):
                raise ValueError(f"valid must hold {n} flags, got shape {v.shape}")
            n_valid = int(v.sum())
            if n_valid < n:
                if not hasattr(self, "score"):      # the full-cache baseline scores nothing else
                    self.score = torch.empty((self.pos.shape[0], self.capacity), dtype=torch.float32,
                                             device=self.K.device)
                    self._ws_compact = torch.empty(pk.pc_compact_workspace_bytes(self.Hkv, self.capacity,
                                                                                 self.share_heads),
                                                   dtype=torch.uint8, device=self.K.device)
                sc_new = self.score[:, a:a + n]
                sc_new.zero_()
                pk.pc_mask_scores(sc_new, torch.from_numpy(v).to(self.K.device))    # masked -> -1 < 0
                table = self.segments + [(a, n, kind, frame)]
                keep = [s[1] for s in self.segments] + [n_valid]
                self.segments, self.nk = pk.pc_compact(self.K, self.V, self.pos, self.score, table, keep,
                                                       share_heads=self.share_heads, ws=self._ws_compact)
                return
        self.segments.append((a, n, kind, frame))
        self.nk = a + n

    def promote_self(self) -> None:
        """Call when a step begins: the frame that was generated last and sat in the cache as the
        always-kept SELF segment of its own step (commit(..., kind=PC_SEG_SELF)) becomes the newest
        past frame.  A table edit only: its rows are already in place."""
        self.segments = [(a, n, pk.PC_SEG_FRAME if kind == pk.PC_SEG_SELF else kind, f)
                         for (a, n, kind, f) in self.segments]

    def advance_window(self) -> int:
        """Call when a step begins, before reserve(): drops the oldest frame segments that
        are empty and rebases the retained frame rows.  Returns the total shift so far."""
        if self.slide_t_scale is None:
            return self.shift
        first = next((j for j, s in enumerate(self.segments) if s[2] == pk.PC_SEG_FRAME), len(self.segments))
        n_drop = 0
        while first + n_drop < len(self.segments) and self.segments[first + n_drop][1] == 0:
            n_drop += 1
        if n_drop and first + n_drop < len(self.segments):
            delta = self.slide_t_scale * n_drop
            self.segments = self.segments[:first] + self.segments[first + n_drop:]
            a = self.segments[first][0]
            pk.pc_rebase(self.K, self.pos, a, self.nk - a, delta, self.sections, self.base)
            self.shift += delta
        return self.shift

    # ---- one frame step -----------------------------------------------------------------------
    def budgets(self) -> list[int]:
        """Budget of every segment for the cache as it stands (anchors: their length)."""
        if self.mode == "dense":
            return [s[1] for s in self.segments]
        n_past = pk._past_frames(self.segments)
        if self.mode == "pow":
            per_d = pk.pc_budget(pk.PC_BUDGET_POW, self.n_frame, n_past, self.gamma, self.b_min)
        else:
            per_d = pk.pc_budget(MODES[self.mode], self.budget_tokens, n_past, self.gamma, self.b_min)
        return pk.segment_budgets(self.segments, per_d)

    def refresh(self, Q, lse=None) -> None:
        """Score every cached key under the (rotated) queries Q and re-pack the cache in
        place.  lse (fp32 [Hq][n_frame]): log-sum-exp of Q's rows over the cache as it
        stands, e.g. from attend(): scoring then needs one QK^T pass instead of two."""
        if self.mode == "dense":
            return
        budgets = self.budgets()
        # only segments that lose rows at this step need scores (anchors never do, a frame that sits at
        # its budget does not either): the scoring covers the span from the first to the last of them
        span = pk._prunable_span(self.segments, budgets)
        if span is None:
            return   # every frame is within its budget: nothing to score, nothing to move
        pk.pc_score(Q, self.K, self.nk, self.call_scale, lse=lse, score=self.score, share_heads=self.share_heads,
                    ws=self._ws_score, q_rows=self.q_rows, key_range=span)
        self.segments, self.nk = pk.pc_compact(self.K, self.V, self.pos, self.score, self.segments,
                                               budgets, share_heads=self.share_heads, ws=self._ws_compact)

    def attend(self, Q, O=None, lse=None):
        """The (rotated) queries Q over the cache as it stands -> O (and the log-sum-exp).  It only reads
        the cache, and each call's key shares go to a workspace of its own: passes on several streams
        or from several threads may overlap."""
        return pk.pc_frame_attn(Q, self.K, self.V, self.nk, self.call_scale, O=O, lse=lse)

    def step(self, Q, O=None, q_pos=None, lse=None):
        """Queries Q [Hq][n_frame][D] of the frame being generated -> O.  q_pos (int32
        [n_frame][3], device): rotate Q in place first (with fold_scale, times scale * log2(e))."""
        if q_pos is not None:
            pk.pc_rope3d(Q, q_pos, self.sections, self.base, out_scale=self.q_out_scale)
        self.refresh(Q)
        return self.attend(Q, O=O, lse=lse)


class RollingStack:
    """The packed caches of a stack of layers in one allocation, re-packed TOGETHER when a frame
    step ends (Sec. 3.4 re-packs the cache at the frame step, not per attention call).

    Per frame step:
        reserve()/commit()   the frame generated last is appended whole to every layer's cache
        per layer:           attend() over the cache as it stands, with the log-sum-exp of the pass;
                             score_layer() turns that log-sum-exp into importances with ONE QK^T pass
        repack()             budgets, then one pc_compact_batch for the whole stack

    All layers share one segment table: budgets depend on the temporal distance only, so every
    layer keeps the same COUNT of rows per frame (each its own rows).  The cache a step attends
    over is the one the previous step packed plus the whole newest frame; the cache repack()
    leaves is the one RollingLayer.step() would have attended over at the same step (same keys
    scored by the same queries under the same budgets).
    """

    def __init__(self, n_layers: int, Hq: int, Hkv: int, D: int, capacity: int, n_frame: int, scale: float,
                 mode: str = "pow", gamma: float = 0.85, b_min: int = 512, budget_tokens: int | None = None,
                 n_score: int = 512, sections=(32, 48, 48), base: float = 10000.0, dtype=None, device="cuda:0",
                 share_heads: bool = False, fold_scale: bool = False):
        import torch
        if mode not in MODES or mode == "dense":
            raise ValueError(f"mode {mode!r} not in {sorted(m for m in MODES if m != 'dense')}")
        self.L, self.Hq, self.Hkv, self.D, self.capacity, self.n_frame = n_layers, Hq, Hkv, D, capacity, n_frame
        self.scale, self.mode, self.gamma, self.b_min = scale, mode, gamma, b_min
        self.fold_scale = fold_scale
        self.q_out_scale = pk.folded_q_scale(scale) if fold_scale else 1.0
        self.call_scale = pk.PC_SCALE_FOLDED if fold_scale else scale
        self.budget_tokens = n_frame if budget_tokens is None else budget_tokens
        self.sections, self.base, self.share_heads = tuple(sections), base, share_heads
        dtype = torch.bfloat16 if dtype is None else dtype
        hsel = 1 if share_heads else Hkv
        self.K = torch.empty((n_layers, Hkv, capacity, D), dtype=dtype, device=device)
        self.V = torch.empty_like(self.K)
        self.pos = torch.empty((n_layers, hsel, capacity, 3), dtype=torch.int32, device=device)
        self.score = torch.empty((n_layers, hsel, capacity), dtype=torch.float32, device=device)
        self.segments: list[tuple[int, int, int, int]] = []
        self.nk = 0
        n_rows = min(n_score, n_frame)
        self.q_rows = ((torch.arange(n_rows, dtype=torch.int64) * n_frame) // n_rows).to(torch.int32).to(device)
        self._ws_score = torch.empty(pk.pc_score_workspace_bytes(Hq, Hkv, n_rows, capacity, share_heads),
                                     dtype=torch.uint8, device=device)
        self._ws_compact = torch.empty(pk.pc_compact_batch_workspace_bytes(n_layers, Hkv, capacity, share_heads),
                                       dtype=torch.uint8, device=device)

    def reserve(self, n: int):
        """Views of the next n free rows of every layer: K, V [L][Hkv][n][D], pos [L][Hsel][n][3]."""
        if self.nk + n > self.capacity:
            raise ValueError(f"cache capacity {self.capacity} < {self.nk} + {n}")
        return pk._rows(self.K, self.V, self.pos, 2, self.nk, n)

    def commit(self, n: int, kind: int, frame: int, rotate_with=None) -> None:
        """Make the n reserved rows part of every layer's cache; rotate_with (int32 [n][3], device)
        rotates the new keys of all layers in place with one call (layers x KV heads as heads)."""
        a = self.nk
        if rotate_with is not None:
            pk.pc_rope3d(self.K.view(self.L * self.Hkv, self.capacity, self.D)[:, a:a + n], rotate_with,
                         self.sections, self.base)
        self.segments.append((a, n, kind, frame))
        self.nk = a + n

    def budgets(self) -> list[int]:
        n_past = pk._past_frames(self.segments)
        if self.mode == "pow":
            per_d = pk.pc_budget(pk.PC_BUDGET_POW, self.n_frame, n_past, self.gamma, self.b_min)
        else:
            per_d = pk.pc_budget(MODES[self.mode], self.budget_tokens, n_past, self.gamma, self.b_min)
        return pk.segment_budgets(self.segments, per_d)

    def attend(self, layer: int, Q, O=None, lse=None):
        """Layer `layer`'s (rotated) queries over its cache as it stands -> O (and the log-sum-exp).  As
        RollingLayer.attend: calls may overlap."""
        return pk.pc_frame_attn(Q, self.K[layer], self.V[layer], self.nk, self.call_scale, O=O, lse=lse)

    def score_layer(self, layer: int, Q, lse=None) -> None:
        """Importance of layer `layer`'s cached keys under Q (lse: the log-sum-exp attend() gave for
        the same queries over the same cache; without it pc_score takes its extra pass)."""
        span = pk._prunable_span(self.segments, self.budgets())
        if span is None:
            return
        pk.pc_score(Q, self.K[layer], self.nk, self.call_scale, lse=lse, score=self.score[layer],
                    share_heads=self.share_heads, ws=self._ws_score, q_rows=self.q_rows, key_range=span)

    def repack(self) -> None:
        """End of the frame step: every layer keeps, per past frame, its top-budget keys; one
        select launch and one gather launch (small caches: one for both) for the whole stack, in place."""
        budgets = self.budgets()
        if pk._prunable_span(self.segments, budgets) is None:
            return
        self.segments, self.nk = pk.pc_compact_batch(self.K, self.V, self.pos, self.score, self.segments, budgets,
                                                     share_heads=self.share_heads, ws=self._ws_compact)


class EvictingStack:
    """The caches of a stack of layers in 4 bits, kept to `budget` rows per head by accumulated attention weight.

    Per step:
        append(layer, K, V, pos)   the step's keys (rotated on insertion) and values enter the layer's cache
        attend(layer, Q)           the step's queries over the cache with the new rows in it; every key's
                                   attention weight is added to `decay` times its sum, in every call
        end_step()                 a cache above its budget loses the rows of least weight, all layers in one call

    Rows below n_anchor (the prompt) and rows whose t coordinate is within recent_t of the newest row's are kept
    whatever their weight.  New rows need that: a row's sum begins at 0 and competes with sums over all earlier steps, so
    without a window (recent_t = 0 and no decay) a step's own rows tend to be the ones that leave, and the cache stays what
    it was when it filled up.  The default window is half of what the anchors leave.  A window is counted in t: where rows
    share one (the tokens of a frame), rows_per_t says how many, and anchors and window together have to fit the budget (of
    more protected rows than that the lowest would stay, and the newest leave).

    attend() applies no mask: the rows of one step see each other.  Text that must not look ahead goes in token by token.

    With the budget reached, a step of n rows goes from budget to budget + n rows and back:
    the same launches every time, so a step can be recorded into a HIP graph and replayed.
    """

    def __init__(self, n_layers: int, Hq: int, Hkv: int, D: int, budget: int, scale: float, step_rows: int = 1,
                 n_anchor: int = 0, recent_t: int | None = None, decay: float = 1.0, sections=(32, 48, 48),
                 base: float = 10000.0, device="cuda:0", share_heads: bool = False, rows_per_t: int = 1):
        import torch
        if not 0 <= n_anchor <= budget or budget < 1 or step_rows < 1 or rows_per_t < 1:
            raise ValueError(f"budget {budget} rows, {n_anchor} of them anchors, {step_rows} new ones per step, {rows_per_t} per t")
        room = budget - n_anchor
        if recent_t is None:
            recent_t = max(room // 2 // rows_per_t, int(room >= rows_per_t))
        if recent_t < 0 or recent_t * rows_per_t > room:
            raise ValueError(f"{n_anchor} anchors and the rows of {recent_t} t, {rows_per_t} each, in a budget of {budget}")
        self.L, self.Hq, self.Hkv, self.D, self.budget, self.scale = n_layers, Hq, Hkv, D, budget, scale
        self.capacity, self.n_anchor, self.recent_t, self.decay = budget + step_rows, n_anchor, recent_t, decay
        self.sections, self.base, self.hsel = tuple(sections), base, 1 if share_heads else Hkv
        # layers x heads are the heads of one cache, so that one call evicts from all of them
        self.cache = pk.q4_cache(n_layers * Hkv, self.capacity, D, device)
        self.pos = torch.zeros((n_layers * self.hsel, self.capacity, 3), dtype=torch.int32, device=device)
        self.weights = torch.zeros((n_layers * self.hsel, self.capacity), dtype=torch.float32, device=device)
        self.nk = 0      # rows when a step begins
        self.n_new = 0   # rows of the step under way
        self._appended: set[int] = set()   # layers that have them

    def layer(self, layer: int):
        """The layer's part: (4-bit cache, pos, weights), as views."""
        if not 0 <= layer < self.L:
            raise ValueError(f"layer {layer} of {self.L}")
        a, s = layer * self.Hkv, layer * self.hsel
        return (tuple(t[a:a + self.Hkv] for t in self.cache), self.pos[s:s + self.hsel], self.weights[s:s + self.hsel])

    def append(self, layer: int, K, V, pos_new, rotate: bool = True) -> None:
        """K, V [Hkv][n][D] of the step become the layer's newest rows, at coordinates pos_new (int32 [n][3], device);
        with `rotate` the keys are rotated in place first.  Every layer of a step appends once, the same number of rows."""
        n = K.shape[1]
        if n < 1:
            raise ValueError("a step appends at least one row")
        if self.nk + n > self.capacity:
            raise ValueError(f"cache capacity {self.capacity} < {self.nk} + {n}")
        if self.n_new not in (0, n):
            raise ValueError(f"{n} rows after {self.n_new} in another layer of the same step")
        if layer in self._appended:
            raise ValueError(f"layer {layer} has its rows of this step; end_step() begins the next one")
        cache, pos, weights = self.layer(layer)
        if rotate:
            pk.pc_rope3d(K, pos_new, self.sections, self.base)
        pk.pc_q4_store(K, V, cache, self.nk, pos_new=pos_new, pos=pos, weights=weights)
        self.n_new = n
        self._appended.add(layer)

    def attend(self, layer: int, Q, O=None, q_pos=None, lse=None, accumulate: bool = True):
        """Queries Q [Hq][n][D] over the layer's cache -> O.  q_pos (int32 [n][3], device): rotate Q in place first."""
        if self._appended and layer not in self._appended:
            raise ValueError(f"layer {layer} has no rows of this step yet")
        if q_pos is not None:
            pk.pc_rope3d(Q, q_pos, self.sections, self.base)
        cache, _, weights = self.layer(layer)
        return pk.pc_q4_attn(Q, cache, self.nk + self.n_new, self.scale, O=O, lse=lse,
                             weights=weights if accumulate else None, decay=self.decay)

    def end_step(self) -> int:
        """The step's rows are part of the cache; above the budget all layers are cut to it.  Returns the rows left."""
        if self._appended and len(self._appended) < self.L:
            raise ValueError(f"layers {sorted(set(range(self.L)) - self._appended)} have no rows of this step")
        self._appended.clear()
        self.nk, self.n_new = self.nk + self.n_new, 0
        if self.nk > self.budget:
            self.nk = pk.pc_q4_evict(self.cache, self.pos, self.weights, self.nk, self.budget, self.n_anchor, self.recent_t)
        return self.nk


class PagedStack:
    """The caches of a stack of layers for several sequences, in pages of one pool.

        a = s.open()                      a sequence without rows
        b, c = s.fork(a, 2)               sequences that begin with a's rows; the pages are common, one that is not full is
                                          copied when either goes on
        s.begin([a, b, c], rows)          a step: new rows of each, one number or one per sequence
        O = s.attend(layer, Q, K, V, pos) their rows, one sequence behind the other: stored in the layer's pages with the
                                          rotation on the way, then attended to; row i of a sequence sees its rows up to its own
        s.close(a)                        its pages are free, but for those that others have in common with it

    Q [Hq][T][D] and K, V [Hkv][T][D] of the step are not rotated yet; Q is rotated in place, and so is K in a step of new
    sequences.  pos int32 [T][3] on the device.  A step in which every sequence is new runs pc_prompt_attn over its own rows,
    every other one pc_page_attn over the pages, with the pages that all of the step's sequences begin with read once for all.

    Every layer of a step is attended to once; a further pass over the same rows says so (again=True) and gives them anew.  A step is not over while some layers have its rows and others do not: begin() refuses
    the next one, and if close() ends it, its sequences can only be closed.  (A step that no layer is attended to stands for one
    that a graph replays; layers that have been recorded are taken to have theirs.)

    The pages of a step are decided in begin(), on the host; attend() only launches.  With the same sequences and one row each, a
    step's launches are the same while n_shared and max_len are, so that attend() can be recorded into a HIP graph: begin()
    writes the lengths and tables into the same device buffers before every replay (max_len: a bound for as long as the graph
    is to last).
    """

    def __init__(self, n_layers: int, Hq: int, Hkv: int, D: int, n_pages: int, scale: float, page_rows: int = 64,
                 max_seqs: int = 64, max_rows: int | None = None, sections=(32, 48, 48), base: float = 10000.0, dtype=None,
                 device="cuda:0", fold_scale: bool = True):
        import torch
        if n_layers < 1 or Hkv < 1 or Hq < 1 or Hq % Hkv or n_pages < 1 or max_seqs < 1:
            raise ValueError(f"{n_layers} layers of {Hq}/{Hkv} heads, {n_pages} pages, {max_seqs} sequences")
        self.L, self.Hq, self.Hkv, self.D, self.page_rows, self.scale = n_layers, Hq, Hkv, D, page_rows, scale
        self.sections, self.base = tuple(sections), base
        # the softmax scale rides on the query rotation (see RollingLayer)
        self.q_out_scale = pk.folded_q_scale(scale) if fold_scale else 1.0
        self.call_scale = pk.PC_SCALE_FOLDED if fold_scale else scale
        pools = pk.page_cache(n_layers * n_pages, Hkv, page_rows, D, dtype, device)
        self.K, self.V = (t.view(n_layers, n_pages, Hkv, page_rows, D) for t in pools)
        max_rows = n_pages * page_rows if max_rows is None else max_rows
        self.width = max(1, -(-max_rows // page_rows))     # pages of a sequence at most
        self.table = torch.zeros((max_seqs, self.width), dtype=torch.int32, device=device)
        self.lens = torch.zeros((max_seqs,), dtype=torch.int32, device=device)
        self.shared = torch.zeros((self.width,), dtype=torch.int32, device=device)
        self._free = list(range(n_pages - 1, -1, -1))
        self._users = [0] * n_pages                        # sequences that a page belongs to
        self._pages: dict[int, list[int]] = {}
        self._rows: dict[int, int] = {}
        self._next = 0
        self._step = None                                  # (sequences, offsets, one number of rows each, fresh)
        self._growing: list[int] = []                      # the step's sequences with new rows
        self._attended: set[int] = set()                   # layers that have them
        self._recorded: set[int] = set()                   # layers that a graph may attend to
        self._torn: set[int] = set()                       # sequences with rows that not every layer has
        self.n_shared = self.max_len = 0

    # ---- sequences (host only) ----------------------------------------------------------------
    def open(self) -> int:
        self._next += 1
        self._pages[self._next], self._rows[self._next] = [], 0
        return self._next

    def rows(self, seq: int) -> int:
        """Rows of a sequence."""
        return self._rows[self._known(seq)]

    def free_pages(self) -> int:
        return len(self._free)

    def _known(self, seq: int) -> int:
        if seq not in self._rows:
            raise ValueError(f"sequence {seq} is not open")
        return seq

    def _whole(self, seq: int) -> int:
        if self._known(seq) in self._torn:
            raise ValueError(f"sequence {seq} has rows that not every layer has: it can only be closed")
        return seq

    def _missing(self) -> list[int]:
        """Layers that have not got the step's rows, if others have."""
        if not self._attended or not self._growing:
            return []
        return [layer for layer in range(self.L) if layer not in self._attended and layer not in self._recorded]

    def fork(self, seq: int, n: int = 1) -> list[int]:
        """n further sequences that begin with seq's rows."""
        self._whole(seq)
        out = []
        for _ in range(n):
            new = self.open()
            self._pages[new], self._rows[new] = list(self._pages[seq]), self._rows[seq]
            for p in self._pages[new]:
                self._users[p] += 1
            if seq in self._growing:
                self._growing.append(new)
            out.append(new)
        return out

    def close(self, seq: int) -> None:
        """The step under way is over, too."""
        for p in self._pages.pop(self._known(seq)):
            self._users[p] -= 1
            if self._users[p] == 0:
                self._free.append(p)
        del self._rows[seq]
        if self._missing():
            self._torn.update(self._growing)
        self._torn &= self._rows.keys()
        self._step, self._growing = None, []

    # ---- one step -----------------------------------------------------------------------------
    def begin(self, seqs, rows=1, max_len: int | None = None) -> None:
        """The step's sequences and how many new rows each of them gets.  max_len: a bound on the rows of any of them, for
        attend() to lay its work out for (None: the longest)."""
        import torch
        if self._missing():
            raise ValueError(f"layers {self._missing()} have not been attended to in the step under way")
        seqs = [self._whole(q) for q in seqs]
        counts = [int(rows)] * len(seqs) if isinstance(rows, int) else [int(r) for r in rows]
        if not seqs or len(set(seqs)) < len(seqs) or len(seqs) > self.table.shape[0] or len(counts) != len(seqs) or min(counts) < 0:
            raise ValueError(f"a step of {len(seqs)} sequences (each once, {self.table.shape[0]} at most), new rows {rows}")
        R = self.page_rows
        # what the step needs: whole new pages, and a copy of a page that is not full and not the sequence's alone (one that
        # several of the step's sequences leave for copies may keep its last user)
        longest = max(self._rows[q] + n for q, n in zip(seqs, counts))
        if max_len is not None and not longest <= max_len <= self.width * R:
            raise ValueError(f"max_len {max_len}: {longest} rows, {self.width * R} at most")
        need, users = 0, {}
        for q, n in zip(seqs, counts):
            have, after = self._rows[q], self._rows[q] + n
            if -(-after // R) > self.width:
                raise ValueError(f"sequence {q}: {after} rows, {self.width * R} at most")
            need += -(-after // R) - len(self._pages[q])
            if n and have % R:
                p = self._pages[q][-1]
                if users.setdefault(p, self._users[p]) > 1:
                    users[p] -= 1
                    need += 1
        if need > len(self._free):
            raise ValueError(f"{need} pages needed, {len(self._free)} free")
        fresh = all(self._rows[q] == 0 for q in seqs)
        copies = []
        for q, n in zip(seqs, counts):
            pages = self._pages[q]
            if n and self._rows[q] % R and self._users[pages[-1]] > 1:
                p = self._free.pop()
                copies.append((pages[-1], p))
                self._users[pages[-1]] -= 1
                self._users[p], pages[-1] = 1, p
            self._rows[q] += n
            while len(pages) * R < self._rows[q]:
                p = self._free.pop()
                self._users[p] = 1
                pages.append(p)
        device = self.K.device
        if copies:
            old, new = (torch.tensor(v, device=device) for v in zip(*copies))
            for t in (self.K, self.V):
                t[:, new] = t[:, old]
        lists = [self._pages[q] for q in seqs]
        common = 0
        if len(seqs) > 1:
            while all(len(v) > common and v[common] == lists[0][common] for v in lists):
                common += 1
        # (a page that is common and not full has no new rows in it: every sequence of it ends there alike)
        self.n_shared = min([common * R] + [self._rows[q] for q in seqs])
        self.max_len = max(1, longest if max_len is None else int(max_len))
        n_cols = max(1, max(len(v) for v in lists))
        host = torch.zeros((len(seqs), n_cols + 1), dtype=torch.int32)
        for i, v in enumerate(lists):
            host[i, :len(v)] = torch.tensor(v, dtype=torch.int32)
            host[i, n_cols] = self._rows[seqs[i]]
        host = host.to(device)
        self.table[:len(seqs), :n_cols] = host[:, :n_cols]
        self.lens[:len(seqs)] = host[:, n_cols]
        self.shared[:n_cols] = host[0, :n_cols]
        offs = [0]
        for n in counts:
            offs.append(offs[-1] + n)
        even = len(set(counts)) == 1
        self._step = (len(seqs), offs, even, fresh)
        self._growing = [q for q, n in zip(seqs, counts) if n]
        self._attended.clear()

    def attend(self, layer: int, Q, K, V, pos, O=None, lse=None, again: bool = False):
        """The step's rows of one layer: into the pages, and their attention -> O.  again: they take the place of those that the layer
        has of this step (not rotated yet either)."""
        import torch
        if self._step is None:
            raise ValueError("begin() names the step's sequences first")
        if not 0 <= layer < self.L:
            raise ValueError(f"layer {layer} of {self.L}")
        n, offs, even, fresh = self._step
        if Q.shape[1] != offs[-1]:
            raise ValueError(f"{Q.shape[1]} rows in a step of {offs[-1]}")
        if layer in self._attended and self._growing and not again and not torch.cuda.is_current_stream_capturing():
            raise ValueError(f"layer {layer} has the rows of this step; begin() names the next one")
        table, lens, pages = self.table[:n], self.lens[:n], (self.K[layer], self.V[layer])
        o = None if even else offs
        pk.pc_page_store(K, V, pages, table, lens, offs=o, pos=pos, sections=self.sections, base=self.base,
                         K_out=K if fresh else None, Q=Q, Q_out=Q, out_scale=self.q_out_scale)
        (self._recorded if torch.cuda.is_current_stream_capturing() else self._attended).add(layer)
        if O is None:
            O = torch.empty(Q.shape, dtype=Q.dtype, device=Q.device)
        if fresh:
            return pk.pc_prompt_attn(Q, K, V, self.call_scale, offs, O=O, lse=lse)
        return pk.pc_page_attn(Q, pages, table, lens, self.max_len, self.call_scale, offs=o,
                               shared=self.shared if self.n_shared else None, n_shared=self.n_shared, O=O, lse=lse)
