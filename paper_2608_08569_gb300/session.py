"""Host-side driver of the three C-ABI calls for one batch of sequences.

A ``Session`` owns the device cache (K, V, score, pos, len; or, paged, the page pools, the page
table and the free-page stack), runs stage 1 once per request, then one decode step per
generated token over all layers and an eviction every ``interval`` steps. It keeps a host-side
upper bound on the cache length (read back once after stage 1) so that every decode launch is
sized without a device-to-host sync; the decode loop of a request can therefore be captured once
in a CUDA graph and replayed (``capture_loop``).

A later turn of the conversation joins a session by ``extend``: its rows are rotated, appended behind the rows that
the cache has kept, and attend over all of them.

With ``kv_bits=4`` the session's cache holds its rows in 4 bits per channel: stage 1 runs into a staging cache of
plain rows, which is packed right after it, and decode steps and evictions work on the packed rows. The staging
rows are needed during ``prefill`` alone: it makes them and gives them back to torch's allocator. Rows that the caller
keeps (``staging``) may serve several sessions: each prefill on them waits for the one before, on whatever stream.
"""
from __future__ import annotations

import threading

import torch

from . import _native as N


class _Turn:
    """Whose prefill has a staging cache that sessions share: one at a time. `done` is recorded behind the last one's
    packing."""

    def __init__(self):
        self.lock = threading.Lock()
        self.done = None


def _torch_stream(stream):
    """A call's `stream` (None, or anything with a cuda_stream) for torch's own work."""
    if stream is None or hasattr(stream, "wait_event"):
        return stream
    return torch.cuda.ExternalStream(stream.cuda_stream)


class Session:
    """`budget` holds one budget per sequence, or per sequence and layer ([B][L]); `history` and
    `compaction` select the eviction policy (see voxzip_evict_ex). `kv_bits` is 16 (rows in the descriptor's
    dtype) or 4; `staging`, with 4, a dict of k and v [B][L][Hkv][C][D] that stage 1 may overwrite (the same dict for
    every session that shares them: it holds their order too, under "turn")."""

    def __init__(self, desc: N.CacheDesc, budget, gamma: float, *, sink: int = 4, recent_frac: float = 0.2,
                 history: bool = True, compaction: str = "ordered", device="cuda", cache=None,
                 pages: int | None = None, kv_bits: int = 16, staging=None):
        if kv_bits not in (4, 16):
            raise ValueError("kv_bits must be 4 or 16")
        if kv_bits == 4 and pages is not None:
            raise ValueError("a paged cache holds its rows in the descriptor's dtype: kv_bits=4 needs pages=None")
        self.kv_bits = kv_bits
        self.staging = staging
        self.desc = desc
        self.device = torch.device(device)
        self.gamma = float(gamma)
        self.sink = int(sink)
        self.recent_frac = float(recent_frac)
        self.history = bool(history)
        self.compaction = compaction
        self.budget = torch.tensor(budget, dtype=torch.int32, device=self.device)
        self.budget_host = [int(b) for b in self.budget.flatten().tolist()]
        self.paged = pages is not None
        if cache is not None:
            self.cache = cache
        elif self.paged:
            self.cache = N.allocate_paged_cache(desc, pages, self.device)
        elif kv_bits == 4:
            self.cache = N.allocate_q4_cache(desc, self.device)
        else:
            self.cache = N.allocate_cache(desc, self.device)
        self.n_max = 0
        self.workspace = None

    # stage 1 -------------------------------------------------------------------------------------
    def prefill(self, k_prefill, v_prefill, in_len, audio_begin, audio_len, span_off, span_start, span_end,
                span_groups, *, anchor_k=None, anchor_v=None, slot_map=None, stream=None, read_back=True):
        """Stage-1 fusion of the prefilled cache (all device tensors, see voxzip_anchor_fuse)."""
        c = self.cache
        need = N.voxzip_anchor_fuse_workspace_size(self.desc, k_prefill.shape[3], span_start.numel())
        if self.workspace is None or self.workspace.numel() < need:
            with torch.cuda.stream(_torch_stream(stream)):  # the launches' own, as it is what they use it on
                self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        if self.paged:
            N.voxzip_anchor_fuse_paged(self.desc, c, k_prefill, v_prefill, in_len, audio_begin, audio_len, span_off,
                                       span_start, span_end, span_groups, slot_map=slot_map, anchor_k=anchor_k,
                                       anchor_v=anchor_v, workspace=self.workspace, stream=stream)
        else:
            def launch(rows):
                N.voxzip_anchor_fuse(self.desc, k_prefill, v_prefill, in_len, audio_begin, audio_len, span_off,
                                     span_start, span_end, span_groups, rows["k"], rows["v"], c["score"], c["pos"],
                                     c["len"], slot_map=slot_map, anchor_k=anchor_k, anchor_v=anchor_v,
                                     workspace=self.workspace, stream=stream)
                if self.kv_bits == 4:
                    N.voxzip_q4_pack(self.desc, c, 0, self.desc.layers, rows["k"], rows["v"], stream=stream)

            if self.kv_bits == 4:
                self._staged(launch, stream)
            else:
                launch(c)
        if read_back:
            with torch.cuda.stream(_torch_stream(stream)):
                self.n_max = int(c["len"].max().item())
        else:
            self.n_max = int(k_prefill.shape[3])  # stage 1 never lengthens a prompt

    def _staged(self, launch, stream):
        """Runs launch(rows) with rows for stage 1 that nothing else uses until it is done on the GPU."""
        stream = _torch_stream(stream)
        with torch.cuda.stream(stream):  # memory made here is the launches' own: who gets it next is ordered behind them
            rows = self.staging
            if rows is None:
                new = lambda: torch.empty(self.desc._rows, dtype=self.desc.dtype, device=self.device)  # noqa: E731
                rows = dict(k=new(), v=new())
            alone = self.staging is None or torch.cuda.is_current_stream_capturing()
        if alone:  # (a graph's replays are ordered by who replays them)
            launch(rows)
        else:
            turn = self.staging.setdefault("turn", _Turn())
            with turn.lock:
                at = stream if stream is not None else torch.cuda.current_stream()
                if turn.done is not None:
                    at.wait_event(turn.done)
                try:
                    launch(self.staging)
                finally:
                    turn.done = at.record_event()

    # a later turn -------------------------------------------------------------------------------
    def extend(self, q, k, v, new_pos, seq_off, out, *, max_rows: int, rotary=None, positions=None, q_out=None,
               sm_scale: float = 0.0, layer_begin=0, layer_count=None, stream=None):
        """A turn's prompt for a layer range (all layers by default): packed rows q, k and v [layers][tokens][heads][D] of
        every sequence (see voxzip_append) join its units, k and q rotated on the way, and the queries' causal attention
        over all rows goes to `out`. `max_rows` bounds the tokens of one sequence (0: the packed tokens do). With a rotation
        and no `q_out` the rotated queries live for the call."""
        if self.kv_bits != 16:
            raise ValueError("extend needs a cache whose rows are in the descriptor's dtype (kv_bits=16)")
        if max_rows < 0:
            raise ValueError("max_rows must bound the tokens of a sequence")
        c = self.cache
        lc = self.desc.layers if layer_count is None else layer_count
        tokens = k.shape[1]
        max_rows = min(int(max_rows), tokens) if max_rows else tokens
        longest = min(self.n_max + max_rows, self.desc.capacity)
        if rotary is not None and q_out is None:
            with torch.cuda.stream(_torch_stream(stream)):  # the launches' own, as it is what they use it on
                q_out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        turn = dict(rotary=rotary, positions=positions, max_rows=max_rows, stream=stream)
        if q_out is not None:
            turn.update(q=q, q_out=q_out)
        attend = dict(sm_scale=sm_scale, max_rows=max_rows, max_len=longest, stream=stream)
        queries = q if q_out is None else q_out
        if self.paged:
            N.voxzip_append_paged(self.desc, c, layer_begin, lc, k, v, new_pos, seq_off, **turn)
            N.voxzip_prompt_attention_paged(self.desc, c, layer_begin, lc, queries, seq_off, out, **attend)
        else:
            N.voxzip_append(self.desc, layer_begin, lc, k, v, new_pos, seq_off, c["k"], c["v"], c["score"], c["pos"],
                            c["len"], **turn)
            N.voxzip_prompt_attention(self.desc, layer_begin, lc, queries, seq_off, c["k"], c["v"], c["len"], out, **attend)
        if layer_begin + lc == self.desc.layers:
            self.n_max = longest

    # stage 2 -------------------------------------------------------------------------------------
    def decode(self, q, k_new, v_new, new_pos, out, *, layer_begin=0, layer_count=None, stream=None):
        """One decode step for a layer range (all layers by default)."""
        c = self.cache
        lc = self.desc.layers if layer_count is None else layer_count
        if self.paged:
            N.voxzip_decode_step_paged(self.desc, c, layer_begin, lc, q, k_new, v_new, new_pos, self.gamma, out,
                                       max_len=self.n_max + 1, stream=stream)
        elif self.kv_bits == 4:
            N.voxzip_decode_step_q4(self.desc, c, layer_begin, lc, q, k_new, v_new, new_pos, self.gamma, out,
                                    max_len=self.n_max + 1, stream=stream)
        else:
            N.voxzip_decode_step(self.desc, layer_begin, lc, q, k_new, v_new, new_pos, c["k"], c["v"], c["score"],
                                 c["pos"], c["len"], self.gamma, out, max_len=self.n_max + 1, stream=stream)
        if layer_begin + lc == self.desc.layers:
            self.n_max += 1

    def evict(self, *, layer_begin=0, layer_count=None, stream=None):
        c = self.cache
        lc = self.desc.layers if layer_count is None else layer_count
        if self.paged:
            N.voxzip_evict_paged(self.desc, c, layer_begin, lc, self.budget, sink=self.sink,
                                 recent_frac=self.recent_frac, history=self.history, compaction=self.compaction,
                                 stream=stream)
        elif self.kv_bits == 4:
            N.voxzip_evict_q4(self.desc, c, layer_begin, lc, self.budget, sink=self.sink, recent_frac=self.recent_frac,
                              history=self.history, compaction=self.compaction, stream=stream)
        elif self.history and self.compaction == "ordered" and self.budget.dim() == 1:
            N.voxzip_evict(self.desc, layer_begin, lc, c["k"], c["v"], c["score"], c["pos"], c["len"], self.budget,
                           sink=self.sink, recent_frac=self.recent_frac, stream=stream)
        else:
            N.voxzip_evict_ex(self.desc, layer_begin, lc, c["k"], c["v"], c["score"], c["pos"], c["len"],
                              self.budget, sink=self.sink, recent_frac=self.recent_frac, history=self.history,
                              compaction=self.compaction, stream=stream)
        if layer_begin + lc == self.desc.layers:
            self.n_max = min(self.n_max, max(self.budget_host))

    # decode loop in a CUDA graph ---------------------------------------------------------------------
    def capture_loop(self, q, k_new, v_new, new_pos, out, interval: int, *, launch_events=None,
                     segments: bool = False):
        """Captures the decode loop of one request: step t (1-based) decodes with q[t-1], k_new[t-1],
        v_new[t-1], new_pos[t-1] into out[t-1], and evicts when t % interval == 0. Call it right
        after a prefill of the request's shape (it starts from that cache length bound); replaying
        the returned graph after each later prefill of the same shape runs the whole loop with one
        host call. With `launch_events` (a list), timing events (created with external=True) are
        captured too and appended as (kind, start, end, launches): around every decode launch
        ("decode", ..., 1), or with `segments` around each run of decode launches between two
        evictions ("decode", ..., steps in the run: the launches keep overlapping one another as in
        the plain graph), and around every eviction ("evict", ..., 1). The graph records into them
        on every replay, so they must outlive it."""
        n0 = self.n_max
        stream = torch.cuda.Stream(device=self.device)
        stream.wait_stream(torch.cuda.current_stream(self.device))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            with torch.cuda.graph(graph, stream=stream):
                steps = q.shape[0]
                mk = lambda: (torch.cuda.Event(enable_timing=True, external=True),
                              torch.cuda.Event(enable_timing=True, external=True))
                ev, run = None, 0
                for t in range(1, steps + 1):
                    if launch_events is not None and ev is None:
                        ev = mk()
                        ev[0].record()
                    self.decode(q[t - 1], k_new[t - 1], v_new[t - 1], new_pos[t - 1], out[t - 1])
                    run += 1
                    if ev is not None and (not segments or t % interval == 0 or t == steps):
                        ev[1].record()
                        launch_events.append(("decode", ev[0], ev[1], run))
                        ev, run = None, 0
                    if t % interval == 0:
                        eev = None
                        if launch_events is not None:
                            eev = mk()
                            eev[0].record()
                        self.evict()
                        if eev is not None:
                            eev[1].record()
                            launch_events.append(("evict", eev[0], eev[1], 1))
        torch.cuda.current_stream(self.device).wait_stream(stream)
        self.n_max = n0
        return graph
