"""Loops over layers built from the library's calls (Sec. 3.4).

LayerLoop (attention only): per layer the chunk store arrives through the layer-wise preloader,
cached keys are re-positioned, the chosen tokens are recomputed and attended, the question's
attention to every chunk feeds Algorithm 1, and once a request's focused chunks are settled the
other chunks of that request are no longer recomputed.  The batch holds ONE layer's per-token
tensors; a caller that has a different set per layer installs it through the loop's layer_inputs
hook.

DecoderLoop (whole layers): the hidden states of the chosen rows pass through normalisation,
projections, the partial prefill and the feed-forward network of every layer.

AnswerLoop: the answers behind a DecoderLoop's prefill, token by token over the pages it left.

Argument marshalling and call order only; every step runs in libcachecraft.
"""
from __future__ import annotations

import math
from typing import Callable, List, Optional, Sequence

import numpy as np
import torch

from .binding import CC_IMPL_AUTO, FocusTracker, Preloader, preload_depth
from .pipeline import DeviceBatch, product_workspace


class DecoderLoop:
    """The hidden states of the chosen rows through whole decoder layers (Sec. 2.1, Sec. 3.4.3): per
    layer cc_rms_norm -> cc_qkv_project -> cc_sparse_prefill over the re-positioned chunk-caches ->
    cc_linear (output projection + residual) -> cc_rms_norm -> cc_gated_linear -> cc_linear (down
    projection + residual).  The rows are chosen once, before the first layer, from the workload's
    per-token queries (cc_select); every layer sees the same synthetic chunk store.
    weights: one workload.LayerWeights per layer.
    window: if given, the question's attention to every chunk (a by-product of the attention call)
    feeds Algorithm 1 in every layer; once a request's focused chunks are settled, the rows of its
    other chunks leave the list (Sec. 3.2.2) and the surviving rows' hidden states are compacted."""

    def __init__(self, w, weights: Sequence, window: Optional[int] = None, impl: int = CC_IMPL_AUTO,
                 device: str = "cuda", preload: bool = False, depth: int = 1, answer_tokens: int = 0):
        """preload: every layer's chunk store comes from pinned host memory through the layer-wise
        preloader (Algorithm 2), `depth` layers ahead of the one being computed.
        answer_tokens: if given, every layer keeps request pages of its own, with room for that many more tokens
        of each request, so that an AnswerLoop can go on from them (not with preload, whose slots hold the
        values of later layers by then)."""
        assert w.hidden is not None, "the workload must carry hidden states"
        assert not (preload and answer_tokens), "the preloader's slots do not keep a layer's values for the answer"
        self.w, self.window, self.answer_tokens = w, window, answer_tokens
        spare = w.n_requests * ((answer_tokens + 15) // 16 + 1) if answer_tokens else 0
        self.batch = DeviceBatch(w, device=device, impl=impl, spare_blocks=spare)
        b = self.batch
        self.turn = 0                                                  # prefills and answers that have begun on the pages
        self.pages = [(b.k_req, b.v_req, b.v_map)] + [(b.k_req.clone(), b.v_req.clone(), b.v_map.clone())
                                                      for _ in weights[1:]] if answer_tokens else []
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device).to(b.dt)
        self.weights = [{k: up(getattr(lw, k)) for k in ("gain_attn", "gain_ffn", "w_qkv", "w_o", "w_gate", "w_up", "w_down")}
                        for lw in weights]
        self.eps = [float(lw.eps) for lw in weights]
        n, hidden, ffn = max(1, b.n_q_tot), w.hidden.shape[1], weights[0].w_gate.shape[0]
        mk = lambda cols: torch.empty((n, cols), dtype=b.dt, device=device)
        self.h, self.h1, self.x, self.act, self.h_alt = mk(hidden), mk(hidden), mk(hidden), mk(ffn), mk(hidden)
        n_attn = w.spec.n_q_heads * w.spec.head_dim
        self.ws_products = product_workspace(b.n_q_tot, device, lambda r: b.ctx.qkv_project_workspace_bytes(r, hidden),
                                             lambda r: b.ctx.linear_workspace_bytes(r, n_attn, hidden),
                                             lambda r: b.ctx.linear_workspace_bytes(r, ffn, hidden))
        seg = w.segments
        self.chunk_segs = [[s for s in range(int(w.req_seg_off[r]), int(w.req_seg_off[r + 1])) if seg[s][1] == 0]
                           for r in range(w.n_requests)]
        self.trackers = [FocusTracker(max(1, len(c)), window) for c in self.chunk_segs] if window else []
        self.budget = np.array(seg[:, 5], dtype=np.int64)
        self.stop_layer: List[Optional[int]] = [None] * w.n_requests
        self.focused: List[Optional[List[int]]] = [None] * w.n_requests
        self.keep_idx = torch.zeros(n, dtype=torch.int32, device=device)
        self.pre = None
        if preload:
            n_layers = len(weights)
            self.k_host, self.v_host = b.k_store.cpu().pin_memory(), b.v_store.cpu().pin_memory()
            n_slots = min(depth + 1, n_layers)
            self.slots = [(torch.empty_like(b.k_store), torch.empty_like(b.v_store)) for _ in range(n_slots)]
            self.pre = (Preloader(n_layers, depth, n_slots), Preloader(n_layers, depth, n_slots))
            for l in range(n_layers):
                self.pre[0].set_layer(l, self.k_host, self.slots[l % n_slots][0])
                self.pre[1].set_layer(l, self.v_host, self.slots[l % n_slots][1])

    def _shift(self, l):
        """Layer l's chunk-caches (waiting for the preloader's copy if there is one), re-positioned."""
        b = self.batch
        if self.pages:
            b.k_req, b.v_req, b.v_map = self.pages[l]
        if self.pre is not None:
            self.pre[0].acquire(l); self.pre[1].acquire(l)
            b.k_store, b.v_store = self.slots[l % len(self.slots)]
        b.rope_shift()
        if self.pre is not None:                               # the key slot is free once the shift has read it;
            self.pre[0].release(l)                             # the values are read by the attention, unless copied
            if not b.cow:
                self.pre[1].release(l)

    def _drop_rows(self, new_budget):
        """New budgets: rebuild the row list (same scores, same order) and compact the hidden states."""
        b = self.batch
        old = np.array(getattr(b, "_seg_host", self.w.segments), copy=True)
        b.set_budget(new_budget)
        new = b._seg_host
        keep = np.concatenate([np.arange(int(o[7]), int(o[7]) + int(nw[5])) for o, nw in zip(old, new)] or
                              [np.zeros(0)]).astype(np.int32)
        assert len(keep) == b.n_q_tot
        if b.n_q_tot:
            self.keep_idx[: len(keep)].copy_(torch.from_numpy(keep))
            b.ctx.gather_rows(self.h, self.keep_idx[: len(keep)], self.h_alt[: len(keep)])
            self.h, self.h_alt = self.h_alt, self.h
            b.select_from_scores()

    def run(self, keep: bool = False):
        """Returns one record per layer (ms, rows; with keep also h_in, out, lse, h1, h2 as numpy arrays)."""
        b = self.batch
        self.turn += 1
        self._shift(0)
        b.select()
        records = []
        for l, lw in enumerate(self.weights):
            n = b.n_q_tot
            if n == 0:
                break
            t0 = torch.cuda.Event(enable_timing=True); t1 = torch.cuda.Event(enable_timing=True)
            t0.record()
            h, h1, x, act = self.h[:n], self.h1[:n], self.x[:n], self.act[:n]
            o2 = b.out[:n].view(n, -1)
            if l == 0:
                b.ctx.gather_rows(b.hidden, b.q_row[:n], h)
            else:
                self._shift(l)
            rec = {"layer": l + 1, "rows": n}
            if keep:
                rec["h_in"] = h.float().cpu().numpy()
                rec["cu_q"] = np.array(getattr(b, "cu_q_host", self.w.cu_q), copy=True)
            b.ctx.rms_norm(h, lw["gain_attn"], self.eps[l], x)
            b.ctx.qkv_project(x, lw["w_qkv"], b.q_c[:n], b.k_c[:n], b.v_c[:n], workspace=self.ws_products)
            if self.window:
                mass = b.sparse_prefill_mass()
            else:
                b.sparse_prefill()
            if self.pre is not None and b.cow:
                self.pre[1].release(l)
            b.ctx.linear(o2, lw["w_o"], h1, residual=h, workspace=self.ws_products)
            b.ctx.rms_norm(h1, lw["gain_ffn"], self.eps[l], x)
            b.ctx.gated_linear(x, lw["w_gate"], lw["w_up"], act)
            b.ctx.linear(act, lw["w_down"], h, residual=h1, workspace=self.ws_products)
            t1.record()
            rec["_events"] = (t0, t1)
            if keep:
                torch.cuda.synchronize()
                rec.update(out=b.out[:n].float().cpu().numpy(), lse=b.lse[:n].cpu().numpy(),
                           h1=h1.float().cpu().numpy(), h2=h.float().cpu().numpy())
            if self.window:
                m = mass.cpu().numpy()                     # (synchronises; Algorithm 1 runs on the host)
                rec["mass"] = m[: len(self.w.segments)].copy()
                changed = False
                for r, segs in enumerate(self.chunk_segs):
                    if self.stop_layer[r] is not None or not segs:
                        continue
                    stop, focused = self.trackers[r].update([float(m[s]) for s in segs])
                    if stop:
                        self.stop_layer[r], self.focused[r] = l + 1, focused
                        for i, sgi in enumerate(segs):
                            if i not in focused and self.budget[sgi]:
                                self.budget[sgi] = 0
                                changed = True
                rec["stop_layer"] = list(self.stop_layer)
                rec["focused"] = [None if f is None else list(f) for f in self.focused]
                if changed and l + 1 < len(self.weights):
                    self._drop_rows(self.budget)
            records.append(rec)
        torch.cuda.synchronize()
        for rec in records:
            t0, t1 = rec.pop("_events")
            rec["ms"] = t0.elapsed_time(t1)
        return records

    def close(self):
        for t in self.trackers:
            t.close()
        self.trackers = []
        if self.pre is not None:
            for p in self.pre:
                p.close()
            self.pre = None


class AnswerLoop:
    """Answers behind a DecoderLoop's prefill (made with answer_tokens), one token per request and step: cc_sample from the last row's logits ->
    cc_extend_segments (a token more per request) -> the token's embedding -> per layer cc_rms_norm -> cc_qkv_project ->
    cc_append_attention over the layer's pages -> cc_linear -> cc_rms_norm -> cc_gated_linear -> cc_linear, -> logits.
    embed [vocab, hidden], gain_out [hidden], w_out [vocab, hidden]: embedding, last normalisation, output projection (numpy).
    temperature, top_k, top_p, min_p: one value, or one per request; None: off.  stop: a request that draws this token
    gets no further one; neither does one whose logits are all -infinity or NaN, or for which no row is left.  Nothing of a step
    depends on the host, so graph=True captures one and replays it.
    Another answer to the same prompts is another AnswerLoop, which takes the pages over: the one before it cannot go on."""

    def __init__(self, loop: DecoderLoop, embed, gain_out, w_out, eps: float = 1.0e-5, temperature=None, top_k=None, top_p=None,
                 min_p=None, stop: Optional[int] = None):
        assert loop.answer_tokens > 0, "the DecoderLoop must keep its pages (answer_tokens)"
        if loop.turn == 0:
            raise ValueError("AnswerLoop: the DecoderLoop has not run yet")
        loop.turn += 1
        self.turn = loop.turn
        self.loop, self.eps, self.stop = loop, float(eps), stop
        w, b = loop.w, loop.batch
        self.b, self.n = b, w.n_requests
        dev = b.device
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev).to(b.dt)
        self.embed, self.gain_out, self.w_out = up(embed), up(gain_out), up(w_out)
        n, hidden, vocab = self.n, self.embed.shape[1], self.w_out.shape[0]
        ffn = loop.weights[0]["w_gate"].shape[0]
        hq, hkv, d = w.spec.n_q_heads, w.spec.n_kv_heads, w.spec.head_dim
        # tables: every request's last segment moves to a place with room for the answer, its pages stay
        seg, last = np.array(w.segments, copy=True), np.asarray(w.req_seg_off[1:]) - 1
        assert (np.diff(w.req_seg_off) > 0).all() and (seg[last, 1] == 1).all(), "every request needs a question, behind which the answer comes"
        pages = lambda t: (t + 15) // 16
        cap = pages(seg[:, 3])
        tab = [np.asarray(w.req_tab)]
        at = len(w.req_tab)
        for s in last:
            held, room = int(cap[s]), int(pages(seg[s, 3] + loop.answer_tokens))
            tab.append(np.concatenate([w.req_tab[seg[s, 4]: seg[s, 4] + held], np.full(room - held, -1)]))
            seg[s, 4], cap[s] = at, room
            at += room
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)
        self.segs, self.tab_cap, self.block_tab = i32(seg), i32(cap), i32(np.concatenate(tab))
        self.free = i32(np.arange(w.n_req_blocks, b.k_req.shape[0]))
        self.free_left = self.free.clone()
        self.last_seg = torch.from_numpy(last.astype(np.int64)).to(dev)
        self.n_new = i32(np.zeros(len(seg)))
        self.cu_q, self.counts = i32(np.zeros(n + 1)), i32(np.zeros(4))
        self.q_pos, self.slot_map, self.row_req, self.last_row, self.status = (i32(np.zeros(n)) for _ in range(5))
        self.max_ctx = max(w.context_len(r) for r in range(n)) + loop.answer_tokens
        self.max_segs = int(np.diff(w.req_seg_off).max())
        # rows of a step
        mk = lambda cols: torch.zeros((n, cols), dtype=b.dt, device=dev)
        self.h, self.h1, self.x, self.act, self.h_last, self.logits = mk(hidden), mk(hidden), mk(hidden), mk(ffn), mk(hidden), mk(vocab)
        self.q, self.k, self.v, self.o = (torch.zeros((n, heads, d), dtype=b.dt, device=dev) for heads in (hq, hkv, hkv, hq))
        ctx = b.ctx
        self.ws_products = product_workspace(n, dev, lambda r: ctx.qkv_project_workspace_bytes(r, hidden),
                                             lambda r: ctx.linear_workspace_bytes(r, hq * d, hidden), lambda r: ctx.linear_workspace_bytes(r, ffn, hidden),
                                             lambda r: ctx.linear_workspace_bytes(r, hidden, vocab))
        self.ws = torch.empty(max(256, ctx.extend_segments_workspace_bytes(len(seg), n), ctx.sample_workspace_bytes(n, vocab),
                                  ctx.append_attention_workspace_bytes(n, 1, n, self.max_ctx, self.max_segs)), dtype=torch.uint8, device=dev)
        one = lambda a, t: None if a is None else torch.as_tensor(np.broadcast_to(np.asarray(a, dtype=t), (n,)).copy()).to(dev)
        self.settings = dict(temperature=one(temperature, np.float32), top_k=one(top_k, np.int32), top_p=one(top_p, np.float32),
                             min_p=one(min_p, np.float32))
        self.u = torch.zeros(n, dtype=torch.float32, device=dev)
        self.token, self.n_kept = i32(np.zeros(n)), i32(np.zeros(n))
        self.logprob = torch.zeros(n, dtype=torch.float32, device=dev)
        self.alive = torch.ones(n, dtype=torch.bool, device=dev)
        self.drawn = 0                                                 # tokens drawn; all but the last have been through the layers
        self.h_last.copy_(loop.h[b.cu_q[1:].long() - 1])               # the prefill's last row of every request
        self._logits()

    def _logits(self):
        c = self.b.ctx
        c.rms_norm(self.h_last, self.gain_out, self.eps, self.x)
        c.linear(self.x, self.w_out, self.logits, workspace=self.ws_products)

    def _draw(self):
        """The next token of every request from the logits; -1 for those that have ended, or whose logits hold nothing to draw: they end here."""
        self.b.ctx.sample(self.logits, self.logits.shape[1], self.u, self.token, logprob=self.logprob, n_kept=self.n_kept, workspace=self.ws,
                          **self.settings)
        self.token.masked_fill_(~self.alive, -1)
        self.alive &= self.token >= 0
        self.logprob.masked_fill_(~self.alive, -math.inf)
        self.n_kept.masked_fill_(~self.alive, 0)
        if self.stop is not None:
            self.alive &= self.token != self.stop

    def _feed(self):
        """The drawn tokens through the layers."""
        b, c = self.b, self.b.ctx
        self.n_new.index_copy_(0, self.last_seg, self.alive.int())
        c.extend_segments(self.segs, self.n_new, self.tab_cap, b.req_seg_off, self.free_left, self.block_tab, b.k_req.shape[0], self.segs, self.cu_q,
                          self.q_pos, self.slot_map, self.row_req, self.last_row, self.status, self.counts, self.ws)
        self.alive &= self.status == 0                                # (one that got no row has no logits either)
        # (the pages taken leave the list: what is left moves to its front, the end repeats its last entry and is never reached)
        left = torch.arange(self.free.shape[0], device=self.free.device) + self.counts[1]
        self.free_left.copy_(self.free_left[left.clamp(max=self.free.shape[0] - 1)])
        rows = self.token[self.row_req.long().clamp(min=0)].masked_fill(self.row_req < 0, -1)
        c.gather_rows(self.embed, rows, self.h)
        for l, lw in enumerate(self.loop.weights):
            k_pool, v_pool, v_map = self.loop.pages[l]
            c.rms_norm(self.h, lw["gain_attn"], self.loop.eps[l], self.x)
            c.qkv_project(self.x, lw["w_qkv"], self.q, self.k, self.v, workspace=self.ws_products)
            c.append_attention(self.q, self.k, self.v, self.q_pos, self.slot_map, self.cu_q, 1, k_pool, v_pool, self.block_tab, self.segs,
                               b.req_seg_off, self.n, self.max_ctx, self.max_segs, self.o, None, self.ws,
                               shared=(b.v_store, v_map) if b.cow else None)
            c.linear(self.o.view(self.n, -1), lw["w_o"], self.h1, residual=self.h, workspace=self.ws_products)
            c.rms_norm(self.h1, lw["gain_ffn"], self.loop.eps[l], self.x)
            c.gated_linear(self.x, lw["w_gate"], lw["w_up"], self.act)
            c.linear(self.act, lw["w_down"], self.h, residual=self.h1, workspace=self.ws_products)
        c.gather_rows(self.h, self.last_row, self.h_last)
        self._logits()

    def run(self, u, graph: bool = False, keep: bool = False):
        """u [steps, requests]: the uniform numbers the tokens are drawn with (at most answer_tokens + 1 steps in all).  Returns the tokens [steps,
        requests] (-1: none, as the request has ended) and their log-probabilities (-infinity there); with keep also the logits each was drawn from."""
        if self.turn != self.loop.turn:
            raise ValueError("AnswerLoop: a later prefill or answer has taken the pages")
        u = torch.as_tensor(np.ascontiguousarray(u, dtype=np.float32)).to(self.u.device)
        if self.drawn + u.shape[0] > self.loop.answer_tokens + 1:
            raise ValueError("AnswerLoop: more tokens than the pages have room for")
        if u.shape[0] == 0:
            none = np.zeros((0, self.n), dtype=np.int32), np.zeros((0, self.n), dtype=np.float32)
            return none + ([],) if keep else none
        tokens, logprobs, logits, captured, fed = [], [], [], None, False
        for step in range(u.shape[0]):
            if self.drawn == 0:
                pass                                                  # (the prefill's logits)
            elif captured is not None:
                captured.replay()
            else:
                self._feed()
                if graph and fed:                                     # (the second eager step: lazy set-up stays out of the graph)
                    torch.cuda.synchronize()
                    captured = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(captured):
                        self._feed()
                fed = True
            self.u.copy_(u[step])
            if keep:
                logits.append(self.logits.float().cpu().numpy())
            self._draw()
            self.drawn += 1
            tokens.append(self.token.clone())
            logprobs.append(self.logprob.clone())
        torch.cuda.synchronize()
        out = torch.stack(tokens).cpu().numpy(), torch.stack(logprobs).cpu().numpy()
        return out + (logits,) if keep else out


class LayerLoop:
    def __init__(self, w, n_layers: int, window: int,
                 layer_inputs: Optional[Callable[[int, DeviceBatch], None]] = None,
                 impl: int = CC_IMPL_AUTO, preload: bool = True, depth: Optional[int] = None,
                 device: str = "cuda"):
        """layer_inputs(l, batch), if given, runs before layer l's attention on the stream the loop
        uses; it may overwrite batch.q / batch.k_new / batch.v_new (or batch.hidden) in place with
        layer l's tensors.  The attention reads them per token through the row list: the loop
        makes no compact copies unless the workload is projected from hidden states."""
        self.w, self.n_layers, self.window, self.layer_inputs = w, n_layers, window, layer_inputs
        self.batch = DeviceBatch(w, device=device, impl=impl)
        b = self.batch
        seg = w.segments
        self.chunk_segs = [[s for s in range(int(w.req_seg_off[r]), int(w.req_seg_off[r + 1])) if seg[s][1] == 0]
                           for r in range(w.n_requests)]
        self.trackers = [FocusTracker(max(1, len(c)), window) for c in self.chunk_segs]
        self.budget = np.array(seg[:, 5], dtype=np.int64)
        self.stop_layer: List[Optional[int]] = [None] * w.n_requests
        self.focused: List[Optional[List[int]]] = [None] * w.n_requests
        self.mass_host = torch.zeros(max(1, len(seg)), dtype=torch.float32).pin_memory()
        self.mass_ready = torch.cuda.Event()
        self.pre = None
        if preload:
            self.k_host, self.v_host = b.k_store.cpu().pin_memory(), b.v_store.cpu().pin_memory()
            self.depth = depth if depth is not None else 1
            n_slots = min(self.depth + 1, n_layers)
            self.slots = [(torch.empty_like(b.k_store), torch.empty_like(b.v_store)) for _ in range(n_slots)]
            self.pre = (Preloader(n_layers, self.depth, n_slots), Preloader(n_layers, self.depth, n_slots))
            for l in range(n_layers):
                self.pre[0].set_layer(l, self.k_host, self.slots[l % n_slots][0])
                self.pre[1].set_layer(l, self.v_host, self.slots[l % n_slots][1])

    def run(self, scores: Optional[np.ndarray] = None, keep_outputs: bool = False):
        """scores: per-token scores to select from (the ordered list a chunk's metadata keeps); by
        default layer 0 computes them with cc_select and the later layers reuse them.
        Returns one record per layer: rows recomputed, per-request focused sets decided so far."""
        b, w = self.batch, self.w
        if scores is not None:
            b.scores.copy_(torch.from_numpy(np.ascontiguousarray(scores, dtype=np.float32)))
        records = []
        for l in range(self.n_layers):
            t_start = torch.cuda.Event(enable_timing=True); t_end = torch.cuda.Event(enable_timing=True)
            t_start.record()
            if self.pre is not None:
                self.pre[0].acquire(l); self.pre[1].acquire(l)
                b.k_store, b.v_store = self.slots[l % len(self.slots)]
            b.rope_shift()
            if l == 0 and scores is None:
                b.select()
            else:
                b.select_from_scores()
            if self.layer_inputs is not None:
                self.layer_inputs(l, b)
            if b.projected:
                b.gather()
            mass = b.sparse_prefill_mass(fused=not b.projected)   # attention + the question's masses in one call
            self.mass_host.copy_(mass, non_blocking=True)
            self.mass_ready.record()
            if self.pre is not None:
                self.pre[0].release(l); self.pre[1].release(l)
            t_end.record()
            rec = {"layer": l + 1, "rows": b.n_q_tot, "_events": (t_start, t_end)}
            if keep_outputs:
                torch.cuda.synchronize()
                rec["out"] = b.out[: b.n_q_tot].float().cpu().numpy()
                rec["lse"] = b.lse[: b.n_q_tot].cpu().numpy()
                rec["sel_idx"] = b.sel_idx[: b.n_q_tot].cpu().numpy()
                rec["cu_q"] = np.array(getattr(b, "cu_q_host", w.cu_q), copy=True)
            # Algorithm 1 on this layer's masses; a settled request drops its unfocused chunks
            self.mass_ready.synchronize()
            m = self.mass_host.numpy()
            rec["mass"] = m[: len(w.segments)].copy()
            changed = False
            for r, segs in enumerate(self.chunk_segs):
                if self.stop_layer[r] is not None or not segs:
                    continue
                stop, focused = self.trackers[r].update([float(m[s]) for s in segs])
                if stop:
                    self.stop_layer[r], self.focused[r] = l + 1, focused
                    for i, sgi in enumerate(segs):
                        if i not in focused:
                            self.budget[sgi] = 0
                            changed = True
            rec["stop_layer"] = list(self.stop_layer)
            rec["focused"] = [None if f is None else list(f) for f in self.focused]
            if changed and l + 1 < self.n_layers:
                b.set_budget(self.budget)
            records.append(rec)
        torch.cuda.synchronize()
        for rec in records:
            t_start, t_end = rec.pop("_events")
            rec["ms"] = t_start.elapsed_time(t_end)
        return records

    def close(self):
        for t in self.trackers:
            t.close()
        if self.pre is not None:
            for p in self.pre:
                p.close()
            self.pre = None
