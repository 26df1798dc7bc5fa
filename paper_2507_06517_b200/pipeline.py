"""Whole-prompt driver: one object that owns the device buffers of a SpindleKV reduction pass and
issues the four library calls for all layers (plan, evict deep layers, build CodeBooks for shallow
layers, compact).  No arithmetic happens here; this is buffer ownership and call order only.
"""
from __future__ import annotations

import dataclasses
import threading
from typing import Dict, Optional, Sequence

import numpy as np
import torch

from . import binding as B


def record_graph(fn, device="cuda") -> "torch.cuda.CUDAGraph":
    """Records what ``fn()`` enqueues (calls of this library on the current stream and on streams forked from it) as a
    CUDA graph; ``replay()`` on the result repeats it with one launch from the host.  ``fn`` runs once outside the
    recording first, so that whatever is set up on first use (kernel attributes, side streams, workspaces) exists
    before the recording starts; the tensors it uses must stay where they are."""
    dev = torch.device(device)
    warm = torch.cuda.Stream(dev)
    warm.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(warm):
        fn()
    torch.cuda.current_stream(dev).wait_stream(warm)
    torch.cuda.synchronize(dev)
    graph = torch.cuda.CUDAGraph()
    # only this thread's calls belong to the recording (a communication library's watchdog thread may poll its events meanwhile)
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        fn()
    return graph


class SpindleKVPass:
    """Buffers and call sequence for one prompt batch.

    ``K`` and ``V`` are ``[n_layers, B, H_kv, N, d]`` (equal lengths) or packed
    ``[n_layers, total_tokens, H_kv, d]`` with ``cu_seqlens``; ``Q`` is
    ``[n_layers - n_shallow, B, H_q, w, d]`` (window queries of the evicting layers).
    Layers ``[0, n_shallow)`` get CodeBooks, the others are evicted.
    """

    def __init__(self, cfg: B.Config, seq_lens: Sequence[int], dtype: torch.dtype, device="cuda",
                 layers_per_codebook_call: Optional[int] = None, keep_adjacency: bool = False,
                 side_by_side: bool = True):
        self.cfg = cfg
        # run(): the K CodeBooks, the V CodeBooks and the eviction are independent; on three streams the short
        # kernels of one (norms, lists, cover, top-k, gathers: a block per unit, far from filling the device) run
        # beside those of the others.  Costs a second CodeBook workspace.  Off when the adjacency is kept (one
        # buffer for both calls).
        self.side_by_side = side_by_side and not keep_adjacency
        self.seq_lens = [int(x) for x in seq_lens]
        self.dtype = dtype
        self.device = torch.device(device)
        self.n_seqs = len(self.seq_lens)
        self.max_len = max(self.seq_lens)
        self.packed = len(set(self.seq_lens)) > 1
        self.total = sum(self.seq_lens) if self.packed else self.n_seqs * self.max_len
        self.n_deep = cfg.n_layers - cfg.n_shallow
        self.n_shallow = cfg.n_shallow
        dev = self.device
        self.cu = None
        if self.packed:
            cu = np.concatenate([[0], np.cumsum(self.seq_lens)]).astype(np.int32)
            self.cu = torch.from_numpy(cu).to(dev)
        self.mode, self.ratio, self.k_ctx_host = B.spindlekv_plan_layers(cfg, self.seq_lens)
        H, d, T = cfg.n_kv_heads, cfg.head_dim, self.total
        i32 = dict(dtype=torch.int32, device=dev)
        if self.n_deep:
            self.deep_batch = B.Batch(self.n_deep, self.n_seqs, self.max_len, T, self.cu)
            self.k_ctx = torch.from_numpy(np.ascontiguousarray(self.k_ctx_host[self.n_shallow:])).to(dev)
            self.kept_lens = torch.from_numpy(np.ascontiguousarray(self.k_ctx_host[self.n_shallow:] + cfg.window, dtype=np.int32)).to(dev)
            self.keep_idx = torch.zeros((self.n_deep, H, T), **i32)
            self.keep_cnt = torch.zeros((self.n_deep, self.n_seqs, H), **i32)
            self.scores = torch.zeros((self.n_deep, H, T), dtype=torch.float32, device=dev)
            nb = B.spindlekv_workspace_bytes(cfg, self.deep_batch, B.WS_EVICT)
            self.ws_evict = torch.empty(nb, dtype=torch.uint8, device=dev)
            self.K_kept = self._alloc_like_input(self.n_deep, dtype)
            self.V_kept = self._alloc_like_input(self.n_deep, dtype)
        if self.n_shallow:
            per_call = layers_per_codebook_call or self.n_shallow
            self.cb_layers_per_call = min(per_call, self.n_shallow)
            self.cb_batch = B.Batch(self.cb_layers_per_call, self.n_seqs, self.max_len, T, self.cu)
            nb = B.spindlekv_workspace_bytes(cfg, self.cb_batch, B.WS_CODEBOOK)
            self.ws_codebook = torch.empty(nb, dtype=torch.uint8, device=dev)
            self.cb: Dict[str, Dict[str, torch.Tensor]] = {}
            for g in ("K", "V"):
                self.cb[g] = {
                    "mag": torch.zeros((self.n_shallow, H, T), dtype=torch.float32, device=dev),
                    "ref": torch.zeros((self.n_shallow, H, T), **i32),
                    "centre_idx": torch.zeros((self.n_shallow, H, T), **i32),
                    "n_entries": torch.zeros((self.n_shallow, self.n_seqs, H), **i32),
                    "C": self._alloc_like_input(self.n_shallow, dtype),
                }
            self.adj = None
            if keep_adjacency:
                units = self.cb_layers_per_call * self.n_seqs * H
                self.adj = torch.zeros((units, self.max_len, B.row_words(self.max_len)), **i32)

    def _alloc_like_input(self, n_layers: int, dtype: torch.dtype) -> torch.Tensor:
        H, d = self.cfg.n_kv_heads, self.cfg.head_dim
        if self.packed:
            return torch.zeros((n_layers, self.total, H, d), dtype=dtype, device=self.device)
        return torch.zeros((n_layers, self.n_seqs, H, self.max_len, d), dtype=dtype, device=self.device)

    def _desc(self, t: torch.Tensor):
        return B.desc_thd(t) if self.packed else B.desc_bhnd(t)

    # -- the four calls, in order ------------------------------------------------------------
    def evict(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, stream=None) -> None:
        """Deep layers: ``K``/``V`` hold only the evicting layers."""
        cfg = self.cfg
        B.spindlekv_evict_deep(cfg, self.deep_batch, self._desc(K), B.desc_bhnd(Q), self.k_ctx, self.keep_idx,
                               self.keep_cnt, self.scores, self.ws_evict, stream)
        for src, dst in ((K, self.K_kept), (V, self.V_kept)):
            B.spindlekv_compact(self.deep_batch, cfg.n_kv_heads, cfg.head_dim, self._desc(src), self.keep_idx,
                                self.keep_cnt, self._desc(dst), None, None, stream)

    def _codebook_chunk(self, G: torch.Tensor, which: str, l0: int, stream=None) -> None:
        """CodeBooks of ``G.shape[0]`` consecutive shallow layers starting at layer ``l0``."""
        cfg = self.cfg
        n = G.shape[0]
        theta = cfg.theta_k if which == "K" else cfg.theta_v
        out = self.cb[which]
        batch = self.cb_batch if n == self.cb_layers_per_call else B.Batch(n, self.n_seqs, self.max_len, self.total, self.cu)
        sl = slice(l0, l0 + n)
        B.spindlekv_codebook_shallow(cfg, batch, self._desc(G), theta, out["mag"][sl], out["ref"][sl],
                                     out["centre_idx"][sl], out["n_entries"][sl], self.ws_codebook, self.adj, stream)
        B.spindlekv_compact(batch, cfg.n_kv_heads, cfg.head_dim, self._desc(G), out["centre_idx"][sl],
                            out["n_entries"][sl], self._desc(out["C"][sl]), out["mag"][sl], None, stream)

    def codebook(self, G: torch.Tensor, which: str, stream=None) -> None:
        """Shallow layers: ``G`` holds only the CodeBook layers of ``which`` in {"K", "V"}."""
        step = self.cb_layers_per_call
        for l0 in range(0, self.n_shallow, step):
            self._codebook_chunk(G[l0:l0 + min(step, self.n_shallow - l0)], which, l0, stream)

    def run(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, stream=None) -> None:
        """All layers of one prompt batch (``K``/``V`` hold every layer)."""
        ns = self.n_shallow
        if self.side_by_side and ns and (stream is None or isinstance(stream, torch.cuda.Stream)):
            return self._run_side_by_side(K, V, Q, stream)   # (a raw stream handle cannot be joined with: one stream then)
        if self.n_deep:
            self.evict(K[ns:], V[ns:], Q, stream)
        if ns:
            self.codebook(K[:ns], "K", stream)
            self.codebook(V[:ns], "V", stream)

    def capture(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor) -> "torch.cuda.CUDAGraph":
        """Records one ``run`` on these tensors (side streams included) as a CUDA graph and returns it; ``replay()``
        on the result repeats the pass on whatever the same tensors hold by then, with one launch from the host."""
        return record_graph(lambda: self.run(K, V, Q), self.device)

    def _run_side_by_side(self, K, V, Q, stream=None) -> None:
        """``run`` on three streams: K CodeBooks on the caller's stream, V CodeBooks and the eviction on two side
        streams that start after the work already queued on the caller's stream and are joined before returning."""
        dev, ns = self.device, self.n_shallow
        cur = stream if stream is not None else torch.cuda.current_stream(dev)
        if not hasattr(self, "_side"):
            self._side = [torch.cuda.Stream(dev) for _ in range(2)]
            self._ws_codebook_v = torch.empty_like(self.ws_codebook)
        sV, sE = self._side
        ev = torch.cuda.Event()
        ev.record(cur)
        sV.wait_event(ev)
        self.codebook(K[:ns], "K", cur)
        ws = self.ws_codebook
        self.ws_codebook = self._ws_codebook_v
        try:
            self.codebook(V[:ns], "V", sV)
        finally:
            self.ws_codebook = ws
        if self.n_deep:
            sE.wait_event(ev)
            self.evict(K[ns:], V[ns:], Q, sE)
            cur.wait_stream(sE)
        cur.wait_stream(sV)

    def store_paged(self, K: torch.Tensor, V: torch.Tensor, cache: "SpindleKVPagedCache", stream=None, rope_table: Optional[torch.Tensor] = None) -> None:
        """What the last eviction kept of ``K`` and ``V`` (every layer's, or the evicting layers' alone) becomes the content of
        ``cache``, whose layers are the evicting ones; what it held is given back.  The kept rows go from the prompt's tensors into
        the pages in one step; with ``rope_table`` (``[n_positions, d/2, 2]``) the keys are rotated on the way, each by the position that it had in
        the prompt.  Equal-length batches."""
        if self.packed:
            raise ValueError("store_paged needs sequences of equal length")
        if (cache.n_layers, cache.n_seqs, cache.Hkv, cache.d) != (self.n_deep, self.n_seqs, self.cfg.n_kv_heads, self.cfg.head_dim):
            raise ValueError("the cache does not have the evicting layers' shape")
        if K.shape[0] != self.n_deep:
            K, V = K[self.n_shallow:], V[self.n_shallow:]
        for name, t in (("K", K), ("V", V)):               # before anything is given back
            cache._cache_rows(name, t, self.n_deep, self.cfg.n_kv_heads)
            if t.shape[3] != self.max_len:
                raise ValueError(f"{name}: {self.max_len} rows expected, got {t.shape[3]}")
        cache.resize(cache.no_tokens, stream=stream)
        cache.resize(self.kept_lens, stream=stream)
        most = int(self.k_ctx_host[self.n_shallow:].max()) + self.cfg.window
        if rope_table is None:
            cache.append(K, V, idx=self.keep_idx, idx_seq=self.max_len, max_new=most, stream=stream)
        else:
            cache.append_rotated(K, V, rope_table, idx=self.keep_idx, idx_seq=self.max_len, max_new=most, stream=stream)

    # -- the same pass fed from host memory ----------------------------------------------------
    def host_outputs(self) -> Dict[str, torch.Tensor]:
        """Pinned host tensors for everything ``run_from_host`` brings back: index maps, counts,
        magnitudes, kept rows (up to the largest ``k + w`` of any layer) and CodeBook rows."""
        out: Dict[str, torch.Tensor] = {}

        def pin(name, t):
            out[name] = torch.empty(t.shape, dtype=t.dtype, pin_memory=True)

        if self.n_deep:
            pin("keep_idx", self.keep_idx)
            pin("keep_cnt", self.keep_cnt)
            pin("K_kept", self._kept_view(self.K_kept))
            pin("V_kept", self._kept_view(self.V_kept))
        if self.n_shallow:
            for g in ("K", "V"):
                for k in ("ref", "mag", "n_entries", "C"):
                    pin(f"{g}.{k}", self.cb[g][k])
        return out

    def _kept_view(self, t: torch.Tensor) -> torch.Tensor:
        if self.packed:
            return t
        return t[:, :, :, : int(self.k_ctx_host[self.n_shallow:].max()) + self.cfg.window]

    def run_from_host(self, hK: torch.Tensor, hV: torch.Tensor, hQ: Optional[torch.Tensor],
                      host_out: Dict[str, torch.Tensor]) -> None:
        """All layers of one prompt batch whose K, V (every layer) and Q (evicting layers) sit in pinned
        host memory.  Uploads, kernels and downloads run on three streams: while the CodeBooks of one
        group of layers are built, the next group is on its way in and the previous results are on
        their way out.  Returns once everything is enqueued; work that follows on the current stream
        is ordered after the last download."""
        dev, cfg, ns = self.device, self.cfg, self.n_shallow
        cur = torch.cuda.current_stream(dev)
        if not hasattr(self, "_s_in"):
            self._s_in, self._s_out = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
            c = self.cb_layers_per_call if ns else 0
            self._stage = [self._alloc_like_input(c, self.dtype) for _ in range(2)] if ns else []
            if self.n_deep:
                self._dK = self._alloc_like_input(self.n_deep, self.dtype)
                self._dV = self._alloc_like_input(self.n_deep, self.dtype)
                self._dQ = torch.empty(hQ.shape, dtype=hQ.dtype, device=dev)
        s_in, s_out = self._s_in, self._s_out
        s_in.wait_stream(cur)
        s_out.wait_stream(cur)
        free = [None, None]   # event after the kernels that last read a staging buffer

        def send(dst, src, after=None):
            with torch.cuda.stream(s_in):
                if after is not None:
                    s_in.wait_event(after)
                dst.copy_(src, non_blocking=True)
                ev = torch.cuda.Event()
                ev.record(s_in)
            return ev

        def fetch(pairs):
            ev = torch.cuda.Event()
            ev.record(cur)
            with torch.cuda.stream(s_out):
                s_out.wait_event(ev)
                for h, d in pairs:
                    h.copy_(d, non_blocking=True)

        slot = 0
        step = self.cb_layers_per_call if ns else 1
        for l0 in range(0, ns, step):
            n = min(step, ns - l0)
            for which, h in (("K", hK), ("V", hV)):
                buf = self._stage[slot & 1][:n]
                cur.wait_event(send(buf, h[l0:l0 + n], free[slot & 1]))
                self._codebook_chunk(buf, which, l0)
                free[slot & 1] = torch.cuda.Event()
                free[slot & 1].record(cur)
                o = self.cb[which]
                fetch([(host_out[f"{which}.{k}"][l0:l0 + n], o[k][l0:l0 + n]) for k in ("ref", "mag", "n_entries", "C")])
                slot += 1
        if self.n_deep:
            ev_k = send(self._dK, hK[ns:])
            ev_q = send(self._dQ, hQ)
            ev_v = send(self._dV, hV[ns:])
            cur.wait_event(ev_k)
            cur.wait_event(ev_q)
            B.spindlekv_evict_deep(cfg, self.deep_batch, self._desc(self._dK), B.desc_bhnd(self._dQ), self.k_ctx,
                                   self.keep_idx, self.keep_cnt, self.scores, self.ws_evict)
            B.spindlekv_compact(self.deep_batch, cfg.n_kv_heads, cfg.head_dim, self._desc(self._dK), self.keep_idx,
                                self.keep_cnt, self._desc(self.K_kept), None, None)
            fetch([(host_out["keep_idx"], self.keep_idx), (host_out["keep_cnt"], self.keep_cnt),
                   (host_out["K_kept"], self._kept_view(self.K_kept))])
            cur.wait_event(ev_v)
            B.spindlekv_compact(self.deep_batch, cfg.n_kv_heads, cfg.head_dim, self._desc(self._dV), self.keep_idx,
                                self.keep_cnt, self._desc(self.V_kept), None, None)
            fetch([(host_out["V_kept"], self._kept_view(self.V_kept))])
        cur.wait_stream(s_out)

    def device_status(self):
        """Status words of both workspaces (synchronises the device)."""
        torch.cuda.synchronize(self.device)
        out = {}
        if self.n_deep:
            out["evict"] = B.spindlekv_poll_status(self.ws_evict)
        if self.n_shallow:
            out["codebook"] = B.spindlekv_poll_status(self.ws_codebook)
            if hasattr(self, "_ws_codebook_v"):   # the V call of the last side-by-side run
                out["codebook_v"] = B.spindlekv_poll_status(self._ws_codebook_v)
        return out


class SpindleKVLiteralPass:
    """The composition of Section 3 as the paper writes it: every layer evicts under the pyramid of
    Eq. (5)(6) laid over all layers (Eq. (7)), then K and V CodeBooks are built from the tokens the layer
    kept (Algorithm 1), whose number differs from layer to layer.  ``cfg.n_shallow`` must be -1; all
    sequences have the same length.  ``K``, ``V``: ``[n_layers, B, H_kv, N, d]``; ``Q``:
    ``[n_layers, B, H_q, w, d]``.  No arithmetic happens here: buffers and call order only.
    """

    def __init__(self, cfg: B.Config, seq_lens: Sequence[int], dtype: torch.dtype, device="cuda",
                 keep_adjacency: bool = False):
        if cfg.n_shallow != -1:
            raise ValueError("SpindleKVLiteralPass needs cfg.n_shallow == -1")
        if len(set(int(x) for x in seq_lens)) != 1:
            raise ValueError("SpindleKVLiteralPass needs sequences of equal length")
        self.cfg = cfg
        self.device = torch.device(device)
        self.ev = SpindleKVPass(dataclasses.replace(cfg, n_shallow=0), seq_lens, dtype, device)
        self.mode, self.ratio, self.k_ctx_host = B.spindlekv_plan_layers(cfg, list(seq_lens))
        L, nB, H, d = cfg.n_layers, len(seq_lens), cfg.n_kv_heads, cfg.head_dim
        self.kept_host = (self.k_ctx_host + cfg.window).astype(np.int32)          # [L, B] tokens kept per head
        self.max_keep = int(self.kept_host.max())
        self.layer_lens = torch.from_numpy(np.ascontiguousarray(self.kept_host)).to(self.device)
        T = nB * self.max_keep
        self.cb_batch = B.Batch(L, nB, self.max_keep, T, None, self.layer_lens)
        nb = B.spindlekv_workspace_bytes(cfg, self.cb_batch, B.WS_CODEBOOK)
        self.ws_codebook = torch.empty(nb, dtype=torch.uint8, device=self.device)
        i32 = dict(dtype=torch.int32, device=self.device)
        self.cb: Dict[str, Dict[str, torch.Tensor]] = {}
        for g in ("K", "V"):
            self.cb[g] = {
                "mag": torch.zeros((L, H, T), dtype=torch.float32, device=self.device),
                "ref": torch.zeros((L, H, T), **i32),
                "centre_idx": torch.zeros((L, H, T), **i32),
                "n_entries": torch.zeros((L, nB, H), **i32),
                "C": torch.zeros((L, nB, H, self.max_keep, d), dtype=dtype, device=self.device),
            }
        self.adj = None
        if keep_adjacency:
            self.adj = torch.zeros((L * nB * H, self.max_keep, B.row_words(self.max_keep)), **i32)

    def _codebook(self, g: str, ws: torch.Tensor, stream) -> None:
        cfg = self.cfg
        kept = (self.ev.K_kept if g == "K" else self.ev.V_kept)[:, :, :, : self.max_keep]
        o = self.cb[g]
        B.spindlekv_codebook_shallow(cfg, self.cb_batch, B.desc_bhnd(kept), cfg.theta_k if g == "K" else cfg.theta_v,
                                     o["mag"], o["ref"], o["centre_idx"], o["n_entries"], ws, self.adj, stream)
        B.spindlekv_compact(self.cb_batch, cfg.n_kv_heads, cfg.head_dim, B.desc_bhnd(kept), o["centre_idx"],
                            o["n_entries"], B.desc_bhnd(o["C"]), o["mag"], None, stream)

    def run(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, which=("K", "V"), stream=None) -> None:
        self.ev.evict(K, V, Q, stream)
        if self.adj is None and tuple(which) == ("K", "V") and (stream is None or isinstance(stream, torch.cuda.Stream)):
            # the two CodeBook calls are independent: the V call runs on a side stream with a workspace of its own
            cur = stream if stream is not None else torch.cuda.current_stream(self.device)
            if not hasattr(self, "_side"):
                self._side = torch.cuda.Stream(self.device)
                self._ws_codebook_v = torch.empty_like(self.ws_codebook)
            ev = torch.cuda.Event()
            ev.record(cur)
            self._side.wait_event(ev)
            self._codebook("K", self.ws_codebook, cur)
            self._codebook("V", self._ws_codebook_v, self._side)
            cur.wait_stream(self._side)
            return
        for g in which:
            self._codebook(g, self.ws_codebook, stream)

    def entry_counts(self):
        """Host copies of the CodeBook sizes ``[L, B, H]`` for K and V (synchronises)."""
        return self.cb["K"]["n_entries"].cpu().numpy(), self.cb["V"]["n_entries"].cpu().numpy()

    def device_status(self):
        torch.cuda.synchronize(self.device)
        out = {"evict": B.spindlekv_poll_status(self.ev.ws_evict), "codebook": B.spindlekv_poll_status(self.ws_codebook)}
        if hasattr(self, "_ws_codebook_v"):
            out["codebook_v"] = B.spindlekv_poll_status(self._ws_codebook_v)
        return out


class SpindleKVRepeatPass:
    """The GQA "repeat" alternative of Section 3.3 inside the composition as written: the KV vectors of
    a group are taken once per query head, so every query head selects its own tokens (Eq. (2)(7) without
    the group mean of Eq. (3)); the K and V CodeBooks of a KV head are then built from the tokens all
    its query heads kept, listed one head after the other, where a token kept by several heads
    appears several times and collapses into one entry (cosine similarity 1).  ``cfg.n_shallow`` must
    be -1; equal-length sequences.  ``K``, ``V``: ``[L, B, H_kv, N, d]``; ``Q``: ``[L, B, H_q, w, d]``.
    One eviction call with ``per_query_head`` set serves all query heads.  Buffers and call order only.
    """

    def __init__(self, cfg: B.Config, seq_lens: Sequence[int], dtype: torch.dtype, device="cuda",
                 keep_adjacency: bool = False):
        if cfg.n_shallow != -1:
            raise ValueError("SpindleKVRepeatPass needs cfg.n_shallow == -1")
        if len(set(int(x) for x in seq_lens)) != 1:
            raise ValueError("SpindleKVRepeatPass needs sequences of equal length")
        self.cfg = cfg
        self.device = dev = torch.device(device)
        self.h_n = cfg.n_q_heads // cfg.n_kv_heads
        L, nB, H, Hq, d, N = cfg.n_layers, len(seq_lens), cfg.n_kv_heads, cfg.n_q_heads, cfg.head_dim, int(seq_lens[0])
        self.n_seqs, self.max_len = nB, N
        self.ecfg = dataclasses.replace(cfg, n_shallow=0, per_query_head=1)
        self.mode, self.ratio, self.k_ctx_host = B.spindlekv_plan_layers(cfg, list(seq_lens))
        self.k_ctx = torch.from_numpy(np.ascontiguousarray(self.k_ctx_host)).to(dev)
        self.ev_batch = B.Batch(L, nB, N, nB * N)
        i32 = dict(dtype=torch.int32, device=dev)
        self.keep_idx = torch.zeros((L, Hq, nB * N), **i32)              # per query head
        self.keep_cnt = torch.zeros((L, nB, Hq), **i32)
        self.scores = torch.zeros((L, Hq, nB * N), dtype=torch.float32, device=dev)
        self.ws_evict = torch.empty(B.spindlekv_workspace_bytes(self.ecfg, self.ev_batch, B.WS_EVICT), dtype=torch.uint8, device=dev)
        self.kept_host = (self.k_ctx_host + cfg.window).astype(np.int32)                     # per query head
        self.union_host = (self.h_n * self.kept_host).astype(np.int32)                       # per KV head
        self.max_union = int(self.union_host.max())
        self.layer_lens = torch.from_numpy(np.ascontiguousarray(self.union_host)).to(dev)
        T = nB * self.max_union
        self.union_idx = torch.zeros((L, H, T), **i32)
        self.union_cnt = torch.zeros((L, nB, H), **i32)
        self.cb_batch = B.Batch(L, nB, self.max_union, T, None, self.layer_lens)
        self.ws_codebook = torch.empty(B.spindlekv_workspace_bytes(cfg, self.cb_batch, B.WS_CODEBOOK), dtype=torch.uint8, device=dev)
        self.rep = {g: torch.zeros((L, nB, H, self.max_union, d), dtype=dtype, device=dev) for g in ("K", "V")}
        self.cb: Dict[str, Dict[str, torch.Tensor]] = {}
        for g in ("K", "V"):
            self.cb[g] = {
                "mag": torch.zeros((L, H, T), dtype=torch.float32, device=dev),
                "ref": torch.zeros((L, H, T), **i32),
                "centre_idx": torch.zeros((L, H, T), **i32),
                "n_entries": torch.zeros((L, nB, H), **i32),
                "C": torch.zeros((L, nB, H, self.max_union, d), dtype=dtype, device=dev),
            }
        self.adj = torch.zeros((L * nB * H, self.max_union, B.row_words(self.max_union)), **i32) if keep_adjacency else None

    def run(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, which=("K", "V"), stream=None) -> None:
        cfg, H, d = self.cfg, self.cfg.n_kv_heads, self.cfg.head_dim
        B.spindlekv_evict_deep(self.ecfg, self.ev_batch, B.desc_bhnd(K), B.desc_bhnd(Q), self.k_ctx, self.keep_idx,
                               self.keep_cnt, self.scores, self.ws_evict, stream)
        # query head h_n*j + g is list g of KV head j: the per-query-head outputs are [L][H][h_n][...] as they stand
        L = cfg.n_layers
        B.spindlekv_union_lists(L, self.n_seqs, H, self.keep_idx.view(L, H, self.h_n, -1),
                                self.keep_cnt.view(L, self.n_seqs, H, self.h_n), self.max_len,
                                self.union_idx, self.union_cnt, self.max_union, stream, lists_inner=True)
        def codebook(g, ws, st):
            src, rep, o = (K if g == "K" else V), self.rep[g], self.cb[g]
            # rows of the union list, gathered from the KV head (the union list is laid out per max_union tokens,
            # the source per max_len tokens: two batches describe the two sides)
            self._gather(src, rep, st)
            B.spindlekv_codebook_shallow(cfg, self.cb_batch, B.desc_bhnd(rep), cfg.theta_k if g == "K" else cfg.theta_v,
                                         o["mag"], o["ref"], o["centre_idx"], o["n_entries"], ws, self.adj, st)
            B.spindlekv_compact(self.cb_batch, H, d, B.desc_bhnd(rep), o["centre_idx"], o["n_entries"],
                                B.desc_bhnd(o["C"]), o["mag"], None, st)

        if self.adj is None and tuple(which) == ("K", "V") and (stream is None or isinstance(stream, torch.cuda.Stream)):
            # the two CodeBook calls are independent: the V call runs on a side stream with a workspace of its own
            cur = stream if stream is not None else torch.cuda.current_stream(self.device)
            if not hasattr(self, "_side"):
                self._side = torch.cuda.Stream(self.device)
                self._ws_codebook_v = torch.empty_like(self.ws_codebook)
            ev = torch.cuda.Event()
            ev.record(cur)
            self._side.wait_event(ev)
            codebook("K", self.ws_codebook, cur)
            codebook("V", self._ws_codebook_v, self._side)
            cur.wait_stream(self._side)
            return
        for g in which:
            codebook(g, self.ws_codebook, stream)

    def _gather(self, src: torch.Tensor, rep: torch.Tensor, stream=None) -> None:
        # index rows are [L][H][B * max_union]; the compaction call addresses source rows through the batch's
        # max_len and index rows through total_len, so the batch carries the index layout and the source
        # tensor descriptor carries its own strides
        cfg = self.cfg
        B.spindlekv_compact(self.cb_batch, cfg.n_kv_heads, cfg.head_dim, B.desc_bhnd(src), self.union_idx, self.union_cnt,
                            B.desc_bhnd(rep), None, None, stream)

    def device_status(self):
        torch.cuda.synchronize(self.device)
        out = {"evict": B.spindlekv_poll_status(self.ws_evict), "codebook": B.spindlekv_poll_status(self.ws_codebook)}
        if hasattr(self, "_ws_codebook_v"):
            out["codebook_v"] = B.spindlekv_poll_status(self._ws_codebook_v)
        return out


class SpindleKVDecodeMerge:
    """Decode-time merging (Section 3.4, last paragraph) of ``t_new`` new tokens per (layer, sequence, head)
    into existing CodeBooks: match against the entries, build a CodeBook of the unmatched tokens, append
    it.  ``C``: ``[L, B, H, c_rows, d]`` with ``n_entries [L, B, H]`` (both updated in place); new tokens
    ``[L, B, H, t_new, d]``.  Results: ``ref_new``, ``mag_new`` ``[L, H, B * t_new]``.  Call order only.
    """

    def __init__(self, cfg: B.Config, n_layers: int, n_seqs: int, t_new: int, c_rows: int, dtype: torch.dtype,
                 device="cuda", keep_adjacency: bool = False):
        self.cfg, self.L, self.nB, self.t_new, self.c_rows = cfg, n_layers, n_seqs, t_new, c_rows
        self.device = dev = torch.device(device)
        H, d, T = cfg.n_kv_heads, cfg.head_dim, n_seqs * t_new
        i32 = dict(dtype=torch.int32, device=dev)
        self.batch = B.Batch(n_layers, n_seqs, t_new, T)
        self.ws_match = torch.empty(B.spindlekv_match_workspace_bytes(self.batch, H), dtype=torch.uint8, device=dev)
        self.ref_new = torch.zeros((n_layers, H, T), **i32)
        self.mag_new = torch.zeros((n_layers, H, T), dtype=torch.float32, device=dev)
        self.left_idx = torch.zeros((n_layers, H, T), **i32)
        self.left_cnt = torch.zeros((n_layers, n_seqs, H), **i32)
        self.left_rows = torch.zeros((n_layers, n_seqs, H, t_new, d), dtype=dtype, device=dev)
        self.left_batch = B.Batch(n_layers, n_seqs, t_new, T, None, self.left_cnt)   # lengths per head, on the device
        self.ws_codebook = torch.empty(B.spindlekv_workspace_bytes(cfg, self.left_batch, B.WS_CODEBOOK), dtype=torch.uint8, device=dev)
        self.left = {"mag": torch.zeros((n_layers, H, T), dtype=torch.float32, device=dev), "ref": torch.zeros((n_layers, H, T), **i32),
                     "centre_idx": torch.zeros((n_layers, H, T), **i32), "n_entries": torch.zeros((n_layers, n_seqs, H), **i32)}
        self.adj = torch.zeros((n_layers * n_seqs * H, t_new, B.row_words(t_new)), **i32) if keep_adjacency else None

    def run(self, G_new: torch.Tensor, C: torch.Tensor, n_entries: torch.Tensor, theta: float, stream=None) -> None:
        cfg, H, d = self.cfg, self.cfg.n_kv_heads, self.cfg.head_dim
        gd, cd, ld = B.desc_bhnd(G_new), B.desc_bhnd(C), B.desc_bhnd(self.left_rows)
        B.spindlekv_codebook_match(self.batch, H, d, gd, cd, n_entries, self.c_rows, theta, self.mag_new, self.ref_new,
                                   self.left_idx, self.left_cnt, self.ws_match, stream)
        B.spindlekv_compact(self.batch, H, d, gd, self.left_idx, self.left_cnt, ld, None, None, stream)
        o = self.left
        B.spindlekv_codebook_shallow(cfg, self.left_batch, ld, theta, o["mag"], o["ref"], o["centre_idx"], o["n_entries"],
                                     self.ws_codebook, self.adj, stream)
        B.spindlekv_codebook_append(self.batch, H, d, ld, o["mag"], o["ref"], o["centre_idx"], o["n_entries"],
                                    self.left_idx, self.left_cnt, cd, self.c_rows, n_entries, self.ref_new, stream)


class SpindleKVDecodeAttention:
    """Buffers for ``spindlekv_decode_attend``: the table of rotary cosines and sines, the scratch of the split
    pass and the output ``[L, B, H_q, d]`` (fp32).  ``batch`` describes the cached tokens.  Call order only."""

    def __init__(self, batch: B.Batch, n_q_heads: int, n_kv_heads: int, head_dim: int, n_positions: int,
                 rope_base: float = 10000.0, device="cuda"):
        self.batch, self.Hq, self.Hkv, self.d = batch, n_q_heads, n_kv_heads, head_dim
        dev = torch.device(device)
        self.table = torch.empty((n_positions, head_dim // 2, 2), dtype=torch.float32, device=dev)
        B.spindlekv_rope_table(head_dim, n_positions, rope_base, self.table)
        self.ws = torch.empty(B.spindlekv_decode_workspace_bytes(batch, n_q_heads, n_kv_heads, head_dim), dtype=torch.uint8, device=dev)
        self.out = torch.zeros((batch.n_layers, batch.n_seqs, n_q_heads, head_dim), dtype=torch.float32, device=dev)

    def run(self, q: torch.Tensor, pos_q: torch.Tensor, cb_k: Dict[str, torch.Tensor], cb_v: Dict[str, torch.Tensor],
            positions: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """``q``: ``[L, B, H_q, 1, d]`` pre-RoPE queries; ``cb_k`` / ``cb_v``: the ``C``, ``ref``, ``mag`` a CodeBook pass left."""
        B.spindlekv_decode_attend(self.batch, self.Hq, self.Hkv, self.d, B.desc_bhnd(q), pos_q, B.desc_bhnd(cb_k["C"]),
                                  cb_k["ref"], cb_k["mag"], B.desc_bhnd(cb_v["C"]), cb_v["ref"], cb_v["mag"], positions,
                                  self.table, self.out, self.ws, stream)
        return self.out


def _layout(t: Optional[torch.Tensor]):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


class _OnDevice:
    """Calls go to the current device and stream; ``_elsewhere`` says that the owner's device has to be made current first."""

    def _elsewhere(self) -> bool:
        return B.current_device() != self._index

    def _raw(self, stream) -> int:
        return B.raw_stream(self._index) if stream is None else B._stream(stream)

    def _empty(self, shape, dtype, stream, zero: bool = False) -> torch.Tensor:
        """Memory that is made within a call belongs to that call's stream: what the current stream still does with a block that the
        allocator hands out again is in no order with ``stream``."""
        raw, make = self._raw(stream), torch.zeros if zero else torch.empty
        if raw == B.raw_stream(self._index):
            return make(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(torch.cuda.ExternalStream(raw, self.device) if raw else torch.cuda.default_stream(self.device)):
            return make(shape, dtype=dtype, device=self.device)

    def _mine(self, name: str, t: torch.Tensor, dtype=None, shape=None) -> torch.Tensor:
        """``t``, if the library may be given its address as it is."""
        if t.device != self.device or (dtype is not None and t.dtype != dtype) or (shape is not None and t.shape != shape) or not t.is_contiguous():
            want = " ".join(str(x) for x in (dtype, None if shape is None else list(shape)) if x is not None)
            raise ValueError(f"{name}: contiguous {want} on {self.device} expected, got {t.dtype} {list(t.shape)} on {t.device}")
        return t


def _device_of(device) -> torch.device:
    dev = torch.device(device)
    return torch.device(dev.type, torch.cuda.current_device()) if dev.type == "cuda" and dev.index is None else dev


class SpindleKVPagedCache(_OnDevice):
    """A cache in 8 bits on pages: the pool, the page table of ``n_layers`` x ``n_seqs`` sequences, the scratch, and the calls on them.
    A step of decoding is ``resize(add=1)``, then for every layer ``append`` and ``attend``; a step of beam search ends with ``fork``.
    ``max_pages`` bounds a sequence's pages, ``n_pages`` the pool's.  All calls of one object, its construction (on the stream current
    then) included, must be ordered (one stream, or events): they share its scratch.  Buffers and call order only."""

    def __init__(self, n_layers: int, n_seqs: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, max_pages: int,
                 page_size: int = 64, fmt: str = "int8", device="cuda"):
        dev = _device_of(device)
        formats = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
        if fmt not in formats:
            raise ValueError(f"unknown format {fmt!r}: one of {sorted(formats)}")
        codes = dict(dtype=formats[fmt], device=dev)
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        pool = {g + "_codes": torch.zeros(shape, **codes) for g in ("k", "v")}
        pool.update({g + "_scale": torch.zeros((n_pages, n_kv_heads, page_size // B.PAGED_BLOCK), dtype=torch.float32, device=dev) for g in ("k", "v")})
        pool["page_ref"] = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        pages = torch.full((n_layers, n_seqs, max_pages), -1, dtype=torch.int32, device=dev)
        self._init(pool, pages, torch.zeros((n_layers, n_seqs), dtype=torch.int32, device=dev), n_q_heads)

    @classmethod
    def over(cls, pool: Dict[str, torch.Tensor], pages: torch.Tensor, lens: torch.Tensor, n_q_heads: Optional[int] = None):
        """The same over buffers that exist: ``pool`` has ``k_codes``, ``v_codes``, ``k_scale``, ``v_scale`` and ``page_ref``."""
        self = cls.__new__(cls)
        self._init(pool, pages, lens, n_q_heads)
        return self

    def _init(self, pool, pages, lens, n_q_heads) -> None:
        self.pool = B.PagePool(*(pool[k] for k in ("k_codes", "v_codes", "k_scale", "v_scale", "page_ref")))
        self.table = B.PageTable(pages, lens)
        self.device, self.pages, self.lens, self.page_ref = self.pool.device, pages, lens, pool["page_ref"]
        self._index = self.device.index
        if pages.device != self.device:
            raise ValueError(f"pages on {pages.device}, the pool on {self.device}")
        self.n_layers, self.n_seqs, max_pages = pages.shape
        self.Hkv, self.page_size, self.d = pool["k_codes"].shape[1:]
        self.Hq = n_q_heads
        self.capacity = max_pages * self.page_size
        n = B.spindlekv_pages_workspace_bytes(self.pool, self.table)
        if n == 0:
            raise ValueError(f"unsupported page pool: {tuple(pool['k_codes'].shape)}, table {tuple(pages.shape)}")
        self.ws_pages = torch.zeros(n, dtype=torch.uint8, device=self.device)
        self.start = torch.full((self.n_layers, self.n_seqs), -1, dtype=torch.int32, device=self.device)
        self.no_tokens = torch.zeros((self.n_layers, self.n_seqs), dtype=torch.int32, device=self.device)
        self.n_live = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._tables = {}
        self._rotated = (None, None)                       # layouts of the last append_rotated, and what follows from them
        self._writing = threading.Lock()                   # of addresses into these
        self._out: Dict[tuple, torch.Tensor] = {}
        n = B.spindlekv_paged_workspace_bytes(self.pool, self.table, self.Hkv, 1)      # the same for every shape that is served
        self.ws_attend = torch.zeros(n, dtype=torch.uint8, device=self.device)

    def _rows_of(self, layer: Optional[int]) -> B.PageTable:
        """The table of all layers, or of one."""
        if layer is None:
            return self.table
        if layer not in self._tables:
            if not 0 <= layer < self.n_layers:
                raise IndexError(f"layer {layer} of {self.n_layers}")
            self._tables[layer] = B.PageTable(self.pages[layer:layer + 1], self.lens[layer:layer + 1])
        return self._tables[layer]

    def _cache_rows(self, name: str, t: torch.Tensor, n_l: int, heads: int) -> B._Tensor:
        shape, strides = t.shape, t.stride()
        if len(shape) != 5 or shape[0] != n_l or shape[1] != self.n_seqs or shape[2] != heads or shape[4] != self.d or strides[4] != 1 \
                or t.device != self.device:
            raise ValueError(f"{name}: [{n_l}, {self.n_seqs}, {heads}, rows, {self.d}] on {self.device} expected, rows contiguous, got {list(shape)} on {t.device}")
        return B._Tensor(t.data_ptr(), B._dtype_code(t), strides[0], strides[1], strides[2], strides[3])

    def resize(self, new_lens: Optional[torch.Tensor] = None, add: int = 0, stream=None) -> torch.Tensor:
        """Pages for new lengths (``[n_layers, n_seqs]`` int32 on the device, or every length plus ``add``).  Returns ``start``, where
        ``append`` goes on; ``status()`` tells when there were too few pages."""
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.resize(new_lens, add, stream)
        if new_lens is not None:
            self._mine("new_lens", new_lens, torch.int32, (self.n_layers, self.n_seqs))
        B.spindlekv_pages_resize(self.pool, self.table, new_lens, add, self.start, self.ws_pages, self._raw(stream))
        return self.start

    def append(self, K: torch.Tensor, V: torch.Tensor, start: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None,
               idx_seq: Optional[int] = None, max_new: Optional[int] = None, layer: Optional[int] = None, stream=None) -> None:
        """Writes tokens ``start .. lens-1`` (``start`` of the last ``resize`` by default) from rows ``[n_layers or 1, n_seqs, H_kv, rows, d]``;
        with ``idx`` ``[n_layers or 1, H_kv, n_seqs * idx_seq]`` from the rows it names."""
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.append(K, V, start, idx, idx_seq, max_new, layer, stream)
        table = self._rows_of(layer)
        n_l = table.n_layers
        if start is None:
            start = self.start
        if layer is not None and start.shape[0] == self.n_layers:
            start = start[layer:layer + 1]
        self._mine("start", start, torch.int32, (n_l, self.n_seqs))
        if V.shape[3] != K.shape[3]:
            raise ValueError("K and V have different numbers of rows")
        if idx is not None:
            self._mine("idx", idx, torch.int32)
            if idx.dim() != 3 or idx.shape[0] != n_l or idx.shape[1] != self.Hkv:
                raise ValueError(f"idx: [{n_l}, {self.Hkv}, n_seqs * idx_seq] expected, got {list(idx.shape)}")
            idx_seq = idx.shape[2] // self.n_seqs if idx_seq is None else idx_seq
        if max_new is None:
            max_new = K.shape[3] if idx is None else idx_seq
        k, v = self._cache_rows("K", K, n_l, self.Hkv), self._cache_rows("V", V, n_l, self.Hkv)
        B.spindlekv_paged_append(self.pool, table, start, max_new, k, v, K.shape[3], idx, idx_seq or 0, self._raw(stream))

    def append_rotated(self, K: torch.Tensor, V: torch.Tensor, rope_table: torch.Tensor, start: Optional[torch.Tensor] = None,
                       first_pos: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None, idx_seq: Optional[int] = None, max_new: Optional[int] = None,
                       K_out: Optional[torch.Tensor] = None, Q: Optional[torch.Tensor] = None, Q_out: Optional[torch.Tensor] = None, layer: Optional[int] = None,
                       stream=None) -> Optional[torch.Tensor]:
        """``append`` of keys that ``rope_table`` (``[n_positions, d/2, 2]`` fp32, ``spindlekv_rope_table``) rotates on the way: row ``r`` of a sequence by
        position ``first_pos + r`` (``first_pos`` ``[n_layers or 1, n_seqs]`` int32; ``start`` by default, 0 with ``idx``).  ``K_out``, if given, gets the rotated
        keys (it may be ``K``); queries ``Q`` ``[n_layers or 1, n_seqs, H_q, rows, d]`` of the same rows are rotated alike into ``Q_out`` (it may be ``Q``; by
        default a new tensor, zeros behind the new rows), which is returned.  ``K_out`` and ``Q_out`` share memory with no other tensor of the call."""
        if B.current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.append_rotated(K, V, rope_table, start, first_pos, idx, idx_seq, max_new, K_out, Q, Q_out, layer, stream)
        table = self.table if layer is None else self._rows_of(layer)
        start = self.start if start is None else start
        if layer is not None:
            start, first_pos = (t[layer:layer + 1] if t is not None and t.shape[0] == self.n_layers else t for t in (start, first_pos))
        if Q is not None and Q_out is None:
            Q_out = self._empty(Q.shape, Q.dtype, stream, zero=True)
        # arguments laid out as those of the last call have been looked over
        layouts = (layer is None, _layout(K), _layout(V), _layout(rope_table), _layout(start), _layout(first_pos), _layout(idx), _layout(K_out), _layout(Q), _layout(Q_out))
        with self._writing:
            if layouts != self._rotated[0]:
                self._rotated = (layouts, self._look_over_rotated(table.n_layers, K, V, rope_table, start, first_pos, idx, K_out, Q, Q_out))
            kd, vd, kod, qd, qod, hq, n_rows = self._rotated[1]
            kd.ptr, vd.ptr = K.data_ptr(), V.data_ptr()
            if K_out is not None:
                kod.ptr = K_out.data_ptr()
            if Q is not None:
                qd.ptr, qod.ptr = Q.data_ptr(), Q_out.data_ptr()
            if idx is not None and idx_seq is None:
                idx_seq = idx.shape[2] // self.n_seqs
            if max_new is None:
                max_new = n_rows if idx is None else idx_seq
            B.spindlekv_paged_append_rotated(self.pool, table, start, max_new, kd, vd, n_rows, rope_table, first_pos, kod, hq, qd, qod, idx, idx_seq or 0, self._raw(stream))
        return Q_out

    def _look_over_rotated(self, n_l, K, V, rope_table, start, first_pos, idx, K_out, Q, Q_out):
        """Checks of ``append_rotated``; descriptors of its rows, the query heads and the rows of each."""
        self._mine("start", start, torch.int32, (n_l, self.n_seqs))
        if first_pos is not None:
            self._mine("first_pos", first_pos, torch.int32, (n_l, self.n_seqs))
        self._mine("rope_table", rope_table, torch.float32)
        if rope_table.dim() != 3 or rope_table.shape[1:] != (self.d // 2, 2):
            raise ValueError(f"rope_table: [positions, {self.d // 2}, 2] expected, got {list(rope_table.shape)}")
        if idx is not None:
            self._mine("idx", idx, torch.int32)
            if idx.dim() != 3 or idx.shape[0] != n_l or idx.shape[1] != self.Hkv:
                raise ValueError(f"idx: [{n_l}, {self.Hkv}, n_seqs * idx_seq] expected, got {list(idx.shape)}")
        if Q is None and Q_out is not None:
            raise ValueError("Q_out without Q")
        hq = 0 if Q is None else Q.shape[2] if Q.dim() == 5 else -1
        out = []
        for name, t, heads in (("K", K, self.Hkv), ("V", V, self.Hkv), ("K_out", K_out, self.Hkv), ("Q", Q, hq), ("Q_out", Q_out, hq)):
            out.append(B.NO_TENSOR if t is None else self._cache_rows(name, t, n_l, heads))
            if t is not None and t.shape[3] != K.shape[3]:
                raise ValueError(f"{name}: {K.shape[3]} rows expected as in K, got {t.shape[3]}")
        return (*out, hq, K.shape[3])

    def attend(self, q: torch.Tensor, out: Optional[torch.Tensor] = None, max_len: Optional[int] = None, scale: float = 0.0,
               layer: Optional[int] = None, stream=None) -> torch.Tensor:
        """Attention of the last ``rows`` tokens, ``q`` ``[n_layers or 1, n_seqs, H_q, rows, d]``.  Without ``out`` the result lies in a
        buffer of this object that the next call of the same shape overwrites, another layer's too; a buffer per shape is kept as long as the
        object, since recorded graphs write into them.  ``max_len`` (the longest sequence, the capacity by
        default) sizes the split and chooses the kernel: a cache with far more room than tokens is served faster with it."""
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.attend(q, out, max_len, scale, layer, stream)
        table = self.table if layer is None else self._rows_of(layer)
        shape = q.shape
        hq = shape[2] if self.Hq is None else self.Hq
        qd = self._cache_rows("q", q, table.n_layers, hq)
        if out is None:
            held = self._out.get((shape, q.dtype))
            if held is None:
                out = self._empty(shape, q.dtype, stream)
                held = self._out[(shape, q.dtype)] = (out, self._cache_rows("out", out, table.n_layers, hq))
            out, od = held
        else:
            if out.shape != shape:
                raise ValueError(f"out: {list(shape)} expected, got {list(out.shape)}")
            od = self._cache_rows("out", out, table.n_layers, hq)
        if self.ws_attend is None:       # given back by its owner: the kernels need no prepared scratch
            self.ws_attend = self._empty((B.spindlekv_paged_workspace_bytes(self.pool, self.table, self.Hkv, 1),), torch.uint8, stream)
        B.spindlekv_paged_attend(self.pool, table, hq, shape[3], max_len or self.capacity, scale, qd, od, self.ws_attend, self._raw(stream))
        return out

    def fork(self, parent: torch.Tensor, stream=None) -> None:
        """Sequence ``i`` becomes what sequence ``parent[i]`` was (int32 ``[n_seqs]`` on the device; -1: empty), in every layer."""
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.fork(parent, stream)
        self._mine("parent", parent, torch.int32, (self.n_seqs,))
        B.spindlekv_pages_fork(self.pool, self.table, parent, self.ws_pages, self._raw(stream))

    def compact(self, stream=None) -> torch.Tensor:
        """Live pages to the lowest page numbers; returns their number (a device tensor)."""
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.compact(stream)
        B.spindlekv_pages_compact(self.pool, self.table, self.n_live, self.ws_pages, self._raw(stream))
        return self.n_live

    def status(self) -> int:
        """Status word of the last ``resize``, ``fork`` or ``compact``, or else of the last ``attend`` (synchronises the device)."""
        torch.cuda.synchronize(self.device)
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.status()
        st = B.spindlekv_poll_status(self.ws_pages)[0]
        return B.spindlekv_poll_status(self.ws_attend)[0] if st == B.OK and self.ws_attend is not None else st


class SpindleKVPromptAttention(_OnDevice):
    """Causal attention of a prompt batch, or of the last rows of one: scratch of ``spindlekv_prompt_attend`` for batches of one shape.  ``keys`` describes
    K and V, ``rows`` the queries (every token by default).  Tensors are ``[L, B, H, N, d]``, or packed ``[L, T, H, d]`` where their batch has
    ``cu_seqlens``.  All calls of one object must be ordered: they share the scratch."""

    def __init__(self, keys: B.Batch, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, rows: Optional[B.Batch] = None, device="cuda"):
        self.keys, self.rows, self.Hq, self.Hkv, self.d, self.dtype = keys, rows or keys, n_q_heads, n_kv_heads, head_dim, dtype
        self.device = dev = _device_of(device)
        self._index = dev.index
        codes = {torch.float32: B.F32, torch.bfloat16: B.BF16}
        if dtype not in codes:
            raise TypeError(f"unsupported dtype {dtype}")
        for b in (self.keys, self.rows):
            for t, n in ((b.cu_seqlens, b.n_seqs + 1), (b.layer_lens, b.n_layers * b.n_seqs)):
                if t is not None and (t.device != dev or t.dtype != torch.int32 or not t.is_contiguous() or t.numel() != n):
                    raise ValueError(f"lengths: {n} contiguous int32 on {dev} expected, got {t.dtype} {list(t.shape)} on {t.device}")
        n = B.spindlekv_prompt_workspace_bytes(self.keys, self.rows, n_q_heads, n_kv_heads, head_dim, codes[dtype])
        if n == 0:
            raise ValueError(f"unsupported attention: {n_q_heads} query heads, {n_kv_heads} KV heads of {head_dim}, {self.keys}, {self.rows}")
        self.ws = torch.empty(n, dtype=torch.uint8, device=dev)
        self._c = self.keys.c(), self.rows.c()
        self._seen = (None, None)                          # layouts of the last call, and the descriptors that follow from them
        self._writing = threading.Lock()                   # of addresses into these

    def _rows_of(self, name: str, t: torch.Tensor, b: B.Batch, heads: int) -> B._Tensor:
        shape, strides = t.shape, t.stride()
        want = (b.n_layers, b.total_len, heads, self.d) if b.cu_seqlens is not None else (b.n_layers, b.n_seqs, heads, b.max_len, self.d)
        if shape != want or strides[-1] != 1 or t.dtype != self.dtype or t.device != self.device:
            raise ValueError(f"{name}: {list(want)} {self.dtype} on {self.device} expected, rows contiguous, got {list(shape)} {t.dtype} on {t.device}")
        if b.cu_seqlens is not None:
            return B._Tensor(t.data_ptr(), B._dtype_code(t), strides[0], 0, strides[2], strides[1])
        return B._Tensor(t.data_ptr(), B._dtype_code(t), strides[0], strides[1], strides[2], strides[3])

    def run(self, q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, scale: float = 0.0,
            stream=None) -> torch.Tensor:
        """``out`` (made by the call by default: zeros behind a sequence's rows) and ``lse`` ``[L, H_q, T]`` fp32, if given, are written; returns ``out``."""
        if B.current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.run(q, K, V, out, lse, scale, stream)
        if out is None:
            out = self._empty(q.shape, q.dtype, stream, zero=self.rows.cu_seqlens is not None or self.rows.layer_lens is not None)
        # arguments laid out as those of the last call have been looked over
        layouts = (_layout(q), _layout(K), _layout(V), _layout(out), _layout(lse))
        with self._writing:
            if layouts != self._seen[0]:
                rows = (("q", q, self.rows, self.Hq), ("K", K, self.keys, self.Hkv), ("V", V, self.keys, self.Hkv), ("out", out, self.rows, self.Hq))
                if lse is not None:
                    self._mine("lse", lse, torch.float32, (self.rows.n_layers, self.Hq, self.rows.total_len))
                self._seen = (layouts, tuple(self._rows_of(*r) for r in rows))
            qd, kd, vd, od = self._seen[1]
            qd.ptr, kd.ptr, vd.ptr, od.ptr = q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr()
            B.spindlekv_prompt_attend(self._c[0], self._c[1], self.Hq, self.Hkv, self.d, scale, qd, kd, vd, od, lse, self.ws, self._raw(stream))
        return out

    def status(self) -> int:
        """Status word of the last call (synchronises the device)."""
        torch.cuda.synchronize(self.device)
        with torch.cuda.device(self.device):
            return B.spindlekv_poll_status(self.ws)[0]


class SpindleKVLogits(_OnDevice):
    """Penalties for repeated tokens, biases and masks of allowed tokens (``spindlekv_logits_adjust``) for ``n_rows`` rows of logits over ``vocab`` tokens, e.g. the
    beams of ``SpindleKVBeamSelect``.  No scratch: calls of one object need no order on the device; host threads take an object each."""

    def __init__(self, n_rows: int, vocab: int, device="cuda"):
        if not (0 < n_rows < 65536 and 0 < vocab <= 1 << 30):
            raise ValueError(f"unsupported logits: {n_rows} rows, vocabulary {vocab}")
        self.n_rows, self.vocab = n_rows, vocab
        self.device = _device_of(device)
        self._index = self.device.index
        self._seen = (None, None)                          # layouts of the last call, and the rules that follow from them

    def _logits(self, name: str, t: torch.Tensor, dtype=None) -> torch.Tensor:
        if t.shape != (self.n_rows, self.vocab) or (self.vocab > 1 and t.stride(1) != 1) or t.device != self.device or (dtype is not None and t.dtype != dtype):
            raise ValueError(f"{name}: [{self.n_rows}, {self.vocab}] {dtype or ''} on {self.device} expected, rows contiguous, got {list(t.shape)} {t.dtype} on {t.device}")
        return t

    def adjust(self, logits: torch.Tensor, out: Optional[torch.Tensor] = None, history: Optional[torch.Tensor] = None, history_lens: Optional[torch.Tensor] = None,
               n_prompt: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None, presence: Optional[torch.Tensor] = None,
               frequency: Optional[torch.Tensor] = None, bias_token: Optional[torch.Tensor] = None, bias_value: Optional[torch.Tensor] = None,
               allowed: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """``history`` ``[n_rows, n]`` int32 (any row stride) with ``history_lens`` tokens each, of which the first ``n_prompt`` are the prompt's; ``repetition``,
        ``presence``, ``frequency`` fp32 ``[n_rows]``; ``bias_token`` int32 and ``bias_value`` fp32 ``[n_rows, n]``; ``allowed`` int32 or uint32 ``[n_rows or 1,
        ceil(vocab / 32)]``, a bit per token, the lowest first.  Returns ``out`` (``logits`` itself, in place, by default)."""
        if B.current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.adjust(logits, out, history, history_lens, n_prompt, repetition, presence, frequency, bias_token, bias_value, allowed, stream)
        if out is None:
            out = logits
        # arguments laid out as those of the last call have been looked over
        layouts = (_layout(logits), _layout(out), _layout(history), _layout(history_lens), _layout(n_prompt), _layout(repetition), _layout(presence), _layout(frequency),
                   _layout(bias_token), _layout(bias_value), _layout(allowed))
        if layouts != self._seen[0]:
            self._seen = (layouts, self._look_over(logits, out, history, history_lens, n_prompt, repetition, presence, frequency, bias_token, bias_value, allowed))
        r = self._seen[1]
        if r.max_history:
            r.history = history.data_ptr()
            r.history_lens = None if history_lens is None else history_lens.data_ptr()
            r.n_prompt = None if n_prompt is None else n_prompt.data_ptr()
            r.repetition = None if repetition is None else repetition.data_ptr()
            r.presence = None if presence is None else presence.data_ptr()
            r.frequency = None if frequency is None else frequency.data_ptr()
        if r.n_bias:
            r.bias_token, r.bias_value = bias_token.data_ptr(), bias_value.data_ptr()
        if allowed is not None:
            r.allowed = allowed.data_ptr()
        B.spindlekv_logits_adjust(logits, out, r, self._raw(stream))
        return out

    def _look_over(self, logits, out, history, history_lens, n_prompt, repetition, presence, frequency, bias_token, bias_value, allowed) -> "B._LogitRules":
        """Checks of ``adjust``; the rules without their addresses."""
        r, n = B._LogitRules(), self.n_rows
        self._logits("logits", logits)
        self._logits("out", out, logits.dtype)
        vectors = (("history_lens", history_lens, torch.int32), ("n_prompt", n_prompt, torch.int32), ("repetition", repetition, torch.float32),
                   ("presence", presence, torch.float32), ("frequency", frequency, torch.float32))
        for name, t, dtype in vectors:
            if t is not None:
                if history is None:
                    raise ValueError(f"{name} without a history")
                self._mine(name, t, dtype, (n,))
        if history is not None:
            if history.dim() != 2 or history.shape[0] != n or (history.shape[1] > 1 and history.stride(1) != 1) or history.dtype != torch.int32 or history.device != self.device:
                raise ValueError(f"history: [{n}, tokens] int32 on {self.device} expected, rows contiguous, got {list(history.shape)} {history.dtype} on {history.device}")
            r.history_stride, r.max_history = history.stride(0), history.shape[1]
        if (bias_token is None) != (bias_value is None):
            raise ValueError("bias_token and bias_value belong together")
        if bias_token is not None:
            if bias_token.dim() != 2 or bias_token.shape[0] != n:
                raise ValueError(f"bias_token: [{n}, biases] expected, got {list(bias_token.shape)}")
            self._mine("bias_token", bias_token, torch.int32)
            self._mine("bias_value", bias_value, torch.float32, bias_token.shape)
            r.n_bias = bias_token.shape[1]
        if allowed is not None:
            words = (self.vocab + 31) // 32
            if allowed.dtype not in (torch.int32, torch.uint32) or allowed.dim() != 2 or allowed.shape[0] not in (1, n) or allowed.shape[1] != words:
                raise ValueError(f"allowed: [{n} or 1, {words}] int32 or uint32 expected, got {list(allowed.shape)} {allowed.dtype}")
            self._mine("allowed", allowed)
            r.allowed_stride = words if allowed.shape[0] == n else 0
        return r


class SpindleKVBeamSelect(_OnDevice):
    """Beam search's selection for batches of one shape: scratch and result buffers of ``spindlekv_beam_select``.  All calls of one object
    must be ordered: they share both."""

    def __init__(self, n_seqs: int, n_beams: int, vocab: int, n_out: Optional[int] = None, device="cuda"):
        self.n_seqs, self.n_beams, self.vocab, self.n_out = n_seqs, n_beams, vocab, n_beams if n_out is None else n_out
        self.device = dev = _device_of(device)
        self._index = dev.index
        n = B.spindlekv_beam_workspace_bytes(n_seqs, n_beams, vocab, self.n_out)
        if n == 0:
            raise ValueError(f"unsupported beam search: {n_seqs} x {n_beams} beams, vocabulary {vocab}, {self.n_out} wanted")
        self.ws = torch.empty(n, dtype=torch.uint8, device=dev)
        self.score = torch.empty((n_seqs, self.n_out), dtype=torch.float32, device=dev)
        self.parent = torch.empty((n_seqs, self.n_out), dtype=torch.int32, device=dev)
        self.token = torch.empty((n_seqs, self.n_out), dtype=torch.int32, device=dev)

    def run(self, logits: torch.Tensor, score: torch.Tensor, finished: Optional[torch.Tensor] = None, eos: int = 0, stream=None):
        """``logits`` ``[n_seqs * n_beams, vocab]`` (any row stride), ``score`` and ``finished`` (bool) ``[n_seqs * n_beams]``.  Returns
        ``(score, parent, token)``, each ``[n_seqs, n_out]``, best first, in buffers that the next call overwrites."""
        if self._elsewhere():
            with torch.cuda.device(self.device):
                return self.run(logits, score, finished, eos, stream)
        rows = self.n_seqs * self.n_beams
        if logits.shape != (rows, self.vocab) or (self.vocab > 1 and logits.stride(1) != 1) or logits.device != self.device:
            raise ValueError(f"logits: [{rows}, {self.vocab}] on {self.device} expected, got {list(logits.shape)} on {logits.device}")
        self._mine("score", score, torch.float32, (rows,))
        if finished is not None:
            self._mine("finished", finished, torch.bool, (rows,))
        B.spindlekv_beam_select(self.n_seqs, self.n_beams, self.vocab, self.n_out, logits, score, finished, eos, self.score, self.parent,
                                self.token, self.ws, self._raw(stream))
        return self.score, self.parent, self.token
