"""A cached DiT stack driven through the C ABI: the user-facing step.

`CachedStack` owns the per-layer int8 caches, the workspaces and the index
buffers on the device and runs one denoising step as the paper orders it
(Sec. 3.3): the audio energy once per generation, then per layer the
energy-guided selection and the block on the selected latents.  Step 0 (or
any step with full=True) refreshes every token and fills the caches.  No host
synchronisation happens inside a fixed-ratio step: K follows from the ratio on
the host.  An adaptive step (AdaptiveRate) reads one scalar back: the change
of the step before.
"""
from __future__ import annotations

import json
import os

import torch

from . import echocache as ec


class AdaptiveRate:
    """The step-level update rate of Sec. 3.3 for a CachedStack.

    After every step the change of Eq. 1 between the stack output of that step
    and of the step before is reduced on the device (echo_step_delta) and
    copied into pinned host memory.  The next cached step's budget
    (echo_update_rate) waits for that copy only: r_t follows the most recent
    change, normalised by the first change measured (Delta-hat = 1 before any
    change is known), and K_t = ceil(r_t NT).  Waiting for the copy is the one
    host synchronisation of an adaptive step."""

    def __init__(self, NT: int, r_min: float = 0.1, r_max: float = 0.5, alpha: float = 0.2,
                 xi: float = 1e-6, device="cuda"):
        self.NT, self.r_min, self.r_max, self.alpha, self.xi = NT, r_min, r_max, alpha, xi
        dev = torch.device(device)
        self.out = torch.zeros(3, dtype=torch.float64, device=dev)
        self.host = torch.zeros(3, dtype=torch.float64).pin_memory()
        self.ws = torch.empty(ec.echo_step_delta_workspace_size(0), dtype=torch.uint8, device=dev)
        self.ready = torch.cuda.Event()
        self.pending = False
        self.h_prev = None
        self.deltas: list[float] = []
        self.rates: list[float] = []
        self.budgets: list[int] = []

    def budget(self) -> int:
        """K for the next cached step (waits for the last change's copy)."""
        if self.pending:
            self.ready.synchronize()
            self.deltas.append(float(self.host[0]))
            self.pending = False
        d, ref = (self.deltas[-1], self.deltas[0]) if self.deltas else (1.0, 1.0)
        rate, K = ec.echo_update_rate(d, ref, self.NT, self.r_min, self.r_max, self.alpha)
        self.rates.append(rate)
        self.budgets.append(K)
        return K

    def observe(self, h_cur: torch.Tensor):
        """Enqueue the change between the previous step's output and h_cur on
        the current stream.  The previous output must stay unchanged until
        this work has run."""
        if self.h_prev is not None:
            ec.echo_step_delta(self.h_prev, h_cur, self.xi, out=self.out, workspace=self.ws)
            self.host.copy_(self.out, non_blocking=True)
            self.ready.record()
            self.pending = True
        self.h_prev = h_cur


class CachedStack:
    def __init__(self, T: int, N: int, D: int, H: int, d: int, F: int, Lc: int,
                 blocks: list, device="cuda", lam: float = 0.1, xi: float = 1e-6,
                 mode: int = ec.MODE_ENERGY_DRIFT, cache_kind: int = ec.CACHE_INT8,
                 R_cap: int | None = None, seg_len: int = 1, tau: float = 0.9,
                 selection: str = "energy", seed: int = 0, reuse_kv: bool = False):
        """cache_kind: ec.CACHE_INT8 (plain int8), ec.CACHE_BF16 (full
        precision) or ec.CACHE_REF (reference plus int8 residual, Sec. 3.4,
        with R_cap, seg_len and tau).  selection: "energy" (the energy-guided
        anchors of Sec. 3.3), or the ablations "uniform" and "random" (keys
        drawn on the device from a generator seeded with `seed`).
        reuse_kv (int8 cache only): keep every layer's K/V of all tokens on the
        device (NT x 2D bf16 per layer) and recompute, at layers >= 1, only the
        rows whose input changed: the tokens refreshed at the layer below in
        this step or the step before (echo_block_step_kv).  The outputs are
        bit for bit those without reuse."""
        if selection not in ("energy", "uniform", "random"):
            raise ValueError(f"unknown selection {selection!r}")
        if reuse_kv and cache_kind != ec.CACHE_INT8:
            raise ValueError("reuse_kv needs the int8 cache form")
        self.T, self.N, self.D = T, N, D
        self.NT = T * N
        self.dims = ec.BlockDims(T, N, D, H, d, F, Lc)
        self.blocks = blocks
        self.lam, self.xi, self.mode = lam, xi, mode
        self.cache_kind, self.selection = cache_kind, selection
        dev = torch.device(device)
        L = len(blocks)
        if cache_kind == ec.CACHE_INT8:
            self.cache_q = [torch.zeros(self.NT, D, dtype=torch.int8, device=dev) for _ in range(L)]
            self.cache_s = [torch.zeros(self.NT, dtype=torch.float32, device=dev) for _ in range(L)]
            self.caches = None
            ws = ec.echo_workspace_size(self.dims, self.NT)
        else:
            self.caches = [ec.DeviceCache(cache_kind, self.NT, D, R_cap=R_cap, seg_len=seg_len,
                                          tau=tau, device=dev) for _ in range(L)]
            ws = ec.echo_block_step_cache_workspace_size(self.dims, self.NT, self.caches[0])
        self.reuse_kv = reuse_kv
        if reuse_kv:
            # K/V of every token per layer; the active rows of every layer at
            # the last two steps (slot t & 1), with their counts (NT: a full
            # step, after which the next step recomputes every row)
            ws = ec.echo_workspace_size_kv(self.dims, self.NT, self.NT)
            self.kv = [torch.empty(self.NT, 2 * D, dtype=torch.bfloat16, device=dev)
                       for _ in range(L)]
            self._act = [[torch.empty(self.NT, dtype=torch.int32, device=dev) for _ in range(2)]
                         for _ in range(L)]
            self._act_K = [[self.NT, self.NT] for _ in range(L)]
            self._kv_ok = [False] * L
            self._t = 0
        self.ws = torch.empty(ws, dtype=torch.uint8, device=dev)
        self.keys = torch.empty(self.NT, dtype=torch.float32, device=dev)
        self.gen = torch.Generator(device=dev).manual_seed(seed)
        # ECHO_PROFILE=<path>: bracket every library launch with CUDA events;
        # profile_report() aggregates them (and writes JSON to <path>)
        self.profile_path = os.environ.get("ECHO_PROFILE") or None
        if self.profile_path:
            ec.echo_profile_enable(True)
        self.sel_ws = torch.empty(ec.echo_select_workspace_size(T, N), dtype=torch.uint8, device=dev)
        self.idx = torch.empty(self.NT, dtype=torch.int32, device=dev)
        self.all_idx = torch.arange(self.NT, dtype=torch.int32, device=dev)
        self.scores = torch.empty(self.NT, dtype=torch.float32, device=dev)
        self.y = [torch.empty(self.NT, D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
        # The audio energy runs on a side stream into two alternating buffers:
        # it depends on the audio only, so a step's energy is computed while
        # the previous step's kernels still run; the step waits for it before
        # its first selection.
        self._aud_stream = torch.cuda.Stream(dev)
        self._band = [torch.empty(T, 8, dtype=torch.float32, device=dev) for _ in range(2)]
        self._seg = [torch.zeros(T, dtype=torch.float32, device=dev) for _ in range(2)]
        self._seg_ready = [torch.cuda.Event() for _ in range(2)]
        self._seg_free = [torch.cuda.Event() for _ in range(2)]
        self._next_buf, self._pending, self._in_use = 0, None, 0
        self._audio_key = None
        self.band, self.seg = self._band[0], self._seg[0]
        self.last_K = []
        # Optional inspection hook, called from the host as each layer is
        # enqueued: layer_hook("pre", l, x, None, 0, None) before layer l's
        # selection, layer_hook("post", l, x, idx, K, y) after its block step
        # (x is the layer's input, y its output).  A hook that reads device
        # tensors synchronises with the stream; None (the default) costs nothing.
        self.layer_hook = None

    def set_audio(self, audio: torch.Tensor, n_fft: int = 512, hop: int = 160, n_bands: int = 8):
        """Segment energy of the audio (Sec. 3.3) for the next step.  The result
        is written on a side stream; the next step waits for it, and a caller
        that reads the returned tensors directly calls wait_audio() first."""
        dev = self.seg.device
        main = torch.cuda.current_stream(dev)
        side = self._aud_stream
        b = self._next_buf
        self._next_buf ^= 1
        if self._band[b].shape[1] != n_bands:
            self._band[b] = torch.empty(self.T, n_bands, dtype=torch.float32, device=dev)
        side.wait_event(self._seg_free[b])          # the last step that read buffer b is done
        key = (audio.data_ptr(), audio._version)
        if key != self._audio_key:                  # new audio: order after its writes
            ev = torch.cuda.Event()
            ev.record(main)
            side.wait_event(ev)
            self._audio_key = key
        ec.echo_audio_energy(audio, self.T, n_fft, hop, n_bands, self._band[b], self._seg[b],
                             stream=side)
        self._seg_ready[b].record(side)
        self._pending = b
        self.band, self.seg = self._band[b], self._seg[b]
        return self.band, self.seg

    def wait_audio(self):
        """Make the current stream wait for the last set_audio's result."""
        if self._pending is not None:
            torch.cuda.current_stream(self.seg.device).wait_event(self._seg_ready[self._pending])

    def step(self, x: torch.Tensor, ratio_num: int, ratio_den: int, full: bool = False,
             keep_scores: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
        """One denoising step over every layer; returns the last layer's output
        (written into `out` when given)."""
        main = torch.cuda.current_stream(self.seg.device)
        if self._pending is not None:               # this step uses the newest energy
            main.wait_event(self._seg_ready[self._pending])
            self._in_use, self._pending = self._pending, None
        cur = self._layers(x, ratio_num, ratio_den, full, keep_scores, out)
        self._seg_free[self._in_use].record(main)   # set_audio may now overwrite it
        if self.reuse_kv:
            self._t += 1
        return cur

    def _layers(self, x, ratio_num, ratio_den, full, keep_scores, out):
        cur = x
        self.last_K = []
        last = len(self.blocks) - 1
        hook = self.layer_hook
        for l, blk in enumerate(self.blocks):
            if hook is not None:
                hook("pre", l, cur, None, 0, None)
            if full:
                idx, K = self.all_idx, self.NT
            elif self.selection == "uniform":
                idx, K = ec.echo_select_uniform(self.T, self.N, ratio_num, ratio_den, idx=self.idx)
            elif self.selection == "random":
                torch.rand(self.NT, generator=self.gen, out=self.keys)
                idx, K = ec.echo_select_random(self.keys, self.T, self.N, ratio_num, ratio_den,
                                               idx=self.idx)
            elif self.caches is None:
                idx, K, _ = ec.echo_select(cur, self.cache_q[l], self.cache_s[l], self.seg, self.T,
                                           self.N, ratio_num, ratio_den, self.lam, self.xi,
                                           self.mode, idx=self.idx,
                                           scores=self.scores if keep_scores else None,
                                           workspace=self.sel_ws)
            else:
                idx, K, _ = ec.echo_select_cache(cur, self.caches[l], self.seg, self.T, self.N,
                                                 ratio_num, ratio_den, self.lam, self.xi,
                                                 self.mode, idx=self.idx,
                                                 scores=self.scores if keep_scores else None,
                                                 workspace=self.sel_ws)
            dst = out if (l == last and out is not None) else self.y[l % 2]
            if self.reuse_kv:
                self._block_step_kv(l, blk, cur, idx, K, dst)
            elif self.caches is None:
                ec.echo_block_step(blk, self.dims, cur, idx, K, self.cache_q[l], self.cache_s[l],
                                   y=dst, workspace=self.ws)
            else:
                ec.echo_block_step_cache(blk, self.dims, cur, idx, K, self.caches[l], y=dst,
                                         workspace=self.ws)
            self.last_K.append(K)
            if hook is not None:
                hook("post", l, cur, idx, K, dst)
            cur = dst
        return cur

    def _block_step_kv(self, l, blk, x, idx, K, dst):
        """Layer l's block step with its K/V kept across steps (reuse_kv)."""
        t, NT = self._t, self.NT
        valid, ra, na, rb, nb = False, None, 0, None, 0
        if l > 0 and self._kv_ok[l]:
            na, nb = self._act_K[l - 1][t & 1], self._act_K[l - 1][(t - 1) & 1]
            if na + nb < NT:
                valid = True
                ra, rb = self._act[l - 1][t & 1], self._act[l - 1][(t - 1) & 1]
        if not valid:
            na = nb = 0
        ec.echo_block_step_kv(blk, self.dims, x, idx, K, self.kv[l], valid, self.cache_q[l],
                              self.cache_s[l], ra, na, rb, nb, y=dst, workspace=self.ws)
        self._kv_ok[l] = True
        if l + 1 < len(self.blocks):      # the next layer's changed rows
            if 0 < K < NT:
                self._act[l][t & 1][:K].copy_(idx[:K])
            self._act_K[l][t & 1] = K if K < NT else NT

    def capture_step(self, x: torch.Tensor, ratio_num: int, ratio_den: int,
                     out: torch.Tensor | None = None, audio: torch.Tensor | None = None,
                     n_fft: int = 512, hop: int = 160, n_bands: int = 8):
        """Record one cached step over every layer as a CUDA graph and return
        (graph, output tensor).  graph.replay() re-runs the step on the same
        buffers with one launch from the host: copy each step's input into `x`
        first.  With `audio` the graph starts with the audio energy (on the
        graph's own stream); without it, it reads the energy of the last
        set_audio.  Selection "random" draws keys from a host generator and
        cannot be captured.  Run one eager step of the same ratio first, so
        that every kernel's one-time set-up is done."""
        if self.selection == "random":
            raise ValueError("random selection cannot be captured")
        if self.reuse_kv:
            raise ValueError("reuse_kv steps depend on the steps before them and cannot be captured")
        dev = self.seg.device
        self.wait_audio()
        if self._pending is not None:
            self._in_use, self._pending = self._pending, None
        band, seg = self._band[self._in_use], self._seg[self._in_use]
        torch.cuda.synchronize(dev)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            if audio is not None:
                ec.echo_audio_energy(audio, self.T, n_fft, hop, n_bands, band, seg)
            y = self._layers(x, ratio_num, ratio_den, False, False, out)
        return g, y

    # ---- checkpoint / resume of the cross-step state (the per-layer caches) ----
    def cache_state(self) -> dict:
        """Host copy of every layer's cache (the only state carried across steps)."""
        if self.caches is None:
            layers = [{"q": q.cpu(), "scale": s.cpu()} for q, s in zip(self.cache_q, self.cache_s)]
        else:
            layers = [{n: t.cpu() for n, t in c.t.items()} for c in self.caches]
        return {"kind": int(self.cache_kind), "NT": self.NT, "D": self.D, "layers": layers}

    def load_cache_state(self, state: dict):
        """Restore caches saved by cache_state (same form, shapes and layer count)."""
        if (state["kind"], state["NT"], state["D"]) != (int(self.cache_kind), self.NT, self.D):
            raise ValueError("cache state does not match this stack")
        if len(state["layers"]) != len(self.blocks):
            raise ValueError("cache state has a different number of layers")
        if self.reuse_kv:   # the kept K/V belong to the old state
            self._kv_ok = [False] * len(self.blocks)
            self._act_K = [[self.NT, self.NT] for _ in self.blocks]
        for l, layer in enumerate(state["layers"]):
            if self.caches is None:
                self.cache_q[l].copy_(layer["q"])
                self.cache_s[l].copy_(layer["scale"])
            else:
                for n, t in self.caches[l].t.items():
                    t.copy_(layer[n])

    def save_caches(self, path: str):
        torch.save(self.cache_state(), path)

    def load_caches(self, path: str):
        self.load_cache_state(torch.load(path))

    def profile_report(self) -> dict:
        """Per-kernel totals of the launches recorded since the last report
        (profiling is on when ECHO_PROFILE is set); written as JSON to the
        ECHO_PROFILE path."""
        agg = {}
        for name, m, n, k, ms in ec.echo_profile_read():
            a = agg.setdefault(f"{name}[{m}x{n}x{k}]", {"launches": 0, "ms": 0.0})
            a["launches"] += 1
            a["ms"] += ms
        for a in agg.values():
            a["ms_per_launch"] = a["ms"] / a["launches"]
        if self.profile_path:
            with open(self.profile_path, "w") as f:
                json.dump(agg, f, indent=1)
        return agg

    def cache_bytes(self, right_sized: bool = False) -> int:
        """Device bytes of every layer's cache; with right_sized, a reference
        pool holds only the rows in use (its high-water mark; synchronises)."""
        if self.caches is None:
            return sum(q.numel() + 4 * s.numel() for q, s in zip(self.cache_q, self.cache_s))
        if right_sized and self.cache_kind == ec.CACHE_REF:
            return sum(c.nbytes(pool_rows=c.stats()[1]) for c in self.caches)
        return sum(c.nbytes() for c in self.caches)

    def step_adaptive(self, x: torch.Tensor, rate: AdaptiveRate, full: bool = False,
                      keep_scores: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
        """One step whose budget follows the adaptive update rate (Sec. 3.3):
        every layer refreshes K_t = rate.budget() tokens (all on a full step),
        then the step's change from the previous output is enqueued.  Without
        `out` the output alternates between two buffers of the stack, so the
        previous output stays intact; a caller passing `out` keeps the previous
        step's output unchanged until this step's work has run."""
        K = self.NT if full else rate.budget()
        if out is None:
            if not hasattr(self, "_h"):
                self._h = [torch.empty(self.NT, self.D, dtype=torch.bfloat16,
                                       device=self.seg.device) for _ in range(2)]
                self._h_i = 0
            out = self._h[self._h_i]
            self._h_i ^= 1
        y = self.step(x, K, self.NT, full=full, keep_scores=keep_scores, out=out)
        rate.observe(y)
        return y

    def run_host(self, host_x: list, host_y: list, ratio_num: int, ratio_den: int,
                 audio: torch.Tensor | None = None, rate: AdaptiveRate | None = None):
        """Steps whose inputs and outputs live in pinned host memory.

        Step i copies host_x[i] to the device, runs one step (the audio energy
        first when `audio` is given) and copies the result into host_y[i].  The
        copies run on their own streams into double-buffered device tensors, so
        the upload of step i+1 and the download of step i-1 overlap step i.
        With `rate` every step takes the adaptive budget (ratio_num and
        ratio_den are then unused).  Returns after everything has been
        enqueued; synchronise before reading host_y."""
        dev = self.seg.device
        comp = torch.cuda.current_stream(dev)
        if not hasattr(self, "_h2d"):
            self._h2d, self._d2h = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
            self._xd = [torch.empty(self.NT, self.D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
            self._yd = [torch.empty(self.NT, self.D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
            self._ev = {k: [torch.cuda.Event() for _ in range(2)]
                        for k in ("x_ready", "x_used", "y_ready", "y_copied")}
            for k in ("x_used", "y_copied"):
                for e in self._ev[k]:
                    e.record(comp)
        ev = self._ev
        start = torch.cuda.Event()
        start.record(comp)                  # copies start after work already queued
        self._h2d.wait_event(start)
        for i, (hx, hy) in enumerate(zip(host_x, host_y)):
            b = i % 2
            with torch.cuda.stream(self._h2d):
                self._h2d.wait_event(ev["x_used"][b])
                self._xd[b].copy_(hx, non_blocking=True)
                ev["x_ready"][b].record(self._h2d)
            comp.wait_event(ev["x_ready"][b])
            comp.wait_event(ev["y_copied"][b])
            if audio is not None:
                self.set_audio(audio)
            if rate is not None:
                self.step_adaptive(self._xd[b], rate, out=self._yd[b])
            else:
                self.step(self._xd[b], ratio_num, ratio_den, out=self._yd[b])
            ev["x_used"][b].record(comp)
            ev["y_ready"][b].record(comp)
            with torch.cuda.stream(self._d2h):
                self._d2h.wait_event(ev["y_ready"][b])
                hy.copy_(self._yd[b], non_blocking=True)
                ev["y_copied"][b].record(self._d2h)
        comp.wait_event(ev["y_copied"][(len(host_x) - 1) % 2])


class PageTable:
    """Host bookkeeping of a pool of key/value pages that clips share: which pages are free,
    which a clip has, in order.  The same numbers serve the pools of every layer."""

    def __init__(self, n_pages: int, page_tokens: int):
        self.n_pages, self.page_tokens = n_pages, page_tokens
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages: dict[int, list[int]] = {}
        self.lens: dict[int, int] = {}

    def open(self, clip: int):
        if clip in self.lens:
            raise ValueError(f"clip {clip} is open already")
        self.pages[clip], self.lens[clip] = [], 0

    def close(self, clip: int):
        """Give the clip's pages back.  Work already enqueued may still read them: whoever
        gets them next writes them on the same stream."""
        del self.lens[clip]
        self.free.extend(reversed(self.pages.pop(clip)))

    def extend(self, rows: dict[int, int]):
        """Room for rows[clip] more tokens of each clip; all of them or none."""
        need = {c: -(-(self.lens[c] + n) // self.page_tokens) - len(self.pages[c])
                for c, n in rows.items()}
        if sum(need.values()) > len(self.free):
            raise MemoryError(f"{sum(need.values())} pages needed, {len(self.free)} free")
        for c, n in rows.items():
            self.pages[c].extend(self.free.pop() for _ in range(need[c]))
            self.lens[c] += n

    def shorten(self, rows: dict[int, int]):
        """Take back the last rows[clip] tokens of each clip, and the pages that only they
        needed."""
        for c, n in rows.items():
            self.lens[c] -= n
            keep = -(-self.lens[c] // self.page_tokens)
            self.free.extend(reversed(self.pages[c][keep:]))
            del self.pages[c][keep:]

    def batch(self, rows: dict[int, int], device="cuda") -> ec.KVBatch:
        """The clips of one call with their new rows (rows[clip] each, in the dict's order),
        copied to the device."""
        clips = list(rows)
        width = max([len(self.pages[c]) for c in clips] + [1])
        host = [self.pages[c] + [-1] * (width - len(self.pages[c])) for c in clips]
        row0 = [0]
        for n in rows.values():
            row0.append(row0[-1] + n)
        flat = torch.tensor([p for h in host for p in h] + [self.lens[c] for c in clips] + row0,
                            dtype=torch.int32).pin_memory().to(device, non_blocking=True)
        B = len(clips)
        return ec.KVBatch(flat[:B * width].view(B, width), flat[B * width:B * width + B],
                          flat[B * width + B:], row0[-1], max(rows.values(), default=0))


class DevicePageTable:
    """PageTable with the pages' numbers on the GPU (ec.KVTables): the host keeps how many pages each
    clip has, the device which.  extend() enqueues a step's tables, places and positions and copies
    two numbers a clip; with those in device memory already, echo_kv_extend itself copies nothing and
    can be captured."""

    def __init__(self, n_pages: int, page_tokens: int, max_clips: int, device="cuda"):
        self.n_pages, self.page_tokens, self.device = n_pages, page_tokens, torch.device(device)
        self.tables = ec.KVTables.empty(n_pages, page_tokens, max_clips, n_pages, device)
        self.free_slots = list(range(max_clips - 1, -1, -1))
        self.slots: dict[int, int] = {}
        self.lens: dict[int, int] = {}
        self.n_free = n_pages

    def _pages(self, tokens: int) -> int:
        return -(-tokens // self.page_tokens)

    def _numbers(self, rows: dict[int, int]):
        """(slots, rows) of the clips on the device, from one copy."""
        host = torch.tensor([[self.slots[c] for c in rows], list(rows.values())], dtype=torch.int32)
        both = host.pin_memory().to(self.device, non_blocking=True)
        return both[0], both[1]

    def open(self, clip: int):
        if clip in self.slots:
            raise ValueError(f"clip {clip} is open already")
        if not self.free_slots:
            raise MemoryError("every slot is taken")
        self.slots[clip], self.lens[clip] = self.free_slots.pop(), 0

    def close(self, clip: int):
        """Give the clip's pages back; as for PageTable, to whoever comes next on this stream."""
        self.shorten({clip: self.lens[clip]})
        self.free_slots.append(self.slots.pop(clip))
        del self.lens[clip]

    def extend(self, rows: dict[int, int]) -> ec.KVStep:
        """Room for rows[clip] more tokens of each clip, all of them or none, and the step that
        they make, its rows in the dict's order."""
        if min(rows.values(), default=0) < 0:
            raise ValueError("a clip's rows cannot be negative")
        need = sum(self._pages(self.lens[c] + n) - self._pages(self.lens[c]) for c, n in rows.items())
        if need > self.n_free:
            raise MemoryError(f"{need} pages needed, {self.n_free} free")
        slots, n = self._numbers(rows)
        step = ec.KVStep.empty(self.tables, len(rows), sum(rows.values()), max(rows.values(), default=0))
        # the tables are as wide as the pool; the clips are no longer than this
        step.batch.max_len = max((self.lens[c] + n for c, n in rows.items()), default=0)
        ec.echo_kv_extend(self.tables, n, step, slots)
        self.n_free -= need
        for c, k in rows.items():
            self.lens[c] += k
        return step

    def shorten(self, rows: dict[int, int]):
        """Take back the last rows[clip] tokens of each clip, all where it has fewer, and the pages
        that only they needed."""
        if min(rows.values(), default=0) < 0:
            raise ValueError("a clip's rows cannot be negative")
        slots, n = self._numbers(rows)
        ec.echo_kv_shorten(self.tables, n, slots)
        for c, k in rows.items():
            k = min(k, self.lens[c])
            self.n_free += self._pages(self.lens[c]) - self._pages(self.lens[c] - k)
            self.lens[c] -= k


class ChunkStream:
    """Blocks run chunk by chunk over several clips at once, each clip's earlier keys and
    values in pages of one pool per layer.

    step({clip: x}) takes the new latent tokens of each clip (any number of frames, or a
    single token), appends their keys and values to the clip's pages, and returns the last
    layer's outputs.  Self-attention is causal frame by frame (frame_tokens = 1: token by
    token): a token sees all earlier frames and its own, as far as the clip's chunks have
    come: the tokens of a frame that comes in parts see the parts up to their own, and their
    outputs stand when the rest arrives.  The audio condition of a clip,
    of any length, is written into pages of its own when the clip is opened, and the
    cross-attention reads it from there.  The block is that of echo_block_step on these rows:
      h1 = x + MHA(LN(x)) Wo + bo,  h2 = h1 + MHA(LN(h1) Wqc; audio) Woc + boc,
      y = h2 + GELU(LN(h2) W1 + b1) W2 + b2.
    kind: ec.CACHE_BF16, ec.CACHE_INT8 or ec.CACHE_INT4 pages.

    device_tables: the page tables are kept on the GPU, for up to max_clips clips at a time.  With
    them, rotary turns each token's queries and keys by its number in the clip before the
    self-attention, and step() takes modulations: mods[clip], f32 or bf16 [layers, 6, D], the
    shift, scale and gate of the self-attention and of the FFN,
      h1 = x + gate_a * (MHA(LN(x) (1 + scale_a) + shift_a) Wo + bo),  h2 as above,
      y = h2 + gate_f * (GELU((LN(h2) (1 + scale_f) + shift_f) W1 + b1) W2 + b2)."""

    def __init__(self, blocks: list, H: int, d: int, frame_tokens: int, n_pages: int,
                 cond_pages: int, page_tokens: int = 64, kind: int = ec.CACHE_INT8, device="cuda",
                 device_tables: bool = False, max_clips: int = 64, rotary: ec.Rotary | None = None):
        if rotary is not None and (not device_tables or rotary.columns != 1 or rotary.d != d):
            raise ValueError("rotary needs device_tables, heads of this size and one position a token")
        self.blocks, self.H, self.d, self.frame_tokens = blocks, H, d, frame_tokens
        self.device = torch.device(device)
        pool = lambda n: [ec.KVPool.empty(kind, n, page_tokens, H, d, device) for _ in blocks]
        self.self_pools, self.cond_pools = pool(n_pages), pool(cond_pages)
        self.device_tables, self.rotary = device_tables, rotary
        table = lambda n: (DevicePageTable(n, page_tokens, max_clips, device) if device_tables   # noqa: E731
                           else PageTable(n, page_tokens))
        self.self_table, self.cond_table = table(n_pages), table(cond_pages)
        if device_tables:
            self.norm = ec.GatedNorm(H * d)

    def open(self, clip: int, cond_kv: list):
        """A new clip with its audio condition: per layer the keys and values bf16 [Lc, 2 D]
        of echo_precompute_cross_kv."""
        D = self.H * self.d
        if len(cond_kv) != len(self.blocks):
            raise ValueError(f"{len(cond_kv)} layers' keys and values for {len(self.blocks)} blocks")
        Lc = cond_kv[0].shape[0] if cond_kv else 0
        if any(tuple(kv.shape) != (Lc, 2 * D) for kv in cond_kv):
            raise ValueError(f"every layer's keys and values must be [{Lc}, {2 * D}]")
        self.cond_table.open(clip)
        try:
            if self.device_tables:
                place = self.cond_table.extend({clip: Lc}).place
                for pool, kv in zip(self.cond_pools, cond_kv):
                    ec.echo_kv_write_at(pool, place, kv[:, :D], kv[:, D:])
            else:
                self.cond_table.extend({clip: Lc})
                batch = self.cond_table.batch({clip: Lc}, self.device)
                for pool, kv in zip(self.cond_pools, cond_kv):
                    ec.echo_kv_write(pool, batch, kv[:, :D], kv[:, D:])
            self.self_table.open(clip)
        except BaseException:
            self.cond_table.close(clip)
            raise

    def close(self, clip: int):
        self.self_table.close(clip)
        self.cond_table.close(clip)

    def step(self, chunks: dict[int, torch.Tensor],
             mods: dict[int, torch.Tensor] | None = None) -> dict[int, torch.Tensor]:
        """chunks: bf16 [n, D] per clip; returns bf16 [n, D] per clip.  After an exception the
        clips are as they were before the call."""
        rows = {c: x.shape[0] for c, x in chunks.items()}
        if any(c not in self.self_table.lens for c in rows):
            raise ValueError("a clip is not open")
        D = self.H * self.d
        for x in chunks.values():
            if x.dim() != 2 or x.shape[1] != D or x.device.type != self.device.type:
                raise ValueError(f"a chunk must be [n, {D}] on {self.device.type}")
            if x.dtype not in (torch.bfloat16, torch.float32):
                raise TypeError(f"unsupported dtype {x.dtype}")
        if mods is not None:
            if not self.device_tables:
                raise ValueError("modulations need device_tables")
            shape = (len(self.blocks), 6, D)
            if set(mods) != set(rows) or any(tuple(m.shape) != shape for m in mods.values()):
                raise ValueError(f"modulations are one tensor {list(shape)} per clip of the step")
        if not sum(rows.values()):
            return {c: x.to(torch.bfloat16) for c, x in chunks.items()}
        x = torch.cat(list(chunks.values())) if len(chunks) > 1 else next(iter(chunks.values())).contiguous()
        if self.device_tables:
            step = self.self_table.extend(rows)
            try:
                x = self._layers(x, rows, step, None if mods is None else torch.stack([mods[c] for c in rows]))
            except BaseException:
                self.self_table.shorten(rows)
                raise
            return dict(zip(rows, x.split(list(rows.values()))))
        self.self_table.extend(rows)
        try:
            batch = self.self_table.batch(rows, self.device)
            cond = self.cond_table.batch(rows, self.device)   # the same rows, over the audio's pages
            for blk, pool, cond_pool in zip(self.blocks, self.self_pools, self.cond_pools):
                w = blk.tensors
                n1 = ec.echo_layernorm(x)
                kv = ec.echo_linear(n1, w["Wkv"], w["bkv"])
                ec.echo_kv_write(pool, batch, kv[:, :D], kv[:, D:])
                a = ec.echo_kv_attention(pool, batch, ec.echo_linear(n1, w["Wq"], w["bq"]),
                                         causal_block=self.frame_tokens)
                h1 = ec.echo_linear(a, w["Wo"], w["bo"], resid=x, out_dtype=torch.float32)
                q = ec.echo_linear(ec.echo_layernorm(h1), w["Wqc"], w["bqc"])
                a = ec.echo_kv_attention(cond_pool, cond, q)
                h2 = ec.echo_linear(a, w["Woc"], w["boc"], resid=h1, out_dtype=torch.float32)
                u = ec.echo_linear(ec.echo_layernorm(h2), w["W1"], w["b1"], act=1)
                x = ec.echo_linear(u, w["W2"], w["b2"], resid=h2)
        except BaseException:
            self.self_table.shorten(rows)
            raise
        return dict(zip(rows, x.split(list(rows.values()))))

    def _layers(self, x, rows, step: ec.KVStep, mods):
        """The blocks over a step's rows; mods [clips, layers, 6, D] or none."""
        D, last = self.H * self.d, len(self.blocks) - 1
        # the same rows over the audio's pages: no more tokens, and these rows' numbers
        audio = self.cond_table.extend({c: 0 for c in rows}).batch
        cond = ec.KVBatch(audio.table, audio.lens, step.batch.row0, step.n_rows, step.batch.max_rows, audio.max_len)

        def norm(x, y=None, out=torch.float32, gate=None, scale=None, shift=None, want_n=True):
            """(h, n) with (layer, row of its modulations) for gate, scale and shift; without y, n alone."""
            part = lambda i: None if mods is None or i is None else mods[:, i[0], i[1]]   # noqa: E731
            g, s, t = part(gate), part(scale), part(shift)
            h = None if y is None else torch.empty(x.shape, dtype=out, device=x.device)
            return ec.echo_gated_norm(self.norm, x, y, g, s, t, h=h, want_h=h is not None, want_n=want_n,
                                      mod_rows=None if g is None and s is None else step.seq)

        # a branch meets the residual in fp32: in the product's epilogue, or where it has a gate, in the norm
        n1 = norm(x, scale=(0, 1), shift=(0, 0))[1] if self.blocks else None
        for l, (blk, pool, cond_pool) in enumerate(zip(self.blocks, self.self_pools, self.cond_pools)):
            w, f32 = blk.tensors, torch.float32
            kv = ec.echo_linear(n1, w["Wkv"], w["bkv"])
            q, k = ec.echo_linear(n1, w["Wq"], w["bq"]), kv[:, :D]
            if self.rotary is not None:
                ec.echo_rotary(self.rotary, step.pos, q, k, q_out=q, k_out=k)
            ec.echo_kv_write_at(pool, step.place, k, kv[:, D:])
            a = ec.echo_kv_attention(pool, step.batch, q, causal_block=self.frame_tokens)
            if mods is None:
                h1 = ec.echo_linear(a, w["Wo"], w["bo"], resid=x, out_dtype=f32)
                nq = norm(h1)[1]
            else:
                h1, nq = norm(x, ec.echo_linear(a, w["Wo"], w["bo"], out_dtype=f32), gate=(l, 2))
            a = ec.echo_kv_attention(cond_pool, cond, ec.echo_linear(nq, w["Wqc"], w["bqc"]))
            h2 = ec.echo_linear(a, w["Woc"], w["boc"], resid=h1, out_dtype=f32)
            u = ec.echo_linear(norm(h2, scale=(l, 4), shift=(l, 3))[1], w["W1"], w["b1"], act=1)
            after = (l + 1, 1) if l < last else None           # of the next block's first norm
            if mods is None:
                x = ec.echo_linear(u, w["W2"], w["b2"], resid=h2)
                n1 = norm(x)[1] if l < last else None
            else:
                x, n1 = norm(h2, ec.echo_linear(u, w["W2"], w["b2"], out_dtype=f32), torch.bfloat16, gate=(l, 5),
                             scale=after, shift=None if after is None else (l + 1, 0), want_n=l < last)
        return x
