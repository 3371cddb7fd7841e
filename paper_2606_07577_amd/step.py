"""One compression step on the GPU through the C ABI.

`DeviceStep` uploads a workload (a list of layer dicts as produced by
`synth.make_workload`) to device buffers laid out as the library expects,
owns the output buffers and runs the four stages on a stream.
"""
from __future__ import annotations

import contextlib

import numpy as np
import torch

from . import omnimem as om


class DeviceStep:
    def __init__(self, layers, total_budget, device="cuda", max_tokens=None, max_chunk=None, **options):
        self.device = torch.device(device)
        self.n_layers = len(layers)
        first = layers[0]
        self.dtype_name = first["dtype"]
        self.tdtype = torch.bfloat16 if self.dtype_name == "bf16" else torch.float32
        h_q, _, d = first["q"].shape
        h_kv = first["k"].shape[0]
        self.h_q, self.h_kv, self.d = h_q, h_kv, d
        self.n = [int(l["k"].shape[1]) for l in layers]
        self.n_cache = [int(l["n_cache"]) for l in layers]
        self.max_tokens = max_tokens or max(self.n)
        self.max_chunk = max_chunk or max(n - c for n, c in zip(self.n, self.n_cache))
        self.total_budget = int(total_budget)
        self.ctx = om.Context(self.n_layers, h_q, h_kv, d, self.max_tokens, self.max_chunk,
                              dtype=om.BF16 if self.dtype_name == "bf16" else om.F32, **options)
        dev, td = self.device, self.tdtype
        self.q = [torch.from_numpy(np.ascontiguousarray(l["q"])).to(dev, td) for l in layers]
        self.k = [torch.from_numpy(np.ascontiguousarray(l["k"])).to(dev, td) for l in layers]
        self.v = [torch.from_numpy(np.ascontiguousarray(l["v"])).to(dev, td) for l in layers]
        self.mod = [torch.from_numpy(np.ascontiguousarray(l["modality"])).to(dev) for l in layers]
        self.k_out = [torch.zeros_like(k) for k in self.k]
        self.v_out = [torch.zeros_like(v) for v in self.v]
        # hidden states (redundancy source of Eq. 7 as printed), when the layers carry them
        self.h = [torch.from_numpy(np.ascontiguousarray(l["h"])).to(dev, self.tdtype) if "h" in l else None
                  for l in layers]
        self.h_out = [torch.zeros_like(h) if h is not None else None for h in self.h]
        self.sm_scale = [float(l["sm_scale"]) for l in layers]
        shape = (self.n_layers, h_kv, self.max_tokens)
        self.a = torch.zeros(shape, device=dev, dtype=torch.float32)
        self.s = torch.zeros(shape, device=dev, dtype=torch.float32)
        self.idx = torch.full(shape, -1, device=dev, dtype=torch.int32)
        self.lse = torch.zeros((self.n_layers, h_q, self.max_chunk), device=dev, dtype=torch.float32)
        self.budgets = torch.zeros((self.n_layers, 2), device=dev, dtype=torch.int32)
        self.stats = torch.zeros((self.n_layers, 10), device=dev, dtype=torch.float32)
        self.layer_budgets = torch.zeros(self.n_layers, device=dev, dtype=torch.int32)
        self.fixed_budgets = False          # run() splits self.layer_budgets instead of Eq. (14)
        self.lse_in = [None] * self.n_layers
        self.attn = None                    # made by attend()
        self.descs = self._descs()
        torch.cuda.current_stream(self.device).synchronize()   # (stages may come on streams that do not wait for this one)

    def _descs(self):
        return [om.make_layer(self.q[l], self.k[l], self.v[l], self.mod[l], self.n_cache[l],
                              self.sm_scale[l], self.lse_in[l], self.k_out[l], self.v_out[l],
                              self.h[l], self.h_out[l])
                for l in range(self.n_layers)]

    def set_lse_inputs(self, lse_list):
        """Give each layer a caller-side log-sum-exp ([H_q, C] fp32 device tensors)."""
        self.lse_in = list(lse_list)
        self.descs = self._descs()

    # stages ---------------------------------------------------------------
    def score(self, stream=None, lse_out=True):
        self.ctx.omnimem_score(self.descs, self.a, self.lse if lse_out else None, stream)

    def redundancy(self, stream=None):
        self.ctx.omnimem_redundancy(self.descs, self.s, stream)

    def allocate(self, stream=None, a=None, s=None):
        self.ctx.omnimem_allocate(self.descs, self.a if a is None else a, self.s if s is None else s,
                                  self.total_budget, self.budgets, self.stats, stream)

    def select_compact(self, stream=None, a=None, s=None, budgets=None):
        self.ctx.omnimem_select_compact(self.descs, self.a if a is None else a, self.s if s is None else s,
                                        self.budgets if budgets is None else budgets, self.idx, stream)

    def attend(self, stream=None):
        """The chunk's attention over the working sets (Eq. 1), all layers in
        one call: self.attn_out[l] [H_q, C, d] (query-major in memory, as the
        output projection takes it), and its log-sum-exp, which the score
        stage then takes instead of computing it."""
        if self.attn is None:
            self.attn = om.Attention(self.h_q, self.h_kv, self.d, om.BF16 if self.dtype_name == "bf16" else om.F32)
            chunk = [n - c for n, c in zip(self.n, self.n_cache)]
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
                self.attn_out = [torch.zeros((c, self.h_q, self.d), device=self.device, dtype=self.tdtype).transpose(0, 1)
                                 for c in chunk]
                self._attn_lse = [torch.zeros((self.h_q, c), device=self.device, dtype=torch.float32) for c in chunk]
            self._queries = om.array_of([om.make_query(self.q[l], self.attn_out[l], self.k[l], self.v[l],
                                                       sm_scale=self.sm_scale[l], lse=self._attn_lse[l])
                                         for l in range(self.n_layers)])
        if any(a is not b for a, b in zip(self.lse_in, self._attn_lse)):
            self.set_lse_inputs(self._attn_lse)
        self.attn.omnimem_attend(self._queries, self.ctx.cfg.causal, stream)

    # offline budgets (calibration) ----------------------------------------
    def calibrate(self, stream=None, a=None, s=None):
        self.ctx.omnimem_calibrate(self.descs, self.a if a is None else a, self.s if s is None else s,
                                   self.stats, stream)

    def calibration_budgets(self, stream=None):
        """The calibration's layer budgets into self.layer_budgets."""
        self.ctx.omnimem_calibration_budgets(self.total_budget, self.layer_budgets, stream)

    def allocate_fixed(self, stream=None, a=None, s=None, layer_budgets=None):
        self.ctx.omnimem_allocate_fixed(self.descs, self.a if a is None else a, self.s if s is None else s,
                                        self.layer_budgets if layer_budgets is None else layer_budgets,
                                        self.budgets, self.stats, stream)

    def run(self, stream=None):
        self.score(stream, lse_out=False)
        self.redundancy(stream)
        if self.fixed_budgets:
            self.allocate_fixed(stream)
        else:
            self.allocate(stream)
        self.select_compact(stream)

    # host views -----------------------------------------------------------
    def to_device_f32(self, per_layer):
        """[L] list of [H_kv, N_l] host arrays -> a [L, H_kv, max_tokens] device tensor."""
        out = torch.zeros((self.n_layers, self.h_kv, self.max_tokens), dtype=torch.float32)
        for l, arr in enumerate(per_layer):
            out[l, :, : arr.shape[1]] = torch.from_numpy(np.asarray(arr, dtype=np.float32))
        return out.to(self.device)

    def host(self, name, l):
        t = getattr(self, name)
        if name in ("a", "s", "idx"):
            return t[l, :, : self.n[l]].cpu().numpy()
        if name == "lse":
            return t[l, :, : self.n[l] - self.n_cache[l]].cpu().numpy()
        return t[l].cpu().numpy()

    def close(self):
        if self.attn is not None:
            self.attn.close()
        self.ctx.close()


class StreamRunner:
    """The compression step after every chunk of a stream, on the GPU.

    Each layer's cache is one buffer [H_kv, cap, d] for K, one for V and a
    modality buffer [cap].  A step's working set is the buffer's first
    N = n_cache + C rows: omnimem_append writes the chunk's K/V and modality
    behind the kept rows (Eq. 3), the four stages run, and
    omnimem_select_compact moves the kept rows to the front of the same
    buffers and rewrites their modality (in place, Eqs. 2-5).  With
    in_place=False two buffers per layer alternate instead (out of place).

    The host needs each layer's kept-row count to describe the next working
    set: it copies the budgets back after the allocation stage and waits for
    that copy only, so the compaction of one step overlaps the host's
    preparation of the next.  The descriptors are ctypes arrays built once;
    a step only updates the fields that change.  Calls may come on different
    streams: each waits for the work on the caches that came before it.

    In place, kept audio rows that land behind their own row are staged in
    the context's reserve of `stage_rows` rows per (layer, KV head); there
    are never more of them than the layer's audio budget.  When a step's
    audio budget exceeds the reserve, the runner asks the library whether
    that step's compaction ran and, if it moved nothing for lack of staging
    rows, compacts out of place into temporary buffers and copies back.
    """

    def __init__(self, n_layers, h_q, h_kv, d, chunk_len, total_budget, dtype="bf16", device="cuda",
                 in_place=True, stage_rows=None, keep_working_set=False, timing=False, **options):
        self.device = torch.device(device)
        self.L, self.h_q, self.h_kv, self.d, self.C = n_layers, h_q, h_kv, d, chunk_len
        self.total_budget = int(total_budget)
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        cfg_probe = om.Context.default_config()
        bmax = options.get("b_max_frac", cfg_probe.b_max_frac)
        self.cache_cap = int(bmax * total_budget / n_layers)   # no layer keeps more
        self.cap = self.cache_cap + chunk_len
        self.in_place = bool(in_place)
        self.stage_rows = int(stage_rows if stage_rows is not None else self.cache_cap // 2) if in_place else 0
        self.ctx = om.Context(n_layers, h_q, h_kv, d, self.cap, chunk_len,
                              dtype=om.BF16 if dtype == "bf16" else om.F32,
                              inplace_stage_rows=self.stage_rows, **options)
        dev, td = self.device, self.tdtype
        n_sets = 1 if self.in_place else 2
        self.kbuf = [[torch.zeros((h_kv, self.cap, d), device=dev, dtype=td) for _ in range(n_layers)]
                     for _ in range(n_sets)]
        self.vbuf = [[torch.zeros((h_kv, self.cap, d), device=dev, dtype=td) for _ in range(n_layers)]
                     for _ in range(n_sets)]
        self.mbuf = [[torch.zeros(self.cap, device=dev, dtype=torch.uint8) for _ in range(n_layers)]
                     for _ in range(n_sets)]
        shape = (n_layers, h_kv, self.cap)
        self.a = torch.zeros(shape, device=dev, dtype=torch.float32)
        self.s = torch.zeros(shape, device=dev, dtype=torch.float32)
        self.idx = torch.full(shape, -1, device=dev, dtype=torch.int32)
        self.budgets = torch.zeros((n_layers, 2), device=dev, dtype=torch.int32)
        self.budgets_host = torch.zeros((n_layers, 2), dtype=torch.int32, pin_memory=True)
        self.stats = torch.zeros((n_layers, 10), device=dev, dtype=torch.float32)
        self.layer_budgets = torch.zeros(n_layers, device=dev, dtype=torch.int32)
        self.calibrating = False   # each step also adds its C^(l) to the calibration
        self.fixed = False         # steps split self.layer_budgets instead of Eq. (14)
        self.cur = 0               # buffer set holding the cache (out of place: alternates)
        self.n_cache = [0] * n_layers
        self.steps = 0
        self.tokens = 0            # sum over steps and layers of the working-set size
        self.fallbacks = 0         # steps compacted out of place for lack of staging rows
        self.keep_working_set = keep_working_set
        self.working_set = None    # [L] of (k, v, modality) copies of the last step's working set
        self.attn = None           # made by hold() or restore()
        self._layers = (om.Layer * n_layers)()
        self._chunks = (om.Chunk * n_layers)()
        self._budget_ready = torch.cuda.Event()
        self._pending, self._pending_stream = False, None   # a pushed step whose budgets are unread
        self._last = torch.cuda.current_stream(dev)   # the stream of the last work on the caches
        self.timing = timing       # per step: events before the append, before score, after select_compact
        self.events = []

    # order on the device ---------------------------------------------------
    def _behind(self, stream):
        """The stream (default: the current one) for work on the caches, made
        to wait for what came before on another one: steps, hold() and
        restore(), and what the current stream did with the caches' views.  A
        stream that is captured may not wait for work outside its graph."""
        stream = stream if stream is not None else torch.cuda.current_stream()
        if self._last != stream:
            with torch.cuda.stream(stream):
                if torch.cuda.is_current_stream_capturing():
                    return stream
            stream.wait_stream(self._last)
            self._last = stream
        return stream

    def _settle(self):
        """The caches' sizes are known, their rows ordered for the current stream."""
        self.finish()
        self._behind(None)

    # buffers ------------------------------------------------------------
    def cache_k(self, l):
        """Device view of layer l's kept keys [H_kv, n_cache, d], for the
        current stream."""
        self._settle()
        return self.kbuf[self.cur][l][:, : self.n_cache[l]]

    def cache_v(self, l):
        self._settle()
        return self.vbuf[self.cur][l][:, : self.n_cache[l]]

    def cache_modality(self, l):
        self._settle()
        return self.mbuf[self.cur][l][: self.n_cache[l]]

    def set_cache(self, l, k, v, m_v, m_a):
        """Replace layer l's retained cache: k, v [H_kv, m_v + m_a, d] (host or
        device), visual rows first."""
        self._settle()
        m = int(m_v) + int(m_a)
        if m > self.cache_cap:
            raise ValueError(f"cache of {m} rows exceeds the capacity {self.cache_cap}")
        kb, vb, mb = self.kbuf[self.cur][l], self.vbuf[self.cur][l], self.mbuf[self.cur][l]
        kb[:, :m] = torch.as_tensor(k).to(self.device, self.tdtype)
        vb[:, :m] = torch.as_tensor(v).to(self.device, self.tdtype)
        mb[:m_v] = 0
        mb[m_v:m] = 1
        self.n_cache[l] = m

    # memories ------------------------------------------------------------
    def hold(self, stream=None):
        """The kept rows of every layer in 4 bits (a HeldMemory): what answers
        are read from (see Reader), a quarter of the cache's bytes to keep
        until the stream goes on (see restore)."""
        budgets = self.finish()
        with torch.cuda.stream(self._attention_stream(stream)):
            if budgets is None:
                budgets = self._held_budgets()
            data = [torch.empty(om.memory_shape(self.h_kv, self.d, n), dtype=torch.uint8, device=self.device)
                    for n in self.n_cache]
            self.attn.omnimem_pack(self._held(data, self.n_cache))
            ready = torch.cuda.Event()
            ready.record()
        return HeldMemory(data, list(self.n_cache), [int(b) for b in budgets[:, 0]], ready)

    def restore(self, held, stream=None):
        """Take a held memory's rows, as they are held, for the retained caches."""
        self.finish()
        if len(held.rows) != self.L or max(held.rows) > self.cache_cap:
            raise ValueError("the memory has another number of layers, or more rows than the caches hold")
        rows = self._held(held.data, held.rows)                # (refuses tensors that do not fit)
        stream = self._attention_stream(stream)
        with torch.cuda.stream(stream):
            if not torch.cuda.is_current_stream_capturing():   # (see _behind)
                if held.ready is not None:
                    stream.wait_event(held.ready)
                for data in held.data:
                    data.record_stream(stream)                 # (the memory may be dropped before the stream is here)
            self.attn.omnimem_unpack(rows)
            for mod, n, visual in zip(self.mbuf[self.cur], held.rows, held.visual):
                mod[:visual] = 0
                mod[visual:n] = 1
        self.n_cache = list(held.rows)

    def _attention_stream(self, stream):
        """The stream for hold() and restore(), with their handle made."""
        if self.attn is None:
            self.attn = om.Attention(self.h_q, self.h_kv, self.d, om.BF16 if self.tdtype == torch.bfloat16 else om.F32)
        return self._behind(stream)

    def _held(self, data, rows):
        return [om.make_held(self.kbuf[self.cur][l][:, :n], self.vbuf[self.cur][l][:, :n], data[l]) for l, n in enumerate(rows)]

    def _held_budgets(self):
        """Kept visual and audio rows of the caches as they are."""
        audio = [int(m[:n].sum()) for m, n in zip(self.mbuf[self.cur], self.n_cache)]
        return np.array([[n - a, a] for n, a in zip(self.n_cache, audio)], dtype=np.int32)

    # one step ----------------------------------------------------------
    def _describe(self, chunk, qs, cur):
        """Fill the persistent descriptor arrays for a step's working sets in
        buffer set `cur`, all but the kept-row counts (_set_cache_rows)."""
        other = cur if self.in_place else 1 - cur
        for l, ch in enumerate(chunk):
            kb, vb, mb = self.kbuf[cur][l], self.vbuf[cur][l], self.mbuf[cur][l]
            ko, vo, mo = self.kbuf[other][l], self.vbuf[other][l], self.mbuf[other][l]
            lay = self._layers[l]
            q = qs[l]
            lay.q, lay.q_head_stride, lay.q_row_stride = q.data_ptr(), q.stride(0), q.stride(1)
            lay.k, lay.v = kb.data_ptr(), vb.data_ptr()
            lay.kv_head_stride, lay.kv_row_stride = kb.stride(0), kb.stride(1)
            lay.modality = mb.data_ptr()
            lay.n_chunk = self.C
            lay.sm_scale = float(ch["sm_scale"])
            lay.k_out, lay.v_out = ko.data_ptr(), vo.data_ptr()
            lay.out_head_stride, lay.out_row_stride = ko.stride(0), ko.stride(1)
            lay.out_rows = self.cap
            lay.modality_out = mo.data_ptr()
            c = self._chunks[l]
            ck, cv, cm = ch["k"], ch["v"], ch["modality"]
            c.k, c.v, c.modality = ck.data_ptr(), cv.data_ptr(), cm.data_ptr()
            c.head_stride, c.row_stride, c.n_rows = ck.stride(0), ck.stride(1), ck.shape[1]

    def _set_cache_rows(self):
        for l in range(self.L):
            self._layers[l].n_cache = self.n_cache[l]

    def _on_device(self, chunk):
        dev, td = self.device, self.tdtype
        out = []
        for ch in chunk:
            x = dict(ch)
            for key in ("q", "k", "v"):
                t = torch.as_tensor(ch[key]).to(dev, td)
                x[key] = t if t.is_contiguous() else t.contiguous()
            x["modality"] = torch.as_tensor(ch["modality"]).to(dev, torch.uint8)
            out.append(x)
        return out

    def push(self, chunk, stream=None, wait=True):
        """Append one chunk (list of per-layer dicts from synth.StreamSource:
        q [H_q, C, d], k, v [H_kv, C, d], modality [C], sm_scale) and run the
        step.  With wait, returns the budgets [L, 2] as a host array (the
        compaction may still be running on the stream).  Without, returns
        None at once: the step's budgets are read by the next push (after it
        has described its chunk, so the host's work overlaps the GPU's) or
        by finish()."""
        stream = self._behind(stream)
        with torch.cuda.stream(stream):
            chunk = self._on_device(chunk)
        cur = self.cur if self.in_place or not self._pending else 1 - self.cur
        self._describe(chunk, [ch["q"] for ch in chunk], cur)
        self.finish()              # the previous step's budgets give this step's kept rows
        self._chunk_refs = chunk   # keep the inputs alive while the stream uses them
        self._set_cache_rows()
        ctx, lays = self.ctx, self._layers
        ev = None
        if self.timing:
            ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
            ev[0].record(stream)
        ctx.omnimem_append(lays, self._chunks, stream)
        if self.keep_working_set:
            with torch.cuda.stream(stream):
                self.working_set = [(self.kbuf[self.cur][l][:, : self.n_cache[l] + self.C].clone(),
                                     self.vbuf[self.cur][l][:, : self.n_cache[l] + self.C].clone(),
                                     self.mbuf[self.cur][l][: self.n_cache[l] + self.C].clone())
                                    for l in range(self.L)]
        if ev:
            ev[1].record(stream)
        ctx.omnimem_score(lays, self.a, None, stream)
        ctx.omnimem_redundancy(lays, self.s, stream)
        if self.calibrating:
            ctx.omnimem_calibrate(lays, self.a, self.s, None, stream)
        if self.fixed:
            ctx.omnimem_allocate_fixed(lays, self.a, self.s, self.layer_budgets, self.budgets, self.stats, stream)
        else:
            ctx.omnimem_allocate(lays, self.a, self.s, self.total_budget, self.budgets, self.stats, stream)
        with torch.cuda.stream(stream):
            self.budgets_host.copy_(self.budgets, non_blocking=True)
            self._budget_ready.record(stream)
        ctx.omnimem_select_compact(lays, self.a, self.s, self.budgets, self.idx, stream)
        if ev:
            ev[2].record(stream)
            self.events.append(ev)
        for l in range(self.L):
            self.tokens += self.n_cache[l] + self.C
        self._pending, self._pending_stream = True, stream
        return self.finish() if wait else None

    def finish(self):
        """Wait for the last pushed step's budgets and take its kept-row
        counts as the caches' sizes; returns the budgets [L, 2] (None when no
        step is pending)."""
        if not self._pending:
            return None
        self._pending = False
        self._budget_ready.synchronize()
        budgets = self.budgets_host.numpy().copy()
        if self.in_place and int(budgets[:, 1].max()) > self.stage_rows:
            self._check_staging(self._pending_stream)
        for l in range(self.L):
            self.n_cache[l] = int(budgets[l, 0]) + int(budgets[l, 1])
        if not self.in_place:
            self.cur = 1 - self.cur
        self.steps += 1
        return budgets

    def _check_staging(self, stream):
        """A step whose audio budget exceeds the staging reserve: if its
        in-place compaction moved nothing, compact out of place into
        temporaries and copy the kept rows back."""
        stream.synchronize()
        try:
            self.ctx.omnimem_inplace_status()
            return
        except om.OmnimemError as e:
            if e.status != om.ERR_CAPACITY:
                raise
        self.fallbacks += 1
        tmp = []
        lays = (om.Layer * self.L)()
        for l in range(self.L):
            lay = om.Layer.from_buffer_copy(self._layers[l])
            ko = torch.empty_like(self.kbuf[self.cur][l])
            vo = torch.empty_like(self.vbuf[self.cur][l])
            lay.k_out, lay.v_out = ko.data_ptr(), vo.data_ptr()
            tmp.append((ko, vo))
            lays[l] = lay
        self.ctx.omnimem_select_compact(lays, self.a, self.s, self.budgets, self.idx, stream)
        with torch.cuda.stream(stream):
            for l, (ko, vo) in enumerate(tmp):
                self.kbuf[self.cur][l].copy_(ko)
                self.vbuf[self.cur][l].copy_(vo)
        stream.synchronize()

    def timings(self):
        """Summed milliseconds over the timed steps: (appends, four stages)."""
        torch.cuda.synchronize()
        app = sum(e[0].elapsed_time(e[1]) for e in self.events)
        abi = sum(e[1].elapsed_time(e[2]) for e in self.events)
        return app, abi

    def freeze_budgets(self, stream=None):
        """Layer budgets from the steps calibrated so far; later steps split them."""
        self.finish()
        self.ctx.omnimem_calibration_budgets(self.total_budget, self.layer_budgets, self._behind(stream))
        self.calibrating = False
        self.fixed = True

    def close(self):
        self.finish()
        if self.attn is not None:
            self.attn.close()
        self.ctx.close()


class HeldMemory:
    """A stream's kept rows in 4 bits: data[l] uint8 [H_kv, blocks, 34 d],
    rows[l] kept rows, visual[l] of them visual (in front).  ready: the event
    behind what writes the data, or None if nothing has to be waited for;
    restore() and Reader wait for it."""

    ready = None                                   # (of memories saved without one)

    def __init__(self, data, rows, visual, ready=None):
        self.data, self.rows, self.visual, self.ready = data, rows, visual, ready

    def __getstate__(self):                        # copies, and what is saved, hold what is written
        if self.ready is not None:
            self.ready.synchronize()
        return dict(self.__dict__, ready=None)


class Reader:
    """Answers from the memories of several streams at once: every layer's
    tokens so far lie in a tail of their own behind each stream's memory.

    A model calls layer() for each of its layers with the projections of the
    streams' next tokens (a prompt's, or one each), in order, and next() after
    the last layer.  `capacity`: tail rows of a stream.  Calls on different HIP
    streams are the caller's to order (they share the tails and a handle); what
    the constructor fills, and the memories, are there before it returns.

    The calls' descriptors are made once; layer() sets what changes.  Where
    every stream has the same number of tokens it takes the streams' tensors
    stacked, at a host cost that does not grow with them (lists: some
    microseconds for each stream).
    """

    def __init__(self, memories, h_q, h_kv, d, rope, capacity, dtype="bf16", device="cuda", sm_scale=0.0):
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.h_q, self.h_kv, self.d, self.cap = h_q, h_kv, d, int(capacity)
        self.memories, self.rope, self.sm_scale = list(memories), rope, float(sm_scale)
        if not self.memories or len({len(m.data) for m in self.memories}) != 1:
            raise ValueError("one memory at least, all of one number of layers")
        n_layers, streams, elt = len(self.memories[0].data), len(self.memories), self.tdtype.itemsize
        self.attn = om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)
        shape = (n_layers, streams, h_kv, self.cap, d)
        self.k, self.v = (torch.zeros(shape, device=device, dtype=self.tdtype) for _ in range(2))
        self.device = self.k.device
        # (calls come on streams that do not wait for this one, and into captures, which may not wait for it)
        torch.cuda.current_stream(self.device).synchronize()
        for m in self.memories:
            if m.ready is not None:
                m.ready.synchronize()
        self.tail = [0] * streams                # tail rows of each stream
        self._new = None                         # and those that the current tokens add
        layouts = {om._Layout(h_q, h_kv, d, self.tdtype, self.device.index, rope.n_axes)}
        self._rows = (om.Projection * streams)()
        self._rows._layouts = layouts
        row = self._row = om.columns_of(self._rows)
        row["q_out_head_stride"], row["q_out_row_stride"] = d, h_q * d
        row["out_head_stride"], row["out_row_stride"] = self.k.stride(2), d
        self._queries, self._query = [], []
        at = np.arange(n_layers * streams, dtype=np.uint64).reshape(n_layers, streams) * np.uint64(h_kv * self.cap * d * elt)
        self._k_at, self._v_at = at + np.uint64(self.k.data_ptr()), at + np.uint64(self.v.data_ptr())
        for l in range(n_layers):
            queries = (om.Query * streams)()
            queries._layouts = layouts
            x = om.columns_of(queries)
            x["q_head_stride"] = x["out_head_stride"] = d
            x["q_row_stride"] = x["out_row_stride"] = h_q * d
            x["k"], x["v"] = self._k_at[l], self._v_at[l]
            x["kv_head_stride"], x["kv_row_stride"], x["sm_scale"] = self.k.stride(2), d, self.sm_scale
            for b, m in enumerate(self.memories):
                if m.rows[l]:
                    om._memory(m.data[l], m.rows[l], self.k[l, b])
                    if m.data[l].device != self.device:
                        raise ValueError("the memories must lie on the reader's device")
                    queries[b].memory, queries[b].memory_head_stride = m.data[l].data_ptr(), m.data[l].stride(0)
                    queries[b].memory_rows = m.rows[l]
            self._queries.append(queries)
            self._query.append(x)

    def _columns(self, what, x, heads, last):
        """Pointers, strides and sizes of the streams' tensors x [heads, n, last] (pos: [axes, n], `last` None): a list
        of them, or the tensors stacked."""
        stacked = isinstance(x, torch.Tensor)
        dims, dtype = (2, torch.int32) if last is None else (3, self.tdtype)
        if len(x) != len(self.memories):
            raise ValueError(f"q, k, v and pos are lists of {len(self.memories)} streams' tensors, or those stacked")
        for t in (x,) if stacked else x:
            lead = t.dim() - dims
            if (lead != int(stacked) or t.dtype != dtype or t.device != self.device or (t.stride(-1) != 1 and t.shape[-1] > 1) or
                    (t.shape[lead] < heads if last is None else (t.shape[lead], t.shape[-1]) != (heads, last))):
                raise ValueError(f"{what}: tensors of the reader's device, heads, width and type (positions int32) with "
                                 "their last axis contiguous")
        if stacked:
            count = len(x)
            ptr = np.uint64(x.data_ptr()) + np.arange(count, dtype=np.uint64) * np.uint64(x.stride(0) * x.element_size())
            return ptr, x.stride(1), x.stride(2), [x.shape[2]] * count
        return ([t.data_ptr() for t in x], [t.stride(0) for t in x], [t.stride(1) for t in x], [t.shape[1] for t in x])

    def layer(self, l, q, k, v, pos, stream=None):
        """One layer of the streams' next tokens: for each stream b q[b] [H_q,
        n_b, d], k[b] and v[b] [H_kv, n_b, d] as projected, and their positions
        pos[b] int32 [axes, n_b].  Keys and queries are normalised and rotated,
        keys and values go behind the stream's tail, and the queries attend to
        its memory and tail.  Returns [H_q, n_b, d] for each stream.  Each of
        the four is a list, or the streams' tensors stacked; with q stacked the
        result is [streams, H_q, n, d]."""
        qp, qh, qr, new = self._columns("q", q, self.h_q, self.d)
        kp, kh, kr, nk = self._columns("k", k, self.h_kv, self.d)
        vp, vh, vr, nv = self._columns("v", v, self.h_kv, self.d)
        pp, ps, _, np_ = self._columns("pos", pos, self.rope.n_axes, None)
        if not new == nk == nv == np_:
            raise ValueError("q, k, v and pos have different numbers of tokens")
        if np.any(np.not_equal(kh, vh)) or np.any(np.not_equal(kr, vr)):
            raise ValueError("k and v must share their strides")
        if self._new is not None and new != self._new:
            raise ValueError("every layer takes the same numbers of tokens (next() begins the next ones)")
        if any(t + n > self.cap for t, n in zip(self.tail, new)):
            raise ValueError(f"more than {self.cap} tail rows")
        total, elt = sum(new), self.tdtype.itemsize
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            rotated, out = (torch.empty((total, self.h_q, self.d), device=self.device, dtype=self.tdtype) for _ in range(2))
        first = np.cumsum([0] + new)
        at = first[:-1].astype(np.uint64) * np.uint64(self.h_q * self.d * elt)
        tail = np.array(self.tail, dtype=np.uint64) * np.uint64(self.d * elt)
        row, query = self._row, self._query[l]
        row["q"], row["q_head_stride"], row["q_row_stride"] = qp, qh, qr
        row["k"], row["v"], row["kv_head_stride"], row["kv_row_stride"] = kp, vp, kh, kr
        row["pos"], row["pos_stride"], row["n_rows"] = pp, ps, new
        row["q_out"] = query["q"] = at + np.uint64(rotated.data_ptr())
        row["k_out"], row["v_out"] = self._k_at[l] + tail, self._v_at[l] + tail
        query["out"], query["n_queries"] = at + np.uint64(out.data_ptr()), new
        query["n_tail"] = np.add(self.tail, new)
        self.attn.omnimem_rotate(self.rope, self._rows, stream)
        self.attn.omnimem_attend(self._queries[l], True, stream)
        self._new = new                          # (a call that was refused has added nothing)
        if isinstance(q, torch.Tensor):
            return out.view(len(new), -1, self.h_q, self.d).transpose(1, 2) if total else out.new_empty((len(new), self.h_q, 0, self.d))
        return [out[i: j].transpose(0, 1) for i, j in zip(first[:-1], first[1:])]

    def next(self):
        """The tokens of the last layer() calls are part of the tails."""
        if self._new is not None:
            self.tail = [t + n for t, n in zip(self.tail, self._new)]
        self._new = None

    def close(self):
        self.attn.close()
