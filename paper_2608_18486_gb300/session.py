"""Device-memory owner around the C ABI, for Python callers.

PyTorch provides device memory and streams only: a DecodeSession allocates
the cache buffer, the two workspaces and the status word once, and forwards
each call to libwm through the ctypes binding.  Nothing here computes any
part of the decode path.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib as W

_I32, _F32 = torch.int32, torch.float32
_LARGE = 1 << 25  # bytes of scratch beyond which no more is held than calls ask for


def torch_dtype(dtype: str):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


class Q4Cache:
    def __init__(self, cfg: W.wm_config, num_pages: int, device: str | torch.device = "cuda:0",
                 cache_buf: torch.Tensor | None = None):
        """The device memory of a cache held in 4 bits (wm_q4_cache), for the
        q4_* calls of sessions of the same config.  cache_buf: a contiguous
        uint8 tensor that holds it; allocated if None."""
        rc = W.wm_config_check(cfg)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_config_check")
        self.cfg, self.num_pages = cfg, int(num_pages)
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        # (the binding would keep the low 32 bits)
        nbytes = W.wm_q4_cache_bytes(cfg, num_pages) if 0 < self.num_pages < 1 << 31 else 0
        if nbytes == 0:
            raise W.WMError(W.WM_ERR_INVALID_ARG, "wm_q4_cache_bytes")
        if cache_buf is None:
            cache_buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        elif cache_buf.dtype != torch.uint8 or not cache_buf.is_contiguous() or \
                cache_buf.device != self.device:
            raise ValueError("cache_buf must be a contiguous uint8 tensor on the cache's device")
        self.cache_buf = cache_buf
        self.cache = W.wm_q4_cache_alloc(cfg, cache_buf, cache_buf.numel(), num_pages)
        self._index = -1 if self.device.type == "cpu" else self.device.index
        self._ref = ctypes.byref(self.cache)


class DecodeSession:
    def __init__(self, cfg: W.wm_config, B: int, num_pages: int, max_pages: int,
                 device: str | torch.device = "cuda:0", cache_buf: torch.Tensor | None = None):
        """cache_buf: a contiguous uint8 tensor that holds the cache (K pool,
        then V pool, as wm_cache_alloc lays them out); allocated if None."""
        rc = W.wm_config_check(cfg)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_config_check")
        self.cfg = cfg
        self.B, self.num_pages, self.max_pages = int(B), int(num_pages), int(max_pages)
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            # one device for the session's buffers, streams and checks
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = torch.float32 if cfg.dtype == W.WM_DT_F32 else torch.bfloat16
        nbytes = W.wm_cache_bytes(cfg, num_pages)
        if nbytes == 0:
            raise W.WMError(W.WM_ERR_INVALID_ARG, "wm_cache_bytes")
        if cache_buf is None:
            cache_buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        elif cache_buf.dtype != torch.uint8 or not cache_buf.is_contiguous() or \
                cache_buf.device != self.device:
            raise ValueError("cache_buf must be a contiguous uint8 tensor on the session's device")
        elif cache_buf.numel() < nbytes:
            raise W.WMError(W.WM_ERR_INVALID_ARG, "wm_cache_alloc")
        self.cache_buf = cache_buf
        self.cache = W.wm_cache_alloc(cfg, self.cache_buf, nbytes, num_pages)
        shape = (cfg.k, num_pages, cfg.Hkv, cfg.page_size, cfg.d)
        esz = 4 if cfg.dtype == W.WM_DT_F32 else 2
        n = cfg.k * num_pages * cfg.Hkv * cfg.page_size * cfg.d
        koff = self.cache.k_pool - self.cache_buf.data_ptr()
        voff = self.cache.v_pool - self.cache_buf.data_ptr()
        self.k_pool = self.cache_buf[koff:koff + n * esz].view(self.dtype).view(shape)
        self.v_pool = self.cache_buf[voff:voff + n * esz].view(self.dtype).view(shape)
        self.mix_ws_bytes = W.wm_kv_mix_workspace(cfg, B)
        self.attn_ws_bytes = W.wm_decode_attn_workspace(cfg, B, max_pages)
        self.mix_ws = torch.empty(self.mix_ws_bytes, dtype=torch.uint8, device=self.device)
        # the attention workspace holds arrival tickets that must start at zero
        self.attn_ws = torch.zeros(self.attn_ws_bytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._weights = None
        self._weight_refs = None
        self._scratch = {}   # per stream
        self._large_scratch = {}  # per stream, for calls that need more than _LARGE bytes
        self._in_graphs = set()   # streams whose large scratch a graph was captured with
        self._outgrown = []  # scratch replaced by larger: graphs captured before may use it
        self._need = {}      # workspace bytes by call and shape
        self._lib = W.lib()
        # the session's own arguments of the long-context calls, made once: a small
        # launch takes about as long on the GPU as its call on the host
        self._refs = (ctypes.byref(self.cfg), ctypes.byref(self.cache))
        self._status_ptr = self.status.data_ptr()
        # what the long-context calls check their tensors against
        self._index = -1 if self.device.type == "cpu" else self.device.index
        self._row_bytes = cfg.Hq * cfg.d * esz  # of q and out
        self._units = cfg.k * cfg.Hkv           # (channel, kv head) pairs of a sequence
        self._slots = self.max_pages * cfg.page_size

    # ------------------------------------------------------------------ setup
    def set_weights(self, pre_g, Wr, br, ch_g, Wkv, qk_g) -> None:
        """Per-branch sequences (index 0 = K, 1 = V) of device tensors."""
        self._weight_refs = (pre_g, Wr, br, ch_g, Wkv, qk_g)
        self._weights = W.mix_weights(pre_g, Wr, br, ch_g, Wkv, qk_g)

    def _check_device(self) -> None:
        # a launch goes to the current device, whatever its stream and pointers
        if self._index >= 0 and torch._C._cuda_getDevice() != self._index:
            raise ValueError(f"the session is on {self.device}, the current device is "
                             f"{torch._C._cuda_getDevice()}")

    def _stream(self, stream) -> ctypes.c_void_p:
        self._check_device()
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        return ctypes.c_void_p(s.cuda_stream)

    # ------------------------------------------------------------------ calls
    def decode_attn(self, layer: int, q, page_table, seq_lens, out, B: int | None = None,
                    stream=None, inputs_ready: bool = False, dynamic_split: bool = False,
                    unit_split: bool = False) -> None:
        """inputs_ready: the previous work on the stream wrote no cache, page
        table, lengths or workspace (true for layers 1..L-1 of a decode step).
        dynamic_split: chunks handed out by a device counter whatever the
        launch size (WM_ATTN_DYNAMIC_SPLIT).  unit_split: one cluster of CTAs
        per (sequence, kv head) unit whatever the launch size
        (WM_ATTN_UNIT_SPLIT)."""
        B = self.B if B is None else B
        flags = (W.WM_ATTN_INPUTS_READY if inputs_ready else 0) | \
            (W.WM_ATTN_DYNAMIC_SPLIT if dynamic_split else 0) | \
            (W.WM_ATTN_UNIT_SPLIT if unit_split else 0)
        rc = W.wm_decode_attn_flags(self.cfg, self.cache, layer, q, page_table, seq_lens, B,
                                    self.max_pages, out, self.attn_ws, self.attn_ws_bytes, flags,
                                    self.status, self._stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_decode_attn_flags")

    def prefill_attn(self, layer: int, q, pos, page_table, out, stream=None) -> None:
        """Causal attention of query rows q [B][Tq][Hq][d] at token positions
        pos [B][Tq] over layer ``layer``'s channel (prefill / parallel passes)."""
        B, Tq = int(q.shape[0]), int(q.shape[1])
        rc = W.wm_prefill_attn(self.cfg, self.cache, layer, q, pos, page_table, B, Tq,
                               self.max_pages, out, self.status, self._stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_prefill_attn")

    def kv_mix(self, h, page_table, slot, B: int | None = None, stream=None, pos=None) -> None:
        """pos: int32 positions of the tokens where they are not slot - 1
        (after an eviction)."""
        if self._weights is None:
            raise RuntimeError("set_weights() first")
        B = self.B if B is None else B
        if pos is not None:
            self._check((pos, _I32, B))
            rc = W.wm_kv_mix_at(self.cfg, self.cache, self._weights, h, page_table, slot, pos, B,
                                self.max_pages, self.mix_ws, self.mix_ws_bytes, self.status,
                                self._stream(stream))
            if rc != W.WM_OK:
                raise W.WMError(rc, "wm_kv_mix_at")
            return
        rc = W.wm_kv_mix(self.cfg, self.cache, self._weights, h, page_table, slot, B,
                         self.max_pages, self.mix_ws, self.mix_ws_bytes, self.status,
                         self._stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_kv_mix")

    # ---------------------------------------------------------- long contexts
    # The library takes addresses: a view with gaps or another order of its
    # dimensions, another type, fewer rows or another device's memory would be
    # read as if they were right.  The calls' checks are written out, since a
    # loop over the tensors takes about twice as long (1.6 against 0.9 us a call).
    # A page table of exactly the call's bytes is taken for [B][max_pages].
    def _check(self, *needs) -> None:
        """needs: (tensor, type, elements it holds at least)."""
        for t, dtype, n in needs:
            if not t.is_contiguous():
                raise ValueError("the library reads contiguous tensors only")
            if t.dtype is not dtype:
                raise ValueError(f"the library reads {dtype} here, not {t.dtype}")
            if t.numel() < n:
                raise ValueError(f"{t.numel()} elements where the call reads or writes {n}")
            if t.get_device() != self._index:
                raise ValueError(f"a tensor on {t.device} in a session on {self.device}")

    def _check_rows(self, q, index, page_table, out, B: int, n: int) -> None:
        """n query rows of B sequences; index: lengths or positions, one per row."""
        dt, dev, row, pages = self.dtype, self._index, n * self._row_bytes, self.max_pages
        if not (q.is_contiguous() and index.is_contiguous() and page_table.is_contiguous() and out.is_contiguous()
                and q.dtype is dt and out.dtype is dt and index.dtype is _I32 and page_table.dtype is _I32
                and q.nbytes >= row and out.nbytes >= row and index.nbytes >= 4 * n
                and page_table.nbytes == 4 * B * pages
                and q.get_device() == index.get_device() == page_table.get_device() == out.get_device() == dev):
            e = n * self.cfg.Hq * self.cfg.d
            self._check((q, dt, e), (index, _I32, n), (out, dt, e))
            self._check_table(page_table, B)

    def _check_table(self, page_table, B: int) -> None:
        self._check((page_table, _I32, B * self.max_pages))
        if page_table.dim() > 1 and page_table.shape[-1] != self.max_pages:
            raise ValueError(f"rows of {page_table.shape[-1]} pages in a session of {self.max_pages}")

    def _check_sums(self, B: int, *needs) -> None:
        """needs: (tensor, type, elements of every (channel, sequence, kv head) of a
        call of B sequences).  One made for more sequences is laid out otherwise."""
        for t, dtype, per in needs:
            n = self._units * B * per
            self._check((t, dtype, n))
            if t.numel() != n:
                raise ValueError(f"{t.numel()} elements where the call's sizes make {n}")

    @staticmethod
    def _counts(*counts: int):
        # the binding would keep the low 32 bits; no sequence has as many slots
        return (min(max(n, -1), 0x7FFFFFFF) for n in counts)

    def _raw_stream(self, stream) -> int:
        if torch._C._cuda_getDevice() != self._index:
            self._check_device()
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.device.index)
        return stream.cuda_stream

    def _scratch_for(self, nbytes: int, raw: int, stream):
        # one buffer per stream for the calls below (they need nothing in it,
        # so calls on one stream share it), allocated on that stream.  One that
        # is too small is replaced by one of at least twice its size, so that
        # all the outgrown ones together are smaller than the live one, which is
        # less than twice the largest size asked for.  The first call of a size
        # may allocate: make it before a graph capture.  Graphs captured on one
        # stream share its buffer: their replays must not overlap.
        if nbytes > _LARGE:
            return self._large_scratch_for(nbytes, raw, stream)
        buf = self._scratch.get(raw)
        if buf is None or buf.numel() < nbytes:
            if buf is not None:
                self._outgrown.append(buf)
                nbytes = max(nbytes, 2 * buf.numel())
            s = torch.cuda.current_stream(self.device) if stream is None else stream
            with torch.cuda.stream(s):
                buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self._scratch[raw] = buf
        return buf.data_ptr()

    def _large_scratch_for(self, nbytes: int, raw: int, stream):
        # as above, but of the size asked for, and an outgrown buffer is kept (and the
        # next one made twice its size) only where a graph was captured with it
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        with torch.cuda.stream(s):
            buf = self._large_scratch.get(raw)
            if buf is None or buf.numel() < nbytes:
                if raw in self._in_graphs:
                    self._in_graphs.remove(raw)
                    self._outgrown.append(buf)
                    nbytes = max(nbytes, 2 * buf.numel())
                buf = None
                self._large_scratch.pop(raw, None)  # (freed on its stream, before the next is allocated)
                buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
                self._large_scratch[raw] = buf
            if torch.cuda.is_current_stream_capturing():
                self._in_graphs.add(raw)
        return buf.data_ptr()

    def _bytes(self, key, query, *args) -> int:
        n = self._need.get(key)
        if n is None:
            n = query(self.cfg, *args)
            if n == 0:
                raise W.WMError(W.WM_ERR_INVALID_ARG, query.__name__)
            self._need[key] = n
        return n

    def window_attn(self, layer: int, q, page_table, seq_lens, out, *, sinks: int, window: int,
                    B: int | None = None, stream=None) -> None:
        """Decode attention over the first ``sinks`` slots and the last
        ``window`` slots of each sequence."""
        cfg, cache = self._refs
        B = self.B if B is None else B
        self._check_rows(q, seq_lens, page_table, out, B, B)
        if (sinks | window) >> 31:
            sinks, window = self._counts(sinks, window)
        rc = self._lib.wm_window_attn(cfg, cache, layer, q.data_ptr(), page_table.data_ptr(),
                                      seq_lens.data_ptr(), sinks, window, B, self.max_pages,
                                      out.data_ptr(), self._status_ptr, self._raw_stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_window_attn")

    def window_prefill_attn(self, layer: int, q, pos, page_table, out, *, sinks: int, window: int,
                            stream=None) -> None:
        """window_attn's mask for query rows q [B][Tq][Hq][d] at positions pos
        [B][Tq]: position i sees slots t <= i, t < sinks or t > i - window."""
        cfg, cache = self._refs
        B, Tq = q.shape[:2]
        self._check_rows(q, pos, page_table, out, B, B * Tq)
        if (sinks | window) >> 31:
            sinks, window = self._counts(sinks, window)
        rc = self._lib.wm_window_prefill_attn(cfg, cache, layer, q.data_ptr(), pos.data_ptr(),
                                              page_table.data_ptr(), sinks, window, B, Tq,
                                              self.max_pages, out.data_ptr(), self._status_ptr,
                                              self._raw_stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_window_prefill_attn")

    def prefix_attn(self, layer: int, q, page_table, seq_lens, out, *, shared_pages: int,
                    B: int | None = None, stream=None) -> None:
        """Decode attention of sequences whose first ``shared_pages`` pages are
        the same ones: those are read once for the batch."""
        cfg, cache = self._refs
        B = self.B if B is None else B
        self._check_rows(q, seq_lens, page_table, out, B, B)
        need = self._bytes(("prefix", B, self.max_pages, shared_pages), W.wm_prefix_attn_workspace, B,
                           self.max_pages, shared_pages)
        raw = self._raw_stream(stream)
        rc = self._lib.wm_prefix_attn(cfg, cache, layer, q.data_ptr(), page_table.data_ptr(),
                                      seq_lens.data_ptr(), shared_pages, B, self.max_pages,
                                      out.data_ptr(), self._scratch_for(need, raw, stream), need,
                                      self._status_ptr, raw)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_prefix_attn")

    def decode_attn_mass(self, layer: int, q, page_table, seq_lens, mass, out, *,
                         B: int | None = None, stream=None) -> None:
        """Decode attention that adds every slot's softmax weight, summed over
        the query heads of a kv head, to mass [k][B][Hkv][slots] (fp32)."""
        cfg, cache = self._refs
        B = self.B if B is None else B
        self._check_rows(q, seq_lens, page_table, out, B, B)
        need = 4 * self._units * B * self._slots
        if not (mass.is_contiguous() and mass.dtype is _F32 and mass.nbytes == need
                and mass.get_device() == self._index):
            self._check_sums(B, (mass, _F32, self._slots))
        need = self._bytes(("mass", B, self.max_pages), W.wm_decode_attn_mass_workspace, B, self.max_pages)
        raw = self._raw_stream(stream)
        rc = self._lib.wm_decode_attn_mass(cfg, cache, layer, q.data_ptr(), page_table.data_ptr(),
                                           seq_lens.data_ptr(), mass.data_ptr(), B, self.max_pages,
                                           out.data_ptr(), self._scratch_for(need, raw, stream),
                                           need, self._status_ptr, raw)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_decode_attn_mass")

    def evict(self, mass, page_table, seq_lens, mass_out, kept, new_lens, *, budget: int,
              sinks: int, recent: int, B: int | None = None, stream=None) -> None:
        """Cut every (channel, sequence, kv head) to ``budget`` slots: the
        first ``sinks``, the last ``recent`` and those with the largest mass.
        Writes mass_out (may be mass), kept [k][B][Hkv][budget] and new_lens."""
        cfg, cache = self._refs
        B = self.B if B is None else B
        dev, pages, units = self._index, self.max_pages, 4 * self._units * B
        if not (mass.is_contiguous() and mass_out.is_contiguous() and kept.is_contiguous() and seq_lens.is_contiguous()
                and new_lens.is_contiguous() and page_table.is_contiguous()
                and mass.dtype is _F32 and mass_out.dtype is _F32 and kept.dtype is _I32 and seq_lens.dtype is _I32
                and new_lens.dtype is _I32 and page_table.dtype is _I32
                and mass.nbytes == mass_out.nbytes == units * self._slots and kept.nbytes == units * budget
                and seq_lens.nbytes >= 4 * B and new_lens.nbytes >= 4 * B and page_table.nbytes == 4 * B * pages
                and mass.get_device() == mass_out.get_device() == kept.get_device() == seq_lens.get_device()
                == new_lens.get_device() == page_table.get_device() == dev):
            self._check((seq_lens, _I32, B), (new_lens, _I32, B))
            self._check_sums(B, (mass, _F32, self._slots), (mass_out, _F32, self._slots), (kept, _I32, budget))
            self._check_table(page_table, B)
        if (budget | sinks | recent) >> 31:
            budget, sinks, recent = self._counts(budget, sinks, recent)
        rc = self._lib.wm_cache_evict(cfg, cache, mass.data_ptr(), mass_out.data_ptr(),
                                      page_table.data_ptr(), seq_lens.data_ptr(), budget, sinks,
                                      recent, B, self.max_pages,
                                      kept.data_ptr(), new_lens.data_ptr(), self._status_ptr,
                                      self._raw_stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_cache_evict")

    # ------------------------------------------------------- caches held in 4 bits
    def _q4_ref(self, q4: Q4Cache):
        if q4._index != self._index:
            raise ValueError(f"a 4-bit cache on {q4.device} in a session on {self.device}")
        return q4._ref

    def _q4_copy(self, call, name, q4, src_table, dst_table, first, last, span, B, stream, write):
        cfg, cache = self._refs
        q4r = self._q4_ref(q4)
        B = self.B if B is None else B
        dev, table = self._index, 4 * B * self.max_pages
        if not (src_table.is_contiguous() and dst_table.is_contiguous() and first.is_contiguous()
                and last.is_contiguous() and src_table.dtype is _I32 and dst_table.dtype is _I32
                and first.dtype is _I32 and last.dtype is _I32 and src_table.nbytes == dst_table.nbytes == table
                and first.nbytes >= 4 * B and last.nbytes >= 4 * B
                and src_table.get_device() == dst_table.get_device() == first.get_device() == last.get_device() == dev):
            self._check((first, _I32, B), (last, _I32, B))
            self._check_table(src_table, B)
            self._check_table(dst_table, B)
        if span >> 31:
            span, = self._counts(span)
        src, dst = (cache, q4r) if write else (q4r, cache)
        rc = call(cfg, src, src_table.data_ptr(), dst, dst_table.data_ptr(), first.data_ptr(),
                  last.data_ptr(), span, B, self.max_pages, self._status_ptr, self._raw_stream(stream))
        if rc != W.WM_OK:
            raise W.WMError(rc, name)

    def q4_write(self, q4: Q4Cache, page_table, q4_table, first, last, *, span: int,
                 B: int | None = None, stream=None) -> None:
        """Slots first[b] .. last[b] - 1 of the session's cache (page_table) to
        the 4-bit cache (q4_table), all channels; no range longer than span."""
        self._q4_copy(self._lib.wm_q4_write, "wm_q4_write", q4, page_table, q4_table, first, last, span, B,
                      stream, True)

    def q4_read(self, q4: Q4Cache, q4_table, page_table, first, last, *, span: int,
                B: int | None = None, stream=None) -> None:
        """Slots first[b] .. last[b] - 1 of the 4-bit cache (q4_table) back into
        the session's cache (page_table), all channels."""
        self._q4_copy(self._lib.wm_q4_read, "wm_q4_read", q4, q4_table, page_table, first, last, span, B,
                      stream, False)

    def q4_kv_mix(self, h, q4: Q4Cache, page_table, slot, *, pos=None, B: int | None = None,
                  stream=None) -> None:
        """kv_mix that appends the tokens to a 4-bit cache (its pages: page_table)."""
        if self._weights is None:
            raise RuntimeError("set_weights() first")
        B = self.B if B is None else B
        q4r = self._q4_ref(q4)
        self._check((h, self.dtype, B * self.cfg.L * self.cfg.D), (slot, _I32, B))
        if pos is not None:
            self._check((pos, _I32, B))
        self._check_table(page_table, B)
        need = self._bytes(("q4 mix", B), W.wm_q4_kv_mix_workspace, B)
        raw = self._raw_stream(stream)
        rc = self._lib.wm_q4_kv_mix(self._refs[0], q4r, ctypes.byref(self._weights), h.data_ptr(),
                                    page_table.data_ptr(), slot.data_ptr(),
                                    None if pos is None else pos.data_ptr(), B, self.max_pages,
                                    self._scratch_for(need, raw, stream), need, self._status_ptr, raw)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_q4_kv_mix")

    def q4_decode_attn(self, layer: int, q, q4: Q4Cache, page_table, seq_lens, out, *,
                       B: int | None = None, stream=None) -> None:
        """Decode attention of layer ``layer`` over a 4-bit cache (its pages:
        page_table)."""
        B = self.B if B is None else B
        if layer >> 31:
            layer = -1  # (the binding would keep the low 32 bits)
        q4r = self._q4_ref(q4)
        self._check_rows(q, seq_lens, page_table, out, B, B)
        need = self._bytes(("q4", B, self.max_pages), W.wm_q4_decode_attn_workspace, B, self.max_pages)
        raw = self._raw_stream(stream)
        rc = self._lib.wm_q4_decode_attn(self._refs[0], q4r, layer, q.data_ptr(), page_table.data_ptr(),
                                         seq_lens.data_ptr(), B, self.max_pages, out.data_ptr(),
                                         self._scratch_for(need, raw, stream), need, self._status_ptr, raw)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_q4_decode_attn")

    def q4_rows_attn(self, layer: int, q, pos, q4: Q4Cache, page_table, out, *, stream=None) -> None:
        """Causal attention of query rows q [B][Tq][Hq][d] at positions pos
        [B][Tq] over a 4-bit cache: position i sees slots 0 .. i."""
        B, Tq = q.shape[:2]
        if layer >> 31:
            layer = -1
        q4r = self._q4_ref(q4)
        self._check_rows(q, pos, page_table, out, B, B * Tq)
        need = self._bytes(("q4 rows", B, Tq, self.max_pages), W.wm_q4_rows_attn_workspace, B, Tq, self.max_pages)
        raw = self._raw_stream(stream)
        rc = self._lib.wm_q4_rows_attn(self._refs[0], q4r, layer, q.data_ptr(), pos.data_ptr(),
                                       page_table.data_ptr(), B, Tq, self.max_pages, out.data_ptr(),
                                       self._scratch_for(need, raw, stream), need, self._status_ptr, raw)
        if rc != W.WM_OK:
            raise W.WMError(rc, "wm_q4_rows_attn")

    def read_status(self, reset: bool = True) -> int:
        v = int(self.status.item())
        if reset:
            self.status.zero_()
        return v
