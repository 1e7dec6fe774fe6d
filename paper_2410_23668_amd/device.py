"""Device-memory plumbing around the C ABI (torch is used only to allocate
device buffers and to name the stream).  Every step of the decode path runs
in libkl.so."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as kb

_DTYPES = {torch.bfloat16: kb.KL_DTYPE_BF16, torch.float16: kb.KL_DTYPE_FP16,
           torch.float32: kb.KL_DTYPE_FP32, torch.float8_e4m3fn: kb.KL_DTYPE_E4M3}


def _dev_u16(a, device) -> torch.Tensor:
    """Host bf16 bit patterns (uint16) -> device int16 tensor with the same bits
    (a device tensor of 16-bit values is taken as it is)."""
    if isinstance(a, torch.Tensor):
        assert a.element_size() == 2 and a.is_contiguous()
        return a.view(torch.int16).to(device)
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)


def stream_handle(stream: torch.cuda.Stream | None = None) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


class GpuModel:
    """A model loaded into libkl's packed arena."""

    def __init__(self, model_cfg: dict, weights: dict, max_batch: int, max_seq: int,
                 device="cuda", stream: torch.cuda.Stream | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("GpuModel needs a GPU")
        self.model_cfg = dict(model_cfg)
        self.device = torch.device(device)
        self.cfg = kb.make_config(model_cfg, max_batch, max_seq)
        self.max_batch, self.max_seq = max_batch, max_seq
        src = {}
        layers = []
        for l, lay in enumerate(weights["layers"]):
            ptrs = {}
            for n in kb.PTR_FIELDS:
                if n not in lay:
                    continue
                t = _dev_u16(lay[n], self.device)
                src[(l, n)] = t
                ptrs[n] = t.data_ptr()
            layers.append(ptrs)
        g = {n: _dev_u16(weights[n], self.device) for n in ("embed", "final_norm", "lm_head")}
        torch.cuda.synchronize(self.device)
        self.state = kb.kl_load_model(self.cfg, g["embed"].data_ptr(), g["final_norm"].data_ptr(),
                                      g["lm_head"].data_ptr(), layers, stream_handle(stream))
        del src, g   # kl_load_model copied and repacked everything

    @classmethod
    def from_layers(cls, model_cfg: dict, layer_fn, globals_fn, max_batch: int, max_seq: int,
                    device="cuda", stream: torch.cuda.Stream | None = None) -> "GpuModel":
        """Load one layer at a time (kl_model_create + kl_model_set_layer): only
        one layer's source weights are on the device at once.  layer_fn(l) and
        globals_fn() return host bf16 arrays by name (as in model_host)."""
        if not torch.cuda.is_available():
            raise RuntimeError("GpuModel needs a GPU")
        self = cls.__new__(cls)
        self.model_cfg = dict(model_cfg)
        self.device = torch.device(device)
        self.cfg = kb.make_config(model_cfg, max_batch, max_seq)
        self.max_batch, self.max_seq = max_batch, max_seq
        self.state = kb.kl_model_create(self.cfg)
        h = stream_handle(stream)
        for l in range(model_cfg["n_layers"]):
            lay = layer_fn(l)
            src = {n: _dev_u16(lay[n], self.device)
                   for n in kb.PTR_FIELDS if n in lay}
            torch.cuda.synchronize(self.device)
            kb.kl_model_set_layer(self.state, l, {n: t.data_ptr() for n, t in src.items()}, h)
            del src, lay
        g = globals_fn()
        src = {n: _dev_u16(g[n], self.device) for n in ("embed", "final_norm", "lm_head")}
        torch.cuda.synchronize(self.device)
        kb.kl_model_set_globals(self.state, src["embed"].data_ptr(), src["final_norm"].data_ptr(),
                                src["lm_head"].data_ptr(), h)
        del src, g
        return self

    def info(self) -> kb.kl_info:
        return kb.kl_get_info(self.state)

    def device_error(self) -> int:
        return kb.kl_get_device_error(self.state)

    def _batch(self, tokens, positions, logits, hidden, device) -> int:
        """The batch of a step's tensors, which are contiguous and on the cache's device."""
        B = tokens.numel()
        assert tokens.dtype == torch.int32 and positions.dtype == torch.int32
        assert positions.numel() == B
        assert logits.dtype == torch.float32 and logits.shape == (B, self.model_cfg["vocab"])
        if hidden is not None:
            assert hidden.dtype == torch.float32 and hidden.shape == (B, self.model_cfg["hidden"])
        for x in (tokens, positions, logits, hidden):
            assert x is None or (x.is_contiguous() and x.device == device)
        return B

    def step(self, tokens: torch.Tensor, positions: torch.Tensor, kv: "KvCache",
             logits: torch.Tensor, hidden: torch.Tensor | None, mode: int,
             stream: torch.cuda.Stream | None = None) -> None:
        B = self._batch(tokens, positions, logits, hidden, kv.k.device)
        kb.kl_decode_step(self.state, tokens.data_ptr(), positions.data_ptr(), B,
                          kv.k.data_ptr(), kv.v.data_ptr(), kv.batch, kv.capacity,
                          logits.data_ptr(), hidden.data_ptr() if hidden is not None else None,
                          stream_handle(stream), mode)

    def step_paged(self, tokens: torch.Tensor, positions: torch.Tensor, pool: "PagedKvCache",
                   table: torch.Tensor, logits: torch.Tensor, hidden: torch.Tensor | None = None,
                   stream: torch.cuda.Stream | None = None) -> None:
        """step() over a paged cache: row b of the table holds sequence b's pages.
        May be captured into a graph."""
        B = self._batch(tokens, positions, logits, hidden, pool.device)
        kb.kl_decode_step_paged(self.state, tokens.data_ptr(), positions.data_ptr(), B, pool.c,
                                pool._table(table), logits.data_ptr(),
                                hidden.data_ptr() if hidden is not None else None,
                                stream_handle(stream))

    def greedy(self, tokens: torch.Tensor, positions: torch.Tensor, kv: "KvCache", n_steps: int,
               tokens_out: torch.Tensor, logits: torch.Tensor, mode: int,
               stream: torch.cuda.Stream | None = None) -> None:
        B = self._batch(tokens, positions, logits, None, kv.k.device)
        assert tokens_out.dtype == torch.int32 and tokens_out.shape == (n_steps, B)
        assert tokens_out.is_contiguous() and tokens_out.device == kv.k.device
        kb.kl_decode_greedy(self.state, tokens.data_ptr(), positions.data_ptr(), B, n_steps,
                            kv.k.data_ptr(), kv.v.data_ptr(), kv.batch, kv.capacity,
                            tokens_out.data_ptr(), logits.data_ptr(), stream_handle(stream), mode)

    def close(self):
        if getattr(self, "state", None):
            kb.kl_free_model(self.state)
            self.state = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KvCache:
    """K and V caches [L][batch][n_kv][capacity][d] bf16 (as int16 tensors)."""

    def __init__(self, model_cfg: dict, batch: int, capacity: int, device="cuda",
                 k_host: np.ndarray | None = None, v_host: np.ndarray | None = None):
        shape = (model_cfg["n_layers"], batch, model_cfg["n_kv_heads"], capacity,
                 model_cfg["head_dim"])
        self.batch, self.capacity = batch, capacity
        if k_host is not None:
            assert k_host.shape == shape and v_host.shape == shape
            self.k = _dev_u16(k_host, device)
            self.v = _dev_u16(v_host, device)
        else:
            self.k = torch.zeros(shape, dtype=torch.int16, device=device)
            self.v = torch.zeros(shape, dtype=torch.int16, device=device)

    def host(self):
        return (self.k.cpu().numpy().view(np.uint16), self.v.cpu().numpy().view(np.uint16))


class PagedKvCache:
    """A pool of KV cache pages for sequences of any length: k and v
    [L][pages][n_kv][page_size][d], bf16 or e4m3; an e4m3 pool has a scale byte
    (biased exponent of a power of two) per row in k_scale and v_scale
    [L][pages][n_kv][page_size].  Which pages hold a sequence is the caller's
    to decide: a table [batch][max_pages] int32 of page numbers, of which those
    of positions not in use may be anything."""

    def __init__(self, model_cfg: dict, n_pages: int, page_size: int = 64,
                 dtype: torch.dtype = torch.bfloat16, device="cuda"):
        shape = (model_cfg["n_layers"], n_pages, model_cfg["n_kv_heads"], page_size,
                 model_cfg["head_dim"])
        scales = [None, None]
        if dtype == torch.float8_e4m3fn:
            # (127: the codes of a cleared pool stand for themselves)
            scales = [torch.full(shape[:-1], 127, dtype=torch.uint8, device=device)
                      for _ in range(2)]
        self._bind(torch.zeros(shape, dtype=dtype, device=device),
                   torch.zeros(shape, dtype=dtype, device=device), *scales)

    @classmethod
    def from_tensors(cls, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                     v_scale: torch.Tensor | None = None) -> "PagedKvCache":
        """A pool over the caller's tensors (which stay in use)."""
        self = cls.__new__(cls)
        self._bind(k, v, k_scale, v_scale)
        return self

    def _bind(self, k, v, k_scale, v_scale):
        assert k.dim() == 5 and k.shape == v.shape and k.dtype == v.dtype
        assert k.dtype in (torch.bfloat16, torch.float8_e4m3fn)
        assert k.is_contiguous() and v.is_contiguous() and k.device == v.device
        assert k.device.type == "cuda"
        if k.dtype == torch.float8_e4m3fn:
            for s in (k_scale, v_scale):
                assert s is not None and s.dtype == torch.uint8 and s.shape == k.shape[:-1]
                assert s.is_contiguous() and s.device == k.device
        else:
            assert k_scale is None and v_scale is None
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device = k.device
        L, pages, n_kv, ps, d = k.shape
        self.n_kv, self.page_size, self.head_dim = n_kv, ps, d
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.c = kb.kl_paged_cache(
            k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
            None if v_scale is None else v_scale.data_ptr(), _DTYPES[k.dtype], L, pages, n_kv, ps, d,
            self.device.index)
        self._filled()

    def _filled(self) -> None:
        """What has been filled on the current stream is there for calls on any stream
        (in a capture the fill is a part of the graph instead, before the calls there)."""
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.device).synchronize()

    def _table(self, table: torch.Tensor) -> kb.kl_page_table:
        (batch, n), (row, one) = table.shape, table.stride()
        assert table.dtype == torch.int32 and table.device == self.device
        assert one == 1 or n <= 1
        return kb.kl_page_table(table.data_ptr(), batch, n, row if batch > 1 else n)

    def _rows(self, x: torch.Tensor, rows: int, heads: int) -> kb.kl_rows:
        row, head, one = x.stride()
        assert x.shape == (rows, heads, self.head_dim) and one == 1 and x.device == self.device
        assert x.dtype in _DTYPES
        return kb.kl_rows(x.data_ptr(), _DTYPES[x.dtype], row, head)

    def _stream(self, stream: torch.cuda.Stream | None) -> int:
        if stream is not None:
            return stream.cuda_stream
        # (the current stream without a Stream object, which takes 2.6 us to make)
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    def _slots(self, positions, seq) -> tuple:
        assert positions.dtype == torch.int32 and positions.dim() == 1
        assert positions.is_contiguous() and positions.device == self.device
        if seq is not None:
            assert seq.dtype == torch.int32 and seq.shape == positions.shape
            assert seq.is_contiguous() and seq.device == self.device
        return seq.data_ptr() if seq is not None else None, positions.data_ptr(), positions.numel()

    def append(self, layer: int, table: torch.Tensor, positions: torch.Tensor, k: torch.Tensor,
               v: torch.Tensor, seq: torch.Tensor | None = None,
               stream: torch.cuda.Stream | None = None) -> None:
        """Rows [n][n_kv][d] of k and v to the slots of (seq[i], positions[i])
        (seq None: row i is sequence i's; a negative position is skipped)."""
        s, p, n = self._slots(positions, seq)
        kb.kl_paged_append(self.c, layer, self._table(table), s, p, n,
                           self._rows(k, n, self.n_kv), self._rows(v, n, self.n_kv),
                           self.error.data_ptr(), self._stream(stream))

    def read(self, layer: int, table: torch.Tensor, positions: torch.Tensor, k: torch.Tensor,
             v: torch.Tensor, seq: torch.Tensor | None = None,
             stream: torch.cuda.Stream | None = None) -> None:
        """The slots' values into rows [n][n_kv][d] of k and v (arguments as for append)."""
        s, p, n = self._slots(positions, seq)
        kb.kl_paged_read(self.c, layer, self._table(table), s, p, n,
                         self._rows(k, n, self.n_kv), self._rows(v, n, self.n_kv),
                         self.error.data_ptr(), self._stream(stream))

    def workspace(self, batch: int) -> torch.Tensor:
        """A workspace for attention calls of up to 'batch' sequences, one after
        the other (calls that may overlap, graphs replayed side by side
        included, need one each), on any stream."""
        n = kb.kl_paged_attention_workspace(self.c, batch)
        if n == 0:
            raise kb.KlError(kb.KL_ERR_INVALID_ARGUMENT, kb.kl_last_error())
        ws = torch.zeros(n, dtype=torch.uint8, device=self.device)
        self._filled()
        return ws

    def attention(self, layer: int, table: torch.Tensor, lengths: torch.Tensor, q: torch.Tensor,
                  out: torch.Tensor, workspace: torch.Tensor, scale: float | None = None,
                  window: int = 0, lse: torch.Tensor | None = None,
                  stream: torch.cuda.Stream | None = None) -> None:
        """One new token per sequence over its first lengths[b] positions: q and
        out [batch][heads][d], lse [batch][heads] fp32; scale 1/sqrt(d) unless given."""
        B, heads = q.shape[0], q.shape[1]
        assert lengths.dtype == torch.int32 and lengths.shape == (B,) and lengths.is_contiguous()
        assert lengths.device == self.device and table.shape[0] == B
        assert workspace.dtype == torch.uint8 and workspace.is_contiguous()
        assert workspace.device == self.device
        if lse is not None:
            assert lse.dtype == torch.float32 and lse.shape == (B, heads) and lse.is_contiguous()
            assert lse.device == self.device
        kb.kl_paged_attention(self.c, layer, self._table(table), lengths.data_ptr(),
                              self._rows(q, B, heads), heads,
                              self.head_dim ** -0.5 if scale is None else scale, window,
                              self._rows(out, B, heads),
                              lse.data_ptr() if lse is not None else None, workspace.data_ptr(),
                              workspace.numel(), self.error.data_ptr(), self._stream(stream))

    def device_error(self) -> int:
        """Waits for all of the device's streams; the error bits of this pool's calls so
        far, which are then cleared (before any later call on any stream)."""
        torch.cuda.synchronize(self.device)
        code = int(self.error.item())
        if code:
            self.error.zero_()
            torch.cuda.synchronize(self.device)
        return code
