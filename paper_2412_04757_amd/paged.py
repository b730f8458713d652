"""Binding of include/ltri_paged.h: a key-value cache in pages (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import LTRI_BF16, LTRI_F32, LtriError, LtriPagedConfig, _ptr, load_library


def paged_config(n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: str, page_tokens: int, n_pages: int,
                 table_pages: int, max_seqs: int, rows_max: int = 1, weights: bool = False, page_stride: int = 0,
                 head_stride: int = 0, token_stride: int = 0) -> LtriPagedConfig:
    """dtype: "f32" or "bf16". Strides (elements) of the pools: all 0 = dense, or those of the tensors LtriPagedCache is given."""
    if dtype not in ("f32", "bf16"):
        raise ValueError(f"dtype {dtype!r}: 'f32' or 'bf16'")
    return LtriPagedConfig(n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                           dtype=LTRI_F32 if dtype == "f32" else LTRI_BF16, page_tokens=page_tokens, n_pages=n_pages,
                           table_pages=table_pages, max_seqs=max_seqs, rows_max=rows_max, weights=int(weights),
                           page_stride=page_stride, head_stride=head_stride, token_stride=token_stride)


class LtriPagedCache:
    """One attention layer's cache in pages: its pools, weights and positions (torch tensors) and the ltri_paged handle.

    k_pages, v_pages: [n_pages][n_kv_heads][page_tokens][head_dim], views of another order of the first three included
    (allocated here, zeroed, if not given); weight (fp32), pos (int32): [n_pages][n_kv_heads][page_tokens], with weights = 1.
    scratch: a uint8 tensor of at least scratch_bytes that caches whose calls do not overlap may share.
    Work goes to the stream given here (default: the current one) or to set_stream(); what is enqueued on other streams is the caller's
    to order, and a call's tensors to keep until its work is done. The cache's own buffers may go at any time: the allocator is told of
    every stream that used them. (A captured graph of its calls needs the cache as long as it is replayed.)"""

    def __init__(self, cfg: LtriPagedConfig, device: Optional[torch.device], dry: bool = False,
                 stream: Optional[torch.cuda.Stream] = None, k_pages: Optional[torch.Tensor] = None,
                 v_pages: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None):
        self.lib = load_library()
        self.handle = C.c_void_p()
        self.dry = dry
        self.cfg = cfg = LtriPagedConfig.from_buffer_copy(cfg)
        self.tdtype = torch.float32 if cfg.dtype == LTRI_F32 else torch.bfloat16
        self._index = -1                                     # of the device, as tensors say it (-1: the CPU)
        shape = (cfg.n_pages, cfg.n_kv_heads, cfg.page_tokens, cfg.head_dim)
        if (k_pages is None) != (v_pages is None):
            raise ValueError("k_pages and v_pages: both or neither")
        if k_pages is not None:
            for t in (k_pages, v_pages):
                if tuple(t.shape) != shape or t.dtype != self.tdtype or t.stride(3) != 1:
                    raise ValueError(f"pools are {self.tdtype} {shape} with dense rows; got {t.dtype} {tuple(t.shape)}, "
                                     f"strides {tuple(t.stride())}")
            if any(n > 1 and step == 0 for n, step in zip(shape, k_pages.stride())):     # (three zeros would say "dense" to the library)
                raise ValueError(f"pools whose rows overlap: strides {tuple(k_pages.stride())} of an expanded tensor")
            if k_pages.stride() != v_pages.stride():
                raise ValueError(f"k_pages and v_pages differ in strides: {k_pages.stride()}, {v_pages.stride()}")
            cfg.page_stride, cfg.head_stride, cfg.token_stride = k_pages.stride()[:3]
        sb, cb = C.c_size_t(), C.c_size_t()
        self._check(self.lib.ltri_paged_workspace_bytes(C.byref(cfg), C.byref(sb), C.byref(cb)))
        self.state_bytes, self.scratch_bytes = sb.value, cb.value
        if dry:
            self._check(self.lib.ltri_paged_create_dry(C.byref(cfg), C.byref(self.handle)))
            return
        self.device = device = torch.device(device.type, torch.cuda.current_device() if device.index is None else device.index)
        self._index = device.index
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        if self.stream.device != device:
            raise ValueError(f"a stream of {self.stream.device}, the cache is on {device}")
        with torch.cuda.stream(self.stream):                 # (what is allocated here is filled and used there)
            if k_pages is None:
                k_pages = torch.zeros(shape, dtype=self.tdtype, device=device)
                v_pages = torch.zeros(shape, dtype=self.tdtype, device=device)
                cfg.page_stride, cfg.head_stride, cfg.token_stride = k_pages.stride()[:3]
            if cfg.weights:
                weight = torch.zeros(shape[:3], dtype=torch.float32, device=device) if weight is None else weight
                pos = torch.zeros(shape[:3], dtype=torch.int32, device=device) if pos is None else pos
            for name, t, dtype in (("weight", weight, torch.float32), ("pos", pos, torch.int32)):
                if t is not None and (tuple(t.shape) != shape[:3] or not cfg.weights):
                    raise ValueError(f"{name}: {shape[:3]} with weights, else None")
                _ptr(t, dtype)
            if scratch is not None and (scratch.dtype != torch.uint8 or scratch.numel() < self.scratch_bytes):
                raise ValueError(f"scratch: uint8, at least {self.scratch_bytes} bytes")
            for t in (k_pages, v_pages, weight, pos, scratch):
                if t is not None and t.device != device:
                    raise ValueError(f"a tensor of the cache is on {t.device}, the cache on {device}")
            self.k_pages, self.v_pages, self.weight, self.pos = k_pages, v_pages, weight, pos
            self.state = torch.empty(self.state_bytes, dtype=torch.uint8, device=device)
            self.scratch = torch.empty(self.scratch_bytes, dtype=torch.uint8, device=device) if scratch is None else scratch
            self._used_on(self.stream)
            self._check(self.lib.ltri_paged_create(C.byref(cfg), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(weight), _ptr(pos),
                                                   self.state.data_ptr(), _ptr(self.scratch), self.stream.cuda_stream,
                                                   C.byref(self.handle)))

    def _used_on(self, stream: "torch.cuda.Stream") -> None:
        """The buffers' memory is not given to others before the work that this stream has by then is done, wherever they were allocated."""
        for t in (self.k_pages, self.v_pages, self.weight, self.pos, self.state, self.scratch):
            if t is not None:
                t.record_stream(stream)

    def _check(self, status: int) -> None:
        if status != 0:
            detail = self.lib.ltri_paged_last_error(self.handle).decode() if self.handle else ""
            raise LtriError(status, f"{self.lib.ltri_strerror(status).decode()}: {detail}")

    def close(self) -> None:
        if self.handle:
            self.lib.ltri_paged_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _arg(self, name: str, t: Optional[torch.Tensor], shape: tuple, dtype: torch.dtype) -> Optional[int]:
        """Address of a dense tensor of this shape on the cache's device. (A decoding step is as long as a few of these calls: one condition.)"""
        if t is None:
            return None
        if t.shape != shape or t.dtype is not dtype or not t.is_contiguous() or t.get_device() != self._index:
            raise ValueError(f"{name}: expected a dense {dtype} {shape} on {'the CPU' if self.dry else self.device}; got {t.dtype} "
                             f"{tuple(t.shape)}, strides {tuple(t.stride())}, on {t.device}")
        return t.data_ptr()

    def _places(self, table, lens, seen=None):
        n = len(table)
        return (n, self._arg("table", table, (n, self.cfg.table_pages), torch.int32), self._arg("lens", lens, (n,), torch.int32),
                self._arg("seen", seen, (n,), torch.int32))

    def _rows(self, n: int, k_new: torch.Tensor, v_new: torch.Tensor):
        c, n_new = self.cfg, k_new.shape[2] if k_new.dim() == 4 else 0
        shape = (n, c.n_kv_heads, n_new, c.head_dim)
        return self._arg("k_new", k_new, shape, self.tdtype), self._arg("v_new", v_new, shape, self.tdtype), n_new

    def _outputs(self, n: int, q: torch.Tensor, out, lse):
        c, n_q = self.cfg, q.shape[1] if q.dim() == 4 else 0
        shape = (n, n_q, c.n_q_heads, c.head_dim)
        q_ptr = self._arg("q", q, shape, self.tdtype)
        if out is None:
            if self.dry or torch.cuda.current_stream(self._index) == self.stream:
                out = torch.empty_like(q)
            else:                                            # its memory belongs to the stream that writes it
                with torch.cuda.stream(self.stream):
                    out = torch.empty_like(q)
        return q_ptr, n_q, out, self._arg("out", out, shape, self.tdtype), self._arg("lse", lse, shape[:3], torch.float32)

    # ---- the C ABI, same names ----
    def set_stream(self, stream: "torch.cuda.Stream") -> None:
        """ltri_paged_set_stream: the caller orders the new stream behind the old one's work (stream.wait_stream), creation included."""
        if not self.dry:
            if stream.device != self.device:
                raise ValueError(f"a stream of {stream.device}, the cache is on {self.device}")
            self._used_on(stream)
        self._check(self.lib.ltri_paged_set_stream(self.handle, stream.cuda_stream))
        self.stream = stream

    def append(self, table: torch.Tensor, lens: torch.Tensor, seen: Optional[torch.Tensor], k_new: torch.Tensor,
               v_new: torch.Tensor, w_new: Optional[torch.Tensor] = None) -> None:
        """ltri_paged_append: k_new, v_new [n][n_kv_heads][n_new][head_dim], w_new fp32 [n][n_kv_heads][n_new]."""
        n, t, l, s = self._places(table, lens, seen)
        k, v, n_new = self._rows(n, k_new, v_new)
        w = self._arg("w_new", w_new, (n, self.cfg.n_kv_heads, n_new), torch.float32)
        self._check(self.lib.ltri_paged_append(self.handle, n, t, l, s, k, v, w, n_new))

    def attend(self, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, decay: Optional[float] = None) -> torch.Tensor:
        """ltri_paged_attend: q, out [n][n_q][n_q_heads][head_dim], lse fp32 [n][n_q][n_q_heads]; decay None: weights stay."""
        n, t, l, _ = self._places(table, lens)
        q_ptr, n_q, out, o_ptr, lse_ptr = self._outputs(n, q, out, lse)
        self._check(self.lib.ltri_paged_attend(self.handle, n, t, l, q_ptr, n_q, o_ptr, lse_ptr, -1.0 if decay is None else decay))
        return out

    def step(self, table: torch.Tensor, lens: torch.Tensor, seen: Optional[torch.Tensor], k_new: torch.Tensor, v_new: torch.Tensor,
             q: torch.Tensor, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
             decay: Optional[float] = None) -> torch.Tensor:
        """ltri_paged_step: append (weights of new tokens 0) and attend of the same rows."""
        n, t, l, s = self._places(table, lens, seen)
        k, v, n_new = self._rows(n, k_new, v_new)
        if q.shape[1:2] != (n_new,):
            raise ValueError(f"q {tuple(q.shape)} for {n_new} new tokens")
        q_ptr, _, out, o_ptr, lse_ptr = self._outputs(n, q, out, lse)
        self._check(self.lib.ltri_paged_step(self.handle, n, t, l, s, k, v, q_ptr, n_new, o_ptr, lse_ptr,
                                             -1.0 if decay is None else decay))
        return out

    def evict(self, table: torch.Tensor, lens: torch.Tensor, seen: torch.Tensor, keep: int, n_sink: int = 0, n_recent: int = 0) -> None:
        """ltri_paged_evict: sequences of more than `keep` tokens go back to `keep`; lens is written."""
        n, t, l, s = self._places(table, lens, seen)
        self._check(self.lib.ltri_paged_evict(self.handle, n, t, l, s, keep, n_sink, n_recent))

    def sync_status(self) -> int:
        return int(self.lib.ltri_paged_sync_status(self.handle))
