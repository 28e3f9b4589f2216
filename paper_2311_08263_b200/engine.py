"""`Decoder`: owns the device buffers (through torch) and forwards every call to the C ABI.

PyTorch is used for device memory and the stream only; every step of the decode path runs in the
CUDA library.  Method names match the C entry points they call.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Dict, Optional

import numpy as np
import torch

from . import lib as _l


class FcError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        msg = _l.load().fc_strerror(code).decode()
        super().__init__(f"{where}: {msg} ({code}) {detail}".strip())


_GUARD, _GUARD_BYTE = 4096, 0xA5      # canary band on either side of the K/V slab and of the workspace


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


class Decoder:
    def __init__(self, cfg, weights: Dict[str, object], max_batch: int, max_c: int, max_seq: int,
                 flags: int = 0, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required (there is no CPU fallback)")
        self.lib = _l.load()
        self.cfg, self.device = cfg, torch.device(device)
        torch.cuda.set_device(self.device)
        dt = _l.FC_F32 if cfg.dtype == "f32" else _l.FC_BF16
        self.shape = _l.fc_model_shape(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.n_kv_heads, cfg.head_dim,
                                       cfg.d_ffn, cfg.vocab, dt, cfg.rms_eps, cfg.rope_theta,
                                       max_batch, max_c, max_seq, cfg.bias_beta, flags)
        kvb = self.lib.fc_kv_bytes(C.byref(self.shape))
        wsb = self.lib.fc_workspace_bytes(C.byref(self.shape))
        if kvb == 0 or wsb == 0:
            raise FcError(_l.FC_ERR_SHAPE, "fc_kv_bytes")
        # each buffer sits between two canary bands (checked by fc_debug_check_guards)
        self._kv_bytes, self._ws_bytes = kvb, wsb
        self._kv_alloc = torch.full((kvb + 2 * _GUARD,), _GUARD_BYTE, dtype=torch.uint8, device=self.device)
        self._ws_alloc = torch.full((wsb + 2 * _GUARD,), _GUARD_BYTE, dtype=torch.uint8, device=self.device)
        self.kv = self._kv_alloc[_GUARD:_GUARD + kvb]
        self.ws = self._ws_alloc[_GUARD:_GUARD + wsb]
        self.kv.zero_()
        self.ws.zero_()
        self._keep = []

        def dev(t: torch.Tensor) -> int:
            t = t.to(self.device).contiguous()
            assert t.dtype == cfg.torch_dtype, (t.dtype, cfg.torch_dtype)
            self._keep.append(t)
            return t.data_ptr()

        def table(ts):
            arr = (C.c_void_p * len(ts))(*[dev(t) for t in ts])
            self._keep.append(arr)
            return C.cast(arr, _l._PP)

        perm = weights.get("bias_perm")
        perm_ptr = None
        if perm is not None:
            p = perm.to(self.device, torch.int32).contiguous()
            self._keep.append(p)
            perm_ptr = p.data_ptr()
        self.weights = _l.fc_weights(dev(weights["tok_emb"]),
                                     *[table(weights[n]) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up",
                                                                   "w_down", "g_attn", "g_ffn")],
                                     dev(weights["g_final"]), dev(weights["lm_head"]), perm_ptr)
        self.stream = torch.cuda.current_stream(self.device)
        h = C.c_void_p()
        rc = self.lib.fc_init(C.byref(h), C.byref(self.shape), C.byref(self.weights),
                              self.kv.data_ptr(), kvb, self.ws.data_ptr(), wsb, self.stream.cuda_stream)
        if rc != _l.FC_OK:
            raise FcError(rc, "fc_init")
        self.h = h
        self.batch = self.c = 0
        self._logits: Optional[torch.Tensor] = None

    def close(self):
        if getattr(self, "h", None):
            self.lib.fc_destroy(self.h)
            self.h = None

    __del__ = close

    def _check(self, rc: int, where: str):
        if rc != _l.FC_OK:
            raise FcError(rc, where, self.lib.fc_last_cuda_error(self.h).decode())

    # ---- C ABI calls -------------------------------------------------------------------------
    def fc_prefill(self, prompt_ids, prompt_lens, c: int, refill: int = 0, pad_id: int = 0):
        ids, lens = _i32(prompt_ids), _i32(prompt_lens)
        if ids.ndim == 1:
            ids = ids[None]
        self._check(self.lib.fc_prefill(self.h, ids.shape[0], ids.ctypes.data, ids.shape[1],
                                        lens.ctypes.data, c, refill, pad_id), "fc_prefill")
        self.batch, self.c = ids.shape[0], c

    def fc_jacobi_step(self, window_in=None):
        """Returns (accepted_count [B], accepted_tokens [B, c], window_out [B, c])."""
        B, c = self.batch, self.c
        cnt, tok, win = np.zeros(B, np.int32), np.zeros((B, c), np.int32), np.zeros((B, c), np.int32)
        wi = _i32(window_in).reshape(B, c) if window_in is not None else None
        self._check(self.lib.fc_jacobi_step(self.h, wi.ctypes.data if wi is not None else None,
                                            cnt.ctypes.data, tok.ctypes.data, win.ctypes.data), "fc_jacobi_step")
        return cnt, tok, win

    def fc_generate(self, max_tokens: int, eos_id: int = -1, c: int = 0, max_iters: int = 0):
        """Returns (tokens [B, max_tokens], lens [B], stats).  c = 0 keeps the current window size."""
        B = self.batch
        out, lens = np.zeros((B, max_tokens), np.int32), np.zeros(B, np.int32)
        st = _l.fc_stats()
        self._check(self.lib.fc_generate(self.h, max_tokens, c, eos_id, max_iters, out.ctypes.data, lens.ctypes.data,
                                         C.byref(st)), "fc_generate")
        if c > 0:
            self.c = c
        return out, lens, st

    def fc_set_window(self, c: int):
        self._check(self.lib.fc_set_window(self.h, c), "fc_set_window")
        self.c = c

    def fc_finish_with_trigger(self, trigger_ids, max_answer_tokens: int, eos_id: int = -1):
        """Returns (answer tokens [B, max_answer_tokens], lens [B]).  The sequences need fc_prefill afterwards."""
        B = self.batch
        t = _i32(trigger_ids)
        out, lens = np.zeros((B, max(max_answer_tokens, 1)), np.int32), np.zeros(B, np.int32)
        self._check(self.lib.fc_finish_with_trigger(self.h, t.ctypes.data if t.shape[0] else None, t.shape[0],
                                                    max_answer_tokens, eos_id, out.ctypes.data, lens.ctypes.data),
                    "fc_finish_with_trigger")
        return out[:, :max_answer_tokens], lens

    def fc_debug_inject_timeout(self):
        self._check(self.lib.fc_debug_inject_timeout(self.h), "fc_debug_inject_timeout")

    def fc_debug_withhold_arrival(self):
        self._check(self.lib.fc_debug_withhold_arrival(self.h), "fc_debug_withhold_arrival")

    def fc_debug_check_guards(self) -> int:
        """Number of damaged canary bands: those between the workspace slices (kept by the library) plus the ones
        this binding keeps around the K/V slab and the workspace."""
        n = C.c_int32(0)
        self._check(self.lib.fc_debug_check_guards(self.h, C.byref(n)), "fc_debug_check_guards")
        bad = int(n.value)
        for buf, nbytes in ((self._kv_alloc, self._kv_bytes), (self._ws_alloc, self._ws_bytes)):
            lo, hi = buf[:_GUARD], buf[_GUARD + nbytes:]
            bad += int((lo != _GUARD_BYTE).any().item()) + int((hi != _GUARD_BYTE).any().item())
        return bad

    def fc_debug_set_state(self, kv_lens, pending, c: int, pad_id: int = 0):
        kl, pe = _i32(kv_lens), _i32(pending)
        self._check(self.lib.fc_debug_set_state(self.h, kl.shape[0], kl.ctypes.data, pe.ctypes.data, c, pad_id),
                    "fc_debug_set_state")
        self.batch, self.c = kl.shape[0], c

    def fc_debug_logits(self, enable: bool = True) -> Optional[torch.Tensor]:
        """Device tensor [max_batch*max_c, vocab] that receives the logits of every later step."""
        if enable:
            rows = self.shape.max_batch * self.shape.max_c
            self._logits = torch.zeros(rows, self.cfg.vocab, dtype=torch.float32, device=self.device)
            self._check(self.lib.fc_debug_logits(self.h, self._logits.data_ptr()), "fc_debug_logits")
        else:
            self._check(self.lib.fc_debug_logits(self.h, None), "fc_debug_logits")
            self._logits = None
        return self._logits

    def fc_get_state(self):
        kl, ng = np.zeros(self.batch, np.int32), np.zeros(self.batch, np.int32)
        self._check(self.lib.fc_get_state(self.h, kl.ctypes.data, ng.ctypes.data), "fc_get_state")
        return kl, ng

    def fc_bench_steps(self, n_steps: int, commit: bool = False):
        """Returns (device milliseconds for n_steps back-to-back steps, tokens committed)."""
        ms, tok = C.c_float(0), C.c_int64(0)
        self._check(self.lib.fc_bench_steps(self.h, n_steps, int(commit), C.byref(ms), C.byref(tok)),
                    "fc_bench_steps")
        return float(ms.value), int(tok.value)

    def fc_profile_step(self):
        """Returns {class name: (milliseconds, launches)} for one non-committing step."""
        n = len(_l.FC_CLASSES)
        ms, cnt = (C.c_float * n)(), (C.c_int32 * n)()
        self._check(self.lib.fc_profile_step(self.h, ms, cnt), "fc_profile_step")
        return {name: (float(ms[i]), int(cnt[i])) for i, name in enumerate(_l.FC_CLASSES)}

    def fc_last_launch_count(self) -> int:
        return int(self.lib.fc_last_launch_count(self.h))

    def fc_last_route(self) -> int:
        return int(self.lib.fc_last_route(self.h))

    # ---- K/V slab view for the window-step sweep (the caller writes random K/V into it) --------
    def kv_view(self) -> torch.Tensor:
        s = self.shape
        return self.kv.view(self.cfg.torch_dtype).view(s.n_layers, 2, s.max_batch, s.n_kv_heads,
                                                       s.max_seq, s.head_dim)


def fc_op_linear(x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, use_tensor_cores: bool) -> int:
    """y[R, N] += x[R, K] . w[N, K]^T on the device (x, y fp32; w fp32 or bf16)."""
    lib = _l.load()
    R, K = x.shape
    N = w.shape[0]
    assert x.is_cuda and w.is_cuda and y.is_cuda and x.dtype == torch.float32 and y.dtype == torch.float32
    assert x.is_contiguous() and w.is_contiguous() and y.is_contiguous()
    dt = _l.FC_F32 if w.dtype == torch.float32 else _l.FC_BF16
    return lib.fc_op_linear(x.data_ptr(), w.data_ptr(), y.data_ptr(), R, N, K, dt, int(use_tensor_cores),
                            torch.cuda.current_stream().cuda_stream)


def fc_op_accept(window, argmax, kv_len, n_gen, prompt, prompt_lens, refill: int, pad_id: int):
    """Runs the accept kernel on device int32 tensors; returns (accepted_count, accepted_tokens)."""
    lib = _l.load()
    B, c = window.shape
    cnt = torch.zeros(B, dtype=torch.int32, device=window.device)
    tok = torch.zeros(B, c, dtype=torch.int32, device=window.device)
    rc = lib.fc_op_accept(window.data_ptr(), argmax.data_ptr(), kv_len.data_ptr(), n_gen.data_ptr(),
                          cnt.data_ptr(), tok.data_ptr(),
                          prompt.data_ptr() if prompt is not None else None,
                          prompt_lens.data_ptr() if prompt_lens is not None else None,
                          B, c, prompt.shape[1] if prompt is not None else 1, refill, pad_id,
                          torch.cuda.current_stream().cuda_stream)
    if rc != _l.FC_OK:
        raise FcError(rc, "fc_op_accept")
    return cnt, tok


def fc_op_window_attention(q: torch.Tensor, kcache: torch.Tensor, vcache: torch.Tensor, kv_len: torch.Tensor,
                           c: int, n_heads: int, max_len: int) -> torch.Tensor:
    """Window attention of one layer.  q [B*c, n_heads*hd]; kcache/vcache [B, n_kv_heads, max_seq, hd];
    kv_len int32 [B] on the device.  Returns fp32 [B*c, n_heads*hd]."""
    lib = _l.load()
    B, hkv, max_seq, hd = kcache.shape
    dt = _l.FC_F32 if q.dtype == torch.float32 else _l.FC_BF16
    nbytes = lib.fc_op_window_attention_scratch_bytes(B, c, n_heads, hkv, hd, max_len, dt)
    scratch = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    out = torch.empty(B * c, n_heads * hd, dtype=torch.float32, device=q.device)
    rc = lib.fc_op_window_attention(q.data_ptr(), kcache.data_ptr(), vcache.data_ptr(), kv_len.data_ptr(),
                                    out.data_ptr(), B, c, n_heads, hkv, hd, max_seq, max_len, dt,
                                    scratch.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    if rc != _l.FC_OK:
        raise FcError(rc, "fc_op_window_attention")
    return out


def fc_op_fused_window_attention(qkv_acc: torch.Tensor, sumsq: torch.Tensor, rms_eps: float, d_norm: int,
                                 rope_theta: float, kcache: torch.Tensor, vcache: torch.Tensor, kv_len: torch.Tensor,
                                 c: int, n_heads: int, max_len: int, n_splits: int = 0, q_tiles: int = 0) -> torch.Tensor:
    """The fused attention kernel of the bf16 step as one operation.  qkv_acc fp32 [B*c, (hq + 2 hkv) * hd] and sumsq
    fp32 [B*c] are consumed (cleared); kcache/vcache bf16 [B, hkv, max_seq, hd] receive the window's rows.
    Returns fp32 [B*c, hq*hd]."""
    lib = _l.load()
    B, hkv, max_seq, hd = kcache.shape
    nbytes = lib.fc_op_fused_window_attention_scratch_bytes(B, c, n_heads, hkv, hd, max_seq, max_len)
    if nbytes == 0:
        raise FcError(_l.FC_ERR_ARG, "fc_op_fused_window_attention_scratch_bytes")
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=qkv_acc.device)
    out = torch.empty(B * c, n_heads * hd, dtype=torch.float32, device=qkv_acc.device)
    rc = lib.fc_op_fused_window_attention(qkv_acc.data_ptr(), sumsq.data_ptr(), rms_eps, d_norm, rope_theta,
                                          kcache.data_ptr(), vcache.data_ptr(), kv_len.data_ptr(), out.data_ptr(),
                                          B, c, n_heads, hkv, hd, max_seq, max_len, n_splits, q_tiles,
                                          scratch.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    if rc != _l.FC_OK:
        raise FcError(rc, "fc_op_fused_window_attention")
    return out


def fc_op_short_window_attention(qkv_acc: torch.Tensor, sumsq: torch.Tensor, rms_eps: float, d_norm: int, rope_theta: float,
                                 kv: torch.Tensor, kv_len: torch.Tensor, c: int, n_heads: int, max_len: int) -> torch.Tensor:
    """The attention kernel behind the one-writer projections as one operation.  kv: bf16 [2, B, hkv, max_seq, hd], keys and values;
    receives the window's rows.  Returns fp32 [B*c, hq*hd], the sum of the bf16 pair that the kernel writes."""
    lib = _l.load()
    _, B, hkv, max_seq, hd = kv.shape
    nbytes = lib.fc_op_fused_window_attention_scratch_bytes(B, c, n_heads, hkv, hd, max_seq, max_len)
    if nbytes == 0:
        raise FcError(_l.FC_ERR_ARG, "fc_op_fused_window_attention_scratch_bytes")
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=kv.device)
    pair = torch.empty(2, B * c, n_heads * hd, dtype=torch.bfloat16, device=kv.device)
    rc = lib.fc_op_short_window_attention(qkv_acc.data_ptr(), sumsq.data_ptr(), rms_eps, d_norm, rope_theta, kv[0].data_ptr(),
                                          kv[1].data_ptr(), kv_len.data_ptr(), pair.data_ptr(), B, c, n_heads, hkv, hd, max_seq,
                                          max_len, scratch.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    if rc != _l.FC_OK:
        raise FcError(rc, "fc_op_short_window_attention")
    return pair.float().sum(0)


# ---- paged K/V cache ------------------------------------------------------------------------------------------------
# Pools are tensors [layers, pages, kv heads, slots, head size] (one layer: without the first dimension) of any strides with adjacent
# elements; a layout with the slots outside the heads is a transposed view.  The calls enqueue work on the current stream of the tensors'
# device and return; they can be captured into CUDA graphs.

_CACHE_TYPES = {torch.float32: _l.FC_F32, torch.bfloat16: _l.FC_BF16}
_POOL = ("k and v: fp32 or bf16 tensors of the same shape and strides on one CUDA device, adjacent elements, "
         "[layers, pages, kv heads, slots, head size] (operations on one layer: without the first dimension)")
_raw_stream = torch._C._cuda_getCurrentRawStream        # a stream object costs two microseconds


# What these calls cost is mostly what Python does for them, so each looks at a tensor's properties once and by the cheapest accessor.
def _pool(k: torch.Tensor, v: torch.Tensor, dims: int) -> _l.fc_pages:
    shape, stride, dtype = k.shape, k.stride(), _CACHE_TYPES.get(k.dtype)
    if (dtype is None or len(shape) != dims or v.shape != shape or v.stride() != stride or v.dtype is not k.dtype or stride[-1] != 1
            or k.get_device() < 0 or v.get_device() != k.get_device()):
        raise ValueError(_POOL)
    if dims == 4:
        return _l.fc_pages(k.data_ptr(), v.data_ptr(), dtype, 1, *shape, 0, *stride[:3])
    return _l.fc_pages(k.data_ptr(), v.data_ptr(), dtype, *shape, *stride[:4])


def _ints(name: str, t: torch.Tensor, dims: int, device: int) -> int:
    if t.dtype is not torch.int32 or t.dim() != dims or not t.is_contiguous() or t.get_device() != device or device < 0:
        raise ValueError(f"{name}: contiguous int32 tensor of {dims} dimension(s) on the pool's CUDA device")
    return t.data_ptr()


def _lengths(kv_len: torch.Tensor, n: int, device: int) -> int:
    if kv_len.numel() != n:
        raise ValueError("kv_len: one length per row of the table")
    return _ints("kv_len", kv_len, 1, device)


def _rows(x: torch.Tensor):
    """Strides of a matrix; that of a single row says nothing."""
    row, elem = x.stride()
    return (row, elem) if x.shape[0] > 1 else (x.shape[1], elem)


def _in_int32(*numbers: int) -> None:
    """ctypes drops the bits beyond 32 without a word; what C refuses within them (negative numbers among it) is left to C."""
    if max(numbers) > 0x7fffffff or min(numbers) < -0x80000000:
        raise ValueError("numbers beyond 32 bits")


def _list(ids):
    if len(ids):
        _in_int32(*ids)
    return (C.c_int32 * len(ids))(*ids)


def _enqueue(device: int, fn, *args) -> None:
    """The call on the current stream of the tensors' device."""
    if device == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _raw_stream(device))
    if rc:
        raise FcError(rc, fn.__name__)


@functools.lru_cache(maxsize=1024)
def _scratch_bytes(name: str, *sizes: int) -> int:
    return getattr(_l.load(), name)(*sizes)


def fc_op_paged_store(qkv: torch.Tensor, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, c: int, n_heads: int,
                      rope_theta: float) -> torch.Tensor:
    """QKV rows of one layer into pages.  qkv fp32 [B*c, (n_heads + 2 n_kv_heads) * hd], rows adjacent or not; k/v [pages, n_kv_heads,
    slots, hd]; table int32 [B, width]; kv_len int32 [B].  Returns the rotated queries [B*c, n_heads * hd] in the pool's type; those of
    table rows without a sequence are not written."""
    pool, device = _pool(k, v, 4), k.get_device()
    tab = _ints("table", table, 2, device)
    B, width = table.shape
    row, elem = _rows(qkv)
    if (qkv.dtype is not torch.float32 or qkv.shape != (B * c, (n_heads + 2 * pool.n_kv_heads) * pool.head_dim) or elem != 1
            or qkv.get_device() != device):
        raise ValueError("qkv: fp32 [B * c, (n_heads + 2 n_kv_heads) * head size] with adjacent elements, on the pool's device")
    q = torch.empty(B * c, n_heads * pool.head_dim, dtype=k.dtype, device=k.device)
    _enqueue(device, _l.load().fc_op_paged_store, pool, 0, tab, width, _lengths(kv_len, B, device), qkv.data_ptr(), row, q.data_ptr(), B, c,
             n_heads, rope_theta)
    return q


def fc_op_paged_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, c: int,
                          n_heads: int, window: int = 0, n_sink: int = 0) -> torch.Tensor:
    """Window attention of one layer over pages, optionally under a sliding window with sinks.  q [B*c, n_heads * hd] in the pool's type,
    rows adjacent or not; the rest as in fc_op_paged_store, the rows' own keys and values stored.  Returns fp32 [B*c, n_heads * hd]."""
    _in_int32(window, n_sink)
    pool, device = _pool(k, v, 4), k.get_device()
    tab = _ints("table", table, 2, device)
    B, width = table.shape
    hd = pool.head_dim
    row, elem = _rows(q)
    if q.dtype is not k.dtype or q.shape != (B * c, n_heads * hd) or elem != 1 or q.get_device() != device:
        raise ValueError("q: [B * c, n_heads * head size] in the pool's type with adjacent elements, on the pool's device")
    nbytes = _scratch_bytes("fc_op_paged_attention_scratch_bytes", B, c, n_heads, pool.n_kv_heads, hd, pool.dtype, width, pool.page_size, window, n_sink)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=k.device) if nbytes > 256 else None         # 256: none is used
    out = torch.empty(B * c, n_heads * hd, dtype=torch.float32, device=k.device)
    _enqueue(device, _l.load().fc_op_paged_attention, pool, 0, tab, width, _lengths(kv_len, B, device), q.data_ptr(), row, out.data_ptr(), B, c,
             n_heads, window, n_sink, scratch.data_ptr() if scratch is not None else None, nbytes)
    return out


def fc_op_pages_fork(table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor, page_size: int, src, dst) -> None:
    """Table rows dst[i] share the pages of rows src[i]'s committed tokens (lists of row numbers on the host)."""
    _in_int32(page_size, refs.numel())
    device, (rows, width), n = table.get_device(), table.shape, len(dst)
    if len(src) != n:
        raise ValueError("src and dst: two lists of the same length")
    _enqueue(device, _l.load().fc_op_pages_fork, _ints("table", table, 2, device), width, rows, _lengths(kv_len, rows, device),
             _ints("refs", refs, 1, device), refs.numel(), page_size, _list(src), _list(dst), n)


def fc_op_pages_free(table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor, page_size: int, seqs, window: int = 0,
                     n_sink: int = 0) -> None:
    """Release the pages of table rows `seqs` (a list on the host): all of them, or those that no later row of a sliding window sees."""
    _in_int32(page_size, refs.numel(), window, n_sink)
    device, (rows, width) = table.get_device(), table.shape
    _enqueue(device, _l.load().fc_op_pages_free, _ints("table", table, 2, device), width, rows, _lengths(kv_len, rows, device),
             _ints("refs", refs, 1, device), refs.numel(), page_size, _list(seqs), len(seqs), window, n_sink)


def fc_op_pages_reserve(k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor,
                        rows: int) -> torch.Tensor:
    """Pages for positions kv_len .. kv_len + rows - 1 of every sequence, copies of shared ones.  k/v [layers, pages, n_kv_heads, slots, hd].
    Returns int32 [n_seqs]: 1 where the positions can be written."""
    _in_int32(rows, rows)
    pool, device = _pool(k, v, 5), k.get_device()
    tab, counts = _ints("table", table, 2, device), _ints("refs", refs, 1, device)
    n, width = table.shape
    if refs.numel() != pool.n_pages:
        raise ValueError("refs: one count per page")
    nbytes = _scratch_bytes("fc_op_pages_reserve_scratch_bytes", pool.n_pages, n)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=k.device)
    served = torch.empty(n, dtype=torch.int32, device=k.device)
    _enqueue(device, _l.load().fc_op_pages_reserve, pool, tab, width, n, _lengths(kv_len, n, device), counts, rows, served.data_ptr(),
             scratch.data_ptr(), nbytes)
    return served


def fc_op_pages_compact(k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, refs: torch.Tensor) -> torch.Tensor:
    """Move the pages in use to the front of the pool, in all layers; table and refs follow.  Returns int32 [1]: how many are in use."""
    pool, device = _pool(k, v, 5), k.get_device()
    tab, counts = _ints("table", table, 2, device), _ints("refs", refs, 1, device)
    n, width = table.shape
    if refs.numel() != pool.n_pages:
        raise ValueError("refs: one count per page")
    nbytes = _scratch_bytes("fc_op_pages_compact_scratch_bytes", pool.n_pages)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=k.device)
    n_live = torch.empty(1, dtype=torch.int32, device=k.device)
    _enqueue(device, _l.load().fc_op_pages_compact, pool, tab, width, n, counts, n_live.data_ptr(), scratch.data_ptr(), nbytes)
    return n_live
