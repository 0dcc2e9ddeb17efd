"""Device-memory plumbing around the C ABI for tests, the smoke check and the benchmark.

PyTorch is used for nothing but allocating device buffers, host<->device copies
and the stream handle; every computation of the path happens inside libpac.so.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as pb
from .inputs import Workload


def _stream_handle() -> int:
    return int(torch.cuda.current_stream().cuda_stream)


class Session:
    """Owns the device buffers of one configuration (cache, workspace, params, optimizer state)."""

    def __init__(self, w: Workload, cache_samples: int | None = None, lens=None, device: str = "cuda:0",
                 flags: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("libpac needs a GPU: no HIP device is visible")
        self.w = w
        self.dev = torch.device(device)
        self.dtype = pb.PAC_BF16 if w.cache_dtype == "bf16" else pb.PAC_F32
        self.ctx = pb.pac_create(w.L, w.d, w.n_max, w.r, w.C, w.B, w.N, self.dtype, flags)
        self.P = pb.pac_param_count(self.ctx)
        n = w.N if cache_samples is None else cache_samples
        self.cache_bytes = pb.pac_cache_bytes(self.ctx, lens, n)
        assert self.cache_bytes > 0
        self.cache = torch.empty(self.cache_bytes, dtype=torch.uint8, device=self.dev)
        self.ws_bytes = pb.pac_workspace_bytes(self.ctx)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev)
        self.params = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.m = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.v = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.grads = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=self.dev)
        self.logits = torch.zeros(w.B * w.C, dtype=torch.float32, device=self.dev)
        self.step_count = 0
        self.hp = pb.pac_adamw(1e-3, 0.9, 0.999, 1e-8, 0.01)

    def close(self):
        if self.ctx:
            pb.pac_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- state -----------------------------------------------------------
    def set_params(self, p: np.ndarray) -> None:
        self.params.copy_(torch.from_numpy(np.ascontiguousarray(p, dtype=np.float32)))
        self.m.zero_()
        self.v.zero_()
        self.step_count = 0

    # ---- the two calls ---------------------------------------------------
    def cache_fill(self, sample_ids, acts, lens=None) -> None:
        """acts: device tensor [count][L][n_max][d], float32 or bfloat16 (or a numpy float32 array)."""
        if isinstance(acts, np.ndarray):
            acts = torch.from_numpy(np.ascontiguousarray(acts, dtype=np.float32)).to(self.dev)
        assert acts.is_contiguous() and acts.device.type == "cuda"
        dt = pb.PAC_BF16 if acts.dtype == torch.bfloat16 else pb.PAC_F32
        assert acts.dtype in (torch.bfloat16, torch.float32)
        pb.pac_cache_fill(self.ctx, self.cache.data_ptr(), self.cache_bytes, sample_ids, acts.data_ptr(), dt,
                          lens, _stream_handle())

    def loss_grad(self, sample_ids, labels_dev, want_grads: bool = True, want_logits: bool = True) -> None:
        pb.pac_adapter_loss_grad(self.ctx, self.cache.data_ptr(), sample_ids, labels_dev.data_ptr(),
                                 self.params.data_ptr(), self.ws.data_ptr(), self.ws_bytes,
                                 self.loss.data_ptr(), self.logits.data_ptr() if want_logits else None,
                                 self.grads.data_ptr() if want_grads else None, _stream_handle())

    def step(self, sample_ids, labels_dev, keep_grads: bool = True) -> None:
        self.step_count = pb.pac_adapter_step(
            self.ctx, self.cache.data_ptr(), sample_ids, labels_dev.data_ptr(), self.params.data_ptr(),
            self.m.data_ptr(), self.v.data_ptr(), self.step_count, self.hp, self.ws.data_ptr(), self.ws_bytes,
            self.loss.data_ptr(), self.grads.data_ptr() if keep_grads else None, _stream_handle())

    # ---- read-back -------------------------------------------------------
    def cache_block(self, sample_id: int) -> np.ndarray:
        """Stored values of one sample: uint16 bf16 bits or float32, [L][len][d]."""
        off, ln = pb.pac_cache_lookup(self.ctx, sample_id)
        es = 2 if self.dtype == pb.PAC_BF16 else 4
        n = self.w.L * ln * self.w.d
        raw = self.cache[off * es:(off + n) * es].cpu().numpy()
        return raw.view(np.uint16 if es == 2 else np.float32).reshape(self.w.L, ln, self.w.d)


class LadderSession(Session):
    """The same cache trained through the paper's default architecture (include/pac_ladder.h): own parameter vector
    and workspace, the ladder's two calls."""

    def __init__(self, w: Workload, heads: int, cache_samples: int | None = None, lens=None, device: str = "cuda:0"):
        super().__init__(w, cache_samples=cache_samples, lens=lens, device=device)
        self.heads = heads
        self.P = pb.pac_ladder_param_count(self.ctx)
        self.ws_bytes = pb.pac_ladder_workspace_bytes(self.ctx, heads)
        if self.P <= 0 or self.ws_bytes <= 0:
            raise ValueError("configuration not supported by the ladder path")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev)
        self.params = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.m = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.v = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.grads = torch.zeros(self.P, dtype=torch.float32, device=self.dev)

    def loss_grad(self, sample_ids, labels_dev, want_grads: bool = True, want_logits: bool = True) -> None:
        pb.pac_ladder_loss_grad(self.ctx, self.cache.data_ptr(), sample_ids, labels_dev.data_ptr(), self.heads,
                                self.params.data_ptr(), self.ws.data_ptr(), self.ws_bytes, self.loss.data_ptr(),
                                self.logits.data_ptr() if want_logits else None,
                                self.grads.data_ptr() if want_grads else None, _stream_handle())

    def step(self, sample_ids, labels_dev, keep_grads: bool = True) -> None:
        self.step_count = pb.pac_ladder_step(
            self.ctx, self.cache.data_ptr(), sample_ids, labels_dev.data_ptr(), self.heads, self.params.data_ptr(),
            self.m.data_ptr(), self.v.data_ptr(), self.step_count, self.hp, self.ws.data_ptr(), self.ws_bytes,
            self.loss.data_ptr(), self.grads.data_ptr() if keep_grads else None, _stream_handle())


class TieredSession(Session):
    """The same buffers with the cache in pinned host memory and two device windows: batch k + 1 is reloaded on a
    copy stream while batch k trains on the compute stream (events order the two; default stream priorities)."""

    def __init__(self, w: Workload, cache_samples: int | None = None, lens=None, device: str = "cuda:0", flags: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("libpac needs a GPU: no HIP device is visible")
        self.w = w
        self.dev = torch.device(device)
        self.dtype = pb.PAC_BF16 if w.cache_dtype == "bf16" else pb.PAC_F32
        self.ctx = pb.pac_create(w.L, w.d, w.n_max, w.r, w.C, w.B, w.N, self.dtype, flags)
        self.P = pb.pac_param_count(self.ctx)
        n = w.N if cache_samples is None else cache_samples
        self.cache_bytes = pb.pac_cache_bytes(self.ctx, lens, n)
        assert self.cache_bytes > 0
        self.host_cache = torch.empty(self.cache_bytes, dtype=torch.uint8, pin_memory=True)
        self.window_bytes = pb.pac_tier_window_bytes(self.ctx)
        self.windows = [torch.empty(self.window_bytes, dtype=torch.uint8, device=self.dev) for _ in range(2)]
        self.copy_stream = torch.cuda.Stream(device=self.dev)
        self.ready = [torch.cuda.Event() for _ in range(2)]
        self.free = [torch.cuda.Event() for _ in range(2)]
        for e in self.free:
            e.record()
        self.ws_bytes = pb.pac_workspace_bytes(self.ctx)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev)
        self.params = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.m = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.v = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.grads = torch.zeros(self.P, dtype=torch.float32, device=self.dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=self.dev)
        self.logits = torch.zeros(w.B * w.C, dtype=torch.float32, device=self.dev)
        self.step_count = 0
        self.hp = pb.pac_adamw(1e-3, 0.9, 0.999, 1e-8, 0.01)

    def cache_fill(self, sample_ids, acts, lens=None) -> None:
        if isinstance(acts, np.ndarray):
            acts = torch.from_numpy(np.ascontiguousarray(acts, dtype=np.float32)).to(self.dev)
        assert acts.is_contiguous() and acts.device.type == "cuda"
        dt = pb.PAC_BF16 if acts.dtype == torch.bfloat16 else pb.PAC_F32
        pb.pac_tier_fill(self.ctx, self.host_cache.data_ptr(), self.cache_bytes, sample_ids, acts.data_ptr(), dt, lens,
                         self.windows[0].data_ptr(), self.window_bytes, _stream_handle())
        self.free[0].record()

    def prefetch(self, k: int, sample_ids) -> None:
        """Reload the batch into window k % 2 on the copy stream, once the step that last read that window is done."""
        slot = k % 2
        self.copy_stream.wait_event(self.free[slot])
        pb.pac_tier_stage(self.ctx, self.host_cache.data_ptr(), sample_ids, self.windows[slot].data_ptr(), self.window_bytes,
                          int(self.copy_stream.cuda_stream))
        self.ready[slot].record(self.copy_stream)

    def step_staged(self, k: int, sample_ids, labels_dev, keep_grads: bool = True) -> None:
        slot = k % 2
        torch.cuda.current_stream().wait_event(self.ready[slot])
        self.step_count = pb.pac_adapter_step_staged(
            self.ctx, self.windows[slot].data_ptr(), sample_ids, labels_dev.data_ptr(), self.params.data_ptr(),
            self.m.data_ptr(), self.v.data_ptr(), self.step_count, self.hp, self.ws.data_ptr(), self.ws_bytes,
            self.loss.data_ptr(), self.grads.data_ptr() if keep_grads else None, _stream_handle())
        self.free[slot].record()

    def loss_grad_staged(self, k: int, sample_ids, labels_dev) -> None:
        slot = k % 2
        torch.cuda.current_stream().wait_event(self.ready[slot])
        pb.pac_adapter_loss_grad_staged(self.ctx, self.windows[slot].data_ptr(), sample_ids, labels_dev.data_ptr(),
                                        self.params.data_ptr(), self.ws.data_ptr(), self.ws_bytes, self.loss.data_ptr(),
                                        self.logits.data_ptr(), self.grads.data_ptr(), _stream_handle())
        self.free[slot].record()

    def cache_block(self, sample_id: int) -> np.ndarray:
        torch.cuda.synchronize()
        off, ln = pb.pac_cache_lookup(self.ctx, sample_id)
        es = 2 if self.dtype == pb.PAC_BF16 else 4
        n = self.w.L * ln * self.w.d
        raw = self.host_cache[off * es:(off + n) * es].numpy()
        return raw.view(np.uint16 if es == 2 else np.float32).reshape(self.w.L, ln, self.w.d).copy()


# ---- blocks of the frozen backbone (include/pac_mx4.h, pac_norm.h, pac_attn.h, pac_kv4.h) ------------------------------------------
# The library takes addresses alone, so what they stand for is checked here.  A single token's kernel takes 4 us: the checks are
# written to cost little beside it.
_KIND = {torch.bfloat16: pb.PAC_BF16, torch.float32: pb.PAC_F32}


def _fits(n: int, what: str) -> int:
    """n, which the library takes in 32 bits (ctypes drops what lies above)."""
    if not -1 << 31 <= n < 1 << 31:
        raise ValueError(f"{what}: {n} is past 2^31 - 1" if n > 0 else f"{what}: {n} is below -2^31")
    return n


def _rows_of(t, name: str, rows: int, cols: int, gpu: int):
    """(row stride, pac_dtype) of a [rows][cols] matrix with neighbouring columns on the GPU of that number (-1: none)."""
    kind = _KIND.get(t.dtype)
    if kind is None or t.get_device() != gpu or gpu < 0 or t.shape != (rows, cols):
        raise ValueError(f"{name}: bfloat16 or float32, ({rows}, {cols}), on GPU {gpu} is wanted, not {t.dtype}, {tuple(t.shape)}, on {t.device}")
    stride = t.stride()
    if stride[1] != 1 and cols > 1:
        raise ValueError(f"{name}: neighbouring columns are wanted")
    return (stride[0] if rows > 1 else max(stride[0], cols)), kind


def _chunked_rows(t, name: str, rows: int, cols: int, gpu: int) -> int:
    """The row stride of a bf16 matrix that is read in 16-byte pieces, in the last row too."""
    stride, kind = _rows_of(t, name, rows, cols, gpu)
    if kind != pb.PAC_BF16:
        raise ValueError(f"{name}: bfloat16 is wanted")
    if cols % 8:
        pad = (cols + 7) // 8 * 8
        if rows == 1:
            stride = pad
        if rows and 2 * (t.storage_offset() + (rows - 1) * stride + pad) > t.untyped_storage().nbytes():
            raise ValueError(f"{name}: rows are read up to a multiple of 8 columns, the last one too")
    elif rows == 1:
        stride = cols
    return stride


def _stored(codes, scales, rows: int, cols: int, device) -> None:
    _fits(cols, "columns")
    for t, pitch, name in ((codes, pb.pac_mx4_code_pitch(cols), "codes"), (scales, pb.pac_mx4_scale_pitch(cols), "scales")):
        if t.dtype != torch.uint8 or t.shape != (rows, pitch) or t.device != device or not t.is_contiguous():
            raise ValueError(f"{name}: dense uint8, ({rows}, {pitch}), on {device} is wanted")


def _call(gpu: int, name: str, *args) -> None:
    """The library's function of that name on args and that GPU's current stream, with that GPU current."""
    if torch._C._cuda_getDevice() != gpu:
        with torch.cuda.device(gpu):
            return _call(gpu, name, *args)
    status = getattr(_lib(), name)(*args, torch._C._cuda_getCurrentRawStream(gpu))
    if status:
        raise pb.PacError(status, name)


_lib = pb.lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def mx4_empty(rows: int, cols: int, device="cuda:0"):
    """Buffers for a matrix in the stored form: (codes, scales)."""
    _fits(cols, "columns")
    return (torch.empty(rows, pb.pac_mx4_code_pitch(cols), dtype=torch.uint8, device=device),
            torch.empty(rows, pb.pac_mx4_scale_pitch(cols), dtype=torch.uint8, device=device))


def mx4_quantize(x, codes, scales) -> None:
    """x (bf16 or fp32, any row stride) into the stored form."""
    rows, cols = x.shape
    gpu = x.get_device()
    stride, kind = _rows_of(x, "x", rows, cols, gpu)
    _stored(codes, scales, rows, cols, x.device)
    _call(gpu, "pac_mx4_quantize", x.data_ptr(), kind, rows, cols, stride, codes.data_ptr(), scales.data_ptr())


def mx4_dequantize(codes, scales, out) -> None:
    """The values a stored matrix stands for, into out (bf16 or fp32, both exact)."""
    rows, cols = out.shape
    gpu = out.get_device()
    stride, kind = _rows_of(out, "out", rows, cols, gpu)
    _stored(codes, scales, rows, cols, out.device)
    _call(gpu, "pac_mx4_dequantize", codes.data_ptr(), scales.data_ptr(), rows, cols, out.data_ptr(), kind, stride)


class Mx4Linear:
    """A frozen linear layer with weights in the stored form: y = act(x W^T + bias), and dx = dy W on the way back.  Between calls its
    tensors may be changed in place, and may be given other storage.  bf16 rows have to start on 16 bytes (a view of rows padded to a
    multiple of 8 columns, where K or N is none); BlockNorm's states are dense, so that such widths are copied between the two."""

    def __init__(self, codes, scales, K: int, bias=None):
        self.N, self.K, self.dev = _fits(codes.shape[0], "outputs"), K, codes.device
        self._gpu = codes.get_device()
        if self._gpu < 0:
            raise ValueError("codes: on a GPU")
        self.codes, self.scales, self.bias = codes, scales, bias
        self._w = None
        self._weights()
        self._x_bytes = pb.pac_mx4_linear_qx_workspace_bytes(1, K)

    def _weights(self):
        """(codes, scales, bias): addresses as they are now, looked at again where they are not what they were."""
        w = self.codes.data_ptr(), self.scales.data_ptr(), _ptr(self.bias)
        if w != self._w:
            bias = self.bias
            _stored(self.codes, self.scales, self.N, self.K, self.dev)
            if bias is not None and (bias.shape != (self.N,) or bias.dtype != torch.float32 or bias.device != self.dev or not bias.is_contiguous()):
                raise ValueError("bias: float32, one value an output, on the weights' device")
            self._w = w
        return w

    @classmethod
    def from_weights(cls, w, bias=None):
        """w [N][K], bf16 or fp32, is quantised; the layer keeps the stored form only."""
        codes, scales = mx4_empty(w.shape[0], w.shape[1], w.device)
        mx4_quantize(w, codes, scales)
        return cls(codes, scales, w.shape[1], bias)

    def forward(self, x, y, gelu: bool = False, x4: bool = False) -> None:
        """x [M][K] bf16, rows on 16 bytes; y [M][N] bf16 or fp32.  x4: x (bf16 or fp32, any row stride) is quantised too, and the
        product runs on 4-bit operands."""
        M, gpu = _fits(x.shape[0], "rows"), self._gpu
        sy, kind = _rows_of(y, "y", M, self.N, gpu)
        act = pb.PAC_MX4_ACT_GELU if gelu else pb.PAC_MX4_ACT_NONE
        codes, scales, bias = self._weights()
        if x4:
            sx, xkind = _rows_of(x, "x", M, self.K, gpu)
            need = M * self._x_bytes  # x in the stored form, for this call, on this stream
            ws = torch.empty(need, dtype=torch.uint8, device=self.dev)
            _call(gpu, "pac_mx4_linear_qx", x.data_ptr(), xkind, M, self.K, sx, codes, scales, self.N, bias, act, y.data_ptr(), kind, sy,
                  ws.data_ptr(), need)
        else:
            sx = _chunked_rows(x, "x", M, self.K, gpu)
            _call(gpu, "pac_mx4_linear", x.data_ptr(), M, self.K, sx, codes, scales, self.N, bias, act, y.data_ptr(), kind, sy)

    def forward_stored(self, codes, scales, y, gelu: bool = False) -> None:
        """The same with x [M][K] already in the stored form (mx4_quantize): layers that share an input quantise it once.  The same bits as
        forward with x4."""
        M, gpu = _fits(codes.shape[0], "rows"), self._gpu
        _stored(codes, scales, M, self.K, self.dev)
        sy, kind = _rows_of(y, "y", M, self.N, gpu)
        w, ws, bias = self._weights()
        _call(gpu, "pac_mx4_linear_x4", codes.data_ptr(), scales.data_ptr(), M, self.K, w, ws, self.N, bias,
              pb.PAC_MX4_ACT_GELU if gelu else pb.PAC_MX4_ACT_NONE, y.data_ptr(), kind, sy)

    def input_grad(self, dy, dx) -> None:
        """dy [M][N] bf16, rows on 16 bytes; dx [M][K] bf16 or fp32."""
        M, gpu = _fits(dy.shape[0], "rows"), self._gpu
        sdy = _chunked_rows(dy, "dy", M, self.N, gpu)
        sdx, kind = _rows_of(dx, "dx", M, self.K, gpu)
        codes, scales, _ = self._weights()
        _call(gpu, "pac_mx4_linear_dx", dy.data_ptr(), M, self.N, sdy, codes, scales, self.K, dx.data_ptr(), kind, sdx)


class BlockNorm:
    """The norms after and before a block with its gate and the residual scale (include/pac_norm.h).  Parameters are float32
    tensors that the caller owns; between calls they may be changed in place, and may be given other storage."""

    def __init__(self, d: int, layer: bool = False, eps: float = 1e-5, w_post=None, b_post=None, gate=None, res=None, w_pre=None,
                 b_pre=None):
        # in the order of the library's structure and of its gradients
        self.d, self.params = _fits(d, "d"), dict(w_post=w_post, b_post=b_post, gate=gate, res=res, w_pre=w_pre, b_pre=b_pre)
        self._shapes = {name: p.shape for name, p in self.params.items() if p is not None}
        for name, shape in self._shapes.items():
            lens = {"gate": (1, d), "res": (1,)}.get(name, (d,))
            if len(shape) != 1 or shape[0] not in lens:
                raise ValueError(f"{name}: {' or '.join(map(str, lens))} values")
        self.dev = next((p.device for p in self.params.values() if p is not None), None)
        self._gpu = None if self.dev is None else self.dev.index
        self._b = {dtype: pb.pac_block_norm(d, kind, int(layer), 0 if gate is None else gate.shape[0], eps) for dtype, kind in _KIND.items()}
        self._at = None
        self._structure(torch.float32)

    def _structure(self, dtype):
        """The library's structure for states of that type, with the parameters' addresses as they are now, looked at again where they
        are not what they were."""
        at = [None if p is None else p.data_ptr() for p in self.params.values()]
        if at != self._at:
            for name, p in self.params.items():
                if (p is None) != (name not in self._shapes):
                    raise ValueError(f"{name}: there or not as in the beginning")
                if p is not None and (p.dtype != torch.float32 or p.shape != self._shapes[name] or not p.is_contiguous() or p.device != self.dev
                                      or self.dev.type != "cuda"):
                    raise ValueError(f"{name}: float32, dense, of the length it had, on one GPU with the other parameters")
            for b in self._b.values():
                b.w_post, b.b_post, b.gate, b.res, b.w_pre, b.b_pre = at
            self._at = at
        return self._b[dtype]

    def _rows(self, x, *others):
        """(rows, GPU) of states."""
        shape, dtype, gpu = x.shape, x.dtype, x.get_device()
        if len(shape) != 2 or shape[1] != self.d or dtype not in _KIND or gpu < 0 or not x.is_contiguous() or self._gpu not in (gpu, None):
            raise ValueError(f"states: dense, bfloat16 or float32, [rows][{self.d}], on the parameters' device")
        for t in others:
            if t is not None and (t.shape != shape or t.dtype is not dtype or t.get_device() != gpu or not t.is_contiguous()):
                raise ValueError(f"states: dense, [rows][{self.d}], of one type, on one device")
        return shape[0], gpu

    def forward(self, x, o=None, y=None, n=None) -> None:
        """y and n of x and a block's output o (None: no block yet), into the buffers given."""
        rows, gpu = self._rows(x, o, y, n)
        _call(gpu, "pac_block_norm_forward", self._structure(x.dtype), rows, x.data_ptr(), _ptr(o), _ptr(y), _ptr(n))

    def backward(self, x, o, dy, dn, dx=None, do=None, dparams=None) -> None:
        """Gradients, given dy (None: zero) and dn (None without w_pre), into the buffers given; dparams: {name: float32 tensor like
        the parameter} for those that are wanted."""
        rows, gpu = self._rows(x, o, dy, dn, dx, do)
        b, grads, ws, need = self._structure(x.dtype), [None] * 6, None, 0
        if dparams:
            dev = x.device
            for name, g in dparams.items():
                if g.shape != self._shapes.get(name) or g.dtype is not torch.float32 or g.device != dev or not g.is_contiguous():
                    raise ValueError(f"d{name}: like the parameter of that name")
            grads = [_ptr(dparams.get(name)) for name in self.params]
            need = _lib().pac_block_norm_workspace_bytes(b, rows)
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)  # for this call, on this stream
        _call(gpu, "pac_block_norm_backward", b, rows, x.data_ptr(), _ptr(o), _ptr(dy), _ptr(dn), _ptr(dx), _ptr(do), *grads, _ptr(ws), need)


def _head_rows(t, name: str, rows: int, cols: int, gpu: int) -> int:
    """The row stride of a bf16 matrix of heads."""
    if t.dtype != torch.bfloat16 or t.get_device() != gpu or t.shape != (rows, cols):
        raise ValueError(f"{name}: bfloat16, ({rows}, {cols}), on GPU {gpu} is wanted, not {t.dtype}, {tuple(t.shape)}, on {t.device}")
    stride = t.stride()
    if stride[1] != 1 and cols > 1:
        raise ValueError(f"{name}: neighbouring columns are wanted")
    return stride[0] if rows > 1 else cols


def _scale(scale, d: int) -> float:
    return d ** -0.5 if scale is None else float(scale)


def packed_offsets(lens, device="cuda:0"):
    """Where sequences of those lengths begin and end in packed rows: int32 [batch + 1]."""
    at = [0]
    for n in lens:
        if n < 0:
            raise ValueError(f"lens: {n} rows")
        at.append(at[-1] + int(n))
    _fits(at[-1], "rows")
    return torch.tensor(at, dtype=torch.int32, device=device)


class Attention:
    """Attention over sequences packed one after the other, and its gradients (include/pac_attn.h).  q and o are [rows][heads d], k and v
    [rows][kv_heads d], bf16, rows on 16 bytes and any multiple of 8 apart (q, k and v may be columns of one matrix); offsets as
    packed_offsets makes them.  lse is float32 [heads][rows], what the way back needs besides o.  scale: 1 / sqrt(d) where none is given."""

    def __init__(self, heads: int, d: int, kv_heads: int | None = None, causal: bool = False, scale: float | None = None):
        kv_heads = heads if kv_heads is None else kv_heads
        self._a = pb.pac_attn(_fits(heads, "heads"), _fits(kv_heads, "kv_heads"), _fits(d, "d"), int(causal), _scale(scale, d) if d > 0 else 1.0)
        if pb.pac_attn_workspace_bytes(self._a, 0, 0) < 0:
            raise ValueError("heads: a multiple of kv_heads, 1..4096; d: a multiple of 8, 8..128; scale: positive, up to 2.35e38")
        self.heads, self.kv_heads, self.d = heads, kv_heads, d

    def _rows(self, q, offsets):
        """(batch, rows, GPU)"""
        gpu = q.get_device()
        if gpu < 0 or q.dim() != 2 or offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.shape[0] < 1 or offsets.get_device() != gpu \
                or not offsets.is_contiguous():
            raise ValueError("q: a matrix on a GPU; offsets: int32, dense, [batch + 1], beside it")
        return offsets.shape[0] - 1, _fits(q.shape[0], "rows"), gpu

    def _lse(self, lse, rows, gpu):
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != (self.heads, rows) or lse.get_device() != gpu or not lse.is_contiguous()):
            raise ValueError(f"lse: dense float32, ({self.heads}, {rows}), on GPU {gpu} is wanted")
        return _ptr(lse)

    def _matrix(self, t, name, cols, rows, gpu):
        return t.data_ptr(), _head_rows(t, name, rows, cols, gpu)

    def forward(self, q, k, v, offsets, o, lse=None) -> None:
        """o, and lse where it is given, of the rows that sequences have; others are left as they are."""
        batch, rows, gpu = self._rows(q, offsets)
        qc, kc, m = self.heads * self.d, self.kv_heads * self.d, self._matrix
        _call(gpu, "pac_attn_forward", self._a, offsets.data_ptr(), batch, rows, *m(q, "q", qc, rows, gpu), *m(k, "k", kc, rows, gpu),
              *m(v, "v", kc, rows, gpu), *m(o, "o", qc, rows, gpu), self._lse(lse, rows, gpu))

    def backward(self, q, k, v, offsets, o, lse, do, dq, dk, dv) -> None:
        """Gradients of q, k and v, given that of o, into the buffers given; o and lse as forward wrote them."""
        batch, rows, gpu = self._rows(q, offsets)
        qc, kc, m = self.heads * self.d, self.kv_heads * self.d, self._matrix
        if lse is None:
            raise ValueError("lse: what forward wrote")
        need = pb.pac_attn_backward_bytes(self._a, batch, rows)
        if need < 0:
            raise ValueError("rows: too many of them by heads")
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)  # for this call, on this stream
        _call(gpu, "pac_attn_backward", self._a, offsets.data_ptr(), batch, rows, *m(q, "q", qc, rows, gpu), *m(k, "k", kc, rows, gpu),
              *m(v, "v", kc, rows, gpu), *m(o, "o", qc, rows, gpu), self._lse(lse, rows, gpu), *m(do, "do", qc, rows, gpu),
              *m(dq, "dq", qc, rows, gpu), *m(dk, "dk", kc, rows, gpu), *m(dv, "dv", kc, rows, gpu), ws.data_ptr(), need)


class Kv4Cache:
    """Keys and values of one layer in 4 bits, in pages (include/pac_kv4.h).  Slot s is place s % page of page s / page; which pages a
    sequence has is the caller's: a row of a table."""

    def __init__(self, pages: int, page: int, kv_heads: int, d: int, device="cuda:0"):
        self._c = pb.pac_kv4(None, _fits(pages, "pages"), _fits(page, "page"), _fits(kv_heads, "kv_heads"), _fits(d, "d"))
        need = pb.pac_kv4_bytes(self._c)
        if need < 0:
            raise ValueError("pages: 0..2^31 - 1; page: a power of two, 8..65536; kv_heads: 1..4096; d: a multiple of 8, 8..128")
        if torch.device(device).type != "cuda":
            raise ValueError("device: a GPU")
        self.pages, self.page, self.kv_heads, self.d = pages, page, kv_heads, d
        self.data = torch.zeros(need, dtype=torch.uint8, device=device)
        self._gpu = self.data.get_device()
        self._room = None, 0  # sizes of the last attend, and bytes of workspace for them

    def _at(self):
        self._c.at = self.data.data_ptr()
        return self._c

    def _io(self, slots, k, v):
        rows, cols, gpu = _fits(k.shape[0], "rows"), self.kv_heads * self.d, self._gpu
        (sk, kind), (sv, other) = _rows_of(k, "k", rows, cols, gpu), _rows_of(v, "v", rows, cols, gpu)
        if kind != other:
            raise ValueError("k and v: of one type")
        if slots.dtype != torch.int64 or slots.shape != (rows,) or slots.get_device() != gpu or not slots.is_contiguous():
            raise ValueError(f"slots: dense int64, ({rows},), on GPU {gpu} is wanted")
        return rows, slots.data_ptr(), k.data_ptr(), sk, v.data_ptr(), sv, kind

    def write(self, k, v, slots) -> None:
        """Row r of k and v [rows][kv_heads d] (bf16 or fp32, any row stride), quantised, into slot slots[r]; rows with a slot outside the
        cache are left out.  No slot may be named twice."""
        _call(self._gpu, "pac_kv4_write", self._at(), *self._io(slots, k, v))

    def read(self, slots, k, v) -> None:
        """The values that slots hold, into rows of k and v; rows with a slot outside the cache are left as they are."""
        _call(self._gpu, "pac_kv4_read", self._at(), *self._io(slots, k, v))

    def attend(self, q, table, lens, o, scale: float | None = None) -> None:
        """o [batch][heads d] of one query a sequence, q alike (bf16, rows on 16 bytes), over the first lens[b] (int32) tokens in the pages of
        row b of table (int32 [batch][pages at most]; a page outside the cache counts as masked).  No tokens: zeros."""
        batch, gpu, d = _fits(q.shape[0], "sequences"), self._gpu, self.d
        if q.dim() != 2 or q.shape[1] < d or q.shape[1] % d:
            raise ValueError(f"q: [sequences][heads {d}]")
        heads = q.shape[1] // d
        sq, so = _head_rows(q, "q", batch, heads * d, gpu), _head_rows(o, "o", batch, heads * d, gpu)
        if lens.dtype != torch.int32 or lens.shape != (batch,) or lens.get_device() != gpu or not lens.is_contiguous():
            raise ValueError(f"lens: dense int32, ({batch},), on GPU {gpu} is wanted")
        if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != batch or table.get_device() != gpu or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError(f"table: int32, ({batch}, pages), neighbouring columns, on GPU {gpu} is wanted")
        pages = _fits(table.shape[1], "pages of a sequence")
        c, st = self._at(), table.stride(0) if batch > 1 else pages
        sizes, need = self._room
        if sizes != (heads, batch, pages):
            need = max(_lib().pac_kv4_attend_bytes(c, heads, batch, pages), 0)
            self._room = (heads, batch, pages), need
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)  # for this call, on this stream
        _call(gpu, "pac_kv4_attend", c, heads, _scale(scale, d), batch, table.data_ptr(), pages, st, lens.data_ptr(), q.data_ptr(), sq, o.data_ptr(), so,
              ws.data_ptr(), need)
