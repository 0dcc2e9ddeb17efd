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


# ---- blocks of the frozen backbone (include/pac_mx4.h, include/pac_norm.h) ------------------------------------------
def _kind(t) -> int:
    if t.dtype == torch.bfloat16:
        return pb.PAC_BF16
    if t.dtype == torch.float32:
        return pb.PAC_F32
    raise ValueError(f"bfloat16 or float32 is wanted, not {t.dtype}")


def _matrix(t, name: str, shape=None, dtype=None, device=None):
    """The row stride of a device matrix whose columns are neighbours (the launch takes addresses alone, so what they stand
    for is checked here)."""
    have, dev = t.shape, t.device
    if len(have) != 2 or dev.type != "cuda" or (device is not None and dev != device):
        raise ValueError(f"{name}: a matrix on the device is wanted")
    if shape is not None and have != shape:
        raise ValueError(f"{name}: shape {shape} is wanted, not {tuple(have)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: {dtype} is wanted, not {t.dtype}")
    row, col = t.stride()
    if col != 1 and have[1] > 1:
        raise ValueError(f"{name}: neighbouring columns are wanted")
    return row if have[0] > 1 else max(row, have[1])


def _stored(codes, scales, cols: int, rows=None, device=None):
    rows = codes.shape[0] if rows is None else rows
    for t, pitch, name in ((codes, pb.pac_mx4_code_pitch(cols), "codes"), (scales, pb.pac_mx4_scale_pitch(cols), "scales")):
        _matrix(t, name, (rows, pitch), torch.uint8, device)
        if not t.is_contiguous():
            raise ValueError(f"{name}: a dense matrix is wanted")


def _padded_stride(t, name: str, cols: int, device):
    """The row stride of a bf16 matrix that is read in 16-byte pieces, in the last row too."""
    stride = _matrix(t, name, (t.shape[0], cols), torch.bfloat16, device)
    pad = (cols + 7) // 8 * 8
    if t.shape[0] == 1:
        stride = max(stride, pad) // 8 * 8
    if t.shape[0] and cols % 8:
        after = t.storage_offset() + (t.shape[0] - 1) * stride + pad
        if after * 2 > t.untyped_storage().nbytes():
            raise ValueError(f"{name}: rows are read up to a multiple of 8 columns, the last one too")
    return stride


def _launch(device, call, *args) -> None:
    """call(*args, the device's current stream), with that device current (switching costs more than looking)."""
    i = device.index
    if torch.cuda.current_device() == i:
        call(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            call(*args, torch._C._cuda_getCurrentRawStream(i))


def _ptr(t):
    return None if t is None else t.data_ptr()


def mx4_empty(rows: int, cols: int, device="cuda:0"):
    """Buffers for a matrix in the stored form: (codes, scales)."""
    return (torch.empty(rows, pb.pac_mx4_code_pitch(cols), dtype=torch.uint8, device=device),
            torch.empty(rows, pb.pac_mx4_scale_pitch(cols), dtype=torch.uint8, device=device))


def mx4_quantize(x, codes, scales) -> None:
    """x (bf16 or fp32, any row stride) into the stored form."""
    stride = _matrix(x, "x")
    _stored(codes, scales, x.shape[1], x.shape[0], x.device)
    _launch(x.device, pb.pac_mx4_quantize, x.data_ptr(), _kind(x), x.shape[0], x.shape[1], stride, codes.data_ptr(), scales.data_ptr())


def mx4_dequantize(codes, scales, out) -> None:
    """The values a stored matrix stands for, into out (bf16 or fp32, both exact)."""
    stride = _matrix(out, "out")
    _stored(codes, scales, out.shape[1], out.shape[0], out.device)
    _launch(out.device, pb.pac_mx4_dequantize, codes.data_ptr(), scales.data_ptr(), out.shape[0], out.shape[1], out.data_ptr(), _kind(out),
            stride)


class Mx4Linear:
    """A frozen linear layer with weights in the stored form: y = act(x W^T + bias), and dx = dy W on the way back."""

    def __init__(self, codes, scales, K: int, bias=None):
        _stored(codes, scales, K)
        self.codes, self.scales, self.bias = codes, scales, bias
        self.N, self.K, self.dev = codes.shape[0], K, codes.device
        if bias is not None and (bias.shape != (self.N,) or bias.dtype != torch.float32 or bias.device != self.dev or not bias.is_contiguous()):
            raise ValueError("bias: float32, one value an output, on the weights' device")
        self._w = (codes.data_ptr(), scales.data_ptr())
        self._b = None if bias is None else bias.data_ptr()

    @classmethod
    def from_weights(cls, w, bias=None):
        """w [N][K], bf16 or fp32, is quantised; the layer keeps the stored form only."""
        codes, scales = mx4_empty(w.shape[0], w.shape[1], w.device)
        mx4_quantize(w, codes, scales)
        return cls(codes, scales, w.shape[1], bias)

    def forward(self, x, y, gelu: bool = False, x4: bool = False) -> None:
        """x [M][K] bf16, rows on 16 bytes; y [M][N] bf16 or fp32.  x4: x is quantised too, and the product runs on 4-bit operands."""
        M = x.shape[0]
        sy = _matrix(y, "y", (M, self.N), None, self.dev)
        act = pb.PAC_MX4_ACT_GELU if gelu else pb.PAC_MX4_ACT_NONE
        if x4:
            sx = _matrix(x, "x", (M, self.K), None, self.dev)
            # x in the stored form lives for this call, on this stream: codes (whole multiples of 128 bytes), then scales
            c = M * self.codes.shape[1]
            buf = torch.empty(c + M * self.scales.shape[1], dtype=torch.uint8, device=self.dev)
            c, s = buf.data_ptr(), buf.data_ptr() + c
            _launch(self.dev, pb.pac_mx4_quantize, x.data_ptr(), _kind(x), M, self.K, sx, c, s)
            _launch(self.dev, pb.pac_mx4_linear_x4, c, s, M, self.K, *self._w, self.N, self._b, act, y.data_ptr(), _kind(y), sy)
        else:
            sx = _padded_stride(x, "x", self.K, self.dev)
            _launch(self.dev, pb.pac_mx4_linear, x.data_ptr(), M, self.K, sx, *self._w, self.N, self._b, act, y.data_ptr(), _kind(y), sy)

    def input_grad(self, dy, dx) -> None:
        """dy [M][N] bf16, rows on 16 bytes; dx [M][K] bf16 or fp32."""
        M = dy.shape[0]
        sdy = _padded_stride(dy, "dy", self.N, self.dev)
        sdx = _matrix(dx, "dx", (M, self.K), None, self.dev)
        _launch(self.dev, pb.pac_mx4_linear_dx, dy.data_ptr(), M, self.N, sdy, *self._w, self.K, dx.data_ptr(), _kind(dx), sdx)


class BlockNorm:
    """The norms after and before a block with its gate and the residual scale (include/pac_norm.h).  Parameters are float32
    tensors that the caller owns and may change in place."""

    def __init__(self, d: int, layer: bool = False, eps: float = 1e-5, w_post=None, b_post=None, gate=None, res=None, w_pre=None,
                 b_pre=None):
        self.d, self.params = d, dict(w_post=w_post, b_post=b_post, gate=gate, res=res, w_pre=w_pre, b_pre=b_pre)
        self.dev = None
        for name, p in self.params.items():
            if p is None:
                continue
            lens = {"gate": (1, d), "res": (1,)}.get(name, (d,))
            if p.dtype != torch.float32 or p.dim() != 1 or p.shape[0] not in lens or not p.is_contiguous() or p.device.type != "cuda":
                raise ValueError(f"{name}: float32 on the device, {' or '.join(map(str, lens))} values")
            if self.dev not in (None, p.device):
                raise ValueError(f"{name}: on another device than the parameters before it")
            self.dev = p.device
        self._b = {kind: pb.pac_block_norm(d, kind, int(layer), 0 if gate is None else gate.shape[0], eps,
                                           *(_ptr(self.params[k]) for k in ("w_post", "b_post", "gate", "res", "w_pre", "b_pre")))
                   for kind in (pb.PAC_BF16, pb.PAC_F32)}

    def _rows(self, x, *others):
        shape, dtype, dev = x.shape, x.dtype, x.device
        if len(shape) != 2 or shape[1] != self.d or dev.type != "cuda" or not x.is_contiguous() or self.dev not in (None, dev):
            raise ValueError(f"states: dense, [rows][{self.d}], on the parameters' device")
        for t in others:
            if t is not None and (t.shape != shape or t.dtype != dtype or t.device != dev or not t.is_contiguous()):
                raise ValueError(f"states: dense, [rows][{self.d}], of one type, on one device")
        return shape[0]

    def forward(self, x, o=None, y=None, n=None) -> None:
        rows = self._rows(x, o, y, n)
        _launch(x.device, pb.pac_block_norm_forward, self._b[_kind(x)], rows, x.data_ptr(), _ptr(o), _ptr(y), _ptr(n))

    def backward(self, x, o, dy, dn, dx=None, do=None, dparams=None) -> None:
        """Gradients; dparams: {name: float32 tensor like the parameter} for those that are wanted."""
        rows = self._rows(x, o, dy, dn, dx, do)
        dparams = dparams or {}
        for name, g in dparams.items():
            p = self.params.get(name)
            if p is None or g.shape != p.shape or g.dtype != torch.float32 or g.device != p.device or not g.is_contiguous():
                raise ValueError(f"d{name}: like the parameter of that name")
        b = self._b[_kind(x)]
        need = pb.pac_block_norm_workspace_bytes(b, rows) if dparams else 0
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        _launch(x.device, pb.pac_block_norm_backward, b, rows, x.data_ptr(), _ptr(o), _ptr(dy), _ptr(dn), _ptr(dx), _ptr(do),
                *(_ptr(dparams.get(k)) for k in ("w_post", "b_post", "gate", "res", "w_pre", "b_pre")), _ptr(ws), need)
