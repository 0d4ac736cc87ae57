"""Python binding of libqmlp, the MI355X (gfx950) W4/W2-GateUp decode-MLP library.

Argument marshalling only: every step of the hot path runs in the HIP
kernels behind ``include/qmlp.h``.  PyTorch provides device memory and the
current stream.  The module fails loudly if the built library is missing;
there is no CPU fallback.

Functions keep the names of the C entry points:

* ``pack_w2`` / ``pack_w4``       -- quantize fp32 weights to packed 2/4-bit (Sec. 4.1, Sec. 7)
* ``gateup_w2_lora``              -- h = SiLU(W2g x + s B_g A_g x) * (W2u x + s B_u A_u x)
* ``down_w4``                     -- y = W4down h
* ``forward``                     -- the whole block x -> y
* ``forward_layers``              -- L independent blocks, y_l = block_l(x_l)
* ``forward_stack``               -- L blocks on a residual stream, x_{l+1} = x_l + block_l(RMSNorm(x_l))
* ``linear_lora``                 -- a linear with adapters of many requests, y[m] = W x[m] + s_a B_a (A_a x[m])
* ``moe_route`` / ``moe_layer``   -- a router's top-k choice and weights; a whole MoE layer for a few tokens
* ``kv_plan`` / ``qk_norm_rope`` / ``kv_read`` / ``kv_attention`` -- a step's pages and slots, head norms and rotation with
  the write into a 4-bit cache of keys and values, what the cache holds, causal attention over it
* ``unpack`` / ``dequant``        -- inspection of a packed matrix (not timed)
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# QMLP_LIB_PATH: another build of the same sources (the host-sanitized one
# of build.py --host-sanitize); by default the library next to this file
LIB_PATH = os.environ.get("QMLP_LIB_PATH") or os.path.join(_HERE, "libqmlp.so")

F16, BF16 = 0, 1
_STATUS = {0: "QMLP_OK", 1: "QMLP_ERR_NULL", 2: "QMLP_ERR_SHAPE", 3: "QMLP_ERR_ALIGN",
           4: "QMLP_ERR_UNSUPPORTED", 5: "QMLP_ERR_WORKSPACE", 6: "QMLP_ERR_HIP"}


class QmlpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%s)" % (where, _STATUS.get(status, status),
                                          _lib().qmlp_status_string(status).decode()))


class QWeightC(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("n_out", ctypes.c_int32), ("k_in", ctypes.c_int32),
                ("group", ctypes.c_int32), ("codes", ctypes.c_void_p), ("meta", ctypes.c_void_p)]


class MlpC(ctypes.Structure):
    _fields_ = [("gate", QWeightC), ("up", QWeightC), ("down", QWeightC),
                ("A_gate", ctypes.c_void_p), ("B_gate", ctypes.c_void_p),
                ("A_up", ctypes.c_void_p), ("B_up", ctypes.c_void_p),
                ("rank", ctypes.c_int32), ("lora_scale", ctypes.c_float)]


class AdaptersC(ctypes.Structure):
    _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("count", ctypes.c_int32), ("rank", ctypes.c_int32)]


class MoeC(ctypes.Structure):
    _fields_ = [("router", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("experts", ctypes.c_int32),
                ("topk", ctypes.c_int32), ("score", ctypes.c_int32), ("mlp", MlpC)]


class KVCacheC(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page", ctypes.c_int32)]


class HeadsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v")] + [(n, ctypes.c_int64) for n in ("ldq", "ldk", "ldv")] + \
               [(n, ctypes.c_void_p) for n in ("q_out", "k_out")] + [(n, ctypes.c_int64) for n in ("ldq_out", "ldk_out")] + \
               [(n, ctypes.c_void_p) for n in ("q_weight", "k_weight", "positions", "inv_freq", "slots")] + \
               [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "head_dim", "rot", "pairs")] + \
               [(n, ctypes.c_float) for n in ("eps", "mul")]


class PlanC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("lens", "new_tokens", "table", "free_pages", "n_free", "slots", "positions",
                                               "starts", "lens_out", "n_free_out", "short_out")] + \
               [(n, ctypes.c_int32) for n in ("B", "page", "W", "N", "tokens")]


class AttentionC(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("y", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("ldy", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("table", "lens", "starts", "sinks", "ws")] + [("ws_bytes", ctypes.c_size_t)] + \
               [(n, ctypes.c_int32) for n in ("T", "heads", "B", "W", "max_new", "window")] + [("scale", ctypes.c_float)]


# The same structures as packed bytes: to fill one of ctypes' own costs about 1.5 us a call, to pass its members one by one
# 4 us, this 0.3 us (their members are ordered so that nothing is padded between them).
_HEADS, _PLAN, _ATTENTION = struct.Struct("@3P3q2P2q5P5i2f"), struct.Struct("@11P5i"), struct.Struct("@2P2q5PN6if")


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libqmlp.so is not built (run __graft_entry__.build()); "
                              "there is no fallback path: %s" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        P, I, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        pq = ctypes.POINTER(QWeightC)
        pm = ctypes.POINTER(MlpC)
        po = ctypes.POINTER(MoeC)
        pa, L = ctypes.POINTER(AdaptersC), ctypes.c_int64
        pc = ctypes.POINTER(KVCacheC)
        sig = {
            "qmlp_codes_bytes": (Z, [I, I, I]),
            "qmlp_meta_bytes": (Z, [I, I, I]),
            "qmlp_workspace_bytes": (Z, [pm, I, I]),
            "qmlp_pack_w2": (I, [P, I, I, I, pq, P, P]),
            "qmlp_pack_w3": (I, [P, I, I, I, pq, P, P]),
            "qmlp_pack_w4": (I, [P, I, I, I, pq, P, P]),
            "qmlp_gateup_w2_lora": (I, [pm, P, I, I, P, P, Z, P]),
            "qmlp_down_w4": (I, [pq, P, I, I, P, P]),
            "qmlp_forward": (I, [pm, P, I, I, P, P, Z, P]),
            "qmlp_unpack": (I, [pq, P, P, P, P]),
            "qmlp_dequant": (I, [pq, P, P]),
            "qmlp_forward_launches": (I, [pm, I, I]),
            "qmlp_stack_workspace_bytes": (Z, [pm, I, I, I]),
            "qmlp_forward_stack": (I, [pm, I, P, I, I, P, P, P, Z, P]),
            "qmlp_stack_launches": (I, [pm, I, I, I]),
            "qmlp_stack_error_offset": (Z, [pm, I, I, I]),
            "qmlp_moe_lanes": (I, [I, I, I, I, I, I, I, ctypes.POINTER(I), ctypes.POINTER(I)]),
            "qmlp_layers_workspace_bytes": (Z, [pm, I, I, I]),
            "qmlp_forward_layers": (I, [pm, I, P, I, I, P, P, Z, P]),
            "qmlp_layers_launches": (I, [pm, I, I, I]),
            "qmlp_batch_workspace_bytes": (Z, [pm, I, I, I]),
            "qmlp_linear_batch": (I, [ctypes.POINTER(QWeightC), I, P, I, I, P, P]),
            "qmlp_moe_workspace_bytes": (Z, [pm, I, I, I, I]),
            "qmlp_forward_moe": (I, [pm, I, P, I, I, P, P, I, P, P, Z, P]),
            "qmlp_forward_batch": (I, [pm, I, P, I, I, P, P, Z, P]),
            "qmlp_status_string": (ctypes.c_char_p, [I]),
            "qmlp_probe_stream_read": (I, [P, Z, P, I, I, P]),
            "qmlp_forward_noalloc": (I, [pm, P, I, I, P, P]),
            "qmlp_layers_path": (I, [pm, I, I, I]),
            "qmlp_noalloc_scratch_bytes": (Z, []),
            "qmlp_linear_lora_workspace_bytes": (Z, [pq, pa, I, I]),
            "qmlp_moe_route_workspace_bytes": (Z, [I, I]),
            "qmlp_moe_route": (I, [P, P, P, I, I, I, I, I, I, P, P, P, Z, P]),
            "qmlp_moe_layer_workspace_bytes": (Z, [po, I, I]),
            "qmlp_moe_layer": (I, [po, P, I, I, P, P, Z, P]),
            "qmlp_linear_lora": (I, [pq, pa, P, P, L, I, I, P, L, P, Z, P]),
            "qmlp_kv_cache_bytes": (Z, [I, I, I, I]),
            "qmlp_kv_plan": (I, [ctypes.c_char_p, P]),
            "qmlp_qk_norm_rope": (I, [ctypes.c_char_p, I, I, P, P]),
            "qmlp_kv_read": (I, [P, P, I, I, P, P, P]),
            "qmlp_kv_attention_workspace_bytes": (Z, [pc, I, I]),
            "qmlp_kv_attention": (I, [P, ctypes.c_char_p, I, P]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


def library():
    """The loaded ctypes library (raises if it is not built)."""
    return _lib()


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    # (the handle alone: torch.cuda.current_stream() makes an object of it, 2.7 us a call here against 0.3)
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _check(status: int, where: str):
    if status != 0:
        raise QmlpError(status, where)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return F16
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("activations must be float16 or bfloat16, got %s" % t.dtype)


def codes_bytes(bits: int, n_out: int, k_in: int) -> int:
    return int(_lib().qmlp_codes_bytes(bits, n_out, k_in))


def meta_bytes(n_out: int, k_in: int, group: int) -> int:
    return int(_lib().qmlp_meta_bytes(n_out, k_in, group))


class QWeight:
    """A packed quantized matrix: device tensors ``codes`` and ``meta`` plus its C view."""

    def __init__(self, bits, n_out, k_in, group, codes, meta, status=None):
        self.bits, self.n_out, self.k_in, self.group = bits, n_out, k_in, group
        self.codes = codes          # uint8 device tensor, codes_bytes() long
        self.meta = meta            # uint8 device tensor, meta_bytes() long
        self.status = status        # int32 device tensor set by the packer (bit 0: invalid group)

    def c(self) -> QWeightC:
        return QWeightC(self.bits, self.n_out, self.k_in, self.group,
                        self.codes.data_ptr(), self.meta.data_ptr())

    def invalid_groups(self) -> bool:
        """True if the packer flagged a non-finite weight or an overflowing scale (syncs)."""
        return bool(self.status is not None and int(self.status.item()) & 1)

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.meta.numel()


def _pack(bits: int, W: torch.Tensor, group: int) -> QWeight:
    if W.dtype != torch.float32 or not W.is_cuda or W.dim() != 2:
        raise TypeError("W must be a 2-D float32 CUDA tensor")
    W = W.contiguous()
    n, k = W.shape
    cb, mb = codes_bytes(bits, n, k), meta_bytes(n, k, group)
    if cb == 0 or mb == 0:
        raise QmlpError(2, "pack_w%d" % bits)
    codes = torch.empty(cb, dtype=torch.uint8, device=W.device)
    meta = torch.empty(mb, dtype=torch.uint8, device=W.device)
    status = torch.zeros(1, dtype=torch.int32, device=W.device)
    qw = QWeightC(0, 0, 0, 0, codes.data_ptr(), meta.data_ptr())
    fn = {2: _lib().qmlp_pack_w2, 3: _lib().qmlp_pack_w3, 4: _lib().qmlp_pack_w4}[bits]
    _check(fn(_ptr(W), n, k, group, ctypes.byref(qw), _ptr(status), _stream()), "pack_w%d" % bits)
    return QWeight(qw.bits, qw.n_out, qw.k_in, qw.group, codes, meta, status)


def pack_w2(W: torch.Tensor, group: int) -> QWeight:
    """Quantize fp32 W [n][k] (device) to 2-bit codes + fp16 scale/zero per group."""
    return _pack(2, W, group)


def pack_w3(W: torch.Tensor, group: int) -> QWeight:
    """Quantize fp32 W [n][k] (device) to 3-bit codes (two-plane layout) + fp16 scale/zero."""
    return _pack(3, W, group)


def pack_w4(W: torch.Tensor, group: int) -> QWeight:
    """Quantize fp32 W [n][k] (device) to 4-bit codes + fp16 scale/zero per group."""
    return _pack(4, W, group)


class MLP:
    """One W4/W2-GateUp block with Recover-LoRA adapters (device tensors); the
    decode path also takes the uniform-W4 / uniform-W2 comparison widths and
    group 32 (see qmlp_mlp in include/qmlp.h)."""

    def __init__(self, gate: QWeight, up: QWeight, down: QWeight, A_gate=None, B_gate=None,
                 A_up=None, B_up=None, lora_scale: float = 1.0):
        self.gate, self.up, self.down = gate, up, down
        self.A_gate, self.B_gate, self.A_up, self.B_up = A_gate, B_gate, A_up, B_up
        self.rank = 0 if A_gate is None else int(A_gate.shape[0])
        self.lora_scale = float(lora_scale)
        self._c = MlpC(gate.c(), up.c(), down.c(), _ptr(A_gate), _ptr(B_gate), _ptr(A_up),
                       _ptr(B_up), self.rank, self.lora_scale)

    @property
    def d(self):
        return self.gate.k_in

    @property
    def f(self):
        return self.gate.n_out

    def c(self) -> MlpC:
        return self._c

    def with_lora_scale(self, lora_scale: float) -> "MLP":
        return MLP(self.gate, self.up, self.down, self.A_gate, self.B_gate, self.A_up, self.B_up,
                   lora_scale)


def workspace_bytes(mlp: MLP, M: int, dtype=torch.float16) -> int:
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_workspace_bytes(ctypes.byref(mlp.c()), M, code))


def forward_launches(mlp: MLP, M: int, dtype=torch.float16) -> int:
    """Kernels qmlp_forward launches for this block at M tokens (1 = fused layer kernel)."""
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_forward_launches(ctypes.byref(mlp.c()), M, code))


def workspace(mlp: MLP, M: int, dtype=torch.float16, device="cuda") -> torch.Tensor:
    """A zeroed workspace (it must start at zero; zero it again before it
    serves a block of another shape or after an error bit)."""
    n = workspace_bytes(mlp, M, dtype)
    return torch.zeros(max(n, 1024), dtype=torch.uint8, device=device)


def workspace_errors(ws: torch.Tensor) -> int:
    """Sticky error bits of a workspace's control block (syncs)."""
    return int(ws[640:644].view(torch.int32).item())


def gateup_w2_lora(mlp: MLP, x: torch.Tensor, h: torch.Tensor | None = None,
                   ws: torch.Tensor | None = None) -> torch.Tensor:
    M = x.shape[0]
    if h is None:
        h = torch.empty((M, mlp.f), dtype=x.dtype, device=x.device)
    if ws is None:
        ws = workspace(mlp, M, x.dtype, x.device)
    _check(_lib().qmlp_gateup_w2_lora(ctypes.byref(mlp.c()), _ptr(x), M, _dtype_code(x), _ptr(h),
                                      _ptr(ws), ws.numel(), _stream()), "gateup_w2_lora")
    return h


def down_w4(down: QWeight, h: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
    M = h.shape[0]
    if y is None:
        y = torch.empty((M, down.n_out), dtype=h.dtype, device=h.device)
    qc = down.c()
    _check(_lib().qmlp_down_w4(ctypes.byref(qc), _ptr(h), M, _dtype_code(h), _ptr(y), _stream()),
           "down_w4")
    return y


def forward(mlp: MLP, x: torch.Tensor, y: torch.Tensor | None = None,
            ws: torch.Tensor | None = None) -> torch.Tensor:
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, mlp.d), dtype=x.dtype, device=x.device)
    if ws is None:
        ws = workspace(mlp, M, x.dtype, x.device)
    _check(_lib().qmlp_forward(ctypes.byref(mlp.c()), _ptr(x), M, _dtype_code(x), _ptr(y),
                               _ptr(ws), ws.numel(), _stream()), "forward")
    return y


def forward_noalloc(mlp: MLP, x: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
    """The whole block x -> y with the library's own per-GPU scratch array as
    workspace (qmlp_forward_noalloc): nothing is allocated by the call."""
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, mlp.d), dtype=x.dtype, device=x.device)
    c = mlp.c()
    _check(_lib().qmlp_forward_noalloc(ctypes.byref(c), _ptr(x), M, _dtype_code(x), _ptr(y), _stream()),
           "qmlp_forward_noalloc")
    return y


def noalloc_scratch_bytes() -> int:
    return int(_lib().qmlp_noalloc_scratch_bytes())


def unpack(w: QWeight):
    """(codes uint8 [n][k], scale bits int16 [n][k/g], zero bits int16 [n][k/g]) on the device."""
    dev = w.codes.device
    codes = torch.empty((w.n_out, w.k_in), dtype=torch.uint8, device=dev)
    scales = torch.empty((w.n_out, w.k_in // w.group), dtype=torch.int16, device=dev)
    zeros = torch.empty_like(scales)
    qc = w.c()
    _check(_lib().qmlp_unpack(ctypes.byref(qc), _ptr(codes), _ptr(scales), _ptr(zeros), _stream()),
           "unpack")
    return codes, scales, zeros


def dequant(w: QWeight) -> torch.Tensor:
    """The dequantized weight as float16 [n][k] (one RNE rounding of scale*(q-zero))."""
    out = torch.empty((w.n_out, w.k_in), dtype=torch.float16, device=w.codes.device)
    qc = w.c()
    _check(_lib().qmlp_dequant(ctypes.byref(qc), _ptr(out), _stream()), "dequant")
    return out


class Layers:
    """L blocks of one shape; holds the C descriptor array that the
    multi-block entry points take."""

    def __init__(self, mlps):
        self.mlps = list(mlps)
        self._arr = (MlpC * len(self.mlps))(*[m.c() for m in self.mlps])

    def __len__(self):
        return len(self.mlps)

    def c(self):
        return self._arr


class Stack(Layers):
    """L blocks of one shape on a residual stream (x_{l+1} = x_l + y_l,
    y_l = block_l(RMSNorm(x_l)))."""


def layers_workspace_bytes(layers: Layers, M: int, dtype=torch.float16) -> int:
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_layers_workspace_bytes(layers.c(), len(layers), M, code))


LAYERS_PATHS = {0: "rejected", 1: "streamed", 2: "batched", 3: "per-block", 4: "mfma"}


def layers_path(layers: Layers, M: int, dtype=torch.float16) -> str:
    """The path qmlp_forward_layers takes (qmlp_layers_path)."""
    code = F16 if dtype == torch.float16 else BF16
    return LAYERS_PATHS[int(_lib().qmlp_layers_path(layers.c(), len(layers), M, code))]


def layers_launches(layers: Layers, M: int, dtype=torch.float16) -> int:
    """Launches forward_layers makes (three per batch of up to 40 blocks on
    the streamed and batched paths, or those of one forward per block)."""
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_layers_launches(layers.c(), len(layers), M, code))


def layers_workspace(layers: Layers, M: int, dtype=torch.float16, device="cuda") -> torch.Tensor:
    """A zeroed workspace for forward_layers."""
    n = layers_workspace_bytes(layers, M, dtype)
    return torch.zeros(max(n, 1024), dtype=torch.uint8, device=device)


def forward_layers(layers: Layers, x: torch.Tensor, y: torch.Tensor | None = None,
                   ws: torch.Tensor | None = None) -> torch.Tensor:
    """y [L][M][d]: y_l = block_l(x_l) for x [L][M][d], every block on its own input."""
    L, M, d = x.shape
    if L != len(layers) or d != layers.mlps[0].d:
        raise ValueError("x must be [L][M][d] for the L blocks")
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = layers_workspace(layers, M, x.dtype, x.device)
    _check(_lib().qmlp_forward_layers(layers.c(), L, _ptr(x), M, _dtype_code(x), _ptr(y), _ptr(ws),
                                      ws.numel(), _stream()), "forward_layers")
    return y


def batch_workspace_bytes(layers: Layers, M: int, dtype=torch.float16) -> int:
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_batch_workspace_bytes(layers.c(), len(layers), M, code))


def batch_workspace(layers: Layers, M: int, dtype=torch.float16, device="cuda") -> torch.Tensor:
    """A zeroed workspace for forward_batch."""
    n = batch_workspace_bytes(layers, M, dtype)
    return torch.zeros(max(n, 1024), dtype=torch.uint8, device=device)


def forward_batch(layers: Layers, x: torch.Tensor, y: torch.Tensor | None = None,
                  ws: torch.Tensor | None = None) -> torch.Tensor:
    """forward_layers on the stand-alone kernels whatever the shape: LoRA-A,
    gate/up and down of every block of a batch of up to 40, three launches."""
    L, M, d = x.shape
    if L != len(layers) or d != layers.mlps[0].d:
        raise ValueError("x must be [L][M][d] for the L blocks")
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = batch_workspace(layers, M, x.dtype, x.device)
    _check(_lib().qmlp_forward_batch(layers.c(), L, _ptr(x), M, _dtype_code(x), _ptr(y), _ptr(ws),
                                     ws.numel(), _stream()), "forward_batch")
    return y


def linear_batch(ws, x: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
    """y [L][M][n] = W_l x_l for L quantized linears of one shape (QWeight list)
    and x [L][M][k] binary16: one launch."""
    L, M, k = x.shape
    if L != len(ws) or k != ws[0].k_in:
        raise ValueError("x must be [L][M][k] for the L linears")
    if y is None:
        y = torch.empty((L, M, ws[0].n_out), dtype=x.dtype, device=x.device)
    arr = (QWeightC * L)(*[w.c() for w in ws])
    _check(_lib().qmlp_linear_batch(arr, L, _ptr(x), M, _dtype_code(x), _ptr(y), _stream()),
           "linear_batch")
    return y


class Adapters:
    """Low-rank adapters of many requests over one linear: A [count][rank][k] and
    B [count][n][rank] in the activation type, scale float32 [count] or None (1.0),
    contiguous on one device.  Lower ranks are padded with zeros."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None):
        if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != B.shape[2]:
            raise ValueError("A must be [count][rank][k] and B [count][n][rank]")
        if A.dtype != B.dtype or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A and B must be contiguous and of one type")
        if scale is not None and (scale.dtype != torch.float32 or scale.shape != A.shape[:1] or not scale.is_contiguous()):
            raise ValueError("scale must be float32 [count]")
        _dtype_code(A)
        _one_device(A, B, scale)
        self.A, self.B, self.scale = A, B, scale
        self.count, self.rank = int(A.shape[0]), int(A.shape[1])
        self._c = AdaptersC(A.data_ptr(), B.data_ptr(), None if scale is None else scale.data_ptr(), self.count, self.rank)

    def c(self) -> AdaptersC:
        return self._c


def _one_device(*tensors):
    """The current device, which the kernels run on; a tensor elsewhere would fault there."""
    here = None
    for t in tensors:
        if t is None:
            continue
        if here is None and t.is_cuda:
            here = torch.cuda.current_device()
        if not t.is_cuda or t.get_device() != here:
            raise ValueError("every tensor must be on the current CUDA device")
    return here


def _addr(t):
    """An address as ctypes takes it where the argument's type is declared (an object of its own costs 0.1 us)."""
    return None if t is None else t.data_ptr()


def linear_lora_workspace_bytes(w: QWeight, adapters: Adapters | None, M: int, dtype=torch.float16) -> int:
    qc = w.c()
    return int(_lib().qmlp_linear_lora_workspace_bytes(ctypes.byref(qc), ctypes.byref(adapters.c()) if adapters else None,
                                                       M, F16 if dtype == torch.float16 else BF16))


def linear_lora_workspace(w: QWeight, adapters: Adapters | None, M: int, dtype=torch.float16,
                          device="cuda") -> torch.Tensor:
    """A workspace for linear_lora of up to this many rows (any contents)."""
    return torch.empty(max(linear_lora_workspace_bytes(w, adapters, M, dtype), 256), dtype=torch.uint8, device=device)


def linear_lora(w: QWeight, adapters: Adapters | None, ids: torch.Tensor | None, x: torch.Tensor,
                y: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """y[m] = W x[m] + s_a B_a (A_a x[m]) with a = ids[m] (int32 [M] on the device; outside
    [0, count): no adapter).  x [M][k] and y [M][n] binary16 or bfloat16, any number of
    rows, each row contiguous (the rows may be part of a wider buffer)."""
    M, k = x.shape
    code = _dtype_code(x)
    if k != w.k_in or (M > 1 and x.stride(0) < k) or (k > 1 and x.stride(1) != 1):
        raise ValueError("x must be [M][k] with contiguous rows")
    if y is None:
        y = torch.empty((M, w.n_out), dtype=x.dtype, device=x.device)
    elif y.dtype != x.dtype or y.shape != (M, w.n_out) or (w.n_out > 1 and y.stride(1) != 1) or \
            (M > 1 and y.stride(0) < w.n_out):
        raise ValueError("y must be [M][n] of x's type with contiguous rows")
    ad = None
    if adapters is not None:
        if adapters.A.dtype != x.dtype or adapters.A.shape[2] != k or adapters.B.shape[1] != w.n_out:
            raise ValueError("the adapters are of another type or shape than the linear")
        if ids is None or ids.dtype != torch.int32 or ids.shape != (M,) or not ids.is_contiguous():
            raise ValueError("ids must be int32 [M]")
        ad = ctypes.byref(adapters._c)
    if ws is None:
        ws = linear_lora_workspace(w, adapters, M, x.dtype, x.device)
    here = _one_device(x, y, ids, ws, w.codes, w.meta, adapters.A if adapters else None)
    _check(_lib().qmlp_linear_lora(ctypes.byref(w.c()), ad, _addr(ids) if ad else None, _addr(x), x.stride(0) if M > 1 else k,
                                   M, code, _addr(y), y.stride(0) if M > 1 else w.n_out, _addr(ws), ws.numel(),
                                   torch._C._cuda_getCurrentRawStream(here)), "linear_lora")
    return y


def moe_workspace_bytes(experts: Layers, M: int, k: int, dtype=torch.float16) -> int:
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_moe_workspace_bytes(experts.c(), len(experts), M, k, code))


def moe_lanes(d: int, f: int, gu_bits: int, dn_bits: int, M: int, k: int, cus: int):
    """(gate/up lanes per row, down lanes per row, down form) of
    qmlp_forward_moe's launches for M tokens with k experts each on `cus`
    compute units (qmlp_moe_lanes; host-only).  Down form: "sum" (the down
    launch forms the routing sum), "pipe" or "plain" (a combine follows)."""
    g, dn = ctypes.c_int(0), ctypes.c_int(0)
    r = int(_lib().qmlp_moe_lanes(d, f, gu_bits, dn_bits, M, k, cus, ctypes.byref(g), ctypes.byref(dn)))
    if r < 0:
        raise ValueError("qmlp_moe_lanes rejected its arguments")
    return g.value, dn.value, ("plain", "pipe", "sum")[r]


def forward_moe(experts: Layers, x: torch.Tensor, topk_idx: torch.Tensor, topk_w: torch.Tensor,
                y: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """y [M][d] = sum_j topk_w[m][j] * expert_{topk_idx[m][j]}(x[m]); topk_idx int32
    and topk_w float32 [M][k] on the device."""
    M, d = x.shape
    k = topk_idx.shape[1]
    if topk_idx.dtype != torch.int32 or topk_w.dtype != torch.float32 or topk_w.shape != topk_idx.shape:
        raise ValueError("topk_idx int32 and topk_w float32, both [M][k]")
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = torch.zeros(max(moe_workspace_bytes(experts, M, k, x.dtype), 1024), dtype=torch.uint8,
                         device=x.device)
    _check(_lib().qmlp_forward_moe(experts.c(), len(experts), _ptr(x), M, _dtype_code(x),
                                   _ptr(topk_idx), _ptr(topk_w), k, _ptr(y), _ptr(ws), ws.numel(),
                                   _stream()), "forward_moe")
    return y


SCORES = {"topk_softmax": 0, "softmax": 1, "sigmoid": 2}


def moe_route_workspace(router: torch.Tensor, M: int) -> torch.Tensor:
    """A workspace for moe_route of up to this many tokens (any contents)."""
    n = int(_lib().qmlp_moe_route_workspace_bytes(router.shape[0], M))
    return torch.empty(max(n, 256), dtype=torch.uint8, device=router.device)


def _router_args(router, bias, d, dtype):
    if router.dim() != 2 or router.shape[1] != d or router.dtype != dtype or not router.is_contiguous():
        raise ValueError("router must be [E][d] of x's type, contiguous")
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != router.shape[:1] or not bias.is_contiguous()):
        raise ValueError("bias must be float32 [E]")


def moe_route(x: torch.Tensor, router: torch.Tensor, k: int, bias: torch.Tensor | None = None,
              score: str = "topk_softmax", topk_idx: torch.Tensor | None = None, topk_w: torch.Tensor | None = None,
              ws: torch.Tensor | None = None):
    """(topk_idx int32 [M][k], topk_w float32 [M][k]) of x [M][d]: the k largest of x Wr^T + bias
    per token, ties to the lower expert, and their weights (score: "topk_softmax",
    "softmax" or "sigmoid"; see qmlp_moe_route).  Unused slots: expert -1, weight 0."""
    M, d = x.shape
    code = _dtype_code(x)
    _router_args(router, bias, d, x.dtype)
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    if topk_idx is None:
        topk_idx = torch.empty((M, k), dtype=torch.int32, device=x.device)
    if topk_w is None:
        topk_w = torch.empty((M, k), dtype=torch.float32, device=x.device)
    if topk_idx.dtype != torch.int32 or topk_w.dtype != torch.float32 or topk_idx.shape != (M, k) or \
            topk_w.shape != (M, k) or not topk_idx.is_contiguous() or not topk_w.is_contiguous():
        raise ValueError("topk_idx int32 and topk_w float32, both [M][k]")
    if ws is None:
        ws = moe_route_workspace(router, M)
    here = _one_device(x, router, bias, topk_idx, topk_w, ws)
    _check(_lib().qmlp_moe_route(_addr(router), _addr(bias), _addr(x), M, d, router.shape[0], k, SCORES[score], code,
                                 _addr(topk_idx), _addr(topk_w), _addr(ws), ws.numel(),
                                 torch._C._cuda_getCurrentRawStream(here)), "moe_route")
    return topk_idx, topk_w


class MoE:
    """A whole mixture-of-experts layer: router [E][d], the experts' matrices stacked along their
    rows (gate and up [E f][d], down [E d][f]; stack_qweights joins packed ones), adapters
    A [E][rank][d] and B [E][f][rank]."""

    def __init__(self, router: torch.Tensor, gate: QWeight, up: QWeight, down: QWeight, topk: int, A_gate=None,
                 B_gate=None, A_up=None, B_up=None, lora_scale: float = 1.0, bias: torch.Tensor | None = None,
                 score: str = "topk_softmax"):
        E, d = router.shape
        f = down.k_in
        _router_args(router, bias, gate.k_in, torch.float16)
        rank = 0
        if any(t is not None for t in (A_gate, B_gate, A_up, B_up)):
            if A_gate is None or A_gate.dim() != 3:
                raise ValueError("adapters must be float16, A [E][rank][d] and B [E][f][rank], all four or none")
            rank = int(A_gate.shape[1])
            for t, s in ((A_gate, (E, rank, d)), (A_up, (E, rank, d)), (B_gate, (E, f, rank)), (B_up, (E, f, rank))):
                if t is None or t.dtype != torch.float16 or tuple(t.shape) != s or not t.is_contiguous():
                    raise ValueError("adapters must be float16, A [E][rank][d] and B [E][f][rank], all four or none")
        _one_device(router, bias, gate.codes, gate.meta, up.codes, up.meta, down.codes, down.meta, A_gate, B_gate, A_up, B_up)
        self.router, self.gate, self.up, self.down, self.bias = router, gate, up, down, bias
        self.adapters = (A_gate, B_gate, A_up, B_up)
        self.experts, self.topk, self.d, self.f, self.rank = int(E), int(topk), int(d), int(f), rank
        p = [None if t is None else t.data_ptr() for t in self.adapters]
        self._c = MoeC(router.data_ptr(), None if bias is None else bias.data_ptr(), self.experts, self.topk, SCORES[score],
                       MlpC(gate.c(), up.c(), down.c(), *p, rank, float(lora_scale)))

    def c(self) -> MoeC:
        return self._c


def stack_qweights(ws) -> QWeight:
    """One packed matrix whose rows are those of packed matrices of one width, group and row length."""
    w = list(ws)
    if any((v.bits, v.k_in, v.group) != (w[0].bits, w[0].k_in, w[0].group) for v in w):
        raise ValueError("stacked matrices must agree in bits, columns and group")
    return QWeight(w[0].bits, sum(v.n_out for v in w), w[0].k_in, w[0].group, torch.cat([v.codes for v in w]),
                   torch.cat([v.meta for v in w]))


def moe_layer_workspace_bytes(moe: MoE, M: int) -> int:
    return int(_lib().qmlp_moe_layer_workspace_bytes(ctypes.byref(moe._c), M, F16))


def moe_layer_workspace(moe: MoE, M: int, device="cuda") -> torch.Tensor:
    """A workspace for moe_layer of up to this many tokens (any contents)."""
    return torch.empty(max(moe_layer_workspace_bytes(moe, M), 256), dtype=torch.uint8, device=device)


def moe_layer(moe: MoE, x: torch.Tensor, y: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """y [M][d] = sum_j w[m][j] expert_{idx[m][j]}(x[m]), routed by the layer's own router (qmlp_moe_layer); binary16,
    up to 64 tokens."""
    M, d = x.shape
    if x.dtype != torch.float16 or d != moe.d or not x.is_contiguous():
        raise ValueError("x must be float16 [M][d], contiguous")
    if y is None:
        y = torch.empty_like(x)
    elif y.dtype != x.dtype or y.shape != x.shape or not y.is_contiguous():
        raise ValueError("y must be float16 [M][d], contiguous")
    if ws is None:
        ws = moe_layer_workspace(moe, M, x.device)
    here = _one_device(x, y, ws, moe.router)
    _check(_lib().qmlp_moe_layer(ctypes.byref(moe._c), _addr(x), M, F16, _addr(y), _addr(ws), ws.numel(),
                                 torch._C._cuda_getCurrentRawStream(here)), "moe_layer")
    return y


class _Keeps:
    """An object whose tensors' addresses the kernels are given: what _KEPT names is set once."""
    _KEPT, _WHY = (), ""

    def __setattr__(self, name, value):
        if name in self._KEPT and self.__dict__.get(name, value) is not value:     # (the same again: lens += 1)
            raise AttributeError(self._WHY)
        super().__setattr__(name, value)

    def __delattr__(self, name):
        if name in self._KEPT:
            raise AttributeError(self._WHY)
        super().__delattr__(name)


class KVCache(_Keeps):
    """A paged cache of keys and values in 4 bits: ``data`` uint8 [pages][kv_heads][2][page * (head_dim/2 + 4)] on the
    device (the storage format of qmlp_kv_cache; kv_cache makes an empty one)."""
    _KEPT = ("data", "page", "pages", "kv_heads", "head_dim", "_c", "_at")
    _WHY = "a cache keeps its tensor (its contents change)"

    def __init__(self, data: torch.Tensor, page: int):
        if data.dim() != 4 or data.dtype != torch.uint8 or data.shape[2] != 2 or not data.is_contiguous() or \
                page < 1 or data.shape[3] % page or data.shape[3] // page not in (36, 68):
            raise ValueError("data must be contiguous uint8 [pages][kv_heads][2][page * (head_dim/2 + 4)], head_dim 64 or 128")
        self.data, self.page = data, int(page)
        self.pages, self.kv_heads = int(data.shape[0]), int(data.shape[1])
        self.head_dim = 2 * (int(data.shape[3]) // self.page - 4)
        if not _lib().qmlp_kv_cache_bytes(self.pages, self.kv_heads, self.head_dim, self.page):
            raise QmlpError(4, "KVCache")
        self._c = KVCacheC(data.data_ptr(), self.pages, self.kv_heads, self.head_dim, self.page)
        self._at = ctypes.addressof(self._c)

    def c(self) -> KVCacheC:
        return self._c


def kv_cache(pages: int, kv_heads: int, head_dim: int, page: int = 64, device="cuda") -> KVCache:
    """An empty cache (all zeros)."""
    return KVCache(torch.zeros((pages, kv_heads, 2, page * (head_dim // 2 + 4)), dtype=torch.uint8, device=device), page)


def _here(*tensors):
    """_one_device for the calls of a decoding step, with one question a tensor (the first is not None)."""
    here = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            here = -1
    if here < 0 or here != torch.cuda.current_device():
        raise ValueError("every tensor must be on the current CUDA device")
    return here


def _at(t):
    return 0 if t is None else t.data_ptr()


def _ints(n, what, *tensors):
    for t in tensors:
        if t is not None and (t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous()):
            raise ValueError("%s must be int32 [%d], contiguous" % (what, n))


def _is_table(table, B):
    if table.dim() != 2 or table.shape[0] != B or table.dtype is not torch.int32 or not table.is_contiguous():
        raise ValueError("table must be int32 [B][W], contiguous")
    return table.shape[1]


class KVPlan(_Keeps):
    """What kv_plan writes for up to ``B`` requests and ``tokens`` new tokens of a step: int32 ``slots`` and ``positions``
    [tokens], ``starts`` [B + 1], ``lens`` [B], ``n_free`` [1], ``short`` [1] (requests refused)."""
    _KEPT = ("slots", "positions", "starts", "short", "lens", "n_free", "B", "tokens", "_out")
    _WHY = "a plan keeps its tensors (their contents change)"

    def __init__(self, B: int, tokens: int, device="cuda", lens: torch.Tensor | None = None,
                 n_free: torch.Tensor | None = None):
        new = lambda n: torch.empty(n, dtype=torch.int32, device=device)
        self.slots, self.positions, self.starts, self.short = new(tokens), new(tokens), new(B + 1), new(1)
        self.lens, self.n_free = new(B) if lens is None else lens, new(1) if n_free is None else n_free
        _ints(B, "lens", self.lens)
        _ints(1, "n_free", self.n_free)
        t = (self.slots, self.positions, self.starts, self.lens, self.n_free, self.short)
        if len({v.device for v in t}) != 1:
            raise ValueError("lens and n_free must be on the plan's device")
        self.B, self.tokens = B, tokens
        self._out = tuple(v.data_ptr() for v in t)


def kv_plan(plan: KVPlan, lens: torch.Tensor, new: torch.Tensor, table: torch.Tensor, free: torch.Tensor,
            n_free: torch.Tensor, page: int) -> KVPlan:
    """The pages of a step (qmlp_kv_plan): requests with ``lens`` cached tokens add ``new`` (-1: ended, pages back on the
    stack ``free`` of ``n_free``); ``table`` [B][W] grows in place and ``plan`` takes starts, slots, positions and the new
    lens and n_free (which may be the same tensors as the old ones).  All int32."""
    B = plan.B
    _ints(B, "lens and new", lens, new)
    _ints(1, "n_free", n_free)
    N = free.numel()
    _ints(N, "free", free)
    W = _is_table(table, B)
    here = _here(plan.slots, lens, new, table, free, n_free)
    _check(_lib().qmlp_kv_plan(_PLAN.pack(lens.data_ptr(), new.data_ptr(), table.data_ptr(), free.data_ptr(), n_free.data_ptr(),
                                          *plan._out, B, page, W, N, plan.tokens),
                               torch._C._cuda_getCurrentRawStream(here)), "kv_plan")
    return plan


PAIRS = {"half": 0, "next": 1}


def _head_rows(t, what, T, D, dtype):
    """(heads, row stride) of [T][heads][D] with the heads of a row side by side."""
    if t.dim() != 3 or t.dtype is not dtype:
        raise ValueError("%s must be [T][heads][head_dim] of q's type" % what)
    (t0, H, d), (ld, hs, ds) = t.shape, t.stride()
    if t0 != T or d != D:
        raise ValueError("%s must be [T][heads][head_dim] of q's type" % what)
    if ds != 1 or (H > 1 and hs != D):
        raise ValueError("the heads of a row of %s must lie side by side" % what)
    return H, ld if T > 1 else H * D


def qk_norm_rope(q: torch.Tensor | None, k: torch.Tensor | None, positions: torch.Tensor | None = None,
                 inv_freq: torch.Tensor | None = None, q_weight: torch.Tensor | None = None,
                 k_weight: torch.Tensor | None = None, eps: float = 1e-6, pairs: str = "half", mul: float = 1.0,
                 q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, cache: KVCache | None = None,
                 v: torch.Tensor | None = None, slots: torch.Tensor | None = None):
    """RMS norm of each head (with a weight) and rotation by position (with inv_freq float32 [rot/2]; positions int32 [T])
    of q [T][heads][D] and k [T][kv_heads][D]; with a cache, k and v are quantized into it at slots int32 [T] (negative: not
    written).  eps and mul are binary32.  Returns (q_out, k_out); without a cache k_out is made if it is not given, with one it is None unless given.
    q_out may be q and k_out may be k."""
    x = q if q is not None else k
    if x is None or x.dim() != 3:
        raise ValueError("q or k must be given, [T][heads][head_dim]")
    T, _, D = x.shape
    code, dtype = _dtype_code(x), x.dtype
    Hq = ldq = ldqo = Hk = ldk = ldko = ldv = rot = 0
    if q is not None:
        Hq, ldq = _head_rows(q, "q", T, D, dtype)
        if q_out is None:
            q_out = torch.empty((T, Hq, D), dtype=dtype, device=q.device)
        H, ldqo = _head_rows(q_out, "q_out", T, D, dtype)
        if H != Hq:
            raise ValueError("q_out must have q's shape")
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        Hk, ldk = _head_rows(k, "k", T, D, dtype)
        if k_out is None and cache is None:
            k_out = torch.empty((T, Hk, D), dtype=dtype, device=k.device)
        if k_out is not None:
            H, ldko = _head_rows(k_out, "k_out", T, D, dtype)
            if H != Hk:
                raise ValueError("k_out must have k's shape")
    elif k_out is not None or cache is not None:
        raise ValueError("a cache and k_out need k")
    if (cache is None) != (v is None) or (cache is None) != (slots is None):
        raise ValueError("cache, v and slots go together")
    if cache is not None:
        H, ldv = _head_rows(v, "v", T, D, dtype)
        if H != Hk:
            raise ValueError("v must have k's shape")
        _ints(T, "slots", slots)
    if (inv_freq is None) != (positions is None):
        raise ValueError("positions and inv_freq go together")
    if inv_freq is not None:
        _ints(T, "positions", positions)
        if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be float32 [rot/2], contiguous")
        rot = 2 * inv_freq.numel()
    for w in (q_weight, k_weight):
        if w is not None and (w.dtype is not dtype or w.shape != (D,) or not w.is_contiguous()):
            raise ValueError("weights must be [head_dim] of q's type, contiguous")
    here = _here(x, k, v, positions, inv_freq, q_weight, k_weight, q_out, k_out, slots, cache.data if cache else None)
    _check(_lib().qmlp_qk_norm_rope(_HEADS.pack(_at(q), _at(k), _at(v), ldq, ldk, ldv, _at(q_out), _at(k_out), ldqo, ldko,
                                                _at(q_weight), _at(k_weight), _at(positions), _at(inv_freq), _at(slots), Hq, Hk, D,
                                                rot, PAIRS[pairs], eps, mul), T, code, cache._at if cache else None,
                                    torch._C._cuda_getCurrentRawStream(here)), "qk_norm_rope")
    return q_out, k_out


def kv_read(cache: KVCache, slots: torch.Tensor, k: torch.Tensor | None = None, v: torch.Tensor | None = None,
            dtype=torch.float16):
    """(k, v) [T][kv_heads][head_dim] as the cache holds them at slots int32 [T]; zeros for a slot outside it.  Both are
    made if neither is given; else the given ones are written."""
    T = slots.numel()
    shape = (T, cache.kv_heads, cache.head_dim)
    _ints(T, "slots", slots)
    if k is None and v is None:
        k, v = (torch.empty(shape, dtype=dtype, device=slots.device) for _ in range(2))
    x = k if k is not None else v
    for t in (k, v):
        if t is not None and (t.shape != shape or not t.is_contiguous() or t.dtype is not x.dtype):
            raise ValueError("k and v must be [T][kv_heads][head_dim], contiguous and of one type")
    code = _dtype_code(x)
    here = _here(slots, k, v, cache.data)
    _check(_lib().qmlp_kv_read(cache._at, slots.data_ptr(), T, code, _addr(k), _addr(v),
                               torch._C._cuda_getCurrentRawStream(here)), "kv_read")
    return k, v


def kv_attention_workspace_bytes(cache: KVCache, heads: int, max_new: int) -> int:
    return int(_lib().qmlp_kv_attention_workspace_bytes(ctypes.byref(cache._c), heads, max_new))


def kv_attention_workspace(q: torch.Tensor, cache: KVCache, table: torch.Tensor | None = None, max_new: int = 1) -> torch.Tensor:
    """A zeroed workspace for kv_attention of steps with up to max_new new tokens a request (zero it again after a call
    that failed)."""
    return torch.zeros(max(kv_attention_workspace_bytes(cache, q.shape[1], max_new), 256), dtype=torch.uint8, device=q.device)


def kv_attention(q: torch.Tensor, cache: KVCache, table: torch.Tensor, lens: torch.Tensor, starts: torch.Tensor | None = None,
                 y: torch.Tensor | None = None, max_new: int | None = None, scale: float | None = None, window: int = 0,
                 sinks: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """y [T][heads][D]: causal attention of a step's rows q over the cache.  Request b has lens[b] cached tokens, pages
    table[b], and the rows starts[b] .. starts[b+1] (None: one row each), which are its last tokens.  scale: head_dim^-0.5
    unless given; window: tokens a row sees, itself among them (0: all); sinks float32 [heads] or None.  max_new: the most
    new tokens of a request (it chooses kernels; unless given, 1 without starts and T with them).  Rows before starts[0]
    and from starts[B] on are left as they are (a y made here starts at zeros)."""
    if q.dim() != 3:
        raise ValueError("q must be [T][heads][head_dim]")
    code, dtype = _dtype_code(q), q.dtype
    T, _, D = q.shape
    H, ldq = _head_rows(q, "q", T, D, dtype)
    if D != cache.head_dim:
        raise ValueError("q and the cache differ in head_dim")
    if y is None:
        y = torch.zeros((T, H, D), dtype=dtype, device=q.device)
    Hy, ldy = _head_rows(y, "y", T, D, dtype)
    if Hy != H:
        raise ValueError("y must have q's shape")
    B = lens.numel()
    _ints(B, "lens", lens)
    _ints(B + 1, "starts", starts)
    W = _is_table(table, B)
    if sinks is not None and (sinks.dtype is not torch.float32 or sinks.shape != (H,) or not sinks.is_contiguous()):
        raise ValueError("sinks must be float32 [heads]")
    if max_new is None:
        max_new = T if starts is not None else 1
    if ws is None:
        ws = kv_attention_workspace(q, cache, table, max_new)
    here = _here(q, y, table, lens, starts, sinks, ws, cache.data)
    _check(_lib().qmlp_kv_attention(cache._at, _ATTENTION.pack(q.data_ptr(), y.data_ptr(), ldq, ldy, table.data_ptr(), lens.data_ptr(),
                                                               _at(starts), _at(sinks), ws.data_ptr(), ws.numel(), T, H, B, W,
                                                               max_new, window, D ** -0.5 if scale is None else scale),
                                    code, torch._C._cuda_getCurrentRawStream(here)), "kv_attention")
    return y


def stack_workspace_bytes(stack: Stack, M: int, dtype=torch.float16) -> int:
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_stack_workspace_bytes(stack.c(), len(stack), M, code))


def stack_launches(stack: Stack, M: int, dtype=torch.float16) -> int:
    """Launches forward_stack makes (persistent launches, or the per-layer kernels)."""
    code = F16 if dtype == torch.float16 else BF16
    return int(_lib().qmlp_stack_launches(stack.c(), len(stack), M, code))


def stack_workspace(stack: Stack, M: int, dtype=torch.float16, device="cuda") -> torch.Tensor:
    """A zeroed workspace for forward_stack."""
    n = stack_workspace_bytes(stack, M, dtype)
    return torch.zeros(max(n, 1024), dtype=torch.uint8, device=device)


def stack_errors(stack: Stack, ws: torch.Tensor, M: int = 1, dtype=torch.float16) -> int:
    """Sticky error bits of the persistent stack launch (syncs): 1/2/4 = a wait for
    the activation / h / the cross-XCD partials gave up, 8 = a workgroup had no place."""
    code = F16 if dtype == torch.float16 else BF16
    off = int(_lib().qmlp_stack_error_offset(stack.c(), len(stack), M, code))
    if off == 0:
        return 0
    return int(ws[off: off + 4].view(torch.int32).item())


def forward_stack(stack: Stack, x: torch.Tensor, y: torch.Tensor | None = None,
                  ws: torch.Tensor | None = None, x_out: torch.Tensor | None = None) -> torch.Tensor:
    """y [L][M][d]: every block's output y_l = block_l(RMSNorm(x_l)) on the
    residual stream x_{l+1} = x_l + y_l (x_out, if given, receives x_L)."""
    M = x.shape[0]
    d = stack.mlps[0].d
    if y is None:
        y = torch.empty((len(stack), M, d), dtype=x.dtype, device=x.device)
    if ws is None:
        ws = stack_workspace(stack, M, x.dtype, x.device)
    _check(_lib().qmlp_forward_stack(stack.c(), len(stack), _ptr(x), M, _dtype_code(x), _ptr(y),
                                     _ptr(x_out), _ptr(ws), ws.numel(), _stream()), "forward_stack")
    return y


def probe_stream_read(buf: torch.Tensor, blocks: int, nontemporal: bool = True,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """Read all of `buf` once with 128-bit loads (measurement hook; see
    qmlp_probe_stream_read).  Returns the per-wave XOR words."""
    if out is None:
        out = torch.empty(4 * blocks, dtype=torch.int32, device=buf.device)
    _check(_lib().qmlp_probe_stream_read(_ptr(buf), buf.numel() * buf.element_size(), _ptr(out),
                                         blocks, int(bool(nontemporal)), _stream()),
           "qmlp_probe_stream_read")
    return out
