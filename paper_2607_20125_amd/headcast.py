"""Python binding of the HeadCast C ABI (include/headcast.h).

Argument marshalling only: every step of the routed-attention path runs in the
HIP library.  torch supplies device memory (``tensor.data_ptr()``) and the
current stream; nothing here computes.  If the library is missing this module
raises on import instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libheadcast.so")

HC_OK, HC_E_INVAL, HC_E_STATE, HC_E_ORDER, HC_E_NOMEM, HC_E_DEVICE = 0, -1, -2, -3, -4, -5
SINK, DUMMY, SPATIAL, GLOBAL = 0, 1, 2, 3
N_STATS = 6
K_DENSE, K_SPATIAL, K_SCATTER, K_STATS, K_COMBINE, K_ROTATE, K_SEQUENCE, K_CACHE = range(8)
BF16, F32 = 0, 1
CLS_O_REF, CLS_O_SINK, CLS_O_DUMMY, CLS_O_SPATIAL = 0, 1, 2, 3

EXPORTS = ("hc_config_default", "hc_validate_config", "hc_status_string", "hc_last_error",
           "hc_ring_slot", "hc_create", "hc_destroy", "hc_classify_heads", "hc_classify_outputs",
           "hc_set_head_types",
           "hc_get_layout", "hc_append_block", "hc_attention", "hc_attention_static",
           "hc_memory_bytes", "hc_profile_enable", "hc_profile_read",
           "hc_rotate", "hc_packed_workspace", "hc_packed_attention", "hc_qcache_bytes",
           "hc_qcache_append", "hc_qcache_read", "hc_qcache_workspace", "hc_qcache_attention")
STATIC_SCRATCH_BYTES = 64 << 20   # HC_STATIC_SCRATCH_BYTES


class HCConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_layers", "n_heads", "head_dim", "grid_h", "grid_w", "frames_per_block",
        "window_blocks", "spatial_radius", "proxy_radius")] + [
        (n, ctypes.c_float) for n in (
            "theta_sink", "theta_dummy", "theta_spatial", "theta_score", "gamma",
            "softmax_scale")] + [("spatial_cell", ctypes.c_int32), ("sd_blocks", ctypes.c_int32)]


def _fields(*groups):
    """ctypes fields from (type, "names") pairs."""
    return [(n, kind) for kind, names in groups for n in names.split()]


_P, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class HCRotateTensor(ctypes.Structure):
    _fields_ = _fields((_P, "x out"), (_I64, "x_token x_head out_token out_head"), (_I32, "n_heads"))


class HCRotateArgs(ctypes.Structure):
    _fields_ = (_fields((_I32, "n_tokens head_dim x_type out_type n_axes"), (_I32 * 4, "axis_dims"),
                        (_I32, "halves joint inverse grid_h grid_w frame0"),
                        (ctypes.c_double, "theta"), (_P, "positions")))


class HCPackedArgs(ctypes.Structure):
    _fields_ = _fields((_P, "q k v out"),
                       (_I64, "q_token q_head k_token k_head v_token v_head out_token out_head"),
                       (_I32, "n_tokens n_keys n_seqs n_heads n_kv_heads head_dim causal_block"),
                       (ctypes.c_float, "softmax_scale"), (_P, "cu_q cu_k workspace"),
                       (_I64, "workspace_bytes"))


class HCQCache(ctypes.Structure):
    _fields_ = _fields((_P, "data"), (_I32, "n_seqs n_heads head_dim capacity"))


class HCQCacheRows(ctypes.Structure):
    _fields_ = _fields((_P, "k v"), (_I64, "k_token k_head v_token v_head"), (_I32, "n_tokens"),
                       (_P, "start cu_seqlens"))


class HCQCacheAttentionArgs(ctypes.Structure):
    _fields_ = _fields((_P, "q out"), (_I64, "q_token q_head out_token out_head"),
                       (_I32, "n_tokens n_heads causal_block max_kv"),
                       (ctypes.c_float, "softmax_scale"), (_P, "kv_len cu_seqlens workspace"),
                       (_I64, "workspace_bytes"))


class HeadCastError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{msg} (status {status})")
        self.status = status


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"HeadCast library not built: {LIB_PATH} is missing "
                          "(run `python -m paper_2607_20125_amd.build`)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, U8P, DP = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                            ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_double))
    I32P = ctypes.POINTER(ctypes.c_int32)
    CP = ctypes.POINTER(HCConfig)
    sig = {
        "hc_config_default": (None, [CP]),
        "hc_validate_config": (ctypes.c_int, [CP]),
        "hc_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "hc_last_error": (ctypes.c_char_p, [P]),
        "hc_ring_slot": (I32, [I64, I32]),
        "hc_create": (ctypes.c_int, [CP, ctypes.c_int, ctypes.POINTER(P)]),
        "hc_destroy": (None, [P]),
        "hc_classify_heads": (ctypes.c_int, [P, ctypes.c_int, I64, P, P, P, U8P, DP, P]),
        "hc_classify_outputs": (ctypes.c_int, [P, ctypes.c_int, P, P]),
        "hc_set_head_types": (ctypes.c_int, [P, ctypes.c_int, U8P, I64, P, P, P]),
        "hc_get_layout": (ctypes.c_int, [P, ctypes.c_int, I32P, I32P]),
        "hc_append_block": (ctypes.c_int, [P, ctypes.c_int, I64, P, P, P]),
        "hc_attention": (ctypes.c_int, [P, ctypes.c_int, P, U8P, P, P]),
        "hc_attention_static": (ctypes.c_int, [P, ctypes.c_int, P, U8P, P, P]),
        "hc_memory_bytes": (ctypes.c_int, [P, ctypes.POINTER(I64)]),
        "hc_profile_enable": (ctypes.c_int, [P, ctypes.c_int]),
        "hc_profile_read": (ctypes.c_int, [P, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(I64)]),
        "hc_rotate": (ctypes.c_int, [P, P, P, ctypes.c_int, P]),
        "hc_packed_workspace": (ctypes.c_int, [P, P, ctypes.POINTER(I64)]),
        "hc_packed_attention": (ctypes.c_int, [P, P, P]),
        "hc_qcache_bytes": (ctypes.c_int, [ctypes.POINTER(HCQCache), ctypes.POINTER(I64)]),
        "hc_qcache_append": (ctypes.c_int, [P, ctypes.POINTER(HCQCache), P, P]),
        "hc_qcache_read": (ctypes.c_int, [P, ctypes.POINTER(HCQCache), P, P]),
        "hc_qcache_workspace": (ctypes.c_int, [P, ctypes.POINTER(HCQCache), P, ctypes.POINTER(I64)]),
        "hc_qcache_attention": (ctypes.c_int, [P, ctypes.POINTER(HCQCache), P, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


lib = _load()


def status_string(s: int) -> str:
    return lib.hc_status_string(s).decode()


def ring_slot(block: int, window_blocks: int) -> int:
    return lib.hc_ring_slot(block, window_blocks)


def default_config() -> HCConfig:
    c = HCConfig()
    lib.hc_config_default(ctypes.byref(c))
    return c


def make_config(**kw) -> HCConfig:
    c = default_config()
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def config_from_workload(w, n_layers=None, spatial_cell=0, sd_blocks=1) -> HCConfig:
    return make_config(n_layers=w.n_layers if n_layers is None else n_layers,
                       n_heads=w.n_heads, head_dim=w.head_dim, grid_h=w.grid_h,
                       grid_w=w.grid_w, frames_per_block=w.frames_per_block,
                       window_blocks=w.window_blocks, spatial_radius=w.spatial_radius,
                       proxy_radius=w.proxy_radius, spatial_cell=spatial_cell,
                       sd_blocks=sd_blocks)


def validate_config(cfg: HCConfig) -> int:
    return lib.hc_validate_config(ctypes.byref(cfg))


def _u8(types) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(types, dtype=np.uint8))


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


# The argument structures as native bytes: packing them costs a call a fifth of what filling ctypes
# structures does, which counts where the kernel takes 4 us.
def _packer(layout, *kinds):
    assert struct.calcsize(layout) == sum(ctypes.sizeof(k) for k in kinds), layout
    return struct.Struct(layout).pack


_PACK_ROTATE = _packer("@15idP", HCRotateArgs)
_PACK_TENSOR = {1: _packer("@2P4qi4x", HCRotateTensor),
                2: _packer("@2P4qi4x2P4qi4x", HCRotateTensor, HCRotateTensor)}
_PACK_PACKED = _packer("@4P8q7if3Pq", HCPackedArgs)
_PACK_ROWS = _packer("@2P4qi4x2P", HCQCacheRows)
_PACK_CACHED = _packer("@2P4q4if4x3Pq", HCQCacheAttentionArgs)
_PACK_WORKSPACE = struct.Struct("@Pq").pack      # their last two fields
torch = None                # loaded by the first call that takes tensors or makes a QCache: the host functions need none


def _use_torch():
    global torch, _BF16, _ROTATE_TYPES, _ROTATE_NONE, _raw_stream
    import torch as module
    _BF16 = (module.bfloat16,)
    # code and what the others of the call must be; any other type is refused by the tensor's check
    _ROTATE_TYPES = {module.bfloat16: (BF16, _BF16), module.float32: (F32, (module.float32,))}
    _ROTATE_NONE = BF16, (module.bfloat16, module.float32)
    # torch's current stream of a device as a hipStream_t: the short way where torch has it
    _raw_stream = (getattr(module._C, "_cuda_getCurrentRawStream", None)
                   or (lambda device: module.cuda.current_stream(device).cuda_stream))
    torch = module


class QCache:
    """A cache of 4-bit keys and values (hc_qcache) in one uint8 tensor: `n_seqs`
    sequences of up to `capacity` tokens.  `Context.qcache` makes one."""

    def __init__(self, n_seqs: int, n_heads: int, head_dim: int, capacity: int, device):
        if torch is None:
            _use_torch()
        for name, value in (("n_seqs", n_seqs), ("n_heads", n_heads), ("capacity", capacity)):
            if not 1 <= value < 1 << 31:
                raise ValueError(f"{name} must be at least 1 and below 2^31, got {value}")
        self.desc = HCQCache(None, n_seqs, n_heads, head_dim, capacity)
        nbytes = ctypes.c_int64()
        st = lib.hc_qcache_bytes(ctypes.byref(self.desc), ctypes.byref(nbytes))
        if st != HC_OK:
            raise HeadCastError(st, f"hc_qcache_bytes: {status_string(st)}")
        self.data = torch.empty(nbytes.value, dtype=torch.uint8, device=device)
        self.desc.data = self.data.data_ptr()
        self.device = self.data.get_device()
        self.n_seqs, self.n_heads = n_seqs, n_heads
        self.head_dim, self.capacity = head_dim, capacity


class Context:
    """Owns one hc_ctx (all layers' compact buffers) on one device."""

    def __init__(self, cfg: HCConfig, device: int = 0):
        self.cfg = cfg
        self.device = device
        self._need = ctypes.c_int64()
        self._h = ctypes.c_void_p()
        st = lib.hc_create(ctypes.byref(cfg), device, ctypes.byref(self._h))
        if st != HC_OK:
            raise HeadCastError(st, f"hc_create: {status_string(st)}")
        self.L = cfg.frames_per_block * cfg.grid_h * cfg.grid_w

    def close(self):
        if self._h:
            lib.hc_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, what: str):
        if st != HC_OK:
            msg = lib.hc_last_error(self._h).decode()
            raise HeadCastError(st, f"{what}: {status_string(st)}: {msg}")

    def _tensor(self, t, dtype_name: str, shape):
        import torch
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype_name]
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"expected a contiguous {dtype_name} CUDA tensor, got "
                             f"{t.dtype} on {t.device} (contiguous={t.is_contiguous()})")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
        return ctypes.c_void_p(t.data_ptr())

    def _win_shape(self, n_blocks):
        c = self.cfg
        return (c.n_heads, n_blocks * self.L, c.head_dim)

    def _blk_shape(self):
        c = self.cfg
        return (c.n_heads, self.L, c.head_dim)

    def set_head_types(self, layer: int, types, cur_block: int, k_win, v_win):
        n = min(cur_block + 1, self.cfg.window_blocks)
        ty = _u8(types)
        self._check(lib.hc_set_head_types(
            self._h, layer, ty.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)), cur_block,
            self._tensor(k_win, "bf16", self._win_shape(n)),
            self._tensor(v_win, "bf16", self._win_shape(n)), _stream()), "hc_set_head_types")

    def classify_heads(self, layer: int, cur_block: int, q, k_win, v_win):
        H = self.cfg.n_heads
        types = np.zeros(H, dtype=np.uint8)
        stats = np.zeros((H, N_STATS), dtype=np.float64)
        W = self.cfg.window_blocks
        self._check(lib.hc_classify_heads(
            self._h, layer, cur_block, self._tensor(q, "bf16", self._blk_shape()),
            self._tensor(k_win, "bf16", self._win_shape(W)),
            self._tensor(v_win, "bf16", self._win_shape(W)),
            types.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
            stats.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), _stream()),
            "hc_classify_heads")
        return types, stats

    def classify_outputs(self, which: int, dst):
        """hc_classify_outputs: copy classification output `which` (CLS_O_REF,
        CLS_O_SINK, CLS_O_DUMMY, CLS_O_SPATIAL) of the last classification into
        `dst` (float32 [H][L][d] on the device)."""
        self._check(lib.hc_classify_outputs(self._h, which,
                                            self._tensor(dst, "f32", self._blk_shape()),
                                            _stream()), "hc_classify_outputs")

    def get_layout(self, layer: int):
        H, W = self.cfg.n_heads, self.cfg.window_blocks
        hs = np.zeros(H, dtype=np.int32)
        ring = np.zeros(W, dtype=np.int32)
        I32P = ctypes.POINTER(ctypes.c_int32)
        self._check(lib.hc_get_layout(self._h, layer, hs.ctypes.data_as(I32P),
                                      ring.ctypes.data_as(I32P)), "hc_get_layout")
        return hs, ring

    def append_block(self, layer: int, block: int, k_blk, v_blk):
        self._check(lib.hc_append_block(
            self._h, layer, block, self._tensor(k_blk, "bf16", self._blk_shape()),
            self._tensor(v_blk, "bf16", self._blk_shape()), _stream()), "hc_append_block")

    def attention(self, layer: int, q, types, o):
        ty = _u8(types)
        self._check(lib.hc_attention(
            self._h, layer, self._tensor(q, "bf16", self._blk_shape()),
            ty.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
            self._tensor(o, "f32", self._blk_shape()), _stream()), "hc_attention")

    def attention_static(self, layer: int, q, types, o):
        """hc_attention_static: the same layer-step in the library's fixed
        device scratch (no device allocation)."""
        ty = _u8(types)
        self._check(lib.hc_attention_static(
            self._h, layer, self._tensor(q, "bf16", self._blk_shape()),
            ty.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
            self._tensor(o, "f32", self._blk_shape()), _stream()), "hc_attention_static")

    def memory_bytes(self) -> int:
        b = ctypes.c_int64()
        self._check(lib.hc_memory_bytes(self._h, ctypes.byref(b)), "hc_memory_bytes")
        return b.value

    def profile_enable(self, on: bool = True):
        self._check(lib.hc_profile_enable(self._h, 1 if on else 0), "hc_profile_enable")

    def profile_read(self, kind: int):
        ms, n = ctypes.c_double(), ctypes.c_int64()
        self._check(lib.hc_profile_read(self._h, kind, ctypes.byref(ms), ctypes.byref(n)),
                    "hc_profile_read")
        return ms.value, n.value

    # --- operators beside the routed attention -----------------------------------
    # Tensors are [tokens][heads][head_dim] with any token and head strides that are
    # multiples of 8; a head-major tensor [heads][tokens][head_dim] is passed as
    # t.transpose(0, 1).  No call records a gradient: a tensor that requires one is refused
    # where torch records them.

    def _rows(self, name, t, dtypes, shape=None):
        """Pointer and strides of a [tokens][heads][head_dim] tensor on this context's device."""
        st = t.stride()
        if (len(st) == 3 and st[2] == 1 and t.dtype in dtypes and t.get_device() == self.device
                and (shape is None or t.shape == shape) and not t.requires_grad):
            return t.data_ptr(), st[0], st[1]
        if t.dtype not in dtypes or t.get_device() != self.device:
            raise ValueError(f"{name}: expected {' or '.join(map(str, dtypes))} on cuda:{self.device}, "
                             f"got {t.dtype} on {t.device}")
        if len(st) != 3 or (shape is not None and t.shape != shape):
            raise ValueError(f"{name}: expected shape {tuple(shape) if shape is not None else '[tokens][heads][head_dim]'}, "
                             f"got {tuple(t.shape)}")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which this call does not record: detach it, or call under "
                             "torch.no_grad() (the gradient of rotate is rotate with inverse=True)")
        if st[2] == 1:
            return t.data_ptr(), st[0], st[1]
        if t.numel():
            raise ValueError(f"{name}: neighbouring dims of a head must be adjacent in memory")
        return t.data_ptr(), 0, 0

    def _ints(self, name, t, shape):
        if t is None:
            return 0
        if (t.dtype is torch.int32 and t.get_device() == self.device and t.shape == shape and t.is_contiguous()):
            return t.data_ptr()
        raise ValueError(f"{name}: expected a contiguous int32 tensor of shape {tuple(shape)} on "
                         f"cuda:{self.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")

    def _work(self, workspace):
        """The caller's workspace, or one of the needed size, which torch keeps from other streams' work
        until it is dropped behind the call."""
        if workspace is None:
            return torch.empty(self._need.value, dtype=torch.uint8, device=torch.device("cuda", self.device))
        if workspace.get_device() != self.device or not workspace.is_contiguous():
            raise ValueError(f"workspace: expected a contiguous tensor on cuda:{self.device}")
        return workspace

    def rotate(self, x, out=None, *, axis_dims, positions=None, grid=None, frame0=0,
               theta=10000.0, halves=False, joint=False, inverse=False):
        """hc_rotate: rotary positions over `len(axis_dims)` axes of one tensor or of a pair
        (queries and keys of the same tokens).  `out`: a tensor or pair of the same shapes
        (bf16 or float32; `x` itself rotates in place), new ones by default.  Positions:
        int32 [axes][tokens], or the (frame, row, column) of the tokens of a `grid` of (height,
        width), the context's by default, from frame `frame0` on.  The outputs of a pair overlap neither
        each other nor the other's input.  Returns `out`."""
        if torch is None:
            _use_torch()
        pair = isinstance(x, (tuple, list))
        xs = x if pair else (x,)
        if out is None:
            outs = tuple([torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in xs])
        else:
            outs = out if isinstance(out, (tuple, list)) else (out,)
        n_tensors, n_axes = len(xs), len(axis_dims)
        if len(outs) != n_tensors or not 1 <= n_tensors <= 2:
            raise ValueError("rotate takes one tensor or a pair, and as many outputs")
        if not 1 <= n_axes <= 4:
            raise ValueError("axis_dims must have one to four entries")
        x_code, x_types = _ROTATE_TYPES.get(xs[0].dtype, _ROTATE_NONE)
        out_code, out_types = _ROTATE_TYPES.get(outs[0].dtype, _ROTATE_NONE)
        tensors, n = [], -1
        for t, o in zip(xs, outs):
            shape = t.shape
            xp, xt, xh = self._rows("x", t, x_types)
            op, ot, oh = self._rows("out", o, out_types, shape)
            if n < 0:
                n, heads, d = shape
            elif shape[0] != n or shape[2] != d:
                raise ValueError("a pair has the same tokens, dims and types")
            else:
                heads = shape[1]
            tensors += xp, op, xt, xh, ot, oh, heads
        if n_tensors == 2 and n:
            x0, o0, x1, o1 = tensors[0], tensors[1], tensors[7], tensors[8]
            if o0 == o1 or o0 == x1 or o1 == x0:
                raise ValueError("the outputs of a pair overlap each other, or one the other's input")
        gh, gw = (self.cfg.grid_h, self.cfg.grid_w) if grid is None else grid
        args = _PACK_ROTATE(n, d, x_code, out_code, n_axes, *axis_dims, *(0,) * (4 - n_axes),
                            1 if halves else 0, 1 if joint else 0, 1 if inverse else 0, gh, gw, frame0, theta,
                            0 if positions is None else self._ints("positions", positions, (n_axes, n)))
        status = lib.hc_rotate(self._h, args, _PACK_TENSOR[n_tensors](*tensors), n_tensors, _raw_stream(self.device))
        if status:
            self._check(status, "hc_rotate")
        return tuple(outs) if pair else outs[0]

    def packed_attention(self, q, k, v, cu_q=None, cu_k=None, out=None, *, causal_block=0,
                         softmax_scale=0.0, workspace=None, n_seqs=None):
        """hc_packed_attention: attention over sequences packed behind one another.  cu_q,
        cu_k: int32 [n_seqs + 1] offsets of the queries and keys; cu_k None takes cu_q's, cu_q
        None makes `n_seqs` (1) equal parts.  Returns `out` (bf16, the shape of q; may be q itself)."""
        if torch is None:
            _use_torch()
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if n_seqs is None:
            n_seqs = 1 if cu_q is None else cu_q.numel() - 1
        qs, ks = q.shape, k.shape
        qp, qt, qh = self._rows("q", q, _BF16)
        kp, kt, kh = self._rows("k", k, _BF16)
        vp, vt, vh = self._rows("v", v, _BF16, ks)
        op, ot, oh = self._rows("out", out, _BF16, qs)
        n, heads, d = qs
        m, kv_heads, kd = ks
        if kd != d:
            raise ValueError(f"k: expected heads of {d} dims, got {tuple(ks)}")
        if op in (qp, kp, vp) and n and (m and op in (kp, vp)
                                         or op == qp and (n > 1 and ot != qt or heads > 1 and oh != qh)):
            raise ValueError("out overlaps an input (it may be q itself, with the same strides)")
        packed = _PACK_PACKED(qp, kp, vp, op, qt, qh, kt, kh, vt, vh, ot, oh, n, m, n_seqs, heads, kv_heads, d,
                              causal_block, softmax_scale,
                              0 if cu_q is None else self._ints("cu_q", cu_q, (n_seqs + 1,)),
                              0 if cu_k is None else self._ints("cu_k", cu_k, (n_seqs + 1,)), 0, 0)
        need = self._need
        status = lib.hc_packed_workspace(self._h, packed, need)
        if status:
            self._check(status, "hc_packed_workspace")
        if need.value:
            workspace = self._work(workspace)
            packed = packed[:-16] + _PACK_WORKSPACE(workspace.data_ptr(), workspace.nbytes)
        status = lib.hc_packed_attention(self._h, packed, _raw_stream(self.device))
        if status:
            self._check(status, "hc_packed_attention")
        return out

    def qcache(self, n_seqs: int, n_heads: int, head_dim: int, capacity: int) -> QCache:
        """A new 4-bit cache on this context's device."""
        return QCache(n_seqs, n_heads, head_dim, capacity, f"cuda:{self.device}")

    def _cache_rows(self, fn, what, writes, cache, k, v, start, cu_seqlens):
        shape = k.shape
        kp, kt, kh = self._rows("k", k, _BF16)
        vp, vt, vh = self._rows("v", v, _BF16, shape)
        n, heads, d = shape
        if cache.device != self.device:
            raise ValueError(f"the cache is on {cache.data.device}, not on cuda:{self.device}")
        if heads != cache.n_heads or d != cache.head_dim:
            raise ValueError(f"k: expected shape [tokens][{cache.n_heads}][{cache.head_dim}], got {tuple(shape)}")
        if writes and kp == vp and n:
            raise ValueError("k and v overlap: each is written")
        rows = _PACK_ROWS(kp, vp, kt, kh, vt, vh, n, self._ints("start", start, (cache.n_seqs,)),
                          0 if cu_seqlens is None else self._ints("cu_seqlens", cu_seqlens, (cache.n_seqs + 1,)))
        status = fn(self._h, cache.desc, rows, _raw_stream(self.device))
        if status:
            self._check(status, what)

    def qcache_append(self, cache: QCache, k, v, start, cu_seqlens=None):
        """hc_qcache_append: stores the rows of k and v (bf16 [tokens][cache heads][head_dim])
        in slots start[s] .. of each sequence (int32 [n_seqs])."""
        self._cache_rows(lib.hc_qcache_append, "hc_qcache_append", False, cache, k, v, start, cu_seqlens)

    def qcache_read(self, cache: QCache, k, v, start, cu_seqlens=None):
        """hc_qcache_read: writes the stored values of those slots into k and v, two tensors."""
        self._cache_rows(lib.hc_qcache_read, "hc_qcache_read", True, cache, k, v, start, cu_seqlens)

    def qcache_attention(self, cache: QCache, q, kv_len, cu_seqlens=None, out=None, *,
                         causal_block=0, softmax_scale=0.0, max_kv=0, workspace=None):
        """hc_qcache_attention: attention of q over the first kv_len[s] (int32 [n_seqs]) slots
        of each sequence of the cache.  Returns `out` (bf16, the shape of q; may be q itself)."""
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        qs = q.shape
        qp, qt, qh = self._rows("q", q, _BF16)
        op, ot, oh = self._rows("out", out, _BF16, qs)
        n, heads, d = qs
        if cache.device != self.device:
            raise ValueError(f"the cache is on {cache.data.device}, not on cuda:{self.device}")
        if d != cache.head_dim:
            raise ValueError(f"q: expected heads of {cache.head_dim} dims, got {tuple(qs)}")
        if op == qp and (n > 1 and ot != qt or heads > 1 and oh != qh):
            raise ValueError("out overlaps q (it may be q itself, with the same strides)")
        packed = _PACK_CACHED(qp, op, qt, qh, ot, oh, n, heads, causal_block, max_kv, softmax_scale,
                              self._ints("kv_len", kv_len, (cache.n_seqs,)),
                              0 if cu_seqlens is None else self._ints("cu_seqlens", cu_seqlens, (cache.n_seqs + 1,)),
                              0, 0)
        need = self._need
        status = lib.hc_qcache_workspace(self._h, cache.desc, packed, need)
        if status:
            self._check(status, "hc_qcache_workspace")
        if need.value:
            workspace = self._work(workspace)
            packed = packed[:-16] + _PACK_WORKSPACE(workspace.data_ptr(), workspace.nbytes)
        status = lib.hc_qcache_attention(self._h, cache.desc, packed, _raw_stream(self.device))
        if status:
            self._check(status, "hc_qcache_attention")
        return out
