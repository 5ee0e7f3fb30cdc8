"""Python binding of libnacl.so (the C ABI declared in include/nacl.h).

Argument marshalling only: every step of the eviction runs in the library's
HIP kernels.  torch tensors provide device memory and the stream.  If the
built library is missing, importing works but every call raises; there is no
CPU fallback.
"""

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libnacl.so")

NACL_OK = 0
NACL_ERR_INVALID_ARG = 1
NACL_ERR_UNSUPPORTED = 2
NACL_ERR_WORKSPACE = 3
NACL_ERR_HIP = 4

NACL_F32 = 0
NACL_BF16 = 1

SAMPLE_SOFTMAX = 0
SAMPLE_PROPORTIONAL = 1
SAMPLE_UNIFORM = 2

EXPORTED = ("nacl_workspace_bytes", "nacl_score", "nacl_select", "nacl_compact", "nacl_compact_slots",
            "nacl_append", "nacl_evict", "nacl_evict_slots", "nacl_evict_noalloc", "nacl_attention",
            "nacl_rotate_append", "nacl_prefix_workspace_bytes", "nacl_prefix_attention",
            "nacl_sample_workspace_bytes", "nacl_sample", "nacl_status_string",
            "nacl_last_error_detail", "nacl_version")


class NaclError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__(f"nacl status {status}: {detail}")
        self.status = status
        self.detail = detail


class _Problem(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("D", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("P", ctypes.c_int32), ("n_protect", ctypes.c_int32),
        ("sm_scale", ctypes.c_float),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3),
        ("proxy_pos", ctypes.POINTER(ctypes.c_int32)),
        ("proxy_pos_dev", ctypes.c_void_p),
        ("q_group", ctypes.c_int32),
    ]


class _Step(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int32), ("row0", ctypes.c_int32), ("lens", ctypes.c_void_p), ("n_new", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("q_out_stride", ctypes.c_int64 * 3),
    ]


class _Rotation(ctypes.Structure):
    _fields_ = [
        ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float),
        ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p),
        ("pos_stride", ctypes.c_int64),
    ]


class _Prefix(ctypes.Structure):
    _fields_ = [
        ("G", ctypes.c_int32), ("L", ctypes.c_int32), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("lens", ctypes.c_void_p),
    ]


class _Draw(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32), ("stride", ctypes.c_int64),
        ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
        ("min_p", ctypes.c_void_p),
    ]


_lib = None


def load_library(path=LIB_PATH):
    """Loads libnacl.so once and declares the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2408_03675_amd.build`")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(_Problem)
    vp, sz, i32, u32, u64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64
    lib.nacl_workspace_bytes.argtypes = [P]
    lib.nacl_workspace_bytes.restype = sz
    lib.nacl_score.argtypes = [P, vp, vp, vp, vp, vp, sz, vp]
    lib.nacl_score.restype = ctypes.c_int
    lib.nacl_select.argtypes = [P, vp, i32, i32, i32, u64, u32, vp, vp, sz, vp]
    lib.nacl_select.restype = ctypes.c_int
    lib.nacl_compact.argtypes = [P, vp, vp, vp, i32, vp, vp, vp]
    lib.nacl_compact.restype = ctypes.c_int
    lib.nacl_compact_slots.argtypes = [P, vp, vp, vp, i32, vp, vp]
    lib.nacl_compact_slots.restype = ctypes.c_int
    lib.nacl_evict_slots.argtypes = [P, vp, vp, vp, i32, i32, i32, u64, u32, vp, vp, vp, vp, sz, vp]
    lib.nacl_evict_slots.restype = ctypes.c_int
    lib.nacl_append.argtypes = [P, vp, vp, i32, vp, vp, i32, vp]
    lib.nacl_append.restype = ctypes.c_int
    lib.nacl_evict.argtypes = [P, vp, vp, vp, i32, i32, i32, u64, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.nacl_evict.restype = ctypes.c_int
    lib.nacl_evict_noalloc.argtypes = [P, vp, vp, vp, i32, i32, i32, u64, u32, vp, vp, vp, vp, vp, vp]
    lib.nacl_evict_noalloc.restype = ctypes.c_int
    lib.nacl_attention.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    lib.nacl_attention.restype = ctypes.c_int
    S, R, X, W = (ctypes.POINTER(t) for t in (_Step, _Rotation, _Prefix, _Draw))
    lib.nacl_rotate_append.argtypes = [P, S, R, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.nacl_rotate_append.restype = ctypes.c_int
    lib.nacl_prefix_workspace_bytes.argtypes = [P, S, X]
    lib.nacl_prefix_workspace_bytes.restype = sz
    lib.nacl_prefix_attention.argtypes = [P, S, X, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.nacl_prefix_attention.restype = ctypes.c_int
    lib.nacl_sample_workspace_bytes.argtypes = [W]
    lib.nacl_sample_workspace_bytes.restype = sz
    lib.nacl_sample.argtypes = [W, vp, vp, vp, vp, vp, sz, vp]
    lib.nacl_sample.restype = ctypes.c_int
    lib.nacl_status_string.argtypes = [ctypes.c_int]
    lib.nacl_status_string.restype = ctypes.c_char_p
    lib.nacl_last_error_detail.argtypes = []
    lib.nacl_last_error_detail.restype = ctypes.c_char_p
    lib.nacl_score_kernel.argtypes = [P, ctypes.c_int, ctypes.c_int]
    lib.nacl_score_kernel.restype = ctypes.c_char_p
    lib.nacl_version.argtypes = []
    lib.nacl_version.restype = ctypes.c_int
    _lib = lib
    return lib


def _check(status):
    if status != NACL_OK:
        lib = load_library()
        raise NaclError(status, lib.nacl_last_error_detail().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _gpu(t, name, dev, shape=None, dtype=None, strides=None, contiguous=False):
    """Checks a tensor argument before its address reaches the kernels: on the
    call's GPU, of the expected shape and dtype, with the problem's strides (Q,
    K, V) or contiguous (scores, indices, outputs, workspace)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on the GPU")
    if t.device != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on {dev}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if strides is not None and (t.dim() != 4 or t.stride(3) != 1 or tuple(t.stride()[:3]) != tuple(strides)):
        raise ValueError(f"{name} has strides {tuple(t.stride())}, the problem has {tuple(strides)} (+ 1)")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.data_ptr() == 0 and t.numel():  # (a null address would mean that it was not given)
        raise ValueError(f"{name} has no memory")
    return t


def _strides(t):
    if t.dim() != 4 or t.stride(3) != 1:
        raise ValueError("Q/K/V must be [B, H, L, D] with a contiguous last dimension")
    return tuple(int(s) for s in t.stride()[:3])


class Problem:
    """nacl_problem for one layer, with its host proxy-position array kept
    alive.  `dtype` is "bf16" or "f32"."""

    def __init__(self, B, H, L, D, dtype, proxy_pos, n_protect=None, sm_scale=None,
                 q_stride=None, k_stride=None, v_stride=None, proxy_pos_dev=None, q_group=1):
        pos = [int(x) for x in proxy_pos]
        self._pos = (ctypes.c_int32 * max(1, len(pos)))(*pos)
        self.proxy_pos = pos
        self.q_group = int(q_group)
        dense = (H * L * D, L * D, D)
        dense_q = (H * self.q_group * L * D, L * D, D)
        s = _Problem()
        s.B, s.H, s.L, s.D = B, H, L, D
        s.dtype = NACL_F32 if dtype in ("f32", torch.float32) else NACL_BF16
        s.P = len(pos)
        s.n_protect = len(pos) if n_protect is None else int(n_protect)
        s.sm_scale = float(sm_scale) if sm_scale else 1.0 / (D ** 0.5)
        s.q_stride[:] = q_stride or dense_q
        s.k_stride[:] = k_stride or dense
        s.v_stride[:] = v_stride or dense
        s.proxy_pos = ctypes.cast(self._pos, ctypes.POINTER(ctypes.c_int32))
        s.q_group = self.q_group
        self.c = s
        self._pos_dev = proxy_pos_dev
        if proxy_pos_dev is not None:
            self._take_pos_dev()

    def _take_pos_dev(self):
        t = self._pos_dev
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and
                t.numel() == len(self.proxy_pos)):
            raise ValueError("proxy_pos_dev must be a contiguous int32 GPU tensor with one entry per proxy")
        self.c.proxy_pos_dev = t.data_ptr()

    @classmethod
    def from_tensors(cls, q, k, v, proxy_pos, n_protect=None, sm_scale=None, proxy_pos_dev=None):
        """q may have a multiple of k's heads (grouped-query attention)."""
        B, H, L, D = k.shape
        if q.dim() != 4 or q.shape[1] % H:
            raise ValueError("q must be [B, H * q_group, L, D] for k of [B, H, L, D]")
        return cls(B, H, L, D, k.dtype, proxy_pos, n_protect, sm_scale,
                   _strides(q), _strides(k), _strides(v), proxy_pos_dev, q_group=q.shape[1] // H)

    @property
    def B(self):
        return self.c.B

    @property
    def H(self):
        return self.c.H

    @property
    def L(self):
        return self.c.L

    @property
    def D(self):
        return self.c.D

    @property
    def torch_dtype(self):
        return torch.float32 if self.c.dtype == NACL_F32 else torch.bfloat16

    def ref(self):
        """The struct for a call.  proxy_pos_dev may have got a new storage since
        the last one (a module's buffer does when it is moved)."""
        if self._pos_dev is not None and self._pos_dev.data_ptr() != self.c.proxy_pos_dev:
            self._take_pos_dev()
        return ctypes.byref(self.c)

    # Shapes the entry points expect.
    def qkv(self, t, name, dev, which):
        st = {"q": self.c.q_stride, "k": self.c.k_stride, "v": self.c.v_stride}[which]
        heads = self.H * self.q_group if which == "q" else self.H
        return _gpu(t, name, dev, (self.B, heads, self.L, self.D), self.torch_dtype, tuple(st))


def workspace_bytes(prob):
    return int(load_library().nacl_workspace_bytes(prob.ref()))


def workspace(prob, device="cuda"):
    """A workspace for prob, zeroed so that its sticky health word starts
    clean (the library itself needs no initialised contents)."""
    n = workspace_bytes(prob)
    if n == 0:
        lib = load_library()
        raise NaclError(NACL_ERR_INVALID_ARG, lib.nacl_last_error_detail().decode())
    return torch.zeros(n, dtype=torch.uint8, device=device)


def health(ws):
    """(this call's, sticky) health words of a workspace (include/nacl.h);
    reading them waits for the stream."""
    w = ws[4:12].view(torch.int32).cpu()
    return int(w[0]), int(w[1])


def score_kernel(prob, lse=False, cus=256):
    """Name of the kernel that scores a call of these sizes (lse: with the
    caller's log-sum-exp) on a device of cus compute units."""
    name = load_library().nacl_score_kernel(prob.ref(), int(bool(lse)), int(cus))
    return None if name is None else name.decode()


def score(prob, q, k, ws, lse=None, out=None):
    """F [B, H, L] fp32 (Section 5.1).  lse: optional [B, H, P] natural
    log-sum-exp from the caller."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    prob.qkv(q, "q", dev, "q")
    prob.qkv(k, "k", dev, "k")
    if lse is not None:
        _gpu(lse, "lse", dev, (prob.B, prob.H * prob.q_group, prob.c.P), torch.float32, contiguous=True)
    _gpu(ws, "ws", dev, dtype=torch.uint8, contiguous=True)
    if out is None:
        out = torch.empty((prob.B, prob.H, prob.L), dtype=torch.float32, device=k.device)
    _gpu(out, "out", dev, (prob.B, prob.H, prob.L), torch.float32, contiguous=True)
    _check(lib.nacl_score(prob.ref(), _ptr(q), _ptr(k), _ptr(lse), _ptr(out), _ptr(ws),
                          ws.numel(), _stream(k.device)))
    return out


def select(prob, scores, C, Cr, sampling=SAMPLE_SOFTMAX, seed=0, layer=0, ws=None, out=None):
    """keep_idx [B, H, C] int32, ascending (Sections 5.1-5.2, Algorithm 1)."""
    lib = load_library()
    dev = _gpu(scores, "scores", scores.device, (prob.B, prob.H, prob.L), torch.float32, contiguous=True).device
    if ws is not None:
        _gpu(ws, "ws", dev, dtype=torch.uint8, contiguous=True)
    if out is None:
        out = torch.empty((prob.B, prob.H, C), dtype=torch.int32, device=scores.device)
    _gpu(out, "out", dev, (prob.B, prob.H, int(C)), torch.int32, contiguous=True)
    _check(lib.nacl_select(prob.ref(), _ptr(scores), int(C), int(Cr), int(sampling), int(seed),
                           int(layer), _ptr(out), _ptr(ws), 0 if ws is None else ws.numel(),
                           _stream(scores.device)))
    return out


def compact(prob, k, v, keep_idx, k_out=None, v_out=None, in_place=False):
    """K', V' [B, H, C, D] (Section 3).  in_place: the kept rows move to rows
    0..C-1 of each head of k and v themselves (generation-phase cache)."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    prob.qkv(k, "k", dev, "k")
    prob.qkv(v, "v", dev, "v")
    C = keep_idx.shape[-1]
    _gpu(keep_idx, "keep_idx", dev, (prob.B, prob.H, C), torch.int32, contiguous=True)
    if in_place:
        k_out, v_out = k, v
    else:
        if k_out is None:
            k_out = torch.empty((prob.B, prob.H, C, prob.D), dtype=k.dtype, device=k.device)
        if v_out is None:
            v_out = torch.empty((prob.B, prob.H, C, prob.D), dtype=v.dtype, device=v.device)
        for t, name in ((k_out, "k_out"), (v_out, "v_out")):
            _gpu(t, name, dev, (prob.B, prob.H, C, prob.D), prob.torch_dtype, contiguous=True)
    _check(lib.nacl_compact(prob.ref(), _ptr(k), _ptr(v), _ptr(keep_idx), int(C), _ptr(k_out),
                            _ptr(v_out), _stream(k.device)))
    return k_out, v_out


def attention(prob, q, k, v, out=None, lse=None, lse_proxy=False):
    """Causal attention of the prefill and each row's log-sum-exp (the
    forward pass whose log-sum-exp Appendix A.7 hands to the score).
    Returns (out [B, H*q_group, L, D] bf16, lse [B, H*q_group, L] fp32,
    lse_proxy [B, H*q_group, P] fp32 or None).  lse_proxy=True needs the
    problem's proxy_pos_dev; the result is nacl_score's lse argument."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    prob.qkv(q, "q", dev, "q")
    prob.qkv(k, "k", dev, "k")
    prob.qkv(v, "v", dev, "v")
    Hq = prob.H * prob.q_group
    if out is None:
        out = torch.empty((prob.B, Hq, prob.L, prob.D), dtype=prob.torch_dtype, device=dev)
    _gpu(out, "out", dev, (prob.B, Hq, prob.L, prob.D), prob.torch_dtype, contiguous=True)
    if lse is None:
        lse = torch.empty((prob.B, Hq, prob.L), dtype=torch.float32, device=dev)
    _gpu(lse, "lse", dev, (prob.B, Hq, prob.L), torch.float32, contiguous=True)
    lp = None
    if lse_proxy is True:
        lp = torch.empty((prob.B, Hq, prob.c.P), dtype=torch.float32, device=dev)
    elif lse_proxy is not False and lse_proxy is not None:
        lp = _gpu(lse_proxy, "lse_proxy", dev, (prob.B, Hq, prob.c.P), torch.float32, contiguous=True)
    _check(lib.nacl_attention(prob.ref(), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(lp),
                              _stream(k.device)))
    return out, lse, lp


def compact_slots(prob, k, v, keep_idx, slot_idx=None):
    """Slot form of the in-place cache update (Section 3, generation phase):
    kept rows below C stay, kept rows at or past C fill the other slots below
    C, in ascending order.  keep_idx [B, H, C] is the ascending keep set.
    Returns slot_idx [B, H, C]: the old row each slot holds afterwards."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    prob.qkv(k, "k", dev, "k")
    prob.qkv(v, "v", dev, "v")
    C = keep_idx.shape[-1]
    _gpu(keep_idx, "keep_idx", dev, (prob.B, prob.H, C), torch.int32, contiguous=True)
    if slot_idx is None:
        slot_idx = torch.empty((prob.B, prob.H, C), dtype=torch.int32, device=dev)
    _gpu(slot_idx, "slot_idx", dev, (prob.B, prob.H, C), torch.int32, contiguous=True)
    _check(lib.nacl_compact_slots(prob.ref(), _ptr(k), _ptr(v), _ptr(keep_idx), int(C), _ptr(slot_idx),
                                  _stream(k.device)))
    return slot_idx


def append(prob, k, v, row0, k_new, v_new):
    """Rows [row0, row0 + m) of every head of the cache k, v take k_new, v_new
    [B, H, m, D] (Algorithm 1, generation phase)."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    prob.qkv(k, "k", dev, "k")
    prob.qkv(v, "v", dev, "v")
    m = k_new.shape[2]
    for t, name in ((k_new, "k_new"), (v_new, "v_new")):
        _gpu(t, name, dev, (prob.B, prob.H, m, prob.D), prob.torch_dtype, contiguous=True)
    _check(lib.nacl_append(prob.ref(), _ptr(k), _ptr(v), int(row0), _ptr(k_new), _ptr(v_new), int(m),
                           _stream(k.device)))


def evict(prob, q, k, v, C, Cr, sampling=SAMPLE_SOFTMAX, seed=0, layer=0, ws=None,
          scores=None, keep_idx=None, k_out=None, v_out=None, in_place=False):
    """score -> select -> compact on the current stream.  Returns
    (scores, keep_idx, k_out, v_out); with in_place the kept rows move to rows
    0..C-1 of each head of k and v, which are returned as k_out and v_out."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        prob.qkv(t, name, dev, name)
    if ws is None:
        ws = workspace(prob, dev)
    if scores is None:
        scores = torch.empty((prob.B, prob.H, prob.L), dtype=torch.float32, device=dev)
    if keep_idx is None:
        keep_idx = torch.empty((prob.B, prob.H, C), dtype=torch.int32, device=dev)
    if in_place:
        k_out, v_out = k, v
    else:
        if k_out is None:
            k_out = torch.empty((prob.B, prob.H, C, prob.D), dtype=k.dtype, device=dev)
        if v_out is None:
            v_out = torch.empty((prob.B, prob.H, C, prob.D), dtype=v.dtype, device=dev)
        for t, name in ((k_out, "k_out"), (v_out, "v_out")):
            _gpu(t, name, dev, (prob.B, prob.H, int(C), prob.D), prob.torch_dtype, contiguous=True)
    _gpu(ws, "ws", dev, dtype=torch.uint8, contiguous=True)
    _gpu(scores, "scores", dev, (prob.B, prob.H, prob.L), torch.float32, contiguous=True)
    _gpu(keep_idx, "keep_idx", dev, (prob.B, prob.H, int(C)), torch.int32, contiguous=True)
    _check(lib.nacl_evict(prob.ref(), _ptr(q), _ptr(k), _ptr(v), int(C), int(Cr), int(sampling),
                          int(seed), int(layer), _ptr(scores), _ptr(keep_idx), _ptr(k_out),
                          _ptr(v_out), _ptr(ws), ws.numel(), _stream(dev)))
    return scores, keep_idx, k_out, v_out


def evict_slots(prob, q, k, v, C, Cr, sampling=SAMPLE_SOFTMAX, seed=0, layer=0, ws=None,
                scores=None, keep_idx=None, slot_idx=None):
    """score -> select -> slot-form in-place update of k, v on the current
    stream (generation-phase eviction, Section 3).  Returns (scores, keep_idx,
    slot_idx): the ascending keep set and the old row each slot below C
    holds afterwards."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        prob.qkv(t, name, dev, name)
    if ws is None:
        ws = workspace(prob, dev)
    if scores is None:
        scores = torch.empty((prob.B, prob.H, prob.L), dtype=torch.float32, device=dev)
    if keep_idx is None:
        keep_idx = torch.empty((prob.B, prob.H, C), dtype=torch.int32, device=dev)
    if slot_idx is None:
        slot_idx = torch.empty((prob.B, prob.H, C), dtype=torch.int32, device=dev)
    _gpu(ws, "ws", dev, dtype=torch.uint8, contiguous=True)
    _gpu(scores, "scores", dev, (prob.B, prob.H, prob.L), torch.float32, contiguous=True)
    for t, name in ((keep_idx, "keep_idx"), (slot_idx, "slot_idx")):
        _gpu(t, name, dev, (prob.B, prob.H, int(C)), torch.int32, contiguous=True)
    _check(lib.nacl_evict_slots(prob.ref(), _ptr(q), _ptr(k), _ptr(v), int(C), int(Cr), int(sampling),
                                int(seed), int(layer), _ptr(scores), _ptr(keep_idx), _ptr(slot_idx),
                                _ptr(ws), ws.numel(), _stream(dev)))
    return scores, keep_idx, slot_idx


NOALLOC_WORKSPACE_MAX = 64 << 20


def evict_noalloc(prob, q, k, v, C, Cr, sampling=SAMPLE_SOFTMAX, seed=0, layer=0,
                  scores=None, keep_idx=None, k_out=None, v_out=None, health=None):
    """nacl_evict_noalloc: the same step with the library's built-in device
    scratch as workspace (no workspace argument).  prob must carry a device
    copy of the proxy positions.  health: optional int32 [2] GPU tensor that
    receives the call's health words.  Outputs must be given or are
    allocated here by torch before the call (the library allocates
    nothing)."""
    lib = load_library()
    dev = _gpu(k, "k", k.device).device
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        prob.qkv(t, name, dev, name)
    if scores is None:
        scores = torch.empty((prob.B, prob.H, prob.L), dtype=torch.float32, device=dev)
    if keep_idx is None:
        keep_idx = torch.empty((prob.B, prob.H, C), dtype=torch.int32, device=dev)
    if k_out is None:
        k_out = torch.empty((prob.B, prob.H, C, prob.D), dtype=k.dtype, device=dev)
    if v_out is None:
        v_out = torch.empty((prob.B, prob.H, C, prob.D), dtype=v.dtype, device=dev)
    _gpu(scores, "scores", dev, (prob.B, prob.H, prob.L), torch.float32, contiguous=True)
    _gpu(keep_idx, "keep_idx", dev, (prob.B, prob.H, int(C)), torch.int32, contiguous=True)
    if k_out is not k:
        for t, name in ((k_out, "k_out"), (v_out, "v_out")):
            _gpu(t, name, dev, (prob.B, prob.H, int(C), prob.D), prob.torch_dtype, contiguous=True)
    if health is not None:
        _gpu(health, "health", dev, (2,), torch.int32, contiguous=True)
    _check(lib.nacl_evict_noalloc(prob.ref(), _ptr(q), _ptr(k), _ptr(v), int(C), int(Cr), int(sampling),
                                  int(seed), int(layer), _ptr(scores), _ptr(keep_idx), _ptr(k_out),
                                  _ptr(v_out), _ptr(health), _stream(dev)))
    return scores, keep_idx, k_out, v_out


# The decoding step between two evictions (Algorithm 1, generation phase).

def _launch(dev, call, *args):
    """call(*args, stream) on dev's current stream, with dev the current device."""
    if dev.index == torch._C._cuda_getDevice():
        status = call(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = call(*args, _raw_stream(dev))
    if status != NACL_OK:
        _check(status)


def _like(t, name, dev, shape, dtype):
    """_gpu's checks of a contiguous tensor in one expression, for calls where
    the host's time counts; what does not pass is reported by _gpu."""
    if not (isinstance(t, torch.Tensor) and t.device == dev and t.shape == shape and t.dtype == dtype and t.is_contiguous()):
        _gpu(t, name, dev, shape, dtype, contiguous=True)


def _rows4(t, name, dev, shape, dtype):
    """A [., ., ., D] tensor with a contiguous last dimension; its strides."""
    if not (isinstance(t, torch.Tensor) and t.device == dev and t.shape == shape and t.dtype == dtype):
        _gpu(t, name, dev, shape, dtype)
    st = t.stride()
    if st[3] != 1:
        raise ValueError(f"{name} must have a contiguous last dimension")
    return st


def _cache(t, name, dev, step, strides):
    """A cache tensor of the step's problem."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == dev and t.shape == step.cache_shape and
            t.dtype == step.dtype and t.stride() == strides):
        _gpu(t, name, dev, step.cache_shape, step.dtype, strides[:3])


def _raw_stream(dev):
    return torch._C._cuda_getCurrentRawStream(dev.index)


class _Keeper:
    """Keeps tensors and their addresses between calls.  A tensor may get a new
    storage meanwhile (a module's parameters do when it is moved), so every call
    compares the addresses and has the tensors checked and taken again."""

    def _take(self):
        """Checks the tensors (before anything is changed), fills the struct and
        calls _keep."""
        raise NotImplementedError

    def _keep(self, *tensors):
        self._kept = tuple((t.data_ptr, t.data_ptr()) for t in tensors if t is not None)

    def current(self):
        for address, at in self._kept:
            if address() != at:
                self._take()
                break


class Step(_Keeper):
    """nacl_step: T new tokens per sequence, token t of sequence b in cache row
    row0 + lens[b] + t.  lens, n_new: optional int32 [B] GPU tensors, read when
    the calls run (a program may advance them in place)."""

    def __init__(self, prob, T=1, lens=None, row0=0, n_new=None):
        if not -2 ** 31 <= min(int(T), int(row0)) <= max(int(T), int(row0)) < 2 ** 31:
            raise ValueError("T and row0 must fit 32 bits")
        self.prob, self.T, self.lens, self.n_new = prob, int(T), lens, n_new
        B, H, L, D, Hq = prob.B, prob.H, prob.L, prob.D, prob.H * max(1, prob.q_group)
        self.dtype = prob.torch_dtype
        self.q_shape, self.new_shape = (B, Hq, self.T, D), (B, H, self.T, D)
        self.cache_shape = (B, H, L, D)
        self.fits = (H, D, self.dtype)
        self.k_stride, self.v_stride = tuple(prob.c.k_stride) + (1,), tuple(prob.c.v_stride) + (1,)
        s = _Step()
        s.T, s.row0 = self.T, int(row0)
        dense = (Hq * self.T * D, self.T * D, D)
        s.q_stride[:] = s.q_out_stride[:] = dense
        s.k_stride[:] = s.v_stride[:] = (H * self.T * D, self.T * D, D)
        self.c = s
        self._take()

    def _take(self):
        lens, n_new = self.lens, self.n_new
        for t, name in ((lens, "lens"), (n_new, "n_new")):
            if t is not None:
                _gpu(t, name, t.device, (self.prob.B,), torch.int32, contiguous=True)
        if lens is not None and n_new is not None and lens.device != n_new.device:
            raise ValueError("lens and n_new are on different devices")
        self.dev = next((t.device for t in (lens, n_new) if t is not None), None)
        self.c.lens = None if lens is None else lens.data_ptr()
        self.c.n_new = None if n_new is None else n_new.data_ptr()
        self._strided = {}  # nacl_step by the strides of the call's tensors
        self._keep(lens, n_new)

    def on(self, prob, dev):
        if prob is not self.prob:
            raise ValueError("the step was made for another problem")
        self.current()
        if self.dev is not None and self.dev != dev:
            raise ValueError(f"the step's lengths are on {self.dev}, the call runs on {dev}")

    def strided(self, q, k=None, v=None, q_out=None):
        key = (q, k, v, q_out)
        s = self._strided.get(key)
        if s is None:
            s = _Step.from_buffer_copy(self.c)
            for field, st in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("q_out_stride", q_out)):
                if st is not None:
                    getattr(s, field)[:] = st[:3]
            if len(self._strided) >= 64:
                self._strided.clear()
            self._strided[key] = s
        return s


class Rotation(_Keeper):
    """nacl_rotation: the angles' frequencies, inv_freq fp32 [rot / 2] (None: no
    rotation), the optional norm weights [D] of the problem's dtype, and how
    entries pair (interleaved: 2i with 2i + 1, else i with i + rot / 2)."""

    def __init__(self, prob, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
        self.inv_freq, self.q_weight, self.k_weight = inv_freq, q_weight, k_weight
        self.fits = (prob.D, prob.torch_dtype)
        self.c = _Rotation()
        self.c.interleaved, self.c.eps = int(bool(interleaved)), float(eps)
        self._take()

    def _take(self):
        inv_freq, q_weight, k_weight = self.inv_freq, self.q_weight, self.k_weight
        D, dtype = self.fits
        if inv_freq is not None:
            _gpu(inv_freq, "inv_freq", inv_freq.device, dtype=torch.float32, contiguous=True)
            if inv_freq.dim() != 1:
                raise ValueError("inv_freq must be one-dimensional")
        for t, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None:
                _gpu(t, name, t.device, (D,), dtype, contiguous=True)
        tensors = tuple(t for t in (inv_freq, q_weight, k_weight) if t is not None)
        dev = tensors[0].device if tensors else None
        if any(t.device != dev for t in tensors):
            raise ValueError("the rotation's tensors are on different devices")
        self.tensors, self.dev = tensors, dev
        r = self.c
        r.rot = 0 if inv_freq is None else 2 * inv_freq.numel()
        r.q_weight = None if q_weight is None else q_weight.data_ptr()
        r.k_weight = None if k_weight is None else k_weight.data_ptr()
        r.inv_freq = None if inv_freq is None else inv_freq.data_ptr()
        self._by_stride = {}  # nacl_rotation by pos_stride
        self._keep(*self.tensors)

    def with_stride(self, n):
        r = self._by_stride.get(n)
        if r is None:
            r = _Rotation.from_buffer_copy(self.c)
            r.pos_stride = n
            self._by_stride[n] = r
        return r


class Prefix(_Keeper):
    """nacl_prefix: k, v [G, H, L, D], shared by B / G consecutive sequences
    each; lens: optional int32 [G] rows in use."""

    def __init__(self, prob, k, v, lens=None):
        self.k, self.v, self.lens = k, v, lens
        self.fits = (prob.H, prob.D, prob.torch_dtype)
        self._take()

    def _take(self):
        k, v, lens = self.k, self.v, self.lens
        H, D, dtype = self.fits
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("the prefix's k must be [G, H, L, D]")
        G, _, L, _ = k.shape
        if max(G, L) >= 2 ** 31:
            raise ValueError("the prefix's groups and rows must fit 32 bits")
        x = _Prefix()
        x.G, x.L = G, L
        dev = _gpu(k, "the prefix's k", k.device).device
        x.k_stride[:] = _rows4(k, "the prefix's k", dev, (G, H, L, D), dtype)[:3]
        x.v_stride[:] = _rows4(v, "the prefix's v", dev, (G, H, L, D), dtype)[:3]
        if lens is not None:
            _gpu(lens, "the prefix's lens", dev, (G,), torch.int32, contiguous=True)
        x.k, x.v = k.data_ptr(), v.data_ptr()
        x.lens = None if lens is None else lens.data_ptr()
        self.c, self.dev = x, dev
        self._keep(k, v, lens)


def rotate_append(prob, step, rotation, positions, q_new, k_new, v_new, k, v, q_out=None):
    """The new tokens' queries and keys normalised and rotated, keys and values
    written into the cache k, v (include/nacl.h: nacl_rotate_append).  q_new
    [B, H*q_group, T, D], k_new, v_new [B, H, T, D] of any strides; positions
    int32 [B, T], or [T] shared by the batch.  Returns q_out (a new tensor, or
    the given one, which may be q_new)."""
    lib = _lib or load_library()
    dev = getattr(k, "device", None)
    _cache(k, "k", dev, step, step.k_stride)
    _cache(v, "v", dev, step, step.v_stride)
    step.on(prob, dev)
    if rotation.fits != step.fits[1:]:
        raise ValueError("the rotation was made for another head size or dtype")
    rotation.current()
    if rotation.dev is not None and rotation.dev != dev:
        raise ValueError(f"the rotation's tensors are on {rotation.dev}, the call runs on {dev}")
    dt = step.dtype
    if q_out is None:
        q_out = torch.empty(step.q_shape, dtype=dt, device=dev)
    s = step.strided(_rows4(q_new, "q_new", dev, step.q_shape, dt), _rows4(k_new, "k_new", dev, step.new_shape, dt),
                     _rows4(v_new, "v_new", dev, step.new_shape, dt), _rows4(q_out, "q_out", dev, step.q_shape, dt))
    pos = None
    if positions is not None:
        per_row = positions.dim() == 2
        _like(positions, "positions", dev, (prob.B, step.T) if per_row else (step.T,), torch.int32)
        pos = positions.data_ptr()
    r = rotation.with_stride(step.T if pos is not None and per_row else 0)
    _launch(dev, lib.nacl_rotate_append, prob.ref(), s, r, pos, q_new.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
            q_out.data_ptr(), k.data_ptr(), v.data_ptr())
    return q_out


def prefix_workspace(prob, step, prefix=None, device="cuda"):
    """A workspace for prefix_attention calls of these sizes."""
    lib = load_library()
    if prefix is not None:
        prefix.current()
    n = int(lib.nacl_prefix_workspace_bytes(prob.ref(), ctypes.byref(step.c),
                                            None if prefix is None else ctypes.byref(prefix.c)))
    if n == 0:
        raise NaclError(NACL_ERR_INVALID_ARG, lib.nacl_last_error_detail().decode())
    return torch.empty(n, dtype=torch.uint8, device=device)


def prefix_attention(prob, step, q, k, v, prefix=None, out=None, lse=None, ws=None):
    """Attention of the step's queries q [B, H*q_group, T, D] to the cache k, v
    (which holds the step's own tokens already) and to the prefix that groups of
    sequences share (include/nacl.h: nacl_prefix_attention).  Returns (out
    [B, H*q_group, T, D], lse [B, H*q_group, T] fp32); lse=False: no lse."""
    lib = _lib or load_library()
    dev = getattr(k, "device", None)
    _cache(k, "k", dev, step, step.k_stride)
    _cache(v, "v", dev, step, step.v_stride)
    step.on(prob, dev)
    if prefix is not None:
        prefix.current()
        if prefix.dev != dev or prefix.fits != step.fits:
            raise ValueError(f"the prefix is on {prefix.dev} with (heads, D, dtype) {prefix.fits}, the call's are on {dev} "
                             f"with {step.fits}")
    s = step.strided(_rows4(q, "q", dev, step.q_shape, step.dtype))
    if out is None:
        out = torch.empty(step.q_shape, dtype=step.dtype, device=dev)
    else:
        _like(out, "out", dev, step.q_shape, step.dtype)
    if lse is None:
        lse = torch.empty(step.q_shape[:3], dtype=torch.float32, device=dev)
    elif lse is False:
        lse = None
    else:
        _like(lse, "lse", dev, step.q_shape[:3], torch.float32)
    if ws is None:
        ws = prefix_workspace(prob, step, prefix, dev)
    n = ws.numel()
    _like(ws, "ws", dev, (n,), torch.uint8)
    _launch(dev, lib.nacl_prefix_attention, prob.ref(), s, None if prefix is None else prefix.c, q.data_ptr(), k.data_ptr(),
            v.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(), ws.data_ptr(), n)
    return out, lse


def _draw(N, V):
    if max(N, V) >= 2 ** 31:
        raise ValueError("N and V must fit 32 bits")
    d = _Draw()
    d.N, d.V, d.dtype, d.stride = int(N), int(V), NACL_F32, int(V)
    return d


def sample_workspace(N, V, device="cuda"):
    """A workspace for sample calls of N rows over a vocabulary of V, of either dtype."""
    lib = load_library()
    n = int(lib.nacl_sample_workspace_bytes(ctypes.byref(_draw(N, V))))
    if n == 0:
        raise NaclError(NACL_ERR_INVALID_ARG, lib.nacl_last_error_detail().decode())
    return torch.empty(n, dtype=torch.uint8, device=device)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, logprobs=None, ws=None):
    """The next token of every row of logits [N, V] (fp32 or bf16, any row stride)
    from uniform numbers u [N] in [0, 1) (include/nacl.h: nacl_sample).  The
    settings are [N] GPU tensors, top_k int32 and the others fp32.  Returns
    (tokens int32 [N], logprobs fp32 [N]); logprobs=False: no logprobs."""
    lib = _lib or load_library()
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be [N, V] of fp32 or bf16")
    N, V = logits.shape
    if max(N, V) >= 2 ** 31:
        raise ValueError("N and V must fit 32 bits")
    dev = logits.device
    if not logits.is_cuda:
        _gpu(logits, "logits", dev)
    stride, one = logits.stride()
    if V > 1 and one != 1:
        raise ValueError("logits must have a contiguous last dimension")
    if N > 1 and stride < V:
        raise ValueError("rows of logits must not overlap")
    rows = (N,)
    _like(u, "u", dev, rows, torch.float32)
    d = _Draw(N, V, NACL_F32 if logits.dtype == torch.float32 else NACL_BF16, stride if N > 1 else V)
    if temperature is not None:
        _like(temperature, "temperature", dev, rows, torch.float32)
        d.temperature = temperature.data_ptr()
    if top_k is not None:
        _like(top_k, "top_k", dev, rows, torch.int32)
        d.top_k = top_k.data_ptr()
    if top_p is not None:
        _like(top_p, "top_p", dev, rows, torch.float32)
        d.top_p = top_p.data_ptr()
    if min_p is not None:
        _like(min_p, "min_p", dev, rows, torch.float32)
        d.min_p = min_p.data_ptr()
    if tokens is None:
        tokens = torch.empty(rows, dtype=torch.int32, device=dev)
    else:
        _like(tokens, "tokens", dev, rows, torch.int32)
    if logprobs is None:
        logprobs = torch.empty(rows, dtype=torch.float32, device=dev)
    elif logprobs is False:
        logprobs = None
    else:
        _like(logprobs, "logprobs", dev, rows, torch.float32)
    if ws is None:
        ws = sample_workspace(N, V, dev)
    n = ws.numel()
    _like(ws, "ws", dev, (n,), torch.uint8)
    _launch(dev, lib.nacl_sample, d, logits.data_ptr(), u.data_ptr(), tokens.data_ptr(),
            None if logprobs is None else logprobs.data_ptr(), ws.data_ptr(), n)
    return tokens, logprobs
