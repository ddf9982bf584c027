"""ctypes binding of libspectrain.so: one Python function per C ABI entry point
(argument marshalling only; every step of the stage runs in the library).

Device buffers are passed as torch tensors (their data pointers) and streams
as torch.cuda.Stream objects; host arrays as float32 NumPy arrays.
"""
import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspectrain.so")

ABI_VERSION = 3
OK, EINVAL, ENOMEM, EHIP, ESTATE, ENONFINITE = range(6)
STATUS_NAMES = {OK: "OK", EINVAL: "EINVAL", ENOMEM: "ENOMEM", EHIP: "EHIP", ESTATE: "ESTATE",
                ENONFINITE: "ENONFINITE"}
FP32, BF16 = 0, 1
KIND_FC, KIND_CONV3X3, KIND_BOTTLENECK, KIND_TRANSFORMER, KIND_RESLSTM = range(5)
HEAD_NONE, HEAD_CE = 0, 1
POLICY_PREDICT, POLICY_STASH = 0, 1
POLICIES = ("spectrain", "vanilla", "stash")
KIND_BY_NAME = {"fc": KIND_FC, "conv3x3": KIND_CONV3X3, "bottleneck": KIND_BOTTLENECK,
                "transformer": KIND_TRANSFORMER, "reslstm": KIND_RESLSTM}

EXPORTED = ("spectrain_version_difference", "spectrain_stage_create", "spectrain_stage_num_params",
            "spectrain_stage_predict", "spectrain_stage_forward", "spectrain_stage_backward",
            "spectrain_stage_backward_noalloc", "spectrain_stage_forward_backward",
            "spectrain_stage_update", "spectrain_stage_get_state", "spectrain_stage_set_state",
            "spectrain_stage_get_predicted", "spectrain_stage_profile", "spectrain_stage_profile_read",
            "spectrain_stage_read_stash", "spectrain_stage_destroy", "spectrain_stage_set_attention",
            "spectrain_stage_set_masks", "spectrain_stage_set_stash", "spectrain_rotary",
            "spectrain_attention_workspace", "spectrain_attention_forward", "spectrain_attention_backward",
            "spectrain_checkpoint_pack", "spectrain_checkpoint_restore", "spectrain_last_error")
ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
CHECKPOINT_GROUP = 32
STASH_FORMATS = {"bf16": 0, "e4m3": 1}


class StageDesc(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_uint32), ("kind", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("head", ctypes.c_int32), ("stage_index", ctypes.c_int32), ("num_stages", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("num_layers", ctypes.c_int32), ("dims", ctypes.c_int32 * 8),
                ("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("weight_policy", ctypes.c_int32)]


class KernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", ctypes.c_int64), ("ms_total", ctypes.c_double),
                ("flops_total", ctypes.c_double), ("bytes_total", ctypes.c_double),
                ("extra_bytes_total", ctypes.c_double)]


class Strides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "dtype", "batch", "tokens", "heads", "head_dim", "rotary_dim", "layout", "scaling", "original_length",
        "first_position", "reserved")] + [("base", ctypes.c_double), ("factor", ctypes.c_double), ("x", Strides),
                                          ("out", Strides)]


class AttentionDesc(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "dtype", "batch", "heads", "kv_heads", "head_dim", "q_len", "kv_len", "q_offset", "causal")] + [
        ("scale", ctypes.c_float), ("cap", ctypes.c_float)] + [
        (n, Strides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]


class AttentionMasks(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("documents", "prefix", "kv_lengths", "slopes")]


class StageAttention(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_uint32), ("causal", ctypes.c_int32), ("cap", ctypes.c_float)] + [
        (n, ctypes.c_int32) for n in ("rotary_dim", "rotary_layout", "rotary_scaling", "rotary_original_length",
                                      "reserved")] + [("rotary_base", ctypes.c_double),
                                                      ("rotary_factor", ctypes.c_double)]


class SpecTrainError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib():
    """Open libspectrain.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_1809_02839_amd.build.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        fp = ctypes.POINTER(ctypes.c_float)
        sig = {
            "spectrain_version_difference": (i32, [i32, i32, i32]),
            "spectrain_stage_create": (ctypes.c_int, [ctypes.POINTER(StageDesc), fp, sz, vp, ctypes.POINTER(vp)]),
            "spectrain_stage_num_params": (ctypes.c_int, [vp, ctypes.POINTER(sz)]),
            "spectrain_stage_predict": (ctypes.c_int, [vp, i32, i32]),
            "spectrain_stage_forward": (ctypes.c_int, [vp, i64, vp, vp, vp, vp]),
            "spectrain_stage_backward": (ctypes.c_int, [vp, i64, vp, vp]),
            "spectrain_stage_backward_noalloc": (ctypes.c_int, [vp, i64, vp, vp]),
            "spectrain_stage_forward_backward": (ctypes.c_int, [vp, i64, vp, vp, vp, vp, i64, vp, vp]),
            "spectrain_stage_update": (ctypes.c_int, [vp, i32, i32]),
            "spectrain_stage_get_state": (ctypes.c_int, [vp, fp, fp]),
            "spectrain_stage_set_state": (ctypes.c_int, [vp, fp, fp]),
            "spectrain_stage_get_predicted": (ctypes.c_int, [vp, i32, fp]),
            "spectrain_stage_profile": (ctypes.c_int, [vp, i32]),
            "spectrain_stage_profile_read": (ctypes.c_int, [vp, ctypes.POINTER(KernelStat), i32,
                                                            ctypes.POINTER(i32)]),
            "spectrain_stage_read_stash": (ctypes.c_int, [vp, i64, i32, vp, sz, ctypes.POINTER(sz)]),
            "spectrain_stage_destroy": (ctypes.c_int, [vp]),
            "spectrain_stage_set_attention": (ctypes.c_int, [vp, ctypes.POINTER(StageAttention), fp]),
            "spectrain_stage_set_masks": (ctypes.c_int, [vp, i64, ctypes.POINTER(AttentionMasks)]),
            "spectrain_stage_set_stash": (ctypes.c_int, [vp, i32]),
            "spectrain_rotary": (ctypes.c_int, [ctypes.POINTER(RotaryDesc), vp, vp, i32, vp, vp]),
            "spectrain_attention_workspace": (ctypes.c_int, [ctypes.POINTER(AttentionDesc), i32, ctypes.POINTER(sz)]),
            "spectrain_attention_forward": (ctypes.c_int, [ctypes.POINTER(AttentionDesc),
                                                           ctypes.POINTER(AttentionMasks)] + [vp] * 6 + [sz, vp]),
            "spectrain_attention_backward": (ctypes.c_int, [ctypes.POINTER(AttentionDesc),
                                                            ctypes.POINTER(AttentionMasks)] + [vp] * 10 + [sz, vp]),
            "spectrain_checkpoint_pack": (ctypes.c_int, [i32, i64, i64, vp, i64, vp, vp, vp]),
            "spectrain_checkpoint_restore": (ctypes.c_int, [i32, i64, i64, vp, vp, vp, i64, vp]),
            "spectrain_last_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _check(code):
    if code != OK:
        raise SpecTrainError(code, lib().spectrain_last_error().decode())


def _fptr(a):
    return None if a is None else a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))


def _dptr(t, dtype=None, what="tensor"):
    """Device pointer of a torch tensor. The library reads raw pointers, so a
    host tensor, a strided view or the wrong element type is refused here
    rather than reaching a kernel."""
    if t is None:
        return None
    if not getattr(t, "is_cuda", False):
        raise ValueError(f"{what} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if dtype is not None and str(t.dtype) != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def version_difference(k: int, N: int, forward: bool) -> int:
    return int(lib().spectrain_version_difference(k, N, 1 if forward else 0))


def policy_versions(policy: str, k: int, N: int):
    """(s before a forward, s before a backward) of stage k of N: Eq. 5 and
    Eq. 6 for SpecTrain; 0 for both under the Vanilla and stashing policies
    (every pass starts from the latest weights; with stashing the backward
    then reads the copy its forward used)."""
    if policy == "spectrain":
        return version_difference(k, N, True), version_difference(k, N, False)
    if policy in ("vanilla", "stash"):
        return 0, 0
    raise ValueError(f"unknown policy {policy!r}")


def make_desc(kind, dtype, head, stage_index, num_stages, batch, num_layers, dims, lr, momentum,
              weight_policy=POLICY_PREDICT) -> StageDesc:
    d = StageDesc()
    d.abi_version = ABI_VERSION
    d.kind = KIND_BY_NAME[kind] if isinstance(kind, str) else int(kind)
    d.dtype = {"fp32": FP32, "bf16": BF16}[dtype] if isinstance(dtype, str) else int(dtype)
    d.head = {"none": HEAD_NONE, "ce": HEAD_CE}[head] if isinstance(head, str) else int(head)
    d.stage_index, d.num_stages, d.batch, d.num_layers = stage_index, num_stages, batch, num_layers
    for i, v in enumerate(dims):
        d.dims[i] = int(v)
    d.lr, d.momentum = lr, momentum
    d.weight_policy = int(weight_policy)
    return d


def desc_from_spec(spec) -> StageDesc:
    policy = getattr(spec, "policy", "spectrain")
    if policy not in POLICIES:
        raise ValueError(f"unknown policy {policy!r}")
    return make_desc(spec.kind, spec.dtype, spec.head, spec.stage_index, spec.num_stages, spec.batch,
                     spec.num_layers, spec.dims, spec.lr, spec.momentum,
                     POLICY_STASH if policy == "stash" else POLICY_PREDICT)


class Stage:
    """Owner of one spectrain_stage_t; methods map 1:1 to the C entry points."""

    def __init__(self, desc: StageDesc, W0: np.ndarray, stream=None):
        W0 = np.ascontiguousarray(W0, dtype=np.float32)
        self._stream = stream
        handle = ctypes.c_void_p()
        sptr = ctypes.c_void_p(stream.cuda_stream) if stream is not None else None
        _check(lib().spectrain_stage_create(ctypes.byref(desc), _fptr(W0), W0.size, sptr, ctypes.byref(handle)))
        self.h = handle
        self.desc = desc
        n = ctypes.c_size_t()
        _check(lib().spectrain_stage_num_params(self.h, ctypes.byref(n)))
        self.n_params = n.value

    def predict(self, s: int, slot: int):
        _check(lib().spectrain_stage_predict(self.h, s, slot))

    @property
    def _act(self):
        return "torch.bfloat16" if self.desc.dtype == BF16 else "torch.float32"

    def forward(self, mb: int, x, y=None, labels=None, loss=None):
        a = self._act
        _check(lib().spectrain_stage_forward(self.h, mb, _dptr(x, a, "x"), _dptr(y, a, "y"),
                                             _dptr(labels, "torch.int32", "labels"),
                                             _dptr(loss, "torch.float32", "loss")))

    def backward(self, mb: int, dy=None, dx=None):
        a = self._act
        _check(lib().spectrain_stage_backward(self.h, mb, _dptr(dy, a, "dy"), _dptr(dx, a, "dx")))

    def backward_noalloc(self, mb: int, dy=None, dx=None):
        a = self._act
        _check(lib().spectrain_stage_backward_noalloc(self.h, mb, _dptr(dy, a, "dy"), _dptr(dx, a, "dx")))

    def forward_backward(self, mb_fwd: int, x, y, mb_bwd: int, dy=None, dx=None, labels=None, loss=None):
        """forward(mb_fwd) then backward(mb_bwd), the two passes running concurrently."""
        a = self._act
        _check(lib().spectrain_stage_forward_backward(self.h, mb_fwd, _dptr(x, a, "x"), _dptr(y, a, "y"),
                                                      _dptr(labels, "torch.int32", "labels"),
                                                      _dptr(loss, "torch.float32", "loss"), mb_bwd,
                                                      _dptr(dy, a, "dy"), _dptr(dx, a, "dx")))

    def update(self, s_next_fwd: int, s_next_bwd: int):
        _check(lib().spectrain_stage_update(self.h, s_next_fwd, s_next_bwd))

    def get_state(self):
        W = np.empty(self.n_params, np.float32)
        v = np.empty(self.n_params, np.float32)
        _check(lib().spectrain_stage_get_state(self.h, _fptr(W), _fptr(v)))
        return W, v

    def set_state(self, W: np.ndarray, v=None):
        W = np.ascontiguousarray(W, dtype=np.float32)
        v = None if v is None else np.ascontiguousarray(v, dtype=np.float32)
        _check(lib().spectrain_stage_set_state(self.h, _fptr(W), _fptr(v)))

    def get_predicted(self, slot: int):
        out = np.empty(self.n_params, np.float32)
        _check(lib().spectrain_stage_get_predicted(self.h, slot, _fptr(out)))
        return out

    def read_stash(self, mb: int, index: int) -> np.ndarray:
        """Stash buffer `index` of mini-batch mb (in flight) as raw bytes
        (uint8; empty when the stage does not use that index)."""
        n = ctypes.c_size_t()
        _check(lib().spectrain_stage_read_stash(self.h, mb, index, None, 0, ctypes.byref(n)))
        out = np.empty(n.value, np.uint8)
        if n.value:
            _check(lib().spectrain_stage_read_stash(self.h, mb, index, ctypes.c_void_p(out.ctypes.data), out.size,
                                                    ctypes.byref(n)))
        return out

    def set_attention(self, causal=False, cap=0.0, slopes=None, rotary_dim=0, rotary_layout="half",
                      rotary_base=10000.0, rotary_scaling="none", rotary_factor=1.0, rotary_original_length=0):
        """Positions and masks of a transformer stage (slopes: `heads` values on the host)."""
        a = StageAttention(ABI_VERSION, int(bool(causal)), cap, rotary_dim, ROTARY_LAYOUTS[rotary_layout],
                           ROTARY_SCALINGS[rotary_scaling], rotary_original_length, 0, rotary_base, rotary_factor)
        s = None if slopes is None else np.ascontiguousarray(slopes, dtype=np.float32)
        if s is not None and s.shape != (self.desc.dims[1],):
            raise ValueError(f"slopes must have {self.desc.dims[1]} values")
        _check(lib().spectrain_stage_set_attention(self.h, ctypes.byref(a), _fptr(s)))

    def clear_attention(self):
        """Back to attention without positions and masks."""
        _check(lib().spectrain_stage_set_attention(self.h, None, None))

    def set_masks(self, mb: int, documents=None, prefix=None, kv_lengths=None):
        """Masks of mini-batch mb for its coming forward and its backward; int32
        device tensors, kept alive by the caller until the backward."""
        B, S = self.desc.batch, self.desc.dims[3]
        for t, shape, what in ((documents, (B, S), "documents"), (prefix, (B,), "prefix"),
                               (kv_lengths, (B,), "kv_lengths")):
            if t is not None and tuple(t.shape) != shape:
                raise ValueError(f"{what} must have shape {shape}")
        i32 = "torch.int32"
        m = AttentionMasks(_dptr(documents, i32, "documents"), _dptr(prefix, i32, "prefix"),
                           _dptr(kv_lengths, i32, "kv_lengths"), None)
        _check(lib().spectrain_stage_set_masks(self.h, mb, ctypes.byref(m)))

    def set_stash(self, format: str):
        """How activations of mini-batches in flight are kept: "bf16" or "e4m3"."""
        _check(lib().spectrain_stage_set_stash(self.h, STASH_FORMATS[format]))

    def configure(self, spec):
        """The attention and stash of a spec that names them (synth.StageSpec)."""
        attention = getattr(spec, "attention", None)
        if attention is not None:
            o = dict(vars(attention))
            o["slopes"] = attention.slope_values(spec.dims[1]) if o.pop("slopes") else None
            self.set_attention(**o)
        if getattr(spec, "stash", "bf16") != "bf16":
            self.set_stash(spec.stash)

    def profile(self, enable: bool, serial: bool = False):
        """Time every launch (serial: each on the stage stream, one at a time)."""
        _check(lib().spectrain_stage_profile(self.h, (2 if serial else 1) if enable else 0))

    def profile_read(self):
        """{family: dict(launches, ms_total, flops_total, bytes_total, extra_bytes_total)} in first-launch order."""
        cap = 64
        arr = (KernelStat * cap)()
        n = ctypes.c_int32()
        _check(lib().spectrain_stage_profile_read(self.h, arr, cap, ctypes.byref(n)))
        return {arr[i].name.decode(): dict(launches=arr[i].launches, ms_total=arr[i].ms_total,
                                           flops_total=arr[i].flops_total, bytes_total=arr[i].bytes_total,
                                           extra_bytes_total=arr[i].extra_bytes_total)
                for i in range(min(n.value, cap))}

    def destroy(self):
        if self.h is not None and self.h.value:
            _check(lib().spectrain_stage_destroy(self.h))
        self.h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---- operators ----

def _dtype_code(t, what):
    name = str(t.dtype)
    if name == "torch.bfloat16":
        return BF16
    if name == "torch.float32":
        return FP32
    raise ValueError(f"{what} must be torch.bfloat16 or torch.float32, got {t.dtype}")


def _on(device, stream, entry, *args):
    """entry(*args, stream pointer) with `device` current, on `stream` (None: the device's current torch stream)."""
    import torch
    if device.type != "cuda":
        raise ValueError("operators take GPU tensors")
    # the current stream's pointer without a Stream object, half of a small call's host time
    raw = torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream
    if device.index == torch.cuda.current_device():
        _check(entry(*args, raw))
        return
    with torch.cuda.device(device):
        _check(entry(*args, raw))


def _heads4(t, shape, dtype, device, what):
    """Pointer of a [batch, token, head, head_dim] tensor, after its checks."""
    if t.device != device:
        raise ValueError(f"{what} must be on {device}, got {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if shape[3] > 1 and t.stride(3) != 1:
        raise ValueError(f"{what} must be contiguous in its last dimension")
    return t.data_ptr()


def _strides(t):
    """The strides of a [batch, token, head, head_dim] tensor; of a single element any would do, and torch keeps odd ones."""
    return Strides(*[0 if n == 1 else s for n, s in zip(t.shape[:3], t.stride())])


def _side(t, shape, dtype, device, what):
    """Pointer of a contiguous side input (None: absent)."""
    if t is None:
        return None
    if t.device != device or str(t.dtype) != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} {tuple(shape)} on {device}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class Rotary:
    """Rotary positions of heads of one width (spectrain_rotary): layout "half"
    or "interleaved"; scaling "none", "linear", "ntk" or "parts"."""

    def __init__(self, head_dim, rotary_dim=None, layout="half", base=10000.0, scaling="none", factor=1.0,
                 original_length=0):
        d = RotaryDesc()
        d.abi_version = ABI_VERSION
        d.head_dim = head_dim
        d.rotary_dim = head_dim if rotary_dim is None else rotary_dim
        d.layout, d.scaling = ROTARY_LAYOUTS[layout], ROTARY_SCALINGS[scaling]
        d.base, d.factor, d.original_length = base, factor, original_length
        self._d = d
        self._last = (None, None)   # layout of the last call and its descriptor, which no later call changes

    def apply(self, x, out=None, positions=None, first_position=0, inverse=False, stream=None):
        """Turn x [batch, token, head, head_dim] into out (None: in place; any
        strides with a contiguous last dimension). positions: int32 [batch,
        token], else first_position + token. Returns out."""
        out = x if out is None else out
        if x.dim() != 4 or x.shape[3] != self._d.head_dim:
            raise ValueError(f"x must be [batch, token, head, {self._d.head_dim}], got {tuple(x.shape)}")
        xp = _heads4(x, x.shape, x.dtype, x.device, "x")
        op = _heads4(out, x.shape, x.dtype, x.device, "out")
        pp = _side(positions, x.shape[:2], "torch.int32", x.device, "positions")
        layout = (x.shape, x.stride(), out.stride(), x.dtype, first_position)
        last, d = self._last
        if layout != last:   # a new one: another thread's call may be reading the old
            d = RotaryDesc.from_buffer_copy(self._d)
            d.dtype = _dtype_code(x, "x")
            d.batch, d.tokens, d.heads = x.shape[:3]
            d.x, d.out = _strides(x), _strides(out)
            d.first_position = first_position
            self._last = (layout, d)
        _on(x.device, stream, lib().spectrain_rotary, ctypes.byref(d), xp, pp, 1 if inverse else 0, op)
        return out


class Attention:
    """Masked attention of one shape (spectrain_attention_forward and
    _backward). Tensors are [batch, token, head, head_dim] bf16 with any strides
    whose last is 1; scale None is 1 / sqrt(head_dim). The masks (each may be
    None) are documents int32 [batch, kv_len], prefix and kv_lengths int32
    [batch], slopes float32 [heads]."""

    def __init__(self, batch, heads, kv_heads, head_dim, q_len, kv_len, causal=False, q_offset=0, scale=None, cap=0.0):
        d = AttentionDesc()
        d.abi_version, d.dtype = ABI_VERSION, BF16
        d.batch, d.heads, d.kv_heads, d.head_dim, d.q_len, d.kv_len = batch, heads, kv_heads, head_dim, q_len, kv_len
        d.q_offset, d.causal = q_offset, int(bool(causal))
        d.scale = head_dim ** -0.5 if scale is None else scale
        d.cap = cap
        self._d = d
        self._last = {}   # forward, backward: strides of the last call and its descriptor, which no later call changes
        self._qs, self._ks = (batch, q_len, heads, head_dim), (batch, kv_len, kv_heads, head_dim)

    def workspace_bytes(self, backward=False):
        n = ctypes.c_size_t()
        _check(lib().spectrain_attention_workspace(ctypes.byref(self._d), int(bool(backward)), ctypes.byref(n)))
        return n.value

    def workspace(self, backward=False, device="cuda"):
        """A workspace for this shape's calls: one for calls that follow each other on a stream."""
        import torch
        return torch.empty(max(256, self.workspace_bytes(backward)), dtype=torch.uint8, device=device)

    def _described(self, pass_, tensors, q):
        """Pointers of (name, tensor, shape), after their checks, and the descriptor with their strides."""
        import torch
        ptr = [_heads4(t, shape, torch.bfloat16, q.device, name) for name, t, shape in tensors]
        strides = tuple([t.stride() for _, t, _ in tensors])
        last, d = self._last.get(pass_, (None, None))
        if strides != last:   # a new one: another thread's call may be reading the old
            d = AttentionDesc.from_buffer_copy(self._d)
            for name, t, _ in tensors:
                setattr(d, name, _strides(t))
            self._last[pass_] = (strides, d)
        return ptr, d

    def _masks(self, device, documents, prefix, kv_lengths, slopes):
        d = self._d
        return AttentionMasks(_side(documents, (d.batch, d.kv_len), "torch.int32", device, "documents"),
                              _side(prefix, (d.batch,), "torch.int32", device, "prefix"),
                              _side(kv_lengths, (d.batch,), "torch.int32", device, "kv_lengths"),
                              _side(slopes, (d.heads,), "torch.float32", device, "slopes"))

    def _scratch(self, workspace, device):
        if workspace.device != device or not workspace.is_contiguous():
            raise ValueError(f"workspace must be contiguous and on {device}")
        return workspace.data_ptr(), workspace.numel() * workspace.element_size()

    def forward(self, q, k, v, out, lse=None, *, workspace, documents=None, prefix=None, kv_lengths=None, slopes=None,
                stream=None):
        """out = attention(q, k, v); lse float32 [batch, heads, q_len] as the backward takes it (None: not wanted)."""
        dev = q.device
        ptr, d = self._described("forward", (("q", q, self._qs), ("k", k, self._ks), ("v", v, self._ks),
                                             ("out", out, self._qs)), q)
        lp = _side(lse, (d.batch, d.heads, d.q_len), "torch.float32", dev, "lse")
        m = self._masks(dev, documents, prefix, kv_lengths, slopes)
        wp, wn = self._scratch(workspace, dev)
        _on(dev, stream, lib().spectrain_attention_forward, ctypes.byref(d), ctypes.byref(m), *ptr, lp, wp, wn)

    def backward(self, q, k, v, out, lse, dout, dq, dk, dv, *, workspace, documents=None, prefix=None, kv_lengths=None,
                 slopes=None, stream=None):
        """dq, dk, dv (overwritten) from the forward's tensors and masks and dout."""
        dev, qs, ks = q.device, self._qs, self._ks
        ptr, d = self._described("backward", (
            ("q", q, qs), ("k", k, ks), ("v", v, ks), ("out", out, qs), ("dout", dout, qs), ("dq", dq, qs),
            ("dk", dk, ks), ("dv", dv, ks)), q)
        lp = _side(lse, (d.batch, d.heads, d.q_len), "torch.float32", dev, "lse")
        m = self._masks(dev, documents, prefix, kv_lengths, slopes)
        wp, wn = self._scratch(workspace, dev)
        _on(dev, stream, lib().spectrain_attention_backward, ctypes.byref(d), ctypes.byref(m), *ptr[:4], lp,
            *ptr[4:], wp, wn)


def _checkpoint_args(t, codes, scales, what):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be [rows, cols] with a contiguous last dimension")
    rows, cols = t.shape
    cp = _side(codes, (rows, cols), "torch.uint8", t.device, "codes")
    sp = _side(scales, (rows, -(-cols // CHECKPOINT_GROUP)), "torch.uint8", t.device, "scales")
    if cp is None or sp is None:
        raise ValueError("codes and scales must be given")
    return _dtype_code(t, what), rows, cols, cp, sp, t.stride(0) if rows > 1 else max(cols, 1)


def checkpoint_pack(x, codes, scales, stream=None):
    """x [rows, cols] to 8-bit codes uint8 [rows, cols] and scales uint8 [rows, ceil(cols / 32)]."""
    dt, rows, cols, cp, sp, ld = _checkpoint_args(x, codes, scales, "x")
    xp = x.data_ptr()
    _on(x.device, stream, lib().spectrain_checkpoint_pack, dt, rows, cols, xp, ld, cp, sp)


def checkpoint_restore(codes, scales, out, stream=None):
    """The values that codes and scales stand for, into out [rows, cols]."""
    dt, rows, cols, cp, sp, ld = _checkpoint_args(out, codes, scales, "out")
    op = out.data_ptr()
    _on(out.device, stream, lib().spectrain_checkpoint_restore, dt, rows, cols, cp, sp, op, ld)
