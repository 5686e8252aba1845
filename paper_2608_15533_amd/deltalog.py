"""ctypes binding of libdeltalog.so -- argument marshalling only.

The entry points keep the C names (``dl_eager_step``, ``dl_append_step``, ``dl_merge``,
``dl_readout``; for whole sequences ``dl_chunk_tables``, ``dl_prefill``,
``dl_prefill_backward``; around a recurrence ``dl_conv_*``, ``dl_ssm_*``,
``dl_qk_norm``, ``dl_qk_norm_backward``) and take torch CUDA tensors; each call checks layouts, builds the C
structs and calls the library, which launches the HIP kernels on the current (or the
given) stream.  No arithmetic of the method happens here.  PyTorch is used only to
own device memory and to name the stream.

Importing this module loads the library and raises ImportError when it has not been
built -- there is no fallback path.
"""

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# DELTALOG_LIB selects another build of the same library (e.g. a tuning variant).
LIB_PATH = os.environ.get("DELTALOG_LIB") or os.path.join(_HERE, "libdeltalog.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2608_15533_amd.build` "
        "(the DeltaLog path has no non-HIP fallback)")

_lib = ctypes.CDLL(LIB_PATH)

# ----------------------------------------------------------------- constants (deltalog.h)
DL_ABI_VERSION = 4
DL_MAX_MERGE_INTERVAL = 64
DL_OK, DL_E_NULL, DL_E_SHAPE, DL_E_DTYPE, DL_E_ALIGN, DL_E_UNSUPPORTED, DL_E_HIP, DL_E_VERSION = (
    0, -1, -2, -3, -4, -5, -6, -7)
DL_E_SCRATCH = -8
DL_NOALLOC_SCRATCH_BYTES = 4 << 20
DL_CHUNK, DL_MAX_HEADS = 32, 65536
DL_MAX_STRIDE = 1 << 24
DL_OP_GDN, DL_OP_KDA, DL_OP_RWKV6, DL_OP_LINATTN, DL_OP_RETNET, DL_OP_GLA = 0, 1, 2, 3, 4, 5
DL_F32, DL_BF16 = 0, 1
OP_IDS = {"gdn": DL_OP_GDN, "kda": DL_OP_KDA, "rwkv6": DL_OP_RWKV6, "linattn": DL_OP_LINATTN,
          "retnet": DL_OP_RETNET, "gla": DL_OP_GLA}
DELTA_OP_IDS = (DL_OP_GDN, DL_OP_KDA)                  # b = beta (v - correction); needs beta
PER_KEY_OP_IDS = (DL_OP_KDA, DL_OP_RWKV6, DL_OP_GLA)   # lambda is [.., dk]; else one per head
DTYPE_IDS = {"f32": DL_F32, "bf16": DL_BF16}
DL_ACT_NONE, DL_ACT_SILU = 0, 1
ACTIVATION_IDS = {"none": DL_ACT_NONE, "silu": DL_ACT_SILU}
NORM_IDS = {"none": 0, "l2": 1, "rms": 2}
TURN_IDS = {"none": 0, "halves": 1, "pairs": 2}
TORCH_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

EXPORTED = ("dl_eager_step", "dl_append_step", "dl_merge", "dl_readout",
            "dl_append_step_tiled", "dl_tiled_workspace_bytes", "dl_status_str",
            "dl_abi_version", "dl_build_flags", "dl_append_step_tiled_noalloc",
            "dl_chunk_tables", "dl_prefill_workspace_bytes", "dl_prefill",
            "dl_prefill_backward",
            "dl_conv_step", "dl_conv_prefill", "dl_conv_workspace_bytes", "dl_conv_backward",
            "dl_qk_norm", "dl_qk_workspace_bytes", "dl_qk_norm_backward",
            "dl_ssm_step", "dl_ssm_prefill", "dl_ssm_workspace_bytes", "dl_ssm_backward")


class dl_desc(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_int32), ("op", ctypes.c_int32),
                ("num_slots", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("dk", ctypes.c_int32), ("dv", ctypes.c_int32),
                ("merge_interval", ctypes.c_int32), ("in_dtype", ctypes.c_int32),
                ("u_log_dtype", ctypes.c_int32), ("state_dtype", ctypes.c_int32)]


class dl_state(ctypes.Structure):
    _fields_ = [("S", ctypes.c_void_p), ("k_log", ctypes.c_void_p),
                ("u_log", ctypes.c_void_p), ("lam_log", ctypes.c_void_p),
                ("len", ctypes.c_void_p), ("err", ctypes.c_void_p)]


class dl_token(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("beta", ctypes.c_void_p), ("lam", ctypes.c_void_p), ("u", ctypes.c_void_p)]


class dl_tables(ctypes.Structure):
    _fields_ = [("cu_tokens", ctypes.c_void_p), ("cu_chunks", ctypes.c_void_p),
                ("chunks", ctypes.c_void_p), ("row_slot", ctypes.c_void_p),
                ("seq_slot", ctypes.c_void_p), ("order", ctypes.c_void_p)]


class dl_grads(ctypes.Structure):
    _fields_ = [("dq", ctypes.c_void_p), ("dk", ctypes.c_void_p), ("dv", ctypes.c_void_p),
                ("dbeta", ctypes.c_void_p), ("dlam", ctypes.c_void_p), ("du", ctypes.c_void_p),
                ("dS", ctypes.c_void_p)]


class dl_conv_desc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("abi_version", "num_slots", "channels", "width",
                                              "activation", "in_dtype")]


class dl_conv_rows(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("w", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class dl_conv_grads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("dx", "dw", "dbias", "ds")]


class dl_qk_desc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("abi_version", "heads", "head_dim", "rep", "norm",
                                              "turn", "rot", "in_dtype")]
    _fields_ += [("eps", ctypes.c_float), ("q_scale", ctypes.c_float)]


class dl_qk_rows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64)]
    _fields_ += [(k, ctypes.c_void_p) for k in ("pos", "freq", "wq", "wk", "used")]


class dl_qk_grads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("dq", "dk", "dwq", "dwk")]


class dl_ssm_desc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("abi_version", "num_slots", "channels", "states",
                                              "in_dtype")]


class dl_ssm_rows(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("x", "dt", "z", "B", "C")]
    _fields_ += [(k, ctypes.c_int64) for k in ("x_stride", "dt_stride", "z_stride", "b_stride",
                                               "c_stride")]
    _fields_ += [(k, ctypes.c_void_p) for k in ("A", "skip", "dt_bias")]


class dl_ssm_grads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("dx", "ddt", "dz", "dB", "dC", "dA", "dskip",
                                               "dbias", "ds")]


_P = ctypes.c_void_p
_lib.dl_eager_step.argtypes = [ctypes.POINTER(dl_desc), _P, ctypes.POINTER(dl_token), _P, _P,
                               ctypes.c_int32, _P]
_lib.dl_append_step.argtypes = [ctypes.POINTER(dl_desc), ctypes.POINTER(dl_state),
                                ctypes.POINTER(dl_token), _P, _P, ctypes.c_int32, _P]
_lib.dl_merge.argtypes = [ctypes.POINTER(dl_desc), ctypes.POINTER(dl_state),
                          ctypes.POINTER(dl_token), _P, _P, ctypes.c_int32, _P]
_lib.dl_readout.argtypes = [ctypes.POINTER(dl_desc), ctypes.POINTER(dl_state), _P, _P, _P,
                            ctypes.c_int32, _P]
_lib.dl_append_step_tiled.argtypes = [ctypes.POINTER(dl_desc), ctypes.POINTER(dl_state),
                                      ctypes.POINTER(dl_token), _P, _P, ctypes.c_int32,
                                      ctypes.c_int32, ctypes.c_int32, _P, ctypes.c_size_t, _P]
_lib.dl_tiled_workspace_bytes.argtypes = [ctypes.POINTER(dl_desc), ctypes.c_int32,
                                          ctypes.POINTER(ctypes.c_size_t)]
_lib.dl_append_step_tiled_noalloc.argtypes = [ctypes.POINTER(dl_desc), ctypes.POINTER(dl_state),
                                              ctypes.POINTER(dl_token), _P, _P, ctypes.c_int32,
                                              ctypes.c_int32, _P]
_lib.dl_chunk_tables.argtypes = [_P, _P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                 ctypes.POINTER(dl_tables), _P, _P]
_lib.dl_prefill_workspace_bytes.argtypes = [ctypes.POINTER(dl_desc), ctypes.c_int32,
                                            ctypes.c_int32, ctypes.c_int32,
                                            ctypes.POINTER(ctypes.c_size_t)]
_lib.dl_prefill.argtypes = [ctypes.POINTER(dl_desc), _P, _P, ctypes.POINTER(dl_token), _P,
                            ctypes.POINTER(dl_tables), ctypes.c_int32, ctypes.c_int32, _P,
                            ctypes.c_size_t, _P]
_lib.dl_prefill_backward.argtypes = [ctypes.POINTER(dl_desc), _P, ctypes.POINTER(dl_token), _P,
                                     _P, ctypes.POINTER(dl_grads), ctypes.POINTER(dl_tables),
                                     ctypes.c_int32, ctypes.c_int32, _P, ctypes.c_size_t, _P]
_I, _PTR, _SIZE = ctypes.c_int32, ctypes.POINTER, ctypes.c_size_t
_lib.dl_conv_step.argtypes = [_PTR(dl_conv_desc), _P, _P, _PTR(dl_conv_rows), _P, _P, _I, _P]
_lib.dl_conv_prefill.argtypes = [_PTR(dl_conv_desc), _P, _P, _PTR(dl_conv_rows), _P,
                                 _PTR(dl_tables), _I, _I, _P]
_lib.dl_conv_workspace_bytes.argtypes = [_PTR(dl_conv_desc), _I, _I, _PTR(_SIZE)]
_lib.dl_conv_backward.argtypes = [_PTR(dl_conv_desc), _P, _PTR(dl_conv_rows), _P, _P,
                                  _PTR(dl_conv_grads), _PTR(dl_tables), _I, _I, _P, _SIZE, _P]
_lib.dl_qk_norm.argtypes = [_PTR(dl_qk_desc), _PTR(dl_qk_rows), _P, _P, _I, _P]
_lib.dl_qk_workspace_bytes.argtypes = [_PTR(dl_qk_desc), _I, _PTR(_SIZE)]
_lib.dl_qk_norm_backward.argtypes = [_PTR(dl_qk_desc), _PTR(dl_qk_rows), _P, _P, _PTR(dl_qk_grads),
                                     _I, _P, _SIZE, _P]
_lib.dl_ssm_step.argtypes = [_PTR(dl_ssm_desc), _P, _P, _PTR(dl_ssm_rows), _P, _P, _I, _P]
_lib.dl_ssm_workspace_bytes.argtypes = [_PTR(dl_ssm_desc), _I, _I, _I, _PTR(_SIZE)]
_lib.dl_ssm_prefill.argtypes = [_PTR(dl_ssm_desc), _P, _P, _PTR(dl_ssm_rows), _P, _PTR(dl_tables),
                                _I, _I, _P, _SIZE, _P]
_lib.dl_ssm_backward.argtypes = [_PTR(dl_ssm_desc), _P, _PTR(dl_ssm_rows), _P, _P,
                                 _PTR(dl_ssm_grads), _PTR(dl_tables), _I, _I, _P, _SIZE, _P]
for _f in ("dl_eager_step", "dl_append_step", "dl_merge", "dl_readout", "dl_append_step_tiled",
           "dl_tiled_workspace_bytes", "dl_abi_version", "dl_append_step_tiled_noalloc",
           "dl_chunk_tables", "dl_prefill_workspace_bytes", "dl_prefill",
           "dl_prefill_backward", "dl_conv_step", "dl_conv_prefill", "dl_conv_workspace_bytes",
           "dl_conv_backward", "dl_qk_norm", "dl_qk_workspace_bytes", "dl_qk_norm_backward",
           "dl_ssm_step", "dl_ssm_workspace_bytes", "dl_ssm_prefill", "dl_ssm_backward"):
    getattr(_lib, _f).restype = ctypes.c_int
_lib.dl_status_str.argtypes = [ctypes.c_int]
_lib.dl_status_str.restype = ctypes.c_char_p
_lib.dl_build_flags.argtypes = []
_lib.dl_build_flags.restype = ctypes.c_char_p

lib = _lib


class DeltaLogError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {dl_status_str(status)} ({status})")


def dl_status_str(status):
    return _lib.dl_status_str(int(status)).decode()


def dl_abi_version():
    return _lib.dl_abi_version()


def dl_build_flags():
    return _lib.dl_build_flags().decode()


if dl_abi_version() != DL_ABI_VERSION:
    raise ImportError(f"libdeltalog ABI {dl_abi_version()} != binding ABI {DL_ABI_VERSION}")


# ----------------------------------------------------------------- descriptors
def make_desc(op, B, H, dk, dv, M, in_dtype="bf16", state_dtype="f32"):
    """dl_desc for operator ``op`` (a key of ``OP_IDS``) with merge interval M."""
    u_dtype = "f32" if OP_IDS[op] in DELTA_OP_IDS else in_dtype
    return dl_desc(DL_ABI_VERSION, OP_IDS[op], B, H, dk, dv, M, DTYPE_IDS[in_dtype],
                   DTYPE_IDS[u_dtype], DTYPE_IDS[state_dtype])


def state_torch_dtype(desc):
    return torch.bfloat16 if desc.state_dtype == DL_BF16 else torch.float32


def decay_width(desc):
    """Width of lambda, ell and the Lam_log snapshots: dk (per-key decay) or 1 (one value
    per head); 0 for linear attention, which has no decay."""
    if desc.op == DL_OP_LINATTN:
        return 0
    return desc.dk if desc.op in PER_KEY_OP_IDS else 1


def _ptr(t):
    return None if t is None else t.data_ptr()


def _need(t, name, dtype, shape, device=None):
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.shape != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class DeltaLogState:
    """Device buffers of the physical state (Sec. 3.1), allocated with torch.

    S [B,H,dk,dv] state dtype, k_log [B,H,C,dk] in_dtype, u_log [B,H,C,dv], lam_log
    [B,H,C,dl] f32 ([B,C,H] for one log-decay per head), len [B,H] int32, err [1] int32.
    ``S`` starts as a copy of ``S0`` (the prefill state, converted to the state dtype);
    the log starts empty (Sec. 4 slot lifecycle).  The cumulative log-decay of Sec. 3.1
    is not a buffer: it is the newest snapshot (0 with an empty log), which the kernels
    read.  Linear attention has no decay, so ``lam_log`` is None (NULL to the library).
    """

    def __init__(self, desc, S0=None, device="cuda"):
        self.desc = desc
        B, H, dk, dv, M = desc.num_slots, desc.heads, desc.dk, desc.dv, desc.merge_interval
        C = M - 1
        dl = decay_width(desc)
        in_t = torch.bfloat16 if desc.in_dtype == DL_BF16 else torch.float32
        u_t = torch.bfloat16 if desc.u_log_dtype == DL_BF16 else torch.float32
        f32 = dict(dtype=torch.float32, device=device)
        st = state_torch_dtype(desc)
        self.S = (torch.zeros((B, H, dk, dv), dtype=st, device=device) if S0 is None else
                  S0.to(device=device, dtype=st).contiguous().clone())
        self.k_log = torch.zeros((B, H, max(C, 0), dk), dtype=in_t, device=device)
        self.u_log = torch.zeros((B, H, max(C, 0), dv), dtype=u_t, device=device)
        # scalar snapshots are entry-major [B, C, H] (the heads of a slot side by side)
        if dl == 1:
            self.lam_log = torch.zeros((B, max(C, 0), H), **f32)
        else:
            self.lam_log = torch.zeros((B, H, max(C, 0), dl), **f32) if dl else None
        self.len = torch.zeros((B, H), dtype=torch.int32, device=device)
        self.err = torch.zeros((1,), dtype=torch.int32, device=device)
        self.struct = dl_state(_ptr(self.S),
                               _ptr(self.k_log) if C > 0 else None,
                               _ptr(self.u_log) if C > 0 else None,
                               _ptr(self.lam_log) if C > 0 and dl else None,
                               _ptr(self.len), _ptr(self.err))

    def buffers(self):
        return dict(S=self.S, k_log=self.k_log, u_log=self.u_log,
                    lam_log=self.lam_log, len=self.len, err=self.err)


def _row_sizes(desc):
    """What of a descriptor the arrays over token rows go by."""
    return (desc.op, desc.heads, desc.dk, desc.dv, desc.in_dtype)


class Token:
    """Device tensors of one decode step's inputs plus the dl_token struct over them."""

    def __init__(self, desc, n, q, k, v, lam, beta=None, u=None):
        H, dk, dv = desc.heads, desc.dk, desc.dv
        dl = decay_width(desc)
        it = torch.bfloat16 if desc.in_dtype == DL_BF16 else torch.float32
        _need(q, "q", it, (n, H, dk))
        _need(k, "k", it, (n, H, dk))
        _need(v, "v", it, (n, H, dv))
        if dl:
            _need(lam, "lam", torch.float32, (n, H) if dl == 1 else (n, H, dl))
        else:
            lam = None                       # linear attention: no decay input
        if desc.op == DL_OP_RWKV6:
            _need(u, "u", torch.float32, (H, dk))
        else:
            u = None
        if desc.op in DELTA_OP_IDS:
            _need(beta, "beta", torch.float32, (n, H))
        else:
            beta = None
        self.n = n
        self.sizes = _row_sizes(desc)
        self.tensors = (q, k, v, lam, beta, u)
        self.struct = dl_token(_ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(lam), _ptr(u))


# Handle of the current device's current stream without building the Stream object that
# torch.cuda.current_stream() wraps around it: 2.8 -> 0.4 us, and with it a 4-slot
# dl_append_step takes 5.2 us of host time instead of 7.3.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _rows(desc, slots, n):
    """(device slot-list pointer or None, rows n of the launch).  Token row i drives slot
    slots[i] for i < n, so a token given with the call must hold at least n rows (extra
    rows are not read); without a slot list n is the token's row count or B."""
    rows = (desc.num_slots if n is None else n) if slots is None else slots.numel()
    if n is not None and n < rows:
        raise ValueError(f"the token holds {n} rows but the launch drives {rows}")
    if slots is None:
        return None, rows
    _need(slots, "slots", torch.int32, (rows,))
    return slots.data_ptr(), rows


def _check(rc, where):
    if rc != DL_OK:
        raise DeltaLogError(rc, where)


# ----------------------------------------------------------------- entry points
def dl_eager_step(desc, S, tok, o, slots=None, stream=None):
    """Eager dense step (Eq. 3) on S [B,H,dk,dv]; writes o [n,H,dv] f32."""
    sp, n = _rows(desc, slots, tok.n)
    _need(o, "o", torch.float32, (n, desc.heads, desc.dv))
    _need(S, "S", state_torch_dtype(desc), (desc.num_slots, desc.heads, desc.dk, desc.dv))
    _check(_lib.dl_eager_step(ctypes.byref(desc), _ptr(S), ctypes.byref(tok.struct), _ptr(o),
                              sp, n, _stream(stream)), "dl_eager_step")


def dl_append_step(desc, state, tok, o, slots=None, stream=None):
    """One DeltaLog step (Alg. 1): append if L < C else merge; writes o [n,H,dv] f32."""
    sp, n = _rows(desc, slots, tok.n)
    _need(o, "o", torch.float32, (n, desc.heads, desc.dv))
    _check(_lib.dl_append_step(ctypes.byref(desc), ctypes.byref(state.struct),
                               ctypes.byref(tok.struct), _ptr(o), sp, n, _stream(stream)),
           "dl_append_step")


def dl_merge(desc, state, tok=None, o=None, slots=None, stream=None):
    """Merge at the current L with the token (writes o), or flush when tok is None."""
    sp, n = _rows(desc, slots, None if tok is None else tok.n)
    if tok is not None:
        _need(o, "o", torch.float32, (n, desc.heads, desc.dv))
    _check(_lib.dl_merge(ctypes.byref(desc), ctypes.byref(state.struct),
                         None if tok is None else ctypes.byref(tok.struct),
                         _ptr(o) if tok is not None else None, sp, n, _stream(stream)),
           "dl_merge")


def dl_readout(desc, state, q, o, slots=None, stream=None):
    """o = q^T S_logical (Eq. 7) for q [n,H,dk]; mutates nothing."""
    n = q.shape[0]
    sp, n = _rows(desc, slots, n)
    it = torch.bfloat16 if desc.in_dtype == DL_BF16 else torch.float32
    _need(q, "q", it, (n, desc.heads, desc.dk))
    _need(o, "o", torch.float32, (n, desc.heads, desc.dv))
    _check(_lib.dl_readout(ctypes.byref(desc), ctypes.byref(state.struct), _ptr(q), _ptr(o),
                           sp, n, _stream(stream)), "dl_readout")


def dl_tiled_workspace_bytes(desc, n):
    """Bytes of scratch dl_append_step_tiled needs for n rows with split replay."""
    out = ctypes.c_size_t(0)
    _check(_lib.dl_tiled_workspace_bytes(ctypes.byref(desc), int(n), ctypes.byref(out)),
           "dl_tiled_workspace_bytes")
    return out.value


def tiled_workspace(desc, n, device="cuda"):
    """A device buffer of the split-replay scratch size for n rows (None if no log)."""
    nbytes = dl_tiled_workspace_bytes(desc, n)
    return torch.empty((nbytes,), dtype=torch.uint8, device=device) if nbytes else None


def dl_append_step_tiled(desc, state, tok, o, slots=None, value_tiles=4, split_replay=True,
                         workspace=None, stream=None):
    """Value-tiled DeltaLog step (Sec. 3.3): the same operation as dl_append_step with
    ``value_tiles`` workgroups per head; ``split_replay`` prepares the replay
    coefficients once per head into ``workspace`` (see ``tiled_workspace``)."""
    sp, n = _rows(desc, slots, tok.n)
    _need(o, "o", torch.float32, (n, desc.heads, desc.dv))
    wp, wn = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() *
                                                  workspace.element_size())
    _check(_lib.dl_append_step_tiled(ctypes.byref(desc), ctypes.byref(state.struct),
                                     ctypes.byref(tok.struct), _ptr(o), sp, n,
                                     int(value_tiles), int(bool(split_replay)), wp, wn,
                                     _stream(stream)), "dl_append_step_tiled")


def dl_append_step_tiled_noalloc(desc, state, tok, o, slots=None, value_tiles=4, stream=None):
    """dl_append_step_tiled with split replay whose coefficient scratch is the library's
    fixed per-GPU array (DL_NOALLOC_SCRATCH_BYTES): the call allocates nothing.  Calls
    that may overlap on one GPU race on that array."""
    sp, n = _rows(desc, slots, tok.n)
    _need(o, "o", torch.float32, (n, desc.heads, desc.dv))
    _check(_lib.dl_append_step_tiled_noalloc(ctypes.byref(desc), ctypes.byref(state.struct),
                                             ctypes.byref(tok.struct), _ptr(o), sp, n,
                                             int(value_tiles), _stream(stream)),
           "dl_append_step_tiled_noalloc")


# ----------------------------------------------------------------- whole sequences
class ChunkTables:
    """Device buffers of the chunk tables and slot maps of ``n`` sequences whose token rows
    are packed into buffers of ``tokens`` rows (dl_tables).  ``num_slots`` bounds the slot
    ids (default n); ``err`` is the device error word (1 = bad slot id, 4 = bad length)."""

    def __init__(self, n, tokens, num_slots=None, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.n, self.tokens = int(n), int(tokens)
        self.num_slots = max(self.n, 1) if num_slots is None else int(num_slots)
        self._words = torch.zeros((2 * self.n + 1,), **i32)
        self.cu_tokens, self.seq_slot = self._words[:self.n + 1], self._words[self.n + 1:]
        self.cu_chunks = torch.zeros((self.n + 1,), **i32)
        self.chunks = torch.zeros((self.tokens // DL_CHUNK + self.n, 4), **i32)
        self.row_slot = torch.zeros((self.tokens,), **i32)
        self.order = torch.zeros((self.n,), **i32)
        self.err = torch.zeros((1,), **i32)
        self.struct = dl_tables(_ptr(self.cu_tokens), _ptr(self.cu_chunks), _ptr(self.chunks),
                                _ptr(self.row_slot), _ptr(self.seq_slot), _ptr(self.order))

    def _kept(self):
        """What the operators around a recurrence read of these tables, copied on the current
        stream: filling the tables again leaves it as it is."""
        return _KeptTables(self)


class _KeptTables:
    def __init__(self, tables):
        self.n, self.tokens, self.num_slots = tables.n, tables.tokens, tables.num_slots
        self.err = tables.err
        words = tables._words + 0            # a kernel, in a captured graph too
        self.cu_tokens, self.seq_slot = words[:self.n + 1], words[self.n + 1:]
        self.struct = dl_tables(_ptr(self.cu_tokens), None, None, None, _ptr(self.seq_slot), None)


class Grads:
    """Device buffers for the gradients of one dl_prefill call (dl_grads), shaped as the
    token's tensors and the state buffer ``S`` (None: no gradient of the initial states)."""

    def __init__(self, desc, tok, S=None):
        q, k, v, lam, beta, u = tok.tensors
        like = lambda t: None if t is None else torch.zeros_like(t)  # noqa: E731
        self.dq, self.dk, self.dv = like(q), like(k), like(v)
        self.dlam, self.dbeta, self.du = like(lam), like(beta), like(u)
        if S is not None:
            _need(S, "S", state_torch_dtype(desc),
                  (desc.num_slots, desc.heads, desc.dk, desc.dv))
        self.dS = like(S)
        self.n, self.sizes = tok.n, tok.sizes
        self.state = None if S is None else (desc.num_slots, desc.state_dtype)
        self.struct = dl_grads(_ptr(self.dq), _ptr(self.dk), _ptr(self.dv), _ptr(self.dbeta),
                               _ptr(self.dlam), _ptr(self.du), _ptr(self.dS))


def _on_current_device(*tensors):
    """Every tensor on the current device, whose stream the call goes to."""
    cur = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.device.index != cur:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{cur}")


def dl_chunk_tables(lens, tables, slots=None, stream=None):
    """Build ``tables`` from the sequences' lengths, lens [n] int32 on the device (slots [n]
    int32, or None: sequence i has slot i)."""
    _need(lens, "lens", torch.int32, (tables.n,))
    if slots is not None:
        _need(slots, "slots", torch.int32, (tables.n,))
    _on_current_device(lens, slots, tables.err)
    _check(_lib.dl_chunk_tables(_ptr(lens), _ptr(slots), tables.n, tables.tokens,
                                tables.num_slots, ctypes.byref(tables.struct),
                                _ptr(tables.err), _stream(stream)), "dl_chunk_tables")


def dl_prefill_workspace_bytes(desc, n, tokens, backward=False):
    """Bytes of workspace dl_prefill needs (with ``backward``: it and dl_prefill_backward)."""
    out = ctypes.c_size_t(0)
    _check(_lib.dl_prefill_workspace_bytes(ctypes.byref(desc), int(n), int(tokens),
                                           int(bool(backward)), ctypes.byref(out)),
           "dl_prefill_workspace_bytes")
    return out.value


def prefill_workspace(desc, n, tokens, backward=False, device="cuda"):
    """A device buffer of the size dl_prefill_workspace_bytes names."""
    return torch.empty((dl_prefill_workspace_bytes(desc, n, tokens, backward),),
                       dtype=torch.uint8, device=device)


def _sequences(desc, tok, tables, workspace, *others):
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor (see prefill_workspace)")
    if tok.sizes != _row_sizes(desc):
        raise ValueError("the token was made for another descriptor")
    if tok.n != tables.tokens:
        raise ValueError(f"the token holds {tok.n} rows but the tables are for {tables.tokens}")
    _on_current_device(*tok.tensors, tables.err, workspace, *others)
    return (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def dl_prefill(desc, S_in, S_out, tok, o, tables, workspace, stream=None):
    """The recurrence over the whole sequences of ``tables``: from S_in[slot] (None: zero) to
    S_out[slot] (may be S_in), o [N,H,dv] in the input dtype."""
    state = (state_torch_dtype(desc), (desc.num_slots, desc.heads, desc.dk, desc.dv))
    if S_in is not None:
        _need(S_in, "S_in", *state)
    _need(S_out, "S_out", *state)
    _need(o, "o", tok.tensors[2].dtype, (tok.n, desc.heads, desc.dv))
    wp, wn = _sequences(desc, tok, tables, workspace, S_in, S_out, o)
    _check(_lib.dl_prefill(ctypes.byref(desc), _ptr(S_in), _ptr(S_out), ctypes.byref(tok.struct),
                           _ptr(o), ctypes.byref(tables.struct), tables.n, tables.tokens, wp, wn,
                           _stream(stream)), "dl_prefill")


def dl_prefill_backward(desc, S_in, tok, d_o, dS_out, grads, tables, workspace, stream=None):
    """Gradients of dl_prefill into ``grads`` (``Grads``) from d_o [N,H,dv] and dS_out
    [B,H,dk,dv] (None: zero).  The forward call must have left S_in as it was."""
    state = (state_torch_dtype(desc), (desc.num_slots, desc.heads, desc.dk, desc.dv))
    _need(d_o, "d_o", tok.tensors[2].dtype, (tok.n, desc.heads, desc.dv))
    for name, t in (("S_in", S_in), ("dS_out", dS_out)):
        if t is not None:
            _need(t, name, *state)
    if grads.n != tok.n or grads.sizes != _row_sizes(desc):
        raise ValueError("the gradients were made for another token or descriptor")
    if grads.state not in (None, (desc.num_slots, desc.state_dtype)):
        raise ValueError("the gradient of the states was made for another descriptor")
    wp, wn = _sequences(desc, tok, tables, workspace, S_in, d_o, dS_out, grads.dq, grads.dS)
    _check(_lib.dl_prefill_backward(ctypes.byref(desc), _ptr(S_in), ctypes.byref(tok.struct),
                                    _ptr(d_o), _ptr(dS_out), ctypes.byref(grads.struct),
                                    ctypes.byref(tables.struct), tables.n, tables.tokens, wp, wn,
                                    _stream(stream)), "dl_prefill_backward")


# ----------------------------------------------------------------- around a recurrence
def _in_torch_dtype(desc):
    return torch.bfloat16 if desc.in_dtype == DL_BF16 else torch.float32


def _need_rows(t, name, dtype, shape):
    """Elements from one row of ``t`` to the next: token rows may be columns of a wider tensor,
    everything behind the first dimension is dense."""
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    width = 1
    for size, stride in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != width:
            raise ValueError(f"{name}: a row must be dense")
        width *= size
    if shape[0] <= 1:
        return width                       # the stride of a single row means nothing
    if t.stride(0) < width or t.stride(0) % 8:
        raise ValueError(f"{name}: rows {t.stride(0)} elements apart, expected a multiple of 8 that "
                         f"is {width} at least")
    return t.stride(0)


def _optional(t, name, dtype, shape):
    if t is not None:
        _need(t, name, dtype, shape)


def _workspace(workspace, maker):
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous device tensor (see {maker})")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


class _Rows:
    """What a call reads besides states: its tensors, the descriptor it was made for, the struct."""

    def _keep(self, desc, n, tensors, struct):
        self.n, self.tensors, self.struct = n, tensors, struct
        self.ref, self.raw, self.sizes = ctypes.byref(struct), bytes(desc), _sizes(desc)
        self.device = tensors[0].get_device()
        for t in tensors:
            if t is not None and t.get_device() != self.device:
                raise ValueError(f"tensors on cuda:{self.device} and {t.device}")


def _made_for(desc, rows, tables=None, grads=None):
    """The rows (and gradients) were made for this descriptor and these tables."""
    if rows.raw != bytes(desc) and rows.sizes != _sizes(desc):
        raise ValueError("the rows were made for another descriptor")
    if tables is not None and rows.n != tables.tokens:
        raise ValueError(f"{rows.n} rows but the tables are for {tables.tokens}")
    if grads is not None and (grads.n != rows.n or grads.sizes != rows.sizes
                              or grads.given != tuple(t is not None for t in rows.tensors)):
        raise ValueError("the gradients were made for other rows or another descriptor")
    if grads is not None and getattr(grads, "slots", None) not in (None, getattr(desc, "num_slots", 0)):
        raise ValueError("the gradient of the states was made for another descriptor")


def _sizes(desc):
    """All of a descriptor but the slots, which rows do not depend on."""
    return tuple(getattr(desc, k) for k, _ in desc._fields_ if k != "num_slots")


def _stream_of(stream, rows, *tensors):
    """The stream to launch on; every tensor has to be on the current device, whose stream it is."""
    cur = torch.cuda.current_device()
    if rows.device != cur:
        raise ValueError(f"tensors are on cuda:{rows.device}, the current device is cuda:{cur}")
    for t in tensors:
        if t is not None and t.get_device() != cur:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{cur}")
    return _raw_stream(cur) if stream is None and _raw_stream is not None else _stream(stream)


def _bytes(call, where, desc, *args):
    out = ctypes.c_size_t(0)
    _check(call(ctypes.byref(desc), *args, ctypes.byref(out)), where)
    return out.value


def make_conv_desc(B, channels, width, in_dtype="bf16", activation="silu"):
    """dl_conv_desc of a short causal convolution: ``width`` taps, states in B slots."""
    return dl_conv_desc(DL_ABI_VERSION, B, channels, width, ACTIVATION_IDS[activation],
                        DTYPE_IDS[in_dtype])


class ConvRows(_Rows):
    """What a convolution reads: token rows x [n,D] in the input dtype (columns of a wider tensor
    will do), w [D,W] and bias [D] (or None) in fp32."""

    def __init__(self, desc, n, x, w, bias=None):
        stride = _need_rows(x, "x", _in_torch_dtype(desc), (n, desc.channels))
        _need(w, "w", torch.float32, (desc.channels, desc.width))
        _optional(bias, "bias", torch.float32, (desc.channels,))
        self._keep(desc, n, (x, w, bias), dl_conv_rows(_ptr(x), stride, _ptr(w), _ptr(bias)))


class ConvGrads:
    """Device buffers for the gradients of one dl_conv_prefill call; ``s``: the states before
    (None: no gradient of them).  Slots without a sequence hold what ``ds`` holds there (None: 0)."""

    def __init__(self, desc, rows, s=None, ds=None):
        x, w, bias = rows.tensors
        self.dx = torch.zeros(x.shape, dtype=x.dtype, device=x.device)
        self.dw = torch.zeros_like(w)
        self.dbias = None if bias is None else torch.zeros_like(bias)
        _optional(s, "s", *_conv_state(desc))
        _optional(ds, "ds", *_conv_state(desc))
        self.ds = None if s is None else torch.zeros_like(s) if ds is None else ds.clone()
        self.n, self.sizes = rows.n, rows.sizes
        self.given = tuple(t is not None for t in rows.tensors)
        self.slots = None if s is None else desc.num_slots
        self.struct = dl_conv_grads(_ptr(self.dx), _ptr(self.dw), _ptr(self.dbias), _ptr(self.ds))


def _conv_state(desc):
    return _in_torch_dtype(desc), (desc.num_slots, desc.width - 1, desc.channels)


def dl_conv_step(desc, s_in, s_out, rows, y, slots=None, stream=None):
    """One token per slot through the convolution: y [n,D], and the slots' new states (the last
    W - 1 inputs) from s_in [B,W-1,D] to s_out (may be s_in)."""
    sp, n = _rows(desc, slots, rows.n)
    _made_for(desc, rows)
    state = _conv_state(desc)
    _need(s_in, "s_in", *state)
    _need(s_out, "s_out", *state)
    _need(y, "y", state[0], (n, desc.channels))
    st = _stream_of(stream, rows, s_in, s_out, y, slots)
    _check(_lib.dl_conv_step(ctypes.byref(desc), _ptr(s_in), _ptr(s_out), rows.ref,
                             _ptr(y), sp, n, st), "dl_conv_step")


def dl_conv_prefill(desc, s_in, s_out, rows, y, tables, stream=None):
    """The convolution over the whole sequences of ``tables``, from s_in[slot] (None: zeros) to
    s_out[slot] (may be s_in), y [N,D] in the input dtype."""
    _made_for(desc, rows, tables)
    _optional(s_in, "s_in", *_conv_state(desc))
    _need(s_out, "s_out", *_conv_state(desc))
    _need(y, "y", _in_torch_dtype(desc), (rows.n, desc.channels))
    st = _stream_of(stream, rows, s_in, s_out, y, tables.err)
    _check(_lib.dl_conv_prefill(ctypes.byref(desc), _ptr(s_in), _ptr(s_out),
                                rows.ref, _ptr(y), ctypes.byref(tables.struct),
                                tables.n, tables.tokens, st), "dl_conv_prefill")


def conv_workspace(desc, n, tokens, device="cuda"):
    """A device buffer of the size dl_conv_workspace_bytes names (dl_conv_backward's scratch)."""
    size = _bytes(_lib.dl_conv_workspace_bytes, "dl_conv_workspace_bytes", desc, int(n), int(tokens))
    return torch.empty((size,), dtype=torch.uint8, device=device)


def dl_conv_backward(desc, s_in, rows, dy, ds_out, grads, tables, workspace, stream=None):
    """Gradients of dl_conv_prefill into ``grads`` (``ConvGrads``) from dy [N,D] and ds_out
    [B,W-1,D] (None: zero).  The forward call must have left s_in as it was."""
    _made_for(desc, rows, tables, grads)
    _optional(s_in, "s_in", *_conv_state(desc))
    _optional(ds_out, "ds_out", *_conv_state(desc))
    _need(dy, "dy", _in_torch_dtype(desc), (rows.n, desc.channels))
    wp, wn = _workspace(workspace, "conv_workspace")
    st = _stream_of(stream, rows, s_in, dy, ds_out, grads.dx, grads.ds, tables.err, workspace)
    _check(_lib.dl_conv_backward(ctypes.byref(desc), _ptr(s_in), rows.ref, _ptr(dy),
                                 _ptr(ds_out), ctypes.byref(grads.struct),
                                 ctypes.byref(tables.struct), tables.n, tables.tokens, wp, wn,
                                 st), "dl_conv_backward")


def make_qk_desc(H, d, norm="l2", turn="none", rot=None, rep=1, in_dtype="bf16", eps=1e-6,
                 q_scale=1.0):
    """dl_qk_desc: ``norm`` "l2", "rms" or "none"; ``turn`` "halves", "pairs" or "none" for the first
    ``rot`` places (None: all of them); ``rep`` output heads for each of the H input heads."""
    rot = (0 if turn == "none" else d) if rot is None else rot
    return dl_qk_desc(DL_ABI_VERSION, H, d, rep, NORM_IDS[norm], TURN_IDS[turn], rot,
                      DTYPE_IDS[in_dtype], eps, q_scale)


class QkRows(_Rows):
    """What the norm of queries and keys reads: q, k [n,H,d] in the input dtype (columns of a wider
    tensor will do), positions pos [n] int32 and frequencies freq [rot/2] fp32 where they turn,
    weights wq, wk [d] fp32 (both or neither).  ``tables``: rows behind its sequences are left out."""

    def __init__(self, desc, n, q, k, pos=None, freq=None, wq=None, wk=None, tables=None):
        H, d, it = desc.heads, desc.head_dim, _in_torch_dtype(desc)
        qs, ks = (_need_rows(t, name, it, (n, H, d)) for t, name in ((q, "q"), (k, "k")))
        if desc.turn == TURN_IDS["none"]:
            pos = freq = None
        else:
            _need(pos, "pos", torch.int32, (n,))
            _need(freq, "freq", torch.float32, (desc.rot // 2,))
        if (wq is None) != (wk is None):
            raise ValueError("weights for both queries and keys, or for neither")
        _optional(wq, "wq", torch.float32, (d,))
        _optional(wk, "wk", torch.float32, (d,))
        if tables is not None and tables.tokens != n:
            raise ValueError(f"{n} rows but the tables are for {tables.tokens}")
        used = None if tables is None else tables.cu_tokens[tables.n:]
        self._keep(desc, n, (q, k, pos, freq, wq, wk, used),
                   dl_qk_rows(_ptr(q), _ptr(k), qs, ks, _ptr(pos), _ptr(freq), _ptr(wq), _ptr(wk),
                              _ptr(used)))


class QkGrads:
    """Device buffers for the gradients of one dl_qk_norm call."""

    def __init__(self, desc, rows):
        q, k, wq, wk = (rows.tensors[i] for i in (0, 1, 4, 5))
        self.dq, self.dk = (torch.zeros(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        self.dwq, self.dwk = (None if t is None else torch.zeros_like(t) for t in (wq, wk))
        self.n, self.sizes = rows.n, rows.sizes
        self.given = tuple(t is not None for t in rows.tensors)
        self.struct = dl_qk_grads(_ptr(self.dq), _ptr(self.dk), _ptr(self.dwq), _ptr(self.dwk))


def dl_qk_norm(desc, rows, q_out, k_out, stream=None):
    """Queries and keys normalised head by head and turned by position, into q_out and k_out
    [n,H rep,d]."""
    _made_for(desc, rows)
    out = (_in_torch_dtype(desc), (rows.n, desc.heads * desc.rep, desc.head_dim))
    _need(q_out, "q_out", *out)
    _need(k_out, "k_out", *out)
    st = _stream_of(stream, rows, q_out, k_out)
    _check(_lib.dl_qk_norm(ctypes.byref(desc), rows.ref, _ptr(q_out), _ptr(k_out),
                           rows.n, st), "dl_qk_norm")


def qk_workspace(desc, n, device="cuda"):
    """A device buffer of the size dl_qk_workspace_bytes names (dl_qk_norm_backward's scratch)."""
    size = _bytes(_lib.dl_qk_workspace_bytes, "dl_qk_workspace_bytes", desc, int(n))
    return torch.empty((size,), dtype=torch.uint8, device=device)


def dl_qk_norm_backward(desc, rows, dq_out, dk_out, grads, workspace, stream=None):
    """Gradients of dl_qk_norm into ``grads`` (``QkGrads``) from dq_out and dk_out [n,H rep,d]."""
    _made_for(desc, rows, grads=grads)
    out = (_in_torch_dtype(desc), (rows.n, desc.heads * desc.rep, desc.head_dim))
    _need(dq_out, "dq_out", *out)
    _need(dk_out, "dk_out", *out)
    wp, wn = _workspace(workspace, "qk_workspace")
    st = _stream_of(stream, rows, dq_out, dk_out, grads.dq, grads.dk, workspace)
    _check(_lib.dl_qk_norm_backward(ctypes.byref(desc), rows.ref, _ptr(dq_out),
                                    _ptr(dk_out), ctypes.byref(grads.struct), rows.n, wp, wn,
                                    st), "dl_qk_norm_backward")


def make_ssm_desc(B, channels, states, in_dtype="bf16"):
    """dl_ssm_desc of a selective scan: ``states`` (16, 32 or 64) states a channel, B slots."""
    return dl_ssm_desc(DL_ABI_VERSION, B, channels, states, DTYPE_IDS[in_dtype])


def _ssm_state(desc):
    return torch.float32, (desc.num_slots, desc.channels, desc.states)


class SsmRows(_Rows):
    """What a selective scan reads: token rows x, dt and z (or None: no gate) [n,D], Bm and Cm [n,S]
    in the input dtype (columns of a wider tensor will do); A [D,S], skip [D] and dt_bias [D] (or
    None) in fp32."""

    def __init__(self, desc, n, x, dt, A, Bm, Cm, skip=None, dt_bias=None, z=None):
        D, S, it = desc.channels, desc.states, _in_torch_dtype(desc)
        strides = [_need_rows(x, "x", it, (n, D)), _need_rows(dt, "dt", it, (n, D)),
                   0 if z is None else _need_rows(z, "z", it, (n, D)),
                   _need_rows(Bm, "Bm", it, (n, S)), _need_rows(Cm, "Cm", it, (n, S))]
        _need(A, "A", torch.float32, (D, S))
        _optional(skip, "skip", torch.float32, (D,))
        _optional(dt_bias, "dt_bias", torch.float32, (D,))
        self._keep(desc, n, (x, dt, z, Bm, Cm, A, skip, dt_bias),
                   dl_ssm_rows(_ptr(x), _ptr(dt), _ptr(z), _ptr(Bm), _ptr(Cm), *strides, _ptr(A),
                               _ptr(skip), _ptr(dt_bias)))


class SsmGrads:
    """Device buffers for the gradients of one dl_ssm_prefill call; ``h``: the states before (None:
    no gradient of them).  Slots without a sequence hold what ``dh`` holds there (None: 0)."""

    def __init__(self, desc, rows, h=None, dh=None):
        like = lambda t: None if t is None else torch.zeros(t.shape, dtype=t.dtype,  # noqa: E731
                                                            device=t.device)
        (self.dx, self.ddt, self.dz, self.dB, self.dC, self.dA, self.dskip,
         self.dbias) = map(like, rows.tensors)
        _optional(h, "h", *_ssm_state(desc))
        _optional(dh, "dh", *_ssm_state(desc))
        self.ds = like(h) if h is None or dh is None else dh.clone()
        self.n, self.sizes = rows.n, rows.sizes
        self.given = tuple(t is not None for t in rows.tensors)
        self.slots = None if h is None else desc.num_slots
        self.struct = dl_ssm_grads(*map(_ptr, (self.dx, self.ddt, self.dz, self.dB, self.dC, self.dA,
                                               self.dskip, self.dbias, self.ds)))


def dl_ssm_step(desc, h_in, h_out, rows, y, slots=None, stream=None):
    """One token per slot through the scan: y [n,D], and the slots' new states from h_in [B,D,S] to
    h_out (may be h_in)."""
    sp, n = _rows(desc, slots, rows.n)
    _made_for(desc, rows)
    state = _ssm_state(desc)
    _need(h_in, "h_in", *state)
    _need(h_out, "h_out", *state)
    _need(y, "y", _in_torch_dtype(desc), (n, desc.channels))
    st = _stream_of(stream, rows, h_in, h_out, y, slots)
    _check(_lib.dl_ssm_step(ctypes.byref(desc), _ptr(h_in), _ptr(h_out), rows.ref,
                            _ptr(y), sp, n, st), "dl_ssm_step")


def ssm_workspace(desc, n, tokens, backward=False, device="cuda"):
    """A device buffer of the size dl_ssm_workspace_bytes names for n and tokens (fewer can need more):
    for dl_ssm_prefill (with ``backward``: and dl_ssm_backward)."""
    size = _bytes(_lib.dl_ssm_workspace_bytes, "dl_ssm_workspace_bytes", desc, int(n), int(tokens),
                  int(bool(backward)))
    return torch.empty((size,), dtype=torch.uint8, device=device)


def dl_ssm_prefill(desc, h_in, h_out, rows, y, tables, workspace, stream=None):
    """The scan over the whole sequences of ``tables``, from h_in[slot] (None: zeros) to h_out[slot]
    (may be h_in), y [N,D] in the input dtype."""
    _made_for(desc, rows, tables)
    _optional(h_in, "h_in", *_ssm_state(desc))
    _need(h_out, "h_out", *_ssm_state(desc))
    _need(y, "y", _in_torch_dtype(desc), (rows.n, desc.channels))
    wp, wn = _workspace(workspace, "ssm_workspace")
    st = _stream_of(stream, rows, h_in, h_out, y, tables.err, workspace)
    _check(_lib.dl_ssm_prefill(ctypes.byref(desc), _ptr(h_in), _ptr(h_out), rows.ref,
                               _ptr(y), ctypes.byref(tables.struct), tables.n, tables.tokens, wp, wn,
                               st), "dl_ssm_prefill")


def dl_ssm_backward(desc, h_in, rows, dy, dh_out, grads, tables, workspace, stream=None):
    """Gradients of dl_ssm_prefill into ``grads`` (``SsmGrads``) from dy [N,D] and dh_out [B,D,S]
    (None: zero).  The forward call must have left h_in as it was."""
    _made_for(desc, rows, tables, grads)
    _optional(h_in, "h_in", *_ssm_state(desc))
    _optional(dh_out, "dh_out", *_ssm_state(desc))
    _need(dy, "dy", _in_torch_dtype(desc), (rows.n, desc.channels))
    wp, wn = _workspace(workspace, "ssm_workspace")
    st = _stream_of(stream, rows, h_in, dy, dh_out, grads.dx, grads.ds, tables.err, workspace)
    _check(_lib.dl_ssm_backward(ctypes.byref(desc), _ptr(h_in), rows.ref, _ptr(dy),
                                _ptr(dh_out), ctypes.byref(grads.struct), ctypes.byref(tables.struct),
                                tables.n, tables.tokens, wp, wn, st), "dl_ssm_backward")
