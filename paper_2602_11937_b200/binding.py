"""Binding of the C ABI: same entry-point names, argument marshalling only (ctypes; the entry points a decode step or a
prompt chunk calls go through a small native module, csrc/call.cpp, because a microsecond of host time counts there)."""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import platform
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "lib", "libpuzzle_attn.so")
_CALL_PATH = os.path.join(_HERE, "lib", "_puzzle_call.so")
_lib = None
_call = None

KV_FP8_E4M3 = 0
KV_BF16 = 1
KV_FP4_E2M1 = 2
FP4_BLOCK_BYTES = 576          # one (block, KV head) of the 4-bit cache: a cache is uint8 [num_blocks][Hkv][576]
DEV_BAD_BLOCK = 1
DEV_SEQ_TOO_LONG = 2
DEV_WAIT_EXPIRED = 4
DEV_BAD_POSITION = 8
STATIC_SCRATCH_BYTES = 8 << 20
SCHED_AUTO, SCHED_CTA, SCHED_WARP = 0, -1, -2      # num_splits values that select the balanced schedule

EXPORTS = (
    "puzzle_kv_amax_update",
    "puzzle_kv_scales_from_amax",
    "puzzle_kv_append",
    "puzzle_kv_append_tokens",
    "puzzle_kv_append_rope",
    "puzzle_kv_read_tokens",
    "puzzle_decode_attn_workspace_bytes",
    "puzzle_decode_attn_workspace_init",
    "puzzle_decode_attn",
    "puzzle_decode_attn_tcgen05",
    "puzzle_decode_attn_static",
    "puzzle_decode_attn_partial",
    "puzzle_decode_step_host",
    "puzzle_decode_step_host_staging_bytes",
    "puzzle_decode_attn_tokens",
    "puzzle_decode_attn_tokens_workspace_bytes",
    "puzzle_decode_attn_tokens_workspace_init",
    "puzzle_attn_merge",
    "puzzle_attn_merge_strided",
    "puzzle_hbm_read_probe",
    "puzzle_status_string",
    "puzzle_launch_count",
    "puzzle_decode_attn_kernel_name",
)


class PuzzleError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: status %d (%s)" % (where, code, puzzle_status_string(code)))


class LayerDesc(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("window", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
                ("sm_scale", ctypes.c_float)]


class _Pointers(ctypes.Structure):
    """A descriptor of pointers, with a note (_held) of what the tensors behind them hold.  A field set by hand may lead to
    other tensors: the note ends with it."""
    _held = None

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name[0] != "_":
            super().__setattr__("_held", None)


class KVView(_Pointers):
    _fields_ = [("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("num_blocks", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("max_blocks_per_seq", ctypes.c_int32),
                ("seq_lens", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]
    # _held, noted by kv_view: device, sequences, scales, bytes of the smaller cache


class Rope(_Pointers):
    _fields_ = [("cos_sin", ctypes.c_void_p), ("num_positions", ctypes.c_int64), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("pos_offset", ctypes.c_void_p)]
    # _held, noted by rope_view: device, sequences that have an offset


class QKV(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
        [(t + which, ctypes.c_int64) for t in "qkv" for which in ("_seq_stride", "_token_stride")]


def library_path() -> str:
    return _LIB_PATH


def _load():
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                "CUDA library %s is missing: build it with `python -m paper_2602_11937_b200.build` "
                "(there is no CPU fallback)" % _LIB_PATH)
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        lib.puzzle_kv_append.restype = ctypes.c_int
        lib.puzzle_kv_append.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, i32, vp, vp]
        lib.puzzle_kv_amax_update.restype = ctypes.c_int
        lib.puzzle_kv_amax_update.argtypes = [vp, ctypes.c_int64, i32, i32, vp, vp]
        lib.puzzle_kv_scales_from_amax.restype = ctypes.c_int
        lib.puzzle_kv_scales_from_amax.argtypes = [vp, i32, i32, vp, vp]
        lib.puzzle_kv_append_tokens.restype = ctypes.c_int
        lib.puzzle_kv_append_tokens.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, i32, i32,
                                                vp, vp]
        lib.puzzle_kv_append_rope.restype = ctypes.c_int
        lib.puzzle_kv_append_rope.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), ctypes.POINTER(Rope),
                                              ctypes.POINTER(QKV), vp, vp, i32, i32, vp, vp]
        lib.puzzle_kv_read_tokens.restype = ctypes.c_int
        lib.puzzle_kv_read_tokens.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, i32, i32,
                                              vp, vp]
        lib.puzzle_decode_attn_workspace_bytes.restype = sz
        lib.puzzle_decode_attn_workspace_bytes.argtypes = [ctypes.POINTER(LayerDesc), i32, i32]
        lib.puzzle_decode_attn_workspace_init.restype = ctypes.c_int
        lib.puzzle_decode_attn_workspace_init.argtypes = [ctypes.POINTER(LayerDesc), i32, vp, sz, vp]
        lib.puzzle_decode_attn.restype = ctypes.c_int
        lib.puzzle_decode_attn.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, vp, i32, i32,
                                           vp, sz, vp, vp]
        lib.puzzle_decode_attn_tcgen05.restype = ctypes.c_int
        lib.puzzle_decode_attn_tcgen05.argtypes = lib.puzzle_decode_attn.argtypes
        lib.puzzle_decode_attn_partial.restype = ctypes.c_int
        lib.puzzle_decode_attn_partial.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, i32, i32,
                                                   vp, sz, vp, vp]
        lib.puzzle_attn_merge_strided.restype = ctypes.c_int
        lib.puzzle_attn_merge_strided.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                                  vp, vp, vp, vp, i32, i32, i32, i32, vp]
        lib.puzzle_decode_attn_static.restype = ctypes.c_int
        lib.puzzle_decode_attn_static.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, vp,
                                                  i32, i32, vp, vp]
        lib.puzzle_decode_step_host_staging_bytes.restype = sz
        lib.puzzle_decode_step_host_staging_bytes.argtypes = [ctypes.POINTER(LayerDesc), i32]
        lib.puzzle_decode_step_host.restype = ctypes.c_int
        lib.puzzle_decode_step_host.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, vp, vp,
                                                i32, i32, vp, sz, vp, sz, vp, vp]
        lib.puzzle_decode_attn_tokens_workspace_bytes.restype = sz
        lib.puzzle_decode_attn_tokens_workspace_bytes.argtypes = [ctypes.POINTER(LayerDesc), i32, i32]
        lib.puzzle_decode_attn_tokens_workspace_init.restype = ctypes.c_int
        lib.puzzle_decode_attn_tokens_workspace_init.argtypes = [ctypes.POINTER(LayerDesc), i32, i32, vp, sz, vp]
        lib.puzzle_decode_attn_tokens.restype = ctypes.c_int
        lib.puzzle_decode_attn_tokens.argtypes = [ctypes.POINTER(LayerDesc), ctypes.POINTER(KVView), vp, vp, vp, vp, vp,
                                                  i32, i32, vp, sz, vp, vp]
        lib.puzzle_attn_merge.restype = ctypes.c_int
        lib.puzzle_attn_merge.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp]
        lib.puzzle_hbm_read_probe.restype = ctypes.c_int
        lib.puzzle_hbm_read_probe.argtypes = [vp, sz, vp, vp]
        lib.puzzle_status_string.restype = ctypes.c_char_p
        lib.puzzle_status_string.argtypes = [ctypes.c_int]
        lib.puzzle_launch_count.restype = ctypes.c_int64
        lib.puzzle_launch_count.argtypes = []
        lib.puzzle_decode_attn_kernel_name.restype = ctypes.c_char_p
        lib.puzzle_decode_attn_kernel_name.argtypes = [vp, vp, i32, i32]
        _bind(lib)
        _lib = lib
    return _lib


# The entry points of the native module, in the order of its Entries.
_CALLS = ("puzzle_kv_append", "puzzle_kv_append_tokens", "puzzle_kv_append_rope", "puzzle_kv_read_tokens",
          "puzzle_decode_attn", "puzzle_decode_attn_tcgen05", "puzzle_decode_attn_tokens")


def _bind(lib):
    """Loads the native module and gives it the addresses of the library's entry points."""
    global _call
    if _call is None:
        if not os.path.exists(_CALL_PATH):
            raise RuntimeError("%s is missing: build it with `python -m paper_2602_11937_b200.build`" % _CALL_PATH)
        loader = importlib.machinery.ExtensionFileLoader("_puzzle_call", _CALL_PATH)
        spec = importlib.util.spec_from_file_location("_puzzle_call", _CALL_PATH, loader=loader)
        module = importlib.util.module_from_spec(spec)
        loader.exec_module(module)
        here = "python %s torch %s" % (".".join(platform.python_version_tuple()[:2]), torch.__version__)
        built_for = getattr(module, "built_for", "an unknown version")
        if built_for != here:
            raise RuntimeError("%s was built for %s, this is %s: build it again with `python -m paper_2602_11937_b200.build`"
                               % (_CALL_PATH, built_for, here))
    else:
        module = _call
    module.bind(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _CALLS))
    _call = module


def _native():
    if _lib is None:
        _load()
    return _call


def _p(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return t.data_ptr()


_ANY = 1 << 62    # as many as a call may want


def _device_of(what: str, *tensors) -> int:
    devices = {t.get_device() for t in tensors if t is not None and t.is_cuda}
    if len(devices) > 1:
        raise ValueError("the tensors of %s lie on several devices" % what)
    return devices.pop() if devices else -1


# The current stream's handle without a Stream object around it: a decode step's call is a few microseconds of host time.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream, tensor=None):
    """Handle of `stream` (None: the current one).  tensor: one of the call's; kernels are launched on the current device,
    so it has to lie there."""
    if tensor is not None and tensor.get_device() != _current_device():
        raise ValueError("the tensors are on cuda:%d, the current device is cuda:%d"
                         % (tensor.get_device(), _current_device()))
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_current_device())
    return torch.cuda.current_stream().cuda_stream


def _arg(t: Optional[torch.Tensor], dtype=None, name="tensor", need: int = 0):
    """Device pointer (None -> NULL) of a tensor that a call is given: contiguous, on the current device, with at least
    `need` elements."""
    p = _p(t, dtype, name)
    if t is None:
        return p
    _same_device(name, t.get_device())
    if t.numel() < need:
        raise ValueError("%s has %d elements, the call needs %d" % (name, t.numel(), need))
    return p


def _same_device(name: str, device: int):
    if device != _current_device():
        raise ValueError("%s is on cuda:%d, the current device is cuda:%d" % (name, device, _current_device()))


def _reach(t: torch.Tensor, dtype, name: str, need: int):
    """_arg of a tensor that names the first of `need` elements of its storage."""
    p = _arg(t, dtype, name)
    if p is not None and t.untyped_storage().nbytes() // t.element_size() - t.storage_offset() < need:
        raise ValueError("%s reaches fewer than the %d elements that the call needs" % (name, need))
    return p


_BLOCK_BYTES = {KV_FP8_E4M3: 16 * 64, KV_BF16: 16 * 64 * 2, KV_FP4_E2M1: FP4_BLOCK_BYTES}


def _taken(desc) -> bool:
    """Whether the library takes this descriptor; others it refuses itself, with a code that says why."""
    return desc.num_kv_heads > 0 and desc.head_dim == 64 and desc.num_q_heads == 8 * desc.num_kv_heads


def _check_view(desc, view, batch: int):
    """Whether what a view points to has room for this descriptor and this many sequences (as in csrc/call.cpp)."""
    if view._held is None:
        return
    device, sequences, scales, cache_bytes = view._held
    if sequences < batch:
        raise ValueError("the cache view has %d sequences, the call needs %d" % (sequences, batch))
    if _taken(desc):
        if scales < desc.num_kv_heads and desc.kv_dtype != KV_BF16:
            raise ValueError("the cache view has %d scales, the call needs %d" % (scales, desc.num_kv_heads))
        need = view.num_blocks * desc.num_kv_heads * _BLOCK_BYTES.get(desc.kv_dtype, 0)
        if cache_bytes < need:
            raise ValueError("the cache has %d bytes, the descriptor's %d blocks need %d" % (cache_bytes, view.num_blocks, need))
    _same_device("the cache view", device)


def _rows(desc, batch: int):
    """Elements of q or out, of their heads, and of k_new or v_new, for `batch` tokens."""
    if not _taken(desc):
        return 0, 0, 0
    return batch * desc.num_q_heads * 64, batch * desc.num_q_heads, batch * desc.num_kv_heads * 64


def layer_desc(window: int = 0, kv_dtype: int = KV_FP8_E4M3, num_q_heads: int = 64, num_kv_heads: int = 8,
               head_dim: int = 64, block_size: int = 16, sm_scale: Optional[float] = None) -> LayerDesc:
    return LayerDesc(num_q_heads, num_kv_heads, head_dim, block_size, int(window), int(kv_dtype),
                     float(sm_scale if sm_scale is not None else head_dim ** -0.5))


def kv_view(k_cache: torch.Tensor, v_cache: torch.Tensor, seq_lens: torch.Tensor,
            block_table: Optional[torch.Tensor] = None, max_blocks_per_seq: Optional[int] = None,
            k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None) -> KVView:
    """Describe one layer's cache ([num_blocks][Hkv][16][D], uint8 codes or bf16; 4-bit: uint8
    [num_blocks][Hkv][FP4_BLOCK_BYTES]) for this batch.

    The view holds raw pointers: keep the tensors alive while it is in use."""
    if block_table is not None:
        max_blocks_per_seq = block_table.shape[1]
    if max_blocks_per_seq is None:
        raise ValueError("max_blocks_per_seq is required without a block table")
    v = KVView()
    v.k_cache = k_cache.data_ptr() if k_cache.is_cuda and k_cache.is_contiguous() else None
    v.v_cache = v_cache.data_ptr() if v_cache.is_cuda and v_cache.is_contiguous() else None
    v.num_blocks = k_cache.shape[0]
    v.block_table = _p(block_table, torch.int32, "block_table")
    v.max_blocks_per_seq = int(max_blocks_per_seq)
    v.seq_lens = _p(seq_lens, torch.int32, "seq_lens")
    v.k_scale = _p(k_scale, torch.float32, "k_scale")
    v.v_scale = _p(v_scale, torch.float32, "v_scale")
    v._held = (_device_of("a cache view", k_cache, v_cache, seq_lens, block_table, k_scale, v_scale),
               min(seq_lens.numel(), _ANY if block_table is None else block_table.shape[0]),
               min(_ANY if t is None else t.numel() for t in (k_scale, v_scale)), min(k_cache.nbytes, v_cache.nbytes))
    return v


def puzzle_status_string(code: int) -> str:
    return _load().puzzle_status_string(int(code)).decode()


def puzzle_launch_count() -> int:
    return int(_load().puzzle_launch_count())


def puzzle_decode_attn_kernel_name(desc: "LayerDesc", kv: "KVView", batch: int, num_splits: int = 0) -> str:
    return _load().puzzle_decode_attn_kernel_name(ctypes.byref(desc), ctypes.byref(kv), int(batch),
                                                  int(num_splits)).decode()


def _check(code: int, where: str):
    if code != 0:
        raise PuzzleError(code, where)


def puzzle_kv_append(desc: LayerDesc, view: KVView, k_new: torch.Tensor, v_new: torch.Tensor,
                     dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(_native().kv_append(desc, view, k_new, v_new, dev_status, stream), "puzzle_kv_append")


def puzzle_kv_amax_update(x: torch.Tensor, amax: torch.Tensor, stream=None) -> None:
    """x: bf16 [n_tokens][Hkv][D] (any leading dims, flattened); amax: float32 [Hkv], raised in place."""
    hkv, d = x.shape[-2], x.shape[-1]
    n_tokens = x.numel() // (hkv * d) if x.numel() else 0
    _check(_load().puzzle_kv_amax_update(_arg(x, torch.bfloat16, "x"), n_tokens, hkv, d, _arg(amax, torch.float32, "amax", hkv),
                                         _stream(stream, x)), "puzzle_kv_amax_update")


def puzzle_kv_scales_from_amax(amax: torch.Tensor, scale_out: torch.Tensor, pow2: bool = False, stream=None) -> None:
    _check(_load().puzzle_kv_scales_from_amax(_arg(amax, torch.float32, "amax"), amax.numel(), int(bool(pow2)),
                                              _arg(scale_out, torch.float32, "scale_out", amax.numel()), _stream(stream)),
           "puzzle_kv_scales_from_amax")


def calibrate_scales(chunks, num_kv_heads: int, pow2: bool = False, device="cuda") -> torch.Tensor:
    """Max-calibrated scales [num_kv_heads] from an iterable of bf16 tensors [..., Hkv, D] (argument
    marshalling only: one amax update per chunk, then the quotient)."""
    amax = torch.zeros(num_kv_heads, dtype=torch.float32, device=device)
    for x in chunks:
        puzzle_kv_amax_update(x, amax)
    scale = torch.empty_like(amax)
    puzzle_kv_scales_from_amax(amax, scale, pow2)
    return scale


def puzzle_kv_append_tokens(desc: LayerDesc, view: KVView, k_new: torch.Tensor, v_new: torch.Tensor,
                            new_lens: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                            stream=None) -> None:
    """k_new, v_new: bf16 [batch][n_new][Hkv][D]; new_lens: int32 [batch] or None (all n_new tokens are real)."""
    _check(_native().kv_append_tokens(desc, view, k_new, v_new, new_lens, dev_status, stream), "puzzle_kv_append_tokens")


def rope_view(cos_sin: torch.Tensor, interleaved: bool = False, pos_offset: Optional[torch.Tensor] = None) -> Rope:
    """Describe a rotation table: float32 [num_positions][rotary_dim], the cosines of a position and then its sines
    (``rope_table`` makes one); pos_offset: int32 [batch] or None.  The description keeps both tensors alive."""
    r = Rope()
    r.cos_sin = _p(cos_sin, torch.float32, "cos_sin")
    r.num_positions, r.rotary_dim = cos_sin.shape
    r.interleaved = int(bool(interleaved))
    r.pos_offset = _p(pos_offset, torch.int32, "pos_offset")
    r._held = (_device_of("a rotation", cos_sin, pos_offset), _ANY if pos_offset is None else pos_offset.numel())
    r._tensors = (cos_sin, pos_offset)
    return r


def puzzle_kv_append_rope(desc: LayerDesc, view: KVView, rope: Rope, q: Optional[torch.Tensor], k_new: torch.Tensor,
                          v_new: torch.Tensor, q_out: Optional[torch.Tensor] = None,
                          new_lens: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    """q, k_new, v_new: bf16 [batch][n_new][heads][D] (or [batch][heads][D] for one token each), contiguous or slices
    of a wider array along the heads; q_out: bf16 [batch][n_new][Hq][D] contiguous, may be q; q None: k and v only."""
    _check(_native().kv_append_rope(desc, view, rope, q, k_new, v_new, q_out, new_lens, dev_status, stream),
           "puzzle_kv_append_rope")


def puzzle_kv_read_tokens(desc: LayerDesc, view: KVView, k_out: torch.Tensor, v_out: torch.Tensor,
                          read_lens: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    """k_out, v_out: bf16 [batch][n_read][Hkv][D]; read_lens: int32 [batch] or None (n_read tokens of every sequence)."""
    _check(_native().kv_read_tokens(desc, view, k_out, v_out, read_lens, dev_status, stream), "puzzle_kv_read_tokens")


def puzzle_decode_attn_tokens_workspace_bytes(desc: LayerDesc, batch: int, n_q: int) -> int:
    return int(_load().puzzle_decode_attn_tokens_workspace_bytes(ctypes.byref(desc), int(batch), int(n_q)))


def puzzle_decode_attn_tokens_workspace_init(desc: LayerDesc, batch: int, n_q: int, workspace: torch.Tensor,
                                             stream=None) -> None:
    _check(_load().puzzle_decode_attn_tokens_workspace_init(ctypes.byref(desc), int(batch), int(n_q), _arg(workspace, None, "workspace"),
                                                            workspace.numel() * workspace.element_size(),
                                                            _stream(stream)), "puzzle_decode_attn_tokens_workspace_init")


def puzzle_decode_attn_tokens(desc: LayerDesc, view: KVView, q: torch.Tensor, sinks: Optional[torch.Tensor],
                              out: torch.Tensor, lse_out: Optional[torch.Tensor] = None,
                              q_lens: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                              dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """q, out: bf16 [batch][n_q][Hq][D]; q_lens: int32 [batch] or None; see include/puzzle_attn.h."""
    if workspace is None:
        raise ValueError("a workspace tensor is required (see puzzle_decode_attn_tokens_workspace_bytes)")
    _check(_native().decode_attn_tokens(desc, view, q, q_lens, sinks, out, lse_out, workspace, dev_status, stream),
           "puzzle_decode_attn_tokens")


def puzzle_decode_attn_workspace_bytes(desc: LayerDesc, batch: int, num_splits: int = 0) -> int:
    return int(_load().puzzle_decode_attn_workspace_bytes(ctypes.byref(desc), int(batch), int(num_splits)))


def puzzle_decode_attn_workspace_init(desc: LayerDesc, batch: int, workspace: torch.Tensor, stream=None) -> None:
    _check(_load().puzzle_decode_attn_workspace_init(ctypes.byref(desc), int(batch), _arg(workspace, None, "workspace"),
                                                     workspace.numel() * workspace.element_size(), _stream(stream)),
           "puzzle_decode_attn_workspace_init")


def puzzle_decode_attn(desc: LayerDesc, view: KVView, q: torch.Tensor, sinks: Optional[torch.Tensor],
                       out: torch.Tensor, lse_out: Optional[torch.Tensor] = None, num_splits: int = 0,
                       workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                       stream=None) -> None:
    if workspace is None:
        raise ValueError("workspace is required (size it with puzzle_decode_attn_workspace_bytes)")
    _check(_native().decode_attn(desc, view, q, sinks, out, lse_out, num_splits, workspace, dev_status, stream),
           "puzzle_decode_attn")


def puzzle_decode_attn_tcgen05(desc: LayerDesc, view: KVView, q: torch.Tensor, sinks: Optional[torch.Tensor],
                               out: torch.Tensor, lse_out: Optional[torch.Tensor] = None, num_splits: int = 0,
                               workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                               stream=None) -> None:
    """puzzle_decode_attn computed by the tcgen05 / tensor-memory kernel (FP8 caches only)."""
    if workspace is None:
        raise ValueError("workspace is required (size it with puzzle_decode_attn_workspace_bytes)")
    _check(_native().decode_attn_tcgen05(desc, view, q, sinks, out, lse_out, num_splits, workspace, dev_status, stream),
           "puzzle_decode_attn_tcgen05")


def puzzle_decode_attn_static(desc: LayerDesc, view: KVView, q: torch.Tensor, sinks: Optional[torch.Tensor],
                              out: torch.Tensor, lse_out: Optional[torch.Tensor] = None, num_splits: int = 0,
                              dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """puzzle_decode_attn on the library's built-in 8 MiB scratch: for callers that cannot allocate device
    memory (no workspace tensor is involved, and nothing is allocated on the way).  Calls that share a
    device must not overlap on the GPU; make the first call on a device outside any stream capture."""
    batch = q.shape[0]
    _check_view(desc, view, batch)
    n, heads, _ = _rows(desc, batch)
    _check(_load().puzzle_decode_attn_static(ctypes.byref(desc), ctypes.byref(view), _arg(q, torch.bfloat16, "q", n),
                                             _arg(sinks, torch.float32, "sinks", heads // batch if batch else 0),
                                             _arg(out, torch.bfloat16, "out", n),
                                             _arg(lse_out, torch.float32, "lse_out", heads), batch, int(num_splits),
                                             _arg(dev_status, torch.int32, "dev_status", 1), _stream(stream, q)),
           "puzzle_decode_attn_static")


def puzzle_decode_step_host_staging_bytes(desc: LayerDesc, batch: int) -> int:
    return int(_load().puzzle_decode_step_host_staging_bytes(ctypes.byref(desc), int(batch)))


def _host_ptr(t: torch.Tensor, name: str, need: int):
    if t.is_cuda or not t.is_contiguous() or t.dtype != torch.bfloat16:
        raise ValueError("%s must be a contiguous bf16 host tensor" % name)
    if t.numel() < need:
        raise ValueError("%s has %d elements, the call needs %d" % (name, t.numel(), need))
    return t.data_ptr()


def puzzle_decode_step_host(desc: LayerDesc, view: KVView, q_host: torch.Tensor, k_new_host: torch.Tensor,
                            v_new_host: torch.Tensor, sinks: Optional[torch.Tensor], out_host: torch.Tensor,
                            staging: torch.Tensor, workspace: torch.Tensor, num_splits: int = 0,
                            dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Append + attention of one layer with q, k_new, v_new and out in host memory (pinned for asynchronous copies);
    staging and workspace are device tensors.  Synchronise the stream before reading out_host."""
    batch = q_host.shape[0]
    n, heads, kn = _rows(desc, batch)
    q, k, v, out = (_host_ptr(t, name, need) for t, name, need in (
        (q_host, "q_host", n), (k_new_host, "k_new_host", kn), (v_new_host, "v_new_host", kn), (out_host, "out_host", n)))
    _check_view(desc, view, batch)
    _check(_load().puzzle_decode_step_host(ctypes.byref(desc), ctypes.byref(view), q, k, v,
                                           _arg(sinks, torch.float32, "sinks", heads // batch if batch else 0), out, batch,
                                           int(num_splits), _arg(staging, None, "staging"),
                                           staging.numel() * staging.element_size(), _arg(workspace, None, "workspace"),
                                           workspace.numel() * workspace.element_size(),
                                           _arg(dev_status, torch.int32, "dev_status", 1), _stream(stream, workspace)),
           "puzzle_decode_step_host")


def puzzle_decode_attn_partial(desc: LayerDesc, view: KVView, q: torch.Tensor, o_part: torch.Tensor,
                               lse_part: torch.Tensor, num_splits: int = 0, workspace: Optional[torch.Tensor] = None,
                               dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """This device's float32 partial (o, lse) over the keys its view holds, no sink: see the header."""
    if workspace is None:
        raise ValueError("workspace is required (size it with puzzle_decode_attn_workspace_bytes)")
    batch = q.shape[0]
    _check_view(desc, view, batch)
    n, heads, _ = _rows(desc, batch)
    _check(_load().puzzle_decode_attn_partial(ctypes.byref(desc), ctypes.byref(view), _arg(q, torch.bfloat16, "q", n),
                                              _arg(o_part, torch.float32, "o_part", n),
                                              _arg(lse_part, torch.float32, "lse_part", heads), batch, int(num_splits),
                                              _arg(workspace, None, "workspace"), workspace.numel() * workspace.element_size(),
                                              _arg(dev_status, torch.int32, "dev_status", 1), _stream(stream, q)),
           "puzzle_decode_attn_partial")


def puzzle_attn_merge_strided(part_o: torch.Tensor, part_lse: torch.Tensor, o_row_stride: int, o_part_stride: int,
                              lse_row_stride: int, lse_part_stride: int, num_parts: Optional[torch.Tensor],
                              sinks: Optional[torch.Tensor], out: torch.Tensor, num_parts_max: int,
                              lse_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """part_o / part_lse: float32 tensors whose first elements are part 0 of row 0 (strides in floats)."""
    batch, hq, d = out.shape
    # with num_parts given, how many parts there are is known on the device alone: one is asked for
    last, parts = max(batch * hq - 1, 0), max(int(num_parts_max) - 1, 0) if num_parts is None else 0
    _check(_load().puzzle_attn_merge_strided(
        _reach(part_o, torch.float32, "part_o", last * int(o_row_stride) + parts * int(o_part_stride) + d),
        _reach(part_lse, torch.float32, "part_lse", last * int(lse_row_stride) + parts * int(lse_part_stride) + 1),
        int(o_row_stride), int(o_part_stride), int(lse_row_stride), int(lse_part_stride),
        _arg(num_parts, torch.int32, "num_parts", batch), _arg(sinks, torch.float32, "sinks", hq),
        _arg(out, torch.bfloat16, "out"), _arg(lse_out, torch.float32, "lse_out", batch * hq), batch, hq, d,
        int(num_parts_max), _stream(stream)), "puzzle_attn_merge_strided")


def puzzle_attn_merge(part_o: torch.Tensor, part_lse: torch.Tensor, num_parts: Optional[torch.Tensor],
                      sinks: Optional[torch.Tensor], out: torch.Tensor, lse_out: Optional[torch.Tensor] = None,
                      stream=None) -> None:
    batch, hq, s, d = part_o.shape
    _check(_load().puzzle_attn_merge(_arg(part_o, torch.float32, "part_o"),
                                     _arg(part_lse, torch.float32, "part_lse", batch * hq * s),
                                     _arg(num_parts, torch.int32, "num_parts", batch), _arg(sinks, torch.float32, "sinks", hq),
                                     _arg(out, torch.bfloat16, "out", batch * hq * d),
                                     _arg(lse_out, torch.float32, "lse_out", batch * hq), batch, hq, d, s, _stream(stream)),
           "puzzle_attn_merge")


def puzzle_hbm_read_probe(buf: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    _check(_load().puzzle_hbm_read_probe(_arg(buf, None, "buf"), buf.numel() * buf.element_size(),
                                         _arg(sink, None, "sink", -(-8 // sink.element_size())), _stream(stream)),
           "puzzle_hbm_read_probe")
