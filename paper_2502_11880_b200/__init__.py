"""Python binding of libbitnet_b200.so: same names as the C ABI, argument marshalling only (ctypes; the calls of the key-value
cache and the attention, which a decode step makes by the dozen, through a small compiled module).

Every step of the path (quantiser, packers, mpGEMV / mpGEMM, rescale) runs in the library's CUDA
kernels.  PyTorch supplies device memory and streams.  There is no CPU fallback: if the shared
library is missing or fails to load, importing a symbol from here raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os

import torch

from . import synth  # noqa: F401  (seeded inputs; holds none of the method's arithmetic)

_PKG = os.path.dirname(os.path.abspath(__file__))
# BITNET_B200_LIB points at another build of the library (e.g. one compiled with different flags)
LIB_PATH = os.environ.get("BITNET_B200_LIB") or os.path.join(_PKG, "libbitnet_b200.so")

FMT_I2S, FMT_TL1, FMT_TL2 = 0, 1, 2
FMT = {"i2s": FMT_I2S, "tl1": FMT_TL1, "tl2": FMT_TL2}

# symbols the header declares (checked by the tests against include/bitnet_b200.h)
SYMBOLS = [
    "bitnet_status_string", "bitnet_last_cuda_error", "bitnet_quant_act", "bitnet_i2s_packed_bytes",
    "bitnet_pack_i2s", "bitnet_tl_packed_bytes", "bitnet_pack_tl", "bitnet_mpgemm_workspace_bytes",
    "bitnet_workspace_init", "bitnet_mpgemm", "bitnet_linear", "bitnet_linear_host", "bitnet_linear_host_batch", "bitnet_unpack_i2s", "bitnet_unpack_tl",
    "bitnet_tl_num_groups", "bitnet_tl_build_lut_debug", "bitnet_mpgemv_tl_noalloc", "bitnet_device_status",
    "bitnet_set_early_start", "bitnet_set_tl2_lookup", "bitnet_device_status_clear", "bitnet_debug_wait_timeout_probe", "bitnet_linear_group", "bitnet_linear_segments", "bitnet_microbench_read_stream", "bitnet_microbench_issue",
    "bitnet_elut_packed_bytes", "bitnet_pack_elut", "bitnet_unpack_elut", "bitnet_elut_linear_group",
    "bitnet_kv_cache_init", "bitnet_kv_append", "bitnet_kv_reserve", "bitnet_kv_workspace_bytes", "bitnet_kv_fork", "bitnet_kv_free",
    "bitnet_kv_trim", "bitnet_kv_compact", "bitnet_kv_copy_pages", "bitnet_attn_workspace_bytes", "bitnet_attn_decode", "bitnet_attn_prompt",
    "bitnet_debug_attn_give_up", "bitnet_attn_shared", "bitnet_attn_shared_workspace_bytes", "bitnet_rope_init", "bitnet_kv_append_rope",
    "bitnet_add_rmsnorm_quant", "bitnet_sample", "bitnet_debug_attn_shared",
]

_lib = None


class BitnetError(RuntimeError):
    pass


def lib():
    """Loads the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise BitnetError(f"{LIB_PATH} is missing: run `python -m paper_2502_11880_b200.build` "
                              "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        i64, vp, ci, sz, fl = C.c_int64, C.c_void_p, C.c_int, C.c_size_t, C.c_float
        L.bitnet_status_string.argtypes = [ci]
        L.bitnet_status_string.restype = C.c_char_p
        L.bitnet_last_cuda_error.restype = ci
        L.bitnet_device_status.argtypes = [vp]
        L.bitnet_debug_wait_timeout_probe.argtypes = [vp]
        L.bitnet_debug_attn_give_up.argtypes = [i64]
        L.bitnet_debug_attn_give_up.restype = None
        L.bitnet_debug_attn_shared.argtypes = [ci]
        L.bitnet_debug_attn_shared.restype = None
        L.bitnet_set_early_start.argtypes = [ci]
        L.bitnet_set_early_start.restype = None
        L.bitnet_set_tl2_lookup.argtypes = [ci]
        L.bitnet_set_tl2_lookup.restype = None
        L.bitnet_quant_act.argtypes = [vp, i64, i64, ci, vp, vp, vp, vp]
        L.bitnet_i2s_packed_bytes.argtypes = [i64, i64]
        L.bitnet_i2s_packed_bytes.restype = sz
        L.bitnet_pack_i2s.argtypes = [vp, i64, i64, vp, sz, vp, vp]
        L.bitnet_tl_packed_bytes.argtypes = [ci, i64, i64, ci]
        L.bitnet_tl_packed_bytes.restype = sz
        L.bitnet_pack_tl.argtypes = [ci, vp, i64, i64, ci, vp, sz, vp, vp]
        L.bitnet_mpgemm_workspace_bytes.argtypes = [ci, i64, i64, i64]
        L.bitnet_mpgemm_workspace_bytes.restype = sz
        L.bitnet_workspace_init.argtypes = [vp, sz, vp]
        L.bitnet_mpgemm.argtypes = [ci, vp, fl, i64, i64, ci, vp, vp, i64, vp, vp, vp, sz, vp]
        L.bitnet_linear.argtypes = [ci, vp, fl, i64, i64, ci, vp, i64, vp, vp, vp, vp, vp, sz, vp]
        L.bitnet_linear_host.argtypes = [ci, vp, fl, i64, i64, ci, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        L.bitnet_linear_host_batch.argtypes = [vp, i64, vp]
        L.bitnet_linear_group.argtypes = [vp, i64, vp]
        L.bitnet_linear_segments.argtypes = [ci, vp, i64, i64, ci, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp, sz, vp]
        L.bitnet_microbench_read_stream.argtypes = [vp, sz, ci, vp, vp]
        L.bitnet_microbench_issue.argtypes = [ci, ci, vp, vp]
        L.bitnet_unpack_i2s.argtypes = [vp, i64, i64, vp, vp, vp]
        L.bitnet_unpack_tl.argtypes = [ci, vp, i64, i64, ci, vp, vp, vp]
        L.bitnet_tl_num_groups.argtypes = [ci, i64, ci]
        L.bitnet_tl_num_groups.restype = i64
        L.bitnet_tl_build_lut_debug.argtypes = [ci, vp, i64, ci, vp, vp]
        L.bitnet_mpgemv_tl_noalloc.argtypes = [ci, vp, fl, i64, i64, ci, vp, vp, i64, vp, vp, vp]
        L.bitnet_elut_packed_bytes.argtypes = [ci, ci, i64, i64]
        L.bitnet_elut_packed_bytes.restype = sz
        L.bitnet_pack_elut.argtypes = [ci, ci, vp, i64, i64, vp, sz, vp, vp]
        L.bitnet_unpack_elut.argtypes = [ci, ci, vp, i64, i64, vp, vp, vp]
        L.bitnet_elut_linear_group.argtypes = [vp, i64, vp]
        L.bitnet_kv_cache_init.argtypes = [vp]
        L.bitnet_kv_append.argtypes = [vp, i64, vp, vp, ci, i64, i64, i64, vp, i64, vp, vp, i64, vp, vp]
        L.bitnet_kv_reserve.argtypes = [vp, i64, vp, i64, i64, vp, vp, i64, vp, vp]
        L.bitnet_kv_workspace_bytes.argtypes = [i64, i64]
        L.bitnet_kv_workspace_bytes.restype = sz
        L.bitnet_kv_fork.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp, i64, vp, sz, vp, vp]
        L.bitnet_kv_free.argtypes = [vp, i64, vp, i64, i64, vp, vp, i64, vp, vp]
        L.bitnet_kv_trim.argtypes = [vp, i64, vp, i64, i64, vp, i64, i64, i64, vp]
        L.bitnet_kv_compact.argtypes = [vp, vp, vp, i64, i64, vp, vp, sz, vp]
        L.bitnet_kv_copy_pages.argtypes = [vp, vp, vp, i64, vp, vp]
        L.bitnet_attn_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.bitnet_attn_workspace_bytes.restype = sz
        L.bitnet_attn_decode.argtypes = [vp, i64, vp, ci, i64, i64, i64, vp, i64, vp, i64, fl, i64, i64, vp, vp, sz, vp, vp]
        L.bitnet_attn_prompt.argtypes = [vp, i64, vp, ci, i64, i64, i64, i64, vp, i64, vp, vp, i64, i64, fl, i64, i64, vp, vp, sz, vp, vp]
        L.bitnet_attn_shared_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.bitnet_attn_shared_workspace_bytes.restype = sz
        L.bitnet_attn_shared.argtypes = [vp, i64, vp, ci, i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, fl, i64, i64, vp, vp, sz, vp, vp]
        L.bitnet_rope_init.argtypes = [vp]
        L.bitnet_kv_append_rope.argtypes = [vp, i64, vp, vp, i64, i64, i64, vp, vp, ci, i64, i64, i64, vp, i64, vp, vp, i64, vp, ci, vp, vp]
        L.bitnet_add_rmsnorm_quant.argtypes = [vp, ci, i64, vp, ci, i64, vp, i64, vp, ci, fl, i64, i64, vp, ci, vp, vp, vp, vp]
        L.bitnet_sample.argtypes = [vp, ci, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp]
        _lib = L
    return _lib


def status_string(rc: int) -> str:
    return lib().bitnet_status_string(rc).decode()


def bitnet_device_status() -> int:
    """Synchronises the device and returns the device-side status flag (0 = no bounded wait ever gave up)."""
    out = C.c_int(0)
    _check(lib().bitnet_device_status(C.byref(out)), "bitnet_device_status")
    return out.value


def bitnet_device_status_clear():
    _check(lib().bitnet_device_status_clear(), "bitnet_device_status_clear")


def bitnet_debug_wait_timeout_probe(stream=None):
    """Test hook: a kernel whose bounded wait runs out (sets the device status flag to BITNET_ERR_TIMEOUT)."""
    _check(lib().bitnet_debug_wait_timeout_probe(_stream(stream)), "bitnet_debug_wait_timeout_probe")


def bitnet_debug_attn_give_up(tile):
    """Test hook: CTAs of the attention kernels give up before their tile-th tile of cached tokens (-1: off)."""
    lib().bitnet_debug_attn_give_up(tile)


def bitnet_debug_attn_shared(always: bool):
    """Test hook: bitnet_attn_shared hands no call to the decode kernel."""
    lib().bitnet_debug_attn_shared(int(bool(always)))


def bitnet_set_early_start(enable: bool):
    lib().bitnet_set_early_start(int(bool(enable)))


def bitnet_set_tl2_lookup(enable: bool):
    """True: TL2 decode batches run the activation-table kernel of Alg. 2 instead of the scan kernel."""
    lib().bitnet_set_tl2_lookup(int(bool(enable)))


def _check(rc: int, what: str):
    if rc != 0:
        extra = f", cudaError {lib().bitnet_last_cuda_error()}" if rc == 5 else ""
        raise BitnetError(f"{what}: {status_string(rc)} (status {rc}{extra})")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _fmt(fmt) -> int:
    return FMT[fmt] if isinstance(fmt, str) else int(fmt)


def _dev(t, dtype, name):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise BitnetError(f"{name}: expected a contiguous CUDA tensor of {dtype}")
    return t


# ------------------------------------------------------------------------------------------------
def bitnet_quant_act(x, per_tensor=False, q=None, act_scale=None, act_sum=None, stream=None):
    """x[T][K] fp32 (CUDA) -> (q int8 [T][K], act_scale fp32 [T], act_sum int32 [T])."""
    _dev(x, torch.float32, "x")
    T, K = x.shape
    q = torch.empty((T, K), dtype=torch.int8, device=x.device) if q is None else q
    act_scale = torch.empty(T, dtype=torch.float32, device=x.device) if act_scale is None else act_scale
    act_sum = torch.empty(T, dtype=torch.int32, device=x.device) if act_sum is None else act_sum
    _check(lib().bitnet_quant_act(_ptr(x), T, K, int(per_tensor), _ptr(q), _ptr(act_scale), _ptr(act_sum),
                                  _stream(stream)), "bitnet_quant_act")
    return q, act_scale, act_sum


def bitnet_i2s_packed_bytes(M, K) -> int:
    return lib().bitnet_i2s_packed_bytes(M, K)


def bitnet_tl_packed_bytes(fmt, M, K, bk3=0) -> int:
    return lib().bitnet_tl_packed_bytes(_fmt(fmt), M, K, bk3)


def packed_bytes(fmt, M, K, bk3=0) -> int:
    return bitnet_i2s_packed_bytes(M, K) if _fmt(fmt) == FMT_I2S else bitnet_tl_packed_bytes(fmt, M, K, bk3)


def _status_word(device):
    return torch.zeros(1, dtype=torch.int32, device=device)


def bitnet_pack_i2s(w, check=True, stream=None):
    """w[M][K] int8 ternary (CUDA) -> uint8 blob.  check=True reads the device status word back."""
    _dev(w, torch.int8, "w")
    M, K = w.shape
    n = bitnet_i2s_packed_bytes(M, K)
    if n == 0:
        _check(2, "bitnet_pack_i2s")
    out = torch.empty(n, dtype=torch.uint8, device=w.device)
    st = _status_word(w.device) if check else None
    _check(lib().bitnet_pack_i2s(_ptr(w), M, K, _ptr(out), n, _ptr(st), _stream(stream)), "bitnet_pack_i2s")
    if check:
        _check(int(st.item()), "bitnet_pack_i2s")
    return out


def bitnet_pack_tl(fmt, w, bk3=0, check=True, stream=None):
    _dev(w, torch.int8, "w")
    M, K = w.shape
    n = bitnet_tl_packed_bytes(fmt, M, K, bk3)
    if n == 0:
        _check(2, "bitnet_pack_tl")
    out = torch.empty(n, dtype=torch.uint8, device=w.device)
    st = _status_word(w.device) if check else None
    _check(lib().bitnet_pack_tl(_fmt(fmt), _ptr(w), M, K, bk3, _ptr(out), n, _ptr(st), _stream(stream)),
           "bitnet_pack_tl")
    if check:
        _check(int(st.item()), "bitnet_pack_tl")
    return out


def pack(fmt, w, bk3=0, check=True):
    return bitnet_pack_i2s(w, check) if _fmt(fmt) == FMT_I2S else bitnet_pack_tl(fmt, w, bk3, check)


def bitnet_unpack_i2s(packed, M, K, stream=None):
    w = torch.empty((M, K), dtype=torch.int8, device=packed.device)
    st = _status_word(packed.device)
    _check(lib().bitnet_unpack_i2s(_ptr(packed), M, K, _ptr(w), _ptr(st), _stream(stream)), "bitnet_unpack_i2s")
    _check(int(st.item()), "bitnet_unpack_i2s")
    return w


def bitnet_unpack_tl(fmt, packed, M, K, bk3=0, stream=None):
    w = torch.empty((M, K), dtype=torch.int8, device=packed.device)
    st = _status_word(packed.device)
    _check(lib().bitnet_unpack_tl(_fmt(fmt), _ptr(packed), M, K, bk3, _ptr(w), _ptr(st), _stream(stream)),
           "bitnet_unpack_tl")
    _check(int(st.item()), "bitnet_unpack_tl")
    return w


def bitnet_tl_num_groups(fmt, K, bk3=0) -> int:
    return lib().bitnet_tl_num_groups(_fmt(fmt), K, bk3)


def bitnet_tl_build_lut_debug(fmt, q_row, bk3=0, stream=None):
    _dev(q_row, torch.int8, "q_row")
    K = q_row.numel()
    ng = bitnet_tl_num_groups(fmt, K, bk3)
    if ng < 0:
        _check(2, "bitnet_tl_build_lut_debug")
    lut = torch.empty((ng, 16), dtype=torch.int16, device=q_row.device)
    _check(lib().bitnet_tl_build_lut_debug(_fmt(fmt), _ptr(q_row), K, bk3, _ptr(lut), _stream(stream)),
           "bitnet_tl_build_lut_debug")
    return lut


def bitnet_mpgemm_workspace_bytes(fmt, T, M, K) -> int:
    return lib().bitnet_mpgemm_workspace_bytes(_fmt(fmt), T, M, K)


def bitnet_workspace_init(workspace, stream=None):
    _check(lib().bitnet_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream(stream)), "bitnet_workspace_init")


def new_workspace(fmt, T, M, K, device="cuda"):
    """A zeroed workspace tensor for bitnet_mpgemm (None when the shape needs none)."""
    n = bitnet_mpgemm_workspace_bytes(fmt, T, M, K)
    if n == 0:
        return None
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    bitnet_workspace_init(ws)
    return ws


def bitnet_mpgemm(fmt, packed, w_scale, M, K, q, act_scale, bk3=0, y=None, acc_out=None, want_acc=False,
                  workspace=None, stream=None):
    """y[T][M] fp32 = (q @ W^T) * act_scale[t] * w_scale from the packed blob.  Returns (y, acc or None)."""
    _dev(q, torch.int8, "q")
    _dev(act_scale, torch.float32, "act_scale")
    T = q.shape[0]
    y = torch.empty((T, M), dtype=torch.float32, device=q.device) if y is None else y
    if want_acc and acc_out is None:
        acc_out = torch.empty((T, M), dtype=torch.int32, device=q.device)
    if workspace is None:
        workspace = new_workspace(fmt, T, M, K, q.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().bitnet_mpgemm(_fmt(fmt), _ptr(packed), float(w_scale), M, K, bk3, _ptr(q), _ptr(act_scale), T,
                               _ptr(y), _ptr(acc_out), _ptr(workspace), ws_bytes, _stream(stream)),
           "bitnet_mpgemm")
    return y, acc_out


def bitnet_linear(fmt, packed, w_scale, M, K, x, bk3=0, q=None, act_scale=None, y=None, acc_out=None, want_acc=False,
                  workspace=None, stream=None):
    """fp32 activations x[T][K] (CUDA) -> (y, q, act_scale, acc or None): quantiser + mpGEMM + rescale."""
    _dev(x, torch.float32, "x")
    T = x.shape[0]
    q = torch.empty((T, K), dtype=torch.int8, device=x.device) if q is None else q
    act_scale = torch.empty(T, dtype=torch.float32, device=x.device) if act_scale is None else act_scale
    y = torch.empty((T, M), dtype=torch.float32, device=x.device) if y is None else y
    if want_acc and acc_out is None:
        acc_out = torch.empty((T, M), dtype=torch.int32, device=x.device)
    if workspace is None:
        workspace = new_workspace(fmt, T, M, K, x.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().bitnet_linear(_fmt(fmt), _ptr(packed), float(w_scale), M, K, bk3, _ptr(x), T, _ptr(q),
                               _ptr(act_scale), _ptr(y), _ptr(acc_out), _ptr(workspace), ws_bytes, _stream(stream)),
           "bitnet_linear")
    return y, q, act_scale, acc_out


def bitnet_linear_host(fmt, packed, w_scale, M, K, x_host, y_host, x_dev, q_dev, scale_dev, y_dev,
                       workspace=None, bk3=0, stream=None):
    """Host fp32 activations in, host fp32 results out (copies queued on the stream; caller synchronises)."""
    T = x_host.shape[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().bitnet_linear_host(_fmt(fmt), _ptr(packed), float(w_scale), M, K, bk3, _ptr(x_host), T,
                                    _ptr(y_host), _ptr(x_dev), _ptr(q_dev), _ptr(scale_dev), _ptr(y_dev),
                                    _ptr(workspace), ws_bytes, _stream(stream)), "bitnet_linear_host")


class HostLinear(C.Structure):
    """Mirror of bitnet_host_linear_t."""
    _fields_ = [("fmt", C.c_int32), ("bk3", C.c_int32), ("packed", C.c_void_p), ("w_scale", C.c_float),
                ("M", C.c_int64), ("K", C.c_int64), ("T", C.c_int64), ("x_host", C.c_void_p), ("y_host", C.c_void_p),
                ("x_dev", C.c_void_p), ("q_dev", C.c_void_p), ("scale_dev", C.c_void_p), ("y_dev", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


def make_host_batch(items):
    """items: dicts with fmt, packed, w_scale, M, K, x_host, y_host, x_dev, q_dev, scale_dev, y_dev and
    optionally workspace, bk3 (tensors).  Returns the ctypes array for bitnet_linear_host_batch; the caller
    keeps the tensors alive."""
    arr = (HostLinear * len(items))()
    for a, d in zip(arr, items):
        ws = d.get("workspace")
        a.fmt, a.bk3, a.packed, a.w_scale = _fmt(d["fmt"]), int(d.get("bk3", 0)), d["packed"].data_ptr(), float(d["w_scale"])
        a.M, a.K, a.T = int(d["M"]), int(d["K"]), int(d["x_host"].shape[0])
        a.x_host, a.y_host = d["x_host"].data_ptr(), d["y_host"].data_ptr()
        a.x_dev, a.q_dev, a.scale_dev, a.y_dev = (d["x_dev"].data_ptr(), d["q_dev"].data_ptr(),
                                                  d["scale_dev"].data_ptr(), d["y_dev"].data_ptr())
        a.workspace = None if ws is None else ws.data_ptr()
        a.workspace_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    return arr


def bitnet_linear_host_batch(batch, stream=None):
    """Queues a batch made by make_host_batch: uploads, kernels and downloads overlap; the caller
    synchronises the stream before reading the host results."""
    _check(lib().bitnet_linear_host_batch(batch, C.c_int64(len(batch)), _stream(stream)), "bitnet_linear_host_batch")


def bitnet_linear_segments(fmt, packed, M, K, seg_end, seg_scale, x, bk3=0, q=None, act_scale=None, y=None, acc_out=None,
                           want_acc=False, workspace=None, stream=None):
    """bitnet_linear for a tensor of row-stacked matrices with one weight scale each: rows [seg_end[s-1], seg_end[s])
    of y carry seg_scale[s].  Returns (y, q, act_scale, acc or None)."""
    _dev(x, torch.float32, "x")
    T = x.shape[0]
    q = torch.empty((T, K), dtype=torch.int8, device=x.device) if q is None else q
    act_scale = torch.empty(T, dtype=torch.float32, device=x.device) if act_scale is None else act_scale
    y = torch.empty((T, M), dtype=torch.float32, device=x.device) if y is None else y
    if want_acc and acc_out is None:
        acc_out = torch.empty((T, M), dtype=torch.int32, device=x.device)
    if workspace is None:
        workspace = new_workspace(fmt, T, M, K, x.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    n = len(seg_end)
    ends = (C.c_int64 * n)(*[int(v) for v in seg_end])
    scales = (C.c_float * n)(*[float(v) for v in seg_scale])
    _check(lib().bitnet_linear_segments(_fmt(fmt), _ptr(packed), M, K, bk3, n, ends, scales, _ptr(x), T, _ptr(q),
                                        _ptr(act_scale), _ptr(y), _ptr(acc_out), _ptr(workspace), ws_bytes, _stream(stream)),
           "bitnet_linear_segments")
    return y, q, act_scale, acc_out


class GroupItem(C.Structure):
    """Mirror of bitnet_group_item_t."""
    _fields_ = [("fmt", C.c_int32), ("bk3", C.c_int32), ("packed", C.c_void_p), ("w_scale", C.c_float),
                ("M", C.c_int64), ("K", C.c_int64), ("T", C.c_int64), ("x", C.c_void_p), ("q", C.c_void_p),
                ("act_scale", C.c_void_p), ("y", C.c_void_p), ("acc_out", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


def make_group(items):
    """items: dicts with fmt, packed, w_scale, M, K, x, q, act_scale, y and optionally acc_out, workspace, bk3
    (CUDA tensors).  Returns the ctypes array for bitnet_linear_group; the caller keeps the tensors alive."""
    arr = (GroupItem * len(items))()
    for a, d in zip(arr, items):
        ws, acc = d.get("workspace"), d.get("acc_out")
        a.fmt, a.bk3, a.packed, a.w_scale = _fmt(d["fmt"]), int(d.get("bk3", 0)), d["packed"].data_ptr(), float(d["w_scale"])
        a.M, a.K, a.T = int(d["M"]), int(d["K"]), int(d["x"].shape[0])
        a.x, a.q, a.act_scale, a.y = d["x"].data_ptr(), d["q"].data_ptr(), d["act_scale"].data_ptr(), d["y"].data_ptr()
        a.acc_out = None if acc is None else acc.data_ptr()
        a.workspace = None if ws is None else ws.data_ptr()
        a.workspace_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    return arr


def bitnet_linear_group(group, stream=None):
    """Queues a list of linears made by make_group (device buffers): one persistent kernel per run of I2_S
    decode items, bitnet_linear for the others."""
    _check(lib().bitnet_linear_group(group, C.c_int64(len(group)), _stream(stream)), "bitnet_linear_group")


# ---- element-wise tables beyond ternary (App. A): weights of cardinality C in groups of g
def bitnet_elut_packed_bytes(C_, g, M, K) -> int:
    return lib().bitnet_elut_packed_bytes(int(C_), int(g), M, K)


def bitnet_pack_elut(C_, g, w, check=True, stream=None):
    """w[M][K] int8 with values -(C//2) .. -(C//2)+C-1 (CUDA) -> uint8 blob of group indices."""
    _dev(w, torch.int8, "w")
    M, K = w.shape
    n = bitnet_elut_packed_bytes(C_, g, M, K)
    if n == 0:
        _check(2, "bitnet_pack_elut")
    out = torch.empty(n, dtype=torch.uint8, device=w.device)
    st = _status_word(w.device) if check else None
    _check(lib().bitnet_pack_elut(int(C_), int(g), _ptr(w), M, K, _ptr(out), n, _ptr(st), _stream(stream)),
           "bitnet_pack_elut")
    if check:
        _check(int(st.item()), "bitnet_pack_elut")
    return out


def bitnet_unpack_elut(C_, g, packed, M, K, stream=None):
    w = torch.empty((M, K), dtype=torch.int8, device=packed.device)
    st = _status_word(packed.device)
    _check(lib().bitnet_unpack_elut(int(C_), int(g), _ptr(packed), M, K, _ptr(w), _ptr(st), _stream(stream)),
           "bitnet_unpack_elut")
    _check(int(st.item()), "bitnet_unpack_elut")
    return w


class ElutItem(C.Structure):
    """Mirror of bitnet_elut_item_t."""
    _fields_ = [("C", C.c_int32), ("g", C.c_int32), ("packed", C.c_void_p), ("w_scale", C.c_float),
                ("M", C.c_int64), ("K", C.c_int64), ("T", C.c_int64), ("x", C.c_void_p), ("q", C.c_void_p),
                ("act_scale", C.c_void_p), ("y", C.c_void_p), ("acc_out", C.c_void_p)]


def make_elut_group(items):
    """items: dicts with C, g, packed, w_scale, M, K, q, act_scale, y and optionally x (fp32 activations: q and
    act_scale are then outputs) and acc_out (CUDA tensors).  Returns the ctypes array for bitnet_elut_linear_group;
    the caller keeps the tensors alive."""
    arr = (ElutItem * len(items))()
    for a, d in zip(arr, items):
        x, acc = d.get("x"), d.get("acc_out")
        a.C, a.g, a.packed, a.w_scale = int(d["C"]), int(d["g"]), d["packed"].data_ptr(), float(d["w_scale"])
        a.M, a.K, a.T = int(d["M"]), int(d["K"]), int(d["q"].shape[0])
        a.x = None if x is None else x.data_ptr()
        a.q, a.act_scale, a.y = d["q"].data_ptr(), d["act_scale"].data_ptr(), d["y"].data_ptr()
        a.acc_out = None if acc is None else acc.data_ptr()
    return arr


def bitnet_elut_linear_group(group, stream=None):
    """Queues a list made by make_elut_group: one persistent kernel per run of items with the same C."""
    _check(lib().bitnet_elut_linear_group(group, C.c_int64(len(group)), _stream(stream)), "bitnet_elut_linear_group")


MICROBENCH_KINDS = {"dp4a": 0, "lop3": 1, "prmt": 2, "imad": 3, "lds32": 4, "lds128": 5, "mma_u8s8_m16n8k32": 6}


def bitnet_microbench_read_stream(buf, depth, sink, stream=None):
    """Queues one read of `buf` (CUDA uint8 tensor) with the grouped decode kernel's copy pattern and no arithmetic."""
    _check(lib().bitnet_microbench_read_stream(_ptr(buf), buf.numel() * buf.element_size(), int(depth), _ptr(sink),
                                               _stream(stream)), "bitnet_microbench_read_stream")


def bitnet_microbench_issue(kind, iters, sink, stream=None):
    """Queues iters * 32 independent instructions of `kind` (a key of MICROBENCH_KINDS) per thread on every SM."""
    _check(lib().bitnet_microbench_issue(MICROBENCH_KINDS[kind], int(iters), _ptr(sink), _stream(stream)),
           "bitnet_microbench_issue")


NOALLOC_MAX_M = 32768
NOALLOC_MAX_K = 32768


def bitnet_mpgemv_tl_noalloc(fmt, packed, w_scale, M, K, q, act_scale, y, acc_out=None, bk3=0, stream=None):
    """TL1/TL2 mpGEMV (T <= 8) for callers that cannot allocate: no workspace argument, and this wrapper
    creates no tensor either -- y (and acc_out, if wanted) must be supplied.  The scratch is a fixed
    array inside the library, shared by every call on the device; see the header for the limits."""
    T = q.shape[0]
    _check(lib().bitnet_mpgemv_tl_noalloc(_fmt(fmt), _ptr(packed), float(w_scale), M, K, bk3, _ptr(q),
                                          _ptr(act_scale), T, _ptr(y), _ptr(acc_out), _stream(stream)),
           "bitnet_mpgemv_tl_noalloc")
    return y, acc_out


# ---- paged key-value cache and the attention over it
KV_DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class KvCacheDesc(C.Structure):
    """Mirror of bitnet_kv_cache_t."""
    _fields_ = [("dtype", C.c_int32), ("kv_heads", C.c_int32), ("page_size", C.c_int32), ("head_dim", C.c_int32),
                ("layers", C.c_int64), ("num_pages", C.c_int64), ("k", C.c_void_p), ("v", C.c_void_p),
                ("stride_layer", C.c_int64), ("stride_page", C.c_int64), ("stride_head", C.c_int64), ("stride_row", C.c_int64),
                ("ready", C.c_uint64), ("maps", C.c_uint64 * 64), ("layer_pages", C.c_int64), ("device", C.c_int32), ("reserved", C.c_int32)]


class KvCache:
    """Handle of a cache whose pools are the CUDA tensors k and v [layers][pages][kv_heads][page_size][head_dim] (bf16 or
    fp16, equal strides, head_dim contiguous; views in another order of the outer dimensions are fine).  Keeps the tensors alive."""

    def __init__(self, k, v):
        # (the stride of a dimension of one entry says nothing)
        stride, other = ([t.stride(i) if t.shape[i] > 1 else 0 for i in range(t.dim())] for t in (k, v))
        if k.dim() != 5 or k.shape != v.shape or stride != other or k.dtype != v.dtype:
            raise BitnetError("KvCache: k and v must be [layers][pages][kv_heads][page_size][head_dim] of one type with equal strides")
        if not (k.is_cuda and v.is_cuda and k.device == v.device) or k.dtype not in (torch.bfloat16, torch.float16):
            raise BitnetError("KvCache: expected CUDA tensors of bfloat16 or float16")
        if k.stride(4) != 1 and k.shape[4] > 1:
            raise BitnetError("KvCache: head_dim must be contiguous")
        self.k, self.v = k, v
        self.layers, self.num_pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.dtype, self.device = k.dtype, k.device
        self.desc = KvCacheDesc(dtype=KV_DTYPE[k.dtype], kv_heads=self.kv_heads, page_size=self.page_size, head_dim=self.head_dim,
                                layers=self.layers, num_pages=self.num_pages, k=k.data_ptr(), v=v.data_ptr(),
                                stride_layer=stride[0], stride_page=stride[1], stride_head=stride[2], stride_row=stride[3])
        _check(lib().bitnet_kv_cache_init(C.byref(self.desc)), "bitnet_kv_cache_init")
        self.ref = C.addressof(self.desc)
        self.scale = self.head_dim ** -0.5


def new_kv_cache(layers, num_pages, kv_heads, page_size, head_dim, dtype=torch.bfloat16, device="cuda"):
    """A cache with zeroed pools (rows padded to a multiple of 8 elements)."""
    shape = (layers, num_pages, kv_heads, page_size, -(-head_dim // 8) * 8)
    k, v = (torch.zeros(shape, dtype=dtype, device=device)[..., :head_dim] for _ in range(2))
    return KvCache(k, v)


_fast = None


def _binding():
    """The compiled part of the binding (csrc/binding.cpp), tied to the loaded library.  Raises if it has not been built."""
    global _fast
    if _fast is None:
        import importlib.machinery
        import importlib.util
        path = os.path.join(_PKG, "_binding.so")
        if not os.path.exists(path):
            raise BitnetError(f"{path} is missing: run `python -m paper_2502_11880_b200.build` (there is no fallback path)")
        loader = importlib.machinery.ExtensionFileLoader(__name__ + "._binding", path)
        m = importlib.util.module_from_spec(importlib.util.spec_from_file_location(__name__ + "._binding", path, loader=loader))
        loader.exec_module(m)
        L = lib()
        m.bind(BitnetError, _check, tuple(C.cast(f, C.c_void_p).value for f in (
            L.bitnet_kv_append, L.bitnet_kv_reserve, L.bitnet_kv_fork, L.bitnet_kv_free, L.bitnet_kv_trim, L.bitnet_kv_compact,
            L.bitnet_kv_copy_pages, L.bitnet_attn_decode, L.bitnet_attn_prompt, L.bitnet_attn_shared, L.bitnet_kv_append_rope,
            L.bitnet_add_rmsnorm_quant, L.bitnet_sample)))
        _fast = m
    return _fast


def _st(stream):
    """None: the current stream of the tensors' device."""
    return None if stream is None else stream.cuda_stream


_here = contextlib.nullcontext()


def _on(stream):
    """Calls that make tensors (results, workspaces) make them on the stream that they run on."""
    return _here if stream is None else torch.cuda.stream(stream)


def bitnet_kv_append(cache, layer, k, v, table, kv_len, q_start=None, dev_status=None, stream=None):
    """Writes new tokens' rows k, v [tokens][kv_heads][head_dim] into their pages; kv_len [seqs] counts them already."""
    (_fast or _binding()).kv_append(cache.ref, layer, k, v, table, kv_len, q_start, dev_status, _st(stream))


def bitnet_kv_reserve(refs, table, from_len, to_len, page_size, dev_status=None, stream=None):
    """Gives the rows of the table the pages that growing from from_len to to_len tokens takes, lowest free pages first."""
    (_fast or _binding()).kv_reserve(refs, table, from_len, to_len, page_size, dev_status, _st(stream))


def bitnet_kv_workspace_bytes(num_pages, n) -> int:
    return lib().bitnet_kv_workspace_bytes(num_pages, n)


def new_kv_workspace(num_pages, n=0, device="cuda"):
    """Workspace of bitnet_kv_fork (up to n children) and bitnet_kv_compact."""
    size = bitnet_kv_workspace_bytes(num_pages, n)
    if size == 0:
        _check(1, "bitnet_kv_workspace_bytes")
    return torch.empty(size, dtype=torch.uint8, device=device)


def bitnet_kv_fork(cache, refs, table, kv_len, parents, children, workspace=None, dev_status=None, stream=None):
    """Rows children[i] become copies of rows parents[i]: full pages shared, a page filled in part copied."""
    with _on(stream):
        if workspace is None:
            workspace = new_kv_workspace(cache.num_pages, parents.shape[0], cache.device)
        (_fast or _binding()).kv_fork(cache.ref, refs, table, kv_len, parents, children, workspace, dev_status, None)


def bitnet_kv_free(refs, table, kv_len, rows, dev_status=None, stream=None):
    """Gives up the listed rows of the table: counts fall, the rows become -1, their lengths 0."""
    (_fast or _binding()).kv_free(refs, table, kv_len, rows, dev_status, _st(stream))


def bitnet_kv_trim(refs, table, kv_len, page_size, window, sinks=0, stream=None):
    """Gives up the pages that attention with this window and these sinks no longer reads."""
    (_fast or _binding()).kv_trim(refs, table, kv_len, page_size, window, sinks, _st(stream))


def bitnet_kv_compact(cache, refs, table, live=None, workspace=None, stream=None):
    """Moves the pages in use to the pool's first places; live (int32 [1], optional) receives their number."""
    with _on(stream):
        if workspace is None:
            workspace = new_kv_workspace(cache.num_pages, 0, cache.device)
        (_fast or _binding()).kv_compact(cache.ref, refs, table, live, workspace, None)


def bitnet_kv_copy_pages(cache, src, dst, dev_status=None, stream=None):
    """Copies pages src[i] to dst[i], K and V, all layers."""
    (_fast or _binding()).kv_copy_pages(cache.ref, src, dst, dev_status, _st(stream))


ATTN_WORKSPACE_HEAD = 65536      # the bytes of a workspace that have to be zero before its first call


def bitnet_attn_workspace_bytes(tokens, q_heads, kv_heads, head_dim) -> int:
    return lib().bitnet_attn_workspace_bytes(tokens, q_heads, kv_heads, head_dim)


def new_attn_workspace(tokens, q_heads, kv_heads, head_dim, device="cuda"):
    """A workspace for bitnet_attn_decode and bitnet_attn_prompt calls, its counters zeroed.  tokens: the most new tokens of a prompt
    call (0: decode calls only, 1.3 MB; otherwise 21 MB, for the parts of prompt calls with few rows)."""
    size = bitnet_attn_workspace_bytes(tokens, q_heads, kv_heads, head_dim)
    if size == 0:
        _check(1, "bitnet_attn_workspace_bytes")
    ws = torch.empty(size, dtype=torch.uint8, device=device)
    bitnet_workspace_init(ws[:ATTN_WORKSPACE_HEAD])
    return ws


def _attn_ws(cache, q, prompt):
    """A workspace for one call; None where the call will refuse q anyway, or has nothing to do."""
    if q.dim() != 3 or q.shape[0] == 0 or q.shape[1] == 0 or q.shape[1] % cache.kv_heads:
        return None
    return new_attn_workspace(prompt * q.shape[0], q.shape[1], cache.kv_heads, cache.head_dim, cache.device)


def bitnet_attn_decode(cache, layer, q, table, kv_len, scale=None, window=0, sinks=0, out=None, workspace=None, dev_status=None,
                       stream=None):
    """Attention of one new token per sequence: q [seqs][q_heads][head_dim] (fp32 or the cache's type) -> out, same shape and type."""
    with _on(stream):
        return (_fast or _binding()).attn_decode(cache.ref, layer, q, table, kv_len, cache.scale if scale is None else scale, window, sinks,
                                                 out, _attn_ws(cache, q, 0) if workspace is None else workspace, dev_status, None)


def bitnet_attn_prompt(cache, layer, q, table, kv_len, q_start, max_new, scale=None, window=0, sinks=0, out=None, workspace=None,
                       dev_status=None, stream=None):
    """Attention of prompts or chunks of prompts: q [tokens][q_heads][head_dim] in the cache's type; sequence s has the tokens
    q_start[s] .. q_start[s + 1] - 1 (at most max_new), the last of them at position kv_len[s] - 1."""
    with _on(stream):
        return (_fast or _binding()).attn_prompt(cache.ref, layer, q, table, kv_len, q_start, max_new, cache.scale if scale is None else scale,
                                                 window, sinks, out, _attn_ws(cache, q, 1) if workspace is None else workspace, dev_status,
                                                 None)


def bitnet_attn_shared_workspace_bytes(seqs, q_heads, kv_heads, head_dim) -> int:
    return lib().bitnet_attn_shared_workspace_bytes(seqs, q_heads, kv_heads, head_dim)


def new_attn_shared_workspace(seqs, q_heads, kv_heads, head_dim, device="cuda"):
    """A workspace for bitnet_attn_shared calls of up to so many sequences, its counters zeroed."""
    size = bitnet_attn_shared_workspace_bytes(seqs, q_heads, kv_heads, head_dim)
    if size == 0:
        _check(1, "bitnet_attn_shared_workspace_bytes")
    ws = torch.empty(size, dtype=torch.uint8, device=device)
    bitnet_workspace_init(ws[:ATTN_WORKSPACE_HEAD])
    return ws


def bitnet_attn_shared(cache, layer, q, table, kv_len, group_start, prefix_len, scale=None, window=0, sinks=0, out=None, workspace=None,
                       dev_status=None, stream=None):
    """bitnet_attn_decode for groups of sequences (group_start [groups + 1]) whose first prefix_len [groups] tokens are the same: read once
    per group.  q [seqs][q_heads][head_dim] in the cache's type -> out, same shape and type."""
    with _on(stream):
        if workspace is None and q.dim() == 3 and q.shape[0] and q.shape[1] and q.shape[1] % cache.kv_heads == 0:
            workspace = new_attn_shared_workspace(q.shape[0], q.shape[1], cache.kv_heads, cache.head_dim, cache.device)
        return (_fast or _binding()).attn_shared(cache.ref, layer, q, table, kv_len, group_start, prefix_len, cache.scale if scale is None else scale,
                                                 window, sinks, out, workspace, dev_status, None)


# ---- rotary positions, norm, drawing of tokens
ROPE_SCALING = {"none": 0, "linear": 1, "bands": 2}


class RopeDesc(C.Structure):
    """Mirror of bitnet_rope_t."""
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scaling", C.c_int32), ("reserved", C.c_int32), ("base", C.c_double),
                ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double), ("context", C.c_double), ("magnitude", C.c_double),
                ("freqs", C.POINTER(C.c_double)), ("ready", C.c_uint64), ("step", C.c_uint64 * 64)]


class Rope:
    """Rotation of the first `rot` elements of a head: pairs (i, i + rot/2) (layout "half") or (2i, 2i + 1) ("interleaved") turn by position *
    base^(-2i/rot).  scaling "linear" divides the frequencies by factor, "bands" those of pairs that make fewer than `high` turns within `context`
    positions (all of it below `low`).  freqs: rot/2 frequencies in radians per position, in place of all that; magnitude multiplies sines and cosines."""

    def __init__(self, rot, base=10000.0, layout="half", scaling="none", factor=1.0, low=1.0, high=4.0, context=8192, freqs=None, magnitude=1.0):
        if layout not in ("half", "interleaved") or scaling not in ROPE_SCALING:
            raise BitnetError("Rope: layout is 'half' or 'interleaved', scaling 'none', 'linear' or 'bands'")
        given = None
        if freqs is not None:
            freqs = [float(f) for f in freqs]
            if len(freqs) != rot // 2:
                raise BitnetError("Rope: freqs must be rot / 2 values")
            given = (C.c_double * len(freqs))(*freqs)
        self.rot, self.layout = rot, layout
        self.desc = RopeDesc(rot_dim=rot, interleaved=int(layout == "interleaved"), scaling=ROPE_SCALING[scaling], base=base, factor=factor, low=low,
                             high=high, context=context, magnitude=magnitude, freqs=given)
        _check(lib().bitnet_rope_init(C.byref(self.desc)), "bitnet_rope_init")
        self.desc.freqs = None                # (read by bitnet_rope_init only)
        self.ref = C.addressof(self.desc)


def bitnet_kv_append_rope(cache, layer, rope, q, k, v, table, kv_len, q_start=None, q_out=None, q_dtype=None, dev_status=None, stream=None):
    """bitnet_kv_append with the rows of q [tokens][q_heads][head_dim] and k rotated by their tokens' positions; returns q's (q_out, or a new tensor of
    q_dtype, by default q's type).  q = None: keys and values only."""
    with _on(stream):
        return (_fast or _binding()).kv_append_rope(cache.ref, layer, rope.ref, q, k, v, table, kv_len, q_start, q_out,
                                                    -1 if q_dtype is None else KV_DTYPE.get(q_dtype, -1), dev_status, None)


def bitnet_add_rmsnorm_quant(x, weight=None, eps=1e-5, residual=None, residual_out=None, y=None, q=None, act_scale=None, act_sum=None, stream=None):
    """h = residual + x (written to residual_out; by default residual itself is updated), y = h / rms(h) * weight (written to y, if that is given), and the int8
    codes that bitnet_quant_act gives for y: returns (q, act_scale)."""
    with _on(stream):
        return (_fast or _binding()).add_rmsnorm_quant(x, weight, eps, residual, residual if residual_out is None else residual_out, y, q, act_scale,
                                                       act_sum, None)


def bitnet_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, prob=None, stream=None):
    """One token per row of logits [rows][vocab] from the random numbers u [rows]; the settings are CUDA vectors of one value per row, or None.
    Returns (tokens int32, prob fp32: the tokens' shares of what was kept)."""
    with _on(stream):
        return (_fast or _binding()).sample(logits, u, temperature, top_k, top_p, min_p, tokens, prob, None)
