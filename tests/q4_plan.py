"""Which attention kernel over the 4-bit cache the library takes for a call: asked of the library, on the CPU."""
import ctypes

import paper_2412_11741_amd as csr


class _Args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "codesK", "paramsK", "codesV", "paramsV", "seq_lens", "q_lens", "out")] + \
               [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "G", "Tq")] + [("T", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("d", "group_k", "group_v", "q_dtype", "out_dtype")] + \
               [("scale", ctypes.c_float), ("causal", ctypes.c_bool), ("q_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
                ("workspace", ctypes.c_void_p), ("stream", ctypes.c_void_p)]


class _Plan(ctypes.Structure):
    _fields_ = [("row_tiles", ctypes.c_int32), ("row_blocks", ctypes.c_int32), ("splits", ctypes.c_int32), ("alone", ctypes.c_bool),
                ("off_ml", ctypes.c_size_t), ("total_bytes", ctypes.c_size_t)]


def plan(B, Hq, Hkv, T, Tq, d, dtype=1):
    """(16s of rows a workgroup, workgroups along the rows, parts of the token axis, eight waves), and the workspace's bytes; dtype: csr_dtype"""
    a = _Args(B=B, Hq=Hq, Hkv=Hkv, G=Hq // Hkv, Tq=Tq, T=T, d=d, group_k=64, group_v=64, q_dtype=dtype, out_dtype=dtype, causal=True)
    p = _Plan()
    call = getattr(csr.lib(), "_ZN3csr12plan_q4_attnERKNS_10Q4AttnArgsEPNS_10Q4AttnPlanE")
    call.restype = None
    call(ctypes.byref(a), ctypes.byref(p))
    return (p.row_tiles, p.row_blocks, p.splits, p.alone), p.total_bytes
