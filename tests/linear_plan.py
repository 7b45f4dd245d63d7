"""The library's own choice of kernel and split for a product (csrc/qlin.hip), asked on the host."""
import ctypes

from paper_2007_06919_amd import aqd

# kernels by their number in csrc/internal.h
ANY, T64x32, T64x64, T128x64, T128x128, T256x128, T256x256, T128x128_ANY, T256x256_ANY, FEW16, FEW64, T128x128_TWO = range(12)
NAMES = ("ANY 64x32 64x64 128x64 128x128 256x128 256x256 128x128_ANY 256x256_ANY FEW16 FEW64 128x128_TWO").split()


class Args(ctypes.Structure):   # QlinArgs
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "w", "x_scales", "w_scales", "bias", "y")] + \
               [(n, ctypes.c_longlong) for n in ("ld_x", "ld_w", "ld_y")] + \
               [(n, ctypes.c_int) for n in ("rows", "n", "k", "wide", "type", "gate", "ksplit", "kchunk")] + \
               [("part", ctypes.c_void_p)] + [(n, ctypes.c_int) for n in ("n_pad", "whole_lines")]


class Plan(ctypes.Structure):   # QlinPlan
    _fields_ = [("shape", ctypes.c_int), ("parts", ctypes.c_int), ("bytes", ctypes.c_size_t)]


def args(rows, n, k, type, act, ld_x=0, ld_w=0, ld_y=0, x=0, w=0):
    return Args(x=x, w=w, ld_x=ld_x or k, ld_w=ld_w or k, ld_y=ld_y or n, rows=rows, n=n, k=k,
                wide=2 * n if act else n, type=type, gate=act)


def plan(a, room=aqd.QLIN_WORKSPACE_BYTES):
    """(kernel, parts, workspace bytes) of a call with `room` bytes of workspace."""
    f = aqd.lib()._ZN3aqd9qlin_planERKNS_8QlinArgsEm
    f.restype, f.argtypes = Plan, [ctypes.POINTER(Args), ctypes.c_size_t]
    p = f(ctypes.byref(a), room)
    return p.shape, p.parts, p.bytes


def launch(a, p):
    """The status of a launch by a plan on the null stream."""
    f = aqd.lib()._ZN3aqd11launch_qlinERKNS_8QlinArgsERKNS_8QlinPlanEP12ihipStream_t
    f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(Args), ctypes.POINTER(Plan), ctypes.c_void_p]
    return f(ctypes.byref(a), ctypes.byref(Plan(*p)), None)
