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


# Sizes that reach every kernel, of those that the plan ever takes, in all types of y: (kernel, act, split, y of whole lines
# past the L2, rows, n, k, row stride of both operands). Short and longer k where k is not split; odd rows, and n and k of no
# multiple, but for whole lines of y.
COVER = [
    (ANY, 0, False, False, 21, 21, 2, 4), (ANY, 0, False, False, 21, 4523, 540, 541),
    (ANY, 0, False, False, 27, 21, 1, 1), (ANY, 0, True, False, 21, 387, 15807, 15807),
    (ANY, 1, False, False, 21, 4302, 449, 449), (ANY, 1, False, False, 23, 26, 1, 1),
    (ANY, 1, False, False, 25, 22, 11, 12), (ANY, 1, True, False, 23, 25, 3803, 3803),
    (FEW16, 0, False, False, 21, 21, 464, 465), (FEW16, 0, False, False, 21, 21, 657, 660),
    (FEW16, 0, False, False, 21, 21, 682, 684), (FEW16, 0, False, False, 23, 21, 18, 19),
    (FEW16, 1, False, False, 21, 21, 20, 21), (FEW16, 1, False, False, 21, 21, 417, 420),
    (FEW16, 1, False, False, 21, 22, 416, 417), (FEW16, 1, False, False, 23, 22, 17, 20),
    (FEW64, 0, False, False, 33, 1362, 16, 17), (FEW64, 0, False, False, 1411, 34, 415, 415),
    (FEW64, 1, False, False, 33, 1445, 453, 453), (FEW64, 1, False, False, 2053, 21, 26, 27),
    (T64x32, 0, False, False, 21, 22, 16, 16), (T64x32, 0, False, False, 23, 23, 406, 408),
    (T64x32, 0, True, False, 23, 26, 11180, 11180), (T64x32, 1, False, False, 21, 2058, 1095, 1096),
    (T64x32, 1, False, False, 1077, 51, 1170, 1172), (T64x32, 1, True, False, 21, 21, 9964, 9964),
    (T64x64, 0, False, False, 8275, 21, 21, 24), (T64x64, 0, False, False, 8927, 21, 415, 416),
    (T64x64, 0, True, False, 887, 67, 3733, 3736), (T128x64, 0, False, False, 8449, 65, 412, 412),
    (T128x64, 0, False, False, 8503, 65, 152, 152), (T128x64, 0, True, False, 3065, 67, 6123, 6124),
    (T128x64, 1, False, False, 21, 2062, 18, 20), (T128x64, 1, False, False, 33, 1410, 445, 448),
    (T128x64, 1, True, False, 23, 26, 7213, 7216), (T128x128, 0, False, False, 67, 16671, 457, 460),
    (T128x128, 0, False, False, 77, 17027, 279, 280), (T128x128, 0, True, False, 81, 3278, 10454, 10456),
    (T128x128, 1, False, False, 16773, 23, 404, 404), (T128x128, 1, False, False, 17525, 21, 147, 148),
    (T128x128, 1, True, False, 3451, 22, 7146, 7148), (T128x128_TWO, 0, False, False, 199, 16435, 19, 20),
    (T128x128_TWO, 0, False, False, 16975, 263, 430, 432), (T128x128_TWO, 0, True, False, 18251, 75, 19147, 19148),
    (T128x128_TWO, 1, False, False, 16717, 137, 419, 420), (T128x128_TWO, 1, False, False, 17577, 139, 18, 20),
    (T128x128_TWO, 1, True, False, 12487, 1, 12738, 12740), (T256x128, 0, False, False, 16405, 209, 161, 164),
    (T256x128, 0, False, False, 16711, 130, 543, 544), (T256x128, 0, False, True, 259, 14784, 408, 408),
    (T256x128, 0, False, True, 1029, 3968, 152, 152), (T256x128, 0, True, False, 6061, 133, 8660, 8660),
    (T256x128, 1, False, False, 65, 16502, 38, 40), (T256x128, 1, False, False, 67, 18557, 401, 404),
    (T256x128, 1, False, True, 259, 7744, 19, 20), (T256x128, 1, False, True, 2537, 832, 414, 416),
    (T256x128, 1, True, False, 5653, 66, 9000, 9000), (T256x256, 0, False, False, 1237, 6617, 515, 516),
    (T256x256, 0, False, False, 8241, 1418, 129, 132), (T256x256, 0, False, True, 3265, 2496, 557, 560),
    (T256x256, 0, False, True, 7377, 1728, 130, 132), (T256x256, 0, True, False, 16561, 129, 11251, 11252),
    (T256x256, 1, False, False, 193, 17066, 406, 408), (T256x256, 1, False, False, 17627, 193, 22, 24),
    (T256x256, 1, False, True, 275, 13312, 22, 24), (T256x256, 1, False, True, 327, 11008, 430, 432),
    (T256x256, 1, True, False, 11631, 70, 17218, 17220), (T128x128_ANY, 0, False, False, 21, 17461, 848, 849),
    (T128x128_ANY, 0, False, False, 23, 16806, 684, 685), (T128x128_ANY, 0, True, False, 25, 23, 14222, 14223),
    (T128x128_ANY, 1, False, False, 21, 8259, 660, 661), (T128x128_ANY, 1, False, False, 23, 8390, 674, 675),
    (T128x128_ANY, 1, True, False, 21, 22, 9518, 9519), (T256x256_ANY, 0, False, False, 16963, 134, 1714, 1715),
    (T256x256_ANY, 0, False, False, 18911, 385, 29, 29), (T256x256_ANY, 0, False, True, 133, 16768, 2116, 2117),
    (T256x256_ANY, 0, False, True, 531, 15168, 20, 21), (T256x256_ANY, 0, True, False, 17079, 134, 1904, 1905),
    (T256x256_ANY, 1, False, False, 147, 16575, 466, 467), (T256x256_ANY, 1, False, False, 197, 17554, 26, 27),
    (T256x256_ANY, 1, False, True, 137, 17600, 425, 425), (T256x256_ANY, 1, False, True, 329, 11456, 26, 27),
    (T256x256_ANY, 1, True, False, 17129, 65, 1684, 1685),
]


def stored_past(kernel, parts, rows, n, type):
    """Whether a packed y is stored in whole lines past the L2, which tiles of 256 x 128 and more can."""
    size = 4 if type == aqd.F32 else 2
    return parts == 1 and kernel in (T256x128, T256x256, T256x256_ANY) and n * size % 128 == 0 and rows * n * size >= 4e6
