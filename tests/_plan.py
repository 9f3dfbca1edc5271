"""The tiles that phase2_quant takes for a call's sizes, as the library plans them."""
import ctypes

from paper_2607_20457_amd import _lib


class Plan(ctypes.Structure):
    """QuantPlan of csrc/common.hpp."""
    _fields_ = [(x, ctypes.c_int) for x in ("columns", "keys", "tokens", "parts")]

    @property
    def waves(self):
        """Of a workgroup."""
        return 8 if self.keys == 32 else 4


def plan(n, Tq, S, Hq, Hkv, d, gen_rows=0):
    fn = _lib.lib()._Z10quant_planiiliiil
    fn.restype = Plan
    fn.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int64] + [ctypes.c_int] * 3 + [ctypes.c_int64]
    return fn(n, Tq, S, Hq, Hkv, d, gen_rows)


# Sizes Hq, Hkv, d, Tq, n, S that take each kernel with room for what a test adds, and that
# kernel's columns and rows of a step.
SHAPES = {
    "16x32_d128": ((8, 2, 128, 3, 2, 300), (16, 32)),
    "16x32_d64": ((4, 1, 64, 5, 2, 300), (16, 32)),
    "48x32_d128": ((64, 8, 128, 6, 3, 12500), (48, 32)),
    "32x32_d128": ((16, 16, 128, 64, 1, 14000), (32, 32)),
    "32x64_d128": ((16, 16, 128, 256, 1, 17600), (32, 64)),
    "32x32_d64": ((64, 64, 64, 128, 1, 8700), (32, 32)),
}
