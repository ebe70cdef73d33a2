"""The forms of the 8-bit projections' kernels, and sizes that take each (test
infrastructure only).

A form is what a launch instantiates: ("one", weight tiles, token tiles, several
token blocks) of k_linear, or ("ring", weight tiles of a wave, token tiles, with K
ranges) of k_linear_ring, as the library's own rule has it.
"""
import ctypes as C

from paper_2506_01979_amd import api


class _Plan(C.Structure):
    _fields_ = [("nt", C.c_int32), ("tblocks", C.c_int32), ("ring_tiles", C.c_int32), ("splits", C.c_int32)]


_rule = getattr(api.lib, "_ZN2sb11linear_planEiii")  # sb::linear_plan(tiles, ks, n_tok)
_rule.restype, _rule.argtypes = _Plan, [C.c_int32] * 3


def form(m, k, n):
    p = _rule(-(-m // 16), -(-(-(-k // 64)) // 4) * 4, n)
    tiles = -(-n // 16)
    if p.ring_tiles:
        return "ring", p.ring_tiles, next(t for t in (2, 3, 5, 7, 9, 12, 16) if tiles <= t), p.splits > 1
    return "one", p.nt, -(-tiles // p.tblocks), p.tblocks > 1


# outputs, inputs, rows: the widths of the 7B, 13B and 70B models that take forms of their
# own, then sizes of none, odd ones among them; together every form that the rule takes
CASES = [
    (15360, 5120, (1, 17, 33, 49, 65, 81, 97, 113, 180)),   # 13B QKV
    (8192, 28672, (17, 33, 65, 81, 129, 177, 256)),         # 70B down
    (5120, 5120, (81, 113)),                                # 13B O
    (12288, 4096, (113, 161)),                              # 7B QKV
    (245, 3847, (9, 25, 41, 57, 73, 89, 105, 121, 145, 177, 209, 233, 249)),
    (6144, 256, (9, 25, 41, 57, 73, 89, 105, 121, 145, 177, 209, 241)),
    (8445, 431, (9, 25, 41, 57, 73, 89, 105, 121, 137, 169, 225)),
    (12544, 789, (9, 25, 41, 57, 73, 89, 105, 121, 145, 177, 209, 241)),
    (2197, 372, (105, 121, 145, 177, 209, 241)),
    (34815, 338, (9, 25, 41, 65, 97, 129, 169, 225)),
    (18671, 351, (25, 41, 57, 73, 97)),
    (1, 15067, (25, 41, 65, 169)),
    (20767, 397, (9, 25, 41)),
    (25688, 347, (9, 25, 41)),
    (18828, 4570, (73, 97, 129, 169, 225)),
]
