"""The forms of the attention over the 8-bit cache, and sizes that take each (test
infrastructure only): row tiles of a wave, and key ranges, as the library's own rule
has them."""
import ctypes as C

from paper_2506_01979_amd import api


class _Plan(C.Structure):
    _fields_ = [("rt", C.c_int32), ("n_rb", C.c_int32), ("chunks", C.c_int32)]


# sb::quant_attn_plan(n_kv, head_dim, n_blocks, tail_keys, rows)
_rule = getattr(api.lib, "_ZN2sb15quant_attn_planEiiiii")
_rule.restype, _rule.argtypes = _Plan, [C.c_int32] * 5


def plan(nh, nkv, d, nb, tail, n):
    """Row tiles of a wave, row blocks, key ranges."""
    p = _rule(nkv, d, nb, tail + n, n * (nh // nkv))
    return p.rt, p.n_rb, p.chunks


# query heads, KV heads, head_dim, blocks, tail, rows
THREE_TILES = [(2, 2, 64, 130, 5, 129), (4, 2, 64, 130, 37, 88), (16, 2, 64, 127, 63, 33), (2, 2, 128, 130, 5, 129),
               (4, 2, 128, 130, 40, 88), (64, 8, 128, 127, 63, 33), (12, 2, 128, 140, 0, 12)]
# more than 64 blocks a wave, whose scales it then loads again
MANY_BLOCKS = [(300, 300, 64, 300, 7, 1), (260, 260, 128, 270, 3, 1), (48, 6, 64, 300, 20, 256), (86, 86, 64, 270, 9, 129),
               (86, 86, 128, 530, 0, 129)]
