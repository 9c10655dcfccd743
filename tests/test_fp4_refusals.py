"""Calls that have no meaning for the 4-bit cache are refused (without a GPU a launch would come back as status 5)."""
import ctypes as C

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build


def test_quantisers_of_queries_and_values():
    """Its queries stay binary16 and its values have 4 bits: INT8 numbers of either are nothing that a call of it uses."""
    sa_build.build()
    lib, null, at = sa.lib(), C.c_void_p(0), C.c_void_p(256)
    for d in (64, 128):
        for rotated in (False, True):
            cfg = sa.make_config(d, 8, 2, sa.SA_KV_FP4, hadamard=rotated)
            # (no vectors: nothing is launched where the configuration is taken)
            assert lib.sa_quantise_query(C.byref(cfg), at, C.c_int(0), at, at, null) == 2
            assert lib.sa_quantise_values(C.byref(cfg), at, C.c_int64(0), at, at, null) == 2
            other = sa.make_config(d, 8, 2, sa.SA_INT8, hadamard=rotated)
            assert lib.sa_quantise_query(C.byref(other), at, C.c_int(0), at, at, null) == 0
            assert lib.sa_quantise_values(C.byref(other), at, C.c_int64(0), at, at, null) == 0
