"""Rotating q in place: only where each row stays where it is (no GPU needed: the call is refused before a launch)."""
import ctypes

import paper_2512_14481_b200 as P

INVALID = 1


def test_in_place_with_another_stride_is_refused():
    buf = (ctypes.c_char * 512)()
    a = (ctypes.addressof(buf) + 63) & ~63             # never dereferenced
    cache = P.KVCacheStruct(a, a, None, None, 16 * 4 * 64, 4 * 64, 64, 8, 16, 4, 64, P.SASQ_KV_16BIT)
    for q_stride, out_stride in ((1024, 512), (512, 1024)):
        batch = P.KVBatchStruct(a, a, a, 8, 2, 8, 4, 2, 100, 0)
        assert P.load_library().sasq_rope_kv_append(ctypes.byref(cache), ctypes.byref(batch), a, a, a, a, q_stride, 256, 256, out_stride,
                                                    8, a, 100, 64, 0, P.SASQ_BF16, None) == INVALID
