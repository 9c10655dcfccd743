"""Host-side validation of the 4-bit cache, sa_read_kv and sa_rotate_qkv: what is refused, and that it is before anything is launched
(without a GPU a launch would come back as status 5)."""
import ctypes as C

import numpy as np
import pytest

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


NULL, ONE = C.c_void_p(0), C.c_void_p(256)      # ONE: a non-null, aligned address that nothing may follow


def _status(fn, *args):
    try:
        fn(*args)
    except sa.SaError as e:
        return e.status
    return 0


@pytest.mark.parametrize("d,want", [(64, 72), (128, 144)])
def test_layout_of_the_4_bit_cache(d, want):
    lay = sa.get_layout(sa.make_config(d, 32, 4, sa.SA_KV_FP4, hadamard=True))
    assert (lay.page_bytes, lay.kcode_off, lay.meta_off, lay.v_off, lay.align) == (64 * want, 0, 16 * d, 18 * d, 256)
    assert lay.page_bytes % 256 == 0 and lay.page_bytes // 2 % 16 == 0


def test_configurations_of_the_4_bit_cache():
    for bad in (dict(nibble=True), dict(headroom_F=7), dict(shift_add=True), dict(add_on_alu=True), dict(shift_by_multiply=True)):
        assert _status(sa.get_layout, sa.make_config(64, 32, 4, sa.SA_KV_FP4, **bad)) == 2, bad
    assert _status(sa.get_layout, sa.make_config(96, 32, 4, sa.SA_KV_FP4)) == 2
    cfg = sa.make_config(64, 32, 4, sa.SA_KV_FP4)
    cache, lib = sa.SaCache(256, 256, 256, 2, 4, 8), sa.lib()
    big = C.c_size_t(1 << 30)
    assert lib.sa_encode_keys(C.byref(cfg), ONE, C.c_int64(4), ONE, ONE, NULL) == 2
    assert lib.sa_debug_unpack(C.byref(cfg), C.byref(cache), C.c_int(0), C.c_int(1), NULL, NULL, NULL, NULL, NULL) == 2
    assert _status(sa.shiftav_workspace_bytes, cfg, 2, 64) == 2
    assert lib.sa_decode_attention_shiftav(C.byref(cfg), C.byref(cache), ONE, ONE, ONE, big, C.c_int(15), C.c_int(15), NULL, NULL, NULL) == 2
    assert lib.sa_decode_attention_fp16(C.byref(cfg), C.byref(cache), ONE, ONE, ONE, big, NULL) == 2
    assert lib.sa_debug_decode_lost_copy(C.byref(cfg), C.byref(cache), ONE, ONE, ONE, big, C.c_int(0), C.c_int(0), C.c_int(0), NULL) == 2
    assert lib.sa_decode_attention(C.byref(cfg), C.byref(cache), ONE, ONE, ONE, big, ONE, NULL) == 2          # no integer scores
    assert lib.sa_decode_attention(C.byref(cfg), C.byref(cache), ONE, ONE, ONE, C.c_size_t(8), NULL, NULL) == 4
    for pages in (1, 64, 513, 1 << 16, 1 << 20):
        assert sa.workspace_bytes(cfg, 1, pages) <= sa.STATIC_SCRATCH_BYTES


def test_read_refuses():
    lib, i64 = sa.lib(), lambda *v: (C.c_int64 * len(v))(*v)
    cfg = sa.make_config(64, 32, 4, sa.SA_KV_FP4)
    good = sa.SaCache(256, 256, 256, 2, 4, 8)
    call = lambda cu, starts=None, cache=good, K=ONE, V=ONE, cfg=cfg: lib.sa_read_kv(C.byref(cfg), C.byref(cache), starts, cu, K, V, NULL)
    assert call(None) == 1 and call(i64(0, 1, 2), K=NULL, V=NULL) == 1
    assert call(i64(0, 1, 2), cache=sa.SaCache(0, 256, 256, 2, 4, 8)) == 1 and call(i64(0, 1, 2), cache=sa.SaCache(264, 256, 256, 2, 4, 8)) == 3
    assert call(i64(0, 1, 2), K=C.c_void_p(264)) == 3 and call(i64(0, 1, 2), V=C.c_void_p(264), K=NULL) == 3
    assert call(i64(0, 2, 1)) == 1 and call(i64(-1, 2, 3)) == 1 and call(i64(0, 1, 2), i64(0, -1)) == 1
    assert call(i64(0, 257, 258)) == 4 and call(i64(0, 1, 2), i64(0, 256)) == 4 and call(i64(0, 0, 0), i64(257, 0)) == 4
    assert call(i64(0, 1, 2), i64(0, (1 << 63) - 1)) == 4
    assert call(i64(5, 5, 5)) == 0                              # nothing to do
    wide = sa.SaCache(256, 256, 256, 2, 1 << 26, 8)             # lengths beyond 32 bits
    assert call(i64(0, 1 << 31, 1 << 31), cache=wide) == 4
    many = sa.make_config(64, 256, 256, sa.SA_KV_FP4)           # more warps than a grid holds
    assert call(i64(0, (1 << 31) - 1, (1 << 31) - 1), cache=wide, cfg=many) == 4
    assert call(i64(0, 1, 2), cfg=sa.make_config(96, 32, 4, sa.SA_KV_FP4)) == 2


def test_rotate_refuses():
    lib, cfg = sa.lib(), sa.make_config(64, 4, 2, sa.SA_KV_FP4)
    fields = dict(dtype=sa.SA_F16, rotary_dim=64, pairs=0, n_axes=1, norm=0, eps=1e-6, scale=1.0, q_weight=0, k_weight=0, inv_freq=256, pair_axis=0)

    def call(n=4, Q=ONE, K=ONE, V=ONE, strides=(256, 128, 128), pos=ONE, outs=(ONE, ONE, ONE), **rot):
        r = sa.SaRotary(**{**fields, **rot})
        return lib.sa_rotate_qkv(C.byref(cfg), C.byref(r), Q, C.c_int64(strides[0]), K, C.c_int64(strides[1]), V, C.c_int64(strides[2]), pos, C.c_int64(n),
                                 *outs, NULL)

    assert call(n=0) == 0
    assert lib.sa_rotate_qkv(C.byref(cfg), NULL, ONE, C.c_int64(256), NULL, C.c_int64(0), NULL, C.c_int64(0), ONE, C.c_int64(0), ONE, NULL, NULL, NULL) == 1
    for bad in (dict(dtype=3), dict(rotary_dim=60), dict(rotary_dim=72), dict(rotary_dim=-8)):
        assert call(n=0, **bad) == 2, bad
    for bad in (dict(pairs=2), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2), dict(norm=2), dict(eps=-1.0), dict(eps=float("nan")), dict(inv_freq=0),
                dict(pos=NULL), dict(Q=NULL), dict(outs=(ONE, NULL, ONE)), dict(n=-1), dict(Q=NULL, K=NULL, V=NULL, outs=(NULL,) * 3),
                dict(strides=(255, 128, 128)), dict(strides=(256, 64, 128))):
        assert call(**{"n": 4, **bad}) == 1, bad
    odd = C.c_void_p(264)
    for bad in (dict(Q=odd), dict(outs=(ONE, ONE, odd)), dict(strides=(260, 128, 128)), dict(q_weight=264), dict(inv_freq=257), dict(pos=C.c_void_p(258))):
        assert call(**bad) == 3, bad
    assert call(n=1 << 31) == 4
    assert call(n=0, rotary_dim=0, inv_freq=0, pos=NULL) == 0 and call(n=0, n_axes=3, pair_axis=256) == 0
