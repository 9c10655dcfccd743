"""Host-side validation of sa_append_qkv and sa_chunk_attention: what is refused, and that it is before anything is launched (without a GPU a launch would
come back as status 5); and what the binding takes for a tensor."""
import ctypes as C

import pytest

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from test_binding_types import outcomes

NULL, ONE, FAR = C.c_void_p(0), C.c_void_p(256), C.c_void_p(1 << 40)      # non-null, aligned addresses that nothing may follow


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def i64(*v):
    return (C.c_int64 * len(v))(*v)


def test_chunk_attention_refuses():
    lib, cfg, good = sa.lib(), sa.make_config(64, 32, 4, sa.SA_POTM4), sa.SaCache(256, 256, 256, 2, 4, 8)

    def call(cu=i64(0, 1, 3), window=0, sinks=0, Q=ONE, O=FAR, dtype=sa.SA_F16, ws=ONE, ws_bytes=1 << 40, cache=good, cfg=cfg):
        return lib.sa_chunk_attention(C.byref(cfg), C.byref(cache), Q, cu, C.c_int(window), C.c_int(sinks), O, C.c_int(dtype), ws, C.c_size_t(ws_bytes), NULL)

    for bad in (dict(cu=None), dict(cu=i64(0, 2, 1)), dict(cu=i64(-1, 0, 1)), dict(window=-1), dict(sinks=-1), dict(Q=NULL), dict(O=NULL), dict(ws=NULL),
                dict(O=ONE), dict(O=C.c_void_p(256 + 3 * 32 * 64 * 2 - 16)), dict(Q=C.c_void_p((1 << 40) + 16)), dict(cache=sa.SaCache(0, 256, 256, 2, 4, 8))):
        assert call(**bad) == 1, bad
    for bad in (dict(dtype=sa.SA_F32), dict(dtype=7), dict(cfg=sa.make_config(96, 32, 4, sa.SA_POTM4)), dict(cfg=sa.make_config(64, 32, 4, sa.SA_POTM4, shift_add=True)),
                dict(cfg=sa.make_config(64, 32, 4, sa.SA_POT4, add_on_alu=True)), dict(cfg=sa.make_config(64, 32, 4, sa.SA_POTM1, shift_by_multiply=True))):
        assert call(**bad) == 2, bad
    for bad in (dict(Q=C.c_void_p(264)), dict(O=C.c_void_p(264)), dict(ws=C.c_void_p(272)), dict(cache=sa.SaCache(264, 256, 256, 2, 4, 8))):
        assert call(**bad) == 3, bad
    need = C.c_size_t()
    assert lib.sa_chunk_workspace_bytes(C.byref(cfg), C.c_int(2), C.c_int64(3), C.byref(need)) == 0
    for bad in (dict(cu=i64(0, 257, 258)), dict(ws_bytes=need.value - 1), dict(cu=i64(0, 100, 101), ws_bytes=need.value)):
        assert call(**bad) == 4, bad
    wide = sa.SaCache(256, 256, 256, 2, 1 << 26, 8)
    assert call(cu=i64(0, 1 << 28, 1 << 28), cache=wide) == 4          # rows (tokens and heads of a group) beyond 32 bits
    assert call(cu=i64(1 << 60, (1 << 60) + 1, (1 << 60) + 1)) == 4     # addresses beyond 64
    assert call(cu=i64(5, 5, 5), Q=NULL, O=NULL, ws=NULL) == 0          # nothing to do


def test_sizes_of_the_workspace():
    for d in (64, 128):
        cfg = sa.make_config(d, 32, 4, sa.SA_KV_FP4)
        small, large = sa.chunk_workspace_bytes(cfg, 8, 16), sa.chunk_workspace_bytes(cfg, 8, 17)
        assert 0 < small < large == sa.chunk_workspace_bytes(cfg, 1000, 1 << 40) < 64 << 20
    for bad in ((cfg, 0, 5), (cfg, 1, -1)):
        with pytest.raises(sa.SaError) as e:
            sa.chunk_workspace_bytes(*bad)
        assert e.value.status == 1
    with pytest.raises(sa.SaError):
        sa.chunk_workspace_bytes(sa.make_config(96, 32, 4, sa.SA_KV_FP4), 1, 1)


def test_append_refuses():
    lib, cfg, good = sa.lib(), sa.make_config(64, 4, 2, sa.SA_KV_FP4), sa.SaCache(256, 256, 256, 2, 4, 8)
    fields = dict(dtype=sa.SA_F16, rotary_dim=64, pairs=0, n_axes=1, norm=0, eps=1e-6, scale=1.0, q_weight=0, k_weight=0, inv_freq=256, pair_axis=0)

    def call(n=4, cu=i64(0, 1, 4), Q=ONE, K=ONE, V=ONE, strides=(256, 128, 128), pos=ONE, out=ONE, cache=good, cfg=cfg, **rot):
        r = sa.SaRotary(**{**fields, **rot})
        return lib.sa_append_qkv(C.byref(cfg), C.byref(cache), C.byref(r), Q, C.c_int64(strides[0]), K, C.c_int64(strides[1]), V, C.c_int64(strides[2]), pos, C.c_int64(n),
                                 cu, out, C.c_int(1), NULL)

    assert call(cu=i64(2, 2, 2)) == 0 and call(n=0, cu=i64(0, 0, 0)) == 0
    for bad in (dict(cu=None), dict(cu=i64(0, 2, 1)), dict(cu=i64(-1, 0, 1)), dict(cu=i64(0, 1, 5)), dict(n=3), dict(n=-1), dict(K=NULL), dict(V=NULL), dict(Q=NULL), dict(out=NULL),
                dict(pos=NULL), dict(inv_freq=0), dict(n_axes=5), dict(pairs=2), dict(norm=3), dict(eps=-1.0), dict(strides=(255, 128, 128)), dict(strides=(256, 64, 128)),
                dict(cache=sa.SaCache(256, 0, 256, 2, 4, 8))):
        assert call(**bad) == 1, bad
    for bad in (dict(dtype=3), dict(rotary_dim=60), dict(cfg=sa.make_config(96, 4, 2, sa.SA_KV_FP4)), dict(cfg=sa.make_config(64, 201, 201, sa.SA_KV_FP4), strides=(1 << 20,) * 3)):
        assert call(**bad) == 2, bad
    odd = C.c_void_p(264)
    for bad in (dict(K=odd), dict(out=odd), dict(strides=(260, 128, 128)), dict(q_weight=264), dict(cache=sa.SaCache(264, 256, 256, 2, 4, 8))):
        assert call(**bad) == 3, bad
    assert call(n=300, cu=i64(0, 257, 258)) == 4 and call(n=1 << 31) == 4


def test_what_the_binding_takes():
    """Stand-ins for tensors at an address between two 16-byte places: the library stops what the binding lets through with status 3."""
    got = outcomes("""(lambda cu: {
        'good': [outcome(lambda: sa.chunk_attention(cfg, cache, Stand(q, 9, 4, 64), Stand(o, 9, 4, 64), ws, cu)) for q in (torch.float16, torch.int16, torch.uint16) for o in (torch.float16, torch.bfloat16)],
        'bad': [outcome(lambda: sa.chunk_attention(cfg, cache, Stand(*q), Stand(*o), ws, c)) for q, o, c in (
            ((torch.bfloat16, 9, 4, 64), (torch.float16, 9, 4, 64), cu), ((torch.bfloat16, 9, 4, 64), (torch.bfloat16, 9, 4, 64), cu), ((torch.float16, 9, 4, 64), (torch.float32, 9, 4, 64), cu),
            ((torch.float16, 8, 4, 64), (torch.float16, 9, 4, 64), cu), ((torch.float16, 9, 4, 64), (torch.float16, 8, 4, 64), cu), ((torch.float16, 9, 2, 64), (torch.float16, 9, 2, 64), cu),
            ((torch.float16, 9, 4, 64), (torch.float16, 9, 4, 64), cu[:2]), ((torch.float16, 9, 4, 64), (torch.float16, 9, 4, 64), cu.astype(np.int32)))],
        'append': [outcome(lambda: sa.append_qkv(rot, cache, Stand(torch.bfloat16, 9, 4, 64), Stand(k, 9, 2, 64), Stand(torch.bfloat16, n, 2, 64), Stand(pos, 1, 9), c, Stand(out, m, 4, 64))) for k, n, pos, c, out, m in (
            (torch.bfloat16, 9, torch.int32, cu, torch.float16, 9), (torch.float16, 9, torch.int32, cu, torch.float16, 9), (torch.bfloat16, 8, torch.int32, cu, torch.float16, 9),
            (torch.bfloat16, 9, torch.int64, cu, torch.float16, 9), (torch.bfloat16, 9, torch.int32, cu[:2], torch.float16, 9), (torch.bfloat16, 9, torch.int32, cu, torch.bfloat16, 9),
            (torch.bfloat16, 9, torch.int32, cu, torch.float16, 10))],
        })(np.array([0, 5, 9])) if [globals().update(ws=type('W', (), dict(nbytes=1 << 30, data_ptr=lambda self: 256))())] else None""")
    assert got["good"] == [3] * 6
    assert got["bad"] == ["refused"] * 8
    assert got["append"] == [3] + ["refused"] * 6


def test_windows_that_are_no_32_bit_numbers():
    """2^32 + 5 is not a window of 5, nor 2^32 none at all."""
    got = outcomes("""(lambda cu: [outcome(lambda: sa.chunk_attention(cfg, cache, Stand(torch.float16, 9, 4, 64), Stand(torch.float16, 9, 4, 64), ws, cu, w, s)) for w, s in (
        (5, 2), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 0), (2 ** 32, 0), (2 ** 32 + 5, 0), (5, 2 ** 32), (5, -2 ** 32))])(np.array([0, 5, 9]))
        if [globals().update(ws=type('W', (), dict(nbytes=1 << 30, data_ptr=lambda self: 256))())] else None""")
    assert got == [3, 3] + ["refused"] * 5


def test_lost_copy_hook_refuses():
    lib, good, cache = sa.lib(), sa.make_config(64, 32, 4, sa.SA_POTM4), sa.SaCache(256, 256, 256, 2, 4, 8)

    def call(cfg=good, b=0, kv_head=0, tile=0, cu=i64(0, 1, 3), ws_bytes=1 << 40):
        return lib.sa_debug_chunk_lost_copy(C.byref(cfg), C.byref(cache), ONE, cu, FAR, ONE, C.c_size_t(ws_bytes), C.c_int(b), C.c_int(kv_head), C.c_int(tile), NULL)

    for cfg in (sa.make_config(128, 32, 4, sa.SA_POTM4), sa.make_config(64, 32, 4, sa.SA_POTM2), sa.make_config(64, 32, 4, sa.SA_KV_FP4), sa.make_config(64, 32, 4, sa.SA_POTM1, nibble=True)):
        assert call(cfg=cfg) == 2
    for bad in (dict(b=2), dict(b=-1), dict(kv_head=4), dict(kv_head=-1), dict(cu=i64(0, 2, 1))):
        assert call(**bad) == 1, bad
    assert call(ws_bytes=8) == 4 and call(cu=i64(0, 0, 0), tile=-3) == 0
