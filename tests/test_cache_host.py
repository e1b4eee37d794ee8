"""The calls on a paged cache: sizes, struct layout and what is refused, without a GPU."""
import ctypes as C
import math
import types

import pytest
import torch

import cache_cases


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import build, heart as h

    build.build()
    return h


GOOD = dict(S=2, T=10, Hq=8, Hkv=2, page=64, n_pages=9, table_stride=4)


def config(heart, **kw):
    c = heart.make_cache_config(**GOOD)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_struct_layout_matches_header(heart):
    # int32 x13, uint32, int64 x7, double
    assert C.sizeof(heart.CacheConfig) == 14 * 4 + 7 * 8 + 8
    assert heart.CacheConfig.flags.offset == 52 and heart.CacheConfig.q_stride_t.offset == 56 and heart.CacheConfig.scale.offset == 112
    assert C.sizeof(heart.CacheStruct) == 32


BAD = [(dict(S=0), 1), (dict(T=0), 1), (dict(Hq=0), 1), (dict(Hkv=0), 1), (dict(n_pages=0), 1), (dict(table_stride=0), 1), (dict(S=-1), 1),
       (dict(Hq=7), 1), (dict(Hq=2 * 129), 2), (dict(D=64), 2), (dict(page=48), 2), (dict(page=256), 2), (dict(page=0), 2), (dict(kind=2), 1),
       (dict(kind=-1), 1), (dict(causal=-1), 1), (dict(window=-1), 1), (dict(sink=-1), 1), (dict(max_new=-1), 1), (dict(flags=1), 1),
       (dict(table_stride=1 << 25), 2), (dict(T=1 << 28), 2), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1), (dict(scale=1e31), 1),
       (dict(scale=1e-31), 1), (dict(q_stride_t=1024), 1), (dict(q_stride_t=1020, q_stride_h=128), 1), (dict(q_stride_t=64, q_stride_h=128), 1),
       (dict(kv_stride_t=-256, kv_stride_h=128), 1), (dict(pool_stride_page=16384), 1), (dict(kind=1, pool_stride_page=16392, pool_stride_h=8192, pool_stride_t=128), 1),
       (dict(q_stride_t=1 << 40, q_stride_h=128), 1)]


@pytest.mark.parametrize("change,code", BAD)
def test_bad_configs_are_refused(heart, change, code):
    cfg = config(heart, **change)
    fake, lib = C.c_void_p(256), heart.lib()  # never dereferenced: validation fails first
    cache = heart.CacheStruct(256, 256, 256, 256)
    assert heart.cache_workspace_bytes(cfg) == 0
    assert lib.heart_cache_write(C.byref(cfg), fake, fake, C.byref(cache), fake, fake, fake, fake, None) == code
    assert lib.heart_cache_read(C.byref(cfg), C.byref(cache), fake, fake, fake, fake, fake, fake, None) == code
    assert lib.heart_cache_attn(C.byref(cfg), fake, C.byref(cache), fake, fake, fake, fake, None, fake, None) == code
    with pytest.raises(heart.HeartError):
        heart.new_cache_workspace(cfg)


def test_good_configs_have_workspaces(heart):
    for change in (dict(), dict(kind=1), dict(page=16), dict(page=128), dict(Hq=256), dict(Hq=6), dict(scale=0.1), dict(causal=1, window=5, sink=3),
                   dict(pool_stride_page=16384 + 8, pool_stride_h=8192, pool_stride_t=128), dict(q_stride_t=128, q_stride_h=1280)):
        n = heart.cache_workspace_bytes(config(heart, **change))
        assert n > 0 and n % 256 == 0, change


def test_null_and_misaligned_pointers_are_refused(heart):
    lib, fake, null = heart.lib(), 256, None
    for kind in (0, 1):
        cfg = config(heart, kind=kind)
        good = [256, 256, 256, 256]
        for i, bad in [(0, 0), (1, 0), (0, 264), (1, 264)] + ([(2, 0), (3, 0), (2, 264), (3, 260)] if kind else []):
            ptrs = list(good)
            ptrs[i] = bad
            cache = heart.CacheStruct(*ptrs)
            assert lib.heart_cache_write(C.byref(cfg), fake, fake, C.byref(cache), fake, fake, fake, fake, None) == heart.ERR_INVALID
            assert lib.heart_cache_read(C.byref(cfg), C.byref(cache), fake, fake, fake, fake, fake, fake, None) == heart.ERR_INVALID
            assert lib.heart_cache_attn(C.byref(cfg), fake, C.byref(cache), fake, fake, fake, fake, null, fake, None) == heart.ERR_INVALID
        cache = heart.CacheStruct(*good)
        for i in range(7):  # K, V, (cache), table, row_start, kv_len, workspace
            for bad in (null, 264 if i in (0, 1, 6) else 258):
                if i == 2:
                    continue
                args = [C.byref(cfg), fake, fake, C.byref(cache), fake, fake, fake, fake, None]
                args[1 + (i if i < 2 else i)] = bad if i < 2 else args[1 + i]
                if i > 2:
                    args[1 + i] = bad
                assert lib.heart_cache_write(*args) == heart.ERR_INVALID, (i, bad)
        assert lib.heart_cache_write(None, fake, fake, C.byref(cache), fake, fake, fake, fake, None) == heart.ERR_INVALID
        assert lib.heart_cache_write(C.byref(cfg), fake, fake, None, fake, fake, fake, fake, None) == heart.ERR_INVALID
        assert lib.heart_cache_read(C.byref(cfg), C.byref(cache), fake, fake, fake, null, fake, fake, None) == heart.ERR_INVALID
        assert lib.heart_cache_read(C.byref(cfg), C.byref(cache), fake, fake, fake, fake, 264, fake, None) == heart.ERR_INVALID
        assert lib.heart_cache_attn(C.byref(cfg), null, C.byref(cache), fake, fake, fake, fake, null, fake, None) == heart.ERR_INVALID
        assert lib.heart_cache_attn(C.byref(cfg), fake, C.byref(cache), fake, fake, fake, 264, null, fake, None) == heart.ERR_INVALID
        assert lib.heart_cache_attn(C.byref(cfg), fake, C.byref(cache), fake, fake, fake, fake, 258, fake, None) == heart.ERR_INVALID


def test_pools_on_the_host_are_refused(heart):
    cfg = config(heart)
    k = torch.zeros((9, 2, 64, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        heart.Cache(cfg, k, k)


def fake_cache(heart, cfg):
    """As far as the checks of a call look at it, on the host."""
    return types.SimpleNamespace(device=-1, layout=heart._cache_layout(cfg), fields=heart._cache_fields(cfg))


def call(heart, cfg, cache, x, strides=(0, 0)):
    cfg = heart.CacheConfig.from_buffer_copy(cfg)
    cfg.kv_stride_t, cfg.kv_stride_h = strides
    ints = [torch.zeros(n, dtype=torch.int32) for n in (cfg.S * cfg.table_stride, cfg.S + 1, cfg.S)]
    ws = torch.zeros(heart.cache_workspace_bytes(cfg), dtype=torch.uint8)
    heart._cache_call(cfg, cache, False, (x,), *ints, ws)


def test_a_cache_of_other_pools_is_refused(heart):
    cfg = config(heart)
    cache = fake_cache(heart, cfg)
    x = torch.zeros((cfg.T, 2, 128), dtype=torch.bfloat16)
    call(heart, cfg, cache, x)
    call(heart, config(heart, causal=3, window=5, max_new=2), cache, x)
    call(heart, config(heart, pool_stride_page=2 * cfg.page * 128, pool_stride_h=cfg.page * 128, pool_stride_t=128), cache, x)  # the same, spelt out
    for change in (dict(n_pages=cfg.n_pages + 1), dict(page=2 * cfg.page), dict(kind=1), dict(Hkv=1),
                   dict(pool_stride_page=2 * cfg.page * 128, pool_stride_h=128, pool_stride_t=256)):
        with pytest.raises(ValueError):
            call(heart, config(heart, **change), cache, x)


def test_packed_tensors_that_do_not_hold_their_strides_are_refused(heart):
    cfg = config(heart)
    cache, T = fake_cache(heart, cfg), cfg.T
    plain = torch.zeros((T, 2, 128), dtype=torch.bfloat16)
    wide = torch.zeros((T, 3, 128), dtype=torch.bfloat16)
    call(heart, cfg, cache, plain)
    call(heart, cfg, cache, plain, strides=(256, 128))
    call(heart, cfg, cache, wide[:, :2], strides=(384, 128))
    call(heart, cfg, cache, wide[:, 1:], strides=(384, 128))
    call(heart, cfg, cache, torch.zeros((2, T, 128), dtype=torch.bfloat16), strides=(128, T * 128))
    call(heart, cfg, cache, torch.zeros((1, 2, T, 128), dtype=torch.bfloat16), strides=(128, T * 128))
    call(heart, cfg, cache, plain.flatten(), strides=(256, 128))
    for x, strides in ((wide[:, :2], (0, 0)), (plain, (384, 128)), (plain, (128, T * 128)), (wide[:, :2], (256, 128)),
                       (plain.flatten(), (384, 128)), (plain.transpose(1, 2), (256, 128)), (plain, (256, -128)), (plain.float(), (256, 128)),
                       (torch.zeros((2, T, 128), dtype=torch.bfloat16), (256, 128))):
        with pytest.raises(ValueError):
            call(heart, cfg, cache, x, strides=strides)


def test_the_definition_of_the_codes():
    """The tests' own quantisation: scales are the smallest that fit, codes the nearest, halves to even."""
    x = torch.zeros((7, 128), dtype=torch.bfloat16)
    x[0, 0], x[0, 1], x[0, 2] = 448.0, 17.0, 19.0       # 2^0; halfway between 16 and 18, 18 and 20
    x[1, 5] = -450.0                                     # 2^1
    x[2, 7] = 2.0 ** -120                                # the smallest scale
    x[3, 9] = math.inf
    x[4, 9] = math.nan
    x[6, 1] = 3.3e38
    codes, scale = cache_cases.quantise(x)
    assert scale.tolist() == [127, 128, 17, 255, 255, 17, 247]
    assert codes[0, :3].float().tolist() == [448.0, 16.0, 20.0]
    back = cache_cases.dequantise(codes, scale)
    assert float(back[1, 5]) == -448.0 and float(back[2, 7]) == 0.0 and torch.isnan(back[3:5]).all() and (back[5] == 0).all()
    assert torch.equal(back[6].to(torch.bfloat16).double(), back[6]) and float(back[6, 1]) == 1.875 * 2.0 ** 127
