"""Page tables of a cache: what the calls refuse, without a GPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import build, heart as h

    build.build()
    return h


GOOD = dict(S=2, T=10, Hq=8, Hkv=2, page=64, n_pages=9, table_stride=4)
EXTEND = ["new_len", "kv_len", "free_pages", "free_count", "page_table", "row_start", "kv_len_out", "free_count_out", "slots", "workspace"]
RELEASE = ["ended", "kv_len", "free_pages", "free_count", "page_table", "kv_len_out", "free_count_out", "workspace"]


def calls(heart, cfg, **change):
    lib = heart.lib()  # (pointers that are never dereferenced: validation fails first)
    cfg = None if cfg is None else C.byref(cfg)
    return (lib.heart_cache_extend(cfg, *(change.get(x, 256) for x in EXTEND), None), lib.heart_cache_release(cfg, *(change.get(x, 256) for x in RELEASE), None))


@pytest.mark.parametrize("change,code", [(dict(S=0), 1), (dict(T=-1), 1), (dict(page=48), 2), (dict(n_pages=0), 1), (dict(table_stride=0), 1),
                                         (dict(table_stride=1 << 25), 2), (dict(Hq=7), 1), (dict(flags=1), 1)])
def test_bad_configs_are_refused(heart, change, code):
    cfg = heart.make_cache_config(**GOOD)
    for k, v in change.items():
        setattr(cfg, k, v)
    assert calls(heart, cfg) == (code, code)
    assert calls(heart, None) == (heart.ERR_INVALID, heart.ERR_INVALID)


def test_null_and_misaligned_pointers_are_refused(heart):
    cfg = heart.make_cache_config(**GOOD)
    for name in set(EXTEND + RELEASE):
        for bad in (None, 258 if name not in ("slots", "workspace") else 260):
            got = calls(heart, cfg, **{name: bad, "workspace": 264 if name != "workspace" else bad})  # (refused for one or the other)
            assert got == (heart.ERR_INVALID, heart.ERR_INVALID)
    lib = heart.lib()
    for i, name in enumerate(EXTEND):
        for bad in ([] if name == "slots" else [None]) + [{"slots": 260, "workspace": 264}.get(name, 258)]:
            p = [256] * 10
            p[i] = bad
            assert lib.heart_cache_extend(C.byref(cfg), *p, None) == heart.ERR_INVALID, (name, bad)
    for i, name in enumerate(RELEASE):
        for bad in [None] + ([] if name == "ended" else [264 if name == "workspace" else 258]):
            p = [256] * 8
            p[i] = bad
            assert lib.heart_cache_release(C.byref(cfg), *p, None) == heart.ERR_INVALID, (name, bad)


def test_tensors_on_the_host_are_refused(heart):
    cfg = heart.make_cache_config(**GOOD)
    i = [torch.zeros(n, dtype=torch.int32) for n in (2, 2, 9, 1, 8, 3)]
    ws = torch.zeros(heart.cache_workspace_bytes(cfg), dtype=torch.uint8)
    with pytest.raises(ValueError):
        heart.heart_cache_extend(cfg, *i, ws)
    with pytest.raises(ValueError):
        heart.heart_cache_release(cfg, torch.zeros(2, dtype=torch.uint8), *i[1:5], ws)
