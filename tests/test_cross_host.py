"""Cross attention: sizes, struct layout and what is refused, without a GPU."""
import ctypes as C
import math

import pytest
import torch

GOOD = dict(S=2, T=10, Tk=30, Hq=8, Hkv=2)


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import build, heart as h

    build.build()
    return h


def config(heart, **kw):
    c = heart.make_cross_config(**GOOD)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def call(heart, cfg, *pointers):
    lib = heart.lib()  # (never dereferenced: validation fails first)
    return lib.heart_cross_attn(None if cfg is None else C.byref(cfg), *pointers, None)


FAKE = [256] * 7 + [None, 256]  # Q, K, V, q_start, k_start, k_len, O, lse, workspace


def test_struct_layout_matches_header(heart):
    # int32 x7, uint32, int64 x4, double
    assert C.sizeof(heart.CrossConfig) == 8 * 4 + 4 * 8 + 8
    assert heart.CrossConfig.flags.offset == 28 and heart.CrossConfig.q_stride_t.offset == 32 and heart.CrossConfig.scale.offset == 64


BAD = [(dict(S=0), 1), (dict(T=0), 1), (dict(Tk=0), 1), (dict(Hq=0), 1), (dict(Hkv=0), 1), (dict(S=-1), 1), (dict(max_q=-1), 1), (dict(Hq=7), 1),
       (dict(Hq=2 * 129), 2), (dict(D=64), 2), (dict(flags=1), 1), (dict(T=1 << 28), 2), (dict(Tk=(1 << 31) - 1), 2), (dict(S=1 << 30), 2),
       (dict(scale=math.nan), 1), (dict(scale=math.inf), 1), (dict(scale=1e31), 1), (dict(scale=1e-31), 1), (dict(q_stride_t=1024), 1),
       (dict(q_stride_t=1020, q_stride_h=128), 1), (dict(q_stride_t=64, q_stride_h=128), 1), (dict(kv_stride_t=-256, kv_stride_h=128), 1),
       (dict(kv_stride_h=128), 1), (dict(q_stride_t=1 << 40, q_stride_h=128), 1), (dict(Hq=128, Hkv=2, q_stride_t=128, q_stride_h=1 << 37), 1)]


@pytest.mark.parametrize("change,code", BAD)
def test_bad_configs_are_refused(heart, change, code):
    cfg = config(heart, **change)
    assert heart.cross_workspace_bytes(cfg) == 0
    assert call(heart, cfg, *FAKE) == code
    with pytest.raises(heart.HeartError):
        heart.new_cross_workspace(cfg)


def test_good_configs_have_workspaces(heart):
    for change in (dict(), dict(Hq=256), dict(Hq=6), dict(scale=0.1), dict(max_q=3), dict(q_stride_t=128, q_stride_h=1280), dict(T=1, Tk=1, S=5)):
        n = heart.cross_workspace_bytes(config(heart, **change))
        assert n > 0 and n % 256 == 0, change


def test_null_and_misaligned_pointers_are_refused(heart):
    cfg = config(heart)
    for i in range(9):
        bad = [258 if i in (3, 4, 5, 7) else 264] + ([] if i == 7 else [None])  # (lse may be NULL)
        for x in bad:
            p = list(FAKE)
            p[i] = x
            assert call(heart, cfg, *p) == heart.ERR_INVALID, (i, x)
    assert call(heart, None, *FAKE) == heart.ERR_INVALID


def test_tensors_on_the_host_are_refused(heart):
    cfg = config(heart)
    Q, K = torch.zeros((10, 8, 128), dtype=torch.bfloat16), torch.zeros((30, 2, 128), dtype=torch.bfloat16)
    i32 = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        heart.heart_cross_attn(cfg, Q, K, K, i32, i32[:2], i32[:2], Q, torch.zeros(heart.cross_workspace_bytes(cfg), dtype=torch.uint8))
