"""Which kernel a call of cross attention takes, asked of the test-hook build, without a GPU."""
import ctypes as C

import pytest

ROWS8, ROWS16, TILES, PAIRS = range(4)  # as CrossKernel has them


@pytest.fixture(scope="module")
def kernel_of():
    from paper_2605_14513_b200 import build, heart

    lib = C.CDLL(build.build_test_hooks())
    return lambda **kw: lib.heart_test_cross_kernel(C.byref(heart.make_cross_config(**kw)))


@pytest.mark.parametrize("T,Hq,Hkv,expected", [
    # by keys 500, 2000, 8000, 32 000: few rows read short states several times, long ones rarely
    (4, 64, 8, (ROWS8, ROWS8, ROWS16, ROWS16)),
    (32, 12, 12, (ROWS8, ROWS8, ROWS16, TILES)),
    (370, 1, 1, (ROWS8, ROWS8, ROWS16, TILES)),
    (300, 1, 1, (ROWS8, ROWS8, ROWS16, TILES)),
    (16, 1, 1, (ROWS8, ROWS8, ROWS8, ROWS8)),
])
def test_few_rows_over_many_keys(kernel_of, T, Hq, Hkv, expected):
    for Tk, kernel in zip((500, 2000, 8000, 32000), expected):
        assert kernel_of(S=1, T=T, Tk=Tk, Hq=Hq, Hkv=Hkv) == kernel, Tk
        # (as many sequences of their own states: as short ones)
        assert kernel_of(S=1000, T=1, Tk=1000 * Tk, Hq=Hq, Hkv=Hkv, max_q=1) == (ROWS8 if Hq // Hkv <= 8 else ROWS16)


def test_rows_of_a_sequence_and_sizes(kernel_of):
    size = dict(Hq=12, Hkv=12)
    assert kernel_of(S=64, T=64, Tk=64 * 32000, max_q=1, **size) == ROWS8
    assert kernel_of(S=64, T=1024, Tk=64 * 100, max_q=16, **size) == ROWS16
    assert kernel_of(S=1, T=4680, Tk=512, **size) == TILES
    assert kernel_of(S=1, T=1000, Tk=32760, **size) == PAIRS
    assert kernel_of(S=2, T=65520, Tk=687, Hq=40, Hkv=40) == PAIRS
    assert kernel_of(S=1, T=1 << 20, Tk=1, Hq=1, Hkv=1) == PAIRS
    big = (1 << 31) - 257
    for S in (1, 7, (1 << 30) - 1):
        for T in (1, 20, big):
            for Tk in (1, big):
                assert kernel_of(S=S, T=T, Tk=Tk, Hq=1, Hkv=1) in range(4)
    assert kernel_of(S=0, T=1, Tk=1, Hq=1, Hkv=1) == -1
