"""Sizes past what a launch or a 32-bit position holds are refused before
anything is enqueued (no call here reaches a launch)."""
import ctypes
import os

import numpy as np
import pytest

from test_abi_cpu import ERR_UNSUPPORTED, FAKE

CU = np.zeros(1, np.int32)
PTR = CU.ctypes.data_as(ctypes.c_void_p)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    import paper_2608_29539_amd as pk
    if not os.path.exists(pk.library_path()):
        from paper_2608_29539_amd.build import build_library
        build_library()
    return pk.library()


def problem(B, N, longest, hq, hkv, d=128, window=64):
    """Without a host copy of the bounds, so that only the sizes are looked at."""
    import paper_2608_29539_amd.binding as b
    return ctypes.byref(b._Problem(B, N, longest, PTR, None, hq, hkv, d, window, 0.0))


def prefix(lib, p, R, total, longest, group):
    import paper_2608_29539_amd.binding as b
    x = b._Prefix(R, total, longest, group, PTR, PTR, None, None)
    return lib.logo_decode_prefix(p, ctypes.byref(x), FAKE, FAKE, FAKE, FAKE, FAKE, None, None,
                                  None, None, None, FAKE, 0, 0.5, None, None, None, 1e-6, FAKE,
                                  None, None, FAKE, BIG, None)


def score(lib, p, cap, lse):
    return lib.logo_cache_score(p, FAKE, FAKE, FAKE, FAKE, cap, FAKE if lse else None, None, FAKE,
                                FAKE, BIG, None)


def step(lib, p):
    return lib.logo_decode_score(p, FAKE, FAKE, FAKE, 0, 0.5, None, None, FAKE, FAKE, BIG, None)


def evict(lib, p, cap, caches=True):
    c = [FAKE if caches else None] * 2
    return lib.logo_cache_evict(p, FAKE, 1 << 30, 0, *c, None, None, *c, None, None, FAKE, FAKE,
                                FAKE, cap, FAKE, BIG, None)


def test_launches_of_2_to_the_32_threads(lib):
    """HIP takes fewer than 2^32 threads in a launch; what needs more is
    unsupported, not a HIP error."""
    # 2^24 workgroups of 256 threads: sequences' heads, a prefix's items
    assert prefix(lib, problem(1 << 21, 1 << 21, 1, 8, 8), 1, 1, 1, 1) == ERR_UNSUPPORTED
    assert prefix(lib, problem(8, 8, 1, 64, 64), 1 << 18, 1 << 18, 1 << 14, 1) == ERR_UNSUPPORTED
    # key blocks of 2^21 sequences, row tiles of 2^21 sequences
    assert score(lib, problem(1 << 21, 1 << 21, 1, 8, 8), 8, True) == ERR_UNSUPPORTED
    assert score(lib, problem(1 << 21, 1 << 21, 1, 8, 8), 8, False) == ERR_UNSUPPORTED
    # 2^25 workgroups of 128 threads, 2^24 of 256
    assert step(lib, problem(1 << 17, 1 << 20, 1 << 13, 32, 32)) == ERR_UNSUPPORTED
    assert step(lib, problem(1 << 21, 1 << 21, 1, 8, 8)) == ERR_UNSUPPORTED
    # 2^22 workgroups of 1024 threads, 2^24 of 256; copies of 2^28 rows of d = 128
    assert evict(lib, problem(1 << 18, 1 << 21, 1 << 14, 8, 8), 1 << 21) == ERR_UNSUPPORTED
    assert evict(lib, problem(1 << 21, 1 << 21, 1, 8, 8), 1 << 21) == ERR_UNSUPPORTED
    assert evict(lib, problem(2, 1 << 25, 1 << 24, 8, 8), 1 << 25) == ERR_UNSUPPORTED


def test_rows_next_to_2_to_the_31(lib):
    """The end of a block of keys behind the last row passes 2^31."""
    for n in ((1 << 31) - 100, (1 << 31) - 1):
        assert score(lib, problem(1, n, n, 1, 1, 64), 8, True) == ERR_UNSUPPORTED
        assert score(lib, problem(1, n, n, 1, 1, 64), 8, False) == ERR_UNSUPPORTED
        assert step(lib, problem(1, n, n, 1, 1, 64)) == ERR_UNSUPPORTED


def test_tiles_of_2_gib(lib):
    """A tile's rows of so many heads that its byte offsets pass 2^31."""
    assert score(lib, problem(1, 100, 100, 1 << 17, 1 << 17), 8, False) == ERR_UNSUPPORTED
    assert step(lib, problem(1, 100, 100, 1 << 19, 1 << 19)) == ERR_UNSUPPORTED
