"""The sizes that the attention refuses are the ones that its header states (no GPU)."""
import ctypes

import pytest

UNSUPPORTED = 2
FAKE = 0x100000   # never dereferenced


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def _status(gs, tokens, n, width, heads=2, kv_heads=2, page=16, max_new=1):
    cache = gs._CacheStruct(FAKE, FAKE + (1 << 28), 4, page, kv_heads, 64)
    batch = gs._BatchStruct(FAKE + (2 << 28), FAKE + (3 << 28), FAKE + (4 << 28), n, width, tokens, max_new)
    size = ctypes.c_size_t()
    return gs.lib.gs_paged_attention_workspace(ctypes.byref(cache), ctypes.byref(batch), heads, ctypes.byref(size))


@pytest.mark.parametrize("tokens,n,heads,kv_heads,page", [(128, 60, 2, 2, 16), (1 << 20, 1, 2, 2, 64), (64, 64, 56, 8, 256),
                                                          (1 << 16, 5, 4, 1, 32)])
def test_work_in_32_bits(gs, tokens, n, heads, kv_heads, page):
    rows = tokens * heads // kv_heads
    per = (rows / 128 + n + 1) * kv_heads                # items; each of (keys / 64 + 6) units at most
    width = int((2e9 / per - 6) * 64 / page)
    assert width * page < 2 ** 31 - 256
    assert _status(gs, tokens, n, width - 1, heads, kv_heads, page) == 0
    assert _status(gs, tokens, n, width + 2, heads, kv_heads, page) == UNSUPPORTED


def test_rows_below_a_thousand_million(gs):
    assert _status(gs, 10 ** 9 - 1, 1, 1, 1, 1) == 0
    assert _status(gs, 10 ** 9, 1, 1, 1, 1) == UNSUPPORTED


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("max_new", [1, 8])
def test_keys_end_a_tile_short_of_32_bits(gs, page, max_new):
    """The key that follows a sequence's last tile has a number of 32 bits too."""
    most = (2 ** 31 - 256) // page
    assert _status(gs, max_new, 1, most, 1, 1, page, max_new) == 0
    if (most + 1) * page < 2 ** 31:
        assert _status(gs, max_new, 1, most + 1, 1, 1, page, max_new) == UNSUPPORTED
