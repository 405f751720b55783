"""Speculative-decoding entry points: what is refused on the host, without a device."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2603_04411_b200 import build
    build.build()
    from paper_2603_04411_b200 import binding
    return binding


def test_calls_without_a_cache_are_refused(B):
    p = ctypes.c_void_p(256)
    assert B.lib.twkv_slot_map(None, 0, p, p, None, 1, 1, p, p, p, None) == B.TWKV_ERR_INVALID_ARG
    assert B.lib.twkv_tree_map(None, p, p, 1, 1, 8, p, p, None) == B.TWKV_ERR_INVALID_ARG
    assert B.lib.twkv_tree_accept(None, p, p, p, p, 1, 1, 8, p, p, p, None) == B.TWKV_ERR_INVALID_ARG
    assert B.lib.twkv_tree_attn(None, 0, p, p, p, p, p, p, p, p, 1, 1, 8, p, p, 1 << 30, None) == B.TWKV_ERR_INVALID_ARG
    assert B.twkv_tree_required_bytes(None, 1, 8) == 0
    assert B.TREE_MAX_NODES == 64
