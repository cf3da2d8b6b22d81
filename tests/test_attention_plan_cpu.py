"""How attention over the 4-bit cache is cut, as far as its workspace shows it (equal shares take one, clusters none)."""

import ctypes

import pytest


@pytest.fixture(scope="module")
def kd():
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _workspace(kd, seqs, most, longest, heads, kv_heads, d=128, starts=True, page=64):
    at = 4096  # an aligned address that is never read
    wide = -(-longest // page)
    cache = kd.KdCache4(at, at, at, at, seqs * wide, kv_heads, page, d, 64)
    s = kd.KdSequences(at, at, at if starts else None, wide, seqs, wide, most, longest)
    return kd.kd_attention_4bit_workspace(ctypes.addressof(cache), ctypes.addressof(s), heads, 0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("seqs,most,longest,heads,kv_heads", [(4, 1000, 1000, 32, 8), (16, 250, 250, 32, 8), (16, 100, 1000, 32, 32),
                                                              (64, 32, 1000, 32, 8), (64, 128, 128, 32, 8), (2, 1000, 1000, 32, 8),
                                                              (8, 8, 100, 64, 8), (3, 64, 40, 4, 4)])
def test_prompts_go_to_clusters(kd, seqs, most, longest, heads, kv_heads, d):
    """Eight blocks of rows of a sequence or more."""
    assert _workspace(kd, seqs, most, longest, heads, kv_heads, d) == 0
    assert _workspace(kd, seqs, most, longest, heads, kv_heads, d, starts=False) == 0


def test_long_sequences_go_to_shares(kd):
    assert _workspace(kd, 1, 1, 131072, 32, 8) > 0
    assert _workspace(kd, 64, 1, 8192, 32, 8) > 0
