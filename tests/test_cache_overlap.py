"""What may not overlap, and sizes that no launch takes, without a GPU: refused before anything is enqueued."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2410_17980_amd import binding
    return binding.load()


P = lambda at: ctypes.c_void_p(at)
MB = 1 << 20
OVERLAP, SHAPE, WORKSPACE = -7, -2, -6


# 32 rows of 4 bytes: 128 bytes of scores
@pytest.mark.parametrize("off,refused", [(16, True), (-16, True), (112, True), (-112, True), (128, False), (-128, False), (0, False)])
def test_scores_in_place_or_apart(lib, off, refused):
    """(What is not refused gets as far as the missing workspace.)"""
    want = OVERLAP if refused else WORKSPACE
    s, out = P(4 * MB), P(4 * MB + off)
    assert lib.sb_attn_decode_kv4(*[P(MB)] * 5, None, None, s, out, P(2 * MB), None, None, 0, 1, 1, 1, 32, 32, 64, None) == want
    assert lib.sb_attn_key_weight(P(MB), P(2 * MB), None, None, s, out, None, 0, 1, 1, 1, 1, 32, 32, 64, None) == want


# spans of an eviction: what it reads and what it writes
READ, WRITTEN = ("score", "lens", "src0", "src1"), ("score_out", "index", "lens_out", "dst0", "dst1")


def evict(lib, **moved):
    at = {n: (i + 1) * MB for i, n in enumerate(READ + WRITTEN)}
    for n, (to, off) in moved.items():
        at[n] = at[to] + off
    two = lambda a, b: (ctypes.c_void_p * 2)(at[a], at[b])
    # B 4, Hkv 2, 8 rows, room for 8, keep 4: the shortest spans are those of lens and lens_out, 16 bytes
    return lib.sb_attn_evict(P(at["score"]), P(at["lens"]), two("src0", "src1"), two("dst0", "dst1"), (ctypes.c_int * 2)(16, 8), 2, P(at["score_out"]),
                             P(at["index"]), P(at["lens_out"]), 4, 2, 8, 8, 8, 4, 1, None)


@pytest.mark.parametrize("written", WRITTEN)
@pytest.mark.parametrize("other", READ + WRITTEN)
def test_eviction_writes_to_places_of_its_own(lib, written, other):
    if written == other:
        pytest.skip("the same span")
    assert evict(lib, **{written: (other, 0)}) == OVERLAP
    if other not in ("lens", "lens_out"):
        assert evict(lib, **{written: (other, 16)}) == OVERLAP


def test_more_heads_than_a_launch_takes(lib):
    need = lambda B, H, Hkv, scores: lib.sb_attn_decode_kv4_workspace_bytes(B, H, Hkv, 32, 32, 32, scores)
    assert need(1, 16 * 65535, 1, 0) > 0 and need(1, 16 * 65535 + 1, 1, 0) == 0
    assert need(8, 1 << 20, 2048, 1) == 0 and need(8, 1 << 20, 2048, 0) > 0
    args = [P(MB)] * 5 + [None] * 4 + [P(MB), None, P(MB), 1 << 40]
    assert lib.sb_attn_decode_kv4(*args, 1, 16 * 65535 + 1, 1, 32, 32, 32, None) == SHAPE
