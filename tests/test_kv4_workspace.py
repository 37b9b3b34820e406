"""What decode on a 4-bit cache and the key weights ask for as workspace (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2410_17980_amd import binding
    return binding.load()


def test_decode_does_not_pay_for_room_in_the_cache(lib):
    """Rows up to T, whatever Tcap is; with scores, and more than one chunk or more than 16 heads a kv head, 4 bytes a query head and row more."""
    need = lib.sb_attn_decode_kv4_workspace_bytes
    for B, H, Hkv, T, d in ((1, 32, 8, 5000, 128), (8, 16, 16, 16384, 64), (2, 40, 2, 700, 32), (70, 16, 16, 4200, 128), (3, 3, 3, 1, 32)):
        cap = (T + 31) // 32 * 32
        for scores in (0, 1):
            least = need(B, H, Hkv, T, cap, d, scores)
            assert 0 < least == need(B, H, Hkv, T, 65536, d, scores) == need(B, H, Hkv, T, 1 << 20, d, scores)
        assert need(B, H, Hkv, T, cap, d, 1) - need(B, H, Hkv, T, cap, d, 0) <= 4 * B * H * cap


def test_decode_in_one_launch_needs_no_room_for_weights(lib):
    need = lib.sb_attn_decode_kv4_workspace_bytes
    for B, H, Hkv, T, d in ((32, 64, 64, 1000, 128), (32, 16, 16, 1800, 64), (1, 12, 4, 333, 128), (64, 64, 4, 700, 32)):
        assert need(B, H, Hkv, T, 65536, d, 1) == need(B, H, Hkv, T, 65536, d, 0) <= 4 * B * H * (d + 4)


def test_key_weights_of_long_prompts_stay_within_two_gigabytes(lib):
    """One number a key from each workgroup, 2^31 bytes of them at a time (or a workgroup a kv head), and two integers a workgroup."""
    need = lib.sb_attn_key_weight_workspace_bytes
    for B, H, Hkv, Tq, T in ((1, 32, 8, 131_072, 131_072), (1, 32, 8, 524_288, 524_288), (16, 32, 32, 65_536, 65_536), (1, 64, 64, 262_144, 524_288), (300, 3, 1, 1, 524_288)):
        assert 0 < need(B, H, Hkv, Tq, T, 128) <= max(2 ** 31, 4 * T * B * Hkv) + 2 ** 20, (B, H, Hkv, Tq, T)
