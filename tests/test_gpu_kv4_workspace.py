"""Decode on a 4-bit cache in a workspace of just the size that it asks for, with more memory behind it: nothing there changes."""
import pytest
import torch

import test_gpu_cache_forms as forms

pytestmark = pytest.mark.gpu

BEHIND = 1 << 20


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


@pytest.mark.parametrize("want_m", [False, True])
@pytest.mark.parametrize("B,H,Hkv,T,cap,d", [(2, 8, 2, 5000, 20000, 128), (1, 6, 3, 1300, 4096, 64), (3, 40, 2, 700, 8192, 32), (40, 16, 8, 4101, 4160, 32), (2, 34, 2, 6001, 6016, 64),
                                             (30, 8, 8, 900, 65536, 64), (1, 1, 1, 1, 32, 32)])
def test_nothing_behind_the_workspace_changes(sb, B, H, Hkv, T, cap, d, want_m):
    q, k, v = forms.activations(B, H, Hkv, T, d, seed=T)
    small, large = forms.new_cache(B, Hkv, (T + 31) // 32 * 32, d), forms.new_cache(B, Hkv, cap, d)
    for cache in (small, large):
        sb.sb_attn_kv4_store(k, v, *cache)
    got = []
    for cache in (small, large):
        room = cache[0].shape[2]
        n = sb.sb_attn_decode_kv4_workspace_bytes(B, H, Hkv, T, room, d, True)
        memory = torch.full((n + BEHIND,), 0xA5, dtype=torch.uint8, device="cuda")
        score = torch.full((B, Hkv, room), 0.25, device="cuda")
        r = sb.sb_attn_decode_kv4(q, *cache, T=T, score=score, want_m=want_m, workspace=memory[:n])
        assert (memory[n:] == 0xA5).all() and (score[:, :, T:] == 0.25).all()
        got.append((*r[:-1], score[:, :, :T]))
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)
