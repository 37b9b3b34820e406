"""Decode on a 4-bit cache where a call has more (entry, kv head, block of query heads) workgroups than leave a head two chunks: 1025 and more, on caches that
are beyond what the near launch takes alone where fewer are."""
import pytest
import torch

import test_gpu_cache_forms as forms
from helpers import nan_bytes

pytestmark = pytest.mark.gpu

SHAPES = [(33, 32, 32, 2100, 32), (129, 16, 8, 2049, 64), (65, 144, 8, 2100, 32), (140, 128, 1, 2800, 32), (128, 144, 1, 4000, 32), (103, 160, 10, 4500, 32)]


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


@pytest.mark.parametrize("want_m", [False, True])
@pytest.mark.parametrize("B,H,Hkv,T,d", SHAPES)
def test_against_the_oracle(sb, oracle, B, H, Hkv, T, d, want_m):
    forms.test_decode_of_many_heads(sb, oracle, B, H, Hkv, T, d, want_m)


@pytest.mark.parametrize("B,H,Hkv,T,d", SHAPES)
def test_every_output_is_written(sb, B, H, Hkv, T, d):
    """Into outputs and a workspace that hold NaN, with and without m and scores; entries alike, so every one gets what the first gets."""
    q, k, v = forms.activations(1, H, Hkv, T, d, seed=T)
    q = q.expand(B, -1, -1).contiguous()
    cap = (T + 31) // 32 * 32
    cache = forms.new_cache(1, Hkv, cap, d)
    sb.sb_attn_kv4_store(k, v, *cache)
    cache = [t.expand(B, -1, -1, -1).contiguous() for t in cache]
    for scores in (False, True):
        for want_m in (False, True):
            nan = lambda *s, t=torch.float32: torch.full(s, float("nan"), dtype=t, device="cuda")
            o, m, s = nan(B, H, d, t=torch.bfloat16), nan(B, H), nan(B, Hkv, cap)
            ws = nan_bytes(sb.sb_attn_decode_kv4_workspace_bytes(B, H, Hkv, T, cap, d, scores))
            sb.sb_attn_decode_kv4(q, *cache, T=T, o=o, m=m if want_m else None, score_out=s if scores else None, workspace=ws)
            assert torch.isfinite(o).all() and torch.equal(o, o[:1].expand_as(o))
            if want_m:
                assert torch.isfinite(m).all() and torch.equal(m, m[:1].expand_as(m)) and (m < 0).all()
            if scores:
                s = s[:, :, :T]
                assert torch.isfinite(s).all() and torch.equal(s, s[:1].expand_as(s)) and (s.sum(-1) > 0.99).all()
