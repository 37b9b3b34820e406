"""Key weights of prompts whose workgroups' numbers are more than the workspace holds at a time."""
import numpy as np
import pytest
import torch

from helpers import to64
from test_gpu_cache_accuracy import U, by_kind, sb, steady  # noqa: F401

pytestmark = pytest.mark.gpu

BEHIND = 1 << 20


def call(sb, q, k, **kw):
    """In a workspace of just the size asked for, with more memory behind it."""
    B, H, Tq, d = q.shape
    n = sb.sb_attn_key_weight_workspace_bytes(B, H, k.shape[1], Tq, kw.get("T") or k.shape[2], d)
    memory = torch.full((n + BEHIND,), 0xA5, dtype=torch.uint8, device="cuda")
    out = sb.sb_attn_key_weight(q, k, workspace=memory[:n], **kw)
    assert (memory[n:] == 0xA5).all()
    return out


@pytest.mark.parametrize("B,H,Hkv,T,d", [(1, 40, 40, 65_536, 32), (5, 12, 6, 65_536, 64)])
def test_a_prompt_is_its_halves(sb, B, H, Hkv, T, d):
    """What all queries give is what the first half's and the second half's give, each a call of its own: equal but for the sums' order, (8 + T G / 128) U of the sum for either side, and for the queries'
    weights, which come of other tiles, 24 U (2 + S) of each with S up to the 88 that fp32 holds.  The whole call: from scores, in place, of entries of different lengths."""
    q, k = (t.cuda() for t in by_kind(B, H, Hkv, T, T, d, seed=B))
    half, G = T // 2, H // Hkv
    lens = [T] + [T - 1000 * b - 3 for b in range(1, B)]
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
    was = torch.rand(B, Hkv, T, generator=torch.Generator().manual_seed(1)).cuda()
    whole = call(sb, q, k, lens=ld, qlens=ld, score=was.clone())
    one = call(sb, q[:, :, :half].contiguous(), k[:, :, :half].contiguous())
    two = torch.zeros_like(was)
    for b in range(B):
        two[b, :, :lens[b]] = call(sb, q[b:b + 1, :, half:lens[b]].contiguous(), k[b:b + 1, :, :lens[b]].contiguous())[0]
    for b in range(B):
        n = lens[b]
        want = two[b].double()
        want[:, :half] += one[b]
        got = whole[b].double() - was[b]
        tol = (2 * (8 + T * G / 128) + 2 * 24 * 90) * U * want + 2 * U * whole[b]
        assert ((got - want).abs()[:, :n] <= tol[:, :n]).all(), b
        assert torch.equal(whole[b, :, n:], was[b, :, n:])


def test_against_the_formula(sb):
    """Logits alike, T = 131072: bounds and formula of test_gpu_key_weight_accuracy.py."""
    T, d, Hkv, G = 131_072, 32, 8, 2
    q, k, z = steady(T, np.array([-16.7, -17.0, -16.62, -13.2])[np.arange(Hkv) % 4], d, Hkv)
    q = q.repeat_interleave(G, 0)[None, :, None].expand(1, Hkv * G, T, d).contiguous().cuda()
    s = to64(call(sb, q, k.cuda()))
    p = 1.0 / (1.0 + np.exp(-z))[:, None]
    log, n = np.log1p(-p), T - 1 - np.arange(T)[None]
    want = G * -np.expm1(n * log)
    S = -n * log
    rel = (4 * np.abs(z) + 2)[:, None] * U * (1 + S) + 24 * U * (2 + S) + (8 + T * G / 128) * U
    assert (np.abs(s - want) <= rel * want + 1e-300).all()
