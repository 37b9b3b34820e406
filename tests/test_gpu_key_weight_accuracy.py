"""How exact the key weights are, in units of fp32's roundings: the bounds do not grow with the length (helpers and derivations: test_gpu_cache_accuracy.py)."""
import numpy as np
import pytest
import torch

from helpers import to64
from test_gpu_cache_accuracy import LEAST, U, by_kind, rows_of, sb, steady  # noqa: F401

pytestmark = pytest.mark.gpu


# One unit a workgroup, four, two units a wave, and chunks of keys
@pytest.mark.parametrize("B,H,Hkv,Tq,T,d", [(1, 2, 1, 700, 700, 64), (8, 16, 16, 2048, 2048, 64), (16, 16, 16, 2048, 2048, 32), (2, 64, 8, 4096, 4096, 64), (1, 8, 8, 4096, 4096, 128), (1, 32, 8, 64, 16384, 128),
                                            (1, 4, 4, 1, 524_288, 32), (1, 8, 4, 40, 65_536, 64), (400, 1, 1, 1, 3000, 32)])
def test_key_weights_of_many_small_weights(sb, B, H, Hkv, Tq, T, d):
    """Every query's logits are z: the key at i gets p (1 - p)^(j - i - 1) from the query at j > i.  A weight's bound is that of decode, and a key's sum takes at most 5 sums over lanes, 3 over waves,
    and one for each of the Tq G / 128 workgroups' numbers."""
    G = H // Hkv
    logits = np.array([-16.7, -17.0, -16.62, -13.2])[np.arange(Hkv) % 4]
    q, k, z = steady(T, logits, d, Hkv)
    q = q.repeat_interleave(G, 0)[None, :, None].expand(B, H, Tq, d).contiguous().cuda()
    s = to64(sb.sb_attn_key_weight(q, k.expand(B, Hkv, T, d).contiguous().cuda()))
    p = 1.0 / (1.0 + np.exp(-z))[:, None]
    i, log = np.arange(T)[None], np.log1p(-p)
    first = np.maximum(i + 1, T - Tq)                     # the first query that sees key i
    want = G * np.exp((first - i - 1) * log) * -np.expm1((T - first) * log)
    S = -(T - 1 - i) * log
    rel = (4 * np.abs(z) + 2)[:, None] * U * (1 + S) + 24 * U * (2 + S) + (8 + Tq * G / 128) * U
    err = np.abs(s - want) / (rel * want + 1e-300)
    print(f"{err.max():.3f} of the bound")
    assert err.max() <= 1.0


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,H,Hkv,Tq,T", [(1, 4, 4, 1, 300), (1, 4, 4, 300, 300), (1, 8, 4, 5, 9000), (1, 32, 4, 32, 2000), (27, 24, 8, 150, 150)])
def test_every_key_weight(sb, B, H, Hkv, Tq, T, d):
    q, k = by_kind(B, H, Hkv, Tq, T, d, seed=Tq + T + d)
    s, worst, G = to64(sb.sb_attn_key_weight(q.cuda(), k.cuda())), 0.0, H // Hkv
    for b in range(0, B, 13):
        for h in range(Hkv):
            seen = np.tile(np.arange(T - Tq, T), G)
            A, rel = rows_of(to64(q)[b, h * G:(h + 1) * G].reshape(G * Tq, d), to64(k)[b, h], seen)
            ref = A.sum(0)
            err = np.abs(s[b, h] - ref) / ((rel * A).sum(0) + (8 + Tq * G / 128 + 1) * U * ref + LEAST)
            worst = max(worst, float(err.max()))
    print(f"{worst:.3f} of the bound")
    assert worst <= 1.0
