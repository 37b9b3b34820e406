"""Decode on a 4-bit cache: the values meet all bits of a weight."""
import numpy as np
import pytest
import torch

from helpers import to64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24            # half a step of fp32, relative


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


def new_cache(B, Hkv, Tcap, d):
    return [torch.full((B, Hkv, Tcap, w), 0xFF, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32, d // 2, d // 32)]


def up32(n):
    return (n + 31) // 32 * 32


def bf16_below(x):
    """x to eight bits, towards zero."""
    unit = 2.0 ** (np.floor(np.log2(x)) - 7)
    return np.floor(x / unit) * unit


# One workgroup a head, spread over the chip, three launches and all keys read (with m); all numbers of copies of a head's column; half as many waves
@pytest.mark.parametrize("want_m", [False, True])
@pytest.mark.parametrize("B,H,Hkv,T,d", [(64, 2, 2, 1, 64), (32, 4, 2, 1, 32), (20, 6, 2, 40, 128), (16, 8, 2, 300, 64), (16, 10, 2, 300, 32), (16, 16, 2, 300, 128),
                                         (16, 24, 2, 300, 64), (8, 40, 2, 300, 64), (4, 8, 2, 3000, 128), (4, 20, 2, 3000, 64), (40, 32, 8, 5000, 32), (300, 2, 2, 600, 64),
                                         (300, 8, 2, 300, 64), (160, 6, 2, 300, 128), (300, 4, 2, 5000, 32), (16, 64, 16, 5000, 64)])
def test_the_output_gets_whole_weights(sb, oracle, B, H, Hkv, T, d, want_m):
    """The nearest key takes A, very nearly 0.6, of the stick, no other key anything (logits of -60), the bias the rest: with values v and -1.5 v, o = (2.5 A - 1.5) v
    is what A differs from 0.6 by, and a bf16 step of it is far below A's last bits.
    Bound: z is exact (three products of few bits), x = z log2(e) off by four roundings, so e by 4 |z| + 2 half steps U, and A by A (1 - A) as much; A and what is left by 8 roundings more each (1 + e, its
    reciprocal, products with what the nearer lanes, tiles and chunks left); o by 4 sums no larger than 1.5; and by half a bf16 step of itself, 2^-8."""
    root, z0 = d ** 0.5, np.log(1.5)
    at = z0 + 4e-4 * np.linspace(-1, 1, B * H).reshape(B, H)
    q1 = bf16_below((z0 * root - 0.01) / 3.0)
    q = torch.zeros(B, H, d, dtype=torch.float64)
    q[..., 1] = q1
    q[..., d - 1] = torch.tensor((at * root - 3.0 * q1) * 4.0)
    q[..., 0] = 15.0 * root
    q = q.bfloat16()
    k = torch.zeros(B, Hkv, T, d)
    k[:, :, :T - 1, 0] = -4.0
    k[:, :, T - 1, 1], k[:, :, T - 1, d - 1] = 3.0, 0.25
    v = torch.where(torch.arange(d) % 3 == 1, -1.0, 1.0).expand(B, Hkv, T, d).contiguous()
    r = (-1.5 * v[0, 0, :1]).expand(H, d).contiguous().bfloat16()
    cache = new_cache(B, Hkv, up32(T), d)
    sb.sb_attn_kv4_store(k.bfloat16().cuda(), v.bfloat16().cuda(), *cache)
    back = sb.sb_attn_kv4_load(*cache, T)
    assert torch.equal(back[0].float().cpu(), k) and torch.equal(back[1].float().cpu(), v)        # (nothing is rounded here)
    got = sb.sb_attn_decode_kv4(q.cuda(), *cache, T=T, r=r.cuda(), want_m=want_m)
    o = to64(got[0] if want_m else got)
    z = (3.0 * to64(q)[..., 1] + to64(q)[..., d - 1] / 4.0) / root
    far = (to64(q)[..., 0] * -4.0) / root
    assert (far < -59).all() and np.abs(z - at).max() < 1e-4
    A = 1.0 / (1.0 + np.exp(-z))
    left = (1.0 - A) * np.exp(-(T - 1) * np.log1p(np.exp(far)))
    ref = (A - 1.5 * left)[..., None] * v[0, 0, 0].double().numpy()
    tol = 2.0 ** -8 * np.abs(ref) + U * (2.5 * A * left * (4 * z + 2) + 8 * (A + 1.5 * left) + 6)[..., None]
    assert np.abs(ref).max() < 5e-4
    worst = np.abs(o - ref) / tol
    print(f"{worst.max():.3f} of the bound")
    assert worst.max() <= 1.0, np.unravel_index(worst.argmax(), worst.shape)
