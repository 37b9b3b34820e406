"""How exact decode on a 4-bit cache and the key weights are, in units of fp32's roundings: the bounds do not grow with the length."""
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


def steady(T, logits, d, Hkv):
    """k [1,Hkv,T,d] and q rows [len(logits),d] whose logits are the same for all keys, one product each; and what they are."""
    k = torch.zeros(1, Hkv, T, d)
    k[..., 3] = -4.0
    q = torch.zeros(len(logits), d)
    q[:, 3] = torch.tensor(logits) * d ** 0.5 / -4.0
    q = q.bfloat16()
    return q, k.bfloat16(), to64(q)[:, 3] * -4.0 / d ** 0.5


# logits at which e is half a last bit of 1 and just above, where few of its bits would be left beside 1, and where the stick is used up half-way
@pytest.mark.parametrize("T", [1500, 65_536, 524_288])
@pytest.mark.parametrize("d,H", [(32, 4), (64, 8), (128, 32)])
@pytest.mark.parametrize("want_m", [False, True])
def test_decode_of_many_small_weights(sb, T, d, H, want_m):
    """The weights of a row whose logits are all z: p (1 - p)^n for the key n places before the last, and m = T log(1 - p).
    Bound: as above, e is off by ze = (4 |z| + 2) U.  What keys take adds up, S = -log of what is left: a weight is off by ze (1 + S) for its own e and those before it, and by 24 U (2 + S)
    for the 24 roundings of its own 32 keys, of the product over all before, taken in more bits, and of reading it (at most so much of what each takes off the stick); m by ze and 40 roundings of itself.  o: its bf16 step, and the same."""
    Hkv = 2
    logits = np.array([-16.7, -17.0, -16.62, -13.2])[np.arange(H) % 4]
    q, k, z = steady(T, logits, d, Hkv)
    cache = new_cache(1, Hkv, up32(T), d)
    v = torch.ones(1, Hkv, T, d, dtype=torch.bfloat16)
    sb.sb_attn_kv4_store(k.cuda(), v.cuda(), *cache)
    got = sb.sb_attn_decode_kv4(q[None].cuda(), *cache, T=T, score_out=torch.zeros(1, Hkv, up32(T), device="cuda"), want_m=want_m)
    p = 1.0 / (1.0 + np.exp(-z))[:, None]
    n = np.arange(T)[::-1]
    S = -n * np.log1p(-p)
    A = p * np.exp(-S)
    ze = (4 * np.abs(z) + 2)[:, None] * U
    rel = ze * (1 + S) + 24 * U * (2 + S)
    sums = lambda x: x.reshape(Hkv, H // Hkv, T).sum(1)
    s = to64(got[-1])[0, :, :T]
    err = np.abs(s - sums(A)) / (sums(rel * A) + (H // Hkv + 1) * U * sums(A))
    end = T * -np.log1p(-p[:, 0])                         # S behind all keys
    ref = -np.expm1(-end)
    o = np.abs(to64(got[0])[0] - ref[:, None]).max(-1) / (ref * (2.0 ** -8 + (ze[:, 0] + 24 * U) * (2 + end)))
    print(f"scores {err.max():.3f}, o {o.max():.3f} of the bound")
    if want_m:
        m = np.abs(to64(got[1])[0] + end) / ((ze[:, 0] + 40 * U) * end)
        print(f"m {m.max():.3f}")
        assert m.max() <= 1.0, m
    assert err.max() <= 1.0 and o.max() <= 1.0


def rows_of(q, k, extra):
    """Weights of queries q [n,d] against keys k [T,d], query t seeing the first extra[t], [n,T], and bounds of their relative errors: a logit is off by d roundings of its products and sums and by the four of
    its scaling, e by that and its own, and the rest as in test_decode_of_many_small_weights."""
    d = q.shape[1]
    z = q @ k.T / np.sqrt(d)
    sees = np.arange(k.shape[0]) < np.asarray(extra)[:, None]
    sp = np.where(sees, np.logaddexp(0.0, z), 0.0)
    S = sp[:, ::-1].cumsum(-1)[:, ::-1] - sp              # of the keys behind
    ze = (d * (np.abs(q) @ np.abs(k).T) / np.sqrt(d) + 4 * np.abs(z) + 2) * U
    return np.where(sees, np.exp(z - np.logaddexp(0.0, z) - S), 0.0), ze.max(-1, keepdims=True) * (1 + S) + 24 * U * (2 + S)


def by_kind(B, H, Hkv, Tq, T, d, seed):
    """By kv head in turn: N(0,1), k * 3, k * 12 (logits of tens), and logits around -6."""
    g = torch.Generator().manual_seed(seed)
    q, k = torch.randn(B, H, Tq, d, generator=g), torch.randn(B, Hkv, T, d, generator=g)
    far, G = (6.0 * d ** 0.5) ** 0.5, H // Hkv
    for h in range(Hkv):
        if h % 4 in (1, 2):
            k[:, h] *= (3.0, 12.0)[h % 4 - 1]
        elif h % 4 == 3:
            k[:, h, :, d - 1] = -far
            q[:, h * G:(h + 1) * G, :, d - 1] = far
    return q.bfloat16(), k.bfloat16()


LEAST = 2.0 ** -100       # (weights below that are left to the bounds of the other tests: subnormal numbers are near)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,H,Hkv,T", [(1, 4, 4, 200), (2, 8, 4, 1500), (1, 4, 4, 20_000), (1, 64, 4, 3000), (80, 16, 8, 400)])
@pytest.mark.parametrize("want_m", [False, True])
def test_every_weight_of_decode(sb, B, H, Hkv, T, d, want_m):
    """Scores from nothing: each is its weight, relative to itself, however small.  m: what e is off by, and 40 roundings, of itself."""
    q, k = by_kind(B, H, Hkv, 1, T, d, seed=T + d)
    cache = new_cache(B, Hkv, up32(T), d)
    sb.sb_attn_kv4_store(k.cuda(), k.cuda(), *cache)
    k4 = to64(sb.sb_attn_kv4_load(*cache, T)[0])
    got = sb.sb_attn_decode_kv4(q[:, :, 0].contiguous().cuda(), *cache, T=T, score_out=torch.zeros(B, Hkv, up32(T), device="cuda"), want_m=want_m)
    s, worst, G = to64(got[-1])[:, :, :T], 0.0, H // Hkv
    for b in range(0, B, 13):
        for h in range(Hkv):
            A, rel = rows_of(to64(q)[b, h * G:(h + 1) * G, 0], k4[b, h], [T] * G)
            ref = A.sum(0)
            err = np.abs(s[b, h] - ref) / ((rel * A).sum(0) + (G + 1) * U * ref + LEAST)
            worst = max(worst, float(err.max()))
            for g in range(h * G, (h + 1) * G if want_m else 0):
                m = -np.logaddexp(0.0, k4[b, h] @ to64(q)[b, g, 0] / d ** 0.5).sum()
                assert abs(to64(got[1])[b, g] - m) <= (rel[g - h * G, -1] + 40 * U) * abs(m), (b, g)         # (rel behind no key: ze + 48 U)
    print(f"{worst:.3f} of the bound")
    assert worst <= 1.0
