"""The ends of the 4-bit format's range, and keys that no stick is left for."""
import pytest
import torch

import test_gpu_cache_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2410_17980_amd import binding
    binding.load(build_if_missing=False)
    return binding


def test_every_scale_and_code(sb, oracle):
    """Loaded as bf16 has them: subnormal numbers at the lower end, infinity where 4 or 6 times the scale is 2^128 and more, NaN at 255."""
    scales = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(1, 1, 256, 1)
    codes = torch.arange(32) % 16
    packed = (codes[0::2] | codes[1::2] << 4).to(torch.uint8).expand(1, 1, 256, 16).contiguous()
    got, again = sb.sb_attn_kv4_load(packed.cuda(), scales.cuda(), packed.cuda(), scales.cuda(), 256)
    want = torch.tensor(oracle.kv4_values(codes.numpy(), scales.numpy())).float().to(torch.bfloat16)       # (fp32 has all of them but those beyond its range)
    assert torch.equal(got.cpu().view(torch.int16)[:, :, :255], want.view(torch.int16)[:, :, :255])
    assert got[:, :, 255].isnan().all() and torch.equal(got.view(torch.int16), again.view(torch.int16))


def test_largest_magnitudes(sb):
    """Up to 1.75 * 2^127 a row comes back finite; beyond, its largest magnitudes are 4 * 2^126, which bf16 has as infinity."""
    x = torch.zeros(1, 1, 3, 32)
    x[0, 0, 0, :3] = torch.tensor([1.75, -1.0, 0.5]) * 2.0 ** 127
    x[0, 0, 1, :3] = torch.tensor([1.9921875, -1.5, 0.5]) * 2.0 ** 127
    x[0, 0, 2, :3] = torch.tensor([-1.7578125, 1.75, 1.0]) * 2.0 ** 127
    cache = forms.new_cache(1, 1, 32, 32)
    sb.sb_attn_kv4_store(x.bfloat16().cuda(), x.bfloat16().cuda(), *cache)
    k, v = sb.sb_attn_kv4_load(*cache, 3)
    inf, unit = float("inf"), 2.0 ** 126
    assert torch.equal(k, v) and k[0, 0, :, :3].double().tolist() == [[3 * unit, -2 * unit, unit], [inf, -3 * unit, unit], [-inf, inf, 2 * unit]]
    assert not k[0, 0, :, 3:].any()


# one launch (a few workgroups, and more than the chip holds), spread, three launches
@pytest.mark.parametrize("want_m", [False, True])
@pytest.mark.parametrize("B,H,Hkv,T", [(1, 4, 2, 300), (300, 4, 2, 300), (2, 4, 2, 2500), (40, 8, 4, 5000)])
def test_finite_keys_behind_a_used_up_stick_change_nothing(sb, B, H, Hkv, T, want_m):
    """The nearest 12 keys, logits of 40, leave 2^-690 of the stick: other rows behind them make no bit of o another one, m of its own keys apart, and get weights of 2^-126 at most."""
    d = 64
    q, k, v = forms.activations(B, H, Hkv, T, d, seed=B + T)
    k[:, :, T - 12:] = 0.0
    k[:, :, T - 12:, 0] = 4.0
    q[..., 0] = 80.0
    k[:, :, :T - 12, 0] = 0.0
    got = []
    for sign in (1.0, -2.0):
        cache = forms.new_cache(B, Hkv, (T + 31) // 32 * 32, d)
        other = torch.where(torch.arange(T, device="cuda")[:, None] < T - 12, sign, 1.0)
        sb.sb_attn_kv4_store((k * other).bfloat16(), (v * other).bfloat16(), *cache)
        got.append(sb.sb_attn_decode_kv4(q, *cache, T=T, score_out=torch.zeros(B, Hkv, cache[0].shape[2], device="cuda"), want_m=want_m))
    (a, b) = got
    assert torch.isfinite(a[0]).all() and torch.equal(a[0], b[0]) and torch.equal(a[-1][:, :, T - 12:], b[-1][:, :, T - 12:])
    assert (a[-1][:, :, T - 1] > 0.99 * H // Hkv).all() and max(float(x[-1][:, :, :T - 12].max()) for x in got) <= (H // Hkv) * 2.0 ** -126
    if want_m:
        assert torch.isfinite(a[1]).all() and (a[1] < -470).all()
