"""The ends of the 4-bit format's range."""
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
