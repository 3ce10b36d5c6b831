"""What packed rings stand for, number by number."""
import pytest
import torch

from paper_2506_15545_amd import binding as rb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_code_with_the_smallest_factors_and_ordinary_ones(dtype):
    """fp32 holds every value; bf16 those that are multiples of its least step, 2^-133, and of the others the nearest multiple, which
    is 2^-134 off at most.  Packing again stands for what was unpacked."""
    factors = [1, 2, 3, 4, 5, 6, 7, 8, 64, 127, 128, 200, 246]      # scale bytes; 448 times the last is below the types' largest number
    W = 4 * len(factors)
    codes = torch.arange(256, dtype=torch.uint8).view(4, 64).repeat(len(factors), 1).view(1, 1, W, 64)
    scale = torch.tensor(factors, dtype=torch.uint8).repeat_interleave(4).view(1, 1, W, 1).repeat(1, 1, 1, 2)
    want = codes.view(torch.float8_e4m3fn).double() * torch.pow(2.0, scale.double() - 127).repeat_interleave(32, -1)
    kc, ks = codes.view(torch.float8_e4m3fn).cuda(), scale.contiguous().view(torch.float8_e8m0fnu).cuda()
    k, v = rb.rattn_ring_unpack(kc, ks, kc, ks, dtype)
    assert torch.equal(k.nan_to_num(), v.nan_to_num())
    got, nan = k.cpu().double(), torch.isnan(want)
    assert bool((torch.isnan(got) == nan).all())
    step = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133
    held = torch.remainder(want, step) == 0
    assert bool((got == want)[held & ~nan].all()) and float((got - want).abs()[~nan].max()) <= step / 2
    assert bool(held[~nan].all()) == (dtype == torch.float32)
    c, s, _, _ = rb.rattn_ring_pack(k, v)
    again = c.cpu().double() * s.cpu().double().repeat_interleave(32, -1)
    assert bool((again == got)[~nan].all())
