"""rift_attention_paged at values near the ends of their types' ranges."""
import pytest
import torch

from test_gpu_attention_paged import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [4, 32])
def test_large_bf16_values(heads, cuda, riftlib):
    """Values whose weighted sums fp32 holds (333 of at most 2^118, below 2^127), with weights of one and less."""
    c = Case(riftlib, cuda, [333, 64, 1, 0], 16, heads, 2, 128, torch.bfloat16, torch.bfloat16)
    c.v.clamp_(-8, 8).mul_(2.0 ** 115)
    c.spoil_tails()
    out, lse = c.run()
    assert bool(torch.isfinite(out).all())
    c.check(out, lse)
    c = Case(riftlib, cuda, [5000], 64, heads, 2, 64, torch.bfloat16, torch.bfloat16)  # cut over CTAs
    c.v.clamp_(-8, 8).mul_(2.0 ** 111)
    out, lse = c.run()
    c.check(out, lse)
    riftlib.sync_status()
