"""rift_attention_paged at values near the ends of their types' ranges, and in place."""
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


@pytest.mark.parametrize("cache", [torch.float16, torch.float8_e4m3fn], ids=["f16", "e4m3"])
@pytest.mark.parametrize("heads,kv", [(8, 8), (8, 1), (40, 1)])
def test_queries_in_place(heads, kv, cache, cuda, riftlib):
    """The output over its own queries: items of one warp, joined within a CTA and between CTAs, empty rows, blocks of heads."""
    for lens in ([5000, 0, 17, 900], [40] * 50, [30000]):
        c = Case(riftlib, cuda, lens, 32, heads, kv, 64, torch.float16, cache, q_pad=64)
        n, w = len(lens), heads * 64
        want, lse = c.run()
        need = riftlib.attention_paged_workspace_bytes(n, heads, kv, 64)
        ws = torch.empty(need, dtype=torch.uint8, device=cuda)
        got = torch.empty(n, heads, dtype=torch.float32, device=cuda)
        queries = c.q.clone()
        for _ in range(3):
            c.q.copy_(queries)
            riftlib.attention_paged(c.pages, c.q, riftlib.RIFT_F16, w + 64, heads, c.seq_lens, n, c.table, c.table.shape[1], 0, 0.0,
                                    c.q, w + 64, got, ws, need)
            assert torch.equal(c.q, want) and torch.equal(got, lse)
    riftlib.sync_status()
