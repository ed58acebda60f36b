"""The counting attention of paged_counts.py sees a single token that is lost, at any length (the mistakes are planted in the
oracle)."""
import pytest
import torch

import paged_counts as counts
import paged_reference as ref


@pytest.mark.parametrize("t", [1, 33, 1000, 9000, 33333, 70000, 100000])
def test_a_lost_token_or_unit_is_seen(t):
    gen = torch.Generator().manual_seed(t)
    table = torch.zeros(1, 1, dtype=torch.int32)
    c = counts.Counts(gen, table, (t,), 1, 1, 2, 1 << 17)
    good = c.want(0, 0)
    assert (good[0].to(counts.BF).double() - good[0]).abs().le(counts.bar(good[0])).all()
    for lost in ((t - 1,), (t // 2,), range(t // 64 * 32, min(t, t // 64 * 32 + 32))):
        bad = c.want(0, 0, lost=lost)[0].to(counts.BF).double()
        assert (bad - good[0]).abs().gt(counts.bar(good[0])).any(), lost


def test_against_the_definition():
    gen, t_ctx, page = torch.Generator().manual_seed(3), (130, 0, 64, 65), 16
    table = torch.randperm(36, generator=gen).view(4, 9).int()
    c = counts.Counts(gen, table, t_ctx, 36, 2, 3, page, share=0.1)
    sel = torch.tensor([0, 2, 1, 2], dtype=torch.int16).expand(4, 2, 1, 4).contiguous()
    cnt = torch.full((4, 2, 1), 4, dtype=torch.int16)
    cnt[2] = 0
    for s, n in ((None, None), (sel, cnt)):
        o, _ = ref.attn(c.q[:, :, 0], c.k, c.v, table, t_ctx, page, s, n, counts.SCALE)
        for b in range(4):
            for h in range(2):
                assert torch.allclose(o[b, 3 * h:3 * h + 3], c.want(b, h, s, n), rtol=1e-12, atol=1e-12), (b, h)
