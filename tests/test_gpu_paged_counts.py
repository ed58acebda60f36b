"""Paged attention on the GPU where every weight is 0 or 1 (paged_counts.py): each token of each unit counts once, with its
own key, by each division of the work and at any length."""
import random

import pytest
import torch

import paged_counts as counts
from test_gpu_paged import dev, n_bad, run_attn, say, shape_of, table_of  # noqa: F401
import paper_2606_04511_amd.sparda as sp

pytestmark = pytest.mark.gpu


def compare(got, c, H, sel=None, cnt=None):
    for b in range(len(c.t_ctx)):
        for h in range(H):
            want = c.want(b, h, sel, cnt)
            far = (got[b, h * c.G:(h + 1) * c.G].double() - want).abs() - counts.bar(want)
            assert (far <= 0).all(), (b, h, int((far > 0).sum()))


def case_of(dev, t_ctx, H, G, page, seed, share=0.5, **kw):  # noqa: F811
    rng, gen = random.Random(seed), torch.Generator().manual_seed(seed)
    table, n_pages = table_of(rng, len(t_ctx), max(t_ctx), page, lens=t_ctx)
    c = counts.Counts(gen, table, t_ctx, n_pages, H, G, page, share)
    shape = shape_of(len(t_ctx), H, G, t_cap=max(t_ctx), **kw)
    return c, shape, sp.SpardaPages(page, table.to(dev), c.k.to(dev), c.v.to(dev)), rng


@pytest.mark.parametrize("case", [
    # t_ctx, kv heads, heads per group, page, share of the tokens that a head attends
    ((2048,), 1, 4, 64, 0.5),                                    # units of one wavefront each
    ((1024,) * 9, 8, 16, 16, 0.02),                              # a few units per wavefront, most of them without a weight
    ((64, 33, 500) * 100, 2, 3, 32, 0.2),                        # a wavefront per row
    ((9000,) + (31, 200, 64) * 40, 2, 2, 128, 0.5),              # the line, rows shared by wavefronts and not
])
def test_units_meet_their_own_keys(dev, case):  # noqa: F811
    """A unit's keys pass through LDS that the units before and behind it use too."""
    t_ctx, H, G, page, share = case
    say("counts", t_ctx[:4], len(t_ctx), H, G, page)
    c, shape, pages, _ = case_of(dev, t_ctx, H, G, page, 7, share)
    t = torch.tensor(t_ctx, dtype=torch.int32)
    compare(run_attn(dev, shape, pages, c.q, t, max(t_ctx), None, None, counts.SCALE), c, H)


def lists_of(c, H, k, rng, order):
    """Sets of up to k blocks: distinct ones in ascending order, or with repeats in any."""
    sel = torch.full((len(c.t_ctx), H, 1, k), -1, dtype=torch.int16)
    cnt = torch.zeros(len(c.t_ctx), H, 1, dtype=torch.int16)
    for b, t in enumerate(c.t_ctx):
        nb = -(-max(t, 0) // 64)
        for h in range(H):
            got = sorted(rng.sample(range(nb), min(nb, k))) if order == "sorted" else [rng.randrange(max(nb, 1)) for _ in range(k)]
            sel[b, h, 0, :len(got)] = torch.tensor(got, dtype=torch.int16)
            cnt[b, h, 0] = len(got)
    return sel, cnt


def run_lists(dev, t_ctx, H, G, k, page, order):  # noqa: F811
    say("lists", t_ctx[:4], len(t_ctx), H, G, k, page, order)
    c, shape, pages, rng = case_of(dev, t_ctx, H, G, page, k, 0.5, k=k)
    sel, cnt = lists_of(c, H, k, rng, order)
    t = torch.tensor(t_ctx, dtype=torch.int32)
    compare(run_attn(dev, shape, pages, c.q, t, max(t_ctx), sel, cnt, counts.SCALE), c, H, sel, cnt)


@pytest.mark.parametrize("case", [
    ((9000,) + tuple(range(0, 620, 20)), 8, 2, 65, 64, "sorted"),       # one list past 128 units per workgroup
    ((30000, 200, 0, 4000) * 8, 8, 1, 400, 32, "sorted"),                # every fourth list long
    ((20000,) + (100, 0, 700) * 5, 2, 16, 300, 128, "repeats"),          # workgroups per row, lists of a few blocks many times over
    ((40000,) + (100, 0, 700) * 21, 2, 4, 300, 128, "sorted"),
])
def test_long_lists_among_short_ones(dev, case):  # noqa: F811
    run_lists(dev, *case)


@pytest.mark.parametrize("case", [
    # t_ctx, kv heads, heads per group: the join takes sixteen wavefronts, four, one
    ((200,) * 30 + (60000,) + (200, 0, -1) * 11, 1, 4),
    ((30000,) + (200, 0) * 32, 4, 4),
    ((100, 0) * 32 + (40000, 700), 2, 16),
    ((50, 0, 64) * 343 + (20000, 1), 1, 16),
    ((9000, 9000, 8000) * 20, 1, 8),
])
def test_one_long_row_on_the_line(dev, case):  # noqa: F811
    t_ctx, H, G = case
    say("line", max(t_ctx), len(t_ctx), H, G)
    c, shape, pages, _ = case_of(dev, t_ctx, H, G, 64, 11)
    t = torch.tensor(t_ctx, dtype=torch.int32)
    compare(run_attn(dev, shape, pages, c.q, t, max(t_ctx), None, None, counts.SCALE), c, H)


@pytest.mark.parametrize("grid,page", [((64, 64), 64), ((32, 16), 16)])
@pytest.mark.parametrize("n_init,n_local", [(1, 2), (0, 1), (4, 32)])
def test_sets_of_the_forced_blocks_alone(dev, grid, page, n_init, n_local):  # noqa: F811
    """A budget of the initial and local blocks only: no key is scored, so none is read and the workspace stays as it is."""
    t_ctx, H, k = (90000, 64 * 40 + 1, 0, 64, 1, 64 * n_local + 1), 2, n_init + n_local
    say("forced", grid, n_init, n_local)
    B, t_max = len(t_ctx), max(t_ctx)
    shape = shape_of(B, H, 1, k, t_max, n_init, n_local, grid)
    table = torch.zeros(B, -(-shape.t_cap // page), dtype=torch.int32, device=dev)
    keys = torch.full((1, H, page // grid[1], 128), float("nan"), dtype=counts.BF, device=dev)
    ws = torch.full((sp.sparda_workspace_size(shape, sp.SPARDA_OP_PAGED_SELECT, 1, t_max - 1),), 0x5A, dtype=torch.uint8, device=dev)
    sel = torch.full((B, H, 1, k), 77, dtype=torch.int16, device=dev)
    cnt = torch.full((B, H, 1), 77, dtype=torch.int16, device=dev)
    sp.sparda_paged_select(shape, sp.SpardaPages(page, table, k_cmp=keys), torch.ones(B, H, 1, 128, dtype=counts.BF, device=dev),
                           torch.tensor(t_ctx, dtype=torch.int32, device=dev), t_max, sel, cnt, ws)
    for b, t in enumerate(t_ctx):
        last = (t - 1) // 64
        want = sorted(set(range(min(n_init, last + 1))) | set(range(max(0, last - n_local + 1), last + 1))) if t > 0 else []
        for h in range(H):
            assert int(cnt[b, h, 0]) == len(want) and sel[b, h, 0].tolist() == want + [-1] * (k - len(want)), (b, h)
    assert (ws == 0x5A).all()


@pytest.mark.parametrize("case", [
    # t_ctx, kv heads, heads per group, page: the longest contexts and the most units per wavefront
    ((70000,), 1, 2, 1024),
    ((33333,), 1, 12, 16),
    ((100001, 99999), 2, 3, 64),
    ((20000, 3, 40000, 17) * 3, 2, 8, 256),
    ((65535, 0, 1, 65537), 1, 1, 65536),
])
def test_every_token_of_long_contexts(dev, case):  # noqa: F811
    t_ctx, H, G, page = case
    say("long", t_ctx, H, G, page)
    c, shape, pages, _ = case_of(dev, t_ctx, H, G, page, 5)
    t = torch.tensor(t_ctx, dtype=torch.int32)
    compare(run_attn(dev, shape, pages, c.q, t, max(t_ctx), None, None, counts.SCALE), c, H)


@pytest.mark.parametrize("case", [
    ((100000,), 1, 2, 1000, 64, "sorted"),
    ((100000,), 1, 2, 1000, 16, "repeats"),
    ((90001,), 2, 16, 1407, 256, "sorted"),          # every block of the context
    ((40000, 39000), 4, 4, 500, 128, "sorted"),
])
def test_every_token_of_long_lists(dev, case):  # noqa: F811
    run_lists(dev, *case)
