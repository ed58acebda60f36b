"""The operators over trees of drafted tokens where their results are most delicate, against the definitions in
float64 (tree_reference.py)."""
import random

import pytest
import torch

import paper_2606_04511_amd.sparda as sp
import tree_reference as ref
from test_gpu_tree import (ATTN, D, L, NAN, attn_inputs, check_verify, dev, exact_rows, run_attn, say,  # noqa: F401
                           shape_of, trees, verify_inputs, workspace)

pytestmark = pytest.mark.gpu


# ---- attention: the last block of the largest cache ------------------------------------------------------

LAST = [
    # nodes, group, entries per list, one list: 16 columns; 32; two tiles of 32; 64 and 128 of wavefronts that share the
    # blocks (the split of the work goes by the entries that lists may hold, not by those they hold)
    (1, 4, 6, False),
    (8, 4, 6, False),
    (9, 4, 8192, True),
    (9, 4, 8192, False),
    (17, 4, 8192, False),
]


@pytest.mark.parametrize("case", range(len(LAST)))
def test_attn_last_block_of_the_largest_cache(dev, case):  # noqa: F811
    """32768 blocks are the most that a cache can have; the last one, number 32767, is a block as any other."""
    n, G, k, shared = LAST[case]
    say("tree attention at 2097152 tokens", LAST[case])
    gen, rng = torch.Generator().manual_seed(case), random.Random(case)
    t_cap = 32768 * L
    t = t_cap - n  # the last block holds 64 - n tokens
    s = shape_of(1, 1, G, k, t, n, t_cap=t_cap)
    blocks = [0, 100, 30720, 32766, 32767]
    rows = torch.cat([torch.arange(j * L, min(j * L + L, t)) for j in blocks])
    caches = []
    for _ in range(2):  # NaN in what no list names and from t on
        x = torch.full((1, 1, t_cap, D), NAN, dtype=torch.bfloat16, device=dev)
        x[0, 0, rows.to(dev)] = torch.randn(len(rows), D, generator=gen).to(torch.bfloat16).to(dev)
        caches.append(x)
    q, kt, vt = (torch.randn(1, h, n, D, generator=gen).to(torch.bfloat16) for h in (G, 1, 1))
    parent = trees(rng, 1, n, "wide")
    ns = 1 if shared else n
    sel, cnt = torch.full((1, 1, ns, k), -1, dtype=torch.int16), torch.full((1, 1, ns), 5, dtype=torch.int16)
    for i in range(ns):
        sel[0, 0, i, :5] = torch.tensor(rng.sample(blocks, 5), dtype=torch.int16)
        cnt[0, 0, i] = 5 if i % 3 < 2 else 3
    o = torch.full(q.shape, NAN, dtype=torch.bfloat16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, t))
    sp.sparda_tree_attn(s, q.to(dev), n, torch.tensor([t], dtype=torch.int32, device=dev), t, parent.to(dev), *caches,
                        kt.to(dev), vt.to(dev), ns, sel.to(dev), cnt.to(dev), ref.SCALE, o, ws)
    torch.cuda.synchronize()
    want, w = ref.attn(q, *(x.cpu() for x in caches), kt, vt, [t], parent, sel, cnt, ref.SCALE)
    assert not torch.isnan(want).any()
    off = (o.cpu().double() - want).abs()
    assert bool((off <= ref.attn_bar(want, w)).all())


# ---- attention: NaN in what a node attends ------------------------------------------------------------------

# nodes, group, kv heads, batch, entries per list, t: 16 and 32 columns with splits and without, the form whose wavefronts
# share the blocks (lists that may hold many entries) with splits, tiles of 32 without splits, the shared form without
SPREAD = [
    (5, 3, 1, 2, 6, 700),
    (7, 4, 2, 2, 8, 1500),
    (3, 4, 64, 4, 6, 700),
    (8, 4, 64, 4, 6, 700),
    (13, 3, 1, 1, 9000, 600000),
    (40, 4, 64, 4, 40, 2600),
    (16, 4, 64, 4, 40, 2600),
]


def spread_inputs(dev, case):  # noqa: F811
    n, G, H, B, k, t = SPREAD[case]
    gen, rng = torch.Generator(device=dev).manual_seed(case), random.Random(case)
    s = shape_of(B, H, G, k, t, n)
    mk = lambda *size: torch.randn(*size, generator=gen, device=dev, dtype=torch.bfloat16)  # noqa: E731
    q, kk, vv = mk(B, H * G, n, D), mk(B, H, s.t_cap, D), mk(B, H, s.t_cap, D)
    kt, vt = mk(B, H, n, D), mk(B, H, n, D)
    parent = trees(rng, B, n, "wide")
    nb, some = -(-t // L), 5
    sel = torch.full((B, H, n, k), -1, dtype=torch.int16, device=dev)
    sel[..., :some] = torch.rand(B, H, n, nb, generator=gen, device=dev).topk(some, dim=3).indices.to(torch.int16)
    cnt = torch.full((B, H, n), some, dtype=torch.int16, device=dev)
    return s, n, [t - 64 * b for b in range(B)], q, parent, kk, vv, kt, vt, sel, cnt


def spread_call(dev, x):  # noqa: F811
    s, n, t_ctx, q, parent, kk, vv, kt, vt, sel, cnt = x
    t = torch.tensor(t_ctx, dtype=torch.int32, device=dev)
    o = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, max(t_ctx)))
    sp.sparda_tree_attn(s, q, n, t, max(t_ctx), parent.to(dev), kk, vv, kt, vt, n, sel, cnt, ref.SCALE, o, ws)
    torch.cuda.synchronize()
    return o


@pytest.mark.parametrize("what", ["query", "context key", "drafted key"])
@pytest.mark.parametrize("case", range(len(SPREAD)))
def test_attn_nan_reaches_those_that_attend_it(dev, case, what):  # noqa: F811
    """A NaN in a node's query, or in a key that it attends, makes that node's output NaN, whatever the number of groups;
    the other nodes' outputs stay as they are, bit for bit."""
    say("tree attention, NaN in a", what, SPREAD[case])
    x = spread_inputs(dev, case)
    s, n, t_ctx, q, parent, kk, vv, kt, vt, sel, cnt = x
    G = s.group_size
    plain = spread_call(dev, x)
    assert not torch.isnan(plain).any()
    bad = torch.zeros(q.shape[:3], dtype=torch.bool)
    for b in range(s.batch):
        up = ref.paths(parent[b].tolist())
        for h in {0, s.n_kv_heads // 2}:
            node = (b + h) % n
            if what == "query":
                q[b, h * G + G - 1, node, 5] = NAN
                bad[b, h * G + G - 1, node] = True
            elif what == "drafted key":
                kt[b, h, node, 77] = NAN
                for i in range(n):
                    bad[b, h * G:h * G + G, i] = node in up[i]
            else:  # the last token of the context that the node's first entry holds
                j = int(sel[b, h, node, 0])
                tok = min(j * L + L, t_ctx[b]) - 1
                if tok < j * L:
                    continue
                kk[b, h, tok, 0] = NAN
                for i in range(n):
                    bad[b, h * G:h * G + G, i] = j in sel[b, h, i, :int(cnt[b, h, i])].tolist()
    assert bad.any()
    got = spread_call(dev, x)
    seen = torch.isnan(got).cpu()
    assert torch.equal(seen.all(3), bad) and torch.equal(seen.any(3), bad)
    keep = ~bad.to(dev)
    assert torch.equal(got[keep].view(torch.int16), plain[keep].view(torch.int16))


# ---- attention: one list, many columns -------------------------------------------------------------------------

ONE_LIST = [
    # nodes, group, kv heads, batch, t: 160 columns of 256 with splits; 1024 in four tiles with splits; 256 of 256 in
    # more workgroups than CUs; 18 of 32 there; 33 of 64
    (40, 4, 12, 5, 900),
    (64, 16, 3, 3, 5000),
    (64, 4, 64, 4, 300),
    (9, 2, 128, 4, 300),
    (11, 3, 64, 4, 300),
]


@pytest.mark.parametrize("case", range(len(ONE_LIST)))
def test_attn_one_list_for_many_columns(dev, case):  # noqa: F811
    n, G, H, B, t = ONE_LIST[case]
    say("tree attention, one list", ONE_LIST[case])
    gen, rng = torch.Generator(device=dev).manual_seed(case), random.Random(case)
    k = 7
    s = shape_of(B, H, G, k, t, n)
    mk = lambda *size: torch.randn(*size, generator=gen, device=dev, dtype=torch.bfloat16)  # noqa: E731
    q, kk, vv, kt, vt = mk(B, H * G, n, D), mk(B, H, s.t_cap, D), mk(B, H, s.t_cap, D), mk(B, H, n, D), mk(B, H, n, D)
    t_ctx = [t - 70 * b for b in range(B)]
    parent = trees(rng, B, n, "wide", pad=[(B - 1, n - 2, n)])
    nb = -(-t // L)
    sel = torch.full((B, H, 1, k), -1, dtype=torch.int16, device=dev)
    some = min(nb, k)
    sel[..., :some] = torch.rand(B, H, 1, nb, generator=gen, device=dev).topk(some, dim=3).indices.to(torch.int16)
    cnt = torch.randint(0, some + 1, (B, H, 1), generator=gen, device=dev).to(torch.int16)
    o = torch.full(q.shape, NAN, dtype=torch.bfloat16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, t))
    sp.sparda_tree_attn(s, q, n, torch.tensor(t_ctx, dtype=torch.int32, device=dev), t, parent.to(dev), kk, vv, kt, vt,
                        1, sel, cnt, ref.SCALE, o, ws)
    torch.cuda.synchronize()
    assert not torch.isnan(o).any()
    for h in {0, H // 2, H - 1}:
        x = [y[:, h:h + 1].cpu() for y in (kk, vv, kt, vt, sel, cnt)]
        want, w = ref.attn(q[:, h * G:(h + 1) * G].cpu(), *x[:4], t_ctx, parent, *x[4:], ref.SCALE)
        off = (o[:, h * G:(h + 1) * G].cpu().double() - want).abs()
        assert bool((off <= ref.attn_bar(want, w)).all())


# ---- attention: weights that must cancel --------------------------------------------------------------------

def fine_bar(o, w, z, terms):
    """How far a bf16 result may be whose weights are held to 2^-16: a logit q . k of bf16 values is a float32 sum of 128
    exact products (at most 129 roundings of 2^-23 of z, the largest sum |q k| scale; a rounding each for the scale, its
    constant, the subtraction and the exponential: 2^-21 of z and 2^-22), which moves a weight by as much of itself,
    numerator and normaliser alike; the weight's two bf16 parts leave 2^-16 of it; sums of `terms` float32 numbers
    (2^-23 each); the division (2^-22) and the bf16 rounding of the result (2^-8 of it and of the error)."""
    e = 2 * (129 * 2.0 ** -23 * z + 2.0 ** -21 * z + 2.0 ** -22) + 2.0 ** -16 + 2 * terms * 2.0 ** -23
    return (e * w) * (1 + 2.0 ** -8) + (2.0 ** -8 + 2.0 ** -22) * o.abs() + 2.0 ** -133


@pytest.mark.parametrize("case", [1, 4, 5, 6, 8, 9, 10])
def test_attn_weights_keep_their_bits(dev, case):  # noqa: F811
    """Small logits, so that the float32 scores are off by little, and outputs near zero, where the rounding of the
    result hides nothing: what is left is how the weights are held for the product with V."""
    say("tree attention, weights' bits", ATTN[case])
    x = list(attn_inputs(ATTN[case], 90 + case))
    x[4] = (x[4].float() / 8).to(torch.bfloat16)
    s, t_max, t_ctx, n, q, k, v, kt, vt, parent, sel, cnt = x
    G = s.group_size
    rows = [torch.cat((k, kt), 2).float().abs()[:, h // G] for h in range(q.shape[1])]
    z = max(float((q[:, h].float().abs() @ rows[h].transpose(1, 2)).max()) for h in range(q.shape[1])) * ref.SCALE
    want, w = ref.attn(q, k, v, kt, vt, t_ctx, parent, sel, cnt, ref.SCALE)
    terms = 64 * sel.shape[3] + n + 64
    off = (run_attn(dev, x).double() - want).abs()
    worst = float((off / fine_bar(want, w, z, terms)).max())
    say(f"  logits up to {z:.2f}, worst error {worst:.3f} of the bar")
    assert worst <= 1.0


# ---- select: the smallest cache of compressed keys -----------------------------------------------------------

SMALL_KC = [
    # t_ctx per sequence, nodes, kv heads, k, n_init, n_local, grid
    ((4096,), 1, 1, 40, 1, 32, (64, 64)),
    ((4096, 3000, 2111), 8, 2, 40, 1, 32, (64, 64)),
    ((9000, 8192), 64, 1, 12, 0, 5, (64, 64)),
    ((4000, 3999), 5, 2, 9, 1, 2, (32, 16)),
    ((4111, 4111), 33, 1, 50, 2, 40, (32, 16)),
    ((2000,), 20, 3, 12, 0, 9, (32, 16)),
]


@pytest.mark.parametrize("case", range(len(SMALL_KC)))
def test_select_with_the_smallest_key_cache(dev, case):  # noqa: F811
    """nc_cap is one more than the last window that can be scored; one less is refused.  The keys end with the tensor."""
    t_ctx, n, H, k, n_init, n_local, grid = SMALL_KC[case]
    say("tree select, smallest key cache", SMALL_KC[case])
    gen, rng = torch.Generator().manual_seed(case), random.Random(case)
    B, t_max, (l, st) = len(t_ctx), max(t_ctx), grid
    last = min((t_max - l) // st, (((t_max + n - 1) // L - n_local + 1) * L - 1) // st)
    s = shape_of(B, H, 1, k, t_max, n, n_init, n_local, grid)
    assert last + 1 < s.nc_cap
    s.nc_cap = last + 1
    f, kc = exact_rows(gen, B, H, n, D), exact_rows(gen, B, H, last + 1, D)
    parent = trees(rng, B, n, "wide" if case % 2 else "chain")
    want = ref.select(f, kc, t_ctx, parent, k, n_init, n_local, grid)
    sel = torch.full((B, H, n, k), 99, dtype=torch.int16, device=dev)
    cnt = torch.full((B, H, n), 99, dtype=torch.int16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, n, t_max))
    args = (f.to(dev), n, torch.tensor(t_ctx, dtype=torch.int32, device=dev), t_max, parent.to(dev), kc.to(dev), sel, cnt, ws)
    sp.sparda_tree_select(s, *args)
    torch.cuda.synchronize()
    assert torch.equal(sel.cpu(), want[0]) and torch.equal(cnt.cpu(), want[1])
    s.nc_cap = last
    with pytest.raises(sp.SpardaError) as ei:
        sp.sparda_tree_select(s, *args)
    assert ei.value.status == sp.SPARDA_ERR_INVALID_ARG


# ---- select: a window that straddles the end of the context ------------------------------------------------------

@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("t", [1024 + x for x in (0, 1, 7, 15, 16, 17, 48, 63)])
def test_select_windows_that_straddle_the_context(dev, t, flat):  # noqa: F811
    """On the (32, 16) grid the last window of a candidate block may end past the context: nodes deep enough to have that
    block as a candidate (50 to 64 of a chain, t % 64 in 1 .. 15) score it by its other windows.  What the cache holds
    there would win every comparison."""
    grid, n, H, k = (32, 16), 64, 2, 6
    say("tree select, straddling windows", t, flat)
    gen, rng = torch.Generator().manual_seed(t), random.Random(t)
    s = shape_of(2, H, 1, k, t, n, 1, 2, grid)
    f, kc = exact_rows(gen, 2, H, n, D).abs(), exact_rows(gen, 2, H, s.nc_cap, D)
    if flat:
        kc.zero_()
    t_ctx = (t, t - 128)
    parent = trees(rng, 2, n, "chain")
    want = ref.select(f, kc, t_ctx, parent, k, 1, 2, grid)
    for b in range(2):
        kc[b, :, (t_ctx[b] - 32) // 16 + 1:] = 100.0
    sel = torch.full((2, H, n, k), 99, dtype=torch.int16, device=dev)
    cnt = torch.full((2, H, n), 99, dtype=torch.int16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, n, t))
    sp.sparda_tree_select(s, f.to(dev), n, torch.tensor(t_ctx, dtype=torch.int32, device=dev), t, parent.to(dev),
                          kc.to(dev), sel, cnt, ws)
    torch.cuda.synchronize()
    assert torch.equal(cnt.cpu(), want[1]) and torch.equal(sel.cpu(), want[0])
    # and the nodes whose candidates do not reach such a window have the sets of an ordinary row at their position
    free = [i for i in range(n) if t % L == 0 or t % L >= 16 or (t + i) // L == t // L]
    one = shape_of(2, H, 1, k, t, n, 1, 2, grid)
    i = free[-1]
    rows = torch.empty(1, H, 1, k, dtype=torch.int16, device=dev), torch.empty(1, H, 1, dtype=torch.int16, device=dev)
    one.batch = 1
    ws = workspace(dev, sp.sparda_workspace_size(one, sp.SPARDA_OP_FORECAST_SELECT, 1, t + i))
    sp.sparda_forecast_select(one, f[:1, :, i:i + 1].contiguous().to(dev), 1, t + i, kc[:1].contiguous().to(dev), *rows, ws)
    torch.cuda.synchronize()
    assert torch.equal(rows[0][0, :, 0], sel[0, :, i]) and torch.equal(rows[1][0, :, 0], cnt[0, :, i])


# ---- verify: many siblings, each rejected ------------------------------------------------------------------------

@pytest.mark.parametrize("V,bf16", [(50021, True), (131072, False)])
def test_verify_a_star_of_rejections(dev, V, bf16):  # noqa: F811
    """63 siblings drawn over a large vocabulary from a q far from p: they are rejected one after another, and every test
    after the first needs the sum of what the earlier ones left."""
    case = (3, 64, "star", V, 0, True, bf16)
    p, q, tokens, parent, u = verify_inputs(case, V, sharp=2.0, near=6.0)
    u[:2] = 0.999 + u[:2] / 2000  # the third sequence: as drawn
    got = check_verify(dev, case, (p, q, tokens, parent, u))
    say("  kept", got[0][:, :3].tolist())


# ---- commit: keys of very different sizes -----------------------------------------------------------------------

@pytest.mark.parametrize("grid", [(64, 64), (32, 16)])
def test_commit_has_the_bits_of_compress_keys(dev, grid):  # noqa: F811
    """Keys from 2^-100 to 2^100, whose sums are not exact in float64: the windows that a commit completes have the bits
    that the ordinary call gives, which adds in the same order."""
    gen = torch.Generator().manual_seed(grid[0])
    B, H, n, t_cap, t0 = 3, 2, 40, 256, (100, 60, 150)
    s = shape_of(B, H, 1, 3, 0, n, grid=grid, t_cap=t_cap)

    def mk(rows):
        x = torch.randn(B, H, rows, D, generator=gen) * 2.0 ** torch.randint(-100, 100, (B, H, rows, D), generator=gen)
        return x.to(torch.bfloat16).to(dev)

    kt, vt, k, v = mk(n), mk(n), mk(t_cap), mk(t_cap)
    kc = torch.zeros(B, H, s.nc_cap, D, dtype=torch.bfloat16, device=dev)
    t, t_new = torch.tensor(t0, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev)
    path = torch.arange(n, dtype=torch.int32, device=dev).expand(B, n).contiguous()
    n_path = torch.full((B,), n, dtype=torch.int32, device=dev)
    sp.sparda_tree_commit(s, n, t, path, n_path, 1, [kt], [vt], [k], [v], [kc], t_new)
    one = shape_of(1, H, 1, 3, 0, n, grid=grid, t_cap=t_cap)
    done = 0
    for b in range(B):
        w0, w1 = ((x - grid[0]) // grid[1] + 1 if x >= grid[0] else 0 for x in (t0[b], t0[b] + n))
        done += w1 - w0
        if w1 == w0:
            continue
        want = torch.zeros(1, H, s.nc_cap, D, dtype=torch.bfloat16, device=dev)
        sp.sparda_compress_keys(one, k[b:b + 1].contiguous(), t0[b] + n, w0, w1, want)
        torch.cuda.synchronize()
        assert torch.equal(kc[b].view(torch.int16), want[0].view(torch.int16))
    assert done > 0
