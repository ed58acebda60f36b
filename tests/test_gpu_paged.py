"""Rotary positions and the operators over paged caches on the GPU, against their definitions in float64
(paged_reference.py), alone and in a run as a serving loop makes it."""
import random
import sys

import pytest
import torch

import paged_reference as ref
import paper_2606_04511_amd.sparda as sp

pytestmark = pytest.mark.gpu
D, L = 128, 64
NAN = float("nan")
BF = torch.bfloat16


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sp.load()
    return torch.device("cuda:0")


def shape_of(B, H, G=1, k=3, t_cap=64, n_init=1, n_local=2, grid=(64, 64)):
    return sp.SpardaShape(batch=B, n_kv_heads=H, group_size=G, k_total=k, t_cap=-(-t_cap // L) * L, nc_cap=0, n_init=n_init,
                          n_local=n_local, cmp_kernel=grid[0], cmp_stride=grid[1])


def workspace(dev, shape, op, t_max):
    n = sp.sparda_workspace_size(shape, op, 1, t_max - 1)
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=dev)  # NaN patterns


def table_of(rng, B, t_cap, page, spare=2, fill=-1, lens=None):
    """int32 [B][pages of t_cap tokens]: distinct pages in no order, `fill` past a sequence's own, and the pages' number."""
    per = -(-(-(-t_cap // L) * L) // page)
    need = [per if lens is None else max(0, -(-t // page)) for t in (lens or [0] * B)]
    ids = list(range(sum(need) + spare))
    rng.shuffle(ids)
    table = torch.full((B, per), fill, dtype=torch.int32)
    for b in range(B):
        for i in range(need[b]):
            table[b, i] = ids.pop()
    return table, sum(need) + spare


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == BF else torch.int32)


# ---- rotate --------------------------------------------------------------------------------------

def freqs(rot, base=10000.0):
    return torch.tensor([base ** (-2 * j / rot) for j in range(rot // 2)], dtype=torch.float64)


ROTATE = [
    # batch, heads, tokens, rot, pairs, back, token first, first position
    (1, 1, 1, 128, False, False, False, 0),
    (1, 40, 1, 128, False, False, True, 131071),
    (2, 3, 5, 128, True, True, False, -7),
    (3, 7, 33, 64, False, True, True, 12345),
    (2, 8, 65, 96, True, False, True, 2097000),
    (1, 2, 100, 16, False, False, False, 99999),
    (1, 5, 17, 32, True, True, True, 2147483000),
    (2, 2, 9, 0, False, False, True, 5),
    (4, 33, 700, 112, False, False, False, 70000),
]


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("case", ROTATE)
def test_rotate(dev, case, dtype):
    B, H, n, rot, pairs, back, first, p0 = case
    say("rotate", case, dtype)
    gen = torch.Generator().manual_seed(100 * n + rot)
    freq, scale = freqs(rot), 1.25
    x = torch.randn(B, n, H, D, generator=gen).to(dtype)
    x = x.transpose(1, 2) if first else x.transpose(1, 2).contiguous()
    pos = (p0 + torch.arange(n)).to(torch.int32) if B == 1 else torch.stack([(p0 - 11 * b + torch.arange(n)) for b in range(B)]).to(
        torch.int32)
    xd, y = x.to(dev) if not first else x.transpose(1, 2).to(dev).transpose(1, 2), torch.full((B, H, n, D), NAN, dtype=dtype, device=dev)
    rope = sp.SpardaRope(rot, sp.SPARDA_ROPE_PAIRS if pairs else sp.SPARDA_ROPE_HALF, freq.to(dev) if rot else None, scale)
    kind = sp.SPARDA_F32 if dtype == torch.float32 else sp.SPARDA_BF16
    sp.sparda_rotate(rope, kind, B, H, n, xd, pos.to(dev), 0 if B == 1 else n, y, back)
    want, size = ref.turn(x, pos if B == 1 else pos[:, None], freq, rot, pairs, scale, back)
    bar = ref.turn_bar(want, size, 2.0 ** 31, 1.0, 2.0 ** -8 if dtype == BF else 0.0)
    if abs(p0) < 2 ** 21:
        bar = ref.turn_bar(want, size, 2.0 ** 21, 1.0, 2.0 ** -8 if dtype == BF else 0.0)
    got = y.cpu()
    assert torch.equal(bits(got[..., rot:]), bits(x[..., rot:]))  # what passes keeps its bits
    assert ((got.double() - want).abs() <= bar).all(), float(((got.double() - want).abs() / bar).max())
    sp.sparda_rotate(rope, kind, B, H, n, xd, pos.to(dev), 0 if B == 1 else n, xd, back)  # in place
    assert torch.equal(bits(xd), bits(y))


def test_rotate_repeats_rows_and_leaves_others(dev):
    """A broadcast input, an output that is a slice of a wider tensor."""
    gen = torch.Generator().manual_seed(1)
    one = torch.randn(1, 1, 6, D, generator=gen).to(dev)
    wide = torch.full((2, 6, 5, D), 7.0, device=dev)
    y = wide[:, :, 1:4].transpose(1, 2)
    rope = sp.SpardaRope(64, sp.SPARDA_ROPE_HALF, freqs(64).to(dev))
    pos = torch.arange(6, dtype=torch.int32, device=dev)
    sp.sparda_rotate(rope, sp.SPARDA_F32, 2, 3, 6, one.expand(2, 3, 6, D), pos, 0, y)
    want, size = ref.turn(one.cpu(), pos.cpu(), freqs(64), 64, False, 1.0)
    for b in range(2):
        for h in range(3):
            assert ((y[b, h].cpu().double() - want[0, 0]).abs() <= ref.turn_bar(want, size, 6, 1, 0.0)[0, 0]).all()
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, 4] == 7).all()


def test_rotation_gradient_against_differences(dev):
    """Backward is the gradient of forward: differences of the GPU's own forward in float32."""
    gen = torch.Generator().manual_seed(2)
    x, g = (torch.randn(1, 2, 5, D, generator=gen) for _ in range(2))
    pos = torch.tensor([0, 1, 500, 8191, 100000], dtype=torch.int32, device=dev)
    rope = sp.SpardaRope(96, sp.SPARDA_ROPE_PAIRS, freqs(96).to(dev), 1.5)

    def run(v, back):
        y = torch.empty(1, 2, 5, D, device=dev)
        sp.sparda_rotate(rope, sp.SPARDA_F32, 1, 2, 5, v.to(dev), pos, 0, y, back)
        return y.cpu().double()

    dx = run(g, True)
    for i in (0, 1, 47, 48, 95, 100):
        d = torch.zeros_like(x)
        d[..., i] = 1.0
        diff = run(x + d, False) - run(x - d, False)  # the rotation is linear: no step error
        want = (diff * g.double()).sum(-1) / 2
        # each forward value: 2^-21.4 of a pair's size below 1.5 (|x| + 1) 2; 128 of them, two sides, over 2
        assert ((dx[..., i] - want).abs() <= 2.0 ** -21 * 1.5 * 2 * 6 * g.abs().sum(-1).double()).all()


# ---- append --------------------------------------------------------------------------------------

APPEND = [
    # t_ctx, n_max, n_new (None: all), kv heads, heads per group, page, grid, rot, pairs
    ((0,), 1, None, 1, 1, 64, (64, 64), 128, False),
    ((63, 64, 127, -1), 1, None, 2, 4, 64, (64, 64), 128, False),          # a block completes; an absent sequence
    ((15, 31, 47, 46, 62, 63), 1, None, 2, 3, 16, (32, 16), 64, True),     # windows complete, or not
    ((0, 5, 63, 64, 100, 17), 70, (70, 0, 1, 69, 33, 64), 2, 2, 64, (64, 64), 96, False),
    ((0, 5, 15, 16, 100, 33), 100, (100, 27, 0, 1, -3, 200), 3, 1, 16, (32, 16), 128, False),
    ((7, 200), 333, (333, 150), 1, 16, 128, (32, 16), 32, True),
    ((0, 30), 290, None, 8, 4, 32, (32, 16), 0, False),
    ((250, 255, 256, 300), 10, None, 1, 2, 256, (64, 64), 128, False),     # past t_cap (256): dropped
]


def rows_view(x):
    """[B][heads][n][128] whose tokens lie one behind the other with their heads side by side."""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


@pytest.mark.parametrize("case", APPEND)
def test_append(dev, case):
    t_ctx, n, n_new, H, G, page, grid, rot, pairs = case
    say("append", case)
    B, rng = len(t_ctx), random.Random(n + rot)
    gen = torch.Generator().manual_seed(100 * n + rot)
    cap = 256 if page == 256 else -(-(max(t_ctx) + n) // L) * L
    shape = shape_of(B, H, G, t_cap=cap, grid=grid)
    table, n_pages = table_of(rng, B, cap, page)
    missing = B > 1 and page == 16  # one page of sequence 0 that is none, one that lies past the pool
    if missing:
        table[0, 1], table[1, 0] = -1, n_pages
    k, v = (torch.randn(n_pages, H, page, D, generator=gen).to(BF) for _ in range(2))
    kc = torch.randn(n_pages, H, page // grid[1], D, generator=gen).to(BF)
    new = {x: rows_view(torch.randn(B, h, n, D, generator=gen).to(BF)) for x, h in (("k", H), ("v", H), ("q", H * G), ("f", H))}
    freq, scale = freqs(rot), 1.1
    rope = sp.SpardaRope(rot, int(pairs), freq.to(dev) if rot else None, scale)
    kd, vd, kcd, t_new = k.to(dev), v.to(dev), kc.to(dev), torch.full((B,), -77, dtype=torch.int32, device=dev)
    pages = sp.SpardaPages(page, table.to(dev), kd, vd, kcd)
    qo, fo = (torch.full((B, h, n, D), 3.0, dtype=BF, device=dev) for h in (H * G, H))
    cnt_d = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device=dev)
    nd = {x: y.transpose(1, 2).to(dev).transpose(1, 2) for x, y in new.items()}
    sp.sparda_paged_append(shape, pages, rope, n, cnt_d, torch.tensor(t_ctx, dtype=torch.int32, device=dev), nd["k"], nd["v"],
                           nd["q"], qo, nd["f"], fo, t_new)
    kg, vg, kcg, qg, fg = (x.cpu() for x in (kd, vd, kcd, qo, fo))
    want_t = []
    touched, windows = torch.zeros(n_pages, page, dtype=torch.bool), torch.zeros(n_pages, page // grid[1], dtype=torch.bool)
    for b, t in enumerate(t_ctx):
        c = n if n_new is None else min(max(n_new[b], 0), n)
        c = 0 if t < 0 else max(0, min(c, cap - t))
        want_t.append(t + c)
        pos = t + torch.arange(c)
        for x, got in (("q", qg), ("f", fg)):
            want, size = ref.turn(new[x][b, :, :c], pos, freq, rot, pairs, scale)
            assert ((got[b, :, :c].double() - want).abs() <= ref.turn_bar(want, size, cap, 1, 2.0 ** -8)).all(), (x, b)
            assert (got[b, :, c:] == 3).all(), (x, b)  # rows past the tokens are left as they were
        want, size = ref.turn(new["k"][b, :, :c], pos, freq, rot, pairs, scale)
        bar = ref.turn_bar(want, size, cap, 1, 2.0 ** -8)
        for j in range(c):
            p = int(table[b, (t + j) // page])
            if not 0 <= p < n_pages:
                continue
            touched[p, (t + j) % page] = True
            assert ((kg[p, :, (t + j) % page].double() - want[:, j]).abs() <= bar[:, j]).all(), (b, j)
            assert torch.equal(bits(vg[p, :, (t + j) % page]), bits(new["v"][b, :, j])), (b, j)
        for w in range((t + c - grid[0]) // grid[1] + 1 if t + c >= grid[0] else 0):
            lo, hi = w * grid[1], w * grid[1] + grid[0]
            pg = [int(table[b, x // page]) for x in range(lo, hi)]
            if hi <= t or not all(0 <= p < n_pages for p in pg):
                continue
            windows[pg[0], lo % page // grid[1]] = True
            # the bits of the mean of what the cache holds, as sparda_compress_keys gives them
            one = torch.zeros(1, H, 64, D, dtype=BF)
            for i, x in enumerate(range(lo, hi)):
                one[0, :, i] = kg[pg[i], :, x % page]
            out = torch.zeros(1, H, 1, D, dtype=BF, device=dev)
            sp.sparda_compress_keys(sp.SpardaShape(batch=1, n_kv_heads=H, group_size=1, k_total=3, t_cap=64, nc_cap=1,
                                                   cmp_kernel=grid[0], cmp_stride=grid[1]), one.to(dev), 64, 0, 1, out)
            got = kcg[pg[0], :, lo % page // grid[1]]
            assert torch.equal(bits(got), bits(out.cpu()[0, :, 0])), (b, w)
            mean = one[0, :, :grid[0]].double().mean(1)
            assert ((got.double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -133).all()
    assert t_new.tolist() == want_t
    keep = ~touched[:, None, :, None]
    assert torch.equal(bits(kg) * keep, bits(k) * keep) and torch.equal(bits(vg) * keep, bits(v) * keep)
    keep = ~windows[:, None, :, None]
    assert torch.equal(bits(kcg) * keep, bits(kc) * keep)


def test_append_without_keys_rotation_or_queries(dev):
    """k_cmp, rope, q and f absent; K and V as slices of one pool with a stride between pages; in-place queries."""
    gen = torch.Generator().manual_seed(8)
    H, n, page = 2, 5, 16
    pool = torch.randn(6, 2, H, page, D, generator=gen).to(BF).to(dev)
    before = pool.clone()
    table = torch.tensor([[4, 1, 0, 5], [2, 3, -1, -1]], dtype=torch.int32, device=dev)
    shape = shape_of(2, H, 2, t_cap=64, grid=(32, 16))
    pages = sp.SpardaPages(page, table, pool[:, 0], pool[:, 1])
    kn, vn = (torch.randn(2, H, n, D, generator=gen).to(BF).to(dev) for _ in range(2))
    t_ctx, t_new = torch.tensor([14, 30], dtype=torch.int32, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    sp.sparda_paged_append(shape, pages, None, n, None, t_ctx, kn, vn, None, None, None, None, t_new)
    assert t_new.tolist() == [19, 35]
    for b, t in ((0, 14), (1, 30)):
        for j in range(n):
            p = int(table[b, (t + j) // page])
            if p >= 0:
                before[p, 0, :, (t + j) % page], before[p, 1, :, (t + j) % page] = kn[b, :, j], vn[b, :, j]
    assert torch.equal(bits(pool), bits(before))
    rope = sp.SpardaRope(128, sp.SPARDA_ROPE_HALF, freqs(128).to(dev))
    q = torch.randn(2, 4, n, D, generator=gen).to(BF).to(dev)
    out = torch.empty_like(q)
    sp.sparda_paged_append(shape, pages, rope, n, None, t_ctx, kn, vn, q, out, None, None, t_new)
    sp.sparda_paged_append(shape, pages, rope, n, None, t_ctx, kn, vn, q, q, None, None, t_new)
    assert torch.equal(bits(q), bits(out))


# ---- select --------------------------------------------------------------------------------------

SELECT = [
    # t_ctx, kv heads, k, n_init, n_local, page, grid
    ((0, 1, 64, 65, 128, 193, 256, 300), 2, 4, 1, 2, 64, (64, 64)),
    ((1, 31, 32, 33, 47, 48, 300, 448, 449, 460), 1, 4, 0, 1, 16, (32, 16)),   # the edge window with n_local = 1
    ((4096, 3000, -5, 100), 8, 16, 1, 2, 64, (64, 64)),
    ((8000, 4097, 517), 2, 20, 2, 3, 32, (32, 16)),
    ((16500, 16384, 9000), 3, 64, 1, 2, 256, (32, 16)),                     # 257 candidates
    ((34000, 33000), 1, 31, 0, 2, 128, (64, 64)),                            # 530
    ((70001,), 2, 96, 1, 32, 64, (64, 64)),                                   # 1061
    ((131072, 131009), 1, 64, 1, 2, 1024, (64, 64)),                          # 2046
    ((270000,), 1, 64, 1, 2, 64, (32, 16)),                                   # 4216: radix passes over memory
    ((200000,), 1, 40, 1, 2, 65536, (64, 64)),                                # 3123
    (tuple(range(64, 64 + 40 * 37, 37)), 8, 9, 1, 2, 64, (64, 64)),           # 320 rows
    ((1100000, 70), 1, 64, 1, 2, 64, (64, 64)),                               # 17185: more than LDS holds
    ((5000, 4000) * 14, 7, 9, 1, 2, 32, (32, 16)),                            # 196 rows, (32, 16), one launch
    (((16384 + 2) * 64,), 1, 64, 1, 2, 64, (64, 64)),                         # 16383: as many as LDS holds
]


def exact_rows(gen, *size):
    """bf16 values on a grid of 1/8: scores of such rows with such keys are exact in float32."""
    return ((torch.randn(*size, generator=gen) * 8).round() / 8).clamp(-4, 4).to(BF)


@pytest.mark.parametrize("case", SELECT)
def test_select(dev, case):
    t_ctx, H, k, n_init, n_local, page, grid = case
    say("select", case)
    B, rng, gen = len(t_ctx), random.Random(5), torch.Generator().manual_seed(len(t_ctx) + k)
    cap, t_max = -(-max(t_ctx) // L) * L, max(t_ctx)
    shape = shape_of(B, H, 1, k, cap, n_init, n_local, grid)
    table, n_pages = table_of(rng, B, cap, page, lens=t_ctx, fill=1 << 30)
    f, kc = exact_rows(gen, B, H, 1, D), exact_rows(gen, n_pages, H, page // grid[1], D)
    for b, t in enumerate(t_ctx):  # keys that are not complete, or of no sequence, count for nothing
        for w in range(max(0, (t - grid[0]) // grid[1] + 1), -(-t // grid[1])):
            kc[int(table[b, w * grid[1] // page]), :, w * grid[1] % page // grid[1]] = NAN
    pages = sp.SpardaPages(page, table.to(dev), k_cmp=kc.to(dev))
    sel = torch.full((B, H, 1, k), 77, dtype=torch.int16, device=dev)
    cnt = torch.full((B, H, 1), 77, dtype=torch.int16, device=dev)
    ws = workspace(dev, shape, sp.SPARDA_OP_PAGED_SELECT, t_max)
    sp.sparda_paged_select(shape, pages, f.to(dev), torch.tensor(t_ctx, dtype=torch.int32, device=dev), t_max, sel, cnt, ws)
    sel, cnt = sel.cpu(), cnt.cpu()
    for b, t in enumerate(t_ctx):
        n_win = (t - grid[0]) // grid[1] + 1 if t >= grid[0] else 0
        for h in range(H):
            want = []
            if t > 0:
                keys = ref.rows_of(kc, table[b], n_win, page, grid[1])[h] if n_win else torch.zeros(0, D)
                want = ref.selection(f[b, h, 0], keys, t, k, n_init, n_local, grid)
            assert int(cnt[b, h, 0]) == len(want), (b, h)
            assert sel[b, h, 0].tolist() == want + [-1] * (k - len(want)), (b, h)


def test_select_ties_missing_pages_and_odd_scores(dev):
    """Equal scores go to the lower block; a window without a page is never preferred; infinities and a NaN in the keys
    leave a valid set."""
    gen, page, k, t = torch.Generator().manual_seed(1), 64, 8, 64 * 40
    shape = shape_of(4, 1, 1, k, t)
    table = torch.arange(160, dtype=torch.int32).view(4, 40).contiguous()
    f, kc = exact_rows(gen, 4, 1, 1, D), torch.ones(160, 1, 1, D, dtype=BF)
    kc[40:80] = exact_rows(gen, 40, 1, 1, D)
    table[1, 1:30:2] = -1
    kc[80:120] = exact_rows(gen, 40, 1, 1, D)
    f[2] = 1.0
    kc[85], kc[90] = float("inf"), float("-inf")
    kc[120:160] = exact_rows(gen, 40, 1, 1, D)
    kc[130, 0, 0, 3] = NAN
    pages = sp.SpardaPages(page, table.to(dev), k_cmp=kc.to(dev))
    sel = torch.empty(4, 1, 1, k, dtype=torch.int16, device=dev)
    cnt = torch.empty(4, 1, 1, dtype=torch.int16, device=dev)
    sp.sparda_paged_select(shape, pages, f.to(dev), torch.full((4,), t, dtype=torch.int32, device=dev), t, sel, cnt,
                           workspace(dev, shape, sp.SPARDA_OP_PAGED_SELECT, t))
    sel = sel.cpu()[:, 0, 0]
    assert cnt.flatten().tolist() == [8] * 4
    assert sel[0].tolist() == [0, 1, 2, 3, 4, 5, 38, 39]
    assert not set(sel[1].tolist()) & set(range(1, 30, 2))
    assert 5 in sel[2].tolist() and 10 not in sel[2].tolist()
    assert sel[3].tolist() == sorted(set(sel[3].tolist())) and sel[3].min() >= 0 and sel[3].max() < 40


def test_select_of_many_rows_of_one_prefix(dev):
    """200 sequences that share their pages, 8192 candidates of each in one launch."""
    gen, B, k = torch.Generator().manual_seed(6), 200, 20
    n_blk = 8192 + 3
    shape, t_max = shape_of(B, 1, 1, k, 64 * n_blk), 64 * n_blk
    table = torch.randperm(n_blk, generator=gen).int().expand(B, n_blk).contiguous()
    f, kc = exact_rows(gen, B, 1, 1, D), exact_rows(gen, n_blk, 1, 1, D)
    t = [t_max - 64 * (b % 7) - b for b in range(B)]
    sel = torch.empty(B, 1, 1, k, dtype=torch.int16, device=dev)
    cnt = torch.empty(B, 1, 1, dtype=torch.int16, device=dev)
    sp.sparda_paged_select(shape, sp.SpardaPages(64, table.to(dev), k_cmp=kc.to(dev)), f.to(dev),
                           torch.tensor(t, dtype=torch.int32, device=dev), t_max, sel, cnt,
                           workspace(dev, shape, sp.SPARDA_OP_PAGED_SELECT, t_max))
    keys = kc[table[0].long(), 0, 0]
    assert cnt.flatten().tolist() == [k] * B
    for b in range(0, B, 9):
        assert sel[b, 0, 0].tolist() == ref.selection(f[b, 0, 0], keys[:t[b] // 64], t[b], k, 1, 2, (64, 64)), b


# ---- attention -----------------------------------------------------------------------------------

def run_attn(dev, shape, pages, q, t_ctx, t_max, sel, cnt, scale=ref.SCALE):
    o = torch.full(q.shape, NAN, dtype=BF, device=dev)
    ws = workspace(dev, shape, sp.SPARDA_OP_PAGED_ATTN, t_max)
    put = lambda x: None if x is None else x.to(dev)  # noqa: E731
    sp.sparda_paged_attn(shape, pages, q.to(dev), t_ctx.to(dev), t_max, put(sel), put(cnt), scale, o, ws)
    first = o.cpu()
    sp.sparda_paged_attn(shape, pages, q.to(dev), t_ctx.to(dev), t_max, put(sel), put(cnt), scale, o, ws)
    assert torch.equal(bits(o.cpu()), bits(first))  # deterministic
    return first[:, :, 0]


def check(got, o, w):
    bar = ref.attn_bar(o, w)
    err = (got.double() - o).abs()
    assert torch.isfinite(got).all() and (err <= bar).all(), float((err / bar).max())
    return float((err / bar).max())


def pools(gen, table, t_ctx, n_pages, H, page):
    """K and V of the sequences' tokens; NaN wherever no sequence has one."""
    k, v = (torch.full((n_pages, H, page, D), NAN, dtype=BF) for _ in range(2))
    for b, t in enumerate(t_ctx):
        for i in range(-(-max(t, 0) // page)):
            p, m = int(table[b, i]), min(page, t - i * page)
            if 0 <= p < n_pages:
                k[p, :, :m], v[p, :, :m] = (torch.randn(H, m, D, generator=gen).to(BF) for _ in range(2))
    return k, v


DENSE = [
    # t_ctx, kv heads, heads per group, page
    ((1,), 1, 1, 16),
    ((0, 1, 15, 16, 17, 31, 32, 33, 64, 65, -3), 2, 4, 16),
    ((100, 0, 257, 1), 3, 5, 32),
    ((1000, 999, 40), 2, 16, 64),
    ((4096,), 8, 4, 64),
    ((4095, 7, 2049), 1, 7, 128),
    ((20000, 3), 2, 8, 256),
    ((33333,), 1, 12, 16),
    ((70000,), 1, 2, 1024),
    (tuple(range(1, 300, 7)), 4, 3, 16),
    ((5, 9) * 300, 2, 1, 16),            # more sequences than threads of a workgroup
    ((0, -1) * 20, 2, 4, 16),            # nothing at all
    ((5000,) + tuple(range(0, 127)), 2, 3, 32),                  # one long context among short ones
    (tuple(range(0, 40)) * 13 + (5000, 700), 1, 4, 16),          # the same with more sequences than threads
    (tuple(range(2300, 500, -55)), 8, 4, 64),                    # 264 rows, most of them long
    ((3, 9000, 0, 4100, 31) * 13, 4, 16, 128),                   # long rows that share workgroups with short ones
    # many short rows, a wavefront each: the last workgroup partly filled, absent sequences, contexts up to the longest that
    # go this way and one past it, for every number of rows
    ((61, 0, 64, 33, -1, 1, 32) * 37, 1, 4, 64),
    ((64, 0, 65, 33, -1, 1, 32) * 37, 1, 4, 64),
    ((192, 17, 0, 100, 31) * 51 + (191,), 3, 5, 16),
    ((193, 17, 0, 100, 31) * 51 + (191,), 3, 5, 16),
    ((512, 3, 0, 510, 250, 64) * 32 + (481,), 8, 16, 128),
    ((513, 3, 0, 510, 250, 64) * 32 + (481,), 8, 2, 128),
]


@pytest.mark.parametrize("case", DENSE)
def test_attention_over_whole_contexts(dev, case):
    t_ctx, H, G, page = case
    say("dense", case)
    B, rng, gen = len(t_ctx), random.Random(B_seed(case)), torch.Generator().manual_seed(H * 100 + G)
    t_max = max(max(t_ctx), 1)
    shape = shape_of(B, H, G, t_cap=t_max)
    table, n_pages = table_of(rng, B, t_max, page, lens=t_ctx, fill=-1)
    k, v = pools(gen, table, t_ctx, n_pages, H, page)
    q = torch.randn(B, H * G, 1, D, generator=gen).to(BF)
    t = torch.tensor(t_ctx, dtype=torch.int32)
    got = run_attn(dev, shape, sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev)), q, t, t_max, None, None)
    o, w = ref.attn(q[:, :, 0], k, v, table, t, page, None, None, ref.SCALE)
    say("worst share of the bar", check(got, o, w))


def B_seed(case):
    return sum(case[0][:5]) + 13 * case[1] + case[2]


SPARSE = [
    # t_ctx, kv heads, heads per group, k, page, order
    ((1, 64, 65, 0), 1, 1, 3, 64, "sorted"),
    ((300, 129, -2, 64), 2, 4, 4, 16, "sorted"),
    ((2000, 700), 2, 3, 11, 32, "mixed"),
    ((5000, 4999, 64 * 30), 8, 4, 16, 64, "sorted"),
    ((5000, 4999, 64 * 30), 2, 16, 97, 64, "mixed"),
    ((40000,), 1, 8, 64, 128, "mixed"),
    ((9000, 8000), 1, 12, 140, 16, "twice"),
    (tuple(range(10, 3000, 73)), 8, 2, 13, 64, "mixed"),       # 328 rows: more than workgroups
    ((600,) * 300, 1, 5, 5, 256, "sorted"),
    ((5000, 0, 70, -1, 640), 2, 4, 40, 64, "sorted"),          # rows of several workgroups, some without tokens
    ((5000, 0, 70, -1, 640), 2, 4, 40, 16, "mixed"),
    (tuple(range(1, 2000, 29)) + (0, -9), 4, 1, 64, 32, "sorted"),  # lists longer than most contexts
    (tuple(range(1, 2000, 29)) + (0, -9), 4, 1, 70, 32, "twice"),
    ((100000,), 1, 2, 1000, 64, "sorted"),
    ((2700, 3, 0) + tuple(range(2600, 2700)), 3, 4, 40, 64, "sorted"),  # 309 rows of up to 40 blocks
    ((2700, 3, 0) + tuple(range(2600, 2700)), 3, 2, 40, 16, "mixed"),
    ((64, 1, 0, 50, -4) * 53, 1, 4, 7, 64, "mixed"),                    # many rows of few blocks, a wavefront each
    ((900, 3, 0, 510, 250, 64) * 22 + (700,), 6, 4, 3, 32, "sorted"),
    ((900, 3, 0, 510, 250, 64) * 32 + (481,), 8, 16, 8, 16, "twice"),
]


@pytest.mark.parametrize("case", SPARSE)
def test_attention_over_listed_blocks(dev, case):
    t_ctx, H, G, k_total, page, order = case
    say("sparse", case)
    B, rng, gen = len(t_ctx), random.Random(B_seed(case)), torch.Generator().manual_seed(H * 100 + G)
    t_max = max(t_ctx)
    shape = shape_of(B, H, G, k=k_total, t_cap=t_max)
    table, n_pages = table_of(rng, B, t_max, page, lens=t_ctx, fill=n_bad(rng))
    k, v = pools(gen, table, t_ctx, n_pages, H, page)
    q = torch.randn(B, H * G, 1, D, generator=gen).to(BF)
    sel = torch.full((B, H, 1, k_total), 5, dtype=torch.int16)  # what lies behind cnt counts for nothing
    cnt = torch.zeros(B, H, 1, dtype=torch.int16)
    for b in range(B):
        nb = max(1, (t_ctx[b] + 63) // 64)
        for h in range(H):
            if order == "sorted":
                got = sorted(rng.sample(range(nb), min(nb, k_total)))
            else:  # any order, repeats, blocks past the context, negative entries
                got = [rng.randrange(nb) if order == "twice" else rng.randrange(-1, nb + 3) for _ in range(k_total)]
                got = got[:rng.randrange(1, k_total + 1)]
            sel[b, h, 0, :len(got)] = torch.tensor(got, dtype=torch.int16)
            cnt[b, h, 0] = len(got)
    if B > 1:
        cnt[1, 0, 0] = 0  # a row that lists nothing
        cnt[0, 0, 0] = min(32767, int(cnt[0, 0, 0]))
    t = torch.tensor(t_ctx, dtype=torch.int32)
    got = run_attn(dev, shape, sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev)), q, t, t_max, sel, cnt)
    o, w = ref.attn(q[:, :, 0], k, v, table, t, page, sel, cnt, ref.SCALE)
    say("worst share of the bar", check(got, o, w))


def n_bad(rng):
    return rng.choice((-1, 1 << 30, -(1 << 31)))


@pytest.mark.parametrize("G", range(1, 17))
def test_attention_of_every_group_size(dev, G):
    gen, rng, t_ctx = torch.Generator().manual_seed(G), random.Random(G), (777, 130)
    table, n_pages = table_of(rng, 2, 777, 32, lens=t_ctx)
    k, v = pools(gen, table, t_ctx, n_pages, 2, 32)
    q = torch.randn(2, 2 * G, 1, D, generator=gen).to(BF)
    t = torch.tensor(t_ctx, dtype=torch.int32)
    got = run_attn(dev, shape_of(2, 2, G, t_cap=777), sp.SpardaPages(32, table.to(dev), k.to(dev), v.to(dev)), q, t, 777, None, None)
    check(got, *ref.attn(q[:, :, 0], k, v, table, t, 32, None, None, ref.SCALE))


def test_attention_skips_what_has_no_page(dev):
    """Pages that are none, inside and at the ends of a context, dense and listed; a row left with nothing."""
    gen, rng, t_ctx, page = torch.Generator().manual_seed(9), random.Random(9), (1000, 500, 64, 90), 16
    table, n_pages = table_of(rng, 4, 1000, page, lens=t_ctx)
    k, v = pools(gen, table, t_ctx, n_pages, 2, page)
    for b, at in ((0, (0, 1, 5, 30, 31, 62)), (1, (3, 30, 31)), (2, (0, 1, 2, 3)), (3, (4, 5))):
        for i in at:
            table[b, i] = rng.choice((-1, n_pages, 2 ** 31 - 1, -2 ** 31))
    q, t = torch.randn(4, 6, 1, D, generator=gen).to(BF), torch.tensor(t_ctx, dtype=torch.int32)
    pages = sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev))
    got = run_attn(dev, shape_of(4, 2, 3, t_cap=1000), pages, q, t, 1000, None, None)
    o, w = ref.attn(q[:, :, 0], k, v, table, t, page, None, None, ref.SCALE)
    check(got, o, w)
    assert (got[2] == 0).all()
    sel = torch.arange(8, dtype=torch.int16).expand(4, 2, 1, 8).contiguous()
    cnt = torch.full((4, 2, 1), 8, dtype=torch.int16)
    got = run_attn(dev, shape_of(4, 2, 3, k=8, t_cap=1000), pages, q, t, 1000, sel, cnt)
    check(got, *ref.attn(q[:, :, 0], k, v, table, t, page, sel, cnt, ref.SCALE))
    assert (got[2] == 0).all()


def test_attention_of_interleaved_pools(dev):
    """K and V as slices of one pool [n_pages][2][Hkv][P][128]."""
    gen, rng, t_ctx, page = torch.Generator().manual_seed(19), random.Random(19), (300, 77), 32
    table, n_pages = table_of(rng, 2, 300, page, lens=t_ctx)
    k, v = pools(gen, table, t_ctx, n_pages, 2, page)
    pool = torch.stack((k, v), 1).to(dev)
    q, t = torch.randn(2, 8, 1, D, generator=gen).to(BF), torch.tensor(t_ctx, dtype=torch.int32)
    got = run_attn(dev, shape_of(2, 2, 4, t_cap=300), sp.SpardaPages(page, table.to(dev), pool[:, 0], pool[:, 1]), q, t, 300, None, None)
    check(got, *ref.attn(q[:, :, 0], k, v, table, t, page, None, None, ref.SCALE))


@pytest.mark.parametrize("longest", [300, 1500, 3000])
def test_attention_of_as_many_sequences_as_fit(dev, longest):
    """65535 rows, by each division of the work: short contexts on shared pages, one long one, absent ones."""
    gen, B, page = torch.Generator().manual_seed(longest), 65535, 16
    n_pages = -(-longest // page) + 7
    table = torch.randint(n_pages, (B, -(-longest // L) * L // page), generator=gen, dtype=torch.int32)
    t = torch.randint(-1, 20, (B,), generator=gen, dtype=torch.int32)
    t[40000], t[-1] = longest, 33
    k, v = (torch.randn(n_pages, 1, page, D, generator=gen).to(BF) for _ in range(2))
    q = torch.randn(B, 2, 1, D, generator=gen).to(BF)
    got = run_attn(dev, shape_of(B, 1, 2, t_cap=longest), sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev)), q, t,
                   longest, None, None)
    rows = torch.cat([torch.arange(0, B, 977), torch.tensor([39999, 40000, 40001, B - 2, B - 1])])
    o, w = ref.attn(q[rows, :, 0], k, v, table[rows], t[rows], page, None, None, ref.SCALE)
    say("worst share of the bar", check(got[rows], o, w))
    assert not got[t <= 0].any() and torch.isfinite(got).all()


def test_attention_nan_and_infinity(dev):
    """A NaN or an infinity in an attended key or value reaches its row, and no other; t_ctx above t_max counts as t_max."""
    gen, rng, page, t = torch.Generator().manual_seed(10), random.Random(10), 64, 700
    table, n_pages = table_of(rng, 5, t, page)
    k, v = pools(gen, table, (t,) * 5, n_pages, 1, page)
    q = torch.randn(5, 2, 1, D, generator=gen).to(BF)
    clean_k, clean_v = k.clone(), v.clone()
    k[int(table[0, 3]), 0, 7, 5] = NAN
    v[int(table[1, 10]), 0, 11, 9] = float("inf")
    k[int(table[2, 2]), 0, :, :] = float("-inf")
    q[3, 1, 0, 0] = NAN
    pages = sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev))
    got = run_attn(dev, shape_of(5, 1, 2, t_cap=704), pages, q, torch.full((5,), 2000, dtype=torch.int32), t, None, None)
    assert torch.isnan(got[0]).all() and torch.isnan(got[3, 1]).all()
    assert not torch.isfinite(got[1, :, 9]).any() and torch.isfinite(got[1, :, :9]).all() and torch.isfinite(got[1, :, 10:]).all()
    o, w = ref.attn(q[:, :, 0], clean_k, clean_v, table, torch.full((5,), t), page, None, None, ref.SCALE)
    check(got[4], o[4], w[4])
    check(got[3, :1], o[3, :1], w[3, :1])


def test_attention_of_large_scores_and_one_hot_rows(dev):
    """Scores far apart (the running maximum moves late and by much), a scale of zero and a negative one."""
    gen, rng, page, t = torch.Generator().manual_seed(11), random.Random(11), 32, 2500
    table, n_pages = table_of(rng, 1, t, page)
    k, v = pools(gen, table, (t,), n_pages, 1, page)
    q = torch.randn(1, 4, 1, D, generator=gen).to(BF)
    for i, at in enumerate((5, 900, 1777, 2499)):
        k[int(table[0, at // page]), 0, at % page] = (q[0, i, 0].float() * (3 + i)).to(BF)
    pages, tt = sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev)), torch.tensor([t], dtype=torch.int32)
    for scale in (1.0, 0.0, -0.05, ref.SCALE):
        got = run_attn(dev, shape_of(1, 1, 4, t_cap=t), pages, q, tt, t, None, None, scale)
        o, w = ref.attn(q[:, :, 0], k, v, table, tt, page, None, None, scale)
        # logits up to |scale| 6 |q|^2 = 1100: a float32 sum is off by up to 2^-17 of that
        big = 2.0 ** -17 * abs(scale) * float((q.float().abs().sum(-1).max() * k[table[0, :78].long()].float().abs().max()))
        assert ((got.double() - o).abs() <= ref.attn_bar(o, w) + 2 * big * w).all()


def test_offsets_past_32_bits(dev):
    """A pool of more than 2^32 elements: append, attention and (below) selection reach its last pages."""
    H, page, n_pages = 1, 65536, 600  # 600 pages of 2^23 elements
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB of free device memory")
    gen = torch.Generator().manual_seed(12)
    k, v = (torch.empty(n_pages, H, page, D, dtype=BF, device=dev) for _ in range(2))
    kc = torch.empty(n_pages, H, page // 64, D, dtype=BF, device=dev)
    table = torch.tensor([[599, 3], [598, 597]], dtype=torch.int32)
    pages, shape = sp.SpardaPages(page, table.to(dev), k, v, kc), shape_of(2, H, 2, k=4, t_cap=131072)
    n = 200
    kn, vn = (torch.randn(2, H, n, D, generator=gen).to(BF) for _ in range(2))
    t_ctx, t_new = torch.zeros(2, dtype=torch.int32, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    sp.sparda_paged_append(shape, pages, None, n, None, t_ctx, kn.to(dev), vn.to(dev), None, None, None, None, t_new)
    for b in range(2):
        assert torch.equal(bits(k[int(table[b, 0]), :, :n].cpu()), bits(kn[b]))
        assert torch.equal(bits(kc[int(table[b, 0]), :, :3].cpu()),
                           bits((kn[b, :, :192].double().view(H, 3, 64, D).mean(2)).float().to(BF)))
    q = torch.randn(2, 2, 1, D, generator=gen).to(BF)
    got = run_attn(dev, shape, pages, q, t_new, 200, None, None)
    small = torch.tensor([[0], [1]], dtype=torch.int32)
    check(got, *ref.attn(q[:, :, 0], kn, vn, small, t_new, n, None, None, ref.SCALE))


# ---- together ------------------------------------------------------------------------------------

class Loop:
    """One layer's serving state: pages, and the same tokens in dense caches, one per sequence, whose ordinary operators
    the paged ones have to agree with."""

    def __init__(self, dev, B, H, G, k, cap, page, grid, seed):
        self.dev, self.gen, self.grid, self.page, self.cap = dev, torch.Generator().manual_seed(seed), grid, page, cap
        self.shape = shape_of(B, H, G, k, cap, 1, 2, grid)
        table, n_pages = table_of(random.Random(seed), B, cap, page)
        self.table = table.to(dev)
        self.k, self.v = (torch.full((n_pages, H, page, D), NAN, dtype=BF, device=dev) for _ in range(2))
        self.kc = torch.full((n_pages, H, page // grid[1], D), NAN, dtype=BF, device=dev)
        self.pages = sp.SpardaPages(page, self.table, self.k, self.v, self.kc)
        self.rope = sp.SpardaRope(128, sp.SPARDA_ROPE_HALF, freqs(128).to(dev))
        self.t, self.t_new = torch.zeros(B, dtype=torch.int32, device=dev), torch.zeros(B, dtype=torch.int32, device=dev)
        self.sel = torch.zeros(B, H, 1, k, dtype=torch.int16, device=dev)
        self.cnt = torch.zeros(B, H, 1, dtype=torch.int16, device=dev)
        self.ws = torch.empty(max(sp.sparda_workspace_size(self.shape, op, 1, cap - 1)
                                  for op in (sp.SPARDA_OP_PAGED_SELECT, sp.SPARDA_OP_PAGED_ATTN)), dtype=torch.uint8, device=dev)
        self.o, self.all = (torch.zeros(B, H * G, 1, D, dtype=BF, device=dev) for _ in range(2))

    def draw(self, n):
        s = self.shape
        return [torch.randn(s.batch, h, n, D, generator=self.gen).to(BF).to(self.dev)
                for h in (s.n_kv_heads, s.n_kv_heads, s.n_q_heads, s.n_kv_heads)]

    def append(self, n, n_new, k, v, q, f, qo, fo):
        sp.sparda_paged_append(self.shape, self.pages, self.rope, n, n_new, self.t, k, v, q, qo, f, fo, self.t_new)

    def attend(self, q, f):
        sp.sparda_paged_select(self.shape, self.pages, f, self.t_new, self.cap, self.sel, self.cnt, self.ws)
        sp.sparda_paged_attn(self.shape, self.pages, q, self.t_new, self.cap, self.sel, self.cnt, ref.SCALE, self.o, self.ws)
        sp.sparda_paged_attn(self.shape, self.pages, q, self.t_new, self.cap, None, None, ref.SCALE, self.all, self.ws)


@pytest.mark.parametrize("page,grid", [(64, (64, 64)), (16, (32, 16)), (128, (32, 16))])
def test_serving_loop_against_dense_caches(dev, page, grid):
    """Prompts of different lengths in two chunks, then decode steps: the sets and outputs are those of the ordinary decode
    operators on dense caches."""
    B, H, G, k, cap = 3, 2, 4, 6, 1024
    loop = Loop(dev, B, H, G, k, cap, page, grid, 21)
    for n, n_new in ((500, (500, 333, 64)), (100, (1, 100, 37))):
        new, counts = loop.draw(n), torch.tensor(n_new, dtype=torch.int32, device=dev)
        loop.append(n, counts, *new, torch.empty_like(new[2]), torch.empty_like(new[3]))
        loop.t.copy_(loop.t_new)
    one = sp.SpardaShape(batch=1, n_kv_heads=H, group_size=G, k_total=k, t_cap=cap, nc_cap=cap // grid[1], cmp_kernel=grid[0],
                         cmp_stride=grid[1])
    for step in range(40):
        kn, vn, q, f = loop.draw(1)
        qo, fo = torch.empty_like(q), torch.empty_like(f)
        loop.append(1, None, kn, vn, q, f, qo, fo)
        loop.attend(qo, fo)
        want, size = ref.turn(q[:, :, 0].cpu(), loop.t.cpu()[:, None], freqs(128), 128, False, 1.0)
        assert ((qo[:, :, 0].cpu().double() - want).abs() <= ref.turn_bar(want, size, cap, 1, 2.0 ** -8)).all()
        if step % 13 == 0:
            for b in range(B):
                t = int(loop.t_new[b])
                kk, vv = (x[loop.table[b].long()].transpose(0, 1).reshape(1, H, cap, D).contiguous() for x in (loop.k, loop.v))
                kc = torch.zeros(1, H, cap // grid[1], D, dtype=BF, device=dev)
                sp.sparda_compress_keys(one, kk, t, 0, (t - grid[0]) // grid[1] + 1, kc)
                paged = loop.kc[loop.table[b].long()].transpose(0, 1).reshape(1, H, cap // grid[1], D)
                n_win = (t - grid[0]) // grid[1] + 1
                assert torch.equal(bits(paged[:, :, :n_win]), bits(kc[:, :, :n_win]))
                sel, cnt = torch.empty_like(loop.sel[:1]), torch.empty_like(loop.cnt[:1])
                ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
                sp.sparda_forecast_select(one, fo[b:b + 1].contiguous(), 1, t - 1, kc, sel, cnt, ws)
                assert torch.equal(cnt, loop.cnt[b:b + 1])
                for h in range(H):  # both sum in float32: a block may differ where its score is within their error of the last
                    a, c = set(sel[0, h, 0].tolist()), set(loop.sel[b, h, 0].tolist())
                    z = (kc[0, h].cpu().double() @ fo[b, h, 0].cpu().double())
                    near = 2 * 2.0 ** -17 * float((kc[0, h].cpu().abs().double() @ fo[b, h, 0].cpu().abs().double()).max())
                    per = [float(z[max(0, (64 * j - grid[0]) // grid[1] + 1):min(n_win, (64 * j + 63) // grid[1] + 1)].max())
                           for j in range(t // 64)]
                    assert all(abs(per[x] - per[y]) <= near for x in a - c for y in c - a)
                kt, vt = kk.cpu(), vv.cpu()
                ident = torch.zeros(1, 1, dtype=torch.int32)
                tt = torch.tensor([t])
                for out, s_, c_ in ((loop.o, loop.sel.cpu()[b:b + 1], loop.cnt.cpu()[b:b + 1]), (loop.all, None, None)):
                    o, w = ref.attn(qo[b:b + 1, :, 0].cpu(), kt, vt, ident, tt, cap, s_, c_, ref.SCALE)
                    check(out[b:b + 1, :, 0].cpu(), o, w)
        loop.t.copy_(loop.t_new)


@pytest.mark.parametrize("page,grid", [(64, (64, 64)), (32, (32, 16))])
def test_shared_prefix(dev, page, grid):
    """Sequences that share the pages of a prefix, its last page copied: the same bits as with pages of their own."""
    B, H, prefix = 3, 2, 5 * page
    own, shared = (Loop(dev, B, H, 4, 6, 1024, page, grid, 9) for _ in range(2))
    new = [x[:1].expand_as(x).contiguous() for x in own.draw(prefix)]
    own.append(prefix, None, *new, torch.empty_like(new[2]), torch.empty_like(new[3]))
    first = torch.tensor([prefix, 0, 0], dtype=torch.int32, device=dev)
    shared.append(prefix, first, *new, torch.empty_like(new[2]), torch.empty_like(new[3]))
    for b in range(1, B):
        for pool in (shared.k, shared.v, shared.kc):
            pool[shared.table[b, 4].long()] = pool[shared.table[0, 4].long()]
        shared.table[b, :4] = shared.table[0, :4]
    for n in (1, 40, 1, 1):
        (kn, vn, q, f), t = own.draw(n), own.t_new.clone()
        for loop in (own, shared):
            loop.t.copy_(t)
            loop.qo, loop.fo = torch.empty_like(q), torch.empty_like(f)
            loop.append(n, None, kn, vn, q, f, loop.qo, loop.fo)
            loop.attend(loop.qo[:, :, -1:].contiguous(), loop.fo[:, :, -1:].contiguous())
        assert torch.equal(own.t_new, shared.t_new) and torch.equal(own.sel, shared.sel)
        assert torch.equal(bits(own.o), bits(shared.o)) and torch.equal(bits(own.all), bits(shared.all))


def test_captured_step_replays(dev):
    """A decode step captured once and replayed while the lengths grow, against eager steps; eager work and
    synchronizations between the replays."""
    args = (dev, 4, 2, 4, 6, 512, 16, (32, 16), 33)
    a, b = Loop(*args), Loop(*args)
    for loop in (a, b):
        new = loop.draw(150)
        loop.append(150, torch.tensor((150, 100, 31, 0), dtype=torch.int32, device=dev), *new, torch.empty_like(new[2]),
                    torch.empty_like(new[3]))
        loop.t.copy_(loop.t_new)
    kn, vn, q, f = a.draw(1)
    qo, fo = torch.empty_like(q), torch.empty_like(f)
    steps = [[torch.randn(x.shape, generator=torch.Generator().manual_seed(100 * i + j)).to(BF).to(dev)
              for j, x in enumerate((kn, vn, q, f))] for i in range(6)]

    def step(loop, kn, vn, q, f, qo, fo):
        loop.append(1, None, kn, vn, q, f, qo, fo)
        loop.attend(qo, fo)
        loop.t.copy_(loop.t_new)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = [x.clone() for x in (a.k, a.v, a.kc, a.t)]
    with torch.cuda.stream(side):
        step(a, kn, vn, q, f, qo, fo)  # warm
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip((a.k, a.v, a.kc, a.t), keep):
        x.copy_(y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, kn, vn, q, f, qo, fo)
    for i, new in enumerate(steps):
        for x, y in zip((kn, vn, q, f), new):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        step(b, *new, torch.empty_like(qo), torch.empty_like(fo))
        for name in ("t", "t_new", "sel", "cnt"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
        for name in ("o", "all"):
            assert torch.equal(bits(getattr(a, name)), bits(getattr(b, name))), (i, name)
    assert a.t.tolist() == [156, 106, 37, 6]


def test_calls_go_to_the_stream_they_are_given(dev):
    """On a side stream, and two calls at once on two streams with a workspace each."""
    gen, rng, t_ctx = torch.Generator().manual_seed(3), random.Random(3), (3000, 10)
    table, n_pages = table_of(rng, 2, 3000, 64, lens=t_ctx)
    k, v = pools(gen, table, t_ctx, n_pages, 4, 64)
    pages, shape = sp.SpardaPages(64, table.to(dev), k.to(dev), v.to(dev)), shape_of(2, 4, 4, t_cap=3000)
    q = torch.randn(2, 16, 1, D, generator=gen).to(BF).to(dev)
    t = torch.tensor(t_ctx, dtype=torch.int32, device=dev)
    want = run_attn(dev, shape, pages, q, t, 3000, None, None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(q) for _ in streams]
    spaces = [workspace(dev, shape, sp.SPARDA_OP_PAGED_ATTN, 3000) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, w in zip(streams, outs, spaces):
            sp.sparda_paged_attn(shape, pages, q, t, 3000, None, None, ref.SCALE, o, w, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(bits(o[:, :, 0].cpu()), bits(want))
