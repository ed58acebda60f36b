"""The operators over trees of drafted tokens on the GPU, against their definitions in float64
(tree_reference.py), alone and in a run as a decode loop makes it."""
import random
import sys

import pytest
import torch

import paper_2606_04511_amd.sparda as sp
import tree_reference as ref

pytestmark = pytest.mark.gpu
D, L = 128, 64
NAN = float("nan")


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    sp.load()
    return torch.device("cuda:0")


def shape_of(B, H, G, k, t_max, n, n_init=1, n_local=2, grid=(64, 64), t_cap=None):
    t_cap = t_cap or -(-(t_max + n) // L) * L
    return sp.SpardaShape(batch=B, n_kv_heads=H, group_size=G, k_total=k, t_cap=t_cap,
                          nc_cap=max(0, (t_cap - grid[0]) // grid[1] + 1), n_init=n_init, n_local=n_local,
                          cmp_kernel=grid[0], cmp_stride=grid[1])


def workspace(dev, n_bytes):
    return torch.full((max(n_bytes, 16),), 0xFF, dtype=torch.uint8, device=dev)  # NaN patterns


def trees(rng, B, n, kind, pad=()):
    p = torch.tensor([ref.tree(rng, n, kind) for _ in range(B)], dtype=torch.int32)
    for b, i, x in pad:
        p[b, i] = x
    return p


def exact_rows(gen, *size):
    """bf16 values on a grid of 1/8: scores of such rows with such keys are exact in float32."""
    return ((torch.randn(*size, generator=gen) * 8).round() / 8).clamp(-4, 4).to(torch.bfloat16)


# ---- select --------------------------------------------------------------------------------------

SELECT = [
    # t_ctx per sequence, nodes, tree, kv heads, k, n_init, n_local, grid
    ((0,), 1, "chain", 1, 3, 1, 2, (64, 64)),                        # no context
    ((0, 1, 63, 64, 65), 5, "wide", 2, 3, 1, 2, (64, 64)),           # no candidate, then one
    ((31, 32, 33, 47, 48, 300), 7, "wide", 1, 4, 0, 2, (32, 16)),    # window edges
    ((200, 447, 448), 64, "chain", 1, 4, 1, 2, (64, 64)),            # nodes of two blocks
    ((1000, 900), 64, "star", 2, 9, 2, 4, (32, 16)),
    ((4096,), 8, "wide", 8, 16, 1, 2, (64, 64)),
    ((4095, 3800, -1, 4000), 21, "wide", 2, 16, 1, 3, (32, 16)),     # an absent sequence
    ((9000, 8321), 17, "wide", 3, 40, 1, 32, (64, 64)),              # 129 to 256 candidates
    ((30001, 29000), 33, "wide", 1, 64, 1, 2, (32, 16)),             # 257 to 512
    ((60000,), 5, "wide", 1, 64, 1, 2, (64, 64)),                    # to 1024
    ((131000, 100000), 16, "wide", 1, 64, 1, 2, (32, 16)),           # to 2048
    ((200000,), 3, "chain", 1, 96, 1, 32, (64, 64)),                 # to 4096
    ((300007,), 3, "chain", 1, 64, 1, 2, (64, 64)),                  # radix passes
    ((5000,), 4, "wide", 1, 300, 1, 2, (64, 64)),                    # every block fits
]


@pytest.mark.parametrize("case,flat", [(c, False) for c in range(len(SELECT))] +
                         [(c, True) for c in range(len(SELECT)) if max(SELECT[c][0]) < 70000])
def test_select(dev, case, flat):
    t_ctx, n, kind, H, k, n_init, n_local, grid = SELECT[case]
    say("tree select", SELECT[case], "flat" if flat else "")
    gen, rng = torch.Generator().manual_seed(100 + case), random.Random(case)
    B, t_max = len(t_ctx), max(max(t_ctx), 0)
    s = shape_of(B, H, 1, k, t_max, n, n_init, n_local, grid)
    f = exact_rows(gen, B, H, n, D)
    kc = exact_rows(gen, B, H, max(s.nc_cap, 1), D)
    if flat:  # every score 0: ties go to the lowest blocks
        f.zero_()
    parent = trees(rng, B, n, kind, pad=[(0, n - 1, n)] if n > 2 else [])
    want_sel, want_cnt = ref.select(f, kc, t_ctx, parent, k, n_init, n_local, grid)
    for b, t in enumerate(t_ctx):  # keys that the context does not complete are not read as numbers
        kc[b, :, max(0, (t - grid[0]) // grid[1] + 1 if t >= grid[0] else 0):] = NAN
    sel = torch.full((B, H, n, k), 99, dtype=torch.int16, device=dev)
    cnt = torch.full((B, H, n), 99, dtype=torch.int16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, n, t_max))
    sp.sparda_tree_select(s, f.to(dev), n, torch.tensor(t_ctx, dtype=torch.int32, device=dev), t_max, parent.to(dev),
                          kc.to(dev), sel, cnt, ws)
    torch.cuda.synchronize()
    assert torch.equal(cnt.cpu(), want_cnt)
    assert torch.equal(sel.cpu(), want_sel)


@pytest.mark.parametrize("t", [9000, 30000, 60000, 131000])
@pytest.mark.parametrize("values", ["two", "steps", "tail", "nan", "inf"])
def test_select_of_awkward_scores(dev, t, values):
    """Scores that share few values, that lie far apart, that are not finite: the best by (score, lower block)."""
    gen, rng = torch.Generator().manual_seed(t), random.Random(t)
    n, k = 6, 64
    s = shape_of(1, 1, 1, k, t, n)
    f = torch.zeros(1, 1, n, D, dtype=torch.bfloat16)
    f[..., 0] = 1  # a block's score is the first element of its key
    kc = torch.zeros(1, 1, s.nc_cap, D, dtype=torch.bfloat16)
    x = torch.randn(s.nc_cap, generator=gen)
    if values == "two":
        x = (x > 1.2).float()
    elif values == "steps":
        x = (x * 2).round()
    elif values == "tail":
        x[torch.rand(s.nc_cap, generator=gen) < 0.01] *= 2.0 ** 60
    elif values == "inf":
        x[torch.rand(s.nc_cap, generator=gen) < 0.02] = float("inf")
        x[torch.rand(s.nc_cap, generator=gen) < 0.02] = -float("inf")
    kc[0, 0, :, 0] = x.to(torch.bfloat16)
    parent = trees(rng, 1, n, "wide")
    want = ref.select(f, kc, [t], parent, k, 1, 2, (64, 64))
    if values == "nan":  # what is chosen then is open; every entry is a block, each once
        kc[0, 0, 5::7, 0] = NAN
    sel = torch.full((1, 1, n + 1, k), 99, dtype=torch.int16, device=dev)
    cnt = torch.full((1, 1, n), 99, dtype=torch.int16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, n, t))
    sp.sparda_tree_select(s, f.to(dev), n, torch.tensor([t], dtype=torch.int32, device=dev), t, parent.to(dev),
                          kc.to(dev), sel, cnt, ws)
    torch.cuda.synchronize()
    assert bool((sel[:, :, n] == 99).all())
    got = sel[:, :, :n].cpu()
    assert torch.equal(cnt.cpu(), want[1])
    if values == "nan":
        assert bool((got[..., 1:] > got[..., :-1]).all()) and int(got.max()) <= (t + n) // L and int(got.min()) == 0
    else:
        assert torch.equal(got, want[0])


def test_select_longer_contexts_count_as_t_max(dev):
    gen, rng = torch.Generator().manual_seed(7), random.Random(7)
    s = shape_of(2, 1, 1, 6, 1000, 5)
    f, kc = exact_rows(gen, 2, 1, 5, D), exact_rows(gen, 2, 1, s.nc_cap, D)
    parent = trees(rng, 2, 5, "wide")
    want = ref.select(f, kc, (1000, 700), parent, 6, 1, 2, (64, 64))
    sel = torch.empty(2, 1, 5, 6, dtype=torch.int16, device=dev)
    cnt = torch.empty(2, 1, 5, dtype=torch.int16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, 5, 1000))
    sp.sparda_tree_select(s, f.to(dev), 5, torch.tensor([2000000000, 700], dtype=torch.int32, device=dev), 1000,
                          parent.to(dev), kc.to(dev), sel, cnt, ws)
    assert torch.equal(sel.cpu(), want[0]) and torch.equal(cnt.cpu(), want[1])


# ---- attention ---------------------------------------------------------------------------------------

ATTN = [
    # t_ctx per sequence, nodes, tree, kv heads, group, k, shared
    ((0,), 1, "chain", 1, 1, 3, True),               # no context: the node alone
    ((0, 1, 63, 64, 65), 3, "chain", 1, 4, 3, False),
    ((100,), 1, "chain", 8, 4, 4, False),            # one token
    ((129, 500, -1), 16, "wide", 2, 1, 4, False),    # an absent sequence
    ((700, 640), 5, "wide", 2, 3, 6, True),
    ((700, 641), 13, "wide", 1, 5, 6, False),
    ((1000,), 64, "wide", 2, 16, 9, False),          # 1024 query rows
    ((1000,), 64, "chain", 1, 7, 9, True),
    ((1030,), 64, "star", 1, 2, 9, False),
    ((4000, 3001), 8, "wide", 2, 4, 16, False),
    ((3000, 2000, 2999, 77), 27, "wide", 2, 4, 20, False),
    ((9000,), 33, "wide", 1, 12, 130, False),        # lists that pass two wavefronts' entries
    ((9000, 4000), 9, "wide", 1, 16, 141, True),
    ((140000,), 6, "wide", 1, 4, 70, False),         # more than 2048 blocks
]


def attn_inputs(case, seed=0):
    t_ctx, n, kind, H, G, k, shared = case
    gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
    B, t_max = len(t_ctx), max(max(t_ctx), 0)
    s = shape_of(B, H, G, k, t_max, n)
    q = torch.randn(B, H * G, n, D, generator=gen).to(torch.bfloat16)
    kk, vv = (torch.randn(B, H, s.t_cap, D, generator=gen).to(torch.bfloat16) for _ in range(2))
    kt, vt = (torch.randn(B, H, n, D, generator=gen).to(torch.bfloat16) for _ in range(2))
    parent = trees(rng, B, n, kind, pad=[(0, n - 1, n - 1)] if n > 2 else [])
    ns = 1 if shared else n
    sel, cnt = torch.full((B, H, ns, k), -1, dtype=torch.int16), torch.zeros(B, H, ns, dtype=torch.int16)
    for b in range(B):
        nb = max(1, -(-max(t_ctx[b], 0) // L))
        for h in range(H):
            hot = rng.sample(range(nb), min(nb, k + 3))  # the nodes share most of their blocks
            for i in range(ns):
                got = rng.sample(hot, rng.randrange(1, min(len(hot), k) + 1))
                if len(got) + 3 <= k:  # entries that must not count: a repeat, one past the context, a negative one
                    got += [got[0], min(nb + 1, s.t_cap // L - 1) if nb * L >= t_ctx[b] else got[0], -5]
                rng.shuffle(got)
                sel[b, h, i, :len(got)] = torch.tensor(got, dtype=torch.int16)
                cnt[b, h, i] = len(got)
    return s, t_max, t_ctx, n, q, kk, vv, kt, vt, parent, sel, cnt


def run_attn(dev, x, scale=ref.SCALE, stream=None):
    s, t_max, t_ctx, n, q, k, v, kt, vt, parent, sel, cnt = x
    o = torch.full(q.shape, NAN, dtype=torch.bfloat16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, t_max))
    d = [y.to(dev) for y in (q, parent, k, v, kt, vt, sel, cnt)]
    t = torch.tensor(t_ctx, dtype=torch.int32, device=dev)
    sp.sparda_tree_attn(s, d[0], n, t, t_max, d[1], d[2], d[3], d[4], d[5], sel.shape[2], d[6], d[7], scale, o, ws)
    torch.cuda.synchronize()
    return o.cpu()


def check_attn(o, x, scale=ref.SCALE):
    s, t_max, t_ctx, n, q, k, v, kt, vt, parent, sel, cnt = x
    want, w = ref.attn(q, k, v, kt, vt, t_ctx, parent, sel, cnt, scale)
    off, bar = (o.double() - want).abs(), ref.attn_bar(want, w)
    assert not torch.isnan(o).any()
    worst = float((off / bar).max())
    say(f"  worst error {worst:.3f} of the bar")
    assert worst <= 1.0
    return want


@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attn(dev, case):
    say("tree attention", ATTN[case])
    x = attn_inputs(ATTN[case], case)
    check_attn(run_attn(dev, x), x)


@pytest.mark.parametrize("case", [1, 5, 6, 10])
def test_attn_ignores_what_it_must(dev, case):
    """NaN in the caches from t_ctx on, in blocks that nobody lists and in the rows of absent nodes."""
    say("tree attention beside NaN", ATTN[case])
    x = list(attn_inputs(ATTN[case], 50 + case))
    plain = run_attn(dev, x)
    s, t_max, t_ctx, n, q, k, v, kt, vt, parent, sel, cnt = x
    for b, t in enumerate(t_ctx):
        listed = {int(j) for j in sel[b].flatten() if j >= 0}
        for j in range(s.t_cap // L):
            if j not in listed:
                k[b, :, j * L:j * L + L] = v[b, :, j * L:j * L + L] = NAN
        k[b, :, max(t, 0):] = v[b, :, max(t, 0):] = NAN
        for i, up in enumerate(ref.paths(parent[b].tolist())):
            if not up:
                kt[b, :, i] = vt[b, :, i] = q[b, :, i] = NAN
    assert torch.equal(run_attn(dev, x).view(torch.int16), plain.view(torch.int16))


def test_attn_scales_and_extremes(dev):
    """Weights that underflow, one that dominates, a scale of zero and a negative one, scores of -inf."""
    for case, scale, big in ((5, 4.0, 1.0), (5, 0.0, 1.0), (10, -ref.SCALE, 1.0), (6, ref.SCALE, 6.0)):
        say("tree attention scale", scale, "inputs times", big)
        x = list(attn_inputs(ATTN[case], 70 + case))
        x[4] = (x[4].float() * big).to(torch.bfloat16)
        s, t_max, t_ctx, n, q, k, v, kt, vt, parent, sel, cnt = x
        want, w = ref.attn(q, k, v, kt, vt, t_ctx, parent, sel, cnt, scale)
        # float32 logits of size z are off by at most 130 roundings of their terms' sum, a weight by as much again
        z = 128 * float(q.abs().max()) * float(k.abs().max()) * abs(scale)
        off = (run_attn(dev, x, scale).double() - want).abs()
        bar = ref.attn_bar(want, w) + 2 * min(1.0, 130 * 2.0 ** -24 * z) * w
        assert float((off / bar).max()) <= 1.0
    x = list(attn_inputs(ATTN[10], 5))
    x[5][:, :, ::3] = -float("inf")  # keys of -inf: scores of -inf or NaN are the inputs' own; with q > 0 all are -inf
    x[4] = x[4].abs() + 0.5
    s, t_max, t_ctx, n, q, k, v, kt, vt, parent, sel, cnt = x
    q = x[4] = q.to(torch.bfloat16)
    want, w = ref.attn(q, k, v, kt, vt, t_ctx, parent, sel, cnt, ref.SCALE)
    off = (run_attn(dev, x).double() - want).abs()
    assert float((off / ref.attn_bar(want, w)).max()) <= 1.0


# Calls whose blocks exceed the last-level cache share them between the wavefronts of a workgroup: 64, 128 or 256
# columns (node, query head) each.  Only some groups are compared.
MANY = [
    # nodes, tree, group, k, t, one list; 1024 groups, or as many as said
    (16, "wide", 4, 9, 700, False),    # 64 columns
    (13, "wide", 3, 9, 700, True),     # 39 of 64
    (21, "chain", 5, 9, 1000, False),  # 105 of 128
    (31, "wide", 4, 9, 640, True),     # 124 of 128
    (40, "wide", 4, 9, 700, False),    # 160 of 256
    (64, "wide", 7, 9, 700, False),    # 448 in two tiles of 256
    (33, "star", 16, 9, 700, True),    # 528 in three, the last of 16
    (16, "wide", 4, 260, 140000, True, 1, 32),  # more than 2048 blocks
]


@pytest.mark.parametrize("case", range(len(MANY)))
def test_attn_many_groups(dev, case):
    n, kind, G, k, t, shared, B, H = (MANY[case] + (4, 256))[:8]
    say("tree attention of many groups", MANY[case])
    gen, rng = torch.Generator(device=dev).manual_seed(case), random.Random(case)
    s = shape_of(B, H, G, k, t, n)
    mk = lambda *size: torch.randn(*size, generator=gen, device=dev, dtype=torch.bfloat16)  # noqa: E731
    q, kk, vv, kt, vt = mk(B, H * G, n, D), mk(B, H, s.t_cap, D), mk(B, H, s.t_cap, D), mk(B, H, n, D), mk(B, H, n, D)
    t_ctx = [t, t - 63, -1, t - 200][:B]
    for b in range(B):
        kk[b, :, max(t_ctx[b], 0):] = vv[b, :, max(t_ctx[b], 0):] = NAN
    parent = trees(rng, B, n, kind, pad=[(B - 1, n - 1, n)])
    ns, nb = (1 if shared else n), -(-t // L)
    sel = torch.rand(B, H, ns, nb, generator=gen, device=dev).topk(k - 1, dim=3).indices.to(torch.int16)
    sel = torch.cat((sel, sel[..., :1]), 3).contiguous()  # one entry twice
    cnt = torch.randint(0, k + 1, (B, H, ns), generator=gen, device=dev).to(torch.int16)
    o = torch.full(q.shape, NAN, dtype=torch.bfloat16, device=dev)
    ws = workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, t))
    sp.sparda_tree_attn(s, q, n, torch.tensor(t_ctx, dtype=torch.int32, device=dev), t, parent.to(dev), kk, vv, kt, vt,
                        ns, sel, cnt, ref.SCALE, o, ws)
    torch.cuda.synchronize()
    assert not torch.isnan(o).any() and not o[2:3].any()
    for h in (0, 7, H // 2, H - 1):
        x = [y[:, h:h + 1].cpu() for y in (kk, vv, kt, vt, sel, cnt)]
        want, w = ref.attn(q[:, h * G:(h + 1) * G].cpu(), *x[:4], t_ctx, parent, *x[4:], ref.SCALE)
        off = (o[:, h * G:(h + 1) * G].cpu().double() - want).abs()
        assert float((off / ref.attn_bar(want, w)).max()) <= 1.0


# ---- verify -------------------------------------------------------------------------------------------

VERIFY = [
    # batch, nodes, tree, vocab, extra elements per row, with q, bf16
    (1, 1, "chain", 1, 0, False, False),
    (3, 1, "chain", 17, 0, True, True),
    (5, 6, "chain", 5, 0, True, False),
    (5, 6, "chain", 33, 3, False, True),
    (7, 64, "star", 40, 1, False, False),
    (7, 64, "star", 40, 1, True, False),
    (9, 21, "wide", 1000, 0, True, True),
    (9, 64, "wide", 4097, 7, True, False),
    (4, 27, "wide", 50021, 0, False, False),
    (4, 27, "wide", 50021, 2, True, True),
    (2, 64, "wide", 131072, 0, False, False),
    (300, 5, "wide", 4099, 0, True, False),
]


def verify_inputs(case, seed=0, sharp=3.0, near=0.7):
    B, n, kind, V, extra, with_q, bf16 = case
    gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
    dt = torch.bfloat16 if bf16 else torch.float32
    z = torch.randn(B, n, V + extra, generator=gen) * sharp
    p = torch.softmax(z, 2).to(dt)
    q = torch.softmax(z + near * torch.randn(B, n, V + extra, generator=gen), 2).to(dt)
    parent = trees(rng, B, n, kind)
    tokens = torch.zeros(B, n, dtype=torch.int32)
    for b in range(B):
        for i in range(1, n):
            tokens[b, i] = int(torch.multinomial(q[b, parent[b, i], :V].float(), 1, generator=gen))
    return p, (q if with_q else None), tokens, parent, torch.rand(B, n, generator=gen)


def run_verify(dev, case, p, q, tokens, parent, u):
    B, n, kind, V, extra, with_q, bf16 = case
    s = sp.SpardaShape(batch=B, n_kv_heads=1, group_size=1, k_total=3, t_cap=64, nc_cap=1)
    path = torch.full((B, n), 77, dtype=torch.int32, device=dev)
    n_path, nxt = (torch.full((B,), 77, dtype=torch.int32, device=dev) for _ in range(2))
    ws = workspace(dev, sp.sparda_tree_verify_workspace_size(s, n, V))
    kind = sp.SPARDA_PROB_BF16 if p.dtype == torch.bfloat16 else sp.SPARDA_PROB_F32
    d = [None if y is None else y.to(dev) for y in (p, q, tokens, parent, u)]
    sp.sparda_tree_verify(s, n, V, p.shape[2], kind, *d, path, n_path, nxt, ws)
    torch.cuda.synchronize()
    return path.cpu(), n_path.cpu(), nxt.cpu()


def check_verify(dev, case, x):
    got, want = run_verify(dev, case, *x), ref.verify(*x, case[3])
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    return got


@pytest.mark.parametrize("case", range(len(VERIFY)))
def test_verify(dev, case):
    say("tree verify", VERIFY[case])
    x = verify_inputs(VERIFY[case], case)
    got = check_verify(dev, VERIFY[case], x)
    say(f"  mean path {got[1].float().mean():.2f}")


@pytest.mark.parametrize("with_q", [False, True])
def test_verify_edges(dev, with_q):
    """Random numbers at both ends, tokens outside the vocabulary, absent nodes and trees, equal tokens among siblings,
    one-hot rows, rows without weight, NaN, infinite and negative entries."""
    case = (12, 16, "wide", 301, 2, with_q, False)
    p, q, tokens, parent, u = verify_inputs(case, 5, sharp=2.0)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    tokens[2, 1::3] = -1
    tokens[2, 2::3] = 301
    parent[3, 4], parent[3, 9] = 4, -1
    parent[4, 0] = 0
    parent[5] = torch.tensor([-1] + [0] * 15)
    tokens[5] = tokens[5, 1]
    p[6] = 0
    p[6, :, 100] = 1
    p[7] = 0
    p[8, :, 3:40] = NAN
    p[8, :, 40:50] = float("inf")
    p[8, :, 50:60] = -1
    if q is not None:
        p[9] = q[9] * 0.5  # a rejection would leave no weight
        u[9] = 0.9
        q[10, :, 5] = float("inf")
        q[11] = 0
    parent[11] = torch.tensor([-1] + [0] * 15)
    p[11] = 0
    p[11, :, 7] = 2.0 ** -30  # all the weight there is lies on the token that is rejected last
    tokens[11] = 9
    tokens[11, 15] = 7
    u[11] = 0.5
    check_verify(dev, case, (p, q, tokens, parent, u))


def test_verify_many_draws(dev):
    """20000 sequences of one small tree: the kept tokens are distributed as the target's own.  The counts of the
    first token after the root are within 5 standard deviations of the target's, for draws from q and for chosen
    tokens."""
    B, n, V = 20000, 5, 7
    gen = torch.Generator().manual_seed(11)
    z = torch.randn(1, n, V, generator=gen)
    p = torch.softmax(z * 1.5, 2).expand(B, n, V).contiguous()
    q = torch.softmax(torch.randn(1, n, V, generator=gen), 2).expand(B, n, V).contiguous()
    parent = torch.tensor([[-1, 0, 0, 0, 1]], dtype=torch.int32).expand(B, n).contiguous()
    for with_q in (True, False):
        tokens = torch.zeros(B, n, dtype=torch.int32)
        for i in range(1, n):
            row = q[:, int(parent[0, i])]
            tokens[:, i] = torch.multinomial(row, 1, generator=gen).squeeze(1).int() if with_q else (2 * i) % V
        u = torch.rand(B, n, generator=gen)
        case = (B, n, "", V, 0, with_q, False)
        path, n_path, nxt = run_verify(dev, case, p, q if with_q else None, tokens, parent, u)
        first = torch.where(n_path > 1, tokens.gather(1, path[:, 1:2].clamp_min(0).long()).squeeze(1), nxt)
        count = torch.bincount(first.long(), minlength=V).double()
        want = p[0, 0].double() * B
        assert bool(((count - want).abs() <= 5 * (want * (1 - want / B)).sqrt()).all())


# ---- commit -----------------------------------------------------------------------------------------------

COMMIT = [
    # t_ctx per sequence, accepted, nodes, kv heads, layers, grid, t_cap
    ((0,), (1,), 1, 1, 1, (64, 64), 64),
    ((0, 63, 64, 127), (1, 1, 2, 3), 8, 2, 1, (64, 64), 192),
    ((0, 30, 31, 47, 100), (64, 1, 2, 17, 50), 64, 1, 2, (32, 16), 192),
    ((10, -1, 50, 60), (5, 3, 0, 64), 64, 2, 3, (64, 64), 128),   # an absent one, none accepted, past the cache
    ((500, 511, 400), (7, 16, 1), 16, 8, 35, (32, 16), 576),      # layers in two launches
]


@pytest.mark.parametrize("case", range(len(COMMIT)))
@pytest.mark.parametrize("with_kc", [True, False])
def test_commit(dev, case, with_kc):
    t_ctx, acc, n, H, layers, grid, t_cap = COMMIT[case]
    say("tree commit", COMMIT[case], with_kc)
    gen, rng = torch.Generator().manual_seed(case), random.Random(case)
    B = len(t_ctx)
    s = shape_of(B, H, 1, 3, 0, n, grid=grid, t_cap=t_cap)
    path = torch.full((B, n), -1, dtype=torch.int32)
    for b in range(B):
        got = sorted([0] + rng.sample(range(1, n), min(max(acc[b], 1), n) - 1))
        path[b, :len(got)] = torch.tensor(got, dtype=torch.int32)
    if case == 4:
        path[1, 5] = n  # dropped from here on
    n_path, t = torch.tensor(acc, dtype=torch.int32), torch.tensor(t_ctx, dtype=torch.int32)
    sets = [[torch.randn(*size, generator=gen).to(torch.bfloat16) for _ in range(layers)] for size in
            ((B, H, n, D), (B, H, n, D), (B, H, t_cap, D), (B, H, t_cap, D), (B, H, s.nc_cap, D))]
    on = [[y.to(dev) for y in z] for z in sets]
    t_new = torch.full((B,), 7, dtype=torch.int32, device=dev)
    sp.sparda_tree_commit(s, n, t.to(dev), path.to(dev), n_path.to(dev), layers, on[0], on[1],
                          sp.layer_pointers(on[2]), on[3], on[4] if with_kc else None, t_new)
    torch.cuda.synchronize()
    for x in range(layers):
        kt, vt, k, v, kc = (z[x] for z in sets)
        want = ref.commit(t, path, n_path, kt, vt, k, v, kc if with_kc else None, grid)
        for g, w in zip((z[x] for z in on[2:]), (k, v, kc)):
            assert torch.equal(g.cpu().view(torch.int16), w.view(torch.int16))
    assert torch.equal(t_new.cpu(), want)


# ---- together -----------------------------------------------------------------------------------------------

class Model:
    """A toy layer for a decode loop: token, position -> Forecast row, query, K and V, and a distribution of the next
    token read off the attention's output."""

    def __init__(self, dev, H, G, V, seed):
        gen = torch.Generator().manual_seed(seed)
        self.H, self.G, self.V, self.dev = H, G, V, dev
        mk = lambda *size: torch.randn(*size, generator=gen)  # noqa: E731
        self.f, self.k = exact_rows(gen, V, H, D).to(dev), exact_rows(gen, V, H, D).to(dev)
        self.q, self.v = mk(V, H * G, D).to(torch.bfloat16).to(dev), mk(V, H, D).to(torch.bfloat16).to(dev)
        self.head = (mk(H * G * D, V) * 0.05).to(dev)

    def rows(self, table, tokens):  # [B][n] -> [B][heads][n][D]
        return table[tokens.long()].transpose(1, 2).contiguous()

    def probs(self, o):  # [B][Hq][n][D] -> [B][n][V]
        x = o.transpose(1, 2).reshape(o.shape[0], o.shape[2], -1).float()
        return torch.softmax(x @ self.head, 2)


def decode_row(m, shape, caches, t, token):
    """One ordinary decode step of one sequence at position t with the framework's own calls; the token is appended."""
    k, v, kc = caches
    tok = torch.tensor([[token]], device=m.dev)
    k[:, :, t], v[:, :, t] = m.rows(m.k, tok)[:, :, 0], m.rows(m.v, tok)[:, :, 0]
    sel = torch.empty(1, m.H, 1, shape.k_total, dtype=torch.int16, device=m.dev)
    cnt = torch.empty(1, m.H, 1, dtype=torch.int16, device=m.dev)
    o = torch.empty(1, m.H * m.G, 1, D, dtype=torch.bfloat16, device=m.dev)
    ws = workspace(m.dev, sp.sparda_workspace_size(shape, sp.SPARDA_OP_DECODE_STEP, 1, t))
    sp.sparda_decode_step(shape, m.rows(m.f, tok), t, kc, m.rows(m.q, tok), k, v, ref.SCALE, sel, cnt, o, ws)
    l, st = shape.cmp_kernel, shape.cmp_stride
    w1 = (t + 1 - l) // st + 1 if t + 1 >= l else 0
    w0 = (t - l) // st + 1 if t >= l else 0
    sp.sparda_compress_keys(shape, k, t + 1, w0, w1, kc)
    return sel, cnt, o


@pytest.mark.parametrize("grid", [(64, 64), (32, 16)])
def test_steps_together_follow_ordinary_decode(dev, grid):
    """Several steps of select, attend, verify, commit on a batch whose lengths drift apart.  Along every accepted path
    the sets are those of ordinary decode steps (bit for bit, up to a window that straddles the context), the outputs
    are within the bar of the definition, and the caches, K~ and lengths end up the same."""
    B, H, G, V, n, k = 3, 2, 4, 50, 13, 7
    rng = random.Random(3)
    m = Model(dev, H, G, V, 9)
    t0 = [600, 655, 707]
    t_cap = 1024
    s = shape_of(B, H, G, k, 0, n, grid=grid, t_cap=t_cap)
    one = shape_of(1, H, G, k, 0, n, grid=grid, t_cap=t_cap)
    gen = torch.Generator().manual_seed(4)
    prompt = torch.randint(0, V, (B, t_cap), generator=gen).to(dev)
    kc0 = torch.zeros(B, H, s.nc_cap, D, dtype=torch.bfloat16, device=dev)
    kk, vv = m.rows(m.k, prompt), m.rows(m.v, prompt)
    for b in range(B):
        kk[b, :, t0[b]:] = NAN
        vv[b, :, t0[b]:] = NAN
        w = (t0[b] - grid[0]) // grid[1] + 1
        sp.sparda_compress_keys(one, kk[b:b + 1].contiguous(), t0[b], 0, w, kc0[b:b + 1])
    k1, v1, kc1 = kk.clone(), vv.clone(), kc0.clone()           # ordinary decode
    root = torch.randint(0, V, (B,), generator=gen).int()
    t = torch.tensor(t0, dtype=torch.int32, device=dev)
    total = 0
    for step in range(8):
        parent = trees(rng, B, n, "wide").to(dev)
        tokens = torch.randint(0, V, (B, n), generator=gen).int()
        tokens[:, 0] = root
        tokens = tokens.to(dev)
        t_max = int(t.max())
        f, q, kt, vt = (m.rows(x, tokens) for x in (m.f, m.q, m.k, m.v))
        sel = torch.empty(B, H, n, k, dtype=torch.int16, device=dev)
        cnt = torch.empty(B, H, n, dtype=torch.int16, device=dev)
        o = torch.full((B, H * G, n, D), NAN, dtype=torch.bfloat16, device=dev)
        sp.sparda_tree_select(s, f, n, t, t_max, parent, kc0, sel, cnt,
                              workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, n, t_max)))
        sp.sparda_tree_attn(s, q, n, t, t_max, parent, kk, vv, kt, vt, n, sel, cnt, ref.SCALE, o,
                            workspace(dev, sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, t_max)))
        p = m.probs(o)
        # small numbers accept tokens of ordinary weight, so that paths get long
        u = torch.rand(B, n, generator=gen).to(dev) * 0.02
        path = torch.empty(B, n, dtype=torch.int32, device=dev)
        n_path, nxt, t_new = (torch.empty(B, dtype=torch.int32, device=dev) for _ in range(3))
        sp.sparda_tree_verify(s, n, V, V, sp.SPARDA_PROB_F32, p, None, tokens, parent, u, path, n_path, nxt,
                              workspace(dev, sp.sparda_tree_verify_workspace_size(s, n, V)))
        sp.sparda_tree_commit(s, n, t, path, n_path, 1, [kt], [vt], [kk], [vv], [kc0], t_new)
        torch.cuda.synchronize()
        want = ref.verify(p.cpu(), None, tokens.cpu(), parent.cpu(), u.cpu(), V)
        assert torch.equal(path.cpu(), want[0]) and torch.equal(n_path.cpu(), want[1]) and torch.equal(nxt.cpu(), want[2])
        for b in range(B):
            tb, view = int(t[b]), [x[b:b + 1] for x in (k1, v1, kc1)]
            for x in range(int(n_path[b])):
                node = int(path[b, x])
                s1, c1, o1 = decode_row(m, one, view, tb + x, int(tokens[b, node]))
                straddles = grid[1] < 64 and tb // L != (tb + x) // L and tb % L < 16
                if not straddles:
                    assert torch.equal(s1[0, :, 0], sel[b, :, node]) and torch.equal(c1[0, :, 0], cnt[b, :, node])
                    at = [y[b:b + 1, :, node:node + 1].cpu() for y in (q, kt, vt)]
                    want_o, w = ref.attn(at[0], view[0].cpu(), view[1].cpu(), at[1], at[2], [tb + x],
                                         torch.tensor([[-1]]), s1.cpu(), c1.cpu(), ref.SCALE)
                    for got in (o1[0, :, 0], o[b, :, node]):
                        gap = (got.double().cpu() - want_o[0, :, 0]).abs()
                        assert bool((gap <= ref.attn_bar(want_o[0, :, 0], w[0, :, 0])).all())
                total += 1
        t, root = t_new, nxt.cpu()
        for b in range(B):
            e = int(t[b])
            assert torch.equal(kk[b, :, :e].view(torch.int16), k1[b, :, :e].view(torch.int16))
            assert torch.equal(vv[b, :, :e].view(torch.int16), v1[b, :, :e].view(torch.int16))
            w = (e - grid[0]) // grid[1] + 1
            assert torch.equal(kc0[b, :, :w].view(torch.int16), kc1[b, :, :w].view(torch.int16))
    say(f"  {total} tokens in 8 steps of {B} sequences, lengths {t.tolist()}")
    assert total > 8 * B


def test_captured_step_replays(dev):
    """One step captured into a graph on a side stream and replayed with other lengths, trees and probabilities, with
    eager steps on the same buffers' copies in between: every replay gives the eager results."""
    B, H, G, n, k, V, t_cap = 2, 2, 4, 11, 6, 3000, 2048
    s = shape_of(B, H, G, k, 0, n, t_cap=t_cap)
    t_max, rng = 1500, random.Random(1)
    gen = torch.Generator(device=dev).manual_seed(1)
    mk = lambda *size: torch.randn(*size, generator=gen, device=dev, dtype=torch.bfloat16)  # noqa: E731
    x = {"f": mk(B, H, n, D), "q": mk(B, H * G, n, D), "kt": mk(B, H, n, D), "vt": mk(B, H, n, D),
         "k": mk(B, H, t_cap, D), "v": mk(B, H, t_cap, D), "kc": mk(B, H, s.nc_cap, D),
         "t": torch.zeros(B, dtype=torch.int32, device=dev), "parent": trees(rng, B, n, "wide").to(dev),
         "p": torch.softmax(torch.randn(B, n, V, generator=gen, device=dev), 2),
         "pq": torch.softmax(torch.randn(B, n, V, generator=gen, device=dev), 2),
         "tok": torch.zeros(B, n, dtype=torch.int32, device=dev), "u": torch.rand(B, n, generator=gen, device=dev)}

    def outputs():
        i32 = dict(dtype=torch.int32, device=dev)
        return {"sel": torch.empty(B, H, n, k, dtype=torch.int16, device=dev), "o": torch.empty_like(x["q"]),
                "cnt": torch.empty(B, H, n, dtype=torch.int16, device=dev), "path": torch.empty(B, n, **i32),
                "n_path": torch.empty(B, **i32), "next": torch.empty(B, **i32), "t_new": torch.empty(B, **i32),
                "ws": [workspace(dev, b) for b in (sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, n, t_max),
                                                   sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_ATTN, n, t_max),
                                                   sp.sparda_tree_verify_workspace_size(s, n, V))]}

    def step(x, y):
        sp.sparda_tree_select(s, x["f"], n, x["t"], t_max, x["parent"], x["kc"], y["sel"], y["cnt"], y["ws"][0])
        sp.sparda_tree_attn(s, x["q"], n, x["t"], t_max, x["parent"], x["k"], x["v"], x["kt"], x["vt"], n, y["sel"],
                            y["cnt"], ref.SCALE, y["o"], y["ws"][1])
        sp.sparda_tree_verify(s, n, V, V, sp.SPARDA_PROB_F32, x["p"], x["pq"], x["tok"], x["parent"], x["u"], y["path"],
                              y["n_path"], y["next"], y["ws"][2])
        sp.sparda_tree_commit(s, n, x["t"], y["path"], y["n_path"], 1, [x["kt"]], [x["vt"]], [x["k"]], [x["v"]],
                              [x["kc"]], y["t_new"])

    def vary(i):
        x["t"].copy_(torch.tensor([1500 - 37 * i, 3 + 300 * i], dtype=torch.int32))
        x["parent"].copy_(trees(rng, B, n, "chain" if i == 2 else "wide"))
        x["p"].copy_(torch.softmax(torch.randn(B, n, V, generator=gen, device=dev) * 2, 2))
        x["tok"].copy_(torch.randint(0, V, (B, n), generator=gen, device=dev))
        x["u"].copy_(torch.rand(B, n, generator=gen, device=dev) * 0.3)

    side = torch.cuda.Stream()
    y = outputs()
    vary(0)
    with torch.cuda.stream(side):
        step(x, y)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(x, y)
    for i in range(5):
        vary(i)
        torch.cuda.synchronize()
        alone, out = {a: b.clone() for a, b in x.items()}, outputs()
        g.replay()
        torch.cuda.synchronize()
        step(alone, out)
        torch.cuda.synchronize()
        for a in ("sel", "cnt", "o", "path", "n_path", "next", "t_new"):
            assert torch.equal(y[a], out[a]), (i, a)
        for a in ("k", "v", "kc"):
            assert torch.equal(x[a].view(torch.int16), alone[a].view(torch.int16)), (i, a)
        y["o"].fill_(NAN)
