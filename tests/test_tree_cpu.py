"""Trees of drafted tokens without a GPU: refusals of the entry points (nothing is launched), workspace sizes, and
checks of the float64 definitions that the GPU tests compare with."""
import itertools
import os
import random

import pytest
import torch

import paper_2606_04511_amd.sparda as sp
import tree_reference as ref

FAKE = 0x7F0000000000  # aligned, never dereferenced: validation fails before any launch
BAD, UNSUP, WS = sp.SPARDA_ERR_INVALID_ARG, sp.SPARDA_ERR_UNSUPPORTED, sp.SPARDA_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(sp.library_path()):
        from paper_2606_04511_amd import build
        build.build()
    return sp.load()


def shape(**kw):
    base = dict(batch=2, n_kv_heads=8, group_size=4, k_total=16, t_cap=8192, nc_cap=128)
    base.update(kw)
    return sp.SpardaShape(**base)


def rc_of(fn, *args):
    with pytest.raises(sp.SpardaError) as ei:
        fn(*args)
    assert sp.last_error_detail() != ""
    return ei.value.status


def replaced(args, **at):
    """args with the named positions replaced ("a3": position 3)."""
    out = list(args)
    for k, v in at.items():
        out[int(k[1:])] = v
    return out


def test_select_refusals():
    f = sp.sparda_tree_select
    s = shape()
    big = 1 << 40
    good = [s, FAKE, 8, FAKE, 4000, FAKE, FAKE, FAKE, FAKE, FAKE, big, 0]
    for at, status in ((dict(a0=shape(head_dim=64)), UNSUP), (dict(a0=shape(n_local=1)), UNSUP), (dict(a1=None), BAD),
                       (dict(a1=FAKE + 8), BAD), (dict(a2=0), BAD), (dict(a2=65), UNSUP), (dict(a3=None), BAD),
                       (dict(a3=FAKE + 2), BAD), (dict(a4=-1), BAD), (dict(a4=8185), BAD), (dict(a5=None), BAD),
                       (dict(a5=FAKE + 1), BAD), (dict(a6=None), BAD), (dict(a7=FAKE + 1), BAD), (dict(a8=None), BAD),
                       (dict(a9=None), WS), (dict(a9=FAKE + 4), WS), (dict(a10=1024), WS),
                       (dict(a0=shape(nc_cap=60)), BAD)):
        assert rc_of(f, *replaced(good, **at)) == status, at


def test_attn_refusals():
    f = sp.sparda_tree_attn
    big = 1 << 40
    good = [shape(), FAKE, 8, FAKE, 4000, FAKE, FAKE, FAKE, FAKE, FAKE, 8, FAKE, FAKE, 0.1, FAKE, FAKE, big, 0]
    for i in (1, 6, 7, 8, 9, 14):
        assert rc_of(f, *replaced(good, **{f"a{i}": None})) == BAD
        assert rc_of(f, *replaced(good, **{f"a{i}": FAKE + 8})) == BAD
    for i, off in ((3, 2), (5, 2), (11, 1), (12, 1)):
        assert rc_of(f, *replaced(good, **{f"a{i}": None})) == BAD
        assert rc_of(f, *replaced(good, **{f"a{i}": FAKE + off})) == BAD
    for at, status in ((dict(a2=0), BAD), (dict(a2=65), UNSUP), (dict(a4=-1), BAD), (dict(a4=8190), BAD),
                       (dict(a10=2), BAD), (dict(a10=0), BAD), (dict(a13=float("nan")), BAD),
                       (dict(a13=float("inf")), BAD)):
        assert rc_of(f, *replaced(good, **at)) == status, at
    need = sp.sparda_workspace_size(shape(), sp.SPARDA_OP_TREE_ATTN, 8, 4000)
    if need:
        for at in (dict(a15=None), dict(a15=FAKE + 8), dict(a16=need - 1)):
            assert rc_of(f, *replaced(good, **at)) == WS


def test_verify_refusals():
    f = sp.sparda_tree_verify
    s = shape()
    need = sp.sparda_tree_verify_workspace_size(s, 8, 1000)
    good = [s, 8, 1000, 1000, sp.SPARDA_PROB_F32, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, 0]
    for at, status in ((dict(a1=0), BAD), (dict(a1=65), UNSUP), (dict(a2=0), BAD), (dict(a3=999), BAD),
                       (dict(a4=2), BAD), (dict(a4=-1), BAD), (dict(a5=None), BAD), (dict(a5=FAKE + 4), BAD),
                       (dict(a6=FAKE + 4), BAD), (dict(a13=None), WS), (dict(a13=FAKE + 8), WS),
                       (dict(a14=need - 1), WS)):
        assert rc_of(f, *replaced(good, **at)) == status, at
    for i in range(7, 13):
        assert rc_of(f, *replaced(good, **{f"a{i}": None})) == BAD
        assert rc_of(f, *replaced(good, **{f"a{i}": FAKE + 2})) == BAD
    assert rc_of(sp.sparda_tree_verify_workspace_size, s, 65, 10) == UNSUP
    assert rc_of(sp.sparda_tree_verify_workspace_size, s, 1, 0) == BAD


def test_commit_refusals():
    f = sp.sparda_tree_commit
    tab = [FAKE, FAKE + 16]
    good = [shape(), 8, FAKE, FAKE, FAKE, 2, tab, tab, tab, tab, tab, FAKE + 4, 0]
    for at, status in ((dict(a1=0), BAD), (dict(a1=65), UNSUP), (dict(a2=None), BAD), (dict(a3=None), BAD),
                       (dict(a4=FAKE + 1), BAD), (dict(a5=0, a6=[], a7=[], a8=[], a9=[], a10=[]), BAD),
                       (dict(a11=None), BAD), (dict(a11=FAKE), BAD)):
        assert rc_of(f, *replaced(good, **at)) == status, at
    for i in range(6, 11):
        assert rc_of(f, *replaced(good, **{f"a{i}": [FAKE, None]})) == BAD
        assert rc_of(f, *replaced(good, **{f"a{i}": [FAKE, FAKE + 8]})) == BAD
    for i in range(6, 10):
        assert rc_of(f, *replaced(good, **{f"a{i}": None})) == BAD
    with pytest.raises(ValueError):
        f(*replaced(good, a6=[FAKE]))


def test_workspace_sizes():
    s = shape(t_cap=131072, nc_cap=2048, k_total=64)
    # block scores of every node, the longest context's candidates padded to 4
    assert sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, 16, 131000) == 2 * 8 * 16 * 2048 * 4
    assert sp.sparda_workspace_size(s, sp.SPARDA_OP_TREE_SELECT, 16, 100) == 0
    for op in (sp.SPARDA_OP_TREE_SELECT, sp.SPARDA_OP_TREE_ATTN):
        assert rc_of(sp.sparda_workspace_size, s, op, 65, 0) == UNSUP
        assert rc_of(sp.sparda_workspace_size, s, op, 8, 131065) == BAD


def test_layer_tables():
    x = [torch.zeros(4, dtype=torch.bfloat16) for _ in range(3)]
    assert list(sp.layer_pointers(x)) == [y.data_ptr() for y in x]


# ---- the definitions ---------------------------------------------------------------------------------

def test_reference_paths():
    assert ref.paths([-1, 0, 1, 0, 7, 4, -1]) == [[0], [1, 0], [2, 1, 0], [3, 0], [], [], []]
    assert ref.paths([0, 0]) == [[], []]


@pytest.mark.parametrize("with_q", [True, False])
def test_reference_verification_keeps_the_targets_distribution(with_q):
    """The probability of the first kept token, integrated over the random numbers and (with q) over what the
    drafter drew, is the target's: the acceptance tests are intervals of u, so their lengths add up exactly."""
    V = 4
    gen = torch.Generator().manual_seed(2)
    p = torch.softmax(torch.randn(V, generator=gen).double(), 0)
    q = torch.softmax(torch.randn(V, generator=gen).double(), 0)
    got = torch.zeros(V, dtype=torch.float64)
    siblings = 2
    draws = itertools.product(range(V), repeat=siblings) if with_q else [(1, 3)]
    for toks in draws:
        weight = float(torch.stack([q[x] for x in toks]).prod()) if with_q else 1.0
        m, c, left = p.clone(), 1.0, weight
        for x in toks:
            qx = float(q[x]) if with_q else 1.0
            acc = min(1.0, float(m[x]) / (c * qx))
            got[x] += left * acc
            left *= 1 - acc
            m = (m - c * q).clamp_min(0) if with_q else m * (torch.arange(V) != x)
            c = float(m.sum())
        got += left * m / m.sum()
    assert torch.allclose(got, p, atol=1e-12)
    # and the reference takes those intervals: just below and just above the edge of the first test
    P = p.float().expand(1, 3, V).contiguous()
    Q = q.float().expand(1, 3, V).contiguous() if with_q else None
    tok = torch.tensor([[0, 1, 3]], dtype=torch.int32)
    par = torch.tensor([[-1, 0, 0]], dtype=torch.int32)
    edge = float(P[0, 0, 1]) / (float(Q[0, 0, 1]) if with_q else 1.0)
    if edge < 1:
        for u, kept in ((edge - 1e-5, 1), (edge + 1e-5, None)):
            path, n, _ = ref.verify(P, Q, tok, par, torch.tensor([[0.5, u, 0.999]]), V)
            assert (int(path[0, 1]) == 1) == (kept == 1)


def test_reference_attention_is_masked_softmax():
    """The tree attention over blocks of the cache equals a dense masked attention over cache and tree."""
    rng = random.Random(1)
    gen = torch.Generator().manual_seed(1)
    t, n, H, G = 150, 6, 2, 3
    q, k, v = (torch.randn(1, x, y, 128, generator=gen) for x, y in ((H * G, n), (H, 192), (H, 192)))
    kt, vt = (torch.randn(1, H, n, 128, generator=gen) for _ in range(2))
    parent = torch.tensor([ref.tree(rng, n, "wide")])
    sel = torch.tensor([[[[2, 0, 0, -1]] * n, [[1, 7, 2, 0]] * n]], dtype=torch.int16)
    cnt = torch.full((1, H, n), 3, dtype=torch.int16)
    o, _ = ref.attn(q, k, v, kt, vt, [t], parent, sel, cnt, 0.1)
    up = ref.paths(parent[0].tolist())
    for h in range(H):
        blocks = {0, 2} if h == 0 else {1, 2}
        seen = torch.zeros(n, 192 + n, dtype=torch.bool)
        for i in range(n):
            seen[i, :t] = torch.tensor([x // 64 in blocks for x in range(t)])
            seen[i, [192 + x for x in up[i]]] = True
        kk, vv = (torch.cat((a[0, h], b[0, h])).double() for a, b in ((k, kt), (v, vt)))
        z = q[0, h * G:(h + 1) * G].double() @ kk.t() * 0.1
        want = torch.softmax(z.masked_fill(~seen, -float("inf")), 2) @ vv
        assert torch.allclose(o[0, h * G:(h + 1) * G], want, atol=1e-12)
