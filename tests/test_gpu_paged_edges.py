"""Paged operators on the GPU where the larger tests do not reach: compressed keys past 32 bits of elements, all operators behind
work of their own stream, scores of -inf."""
import random

import pytest
import torch

import paged_reference as ref
from test_gpu_paged import (BF, NAN, bits, check, dev, exact_rows, freqs, pools, run_attn, say, shape_of, table_of,  # noqa: F401
                            workspace)
import paper_2606_04511_amd.sparda as sp

pytestmark = pytest.mark.gpu
D, L = 128, 64


@pytest.mark.parametrize("grid,n_pages,H", [((64, 64), 34000, 1), ((32, 16), 4200, 2)])
def test_selection_past_32_bits(dev, grid, n_pages, H):  # noqa: F811
    """Compressed keys of more than 2^32 elements: the sequence's lie in the last pages; all others, which offsets cut to 32 bits would
    reach, hold NaN."""
    page = 65536
    per = page // grid[1]  # keys of a page and head
    assert n_pages * H * per * D > 1 << 32
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of free device memory")
    say("keys", n_pages * H * per * D)
    gen, k, t = torch.Generator().manual_seed(4), 20, 100000
    kc = torch.empty(n_pages, H, per, D, dtype=BF, device=dev)
    kc.fill_(NAN)
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32)
    own = exact_rows(gen, 2, H, per, D)
    for i in range(2):
        kc[int(table[0, i])] = own[i].to(dev)
    f = exact_rows(gen, 1, H, 1, D)
    shape = shape_of(1, H, 1, k, 131072, 1, 2, grid)
    sel, cnt = torch.empty(1, H, 1, k, dtype=torch.int16, device=dev), torch.empty(1, H, 1, dtype=torch.int16, device=dev)
    sp.sparda_paged_select(shape, sp.SpardaPages(page, table.to(dev), k_cmp=kc), f.to(dev), torch.tensor([t], dtype=torch.int32, device=dev),
                           t, sel, cnt, workspace(dev, shape, sp.SPARDA_OP_PAGED_SELECT, t))
    n_win = (t - grid[0]) // grid[1] + 1
    for h in range(H):
        keys = torch.cat((own[0, h], own[1, h]))[:n_win]
        assert sel[0, h, 0].tolist() == ref.selection(f[0, h, 0], keys, t, k, 1, 2, grid), h


def behind(dev, work):  # noqa: F811
    """work(stream) on a side stream behind 20 ms or more of products, while the current stream is idle; what it returns."""
    a = torch.randn(4096, 4096, device=dev)
    b = a @ a
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.mm(a, a, out=b)
    out = work(side)
    assert not side.query()  # the calls have returned before the products ended
    torch.cuda.synchronize()
    return out


def test_calls_wait_for_their_stream(dev):  # noqa: F811
    """Inputs that the given stream writes late: each operator reads them, and its output is read by the next, in that stream alone."""
    B, H, G, k, page, t0, n = 2, 2, 4, 6, 64, 600, 3
    gen, rng = torch.Generator().manual_seed(6), random.Random(6)
    cap, shape = 1024, shape_of(B, H, G, 6, 1024)
    table, n_pages = table_of(rng, B, cap, page)
    table = table.to(dev)
    start = [torch.randn(n_pages, H, page, D, generator=gen).to(BF).to(dev) for _ in range(2)]
    kc0 = exact_rows(gen, n_pages, H, 1, D).to(dev)
    new = [torch.randn(B, h, n, D, generator=gen).to(BF).to(dev) for h in (H, H, H * G, H)]
    rope = sp.SpardaRope(128, sp.SPARDA_ROPE_HALF, freqs(128).to(dev))
    pos = torch.arange(n, dtype=torch.int32, device=dev) + t0
    ws = [workspace(dev, shape, op, cap) for op in (sp.SPARDA_OP_PAGED_SELECT, sp.SPARDA_OP_PAGED_ATTN)]

    def state():
        s = {"k": start[0].clone(), "v": start[1].clone(), "kc": kc0.clone()}
        s["pages"] = sp.SpardaPages(page, table, s["k"], s["v"], s["kc"])
        s["in"] = [torch.full_like(x, NAN) for x in new]
        for name, like in (("q", new[2]), ("f", new[3]), ("y", new[0]), ("o", new[2][:, :, :1]), ("all", new[2][:, :, :1]), ("f1", new[3][:, :, :1]),
                           ("q1", new[2][:, :, :1])):
            s[name] = torch.zeros(like.shape, dtype=BF, device=dev)
        s["sel"], s["cnt"] = torch.zeros(B, H, 1, k, dtype=torch.int16, device=dev), torch.zeros(B, H, 1, dtype=torch.int16, device=dev)
        s["t"], s["t_new"] = torch.zeros(B, dtype=torch.int32, device=dev), torch.zeros(B, dtype=torch.int32, device=dev)
        return s

    def run(s, stream):
        with torch.cuda.stream(stream):  # the inputs arrive late
            for x, y in zip(s["in"], new):
                x.copy_(y)
            s["t"].fill_(t0)
        kn, vn, q, f = s["in"]
        sp.sparda_rotate(rope, sp.SPARDA_BF16, B, H, n, kn, pos, 0, s["y"], stream=stream)
        sp.sparda_paged_append(shape, s["pages"], rope, n, None, s["t"], kn, vn, q, s["q"], f, s["f"], s["t_new"], stream=stream)
        with torch.cuda.stream(stream):
            s["f1"].copy_(s["f"][:, :, -1:])
            s["q1"].copy_(s["q"][:, :, -1:])
        sp.sparda_paged_select(shape, s["pages"], s["f1"], s["t_new"], cap, s["sel"], s["cnt"], ws[0], stream=stream)
        sp.sparda_paged_attn(shape, s["pages"], s["q1"], s["t_new"], cap, s["sel"], s["cnt"], ref.SCALE, s["o"], ws[1], stream=stream)
        sp.sparda_paged_attn(shape, s["pages"], s["q1"], s["t_new"], cap, None, None, ref.SCALE, s["all"], ws[1], stream=stream)
        return s

    want = run(state(), torch.cuda.current_stream())
    torch.cuda.synchronize()
    fresh = state()
    got = behind(dev, lambda stream: run(fresh, stream))
    assert want["t_new"].tolist() == [t0 + n] * B and int(want["cnt"].min()) == k
    assert torch.equal(want["t_new"], got["t_new"]) and torch.equal(want["sel"], got["sel"]) and torch.equal(want["cnt"], got["cnt"])
    for name in ("k", "v", "kc", "y", "q", "f", "o", "all"):
        assert torch.equal(bits(want[name]), bits(got[name])), name
    assert torch.isfinite(got["o"]).all() and got["o"].any() and got["y"].any()


@pytest.mark.parametrize("t,listed", [(700, False), (700, True), (30, False), (20000, False)])
def test_a_score_of_minus_infinity_weighs_nothing(dev, t, listed):  # noqa: F811
    """One element of some keys is -inf against positive elements of every query: the outputs are those without these tokens."""
    gen, rng, page, G = torch.Generator().manual_seed(t), random.Random(t), 16, 3
    table, n_pages = table_of(rng, 2, t, page)
    k, v = pools(gen, table, (t, t), n_pages, 1, page)
    q = torch.randn(2, G, 1, D, generator=gen).to(BF)
    q[..., 7] = q[..., 7].abs() + 0.125
    gone = [0, 5, 6, t // 2, t - 1] + list(range(16, 29)) + (list(range(256, 384)) if t > 384 else [])
    for i in gone:
        k[int(table[0, i // page]), 0, i % page, 7] = float("-inf")
    k[table[1].long(), 0, :, 7] = float("-inf")  # nothing is left of the second sequence
    sel = cnt = None
    if listed:
        sel = torch.tensor([0, 2, 4, 5, 10], dtype=torch.int16).expand(2, 1, 1, 5).contiguous()
        cnt = torch.full((2, 1, 1), 5, dtype=torch.int16)
    shape = shape_of(2, 1, G, k=5, t_cap=t)
    got = run_attn(dev, shape, sp.SpardaPages(page, table.to(dev), k.to(dev), v.to(dev)), q, torch.tensor([t, t], dtype=torch.int32), t, sel, cnt)
    left = [i for i in range(t) if i not in set(gone) and (not listed or i // L in (0, 2, 4, 5, 10))]
    kk, vv = (torch.stack([x[int(table[0, i // page]), :, i % page] for i in left], 1)[None] for x in (k, v))
    o, w = ref.attn(q[:1, :, 0], kk, vv, torch.zeros(1, 1, dtype=torch.int32), (len(left),), len(left), None, None, ref.SCALE)
    check(got[:1], o, w)
    assert (got[1] == 0).all()
