"""The operators of speculative decoding over the attended sets, as cases to measure: a model checks
a whole tree of drafted tokens in one step instead of decoding one token.

A case is a dict of plain values.  "op" names the operator:
  select  the Forecast selection of every node of the trees (sparda_tree_select)
  attn    attention of the nodes over their blocks of the cache and their ancestors (sparda_tree_attn)
  verify  which drafted tokens the target's probabilities keep, and the token that follows (sparda_tree_verify)
  commit  the accepted path's K and V packed into the caches of all layers, with their K~ (sparda_tree_commit)
"t" is the longest context of the batch (the others are up to an eighth shorter: after a verification the
sequences of a batch differ in length), "n" the nodes of a tree (node 0 is the last sampled token), "wide"
whether the tree branches (else it is a chain), "grid" the compression window (64: one key per block; 32:
32-token windows at stride 16).

Forecast rows and K~ are rounded to multiples of 1/8 and 1/64: a score then has at most 20 significant bits,
is exact in 32 bits in any order of summation, and the sets are the same whole numbers on every side, ties
(to the lower block) included.
"""
import math

import torch

D, L = 128, 64
SCALE = 1.0 / math.sqrt(D)
own = False


def _case(name, op, **kw):
    return {"op": op, **kw} if name is None else {"name": name, "op": op, **kw}


def _select(name, t, n, batch=1, kvh=8, k=64, n_init=1, n_local=2, grid=64, wide=True):
    return _case(name, "select", t=t, n=n, batch=batch, kvh=kvh, k=k, n_init=n_init, n_local=n_local, grid=grid, wide=wide)


def _attn(name, t, n, batch=1, kvh=8, g=4, k=64, n_init=1, n_local=2, shared=False, wide=True):
    return _case(name, "attn", t=t, n=n, batch=batch, kvh=kvh, g=g, k=k, n_init=n_init, n_local=n_local, shared=shared,
                 wide=wide)


def _verify(name, vocab, n, batch=1, drafts="point", dtype="float32", wide=True):
    return _case(name, "verify", vocab=vocab, n=n, batch=batch, drafts=drafts, dtype=dtype, wide=wide)


def _commit(name, layers, n, batch=1, kvh=8, grid=64, t=960):
    return _case(name, "commit", layers=layers, n=n, batch=batch, kvh=kvh, grid=grid, t=t)


def listed():
    return [
        # one conversation of 4K tokens, a small tree: latency
        _select("select_b1_4k", 4096, 8, k=16),
        # ordinary serving with ragged lengths, the paper's key grid, an odd tree
        _select("select_b8_32k", 32717, 21, batch=8, grid=32),
        # a full batch at 128K, the repository's headline decode workload
        _select("select_b32_128k", 131000, 16, batch=32),
        # one conversation, a small tree: latency
        _attn("attn_b1_4k", 4096, 8, k=16),
        # ordinary serving: every node has its own blocks, odd lengths
        _attn("attn_b8_32k", 32717, 27, batch=8),
        # a full batch at 128K whose trees share the root's blocks
        _attn("attn_b32_128k", 131000, 16, batch=32, shared=True),
        # the paper's model layout (32 query / 2 KV heads, 96 blocks with a 32-block local window), the largest trees
        _attn("attn_paper_b8_64k", 65000, 64, batch=8, kvh=2, g=16, k=96, n_local=32),
        # a chain of drafted tokens with the draft model's probabilities, one conversation
        _verify("verify_chain_b1", 32000, 6, drafts="probs", wide=False),
        # trees with the draft model's probabilities, an odd vocabulary, bf16 probabilities
        _verify("verify_tree_b8", 50021, 27, batch=8, drafts="probs", dtype="bfloat16"),
        # a full batch of the largest trees, drafted without probabilities
        _verify("verify_tree_b32", 131072, 64, batch=32),
        # one layer, one conversation: latency
        _commit("commit_b1", 1, 8, grid=32, t=958),
        # all layers of a model, a full batch, the paper's key grid
        _commit("commit_b16_l32", 32, 16, batch=16, grid=32),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("select", "select", "attn", "attn", "attn", "verify", "verify", "commit"))
    n, kvh, grid = _logint(rng, 1, 64), rng.choice((1, 2, 4, 8)), rng.choice((64, 32))
    n_init, n_local = rng.choice((0, 1, 1, 2)), rng.choice((2, 2, 4, 16, 32))
    k, wide = n_init + n_local + _logint(rng, 8, 64), rng.random() < 0.7
    if op == "select":
        t = _logint(rng, 1000, 131000)
        batch = _logint(rng, 1, max(1, min(32, int(2.5e8 * grid / (kvh * t * n * 4)))))
        return _select(None, t, n, batch, kvh, k, n_init, n_local, grid, wide)
    if op == "attn":
        t, g = _logint(rng, 1000, 65000), rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 12, 16))
        batch = _logint(rng, 1, max(1, min(16, int(1.0e9 / (kvh * g * n * t)))))
        return _attn(None, t, n, batch, kvh, g, k, n_init, n_local, rng.random() < 0.4, wide)
    if op == "verify":
        vocab = _logint(rng, 1000, 131072)
        batch = _logint(rng, 1, max(1, min(64, int(1.3e8 / (vocab * n)))))
        return _verify(None, vocab, n, batch, rng.choice(("point", "probs")), rng.choice(("float32", "bfloat16")), wide)
    layers = _logint(rng, 1, 32)
    return _commit(None, layers, n, _logint(rng, 1, max(1, 512 // (layers * kvh))), kvh, grid, rng.randrange(100, 961))


# ---- inputs ------------------------------------------------------------------------------------

def _stride(c):
    return 16 if c["grid"] == 32 else 64


def _t_cap(c):
    return (c["t"] + c["n"] + L - 1) // L * L


def _nc_cap(c):
    return (_t_cap(c) - c["grid"]) // _stride(c) + 2


def _trees(c, gen):
    """int32 [B][n] parents: a chain, or trees that branch (each node hangs on one of the 8 before it)."""
    B, n = c["batch"], c["n"]
    i = torch.arange(n, device="cuda")
    if not c.get("wide", True):
        return (i - 1).to(torch.int32).expand(B, n).contiguous()
    back = (torch.rand(B, n, generator=gen, device="cuda") * 8).long() + 1
    return torch.where(i > 0, (i - back).clamp_min(0), -1).to(torch.int32).contiguous()


def _lengths(c, gen):
    """int32 [B] contexts: the first is the longest."""
    short = (torch.rand(c["batch"], generator=gen, device="cuda") * (c["t"] / 8)).long()
    short[0] = 0
    return (c["t"] - short).to(torch.int32)


def _coherent(gen, a, *size):
    """Unit normals [.., n, x]; the nodes of a tree share `a` of their variance."""
    base = torch.randn(*size[:-2], 1, size[-1], generator=gen, device="cuda")
    return base * math.sqrt(a) + torch.randn(*size, generator=gen, device="cuda") * math.sqrt(1 - a)


def _sets(c, gen, t_ctx, nodes):
    """Attended sets as a selection gives them, ascending and -1 padded: the forced blocks and the best of coherent
    random scores."""
    B, H, K = c["batch"], c["kvh"], c["k"]
    nb = (c["t"] + c["n"] - 1) // L + 1
    j = torch.arange(nb, device="cuda")
    blk = (t_ctx.long() // L).view(B, 1, 1, 1)
    sc = _coherent(gen, 0.8, B, H, nodes, nb)
    sc = torch.where((j < c["n_init"]) | (j > blk - c["n_local"]), math.inf, sc).masked_fill(j > blk, -math.inf)
    top = sc.topk(min(K, nb), dim=3)
    idx = torch.where(top.values > -math.inf, top.indices, nb).sort(3).values
    sel = torch.full((B, H, nodes, K), -1, device="cuda", dtype=torch.int16)
    sel[..., :idx.shape[3]] = torch.where(idx < nb, idx, -1).to(torch.int16)
    return sel, (sel >= 0).sum(3).to(torch.int16)


def _drafted(c, gen, probs, parent):
    """Tokens int32 [B][n]: independent draws from the parent's row of `probs`."""
    B, n, V = probs.shape
    row = parent.long().clamp_min(0)
    if n == 1:
        return torch.zeros(B, 1, device="cuda", dtype=torch.int32)
    cdf = probs.float().cumsum(2)
    u = torch.rand(B, n, generator=gen, device="cuda") * 0.999
    tok = torch.empty(B, n, device="cuda", dtype=torch.int64)
    for b in range(B):
        tok[b] = torch.searchsorted(cdf[b][row[b]], u[b, :, None] * cdf[b][row[b], -1:]).squeeze(1)
    return tok.clamp_max(V - 1).to(torch.int32)


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    B, n = c["batch"], c["n"]
    s = {"case": c}

    def normal(*size):
        return torch.randn(*size, generator=gen, device=dev, dtype=torch.bfloat16)

    if c["op"] == "verify":
        V, dt = c["vocab"], getattr(torch, c["dtype"])
        s["parent"] = _trees(c, gen)
        logits = torch.randn(B, n, V, generator=gen, device=dev) * 8  # peaked, as a language model's are
        s["p"] = torch.softmax(logits, 2).to(dt)
        logits += torch.randn(B, n, V, generator=gen, device=dev)  # the draft model is near the target
        q = torch.softmax(logits, 2).to(dt)
        s["tokens"] = _drafted(c, gen, q, s["parent"])
        s["q"] = q if c["drafts"] == "probs" else None
        s["u"] = torch.rand(B, n, generator=gen, device=dev)
        s["path"] = torch.empty(B, n, dtype=torch.int32, device=dev)
        s["n_path"], s["next"] = (torch.empty(B, dtype=torch.int32, device=dev) for _ in range(2))
        s["ws"] = torch.empty(64 * B + 16 * B * (V // 1024 + 128), dtype=torch.uint8, device=dev)
        return s
    H = c["kvh"]
    s["t_ctx"] = _lengths(c, gen)
    if c["op"] == "commit":
        rows = (c["layers"], B, H)
        for x in ("k", "v"):
            s[x] = normal(*rows, _t_cap(c), D)
            s[x + "_tree"] = normal(*rows, n, D)
        s["kc"] = torch.zeros(*rows, _nc_cap(c), D, dtype=torch.bfloat16, device=dev)
        # an accepted path: ascending nodes from the root on, one to n of them, -1 padded
        keep = torch.rand(B, n, generator=gen, device=dev) < torch.rand(B, 1, generator=gen, device=dev)
        keep[:, 0] = True
        i = torch.arange(n, device=dev)
        path = torch.where(keep, i, n).sort(1).values
        s["path"] = torch.where(path < n, path, -1).to(torch.int32)
        s["n_path"] = keep.sum(1).to(torch.int32)
        s["t_new"] = torch.empty(B, dtype=torch.int32, device=dev)
        s["layers"] = {x: list(s[x].unbind(0)) for x in ("k", "v", "k_tree", "v_tree", "kc")}
        return s
    s["parent"] = _trees(c, gen)
    if c["op"] == "select":
        nc = _nc_cap(c)
        f = _coherent(gen, 0.8, B, H, n, D)
        kc = torch.randn(B, H, nc, D, generator=gen, device=dev) / math.sqrt(c["grid"])
        # 5 % of the blocks lie along the nodes' common direction
        hot = torch.rand(B, H, nc * _stride(c) // L + 1, generator=gen, device=dev) < 0.05
        hot = hot.repeat_interleave(L // _stride(c), 2)[:, :, :nc]
        kc += hot[..., None] * (f.mean(2, keepdim=True) / f.mean(2, keepdim=True).norm(dim=3, keepdim=True))
        s["f"] = ((f * 8).round() / 8).clamp(-4, 4).to(torch.bfloat16)
        s["kc"] = ((kc * 64).round() / 64).clamp(-2, 2).to(torch.bfloat16)
        s["sel"] = torch.empty(B, H, n, c["k"], dtype=torch.int16, device=dev)
        s["cnt"] = torch.empty(B, H, n, dtype=torch.int16, device=dev)
        s["ws"] = torch.empty(B * H * n * (c["t"] // L + 8) * 4 + 1024, dtype=torch.uint8, device=dev)
        return s
    G = c["g"]
    s["sel"], s["cnt"] = _sets(c, gen, s["t_ctx"], 1 if c["shared"] else n)
    s["q"] = normal(B, H * G, n, D)
    s["k"], s["v"] = normal(B, H, _t_cap(c), D), normal(B, H, _t_cap(c), D)
    s["k_tree"], s["v_tree"] = normal(B, H, n, D), normal(B, H, n, D)
    s["o"] = torch.empty_like(s["q"])
    s["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device=dev)
    return s


# ---- the framework's operators --------------------------------------------------------------------

def _shape(sp, c):
    t_cap = _t_cap(c) if "t" in c else L
    grid, stride = c.get("grid", 64), _stride(c) if "grid" in c else 64
    return sp.SpardaShape(batch=c["batch"], n_kv_heads=c.get("kvh", 1), group_size=c.get("g", 1), k_total=c.get("k", 3),
                          t_cap=t_cap, nc_cap=_nc_cap(c) if "grid" in c else t_cap // L, n_init=c.get("n_init", 1),
                          n_local=c.get("n_local", 2), cmp_kernel=grid, cmp_stride=stride)


def _run_own(s):
    from paper_2606_04511_amd import sparda as sp
    c = s["case"]
    if "shape" not in s:
        s["shape"] = _shape(sp, c)
    shape, n = s["shape"], c["n"]
    if c["op"] == "select":
        sp.sparda_tree_select(shape, s["f"], n, s["t_ctx"], c["t"], s["parent"], s["kc"], s["sel"], s["cnt"], s["ws"])
        return {"sel": s["sel"], "cnt": s["cnt"]}
    if c["op"] == "attn":
        sp.sparda_tree_attn(shape, s["q"], n, s["t_ctx"], c["t"], s["parent"], s["k"], s["v"], s["k_tree"], s["v_tree"],
                            s["sel"].shape[2], s["sel"], s["cnt"], SCALE, s["o"], s["ws"])
        return {"o": s["o"]}
    if c["op"] == "verify":
        kind = sp.SPARDA_PROB_F32 if c["dtype"] == "float32" else sp.SPARDA_PROB_BF16
        sp.sparda_tree_verify(shape, n, c["vocab"], c["vocab"], kind, s["p"], s["q"], s["tokens"], s["parent"], s["u"],
                              s["path"], s["n_path"], s["next"], s["ws"])
        return {"path": s["path"], "n_path": s["n_path"], "next": s["next"]}
    if "tables" not in s:  # the layers' addresses, which stay the same from step to step
        s["tables"] = {x: sp.layer_pointers(y) for x, y in s["layers"].items()}
    tab = s["tables"]
    sp.sparda_tree_commit(shape, n, s["t_ctx"], s["path"], s["n_path"], c["layers"], tab["k_tree"], tab["v_tree"],
                          tab["k"], tab["v"], tab["kc"], s["t_new"])
    return {"k": s["k"], "v": s["v"], "kc": s["kc"], "t": s["t_new"]}


# ---- the same in plain torch ------------------------------------------------------------------------

def _ancestors(parent):
    """float [B][n][n]: 1 where the column's node is the row's or one of its ancestors."""
    B, n = parent.shape
    i = torch.arange(n, device=parent.device)
    a = ((i == i[:, None]) | (i == parent[:, :, None])).float()
    for _ in range(6):  # paths of up to 64 steps
        a = ((a @ a) > 0).float()
    return a


def _plain_select(s):
    c, f, kc, t = s["case"], s["f"], s["kc"], s["t_ctx"].long()
    B, H, n, K, w, st = c["batch"], c["kvh"], c["n"], c["k"], c["grid"], _stride(c)
    nb, nc, dev = (c["t"] + n - 1) // L + 1, kc.shape[2], f.device
    j = torch.arange(nb, device=dev)
    blk = ((t[:, None] + _ancestors(s["parent"]).sum(2).long() - 1) // L)[:, None, :, None]
    ws = f.float() @ kc.float().transpose(2, 3)
    done = torch.arange(nc, device=dev) * st + w <= t.view(B, 1, 1, 1)
    ws = torch.where(done, ws, -math.inf)
    pad = torch.full((B, H, n, 4 * nb + 1), -math.inf, device=dev)
    if w == 64:
        sc = pad[..., :nb].clone()
        sc[..., :min(nc, nb)] = ws[..., :nb]
    else:  # block j: windows 4 j - 1 .. 4 j + 3
        pad[..., 1:1 + min(nc, 4 * nb)] = ws[..., :4 * nb]
        sc = torch.maximum(pad[..., 1:].reshape(B, H, n, nb, 4).amax(4), pad[..., 0:4 * nb:4])
    sc = torch.where((j < c["n_init"]) | (j > blk - c["n_local"]), math.inf, sc)
    sc = torch.where(j > blk, -math.inf, sc)
    top, idx = sc.sort(dim=3, descending=True, stable=True)
    m = min(K, nb)
    idx = torch.where(top[..., :m] > -math.inf, idx[..., :m], nb).sort(3).values
    sel = torch.full((B, H, n, K), -1, device=dev, dtype=torch.int16)
    sel[..., :m] = torch.where(idx < nb, idx, -1).to(torch.int16)
    return {"sel": sel, "cnt": (sel >= 0).sum(3).to(torch.int16)}


def _plain_attn(s):
    c, t = s["case"], s["t_ctx"].long().view(-1, 1, 1, 1)
    B, H, G, n, dev = c["batch"], c["kvh"], c["g"], c["n"], s["q"].device
    nb = (c["t"] - 1) // L + 1
    sel = s["sel"].long()
    if c["shared"]:  # the blocks of one list for all nodes
        bh = torch.arange(B * H, device=dev)[:, None]
        at = sel.view(B * H, -1).clamp_min(0)
        k, v = (s[x].view(B * H, -1, L, D)[bh, at].view(B, H, -1, D) for x in ("k", "v"))
        tok = (sel[..., None] * L + torch.arange(L, device=dev)).view(B, H, 1, -1)
        seen = ((tok >= 0) & (tok < t)).expand(B, H, n, -1)
    else:  # all tokens, masked
        on = torch.zeros(B, H, n, nb + 1, device=dev, dtype=torch.bool)
        on.scatter_(3, torch.where((sel >= 0) & (sel < nb), sel, nb), True)
        k, v = (s[x][:, :, :nb * L] for x in ("k", "v"))
        tok = torch.arange(k.shape[2], device=dev)
        seen = on[..., :nb].repeat_interleave(L, 3)[..., :k.shape[2]] & (tok < t)
    seen = torch.cat((seen, (_ancestors(s["parent"]) > 0)[:, None].expand(B, H, n, n)), 3)
    k, v = torch.cat((k, s["k_tree"]), 2).float(), torch.cat((v, s["v_tree"]), 2).float()
    z = (s["q"].float() * SCALE).view(B, H, G * n, D) @ k.transpose(2, 3)
    z = z.view(B, H, G, n, -1).masked_fill_(~seen[:, :, None], -math.inf)
    z = z.sub_(z.amax(4, keepdim=True)).exp_()
    z = z.div_(z.sum(4, keepdim=True)).view(B, H, G * n, -1)
    return {"o": (z @ v).view(B, H * G, n, D).to(torch.bfloat16)}


def _plain_verify(s):
    c, parent = s["case"], s["parent"].long()
    B, n, V, dev = c["batch"], c["n"], c["vocab"], s["p"].device
    b, q = torch.arange(B, device=dev), s["q"]
    cur = torch.zeros(B, device=dev, dtype=torch.int64)
    kept = torch.zeros(B, n, device=dev, dtype=torch.bool)
    kept[:, 0] = True
    m, mass = s["p"][:, 0].double(), torch.ones(B, device=dev, dtype=torch.float64)
    for i in range(1, n):  # siblings in the order of their nodes
        child, x = parent[:, i] == cur, s["tokens"][:, i].long()
        mx = m[b, x]
        qx = q[b, cur, x].double() if q is not None else 1.0
        yes = child & (s["u"][:, i].double() * mass * qx < mx)
        no = child & ~yes
        if q is not None:
            left = (m - mass[:, None] * q[b, cur].double()).clamp_min(0)
            now = left.sum(1)
        else:
            left, now = m.clone(), (mass - mx).clamp_min(0)
            left[b, x] = 0
        m = torch.where(yes[:, None], s["p"][:, i].double(), torch.where(no[:, None], left, m))
        mass = torch.where(yes, 1.0, torch.where(no, now, mass))
        cur = torch.where(yes, i, cur)
        kept[:, i] = yes
    run = m.cumsum(1)
    nxt = (run <= s["u"][:, 0].double()[:, None] * run[:, -1:]).sum(1)
    path = torch.where(kept, torch.arange(n, device=dev), n).sort(1).values
    return {"path": torch.where(path < n, path, -1).to(torch.int32), "n_path": kept.sum(1).to(torch.int32),
            "next": nxt.clamp_max(V - 1).to(torch.int32)}


def _plain_commit(s):
    c, t, cnt = s["case"], s["t_ctx"].long(), s["n_path"].long()
    n, w, st, dev = c["n"], c["grid"], _stride(c), s["k"].device
    b, i = torch.arange(c["batch"], device=dev)[:, None], torch.arange(n, device=dev)
    at, new = t[:, None] + i, i < cnt[:, None]
    for x in ("k", "v"):  # the rows come to the front: [B][n][layers][Hkv][D]
        cache, tree = s[x].permute(1, 3, 0, 2, 4), s[x + "_tree"].permute(1, 3, 0, 2, 4)
        cache[b, at] = torch.where(new[:, :, None, None, None], tree[b, s["path"].long().clamp_min(0)], cache[b, at])
    first = ((t - w) // st + 1).clamp_min(0)[:, None] + torch.arange(n // st + 1, device=dev)
    full = first * st + w <= (t + cnt)[:, None]
    rows = (first[:, :, None] * st + torch.arange(w, device=dev)).clamp_max(s["k"].shape[3] - 1)
    kc, keys = s["kc"].permute(1, 3, 0, 2, 4), s["k"].permute(1, 3, 0, 2, 4)
    mean = keys[b[:, :, None], rows].double().sum(2) / w
    kc[b, first] = torch.where(full[:, :, None, None, None], mean.to(torch.bfloat16), kc[b, first])
    return {"k": s["k"], "v": s["v"], "kc": s["kc"], "t": (t + cnt).to(torch.int32)}


def run(state):
    if own:
        return _run_own(state)
    return {"select": _plain_select, "attn": _plain_attn, "verify": _plain_verify,
            "commit": _plain_commit}[state["case"]["op"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    c = case
    B, n = c["batch"], c["n"]
    if c["op"] == "verify":
        size = 4 if c["dtype"] == "float32" else 2
        rows = 2 if c["drafts"] == "probs" else 1
        return {"bytes": B * (rows * size * (c["vocab"] + n) + 20 * n), "flops": 4 * B * c["vocab"]}
    rows = B * c["kvh"]
    if c["op"] == "commit":
        mean = 0.5 * n + 0.5
        moved = c["layers"] * rows * D * 2
        return {"bytes": moved * mean * (4 + c["grid"] / _stride(c)), "flops": moved * mean * c["grid"] / _stride(c) / 2}
    t = c["t"] * (15 / 16 if B > 1 else 1)
    if c["op"] == "select":
        nw = t / _stride(c)
        return {"bytes": rows * (2 * D * (nw + n) + 2 * n * (c["k"] + 1)), "flops": 2 * D * rows * n * nw}
    attended = min(c["k"] * L, t)
    # blocks that some node lists, about: the nodes' sets share most of their blocks (0.8 of the scores' variance)
    chosen = max(0, c["k"] - c["n_init"] - c["n_local"])
    blocks = min(t / L, c["k"] + (0 if c["shared"] else chosen * min(n - 1, 0.45 * math.log2(n + 1))))
    return {"bytes": rows * 2 * D * (2 * blocks * L + 2 * n + 2 * n * c["g"]),
            "flops": 4 * D * rows * c["g"] * n * (attended + min(n, 8))}


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _paths(parent):
    """For every sequence and node, the nodes from it up to the root."""
    out = []
    for row in parent.tolist():
        up = []
        for i, p in enumerate(row):
            up.append([i] + (up[p] if i else []))
        out.append(up)
    return out


def _exact_select(c, s):
    w, st, K = c["grid"], _stride(c), c["k"]
    sel = torch.full((c["batch"], c["kvh"], c["n"], K), -1, dtype=torch.int64)
    cnt = torch.zeros(c["batch"], c["kvh"], c["n"], dtype=torch.int64)
    paths = _paths(s["parent"])
    for b, t in enumerate(s["t_ctx"].tolist()):
        n_win = (t - w) // st + 1 if t >= w else 0
        for h in range(c["kvh"]):
            z = (s["f"][b, h].double() @ s["kc"][b, h, :n_win].double().t().contiguous()).cpu()
            for i in range(c["n"]):
                blk = (t + len(paths[b][i]) - 1) // L
                forced = sorted({x for x in range(min(c["n_init"], blk + 1))} |
                                set(range(max(0, blk - c["n_local"] + 1), blk + 1)))
                cand = range(c["n_init"], blk - c["n_local"] + 1)
                if len(cand) and len(forced) + len(cand) > K:
                    if w == 64:
                        sc = z[i, cand.start:cand.stop]
                    else:
                        lo = torch.arange(4 * cand.start - 1, 4 * cand.stop - 1, 4)[:, None] + torch.arange(5)
                        sc = torch.where((lo >= 0) & (lo < n_win), z[i][lo.clamp(0, n_win - 1)], -math.inf).amax(1)
                    order = torch.argsort(-sc, stable=True)[:K - len(forced)] + cand.start
                    got = sorted(forced + order.tolist())
                else:
                    got = sorted(forced + list(cand))
                sel[b, h, i, :len(got)] = torch.tensor(got)
                cnt[b, h, i] = len(got)
    return {"sel": sel, "cnt": cnt}


def _exact_attn(c, s):
    G, n = c["g"], c["n"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    paths = _paths(s["parent"])
    within = torch.arange(L, device="cuda")
    for b, t in enumerate(s["t_ctx"].tolist()):
        for h in range(c["kvh"]):
            k, v = s["k"][b, h], s["v"][b, h]
            for i in range(n):
                up = torch.tensor(paths[b][i], device="cuda")
                r = 0 if c["shared"] else i
                if i == 0 or not c["shared"]:
                    blocks = s["sel"][b, h, r, :int(s["cnt"][b, h, r])].long()
                    tok = (blocks[:, None] * L + within).reshape(-1)
                    tok = tok[tok < t]
                    kc, vc = k[tok].double(), v[tok].double()
                kk = torch.cat((kc, s["k_tree"][b, h, up].double()))
                vv = torch.cat((vc, s["v_tree"][b, h, up].double()))
                z = kk @ s["q"][b, h * G:(h + 1) * G, i].double().t().contiguous() * SCALE
                o[b, h * G:(h + 1) * G, i] = torch.softmax(z, 0).t().contiguous() @ vv
    return {"o": o}


def _exact_verify(c, s):
    out = {"path": [], "n_path": [], "next": []}
    parents, tokens, us = s["parent"].tolist(), s["tokens"].tolist(), s["u"].double().tolist()
    for b in range(c["batch"]):
        at, path, p, mass = 0, [0], s["p"][b, 0].double(), 1.0
        for i in range(1, c["n"]):
            if parents[b][i] != at:
                continue
            x = tokens[b][i]
            if s["q"] is None:
                if us[b][i] * mass < float(p[x]):
                    at, p, mass = i, s["p"][b, i].double(), 1.0
                    path.append(i)
                else:
                    mass = max(mass - float(p[x]), 0.0)
                    p = p.clone()
                    p[x] = 0
            else:
                d = s["q"][b, at].double()
                if us[b][i] * mass * float(d[x]) < float(p[x]):
                    at, p, mass = i, s["p"][b, i].double(), 1.0
                    path.append(i)
                else:
                    p = torch.relu(p - mass * d)
                    mass = float(p.sum())
        edges = p.cumsum(0)
        nxt = int(torch.searchsorted(edges, edges[-1:] * us[b][0], right=True))
        out["path"].append(path + [-1] * (c["n"] - len(path)))
        out["n_path"].append(len(path))
        out["next"].append(min(nxt, c["vocab"] - 1))
    return {x: torch.tensor(y) for x, y in out.items()}


def _exact_commit(c, s):
    w, st = c["grid"], _stride(c)
    k, v, kc = s["k"].double(), s["v"].double(), s["kc"].double()
    t_new = []
    for b, t in enumerate(s["t_ctx"].tolist()):
        nodes = s["path"][b, :int(s["n_path"][b])].long()
        k[:, b, :, t:t + len(nodes)] = s["k_tree"][:, b][:, :, nodes].double()
        v[:, b, :, t:t + len(nodes)] = s["v_tree"][:, b][:, :, nodes].double()
        t_new.append(t + len(nodes))
        for i in range(kc.shape[3]):
            if t < i * st + w <= t_new[-1]:
                kc[:, b, :, i] = k[:, b, :, i * st:i * st + w].mean(2)
    return {"k": k, "v": v, "kc": kc, "t": torch.tensor(t_new)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"select": _exact_select, "attn": _exact_attn, "verify": _exact_verify, "commit": _exact_commit}[case["op"]](case, s)
