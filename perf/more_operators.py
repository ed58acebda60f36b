"""The operators of a paged key-value cache, as cases to measure: rotary positions, the append of new tokens, the
Forecast selection and the attention of one new token, for sequences of different lengths whose tokens lie in pages.

A case is a dict of plain values.  "op" names the operator:
  rotate  rotary positions of rows (sparda_rotate), or the gradient through them
  append  new tokens' K, rotated on the way, and V into the pages, with the compressed keys of the windows they
          complete and the tokens' rotated queries and Forecast rows (sparda_paged_append)
  select  the Forecast selection of each sequence's newest token over paged compressed keys (sparda_paged_select)
  attn    attention of each sequence's newest token over its listed blocks, or over its whole context
          (sparda_paged_attn)
"t" is the longest context of the batch (the others are up to a half shorter where "ragged", else an eighth), "page"
the tokens of a page, "grid" the compression window (64: one key per block; 32: 32-token windows at stride 16), "rot"
the rotated part of the head, "pairs" whether a pair is two neighbours (else it lies half the rotated part apart), "far"
the factor by which positions are scaled beyond the trained context.

Forecast rows and K~ of the selections are rounded to multiples of 1/8 and 1/64: a score then has at most 20
significant bits, is exact in 32 bits in any order of summation, and the sets are the same whole numbers on every
side, ties (to the lower block) included.
"""
import math

import torch

D, L = 128, 64
SCALE = 1.0 / math.sqrt(D)
TRAINED = 8192  # positions of the trained context, which the scaled frequencies stretch
own = False


def _case(name, op, **kw):
    return {"op": op, **kw} if name is None else {"name": name, "op": op, **kw}


def _rotate(name, n, heads, batch=1, rot=128, pairs=False, far=1.0, dtype="bfloat16", back=False, tokens_first=False):
    return _case(name, "rotate", n=n, heads=heads, batch=batch, rot=rot, pairs=pairs, far=far, dtype=dtype, back=back,
                 tokens_first=tokens_first)


def _append(name, t, n, batch=1, kvh=8, g=4, page=64, grid=64, rot=128, pairs=False, far=1.0):
    return _case(name, "append", t=t, n=n, batch=batch, kvh=kvh, g=g, page=page, grid=grid, rot=rot, pairs=pairs, far=far)


def _select(name, t, batch=1, kvh=8, k=64, n_init=1, n_local=2, page=64, grid=64, ragged=False):
    return _case(name, "select", t=t, batch=batch, kvh=kvh, k=k, n_init=n_init, n_local=n_local, page=page, grid=grid,
                 ragged=ragged)


def _attn(name, t, batch=1, kvh=8, g=4, k=0, n_init=1, n_local=2, page=64, ragged=False):
    return _case(name, "attn", t=t, batch=batch, kvh=kvh, g=g, k=k, n_init=n_init, n_local=n_local, page=page, ragged=ragged)


def listed():
    return [
        # the gradient of a training chunk's Forecast rows (256 rows of 8 groups): latency
        _rotate("rotate_grad_256", 256, 8, dtype="float32", back=True),
        # a long prompt's queries as a projection lays them out (token first), positions scaled beyond the trained context
        _rotate("rotate_32k", 32717, 32, far=4.0, tokens_first=True),
        # one conversation, one token: latency
        _append("append_b1", 959, 1, grid=32),
        # a decode step of a full batch
        _append("append_b32", 959, 1, batch=32),
        # a chunk of several prompts of different lengths, small pages, the paper's key grid, half of the head rotated
        _append("append_chunk", 1003, 4001, batch=4, page=16, grid=32, rot=64, pairs=True),
        # one conversation of 4K tokens: latency
        _select("select_b1_4k", 4096, k=16),
        # ordinary serving: very different lengths, small pages, the paper's key grid
        _select("select_b8_32k", 32717, batch=8, page=16, grid=32, ragged=True),
        # a full batch at 128K, the repository's headline decode workload
        _select("select_b32_128k", 131000, batch=32),
        # one conversation of 4K tokens, whole context: latency
        _attn("attn_b1_4k", 4096),
        # ordinary serving without sparsity: very different lengths, whole contexts
        _attn("attn_b8_32k", 32717, batch=8, ragged=True),
        # a full batch at 128K over 64 blocks a row, the repository's headline decode workload
        _attn("attn_b32_128k", 131000, batch=32, k=64),
        # the paper's model layout (32 query / 2 KV heads, 96 blocks with a 32-block local window), small pages
        _attn("attn_paper_b16_64k", 65000, batch=16, kvh=2, g=16, k=96, n_local=32, page=16),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotate", "append", "append", "select", "select", "attn", "attn", "attn"))
    kvh, grid, batch = rng.choice((1, 2, 4, 8)), rng.choice((64, 32)), _logint(rng, 1, 64)
    page = rng.choice((16, 32, 64, 64, 128, 256))
    rot, pairs, far = rng.choice((128, 128, 96, 64, 32)), rng.random() < 0.4, rng.choice((1.0, 1.0, 4.0))
    n_init, n_local = rng.choice((0, 1, 1, 2)), rng.choice((1, 2, 2, 4, 16, 32))
    k, ragged = n_init + n_local + _logint(rng, 4, 64), rng.random() < 0.5
    if op == "rotate":
        heads, batch = _logint(rng, 1, 40), _logint(rng, 1, 8)
        n = _logint(rng, 1, max(1, 1000000 // (heads * batch)))
        return _rotate(None, n, heads, batch, rot, pairs, far, rng.choice(("bfloat16", "bfloat16", "float32")),
                       rng.random() < 0.4, rng.random() < 0.5)
    if op == "append":
        page = max(page, 64) if grid == 64 else page
        g = rng.choice((1, 2, 4, 4, 5, 8, 16))
        n = 1 if rng.random() < 0.5 else _logint(rng, 1, 4096)
        batch = max(1, min(batch, int(600000 // (n * kvh * (g + 3)))))
        return _append(None, rng.randrange(1, 1000), n, batch, kvh, g, page, grid, rot, pairs, far)
    if op == "select":
        page = max(page, 64) if grid == 64 else page
        t = _logint(rng, 1, 131000)
        batch = max(1, min(batch, int(5.0e5 * grid / (kvh * t))))
        return _select(None, t, batch, kvh, k, n_init, n_local, page, grid, ragged)
    t, g = _logint(rng, 1, 100000), rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 12, 16))
    batch = max(1, min(batch, int(2.0e6 // (kvh * t))))
    return _attn(None, t, batch, kvh, g, k if rng.random() < 0.5 else 0, n_init, n_local, page, ragged)


# ---- inputs ------------------------------------------------------------------------------------

def _stride(c):
    return 16 if c["grid"] == 32 else 64


def _t_cap(c):
    """Tokens that a sequence's row of the page table covers: the context, the new tokens, room for a window."""
    return (c["t"] + c.get("n", 0) + 2 * L + L - 1) // L * L


def _lengths(c, gen):
    """int32 [B] contexts: the first is the longest."""
    short = torch.rand(c["batch"], generator=gen, device="cuda") * (c["t"] / (2 if c.get("ragged") else 8))
    short[0] = 0
    return (c["t"] - short.long()).to(torch.int32)


def _table(c, gen):
    """int32 [B][pages of a sequence]: the pool's pages in no order."""
    per = (_t_cap(c) + c["page"] - 1) // c["page"]
    return torch.randperm(c["batch"] * per + 3, generator=gen, device="cuda")[:c["batch"] * per].view(-1, per).to(torch.int32)


def _frequencies(c):
    """Radians per position, float64, and the factor on the rotated part.  Scaled contexts divide the slow
    frequencies, keep the fast ones and blend in between."""
    f = 10000.0 ** (-2.0 * torch.arange(c["rot"] // 2, dtype=torch.float64) / c["rot"])
    turns = TRAINED * f / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    return (f * (keep + (1 - keep) / c["far"])).to("cuda"), 1.0 + 0.1 * math.log(c["far"])


def _sets(c, gen, t_ctx):
    """Attended sets as a selection gives them, ascending and -1 padded: the forced blocks and the best of random
    scores."""
    B, H, K = c["batch"], c["kvh"], c["k"]
    nb = (c["t"] - 1) // L + 1
    j = torch.arange(nb, device="cuda")
    blk = ((t_ctx.long() - 1) // L).view(B, 1, 1)
    sc = torch.randn(B, H, nb, generator=gen, device="cuda")
    sc = torch.where((j < c["n_init"]) | (j > blk - c["n_local"]), math.inf, sc).masked_fill(j > blk, -math.inf)
    top = sc.topk(min(K, nb), dim=2)
    idx = torch.where(top.values > -math.inf, top.indices, nb).sort(2).values
    sel = torch.full((B, H, 1, K), -1, device="cuda", dtype=torch.int16)
    sel[:, :, 0, :idx.shape[2]] = torch.where(idx < nb, idx, -1).to(torch.int16)
    return sel, (sel >= 0).sum(3).to(torch.int16)


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    s = {"case": c}

    def normal(*size, dtype=torch.bfloat16):
        return torch.randn(*size, generator=gen, device=dev, dtype=dtype)

    B = c["batch"]
    if c["op"] == "rotate":
        s["freq"], s["scale"] = _frequencies(c)
        n, h, dt = c["n"], c["heads"], getattr(torch, c["dtype"])
        # rows are seen as [B][heads][n][D]; a projection's output has a token's heads side by side
        s["x"] = normal(B, n, h, D, dtype=dt).transpose(1, 2) if c["tokens_first"] else normal(B, h, n, D, dtype=dt)
        s["y"] = torch.empty(B, h, n, D, dtype=dt, device=dev)
        first = torch.randint(0, int(TRAINED * c["far"]), (B, 1), generator=gen, device=dev)
        s["pos"] = (first + torch.arange(n, device=dev)).to(torch.int32)
        return s
    H = c["kvh"]
    s["t_ctx"], s["table"] = _lengths(c, gen), _table(c, gen)
    pages = s["table"].numel() + 3
    if c["op"] == "append":
        s["freq"], s["scale"] = _frequencies(c)
        n, G = c["n"], c["g"]
        s["k"], s["v"] = normal(pages, H, c["page"], D), normal(pages, H, c["page"], D)
        s["kc"] = torch.zeros(pages, H, c["page"] // _stride(c), D, dtype=torch.bfloat16, device=dev)
        # one projection's output: a token's query, key, value and Forecast heads side by side
        new = normal(B, n, H * (G + 3), D).transpose(1, 2)
        s["q_new"], s["k_new"], s["v_new"], s["f_new"] = new.split((H * G, H, H, H), 1)
        s["q"], s["f"] = torch.zeros(B, H * G, n, D, dtype=torch.bfloat16, device=dev), torch.zeros(
            B, H, n, D, dtype=torch.bfloat16, device=dev)
        less = (torch.rand(B, generator=gen, device=dev) * (n / 2)).long()
        less[0] = 0
        s["n_new"] = (n - less).to(torch.int32)
        s["t_new"] = torch.empty(B, dtype=torch.int32, device=dev)
        return s
    s["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
    if c["op"] == "select":
        f = torch.randn(B, H, 1, D, generator=gen, device=dev)
        kc = torch.randn(pages, H, c["page"] // _stride(c), D, generator=gen, device=dev) / math.sqrt(c["grid"])
        s["f"] = ((f * 8).round() / 8).clamp(-4, 4).to(torch.bfloat16)
        s["kc"] = ((kc * 64).round() / 64).clamp(-2, 2).to(torch.bfloat16)
        s["sel"] = torch.empty(B, H, 1, c["k"], dtype=torch.int16, device=dev)
        s["cnt"] = torch.empty(B, H, 1, dtype=torch.int16, device=dev)
        return s
    s["sel"], s["cnt"] = _sets(c, gen, s["t_ctx"]) if c["k"] else (None, None)
    s["q"] = normal(B, H * c["g"], 1, D)
    s["k"], s["v"] = normal(pages, H, c["page"], D), normal(pages, H, c["page"], D)
    s["o"] = torch.empty_like(s["q"])
    return s


# ---- the framework's operators --------------------------------------------------------------------

def _run_own(s):
    from paper_2606_04511_amd import sparda as sp
    c = s["case"]
    if "shape" not in s:  # what a program keeps from call to call: the shape, the rotation, the layer's pages
        if c["op"] != "rotate":
            cap, grid = _t_cap(c), c.get("grid", 64)
            n_init, n_local = c.get("n_init", 1), c.get("n_local", 2)
            s["shape"] = sp.SpardaShape(batch=c["batch"], n_kv_heads=c["kvh"], group_size=c.get("g", 1),
                                        k_total=c.get("k") or n_init + n_local, t_cap=cap, nc_cap=0, n_init=n_init,
                                        n_local=n_local, cmp_kernel=grid, cmp_stride=16 if grid == 32 else 64)
            s["pages"] = sp.SpardaPages(c["page"], s["table"], s.get("k"), s.get("v"), s.get("kc"))
        else:
            s["shape"] = None
        if "freq" in s:
            s["rope"] = sp.SpardaRope(c["rot"], sp.SPARDA_ROPE_PAIRS if c["pairs"] else sp.SPARDA_ROPE_HALF, s["freq"],
                                      s["scale"])
    if c["op"] == "rotate":
        kind = sp.SPARDA_F32 if c["dtype"] == "float32" else sp.SPARDA_BF16
        sp.sparda_rotate(s["rope"], kind, c["batch"], c["heads"], c["n"], s["x"], s["pos"], c["n"], s["y"], c["back"])
        return {"y": s["y"]}
    shape, pages = s["shape"], s["pages"]
    if c["op"] == "append":
        sp.sparda_paged_append(shape, pages, s["rope"], c["n"], s["n_new"], s["t_ctx"], s["k_new"], s["v_new"], s["q_new"],
                               s["q"], s["f_new"], s["f"], s["t_new"])
        return {x: s[x] for x in ("k", "v", "kc", "q", "f", "t_new")}
    if c["op"] == "select":
        sp.sparda_paged_select(shape, pages, s["f"], s["t_ctx"], c["t"], s["sel"], s["cnt"], s["ws"])
        return {"sel": s["sel"], "cnt": s["cnt"]}
    sp.sparda_paged_attn(shape, pages, s["q"], s["t_ctx"], c["t"], s["sel"], s["cnt"], SCALE, s["o"], s["ws"])
    return {"o": s["o"]}


# ---- the same in plain torch ------------------------------------------------------------------------

def _turned(c, s, x, pos, back=False):
    """float32 [B][heads][n][D]: the rows x turned to the positions pos [B][n]."""
    ang = pos.double()[:, None, :, None] * s["freq"]
    cos, sin = (ang.cos() * s["scale"]).float(), (ang.sin() * (-s["scale"] if back else s["scale"])).float()
    x, m = x.float(), c["rot"] // 2
    y = x.clone()
    a, b = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if c["pairs"] else (slice(0, m), slice(m, 2 * m))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _plain_rotate(s):
    return {"y": _turned(s["case"], s, s["x"], s["pos"], s["case"]["back"]).to(s["x"].dtype)}


def _plain_append(s):
    c, t, cnt = s["case"], s["t_ctx"].long()[:, None], s["n_new"].long()[:, None]
    n, P, w, st, dev = c["n"], c["page"], c["grid"], _stride(c), s["k"].device
    table, b, i = s["table"].long(), torch.arange(c["batch"], device=dev)[:, None], torch.arange(n, device=dev)
    at, new = t + i, i < cnt
    keep = new[:, None, :, None]
    for x in ("q", "f"):
        s[x].copy_(torch.where(keep, _turned(c, s, s[x + "_new"], at).to(torch.bfloat16), s[x]))
    page, row = table[b, at // P], at % P
    for x, val in (("k", _turned(c, s, s["k_new"], at).to(torch.bfloat16)), ("v", s["v_new"])):
        pool = s[x].transpose(1, 2)  # [pages][P][Hkv][D]
        pool[page, row] = torch.where(new[:, :, None, None], val.transpose(1, 2), pool[page, row])
    first = ((t - w) // st + 1).clamp_min(0) + torch.arange(n // st + 1, device=dev)
    full = first * st + w <= t + cnt
    tok = first[:, :, None] * st + torch.arange(w, device=dev)
    mean = s["k"].transpose(1, 2)[table[b[:, :, None], tok // P], tok % P].double().sum(2) / w
    kc, page, row = s["kc"].transpose(1, 2), table[b, first * st // P], first * st % P // st
    kc[page, row] = torch.where(full[:, :, None, None], mean.to(torch.bfloat16), kc[page, row])
    return {"k": s["k"], "v": s["v"], "kc": s["kc"], "q": s["q"], "f": s["f"], "t_new": (t + cnt)[:, 0].to(torch.int32)}


def _in_order(pool, table):
    """[B][Hkv][tokens or windows][D]: the pages of each sequence one behind the other."""
    x = pool[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, D)


def _plain_select(s):
    c, f, t = s["case"], s["f"], s["t_ctx"].long().view(-1, 1, 1)
    B, H, K, w, st, dev = c["batch"], c["kvh"], c["k"], c["grid"], _stride(c), s["f"].device
    nb = (c["t"] - 1) // L + 1
    kc = _in_order(s["kc"], s["table"])
    ws = (kc.float() @ f.float().transpose(2, 3))[..., 0]
    ws = torch.where(torch.arange(kc.shape[2], device=dev) * st + w <= t, ws, -math.inf)
    if w == 64:
        sc = ws[..., :nb]
    else:  # block j: windows 4 j - 1 .. 4 j + 3
        pad = torch.cat((torch.full((B, H, 1), -math.inf, device=dev), ws[..., :4 * nb]), 2)
        sc = torch.maximum(pad[..., 1:].reshape(B, H, nb, 4).amax(3), pad[..., 0:4 * nb:4])
    j, blk = torch.arange(nb, device=dev), (t - 1) // L
    sc = torch.where((j < c["n_init"]) | (j > blk - c["n_local"]), math.inf, sc)
    sc = torch.where(j > blk, -math.inf, sc)
    top, idx = sc.sort(dim=2, descending=True, stable=True)
    m = min(K, nb)
    idx = torch.where(top[..., :m] > -math.inf, idx[..., :m], nb).sort(2).values
    sel = torch.full((B, H, 1, K), -1, device=dev, dtype=torch.int16)
    sel[:, :, 0, :m] = torch.where(idx < nb, idx, -1).to(torch.int16)
    return {"sel": sel, "cnt": (sel >= 0).sum(3).to(torch.int16)}


def _plain_attn(s):
    c, t = s["case"], s["t_ctx"].long().view(-1, 1, 1)
    B, H, G, P, dev = c["batch"], c["kvh"], c["g"], c["page"], s["q"].device
    if c["k"]:  # the tokens of the listed blocks
        tok = (s["sel"].long().view(B, H, -1, 1) * L + torch.arange(L, device=dev)).view(B, H, -1)
        seen, tok = (tok >= 0) & (tok < t), tok.clamp_min(0)
        page = s["table"].long()[torch.arange(B, device=dev).view(B, 1, 1), tok // P]
        k, v = (s[x][page, torch.arange(H, device=dev).view(H, 1), tok % P].float() for x in ("k", "v"))
    else:
        table = s["table"][:, :(c["t"] + P - 1) // P]
        k, v = (_in_order(s[x], table).float() for x in ("k", "v"))
        seen = (torch.arange(k.shape[2], device=dev) < t).expand(B, H, -1)
    z = (s["q"].float() * SCALE).view(B, H, G, D) @ k.transpose(2, 3)
    z = z.masked_fill_(~seen[:, :, None], -math.inf)
    z = z.sub_(z.amax(3, keepdim=True)).exp_()
    o = (z @ v) / z.sum(3, keepdim=True)
    return {"o": o.view(B, H * G, 1, D).to(torch.bfloat16)}


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _plain_rotate, "append": _plain_append, "select": _plain_select,
            "attn": _plain_attn}[state["case"]["op"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    c = case
    B = c["batch"]
    if c["op"] == "rotate":
        rows = B * c["heads"] * c["n"]
        return {"bytes": rows * D * 2 * (4 if c["dtype"] == "float32" else 2) + 4 * B * c["n"],
                "flops": 3 * rows * c["rot"]}
    H = c["kvh"]
    if c["op"] == "append":
        mean = (0.75 * B + 0.25) / B * c["n"] if B > 1 else c["n"]
        rows, windows = B * mean * H * (c["g"] + 3), B * H * mean / _stride(c)
        older = min(c["grid"] - mean, c["t"]) if mean < c["grid"] else 0.5 * c["grid"] * c["grid"] / mean
        return {"bytes": 2 * D * (2 * rows + windows * (older + 1)),
                "flops": 3 * B * mean * H * (c["g"] + 2) * c["rot"] + windows * c["grid"] * D}
    t = c["t"] * ((0.75 if c["ragged"] else 15 / 16) if B > 1 else 1)
    if c["op"] == "select":
        nw = t / _stride(c)
        return {"bytes": B * H * (2 * D * (nw + 1) + 2 * (c["k"] + 1)), "flops": 2 * D * B * H * nw}
    attended = min(c["k"] * L, t) if c["k"] else t
    return {"bytes": B * H * 2 * D * (2 * attended + 2 * c["g"]) + 2 * B * H * c["k"],
            "flops": 4 * D * B * H * c["g"] * attended}


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _exact_turn(c, s, x, pos, back=False):
    """float64: each pair of [.., n, D] as a complex number times a unit one at its position's angle."""
    x, m = x.double(), c["rot"] // 2
    angle = pos.double()[:, None] * s["freq"] * (-1.0 if back else 1.0)
    turn = torch.polar(torch.full_like(angle, s["scale"]), angle)
    part = x[..., :2 * m]
    pair = part.reshape(*x.shape[:-1], m, 2) if c["pairs"] else torch.stack((part[..., :m], part[..., m:]), -1)
    got = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    got = got.reshape(part.shape) if c["pairs"] else torch.cat((got[..., 0], got[..., 1]), -1)
    return torch.cat((got, x[..., 2 * m:]), -1)


def _exact_rotate(c, s):
    return {"y": torch.stack([_exact_turn(c, s, s["x"][b], s["pos"][b], c["back"]) for b in range(c["batch"])])}


def _exact_append(c, s):
    P, w, st = c["page"], c["grid"], _stride(c)
    out = {x: s[x].double() for x in ("k", "v", "kc", "q", "f")}
    t_new = []
    for b, (t, n) in enumerate(zip(s["t_ctx"].tolist(), s["n_new"].tolist())):
        pos = torch.arange(t, t + n, device="cuda")
        row = s["table"][b].long()
        for x in ("q", "f"):
            out[x][b, :, :n] = _exact_turn(c, s, s[x + "_new"][b, :, :n], pos)
        out["k"][row[pos // P], :, pos % P] = _exact_turn(c, s, s["k_new"][b, :, :n], pos).transpose(0, 1)
        out["v"][row[pos // P], :, pos % P] = s["v_new"][b, :, :n].double().transpose(0, 1)
        t_new.append(t + n)
        i = 0
        while i * st + w <= t + n:  # the means are those of the keys that the cache holds, rounded to its type
            if i * st + w > t:
                tok = torch.arange(i * st, i * st + w, device="cuda")
                keys = out["k"][row[tok // P], :, tok % P].to(torch.bfloat16).double()
                out["kc"][int(row[i * st // P]), :, i * st % P // st] = keys.mean(0)
            i += 1
    return {**out, "t_new": torch.tensor(t_new)}


def _exact_select(c, s):
    w, st, K = c["grid"], _stride(c), c["k"]
    sel = torch.full((c["batch"], c["kvh"], 1, K), -1, dtype=torch.int64)
    cnt = torch.zeros(c["batch"], c["kvh"], 1, dtype=torch.int64)
    for b, t in enumerate(s["t_ctx"].tolist()):
        n_win = (t - w) // st + 1 if t >= w else 0
        i = torch.arange(n_win, device="cuda") * st
        keys = s["kc"][s["table"][b].long()[i // c["page"]], :, i % c["page"] // st].double()  # [windows][Hkv][D]
        z = (keys * s["f"][b, :, 0].double()).sum(2).cpu()
        blk = (t - 1) // L
        forced = sorted(set(range(min(c["n_init"], blk + 1))) | set(range(max(0, blk - c["n_local"] + 1), blk + 1)))
        cand = range(c["n_init"], blk - c["n_local"] + 1)
        for h in range(c["kvh"]):
            if len(cand) and len(forced) + len(cand) > K:
                if w == 64:
                    sc = z[cand.start:cand.stop, h]
                else:
                    lo = torch.arange(4 * cand.start - 1, 4 * cand.stop - 1, 4)[:, None] + torch.arange(5)
                    sc = torch.where((lo >= 0) & (lo < n_win), z[lo.clamp(0, n_win - 1), h], -math.inf).amax(1)
                order = torch.argsort(-sc, stable=True)[:K - len(forced)] + cand.start
                got = sorted(forced + order.tolist())
            else:
                got = sorted(forced + list(cand))
            sel[b, h, 0, :len(got)] = torch.tensor(got)
            cnt[b, h, 0] = len(got)
    return {"sel": sel, "cnt": cnt}


def _exact_attn(c, s):
    G, P = c["g"], c["page"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, t in enumerate(s["t_ctx"].tolist()):
        for h in range(c["kvh"]):
            tok = torch.arange(t, device="cuda")
            if c["k"]:
                blocks = s["sel"][b, h, 0, :int(s["cnt"][b, h, 0])].long()
                tok = (blocks[:, None] * L + torch.arange(L, device="cuda")).reshape(-1)
                tok = tok[tok < t]
            page = s["table"][b].long()[tok // P]
            k, v = s["k"][page, h, tok % P].double(), s["v"][page, h, tok % P].double()
            z = k @ s["q"][b, h * G:(h + 1) * G, 0].double().t().contiguous() * SCALE
            o[b, h * G:(h + 1) * G, 0] = torch.softmax(z, 0).t().contiguous() @ v
    return {"o": o}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "select": _exact_select, "attn": _exact_attn}[case["op"]](case, s)
