"""The operators over trees of drafted tokens, written from their definitions in float64 with plain loops
(test infrastructure; shares no code with the library).  Tensors are torch tensors on the CPU; bf16 values are
taken as they are."""
import math

import torch

L = 64


def paths(parent):
    """For every node of one tree the nodes from it up to the root, [] for an absent node."""
    out = []
    for i, p in enumerate(parent):
        if i == 0:
            out.append([0] if p == -1 else [])
        elif 0 <= p < i and out[p]:
            out.append([i] + out[p])
        else:
            out.append([])
    return out


def select(f, kc, t_ctx, parent, k_total, n_init, n_local, grid):
    """sets [B][H][n][k_total] and counts [B][H][n]."""
    l, s = grid
    B, H, n, _ = f.shape
    sel = torch.full((B, H, n, k_total), -1, dtype=torch.int16)
    cnt = torch.zeros(B, H, n, dtype=torch.int16)
    for b in range(B):
        t, up = int(t_ctx[b]), paths(parent[b].tolist())
        n_win = (t - l) // s + 1 if t >= l else 0
        for h in range(H):
            z = f[b, h].double() @ kc[b, h, :n_win].double().t()
            for i in range(n):
                if t < 0 or not up[i]:
                    continue
                blk = (t + len(up[i]) - 1) // L
                forced = set(range(min(n_init, blk + 1))) | set(range(max(0, blk - n_local + 1), blk + 1))
                cand = list(range(n_init, blk - n_local + 1))
                score = {}
                for j in cand:
                    first = max(0, (L * j - l) // s + 1)           # x s + l > L j
                    last = min(n_win - 1, (L * (j + 1) - 1) // s)  # x s < L (j + 1)
                    score[j] = float(z[i, first:last + 1].max())
                take = sorted(cand, key=lambda j: (-score[j], j))[:k_total - len(forced)]
                got = sorted(forced | set(take))
                sel[b, h, i, :len(got)] = torch.tensor(got, dtype=torch.int16)
                cnt[b, h, i] = len(got)
    return sel, cnt


def attn(q, k, v, k_tree, v_tree, t_ctx, parent, sel, cnt, scale):
    """(o, w): the attention [B][Hq][n][D] and sum p |v| / sum p, the size that rounding errors go by."""
    B, HQ, n, D = q.shape
    H = k.shape[1]
    G = HQ // H
    o, w = (torch.zeros(B, HQ, n, D, dtype=torch.float64) for _ in range(2))
    for b in range(B):
        t, up = int(t_ctx[b]), paths(parent[b].tolist())
        if t < 0:
            continue
        for h in range(H):
            for i in range(n):
                if not up[i]:
                    continue
                r = 0 if sel.shape[2] == 1 else i
                listed = sel[b, h, r, :max(0, min(int(cnt[b, h, r]), sel.shape[3]))].tolist()
                tok = [x for j in sorted({j for j in listed if j >= 0}) for x in range(j * L, min(j * L + L, t))]
                kk = torch.cat((k[b, h, tok], k_tree[b, h, up[i]])).double()
                vv = torch.cat((v[b, h, tok], v_tree[b, h, up[i]])).double()
                a = torch.softmax(q[b, h * G:(h + 1) * G, i].double() @ kk.t() * scale, 1)
                o[b, h * G:(h + 1) * G, i] = a @ vv
                w[b, h * G:(h + 1) * G, i] = a @ vv.abs()
    return o, w


def verify(p, q, tokens, parent, u, vocab):
    """path [B][n], n_path [B], next_token [B]."""
    B, n = tokens.shape

    def row(x, b, i):
        y = x[b, i, :vocab].double()
        return torch.where((y > 0) & torch.isfinite(y), y, torch.zeros((), dtype=torch.float64))

    path = torch.full((B, n), -1, dtype=torch.int32)
    n_path, nxt = torch.zeros(B, dtype=torch.int32), torch.full((B,), -1, dtype=torch.int32)
    for b in range(B):
        up = paths(parent[b].tolist())
        if not up[0]:
            continue
        cur, got, c = 0, [0], 1.0
        m = row(p, b, 0)
        before = m  # the weights before the last rejection
        for i in range(1, n):
            x = int(tokens[b, i])
            if not up[i] or int(parent[b, i]) != cur or not 0 <= x < vocab:
                continue
            if q is not None and not m.sum() > 0:
                m = before
            qx = float(row(q, b, cur)[x]) if q is not None else 1.0
            if float(u[b, i]) * c * qx < float(m[x]):
                cur, c = i, 1.0
                got.append(i)
                m = before = row(p, b, i)
                continue
            before = m
            if q is not None:
                m = (m - c * row(q, b, cur)).clamp_min(0)
                c = float(m.sum()) if m.sum() > 0 else c
            else:
                c = max(c - float(m[x]), 0.0)
                m = m.clone()
                m[x] = 0
        if not m.sum() > 0:
            m = before
        path[b, :len(got)] = torch.tensor(got, dtype=torch.int32)
        n_path[b] = len(got)
        if m.sum() > 0:
            run = m.cumsum(0)
            over = torch.nonzero((run > float(u[b, 0]) * float(run[-1])) & (m > 0))
            nxt[b] = int(over[0]) if len(over) else int(torch.nonzero(m > 0)[-1])
    return path, n_path, nxt


def commit(t_ctx, path, n_path, k_tree, v_tree, k, v, kc, grid):
    """The caches of one layer after the append, in place; returns t_new."""
    l, s = grid
    t_new = t_ctx.clone()
    n, t_cap = path.shape[1], k.shape[2]
    for b in range(len(t_ctx)):
        t = int(t_ctx[b])
        if t < 0:
            continue
        got = 0
        for i in range(min(int(n_path[b]), n)):
            node = int(path[b, i])
            if not 0 <= node < n or t + i >= t_cap:
                break
            k[b, :, t + i] = k_tree[b, :, node]
            v[b, :, t + i] = v_tree[b, :, node]
            got += 1
        t_new[b] = t + got
        if kc is not None:
            for w in range(kc.shape[2]):
                if t < w * s + l <= t + got:
                    kc[b, :, w] = (k[b, :, w * s:w * s + l].double().sum(1) / l).to(torch.bfloat16)
    return t_new


def attn_bar(o, w):
    """How far a bf16 result may be: the weights rounded to bf16 (2^-8 of w), float32 logits and sums of at most
    16384 terms (2^-10 of w covers both for logits within +-64), the division (2^-23) and the bf16 rounding of the
    result (2^-8 of it, and of the error itself: 2^-15 w)."""
    return (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -15) * w + (2.0 ** -8 + 2.0 ** -22) * o.abs() + 2.0 ** -133


def tree(rng, n, kind):
    """parents of one tree of n nodes."""
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    return [-1] + [rng.randrange(max(0, i - 6), i) for i in range(1, n)]


SCALE = 1.0 / math.sqrt(128)
