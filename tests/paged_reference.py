"""Rotary positions and the operators over paged caches, written from their definitions in float64 with plain loops (test
infrastructure; shares no code with the library).  Tensors are torch tensors on the CPU; bf16 values are taken as they
are."""
import math

import torch

L = 64
SCALE = 1.0 / math.sqrt(128)


def turn(x, pos, freq, rot, pairs, scale, back=False):
    """(y, size): the rows x [.., n, 128] at the positions pos (broadcast over the rows), and scale (|x_a| + |x_b|) of
    each element's pair, 0 where an element passes."""
    x = x.double()
    y, size = x.clone(), torch.zeros_like(x)
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if pairs else (j, j + rot // 2)
        w = pos.double() * freq[j] * (-1.0 if back else 1.0)
        y[..., a] = scale * (x[..., a] * w.cos() - x[..., b] * w.sin())
        y[..., b] = scale * (x[..., a] * w.sin() + x[..., b] * w.cos())
        size[..., a] = size[..., b] = scale * (x[..., a].abs() + x[..., b].abs())
    return y, size


def turn_bar(y, size, pos_max, freq_max, half_step):
    """How far a turned row may be.  The angle in turns: float64 products (3 roundings of 2^-53 of pos freq, and the
    reference's own), then float32 of at most half a turn (2^-26 turns = 2^-23.3 radians); sine and cosine to 2 units in
    the last place below 1 (2^-23); scale, two products and a sum (3 roundings of 2^-24): 2^-23.3 + 2^-23 + 3 2^-24 <
    2^-21.4 of the pair's size.  Then one rounding by half_step (relative), 0 where float32 is stored: counted above."""
    return (2.0 ** -21.4 + pos_max * freq_max * 2.0 ** -50) * size + half_step * (1 + 2.0 ** -20) * y.abs() + 2.0 ** -133


def rows_of(pool, table, n, page, slot=1):
    """[H][n][128]: rows 0 .. n - 1 of a sequence (row i belongs to token i slot)."""
    tok = torch.arange(n) * slot
    return pool[table[tok // page].long(), :, tok % page // slot].transpose(0, 1)


def selection(f, keys, t, k_total, n_init, n_local, grid):
    """The set of one row at position t - 1: f [128], keys [windows complete][128]."""
    l, s = grid
    z = keys.double() @ f.double()
    blk = (t - 1) // L
    forced = set(range(min(n_init, blk + 1))) | set(range(max(0, blk - n_local + 1), blk + 1))
    cand = list(range(n_init, blk - n_local + 1))
    score = {}
    for j in cand:
        first, last = max(0, (L * j - l) // s + 1), min(len(z) - 1, (L * (j + 1) - 1) // s)
        score[j] = float(z[first:last + 1].max())
    take = sorted(cand, key=lambda j: (-score[j], j))[:max(0, k_total - len(forced))]
    return sorted(forced | set(take))


def attn(q, k_pool, v_pool, table, t_ctx, page, sel, cnt, scale):
    """(o, w): the attention [B][Hq][128] over the pages and sum p |v| / sum p."""
    B, HQ, D = q.shape
    H, n_pages = k_pool.shape[1], k_pool.shape[0]
    G = HQ // H
    o, w = (torch.zeros(B, HQ, D, dtype=torch.float64) for _ in range(2))
    for b in range(B):
        t = int(t_ctx[b])
        for h in range(H):
            if sel is None:
                tok = torch.arange(max(t, 0))
            else:
                listed = sel[b, h, 0, :max(0, min(int(cnt[b, h, 0]), sel.shape[3]))].tolist()
                tok = torch.tensor([x for j in sorted({j for j in listed if j >= 0}) for x in range(j * L, min(j * L + L, t))],
                                   dtype=torch.long)
            pg = table[b].long()[tok // page]
            on = (pg >= 0) & (pg < n_pages)
            tok, pg = tok[on], pg[on]
            if len(tok) == 0:
                continue
            kk, vv = k_pool[pg, h, tok % page].double(), v_pool[pg, h, tok % page].double()
            a = torch.softmax(q[b, h * G:(h + 1) * G].double() @ kk.t() * scale, 1)
            o[b, h * G:(h + 1) * G] = a @ vv
            w[b, h * G:(h + 1) * G] = a @ vv.abs()
    return o, w


def attn_bar(o, w):
    """How far a bf16 result may be.  A weight: its logit is a float32 sum of 128 products (gamma_128 = 2^-17 of
    scale |q| |k|, below 2^4 for unit normals: 2^-13), its exponential and its two bf16 parts 2^-15; sums of at most
    16384 terms a lane 2^-10; the same in the numerator (of w) and the denominator (of |o|); then the bf16 rounding."""
    e = 2.0 ** -10 + 2.0 ** -13 + 2.0 ** -15
    return e * w + (e + 2.0 ** -8 + 2.0 ** -15) * o.abs() + 2.0 ** -133
