"""Attention whose results are whole numbers over a count (test infrastructure; shares no code with the library).

Head g's query is 64 in element g; a key holds 0 there if the head attends the token and -64 if it does not, which at the scale
1 / sqrt(128) is a score of -522 in powers of two below the attended ones: weights are exactly 1 and 0 in float32, whatever the
order, and so is a partial result of unattended tokens once it meets an attended one.  V is +1 or -1.  The sums of weights
and of V are whole numbers below 2^24, and the output is their quotient.  A token that is lost, counted twice or met by
another token's key moves all 128 sums by 1 or 2, of which those near zero show it at any length."""
import torch

BF = torch.bfloat16
SCALE = 128 ** -0.5


def signs(gen, *size):
    return (torch.randint(0, 2, size, generator=gen) * 2 - 1).to(torch.int8)


class Counts:
    """Pools of the sequences' tokens, and the outputs that belong to them.  What no token has is NaN."""

    def __init__(self, gen, table, t_ctx, n_pages, H, G, page, share=0.5):
        self.G, self.page, self.t_ctx, self.table = G, page, t_ctx, table
        self.k, self.v = (torch.full((n_pages, H, page, 128), float("nan"), dtype=BF) for _ in range(2))
        self.on, self.sign = [], []
        for b, t in enumerate(t_ctx):
            t = max(t, 0)
            on = torch.rand(H, G, t, generator=gen) < share
            on[:, 0] = True  # the first head attends everything
            sign = signs(gen, H, t, 128)
            key = torch.randint(-3, 4, (H, t, 128), generator=gen).to(BF)
            key[:, :, :G] = torch.where(on, 0.0, -64.0).transpose(1, 2).to(BF)
            for i in range(-(-t // page)):
                p, m = int(table[b, i]), min(page, t - i * page)
                self.k[p, :, :m], self.v[p, :, :m] = key[:, i * page:i * page + m], sign[:, i * page:i * page + m].to(BF)
            self.on.append(on)
            self.sign.append(sign)
        self.q = torch.zeros(len(t_ctx), H, G, 128)
        self.q[:, :, range(G), range(G)] = 64.0
        self.q = self.q.view(len(t_ctx), H * G, 1, 128).to(BF)

    def want(self, b, h, sel=None, cnt=None, lost=()):
        """float64 [G][128] of a row: (sums of V) / (attended tokens), 0 of none.  lost: tokens left out (planted)."""
        t = max(self.t_ctx[b], 0)
        if sel is None:
            seen = torch.ones(t, dtype=torch.bool)
        else:
            seen = torch.zeros(t, dtype=torch.bool)
            for j in sel[b, h, 0, :int(cnt[b, h, 0])].tolist():
                if j >= 0:
                    seen[64 * j:64 * j + 64] = True
        seen[list(lost)] = False
        on = (self.on[b][h] & seen).double()
        n = on.sum(1, keepdim=True)
        o = on @ self.sign[b][h].double() / n.clamp_min(1)
        # a head that attends none of the tokens seen weighs them all alike
        flat = seen.double() @ self.sign[b][h].double() / max(int(seen.sum()), 1)
        return torch.where(n > 0, o, flat)


def bar(o):
    """The quotient: a reciprocal and a product in float32 (2^-24 each) and the rounding to bf16 (2^-8)."""
    return (2.0 ** -8 + 2.0 ** -22) * o.abs()
