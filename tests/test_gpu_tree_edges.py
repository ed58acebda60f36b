"""The operators over trees of drafted tokens where their results are most delicate, against the definitions in
float64 (tree_reference.py)."""
import pytest
import torch

import tree_reference as ref
from test_gpu_tree import ATTN, attn_inputs, dev, run_attn, say  # noqa: F401

pytestmark = pytest.mark.gpu


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
