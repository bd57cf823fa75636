"""How exact the attention over shared prefixes is, in the 2-norm over all outputs, which a term left out of a product shows in at any length.

Inputs are normal, so what n roundings of independent sign do to a sum grows as the sum itself does: a weight that is off by a share e of itself
moves the outputs by a share e of their norm."""
import pytest
import torch

from tests.test_gpu_beams import ATTENTION, BF16, MANY_STEPS, attention_case, plain_attention, run_attention

pytestmark = pytest.mark.gpu

# lengths that give a row many weights of like size; several rows and parts, causal ones
LONG = [case for case in ATTENTION + MANY_STEPS if max(case[3], default=0) + max(case[5]) >= 100]


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


def attended(x, kv, case):
    hq, hk, d, plens, groups, olens, counts, ppage, opage = case
    q, kc, vc, ptab, otab, starts = attention_case(hq * d + len(olens) + 1, x, kv, hq, hk, d, plens, groups, olens, counts, ppage, opage, pad=8)
    scale = 1.3 * d ** -0.5
    got, lse = run_attention(q, kc, vc, ptab, otab, starts, plens, groups, olens, ppage, opage, scale, all(c == 1 for c in counts))
    want, want_lse, _ = plain_attention(q, kc, vc, scale, plens, ptab, ppage, groups, olens, otab, opage, starts)
    return got, lse, want, want_lse


@pytest.mark.parametrize("case", LONG)
def test_bf16_outputs_are_off_by_their_rounding_alone(case):
    """Rounding the exact outputs to bf16 moves them by some 2^-9.2 of their norm.  What comes before it (weights to 2^-16, float32 sums, scores to
    2^-20) adds a hundredth of that, and in quadrature nothing: a twentieth more is allowed.  (One bf16 term for the weights adds a third.)"""
    got, _, want, _ = attended(BF16, BF16, case)
    assert relative(got, want) <= 1.05 * relative(want.to(BF16), want)
