"""How exact the attention over shared prefixes is, in the 2-norm over all outputs, which a term left out of a product shows in at any length.

Inputs are normal, so what n roundings of independent sign do to a sum grows as the sum itself does: a weight that is off by a share e of itself
moves the outputs by a share e of their norm."""
import math

import pytest
import torch

from tests.test_gpu_beams import ATTENTION, BF16, F32, FEW_ROWS, MANY_STEPS, attention_case, plain_attention, run_attention

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


# float32 queries.  Scores: products to 2^-22 of themselves, some d / 16 additions that truncate (2^-23 of the partial sum, which is a few units at most):
# 2^-20 of a unit, which is what it moves the weights and, by random signs, the outputs by.  Weighted values: products to 2^-22, some ten to twenty
# additions of a run that truncate, towards zero, by half of 2^-23 on average: 2^-20.  Both together, and as much again for the join: 2^-19.
FLOAT_BOUND = 2.0 ** -19


@pytest.mark.parametrize("kv", [BF16, F32])
@pytest.mark.parametrize("case", LONG + [case for case in FEW_ROWS if max(case[3], default=0) + max(case[5]) >= 100])
def test_float32_outputs_have_no_term_left_out(kv, case):
    got, lse, want, want_lse = attended(F32, kv, case)
    assert relative(got, want) <= FLOAT_BOUND
    seen = want_lse > -math.inf
    assert (lse.double() - want_lse)[seen].abs().max() <= 2 * FLOAT_BOUND


def leading(x, bits):
    """The first `bits` significant bits of float32 values, by truncation."""
    return (x.float().view(torch.int32) & (-1 << (24 - bits))).view(F32).double()


@pytest.mark.parametrize("left_out", ["third term of the queries", "third term of the weights", "second part of the keys", "second part of the values",
                                      "second part of the queries", "second part of the weights"])
@pytest.mark.parametrize("positions", [100, 1000, 6000])
def test_a_term_left_out_would_show(left_out, positions):
    """What the outputs would be with one term fewer in one operand (bf16 terms have 8 bits each, tf32 ones 11) is past the bound at every length."""
    g = torch.Generator().manual_seed(positions)
    n, d = 8, 128
    q, k, v = (torch.randn(m, d, generator=g) for m in (n, positions, positions))

    def attend(cut):
        s = (cut("queries", q) @ cut("keys", k).T) * 1.3 * d ** -0.5
        p = torch.exp(s - s.amax(-1, keepdim=True))
        return cut("weights", p) @ cut("values", v) / p.sum(-1, keepdim=True)

    bits = 16 if left_out.startswith("third") else 11
    want = attend(lambda name, x: x.double())
    less = attend(lambda name, x: leading(x, bits) if left_out.endswith(name) else x.double())
    assert relative(less, want) > 2 * FLOAT_BOUND
