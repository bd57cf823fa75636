"""The operators of beams at the far ends of what they take, and calls of other sizes in between."""
import math

import pytest
import torch

import paper_2405_18400_b200 as P
from tests.test_gpu_beams import BF16, DEV, F32, gen, i32, normal

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- attention: many steps in many runs
# (bf16 cache: 16 positions a step, float32 8; steps = sequences x 32 heads x steps of a sequence; products with 2368 runs pass 32 bits at 1 813 754)
@pytest.mark.parametrize("kv,own", [(BF16, 872), (BF16, 900), (BF16, 1023), (BF16, 1040), (F32, 450), (F32, 504), (F32, 520)])
def test_own_parts_of_millions_of_steps(kv, own):
    b, h, d, slots = 1024, 32, 64, 1500
    g = gen(own)
    kc, vc = normal(g, slots, h, d).to(kv), normal(g, slots, h, d).to(kv)
    q = normal(g, b, h, d)
    table = torch.randint(0, slots, (b, own), generator=g, device=DEV).to(torch.int32)     # the sequences' slots are shared, so that the cache is small
    got, lse = P.spd_shared_attention(q, kc, vc, table, i32([own] * b), return_lse=True)
    k, v = kc.double(), vc.double()
    for lo in range(0, b, 64):
        rows = table[lo: lo + 64].long()
        s = torch.einsum("bhd,bphd->bhp", q[lo: lo + 64].double(), k[rows]) * d ** -0.5
        want, want_lse = torch.einsum("bhp,bphd->bhd", torch.softmax(s, -1), v[rows]), torch.logsumexp(s, -1)
        # float32 arithmetic in parts of a hundred steps: scores and sums to some 2^-21 (the sum's terms are of random sign), ten times that to spare
        assert (got[lo: lo + 64].double() - want).abs().max() < 2.0 ** -17
        assert (lse[lo: lo + 64].double() - want_lse).abs().max() < 2.0 ** -17
