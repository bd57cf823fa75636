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


# ---------------------------------------------------------------- selection: one workspace, calls of different sizes in turn
def selection(seed, r, w, v, offset=0):
    g = gen(seed)
    wide = normal(g, r, w, v + 4)
    return wide[..., offset: offset + v], -torch.rand(r, w, generator=g, device=DEV)


def same_selections(z, score, workspace):
    want = P.spd_beam_select(z, score)
    got = P.spd_beam_select(z, score, workspace=workspace)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_selections_workspace_serves_other_numbers_of_requests():
    z, score = selection(1, 100, 4, 3000)
    ws = P.spd_beam_select_workspace(z)
    for n in (100, 10, 100, 1, 65, 100):
        same_selections(z[:n], score[:n], ws)
    big = P.spd_beam_select_workspace(selection(2, 150, 16, 9000)[0])
    for k, (r, w, v, offset) in enumerate([(150, 16, 9000, 0), (7, 5, 40000, 1), (150, 2, 300, 0), (3, 16, 9000, 2), (90, 8, 5000, 0), (150, 16, 9000, 3)]):
        same_selections(*selection(10 + k, r, w, v, offset), big)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("w,v", [(3, 32000), (8, 32000), (2, 100000), (16, 4099), (32, 40000)])
def test_a_selections_workspace_is_enough_for_fewer_requests(dtype, w, v):
    """The fewer requests, the more slices a row is cut into; the room asked for covers that, for rows that begin on a vector and others."""
    z, score = selection(3, 40, w, v)
    z = z.to(dtype)
    ws = P.spd_beam_select_workspace(z)
    for n in (40, 39, 37, 36, 31, 19, 18, 12, 9, 5, 3, 2, 1):
        assert P.spd_beam_select_workspace(z[:n]).numel() <= ws.numel()
        same_selections(z[:n], score[:n], ws)
        if v % 8:
            continue
        skewed = torch.empty(n, w, v + 1, dtype=dtype, device=DEV)[..., 1:].copy_(z[:n])
        same_selections(skewed, score[:n], ws)


# ---------------------------------------------------------------- attention: one workspace for as many rows, sequences and prefixes or fewer
def attention_room(x, kv, heads, kv_heads, dim, n, b, g):
    q, cache = torch.empty(n, heads, dim, dtype=x, device=DEV), torch.empty(1, kv_heads, dim, dtype=kv, device=DEV)
    tables = torch.empty(b, 1, dtype=torch.int32, device=DEV)
    return P.spd_shared_attention_workspace(q, cache, tables, tables[:g] if g else None).numel()


@pytest.mark.parametrize("x,kv,heads,kv_heads,dim,more,fewer", [
    (F32, BF16, 8, 8, 128, (8, 8, 1), (4, 4, 1)), (F32, F32, 8, 8, 128, (9, 9, 1), (8, 8, 1)), (F32, F32, 40, 40, 128, (16, 8, 1), (8, 8, 1)),
    (F32, BF16, 1, 1, 128, (8, 8, 8), (8, 8, 1)), (F32, BF16, 1, 1, 128, (8, 8, 8), (8, 8, 0)), (F32, BF16, 32, 32, 64, (20, 20, 1), (4, 4, 1))])
def test_an_attentions_workspace_is_enough_for_less(x, kv, heads, kv_heads, dim, more, fewer):
    assert attention_room(x, kv, heads, kv_heads, dim, *more) >= attention_room(x, kv, heads, kv_heads, dim, *fewer)


@pytest.mark.parametrize("x,kv", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (8, 2, 128), (6, 1, 256)])
def test_smaller_calls_in_a_larger_ones_workspace(x, kv, heads, kv_heads, dim):
    """A search whose beams and prompts end: fewer rows go to other kernels, with the room that was taken at its start."""
    g = gen(dim)
    groups, beams, prefix, own, slots = 3, 8, 150, 20, 900
    b = groups * beams
    kc, vc = normal(g, slots, kv_heads, dim).to(kv), normal(g, slots, kv_heads, dim).to(kv)
    q = normal(g, b, heads, dim).to(x)
    ptab = torch.randint(0, slots // 10, (groups, prefix // 10), generator=g, device=DEV).to(torch.int32)
    otab = torch.randint(0, slots, (b, own), generator=g, device=DEV).to(torch.int32)
    ws = P.spd_shared_attention_workspace(q, kc, otab, ptab)
    for n in (groups, 2, 1, 0):
        for w in (beams, 5, 4, 2, 1):
            rows = max(n, 1) * w
            kw = dict(prefix_table=ptab[:n], prefix_len=i32([prefix] * n), prefix_page=10, group_start=i32([w * i for i in range(n + 1)])) if n else {}
            call = lambda space: P.spd_shared_attention(q[:rows], kc, vc, otab[:rows], i32([own] * rows), workspace=space, **kw)   # noqa: E731
            assert torch.equal(call(ws), call(None))


# ---------------------------------------------------------------- attention: arrays that are no partition
@pytest.mark.parametrize("x,kv", [(BF16, BF16), (F32, BF16), (F32, F32)])
def test_where_rows_or_groups_fall_nothing_is_seen(x, kv):
    g = gen(11)
    h, d, slots, b = 4, 64, 300, 5
    kc, vc, q = normal(g, slots, h, d).to(kv), normal(g, slots, h, d).to(kv), normal(g, 9, h, d).to(x)
    ptab = torch.randint(0, slots, (2, 70), generator=g, device=DEV).to(torch.int32)
    otab = torch.randint(0, slots, (b, 20), generator=g, device=DEV).to(torch.int32)
    good = ([0, 2, 4, 4, 6, 9], [0, 2, 5])
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def call(rows, groups):
        status.zero_()
        return P.spd_shared_attention(q, kc, vc, otab, i32([20] * b), prefix_table=ptab, prefix_len=i32([70, 33]), group_start=i32(groups), q_start=i32(rows),
                                      return_lse=True, status=status)
    want = call(*good)
    assert int(status) == 0
    for rows, groups in (([5, 6, 0, 3, 6, 9], good[1]), ([1, 2, 0, 9, 9, 9], good[1]), ([0, 9, 0, 9, 0, 9], good[1]), ([0, 2, 4, 4, 9, 7], good[1]),
                         (good[0], [2, 0, 5]), (good[0], [0, 5, 1]), ([9, 7, 5, 3, 1, 0], [5, 3, 0])):
        out, lse = call(rows, groups)
        assert int(status) == -3 and not out.any() and (lse == -math.inf).all()
    out, lse = call([-4, 2, 4, 4, 6, 1000], [-1, 2, 70])       # entries outside the rows and sequences, in order: as far as they lie inside
    assert torch.equal(out[4:6], want[0][4:6]) and int(status) == 0
    again = call(*good)
    assert int(status) == 0 and all(torch.equal(a, b) for a, b in zip(want, again))


# ---------------------------------------------------------------- refusals
def test_workspaces_that_repeat_their_elements_are_refused():
    """A view of a few bytes may count as many: only those that are there may be written."""
    q, kc, table = torch.zeros(3, 2, 64, device=DEV), torch.zeros(8, 2, 64, device=DEV), i32([[0], [1], [2]])
    z, score = torch.zeros(2, 3, 10, device=DEV), torch.zeros(2, 3, device=DEV)
    few = torch.zeros(64, dtype=torch.uint8, device=DEV)
    for space in (few[:1].expand(1 << 26), few[:1, None].expand(1, 1 << 26), few.view(2, 32).t()):
        with pytest.raises(ValueError):
            P.spd_shared_attention(q, kc, kc.clone(), table, i32([1, 1, 1]), workspace=space)
        with pytest.raises(ValueError):
            P.spd_beam_select(z, score, workspace=space)
    assert not few.any()


def test_an_append_to_a_table_without_pages_is_refused():
    """An empty tensor has no address, and no table means that places are slots: nothing may go there."""
    x, pos = torch.ones(2, 1, 8, device=DEV), i32([0, 1])
    for shape in ((0, 4), (2, 0), (0, 0)):
        kc, vc = torch.zeros(6, 1, 8, device=DEV), torch.zeros(6, 1, 8, device=DEV)
        with pytest.raises(ValueError):
            P.spd_cache_append(x, x, kc, vc, pos, None, table=torch.empty(shape, dtype=torch.int32, device=DEV))
        assert not kc.any() and not vc.any()
    P.spd_cache_append(x[:0], x[:0], kc, vc, pos[:0], None, table=torch.empty(0, 0, dtype=torch.int32, device=DEV))   # no tokens: no pages needed


def test_return_lse_is_any_truth_value():
    q, kc, table = torch.ones(3, 2, 64, device=DEV), torch.ones(8, 2, 64, device=DEV), i32([[0], [1], [2]])
    call = lambda lse: P.spd_shared_attention(q, kc, kc.clone(), table, i32([1, 1, 1]), return_lse=lse)   # noqa: E731
    for yes in (True, 1, "yes", [0], torch.ones(1)):
        out, lse = call(yes)
        assert out.shape == q.shape and lse.shape == (3, 2)
    for no in (False, 0, None, ""):
        assert torch.equal(call(no), out)


def test_states_that_lie_on_one_another_are_refused():
    parent = i32([[1, 0], [1, 1]])
    one, other = torch.arange(8.0, device=DEV).view(2, 2, 2), torch.arange(8.0, device=DEV).view(2, 2, 2)
    row = torch.arange(2.0, device=DEV)
    wide = torch.arange(12.0, device=DEV)
    layers = one.expand(3, 2, 2, 2)
    many = [torch.arange(8.0, device=DEV).view(2, 2, 2) for _ in range(10)]
    for states, dim in (([one, one], 0), ([one, other, one], 0), (row.expand(2, 2, 2), 0), (one[:1].expand(2, 2, 2), 0), (layers, 1),
                        (wide.as_strided((2, 2, 2), (4, 1, 1)), 0), (many + [many[0]], 0)):
        with pytest.raises(ValueError):
            P.spd_beam_reorder(states, parent, dim=dim)
    assert all(t.flatten().tolist() == list(range(8)) for t in [one, other] + many)
    pair = torch.arange(16.0, device=DEV).view(2, 2, 2, 2)                    # two states side by side in one buffer lie apart
    P.spd_beam_reorder([pair[:, :, 0], pair[:, :, 1]], parent)
    assert pair.flatten().tolist() == [4, 5, 6, 7, 0, 1, 2, 3, 12, 13, 14, 15, 12, 13, 14, 15]
    P.spd_beam_reorder([row.view(1, 1, 2).expand(2, 1, 2)], i32([[0], [0]]))   # one beam: nothing moves


def test_outputs_that_repeat_their_elements_are_refused():
    x, pos, table = torch.zeros(3, 2, 64, device=DEV), i32([0, 1, 2]), i32([[0], [1], [2]])
    cache = torch.zeros(8, 2, 64, device=DEV)
    for twice in (cache[:1].expand(8, 2, 64), cache[:, :1].expand(8, 2, 64)):
        for caches in ((twice, cache), (cache, twice)):
            with pytest.raises(ValueError):
                P.spd_cache_append(x, x, *caches, pos, None, index=pos)
        with pytest.raises(ValueError):
            P.spd_cache_append(None, None, None, None, pos, None, q=x, q_out=twice[:3])
        with pytest.raises(ValueError):
            P.spd_shared_attention(x, cache, cache, table, i32([1, 1, 1]), out=twice[:3])
        P.spd_shared_attention(twice[:3], twice, twice, table, i32([1, 1, 1]))     # what is read may be
        P.spd_cache_append(twice[:3], twice[:3], cache, cache.clone(), pos, None, q=twice[:3], index=pos)


# ---------------------------------------------------------------- selection: temperatures of any size
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_select_at_an_infinite_temperature(dtype):
    """All tokens that are options are alike; in a beam the larger logit stands first all the same."""
    g = gen(21)
    w, v = 3, 5000
    z = normal(g, 1, w, v).to(dtype)
    z[0, :, 100:4900] = -math.inf
    score = torch.tensor([[-0.25, -1.0, -0.5]], device=DEV)
    token, parent, new, _, _ = P.spd_beam_select(z, score, tau=math.inf)
    order = torch.sort(z[0, 0].float(), descending=True, stable=True).indices[:w]
    assert token[0].tolist() == order.tolist() and parent[0].tolist() == [0, 0, 0]
    assert (new[0].double() + 0.25 + math.log(200)).abs().max() <= 2.0 ** -23 * 16


def test_select_at_a_temperature_near_zero():
    """1 / tau is past float32: the largest logit has all the weight, shared by those that equal it."""
    w, v = 3, 5000
    z = torch.zeros(1, w, v, device=DEV)
    z[0, 0, [7, 4000]] = 0.01
    z[0, 1, 55] = 0.01
    z[0, 2] = -math.inf
    z[0, 2, 9] = -5.0
    score = torch.tensor([[-1.0, -2.0, -3.0]], device=DEV)
    token, parent, new, _, _ = P.spd_beam_select(z, score, tau=1e-39)
    assert list(zip(parent[0].tolist(), token[0].tolist())) == [(0, 7), (0, 4000), (1, 55)]
    assert (new[0].double() - torch.tensor([-1 - math.log(2), -1 - math.log(2), -2.0], device=DEV)).abs().max() <= 2.0 ** -23 * 18


# ---------------------------------------------------------------- append: positions without an angle
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
def test_positions_outside_the_angles_write_no_query_and_no_key(pairs):
    g = gen(31)
    n, h, d = 4, 2, 64
    q, k, v = normal(g, n, h, d), normal(g, n, h, d), normal(g, n, h, d)
    rope = P.spd_rope_table(8, d, device=DEV)
    for index, bad, told in (([3, 1, 0, 2], 2, -3), ([3, 1, -1, 2], 2, 0)):          # a token that is stored; padding
        for place in (8, -1, 2 ** 31 - 1, -2 ** 31):
            pos = [5, 7, 0, 1]
            pos[bad] = place
            kc, vc, out = torch.full((4, h, d), 7.0, device=DEV), torch.full((4, h, d), 7.0, device=DEV), torch.full((n, h, d), 7.0, device=DEV)
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            P.spd_cache_append(k, v, kc, vc, i32(pos), rope, q=q, q_out=out, index=i32(index), pairs=pairs, status=status)
            assert int(status) == told
            assert (out[bad] == 7).all() and (kc[0] == 7).all()
            assert torch.equal(vc[0], v[bad]) if told else (vc[0] == 7).all()
            pos[bad] = 0
            want = P.spd_cache_append(k, v, kc.clone(), vc.clone(), i32(pos), rope, q=q, index=i32(index), pairs=pairs)
            rest = [i for i in range(n) if i != bad]
            assert torch.equal(out[rest], want[rest]) and torch.equal(vc[[3, 1, 2]], v[rest]) and (kc[1:] != 7).any()


# ---------------------------------------------------------------- attention: operands of any size that is said to be taken
@pytest.mark.parametrize("x,kv", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("rows", [1, 20])
def test_values_and_keys_up_to_the_largest(x, kv, rows):
    """Values just below the largest that are taken, whose weighted sum stays inside float32; keys whose scores do with small queries."""
    g = gen(rows)
    h, d, own = 2, 64, 40
    largest = 2.0 ** 128 - 2.0 ** 120 if kv == BF16 else 2.0 ** 128 - 2.0 ** 117
    kc, vc = normal(g, own, h, d).to(kv), normal(g, own, h, d).to(kv)
    q = normal(g, rows, h, d).to(x)
    kc[7] = q[0] * -3
    vc[7, :, :3], vc[7, :, 3:] = largest / 64, 1.0          # 40 weights of 1 at most: the sum stays inside
    kc[9, :, 0], kc[9, :, 1:] = -largest, 0.0
    q[:, :, 1:] *= 2.0 ** -4
    q[:, :, 0] = 2.0 ** -126
    out, lse = P.spd_shared_attention(q, kc, vc, torch.arange(own, device=DEV).to(torch.int32).expand(rows, own).contiguous(), i32([own] * rows), return_lse=True)
    s = torch.einsum("nhd,phd->nhp", q.double(), kc.double()) * d ** -0.5
    want = torch.einsum("nhp,phd->nhd", torch.softmax(s, -1), vc.double())
    assert out.isfinite().all() and lse.isfinite().all()
    assert ((out.double() - want).abs() <= want.abs() * (2.0 ** -8 if x == BF16 else 2.0 ** -18) + 2.0 ** -16).all()
    assert ((lse.double() - torch.logsumexp(s, -1)).abs() <= 2.0 ** -18).all()


def test_pairs_that_are_not_known_are_refused():
    with pytest.raises(P.SpdError):
        P.spd_cache_append(None, None, None, None, i32([0]), P.spd_rope_table(2, 8, device=DEV), q=torch.zeros(1, 1, 8, device=DEV), pairs="neither")
