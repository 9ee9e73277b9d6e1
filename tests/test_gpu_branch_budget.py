"""branch_weights and branch_evict against plain forms in 64 bits, and the operators of a sequence's pages together.

Tolerances of the weights (u = 2^-24): a logit of 128 products summed in float is off by at most 2^-17 A (A: sum |q_i k_i| scale), scaled and shifted
with one rounding each, which the exponential makes a relative error of the weight of 2 * 2^-17 A + 2^-22 |lse| (the logarithm turned to base
two); the exponential 2^-22; a sum of n weights, all of one sign, n u; the old weight and its product with the decay 2 u.  The hardware's exponential
gives zero in the place of a number below 2^-126, the smallest normal float: each of the n weights may lack that much.
The eviction moves bits: equality.
"""
import numpy as np
import pytest

import paper_2504_15364_amd as kd
from test_gpu_branch import close, gen, ints, paged, put_rows, rows_of, tables, wide  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ------------------------------------------------------------------------------------------------ weights
def gathered(q, k, lse, before, new, observe, scale):
    """One sequence: q [hq][T][d], k [hkv][n][d] in double, lse [hq][T]: the weight that each row gets, and the bound of its error."""
    hq, T, d = q.shape
    hkv, n = k.shape[:2]
    x = q.double().reshape(hkv, -1, d)
    a = torch.matmul(x, k.transpose(1, 2).contiguous()).view(hkv, hq // hkv, T, n) * scale
    A = torch.matmul(x.abs(), k.abs().transpose(1, 2).contiguous()).view(hkv, hq // hkv, T, n) * scale
    j = torch.arange(T, device="cuda")[:, None]
    seen = (torch.arange(n, device="cuda")[None] <= before + j) & (j >= (T - observe if observe else 0))
    L = lse.double().view(hkv, hq // hkv, T, 1)
    p = torch.where(seen & (L > float("-inf")), (a - L).exp(), 0.0)
    e = 2.0 ** -16 * A + 2.0 ** -21 * L.abs().nan_to_num(posinf=0.0) + 2.0 ** -21
    return p.sum((1, 2)), (p * (e + hq * T * 2.0 ** -24)).sum((1, 2)) + hq * T * 2.0 ** -126


WEIGHTS = [
    # hq, hkv, d, page, Bt, lens, n_new, observe
    (4, 1, 64, 8, 1, [0], None, 0),                                              # the token's own row alone
    (32, 8, 128, 16, 1, [15, 16, 0, 31, 700, -1], None, 0),
    (28, 4, 128, 32, 4, [3, 30, 64, 100], [4, 0, 2, 9], 0),                      # 28 rows
    (64, 1, 64, 8, 1, [100], None, 0),                                           # 64 query heads: a tile of query rows
    (16, 16, 128, 16, 20, [5, 700], None, 0),
    (8, 2, 64, 1024, 37, [1020, 0, 5000], [37, 1, 36], 0),
    (8, 2, 128, 16, 65, [511, 0, 512, 447], None, 0),                            # rows that end with a block of 512 and behind it
    (6, 2, 128, 32, 90, [3, 30, 64, -1, 100], [90, 0, 2, 90, 1000], 40),
    (32, 8, 128, 64, 200, [3000], None, 32),
    (32, 8, 128, 64, 200, [3000, 77], [200, 5], 7),                              # 28 rows of the last tokens; fewer tokens than are looked at
    (24, 8, 128, 32, 300, [500 * i % 1300 for i in range(8)], [(97 * i + 300) % 301 for i in range(8)], 0),
    (8, 1, 128, 16, 1500, [0], None, 0),                                         # a prompt of its own: the causal triangle
    (8, 1, 64, 16, 1500, [4000], None, 1),
]


@pytest.mark.parametrize("case", WEIGHTS, ids=[str(i) for i in range(len(WEIGHTS))])
@pytest.mark.parametrize("decay", [1.0, 0.75, 0.0])
@pytest.mark.parametrize("size", [1.0, 5.0])
def test_weights(case, decay, size):
    hq, hkv, d, page, Bt, lens, n_new, observe = case
    n = len(lens)
    g = gen(500 + hq + Bt + page)
    new = [0 if L < 0 else (Bt if n_new is None else min(n_new[s], Bt)) for s, L in enumerate(lens)]
    k_pages, _, table = paged(lens, Bt, page, hkv, d, g)
    w_pages = torch.full((len(k_pages), hkv, page), float("nan"), device="cuda")   # weights of rows that are not there yet
    old = []
    for s, L in enumerate(lens):
        old.append(torch.rand((hkv, max(L, 0)), **g))
        if L >= 0:
            put_rows(k_pages, table, s, torch.randn((hkv, L + new[s], d), **g).mul_(size).bfloat16())
            put_rows(w_pages, table, s, old[s] if decay else torch.full_like(old[s], float("nan")))
    q = torch.randn((n, Bt, hq, d), **g).mul_(size).bfloat16().transpose(1, 2)
    lse = torch.full((n, hq, Bt), float("nan"), device="cuda")
    for s, L in enumerate(lens):
        q[s, :, new[s]:] = float("nan")
        if new[s]:
            k = rows_of(k_pages, table, s, L + new[s])
            a = torch.matmul(q[s, :, :new[s]].double().reshape(hkv, -1, d), k.transpose(1, 2).contiguous()).view(hq, new[s], -1) * d ** -0.5
            hidden = torch.arange(L + new[s], device="cuda")[None] > L + torch.arange(new[s], device="cuda")[:, None]
            lse[s, :, :new[s]] = (torch.logsumexp(a.masked_fill(hidden, float("-inf")), -1) + torch.rand((hq, new[s]), **g)).float()
    if new[0] > 2:
        lse[0, :, 1] = float("-inf")                             # a query that saw no key gives no weight
    before = w_pages.clone()
    # (a workspace that holds NaN everywhere)
    work = torch.full((kd.branch_weights_workspace_bytes(n, hq, hkv, d, Bt, observe) + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    kw = dict(n_new=None if n_new is None else ints(n_new), observe=observe, decay=decay)
    kd.branch_weights(q, k_pages, w_pages, table, ints(lens), lse, workspace=work, **kw)
    assert bool((work[-512:] == 0xFF).all())
    again = before.clone()
    kd.branch_weights(q, k_pages, again, table, ints(lens), lse, **kw)
    assert torch.equal(again.view(torch.int32), w_pages.view(torch.int32))
    for s, L in enumerate(lens):
        m = new[s]
        if not m:
            continue
        got = rows_of(w_pages, table, s, L + m)
        want, bound = gathered(q[s, :, :m], rows_of(k_pages, table, s, L + m), lse[s, :, :m], L, m, observe, d ** -0.5)
        if decay:
            want[:, :L] += decay * old[s].double()
        close(got, want, bound + 2.0 ** -22 * want, f"sequence {s}")
        put_rows(before, table, s, got.float())
    assert torch.equal(before.view(torch.int32), w_pages.view(torch.int32))   # nothing else was touched


@pytest.mark.parametrize("hq,Bt", [(4, 3), (4, 40)])
def test_weights_leave_rows_of_absent_pages(hq, Bt):
    hkv, d, page, L = 2, 64, 8, 90
    g = gen(61)
    k_pages, _, table = paged([L], Bt, page, hkv, d, g)
    put_rows(k_pages, table, 0, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    w_pages = torch.rand((len(k_pages), hkv, page), **g)
    q, lse = torch.randn((1, hq, Bt, d), **g).bfloat16(), torch.full((1, hq, Bt), 5.0, device="cuda")
    whole = w_pages.clone()
    kd.branch_weights(q, k_pages, whole, table, ints([L]), lse)
    holes = table.clone()
    holes[0, 2], holes[0, 5], holes[0, L // page] = -1, 10 ** 6, len(k_pages)
    before = w_pages.clone()
    kd.branch_weights(q, k_pages, w_pages, holes, ints([L]), lse)
    for i in (2, 5, L // page):
        whole[table[0, i]] = before[table[0, i]]
    assert torch.equal(whole, w_pages)
    # a length beyond the table: all its rows are old ones and seen by every token
    kd.branch_weights(q, k_pages, w_pages, table[:, :4].contiguous(), ints([10 ** 9]), lse, decay=0.0)
    want, bound = gathered(q[0], rows_of(k_pages, table, 0, 4 * page), lse[0], 4 * page, Bt, 0, d ** -0.5)
    close(rows_of(w_pages, table, 0, 4 * page), want, bound, "beyond its table")


# ------------------------------------------------------------------------------------------------ eviction
def evicted(w, p, late, budget):
    """One head: which rows stay, in the order of (late positions, weight, lower position, lower row); from, to of the moves."""
    n = len(w)
    w = np.where(np.isnan(w), -np.inf, w.astype(np.float64))
    stays = np.zeros(n, dtype=bool)
    stays[np.lexsort((np.arange(n), p, -w, ~(p >= late)))[:budget]] = True
    return budget + np.flatnonzero(stays[budget:]), np.flatnonzero(~stays[:budget])


def evict_case(hkv, d, page, lens, new, budget, g, weights, seqs_pos0, positions="shuffled", Bt=None):
    """Pools of distinct rows, weights and positions; and what they are after the eviction."""
    Bt = max(new) if Bt is None else Bt
    k, v, table = paged(lens, Bt, page, hkv, d, g)
    k, v = torch.randn(k.shape, **g).bfloat16(), torch.randn(k.shape, **g).bfloat16()
    w = torch.full((len(k), hkv, page), float("nan"), device="cuda")
    p = torch.full((len(k), hkv, page), -12345, dtype=torch.int32, device="cuda")
    for s, (L, m) in enumerate(zip(lens, new)):
        if L < 0:
            continue
        put_rows(w, table, s, weights((hkv, L + m), g))
        held = torch.stack([torch.randperm(L + seqs_pos0[s], generator=g["generator"], device="cuda")[:L] for _ in range(hkv)]) if positions == "shuffled" \
            else torch.arange(L, device="cuda").expand(hkv, L)
        put_rows(p, table, s, held.to(torch.int32))
    return k, v, w, p, table


def after_eviction(pools, table, lens, new, pos0, budget, window):
    k, v, w, p = (x.clone() for x in pools)
    page = k.shape[2]
    for s, (L, m) in enumerate(zip(lens, new)):
        if L < 0:
            continue
        r = torch.arange(L, L + m, device="cuda")
        p[table[s, r // page].long(), :, r % page] = (pos0[s] + r)[:, None].to(torch.int32).expand(-1, k.shape[1])
        n = L + m
        if n <= budget:
            continue
        ws, ps = rows_of(w, table, s, n).cpu().numpy(), rows_of(p, table, s, n).cpu().numpy().astype(np.int64)
        for h in range(k.shape[1]):
            fro, to = (torch.from_numpy(x).cuda() for x in evicted(ws[h], ps[h], pos0[s] + n - window, budget))
            for x in (k, v, w, p):
                x[table[s, to // page].long(), h, to % page] = x[table[s, fro // page].long(), h, fro % page]
    return k, v, w, p


def same(got, want):
    for a, b in zip(got, want):
        i = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(a.view(i), b.view(i))


spread = lambda shape, g: torch.exp(3.0 * torch.randn(shape, **g))  # noqa: E731
WEIGHT_KINDS = {
    "spread": spread,
    "ties": lambda shape, g: torch.randint(0, 4, shape, **g).float() * 0.25,                     # whole classes of equal weights
    "zero": lambda shape, g: torch.where(torch.rand(shape, **g) < 0.5, -0.0, 0.0),                # both zeros are one weight
    "odd": lambda shape, g: torch.where(torch.rand(shape, **g) < 0.1, float("nan"), torch.where(torch.rand(shape, **g) < 0.1, float("inf"), torch.where(
        torch.rand(shape, **g) < 0.1, float("-inf"), torch.randn(shape, **g)))),
    "alike": lambda shape, g: torch.full(shape, 0.5, device="cuda"),                               # positions decide
    "close": lambda shape, g: 1.0 + 2.0 ** -23 * torch.randint(0, 40, shape, **g).float(),        # borders in the last bits
}
EVICT = [
    # hkv, d, page, Bt, lens, new, budget, window
    (1, 64, 8, 1, [96], [1], 96, 0),
    (8, 128, 64, 1, [100, 99, 0, 100, -1], [1, 1, 1, 0, 1], 100, 10),           # at, below and far below the budget; without a new token; not in use
    (2, 128, 16, 128, [500, 500, 13], [128, 5, 0], 500, 64),
    (4, 64, 32, 40, [1000, 300], [40, 40], 200, 0),                             # far above the budget
    (2, 64, 8, 3, [50], [3], 1, 0),                                             # one row is left
    (2, 128, 16, 700, [0, 100], [700, 1], 99, 98),                              # all but one row by position
    (1, 128, 1024, 9, [20000], [9], 9000, 100),                                 # more rows than are kept in LDS
    (2, 64, 64, 1, [40000], [1], 39999, 0),
    (3, 64, 16, 2, [33] * 100, [2, 1] * 50, 33, 4),
    (2, 128, 64, 1, [4000, 3999, 1], [1, 1, 1], 4000, 0),                       # up to 4096 rows in registers; one too many, none, none
    (2, 64, 32, 700, [3000, 2500], [700, 64], 1100, 100),                       # more moves than the workgroup makes itself
    (1, 128, 64, 30, [16000], [30], 15999, 500),                                # up to 16384 rows
    (2, 64, 64, 1, [12000, 5000], [1, 0], 6000, 0),                             # half of the rows at once
]


@pytest.mark.parametrize("case", EVICT, ids=[str(i) for i in range(len(EVICT))])
@pytest.mark.parametrize("kind", WEIGHT_KINDS)
def test_eviction(case, kind):
    hkv, d, page, Bt, lens, new, budget, window = case
    g = gen(700 + budget + hkv)
    pos0 = [(37 * s) % 50 for s in range(len(lens))]
    k, v, w, p, table = evict_case(hkv, d, page, lens, new, budget, g, WEIGHT_KINDS[kind], pos0, Bt=Bt)
    want = after_eviction((k, v, w, p), table, lens, new, pos0, budget, window)
    work = torch.full((kd.branch_evict_workspace_bytes(len(lens), hkv, table.shape[1] * page, budget) + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    status = ints([64])
    L, m, first = ints(lens), ints(new), ints(pos0)
    kd.branch_evict(k, v, w, p, table, L, budget, Bt=Bt, n_new=m, pos0=first, window=window, workspace=work, status=status)
    same((k, v, w, p), want)
    assert bool((work[-512:] == 0xFF).all()) and status.tolist() == [64] and L.tolist() == lens and first.tolist() == pos0


def test_eviction_without_new_counts_and_positions():
    hkv, d, page, lens, budget = 2, 128, 16, [40, 64, 7], 50
    g = gen(71)
    k, v, w, p, table = evict_case(hkv, d, page, lens, [20] * 3, budget, g, spread, [0] * 3, positions="held")
    want = after_eviction((k, v, w, p), table, lens, [20] * 3, [0] * 3, budget, 0)
    kd.branch_evict(k, v, w, p, table, ints(lens), budget, Bt=20)
    same((k, v, w, p), want)


@pytest.mark.parametrize("L", [300, 3000, 9000, 20000])
def test_rows_that_are_alike_go_from_the_last_one(L):
    # weights and positions of a few kinds each: whole classes of rows of one rank, cut by the budget
    hkv, d, page = 2, 64, 8
    g = gen(75)
    k, v, w, p, table = evict_case(hkv, d, page, [L], [1], 0, g, WEIGHT_KINDS["ties"], [0])
    for budget in (L, L - 40, L // 3, 1):
        put_rows(p, table, 0, torch.randint(0, 2, (hkv, L), **g).to(torch.int32))
        if budget == 1:
            put_rows(w, table, 0, torch.zeros((hkv, L + 1), device="cuda"))
            put_rows(p, table, 0, torch.full((hkv, L), L, dtype=torch.int32, device="cuda"))
        want = after_eviction((k, v, w, p), table, [L], [1], [0], budget, 0)
        kd.branch_evict(k, v, w, p, table, ints([L]), budget)
        same((k, v, w, p), want)


@pytest.mark.parametrize("weight", [0.0, -0.0, 0.5, -3.0, float("inf"), float("-inf"), float("nan"), None])
@pytest.mark.parametrize("L", [900, 5000, 12000])
def test_rows_of_equal_weight_go_by_positions_of_the_whole_range(L, weight):
    # no weight, one weight, or two of them, and positions from one end of int32 to the other, its ends among them many times
    hkv, d, page = 2, 64, 16
    g = gen(77)
    k, v, w, p, table = evict_case(hkv, d, page, [L], [5], 0, g, spread, [0])
    for budget in (L + 5 - 2, L - 200, L // 2, 3):
        at = torch.randint(-2 ** 31, 2 ** 31, (hkv, L), **g)
        at = torch.where(torch.rand((hkv, L), **g) < 0.1, -2 ** 31, torch.where(torch.rand((hkv, L), **g) < 0.1, 2 ** 31 - 1, at))
        put_rows(p, table, 0, at.to(torch.int32))
        flat = torch.full((hkv, L + 5), weight, device="cuda") if weight is not None else (torch.rand((hkv, L + 5), **g) < 0.5).float() - 0.5
        put_rows(w, table, 0, flat)
        want = after_eviction((k, v, w, p), table, [L], [5], [0], budget, -(1 << 40))   # (no row is late)
        kd.branch_evict(k, v, w, p, table, ints([L]), budget, Bt=5)
        same((k, v, w, p), want)


def test_evicting_again_from_what_is_there_already():
    # rows behind the budget are still there: the same call once more, many times, while copies of rows take over
    hkv, d, page, L, Bt, budget = 2, 64, 16, 500, 200, 450
    g = gen(76)
    pools = evict_case(hkv, d, page, [L], [Bt], budget, g, spread, [0])
    k, v, w, p, table = pools
    for _ in range(12):
        want = after_eviction((k, v, w, p), table, [L], [Bt], [0], budget, 30)
        kd.branch_evict(k, v, w, p, table, ints([L]), budget, Bt=Bt, window=30)
        same((k, v, w, p), want)


def test_positions_that_make_no_sense_do_no_harm():
    # equal positions, and positions behind the last one (all rows look late): the lower row is kept, and nothing but the moves happens
    hkv, d, page, L, budget = 2, 64, 8, 300, 200
    for fill in (7, 2 ** 31 - 1, -2 ** 31):
        g = gen(72)
        k, v, w, p, table = evict_case(hkv, d, page, [L], [1], budget, g, WEIGHT_KINDS["ties"], [0])
        put_rows(p, table, 0, torch.full((hkv, L), fill, dtype=torch.int32, device="cuda"))
        want = after_eviction((k, v, w, p), table, [L], [1], [0], budget, 50)
        if fill == 2 ** 31 - 1:   # late rows are alike whatever they weigh
            ws, ps = rows_of(w, table, 0, L + 1), rows_of(p, table, 0, L + 1)
            assert bool((ps[:, :L] == fill).all()) and ws.shape[1] == L + 1
            k2, v2, w2, p2 = (x.clone() for x in (k, v, w, p))
            r = torch.arange(L, L + 1, device="cuda")
            p2[table[0, r // page].long(), :, r % page] = L
            flat = w2.clone()
            put_rows(flat, table, 0, torch.zeros((hkv, L + 1), device="cuda"))
            moved = after_eviction((k2, v2, flat, p2), table, [L], [1], [0], budget, 50)
            fro, to = evicted(np.zeros(L + 1), rows_of(p2, table, 0, L + 1)[0].cpu().numpy().astype(np.int64), L + 1 - 50, budget)
            fro, to = torch.from_numpy(fro).cuda(), torch.from_numpy(to).cuda()
            w2[table[0, to // page].long(), :, to % page] = w2[table[0, fro // page].long(), :, fro % page]
            want = moved[0], moved[1], w2, moved[3]
        kd.branch_evict(k, v, w, p, table, ints([L]), budget, window=50)
        same((k, v, w, p), want)


@pytest.mark.parametrize("L", [900, 20000])
@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 100, 2 ** 30])
def test_lengths_far_behind_the_table(L, length):
    # rows that no table can name: the sequence is left as it was, whether its length is within the budget or not
    hkv, d, page = 2, 64, 16
    g = gen(79)
    k, v, w, p, table = evict_case(hkv, d, page, [L], [5], 0, g, spread, [0])
    before = [x.clone() for x in (k, v, w, p)]
    for budget, bits in ((2 ** 31 - 1, kd.LEFT_OUT_ROW if length + 5 > 2 ** 31 - 1 else 0), (700, kd.LEFT_OUT_ROW)):
        status = ints([0])
        kd.branch_evict(k, v, w, p, table, ints([length]), budget, Bt=5, status=status)
        assert status.tolist() == [bits]
        same((k, v, w, p), before)
        gathered = w.clone()
        kd.branch_weights(torch.zeros((1, hkv, 5, d), dtype=torch.bfloat16, device="cuda"), k, gathered, table, ints([length]),
                          torch.full((1, hkv, 5), float("-inf"), device="cuda"))
        same((gathered,), (w,))
    q = torch.randn((1, 4, 90, d), **g).bfloat16()   # ... and it sees all rows of the table
    got, want = (kd.branch_chunk_attention(q, k, v, table, ints([x])) for x in (length, table.shape[1] * page))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool(torch.isfinite(want[1]).all())


def test_sequences_with_rows_on_absent_pages_are_left_out():
    hkv, d, page, budget = 2, 64, 8, 60
    lens = [100, 100, 100, 20]
    g = gen(73)
    k, v, w, p, table = evict_case(hkv, d, page, lens, [1] * 4, budget, g, spread, [0] * 4)
    holes = table.clone()
    holes[1, 3] = -1
    holes[3, 1] = 10 ** 6                     # (fewer rows than the budget: nothing is asked of its pages)
    want = after_eviction((k, v, w, p), table, lens, [1, 1, 1, 1], [0] * 4, budget, 0)
    before = tuple(x.clone() for x in (k, v, w, p))
    status = ints([0])
    kd.branch_evict(k, v, w, p, holes, ints(lens), budget, status=status)
    assert status.tolist() == [kd.LEFT_OUT_ROW]
    for got, after, old in zip((k, v, w, p), want, before):
        n = torch.arange(101, device="cuda")
        i = torch.int16 if got.dtype == torch.bfloat16 else torch.int32
        for s in (0, 2, 3):
            rows = n[:21] if s == 3 else n
            number = table[s, rows // page].long()
            keep = torch.ones_like(rows, dtype=torch.bool)
            assert torch.equal(got[number, :, rows % page].view(i)[keep], after[number, :, rows % page].view(i)[keep])
        number = table[1, n[:100] // page].long()
        assert torch.equal(got[number, :, n[:100] % page].view(i), old[number, :, n[:100] % page].view(i))
    # a length beyond the table
    status.zero_()
    kd.branch_evict(k, v, w, p, table[:, :5].contiguous(), ints([39, 40, 10, 10 ** 9]), 30, status=status)
    assert status.tolist() == [kd.LEFT_OUT_ROW]


def test_pools_past_32_bits():
    hkv, d, page, L, budget = 2, 128, 64, 200, 100
    pages = (1 << 31) // (hkv * d * page) + 40
    k, v = (torch.zeros((pages, hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w, p = torch.zeros((pages, hkv, page), device="cuda"), torch.zeros((pages, hkv, page), dtype=torch.int32, device="cuda")
    g = gen(74)
    table = torch.arange(pages - 4, pages, dtype=torch.int32, device="cuda")[None].contiguous()
    for x in (k, v):
        put_rows(x, table, 0, torch.randn((hkv, L + 1, d), **g).bfloat16())
    q = torch.randn((1, 4, 1, d), **g).bfloat16()
    _, lse = kd.branch_chunk_attention(q, k, v, table, ints([L]))
    kd.branch_weights(q, k, w, table, ints([L]), lse)
    want, bound = gathered(q[0], rows_of(k, table, 0, L + 1), lse[0], L, 1, 0, d ** -0.5)
    close(rows_of(w, table, 0, L + 1), want, bound, "weights")
    put_rows(p, table, 0, torch.arange(L, device="cuda", dtype=torch.int32).expand(hkv, L))
    near = [x[pages - 4:].clone() for x in (k, v, w, p)]
    want = after_eviction(near, torch.arange(4, dtype=torch.int32, device="cuda")[None], [L], [1], [0], budget, 0)
    kd.branch_evict(k, v, w, p, table, ints([L]), budget)
    same([x[pages - 4:].contiguous() for x in (k, v, w, p)], want)


# ------------------------------------------------------------------------------------------------ together
class Sequences:
    """Two layers of sequences with a budget, as a program keeps them."""

    def __init__(self, layers, n, hq, hkv, d, page, budget, Bt, window, g):
        self.hq, self.hkv, self.d, self.budget, self.window, self.page = hq, hkv, d, budget, window, page
        width = -(-(budget + Bt) // page)
        self.table = torch.randperm(n * width, generator=g["generator"], device="cuda").to(torch.int32).view(n, width)
        shape = (n * width, hkv, page)
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.k, self.v = ([torch.full(shape + (d,), float("nan"), **bf) for _ in range(layers)] for _ in range(2))
        self.w = [torch.full(shape, float("nan"), device="cuda") for _ in range(layers)]
        self.p = [torch.full(shape, -1, dtype=torch.int32, device="cuda") for _ in range(layers)]
        self.lens, self.pos0 = ints([0] * n), ints([0] * n)
        self.cos, self.sin = tables(4000, d)

    def step(self, xs, n_new, prefix=None, observe=0):
        """One step of all layers: xs[l] [n][heads][Bt][d], views of the layer's projection."""
        outs = []
        for l, x in enumerate(xs):
            q, k, v = x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]
            q = kd.branch_append(q, k, v, self.k[l], self.v[l], self.table, self.lens, n_new=n_new, pos0=self.pos0, cos=self.cos, sin=self.sin)
            out, lse = kd.branch_chunk_attention(q, self.k[l], self.v[l], self.table, self.lens, prefix=prefix, n_new=n_new)
            kd.branch_weights(q, self.k[l], self.w[l], self.table, self.lens, lse, n_new=n_new, observe=observe, decay=0.9)
            kd.branch_evict(self.k[l], self.v[l], self.w[l], self.p[l], self.table, self.lens, self.budget, Bt=x.shape[2], n_new=n_new, pos0=self.pos0,
                            window=self.window)
            outs.append(out)
        n = self.lens + n_new
        kept = n.clamp(max=self.budget)
        self.pos0 += n - kept
        self.lens.copy_(kept)
        return outs


@pytest.mark.parametrize("d,prompt", [(128, True), (64, False)])
def test_sequences_that_live_within_a_budget(d, prompt):
    # a long text in pieces, then token by token: what attention gives is that over the rows which the plain policy keeps
    n, hq, hkv, page, budget, window, layers, N = 3, 8, 2, 8, 100, 20, 2, 60
    g = gen(80 + d)
    seqs = Sequences(layers, n, hq, hkv, d, page, budget, 50, window, g)
    prefix = (torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16(), N) if prompt else None
    # what every (layer, sequence) has ever seen: rotated keys, values; and which tokens are held with which weight
    history = [[[torch.zeros((hkv, 0, d), dtype=torch.float64, device="cuda") for _ in range(2)] for _ in range(n)] for _ in range(layers)]
    held = [[[{} for _ in range(hkv)] for _ in range(n)] for _ in range(layers)]   # position -> weight, from the pages
    total = [0] * n
    for step, Bt in enumerate([50, 50, 33, 50, 1, 1, 1, 4, 1, 50]):
        new = [Bt, max(Bt - 7, 1) if Bt > 1 else 1, 0 if step == 2 else Bt]
        xs = [torch.randn((n, Bt, hq + 2 * hkv, d), **g).bfloat16().transpose(1, 2) for _ in range(layers)]
        first = seqs.lens.tolist()
        rotated = [kd.norm_rope(x[:, :hq], x[:, hq:hq + hkv], seqs.cos, seqs.sin,
                                positions=(ints(total)[:, None] + torch.arange(Bt, dtype=torch.int32, device="cuda")).contiguous()) for x in xs]
        outs = seqs.step(xs, ints(new), prefix=prefix)
        for l in range(layers):
            q, k = rotated[l]
            v = xs[l][:, hq + hkv:]
            for s in range(n):
                m = new[s]
                if not m:
                    continue
                K, V = (torch.cat([a, b[s, :, :m].double()], 1) for a, b in zip(history[l][s], (k, v)))
                history[l][s] = [K, V]
                for h in range(hkv):
                    kept = sorted(held[l][s][h])
                    at = torch.tensor(kept + list(range(total[s], total[s] + m)), device="cuda")
                    kk, vv = K[h, at], V[h, at]
                    if prompt:
                        kk, vv = torch.cat([prefix[0][0, h].double(), kk]), torch.cat([prefix[1][0, h].double(), vv])
                    x = q[s, h * hq // hkv:(h + 1) * hq // hkv, :m].double()
                    a = torch.matmul(x, kk.t()) * d ** -0.5
                    before = len(kk) - m
                    a.masked_fill_(torch.arange(len(kk), device="cuda")[None, None] > (before + torch.arange(m, device="cuda"))[None, :, None], float("-inf"))
                    p = torch.softmax(a, -1)
                    want = torch.matmul(p, vv)
                    got = outs[l][s, h * hq // hkv:(h + 1) * hq // hkv, :m].double()
                    # (16: the largest sum |q_i k_i| scale of such rows is below it, so e < 2^-11)
                    bound = (2.0 ** -8 + 2.0 ** -11) * torch.matmul(p, vv.abs()) + (2.0 ** -8 + 2.0 ** -11) * want.abs()
                    close(got, want, bound, f"step {step}, layer {l}, sequence {s}, head {h}")
                    # weights: what was held, forgotten by the decay, and this step's
                    weight = p.sum((0, 1))[len(kk) - len(at):]
                    weight[:len(kept)] += 0.9 * torch.tensor([held[l][s][h][t] for t in kept], dtype=torch.float64, device="cuda")
                    now = min(first[s] + m, budget)
                    r = torch.arange(now, device="cuda")
                    number = seqs.table[s, r // page].long()
                    ps, ws = seqs.p[l][number, h, r % page].tolist(), seqs.w[l][number, h, r % page].double().tolist()
                    assert len(set(ps)) == now and set(ps) <= set(at.tolist())
                    expect = dict(zip(at.tolist(), weight.tolist()))
                    for t, x_ in zip(ps, ws):
                        assert abs(x_ - expect[t]) <= 2.0 ** -10 * expect[t] + 1e-12, (step, t, x_, expect[t])
                    # the latest stay; of the others none that goes weighs more than one that stays (but for the error of weights)
                    late = total[s] + m - window
                    assert all(t in ps for t in at.tolist() if t >= late)
                    gone = [expect[t] for t in at.tolist() if t not in ps]
                    least = min([expect[t] for t in ps if t < late], default=float("inf"))
                    assert not gone or max(gone) <= least * (1 + 2.0 ** -9)
                    # the rows are those of the tokens
                    assert torch.equal(seqs.k[l][number, h, r % page].double(), K[h, torch.tensor(ps, device="cuda")])
                    assert torch.equal(seqs.v[l][number, h, r % page].double(), V[h, torch.tensor(ps, device="cuda")])
                    held[l][s][h] = dict(zip(ps, ws))
        for s in range(n):
            total[s] += new[s]
        assert (seqs.lens + seqs.pos0).tolist() == total


def test_captured_steps_within_a_budget():
    # a token's step in a graph, replayed while the sequences pass their budget, against eager steps on copies
    n, hq, hkv, d, page, budget, window, layers = 3, 8, 2, 128, 16, 70, 8, 2
    here, there = (Sequences(layers, n, hq, hkv, d, page, budget, 4, window, gen(90)) for _ in range(2))
    xs = [torch.zeros((n, 1, hq + 2 * hkv, d), dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(layers)]
    n_new = ints([1, 1, 1])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        here.step(xs, n_new)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = here.step(xs, n_new)
    for x in (here.lens, here.pos0):
        x.zero_()
    g = gen(91)
    for step in range(110):
        for x in xs:
            x.copy_(torch.randn(x.shape, **g).bfloat16())
        n_new.copy_(ints([1, step % 2, 1 if step != 80 else 0]))
        graph.replay()
        want = there.step(xs, n_new)
        if step % 9 == 0 or 65 < step < 75:
            torch.cuda.synchronize()
            assert torch.equal(here.lens, there.lens) and torch.equal(here.pos0, there.pos0)
            for l in range(layers):
                for s in range(n):
                    if int(n_new[s]):
                        assert torch.equal(outs[l][s], want[l][s]), step
                    rows = int(here.lens[s])
                    for a, b in ((here.k, there.k), (here.v, there.v), (here.w, there.w), (here.p, there.p)):
                        assert torch.equal(rows_of(a[l], here.table, s, rows), rows_of(b[l], there.table, s, rows)), step
