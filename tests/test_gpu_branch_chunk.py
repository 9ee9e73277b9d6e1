"""branch_chunk_attention against a plain form in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, the half step of float; 2^-8 the half step of bf16, relative to the value):

  logits    128 products summed in float, at most 128 u = 2^-17 of sum |q_i k_i| scale = A, and one rounding of the scaled logit: a relative
            error of the weight of 2 * 2^-17 A; the exponential 2^-22; sums of n weights and values in float tile by tile, (n / 32 + 60) u: e in all
  outputs   the weights of the numerator are rounded to bf16, 2^-8 each, those of the denominator are not; a reference that moves scales sums by
            exponentials: within e.  |error| <= (e + 2^-8) sum p |v| + e |o|, and 2^-8 |o| of the output.  The roundings of the weights are
            independent of one another, so their sum is far below that where there are many keys: of all outputs of a sequence together,
            the squares of the errors add up to at most 2^-16 (sum o^2 + sum_i p_i^2 v_i^2) (three times the mean of such sums) and the squares of the e terms
  log sums  the error of a sum of weights relative to it is that of a weight, e; the logarithm 2^-22, two roundings of the reference's size
"""
import gc

import pytest

import paper_2504_15364_amd as kd
from test_gpu_branch import U8, close, gen, ints, paged, put_rows, rows_of, tables, wide  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def reference(q, prefix, own, before, scale, absent=None):
    """One sequence: q [hq][T][d]; prefix, own: (k, v) [hkv][rows][d] in double, `before` own rows held ahead of the tokens; absent: own rows that
    count as no keys.  Outputs and the bound of their error, logarithms and theirs, and sum p^2 v^2 with the squares of e's part."""
    hq, T, d = q.shape
    hkv, n = own[0].shape[:2]
    k, v = (torch.cat([a, b], 1) if a is not None else b for a, b in zip(prefix, own))
    N = k.shape[1] - n
    x = q.double().reshape(hkv, hq // hkv * T, d)
    a = torch.matmul(x, k.transpose(1, 2).contiguous()).view(hkv, hq // hkv, T, -1) * scale
    r = torch.arange(N + n, device="cuda") - N
    hidden = r[None] > before + torch.arange(T, device="cuda")[:, None]
    if absent is not None:
        hidden = hidden | ((r >= 0) & absent[r.clamp(min=0)])[None]
    a = a.masked_fill(hidden, float("-inf"))
    lse = torch.logsumexp(a, -1)
    p = torch.where(lse[..., None] == float("-inf"), 0.0, (a - lse[..., None]).exp()).view(hkv, -1, N + n)
    A = (torch.matmul(x.abs(), k.abs().transpose(1, 2).contiguous()).view(hkv, hq // hkv, T, -1) * scale).masked_fill(hidden, 0).amax(-1)
    e = (2.0 ** -16 * A + 2.0 ** -22 + ((N + n) / 32 + 60) * 2.0 ** -24).view(hkv, -1, 1)
    o, pv = torch.matmul(p, v), torch.matmul(p, v.abs())
    bound = (e + U8) * pv + (e + U8) * o.abs()
    squares = (U8 ** 2 * (o.square() + torch.matmul(p.square(), v.square()))).sum() + ((e * (pv + o.abs())).square()).sum()
    e_lse = e.view(hkv, hq // hkv, T) + 2.0 ** -21 + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0)
    return o.view(hq, T, d), bound.view(hq, T, d), lse.view(hq, T), e_lse.view(hq, T), squares


def check(out, lse, want, what):
    o, bound, log_sum, e_lse, squares = want
    close(out, o, bound, what)
    seen = log_sum > float("-inf")
    assert torch.equal(lse == float("-inf"), ~seen), what
    close(lse[seen], log_sum[seen], e_lse[seen], what + ", log sums")
    assert float((out.double() - o).square().sum()) <= float(squares) + 1e-30, what


CASES = [
    # hq, hkv, d, prompts, fan, N, page, Bt, lens, n_new
    (4, 1, 64, 0, 2, 0, 8, 1, [0, 200], None),                                  # few rows: a token alone
    (28, 4, 128, 1, 3, 257, 16, 4, [5, 0, 61], [4, 0, 3]),                      # 28 rows a sequence
    (4, 1, 64, 0, 1, 0, 8, 9, [0], None),                                       # 36 rows: the smallest piece that is none of few rows
    (4, 4, 128, 0, 2, 0, 8, 33, [0, 7], None),                                  # a KV head for every query head
    (32, 8, 128, 1, 1, 1, 16, 64, [0], None),                                   # one shared row; one block filled to the last row
    (32, 8, 128, 0, 1, 0, 64, 65, [63], None),                                  # ... and one more token
    (28, 4, 128, 2, 2, 63, 16, 100, [0, 1, 64, 129], [100, 37, 1, 99]),
    (6, 2, 128, 1, 5, 64, 32, 90, [3, 30, 64, -1, 100], [90, 0, 2, 90, 1000]),  # more than Bt counts as Bt; a sequence that is not in use
    (8, 2, 64, 1, 3, 65, 8, 200, [0, 500, 77], None),
    (8, 2, 64, 0, 3, 0, 1024, 333, [1020, 0, 5000], [333, 1, 332]),
    (64, 1, 64, 1, 2, 130, 8, 20, [40, 9], None),                               # 64 query heads to one KV head
    (24, 8, 128, 1, 24, 300, 32, 50, [29 * i % 700 for i in range(24)], [(31 * i + 50) % 51 for i in range(24)]),
    (20, 10, 64, 10, 6, 150, 16, 17, [i % 50 - 1 for i in range(60)], None),
    (8, 8, 128, 1, 1, 0, 16, 700, [0], None),                                   # a prompt of its own, a KV head for every query head
    (16, 2, 128, 1, 1, 5000, 64, 129, [9001], None),                            # long: cut into many parts
]


def problem(case, size, g, wide):
    hq, hkv, d, prompts, fan, N, page, Bt, lens, n_new = case
    n = max(prompts, 1) * fan
    new = [0 if L < 0 else (Bt if n_new is None else min(n_new[s], Bt)) for s, L in enumerate(lens)]
    k_pages, v_pages, table = paged(lens, Bt, page, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        if new[s]:   # rows behind the new ones stay NaN
            put_rows(k_pages, table, s, torch.randn((hkv, L + new[s], d), **g).mul_(size).bfloat16())
            put_rows(v_pages, table, s, torch.randn((hkv, L + new[s], d), **g).bfloat16())
    prefix = None
    if prompts:
        kp, vp = torch.randn((prompts, hkv, N + 3, d), **g).mul_(size).bfloat16(), torch.randn((prompts, hkv, N + 3, d), **g).bfloat16()
        kp[:, :, N:] = float("nan")
        vp[:, :, N:] = float("nan")
        prefix = kp, vp, N
    q = torch.randn((n, Bt, hq, d), **g).mul_(size).bfloat16().transpose(1, 2)
    for s in range(n):
        q[s, :, new[s]:] = float("nan")                         # of tokens that are none nothing is read into the others
    return new, k_pages, v_pages, table, prefix, q


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("values", ["plain", "peaked"])
def test_chunk_attention(case, values, wide):  # noqa: F811
    hq, hkv, d, prompts, fan, N, page, Bt, lens, n_new = case
    n = len(lens)
    g = gen(2000 + hq * N + page + Bt)
    new, k_pages, v_pages, table, prefix, q = problem(case, 1.0 if values == "plain" else 6.0, g, wide)
    out = torch.full((n, hq, Bt, d), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, hq, Bt), 7.0, device="cuda")
    # (a workspace that holds NaN everywhere: nothing in it is read before it is written)
    work = torch.full((kd.branch_chunk_workspace_bytes(n, hq, hkv, d, Bt, prompts) + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    kw = dict(prefix=prefix, n_new=None if n_new is None else ints(n_new))
    got = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), out=out, lse=lse, workspace=work, **kw)
    assert got[0] is out and got[1] is lse
    assert bool((work[-512:] == 0xFF).all())
    again, lse2 = torch.full_like(out, 9.0), torch.full_like(lse, 7.0)
    kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), out=again, lse=lse2, **kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    for s, L in enumerate(lens):
        m = new[s]
        assert bool((out[s, :, m:] == 9).all()) and bool((lse[s, :, m:] == 7).all()), f"rows of sequence {s} that are not its own were written"
        if m:
            shared = (prefix[0][s // fan, :, :N].double(), prefix[1][s // fan, :, :N].double()) if prompts else (None, None)
            own = rows_of(k_pages, table, s, L + m), rows_of(v_pages, table, s, L + m)
            check(out[s, :, :m], lse[s, :, :m], reference(q[s, :, :m], shared, own, L, d ** -0.5), f"sequence {s}")


@pytest.mark.parametrize("hq,hkv,d,Bt,page", [(4, 1, 64, 50, 8), (8, 2, 128, 70, 16), (8, 2, 128, 5, 16)])
def test_chunk_attention_absent_pages(hq, hkv, d, Bt, page, wide):  # noqa: F811
    # pages that do not exist in the middle, at the start (the first tokens see no key at all) and behind the table's end
    g = gen(17 + d + Bt)
    lens = [0, 300, 150, 0]
    k_pages, v_pages, table = paged(lens, Bt, page, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    copies = [(rows_of(k_pages, table, s, L + Bt), rows_of(v_pages, table, s, L + Bt)) for s, L in enumerate(lens)]
    gone = {0: [0], 1: [3, 4, 9], 2: list(range((150 + Bt + page - 1) // page)), 3: [(Bt - 1) // page]}
    absent = []
    for s, L in enumerate(lens):
        r = torch.arange(L + Bt, device="cuda")
        absent.append(torch.isin(r // page, torch.tensor(gone[s], device="cuda")))
        for i in gone[s]:
            number = int(table[s, i])
            k_pages[number] = float("nan")
            v_pages[number] = float("nan")
            table[s, i] = [-1, 10 ** 6, len(k_pages)][i % 3]
    q = torch.randn((4, hq, Bt, d), **g).bfloat16()
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), softmax_scale=0.3)
    for s, L in enumerate(lens):
        check(out[s], lse[s], reference(q[s], (None, None), copies[s], L, 0.3, absent[s]), f"sequence {s}")
    assert bool((out[2] == 0).all()) and bool((lse[2] == float("-inf")).all())
    # rows that lie outside the table count as absent as well: lengths beyond it
    short = table[:, :6].contiguous()
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, short, ints([6 * page - 20, 10 ** 9, -1, 6 * page]), softmax_scale=0.3)
    for s, before in ((0, 6 * page - 20), (1, 6 * page), (3, 6 * page)):
        rows = min(6 * page, copies[s][0].shape[1])
        if rows < 6 * page:
            continue
        own = copies[s][0][:, :rows], copies[s][1][:, :rows]
        check(out[s], lse[s], reference(q[s], (None, None), own, before, 0.3, absent[s][:rows]), f"sequence {s} beyond its table")


def test_chunk_attention_of_queries_in_a_projections_output_and_in_place(wide):  # noqa: F811
    hq, hkv, d, Bt, N = 12, 4, 128, 75, 200
    g = gen(31)
    lens = [10, 0, 129]
    fused = torch.randn((3, Bt, hq + 2 * hkv, d), **g).bfloat16().transpose(1, 2)
    k_pages, v_pages, table = paged(lens, Bt, 16, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    prefix = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16(), N
    q = fused[:, :hq]
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), prefix=prefix)
    same = q.contiguous()
    got, lse2 = kd.branch_chunk_attention(same, k_pages, v_pages, table, ints(lens), prefix=prefix, out=same)
    assert got is same and torch.equal(same, out) and torch.equal(lse, lse2)
    # one head and one token after the other, strides of all kinds
    padded = torch.zeros((3, hq + 1, Bt + 2, d + 8), dtype=torch.bfloat16, device="cuda")
    padded[:, :hq, :Bt, :d] = q
    got, _ = kd.branch_chunk_attention(padded[:, :hq, :Bt, :d], k_pages, v_pages, table, ints(lens), prefix=prefix)
    assert torch.equal(got, out)


@pytest.mark.parametrize("power", [-115, -90, 90])
@pytest.mark.parametrize("Bt", [6, 80])
def test_chunk_attention_values_of_extreme_size(power, Bt, wide):  # noqa: F811
    hq, hkv, d, N = 8, 2, 128, 700
    g = gen(300 + power + Bt)
    lens = [0, 33, 500]
    k_pages, v_pages, table = paged(lens, Bt, 16, hkv, d, g, wide=wide)
    size = 2.0 ** (power + torch.randint(-10, 10, (hkv, 1, 1), **g).float())
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
        put_rows(v_pages, table, s, (torch.randn((hkv, L + Bt, d), **g) * size).bfloat16())
    kp, vp = torch.randn((1, hkv, N, d), **g).bfloat16(), (torch.randn((1, hkv, N, d), **g) * size).bfloat16()[:1]
    q = torch.randn((3, hq, Bt, d), **g).bfloat16()
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), prefix=(kp, vp.contiguous(), N))
    for s, L in enumerate(lens):
        own = rows_of(k_pages, table, s, L + Bt), rows_of(v_pages, table, s, L + Bt)
        o, bound, log_sum, e_lse, _ = reference(q[s], (kp[0].double(), vp[0].double()), own, L, d ** -0.5)
        # (near the smallest normal number, 2^-126, sums of such values lose at most it for each key, and an output that lies below it)
        close(out[s], o, bound + (2.0 ** -126 * (N + L + Bt) if power == -115 else 0.0), f"sequence {s}")
        close(lse[s], log_sum, e_lse, f"sequence {s}, log sums")
    # no values at all
    out, _ = kd.branch_chunk_attention(q, k_pages, torch.zeros_like(v_pages), table, ints(lens), prefix=(kp, torch.zeros_like(kp), N))
    assert bool((out == 0).all())


def test_chunk_attention_logits_that_rise_and_fall(wide):  # noqa: F811
    # the reference of a row moves in every tile, or never again behind the first: keys that grow along the sequence, and that shrink
    hq, hkv, d, Bt, L = 4, 1, 128, 70, 900
    g = gen(41)
    for rising in (True, False):
        k_pages, v_pages, table = paged([L], Bt, 32, hkv, d, g, wide=wide)
        q = torch.randn((1, hq, Bt, d), **g).bfloat16()
        along = torch.linspace(0, 1, L + Bt, device="cuda")[None, :, None]
        k = torch.randn((hkv, L + Bt, d), **g) * 0.2 + 10.0 * (along if rising else 1 - along) * torch.sign(q[0, 0, 0].float())
        put_rows(k_pages, table, 0, k.bfloat16())
        put_rows(v_pages, table, 0, torch.randn((hkv, L + Bt, d), **g).bfloat16())
        out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints([L]))
        own = rows_of(k_pages, table, 0, L + Bt), rows_of(v_pages, table, 0, L + Bt)
        check(out[0], lse[0], reference(q[0], (None, None), own, L, d ** -0.5), f"rising {rising}")


def test_chunk_attention_queries_that_are_nan_give_nan(wide):  # noqa: F811
    hq, hkv, d, Bt = 4, 2, 128, 40
    g = gen(43)
    k_pages, v_pages, table = paged([100], Bt, 16, hkv, d, g, wide=wide)
    for pool in (k_pages, v_pages):
        put_rows(pool, table, 0, torch.randn((hkv, 100 + Bt, d), **g).bfloat16())
    q = torch.randn((1, hq, Bt, d), **g).bfloat16()
    q[0, 1, 7, 3] = float("nan")
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints([100]))
    bad = torch.zeros((hq, Bt), dtype=torch.bool, device="cuda")
    bad[1, 7] = True
    assert torch.equal(torch.isnan(out[0]).all(-1), bad) and torch.equal(torch.isnan(out[0]).any(-1), bad) and torch.equal(torch.isnan(lse[0]), bad)


def test_few_rows_are_what_branch_attention_gives(wide):  # noqa: F811
    hq, hkv, d, Bt, N = 32, 8, 128, 3, 700
    g = gen(44)
    lens = [(97 * i) % 400 for i in range(6)]
    k_pages, v_pages, table = paged(lens, Bt, 16, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    prefix = torch.randn((2, hkv, N, d), **g).bfloat16(), torch.randn((2, hkv, N, d), **g).bfloat16(), N
    q = torch.randn((6, hq, Bt, d), **g).bfloat16()
    out, _ = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), prefix=prefix)
    assert torch.equal(out, kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=prefix))


def test_pools_past_32_bits():
    # 2^31 elements and more ahead of the rows that are read
    hkv, d, page, Bt = 2, 128, 64, 40
    pages = (1 << 31) // (hkv * d * page) + 40
    k_pages, v_pages = (torch.zeros((pages, hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = gen(45)
    table = torch.arange(pages - 4, pages, dtype=torch.int32, device="cuda")[None].contiguous()
    for pool in (k_pages, v_pages):
        put_rows(pool, table, 0, torch.randn((hkv, 150 + Bt, d), **g).bfloat16())
    q = torch.randn((1, 4, Bt, d), **g).bfloat16()
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints([150]))
    own = rows_of(k_pages, table, 0, 150 + Bt), rows_of(v_pages, table, 0, 150 + Bt)
    check(out[0], lse[0], reference(q[0], (None, None), own, 150, d ** -0.5), "")
    del k_pages, v_pages
    gc.collect()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("layout", [kd.LAYOUT_FILL, kd.LAYOUT_ORDERED])
def test_pieces_behind_prompts_held_by_keydiff_caches(layout, wide):  # noqa: F811
    # prompts through block steps (their last eviction pending), then a piece of each of two continuations
    hq, hkv, d, N, B, prompts, Bt = 8, 2, 128, 160, 64, 2, 30
    g = gen(46)
    cache = kd.KeyDiffCache(kd.KeyDiffConfig(prompts, hq, hkv, d, N, B, layout=layout, softmax_scale=0.11))
    for t in range(0, 320, B):
        block = [torch.randn((prompts, h, B, d), **g).bfloat16() for h in (hq, hkv, hkv)]
        cache.prefill_block_deferred(*block, t)
    lens = [0, 5, 64, 200]
    k_pages, v_pages, table = paged(lens, Bt, 16, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        for pool in (k_pages, v_pages):
            put_rows(pool, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    q = torch.randn((4, hq, Bt, d), **g).bfloat16()
    out, lse = kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), prefix=cache)
    assert cache.len == N
    for s, L in enumerate(lens):
        shared = cache.key_rows()[s // 2, :, :N].double(), cache.value_rows()[s // 2, :, :N].double()
        own = rows_of(k_pages, table, s, L + Bt), rows_of(v_pages, table, s, L + Bt)
        check(out[s], lse[s], reference(q[s], shared, own, L, float(torch.tensor(0.11))), f"sequence {s}")
    with pytest.raises(ValueError):
        kd.branch_chunk_attention(q, k_pages, v_pages, table, ints(lens), prefix=cache, softmax_scale=0.2)
    assert cache.status() == 0
    cache.close()


def test_captured_pieces_follow_what_they_find(wide):  # noqa: F811
    hq, hkv, d, Bt, N = 8, 2, 128, 48, 100
    g = gen(47)
    most = [400, 300, 200]
    k_pages, v_pages, table = paged(most, Bt, 16, hkv, d, g, wide=wide)
    for s, L in enumerate(most):
        for pool in (k_pages, v_pages):
            put_rows(pool, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    prefix = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16(), N
    q = torch.randn((3, hq, Bt, d), **g).bfloat16()
    lens, n_new = ints([0, 0, 0]), ints([Bt] * 3)
    out, lse = torch.zeros((3, hq, Bt, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, hq, Bt), device="cuda")
    call = lambda: kd.branch_chunk_attention(q, k_pages, v_pages, table, lens, prefix=prefix, n_new=n_new, out=out, lse=lse)  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for now, taken in (([0, 0, 0], [48, 48, 48]), ([400, 1, 77], [48, 3, 0]), ([10, -1, 200], [48, 48, 20]), ([400, 300, 200], [1, 48, 48])):
        lens.copy_(ints(now))
        n_new.copy_(ints(taken))
        out.fill_(9)
        lse.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = torch.full_like(out, 9), torch.full_like(lse, 7)
        kd.branch_chunk_attention(q, k_pages, v_pages, table, lens, prefix=prefix, n_new=n_new, out=want, lse=want_lse)
        assert torch.equal(out, want) and torch.equal(lse, want_lse), now


def test_pieces_on_two_streams_at_once():
    hq, hkv, d, Bt = 16, 4, 128, 200
    g = gen(48)
    lens = [700, 0, 333]
    k_pages, v_pages, table = paged(lens, Bt, 32, hkv, d, g, wide=1 << 14)
    for s, L in enumerate(lens):
        for pool in (k_pages, v_pages):
            put_rows(pool, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    qs = [torch.randn((3, hq, Bt, d), **g).bfloat16() for _ in range(2)]
    L = ints(lens)
    want = [kd.branch_chunk_attention(q, k_pages, v_pages, table, L) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i in range(2):
            got[i].append(kd.branch_chunk_attention(qs[i], k_pages, v_pages, table, L, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
