"""norm_rope, branch_append, branch_attention and the block steps that norm, against plain forms in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, the half step of float; 2^-8 the half step of bf16, relative to the value):

  norm and rotation  the sum of squares of 128 values in float, square root, division, two products, one product and one sum of the
                     rotation: at most 24 roundings on the way of a term (a lane adds 32 numbers, three more steps join the lanes;
                     of a sum of squares half the relative error reaches the root), 2^-19 of the terms' magnitude with a factor of
                     two to spare, then one rounding to bf16
  attention          logits: 128 products summed in float, at most 128 u = 2^-17 of sum |q_i k_i| scale = A, and one rounding of the
                     scaled logit: a relative error of the weight of 2 * 2^-17 A; the exponential 2^-22, the weight as two
                     bf16 numbers 2^-16, sums of n weights and values in float tile by tile (n / 32 + 60) u: e in all, on the
                     weights of numerator and denominator: |error| <= e (sum p |v| + |o|) + 2^-8 |o|
"""
import gc
import math

import pytest

import paper_2504_15364_amd as kd

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U8 = 2.0 ** -8 * 1.001


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(generator=g, device="cuda")


def tables(rows, d):
    inv = 500000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    ang = torch.arange(rows, dtype=torch.float64)[:, None] * inv[None]
    return ang.cos().float().cuda(), ang.sin().float().cuda()


def formed(x, w, cos, sin, positions, eps):
    """Norm and rotation of x [b][h][T][d] in double, positions [b][T]; and the bound of the error."""
    x = x.double()
    d = x.shape[-1]
    if w is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * (w.double() if w.dim() == 1 else w.double()[None, :, None])
    if cos is None:
        return x, U8 * x.abs() + 2.0 ** -19 * x.abs()
    p = positions.long()
    c, s = cos.double()[p][:, None], sin.double()[p][:, None]
    a, b = x[..., :d // 2], x[..., d // 2:]
    y = torch.cat([a * c - b * s, b * c + a * s], -1)
    size = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
    return y, U8 * y.abs() + 2.0 ** -19 * size + 1e-38


def close(got, want, bound, what=""):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} values off, worst {float((off - bound)[bad].max()):.3g} over its bound"


# ------------------------------------------------------------------------------------------------ norms and rotation
@pytest.mark.parametrize("b,hq,hkv,T,d", [(1, 4, 1, 1, 64), (1, 28, 4, 1, 128), (3, 6, 2, 33, 128), (2, 8, 2, 257, 64), (1, 32, 8, 1000, 128),
                                         (5, 1, 1, 7, 64)])
@pytest.mark.parametrize("norm,rope", [("shared", True), ("heads", True), ("none", True), ("heads", False)])
def test_norm_rope(b, hq, hkv, T, d, norm, rope):
    g = gen(hq * T + d)
    fused = torch.randn((b, T, hq + 2 * hkv, d), **g).mul_(3.0).bfloat16().transpose(1, 2)   # views into one projection's output
    q, k = fused[:, :hq], fused[:, hq:hq + hkv]
    cos, sin = tables(2000, d) if rope else (None, None)
    wq = wk = None
    if norm != "none":
        wq = torch.randn((d,) if norm == "shared" else (hq, d), **g).bfloat16()
        wk = torch.randn((d,) if norm == "shared" else (hkv, d), **g).bfloat16()
    pos0 = 911
    positions = torch.randint(0, 2000, (b, T), **g).to(torch.int32)
    for at in (None, positions):
        qo, ko = kd.norm_rope(q, k, cos, sin, pos0=pos0, positions=at, q_weight=wq, k_weight=wk, norm_eps=1e-5)
        p = at if at is not None else (pos0 + torch.arange(T, device="cuda"))[None].expand(b, T)
        for got, x, w in ((qo, q, wq), (ko, k, wk)):
            assert got.is_contiguous() and got.shape == x.shape
            close(got, *formed(x, w, cos, sin, p, 1e-5))


def test_norm_rope_small_rows_and_zero_rows():
    # rows far below sqrt(eps) and rows of zeros: eps keeps the root from zero
    d = 128
    x = torch.zeros((1, 2, 3, d), dtype=torch.bfloat16, device="cuda")
    x[0, 0, 1] = 1e-6
    x[0, 1, 2, 5] = 3e38
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    qo, ko = kd.norm_rope(x, x[:, :1], q_weight=w, k_weight=w, norm_eps=1e-6)
    assert float(qo[0, 0, 0].abs().max()) == 0 and float(ko[0, 0, 0].abs().max()) == 0
    want, bound = formed(x[:, :1], w, None, None, None, 1e-6)
    close(ko, want, bound)
    assert abs(float(qo[0, 0, 1, 0]) - 1e-6 / math.sqrt(1e-6 + 1e-12)) < 1e-5


def test_norm_rope_leaves_tokens_outside_the_tables():
    d = 64
    g = gen(3)
    q, k = torch.randn((2, 4, 5, d), **g).bfloat16(), torch.randn((2, 2, 5, d), **g).bfloat16()
    cos, sin = tables(10, d)
    positions = torch.tensor([[0, 9, 10, -1, 3], [2 ** 31 - 1, -2 ** 31, 1, 2, 9]], dtype=torch.int32, device="cuda")
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    kd.norm_rope(q, k, cos, sin, positions=positions, q_out=qo, k_out=ko)
    inside = (positions >= 0) & (positions < 10)
    assert bool((qo.transpose(1, 2)[~inside] == 7).all()) and bool((ko.transpose(1, 2)[~inside] == 7).all())
    want, bound = formed(q, None, cos, sin, positions.clamp(0, 9), 0)
    sel = inside[:, None, :, None].expand_as(q)
    close(qo[sel], want[sel], bound[sel])


def test_norm_rope_without_norm_is_the_rotation_of_the_block_step():
    # the same products and sums as the rotation ahead of prefill_block_rope, each rounded on its own
    d = 128
    g = gen(4)
    q, k = torch.randn((1, 6, 40, d), **g).bfloat16(), torch.randn((1, 2, 40, d), **g).bfloat16()
    cos, sin = tables(500, d)
    qo, ko = kd.norm_rope(q, k, cos, sin, pos0=77)
    c, s = cos[77:117], sin[77:117]
    for x, got in ((q, qo), (k, ko)):
        a, b = x.float()[..., :d // 2], x.float()[..., d // 2:]
        assert torch.equal(got, torch.cat([a * c - b * s, b * c + a * s], -1).bfloat16())


@pytest.mark.parametrize("layout", [kd.LAYOUT_FILL, kd.LAYOUT_ORDERED])
@pytest.mark.parametrize("layers", [1, 3])
def test_block_steps_that_norm_are_steps_on_what_norm_rope_gives(layout, layers):
    hq, hkv, d, N, B, T = 6, 2, 128, 96, 32, 200
    g = gen(5 + layers)
    cos, sin = tables(T, d)
    cfg = kd.KeyDiffConfig(1, hq, hkv, d, N, B, layout=layout)
    here, there = [kd.KeyDiffCache(cfg) for _ in range(layers)], [kd.KeyDiffCache(cfg) for _ in range(layers)]
    x = torch.randn((layers, 1, T, hq + 2 * hkv, d), **g).bfloat16().transpose(2, 3)
    wq = [torch.randn((hq, d), **g).bfloat16() if l % 2 else torch.randn((d,), **g).bfloat16() for l in range(layers)]
    wk = [torch.randn((hkv, d), **g).bfloat16() if l % 2 else torch.randn((d,), **g).bfloat16() for l in range(layers)]
    for t in range(0, T, B):
        parts = [tuple(y[:, a:b, t:t + B].contiguous() for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))) for y in x]
        formed_ = [kd.norm_rope(q, k, cos, sin, pos0=t, q_weight=wq[l], k_weight=wk[l]) for l, (q, k, _) in enumerate(parts)]
        if layers == 1:
            q, k, v = parts[0]
            got = [here[0].prefill_block_norm_rope(q, k, v, t, cos, sin, wq[0], wk[0])]
            want = [there[0].prefill_block(*formed_[0], v, t)]
        else:
            got = kd.prefill_block_layers(here, [p[0] for p in parts], [p[1] for p in parts], [p[2] for p in parts], t, rope=(cos, sin),
                                          norm=(wq, wk, 1e-6))
            want = kd.prefill_block_layers(there, [f[0] for f in formed_], [f[1] for f in formed_], [p[2] for p in parts], t)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    for a, b in zip(here, there):
        assert a.len == b.len and torch.equal(a.positions(), b.positions())
        assert torch.equal(a.key_rows()[:, :, :a.len], b.key_rows()[:, :, :b.len])
        assert a.status() == 0
        a.close()
        b.close()


def test_block_step_with_norm_alone_and_its_refusals():
    d, T = 64, 16
    g = gen(9)
    cache = kd.KeyDiffCache(kd.KeyDiffConfig(2, 4, 1, d, 32, 16))
    q, k, v = (torch.randn((2, h, T, d), **g).bfloat16() for h in (4, 1, 1))
    w = torch.randn((d,), **g).bfloat16()
    cos, sin = tables(20, d)
    for kw in (dict(cos=None, sin=None, q_weight=None, k_weight=None), dict(cos=cos, sin=sin, q_weight=w, k_weight=w)):
        with pytest.raises(kd.KeyDiffError):
            cache.prefill_block_norm_rope(q, k, v, 10, **kw)   # nothing to do; a block that ends behind the tables
    assert cache.len == 0
    cache.prefill_block_norm_rope(q, k, v, 10, None, None, w, w)
    want, bound = formed(k, w, None, None, None, 1e-6)
    close(cache.key_rows()[:, :, :T], want, bound)
    cache.close()


# ------------------------------------------------------------------------------------------------ continuations
@pytest.fixture(params=[0, 1 << 16], ids=["narrow", "wide"])
def wide(request):
    """Rows that tables could name beyond those that lengths ask for.  A call whose tables name few rows of few sequences is one launch;
    one whose tables could name this many is two."""
    return request.param


def paged(lens, extra, page, hkv, d, g, spare=4, wide=0):
    """Pools whose every row is NaN, a table of shuffled pages for lens[i] + extra rows each."""
    need = [max(0, -(-(max(n, 0) + extra) // page)) for n in lens]
    width, total = max(max(need), 1) + wide // page, sum(need) + spare
    pool = torch.full((total, hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    order = torch.randperm(total, generator=g["generator"], device="cuda").cpu()
    table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return pool, pool.clone(), table.cuda()


def rows_of(pool, table, s, n):
    """The first n own rows of sequence s: [hkv][n][d] in double."""
    r = torch.arange(n, device="cuda")
    page = pool.shape[2]
    return pool[table[s, r // page].long(), :, r % page].transpose(0, 1).double()


def put_rows(pool, table, s, x):
    r = torch.arange(x.shape[1], device="cuda")
    page = pool.shape[2]
    pool[table[s, r // page].long(), :, r % page] = x.transpose(0, 1)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("hq,hkv,d,page,Bt,lens,n_new", [
    (4, 1, 64, 8, 1, [0], None),
    (28, 4, 128, 16, 1, [15, 16, 0, 31, 700], None),
    (6, 2, 128, 32, 5, [3, 30, 64, -1, 100], [5, 0, 2, 5, 9]),     # more than Bt counts as Bt
    (8, 2, 64, 1024, 37, [1020, 0, 5000], [37, 1, 36]),
])
def test_branch_append(hq, hkv, d, page, Bt, lens, n_new):
    g = gen(hq + page)
    n = len(lens)
    k_pages, v_pages, table = paged(lens, Bt, page, hkv, d, g)
    x = torch.randn((n, Bt, hq + 2 * hkv, d), **g).bfloat16().transpose(1, 2)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    wq, wk = torch.randn((d,), **g).bfloat16(), torch.randn((hkv, d), **g).bfloat16()
    cos, sin = tables(9000, d)
    pos0 = ints([100 + 7 * i for i in range(n)])
    q_out = torch.full((n, hq, Bt, d), 5.0, dtype=torch.bfloat16, device="cuda")
    before_k, before_v = k_pages.clone(), v_pages.clone()
    L = ints(lens)
    kd.branch_append(q, k, v, k_pages, v_pages, table, L, n_new=None if n_new is None else ints(n_new), pos0=pos0, cos=cos, sin=sin,
                     q_weight=wq, k_weight=wk, q_out=q_out)
    assert L.tolist() == lens
    for s in range(n):
        m = 0 if lens[s] < 0 else min(Bt, n_new[s] if n_new else Bt)
        assert bool((q_out[s, :, m:] == 5).all())
        if m == 0:
            continue
        at = (100 + 7 * s + lens[s] + torch.arange(m, device="cuda"))[None]
        close(q_out[s:s + 1, :, :m], *formed(q[s:s + 1, :, :m], wq, cos, sin, at, 1e-6), "queries")
        r = lens[s] + torch.arange(m, device="cuda")
        number = table[s, r // page].long()
        want, bound = formed(k[s:s + 1, :, :m], wk, cos, sin, at, 1e-6)
        close(k_pages[number, :, r % page].transpose(0, 1), want[0], bound[0], "keys")
        assert torch.equal(v_pages[number, :, r % page].transpose(0, 1), v[s, :, :m])
        before_k[number, :, r % page] = k_pages[number, :, r % page]
        before_v[number, :, r % page] = v_pages[number, :, r % page]
    # nothing else was touched
    assert torch.equal(before_k.view(torch.int16), k_pages.view(torch.int16))
    assert torch.equal(before_v.view(torch.int16), v_pages.view(torch.int16))


def test_branch_append_without_queries_or_form_and_outside_the_table():
    hkv, d, page = 2, 64, 8
    g = gen(12)
    k_pages, v_pages, table = paged([0, 0, 0], 16, page, hkv, d, g)
    table[1, 0] = 10 ** 6                     # no such page
    table[1, 1] = -5
    k, v = torch.randn((3, hkv, 10, d), **g).bfloat16(), torch.randn((3, hkv, 10, d), **g).bfloat16()
    lens = ints([0, 0, 13])                   # the last sequence's rows 16 .. lie outside its table
    before = k_pages.clone()
    assert kd.branch_append(None, k, v, k_pages, v_pages, table, lens) is None
    assert torch.equal(rows_of(k_pages, table, 0, 10), k[0].double()) and torch.equal(rows_of(v_pages, table, 0, 10), v[0].double())
    r = 13 + torch.arange(3, device="cuda")
    number = table[2, r // page].long()
    assert torch.equal(k_pages[number, :, r % page].transpose(0, 1), k[2, :, :3])
    for s, first, m in ((0, 0, 10), (2, 13, 3)):
        r = first + torch.arange(m, device="cuda")
        before[table[s, r // page].long(), :, r % page] = k[s, :, :m].transpose(0, 1)
    assert torch.equal(before.view(torch.int16), k_pages.view(torch.int16))


def attention_reference(q, prefix, rows, own, j_of, scale):
    """One sequence: q [hq][Bt][d]; prefix (k, v) [hkv][N][d] double, own (k, v) [hkv][n][d]; row j sees own rows [0, j_of(j)).
    Returns the outputs and the bound of their error."""
    hq, Bt, d = q.shape
    hkv = own[0].shape[0]
    out, bound = torch.zeros((hq, Bt, d), dtype=torch.float64, device="cuda"), torch.zeros((hq, Bt, d), dtype=torch.float64, device="cuda")
    for j in range(Bt):
        k = torch.cat([prefix[0][:, :rows], own[0][:, :j_of(j)]], 1)
        v = torch.cat([prefix[1][:, :rows], own[1][:, :j_of(j)]], 1)
        if k.shape[1] == 0:
            continue
        x = q[:, j].double().view(hkv, hq // hkv, d)
        a = torch.bmm(x, k.transpose(1, 2).contiguous()) * scale
        p = torch.softmax(a, -1)
        o = torch.bmm(p, v)
        A = torch.bmm(x.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) * scale
        e = 2.0 ** -16 * A + 2.0 ** -22 + 2.0 ** -16 + (k.shape[1] / 32 + 60) * 2.0 ** -24
        out[:, j] = o.view(hq, d)
        bound[:, j] = ((torch.bmm(p, v.abs()) + o.abs()) * e + U8 * o.abs()).view(hq, d)
    return out, bound


CASES = [
    # hq, hkv, d, prompts, fan, N, page, Bt, lens, n_new
    (4, 1, 64, 1, 1, 1, 8, 1, [0], None),                                       # one shared key and the token's own
    (4, 1, 64, 0, 2, 0, 8, 1, [0, 200], None),                                  # no prompt: the token alone; 201 own rows
    (8, 2, 128, 1, 1, 31, 16, 1, [31], None),
    (8, 2, 128, 1, 3, 33, 16, 1, [32, 0, 33], None),
    (28, 4, 128, 2, 4, 257, 16, 3, [5, 0, 61, 30, 31, 32, 33, 100], [3, 3, 0, 1, 2, 3, 3, 3]),   # 7 query heads: 21 rows a sequence
    (32, 8, 128, 1, 21, 700, 64, 1, [0, 1, 63, 64, 65, 500, -1, 3, 700, 90, 128, 127, 32, 31, 96, 20, 17, -7, 40, 2, 1000], None),
    (6, 2, 128, 3, 2, 100, 32, 14, [7, 0, 18, 100, 64, 3], [14, 5, 14, 14, 1, 14]),   # 42 rows a sequence
    (64, 1, 64, 1, 2, 130, 8, 1, [40, 9], None),                                # 64 query heads to one KV head
    (16, 16, 64, 2, 1, 65, 1024, 2, [0, 1500], None),                           # a KV head for every query head
    (24, 8, 128, 1, 90, 300, 16, 1, [i % 40 for i in range(90)], None),
    # 64, 240, 256 and 500 rows of one KV head over a prompt: two to eight waves share its tiles, in one block or two
    (8, 2, 128, 1, 16, 1500, 16, 1, [3 * i for i in range(16)], None),
    (6, 2, 128, 2, 80, 1000, 16, 1, [i % 7 for i in range(160)], None),
    (8, 2, 64, 1, 64, 97, 32, 1, [i for i in range(64)], None),
    (8, 2, 64, 1, 125, 777, 8, 1, [i % 50 - 1 for i in range(125)], None),
    (8, 2, 64, 1, 16, 3000, 8, 1, [1] * 16, None),
    (16, 4, 128, 1, 30, 2049, 8, 1, [1] * 30, None),
    # more segments of shared rows than workgroups: whole ones in turn, or halves
    (16, 8, 64, 40, 1, 700, 16, 1, [i % 33 for i in range(40)], None),
    (20, 10, 64, 30, 20, 150, 16, 1, [i % 5 - 1 for i in range(600)], None),
    (8, 8, 128, 65, 1, 2500, 8, 1, [0] * 65, None),
    (16, 2, 128, 1, 40, 500, 16, 9, [i % 21 for i in range(40)], [i % 10 for i in range(40)]),   # 72 rows a sequence, 2880 of a prompt
    # blocks of 128 and 256 shared rows, filled in part
    (64, 16, 128, 4, 31, 1021, 16, 1, [i % 35 for i in range(124)], None),
    (80, 20, 64, 10, 30, 1021, 16, 1, [i % 35 for i in range(300)], None),
    (64, 16, 128, 4, 120, 515, 16, 1, [i % 9 - 1 for i in range(480)], None),
    (64, 16, 64, 4, 120, 515, 16, 1, [i % 9 - 1 for i in range(480)], None),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("values", ["plain", "peaked"])
def test_branch_attention(case, values, wide):
    hq, hkv, d, prompts, fan, N, page, Bt, lens, n_new = case
    n = max(prompts, 1) * fan
    g = gen(1000 + hq * N + page)
    k_pages, v_pages, table = paged(lens, Bt, page, hkv, d, g, wide=wide)
    size = 1.0 if values == "plain" else 6.0                    # peaked: logits up to hundreds, one key takes nearly all
    for s, L in enumerate(lens):
        if L >= 0:   # rows behind the new ones stay NaN
            m = L + (Bt if n_new is None else n_new[s])
            put_rows(k_pages, table, s, torch.randn((hkv, m, d), **g).mul_(size).bfloat16())
            put_rows(v_pages, table, s, torch.randn((hkv, m, d), **g).bfloat16())
    kp, vp = torch.randn((max(prompts, 1), hkv, N + 3, d), **g).mul_(size).bfloat16(), torch.randn((max(prompts, 1), hkv, N + 3, d), **g).bfloat16()
    kp[:, :, N:] = float("nan")                                 # rows of the buffer behind the prompt's
    vp[:, :, N:] = float("nan")
    q = torch.randn((n, Bt, hq, d), **g).mul_(size).bfloat16().transpose(1, 2)
    out = torch.full((n, hq, Bt, d), 9.0, dtype=torch.bfloat16, device="cuda")
    # (a workspace that holds NaN everywhere: nothing in it is read before it is written)
    need = kd.branch_workspace_bytes(n, hq, hkv, d, Bt, prompts)
    work = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=(kp, vp, N) if prompts else None,
                        n_new=None if n_new is None else ints(n_new), out=out, workspace=work)
    again = torch.full_like(out, 9.0)
    kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=(kp, vp, N) if prompts else None,
                        n_new=None if n_new is None else ints(n_new), out=again)
    assert torch.equal(out, again)
    for s, L in enumerate(lens):
        m = 0 if L < 0 else (Bt if n_new is None else n_new[s])
        assert bool((out[s, :, m:] == 9).all()), f"rows of sequence {s} that are not its own were written"
        if m:
            own = rows_of(k_pages, table, s, L + m), rows_of(v_pages, table, s, L + m)
            want, bound = attention_reference(q[s, :, :m], (kp[s // fan].double(), vp[s // fan].double()), N, own, lambda j: L + j + 1,
                                              d ** -0.5)
            close(out[s, :, :m], want, bound, f"sequence {s}")


def test_branch_attention_long_prompts_and_long_own_rows():
    hq, hkv, d, N = 8, 2, 128, 20011
    g = gen(77)
    lens = [9000, 40, 1]
    k_pages, v_pages, table = paged(lens, 1, 64, hkv, d, g)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
    kp, vp = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16()
    q = torch.randn((3, hq, 1, d), **g).bfloat16()
    out = kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=(kp, vp, N), softmax_scale=0.25)
    for s, L in enumerate(lens):
        own = rows_of(k_pages, table, s, L + 1), rows_of(v_pages, table, s, L + 1)
        want, bound = attention_reference(q[s], (kp[0].double(), vp[0].double()), N, own, lambda j: L + 1, 0.25)
        close(out[s], want, bound, f"sequence {s}")


def test_branch_attention_dominant_keys_at_the_ends_of_pieces(wide):
    # one key of a row holds nearly all the weight, wherever it lies; all other keys far below
    hq, hkv, d, N, L = 4, 1, 64, 300, 90
    g = gen(78)
    for at in (0, 31, 32, 255, 256, 299, 300, 331, 390):
        k_pages, v_pages, table = paged([L], 1, 16, hkv, d, g, wide=wide)
        k, v = torch.randn((hkv, N + L + 1, d), **g).bfloat16(), torch.randn((hkv, N + L + 1, d), **g).bfloat16()
        q = torch.randn((1, hq, 1, d), **g).bfloat16()
        k[0, at] = (60.0 * q[0, 1, 0].float() / q[0, 1, 0].float().norm()).bfloat16()
        put_rows(k_pages, table, 0, k[:, N:])
        put_rows(v_pages, table, 0, v[:, N:])
        out = kd.branch_attention(q, k_pages, v_pages, table, ints([L]), prefix=(k[None, :, :N].contiguous(), v[None, :, :N].contiguous(), N))
        own = k[:, N:].double(), v[:, N:].double()
        want, bound = attention_reference(q[0], (k.double(), v.double()), N, own, lambda j: L + 1, d ** -0.5)
        close(out[0], want, bound, f"key {at}")


@pytest.mark.parametrize("fan", [3, 16, 40, 64])
@pytest.mark.parametrize("power", [-90, 90])
def test_branch_attention_values_of_extreme_size(fan, power, wide):
    # heads whose values differ by 2^30 from one another, all far from one
    hq, hkv, d, N = 8, 2, 128, 700
    g = gen(300 + fan + power)
    lens = [(7 * i) % 60 for i in range(fan)]
    k_pages, v_pages, table = paged(lens, 1, 16, hkv, d, g, wide=wide)
    size = 2.0 ** (power + torch.randint(-15, 16, (hkv, 1, 1), **g).float())

    def values(n):
        return (torch.randn((hkv, n, d), **g) * size).bfloat16()

    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
        put_rows(v_pages, table, s, values(L + 1))
    kp, vp = torch.randn((1, hkv, N, d), **g).bfloat16(), values(N)[None]
    q = torch.randn((fan, hq, 1, d), **g).bfloat16()
    out = kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=(kp, vp.contiguous(), N))
    for s, L in enumerate(lens):
        own = rows_of(k_pages, table, s, L + 1), rows_of(v_pages, table, s, L + 1)
        want, bound = attention_reference(q[s], (kp[0].double(), vp[0].double()), N, own, lambda j: L + 1, d ** -0.5)
        close(out[s], want, bound, f"sequence {s}")


def test_branch_attention_absent_pages(wide):
    # a page outside the pool: its keys are absent; a query without any key gets zeros
    hq, hkv, d, page = 8, 2, 128, 8
    g = gen(79)
    k_pages, v_pages, table = paged([60, 5, 70], 2, page, hkv, d, g, wide=wide)
    for s, L in enumerate((60, 5, 70)):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 2, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + 2, d), **g).bfloat16())
    k_pages[0], v_pages[0] = float("nan"), float("nan")
    q = torch.randn((3, hq, 2, d), **g).bfloat16()
    table2 = table.clone()
    table2[0, 2], table2[0, 5], table2[1] = -1, k_pages.shape[0], 2 ** 31 - 1
    table2[2, 0] = table2[0, 2]
    lens = ints([60, 5, 1 << 29])    # the last sequence claims more rows than its table has: those are absent as well
    out = kd.branch_attention(q, k_pages, v_pages, table2, lens, prefix=None)
    assert bool((out[1] == 0).all())
    seen = torch.tensor([r for r in range(62) if r // page not in (2, 5)], device="cuda")
    table_ok = table.clone()
    own = rows_of(k_pages, table_ok, 0, 62)[:, seen], rows_of(v_pages, table_ok, 0, 62)[:, seen]
    none = (own[0][:, :0], own[1][:, :0])
    want, bound = attention_reference(q[0], none, 0, own, lambda j: len(seen) - 1 + j, d ** -0.5)
    close(out[0], want, bound)
    rows = 72   # (a wide table's other columns name no pages)
    own = rows_of(k_pages, table_ok, 2, rows)[:, page:], rows_of(v_pages, table_ok, 2, rows)[:, page:]
    want, bound = attention_reference(q[2], none, 0, own, lambda j: rows - page, d ** -0.5)
    close(out[2], want, bound)


def test_branch_attention_shared_own_pages_and_pools_past_32_bits():
    # sequences that read the same pages, at the far end of pools of 5 GB each
    hq, hkv, d, page = 4, 2, 128, 64
    g = gen(80)
    pages = (5 << 30) // (hkv * page * d * 2)
    k_pages = torch.empty((pages, hkv, page, d), dtype=torch.bfloat16, device="cuda")
    v_pages = torch.empty_like(k_pages)
    table = ints([[pages - 1, pages - 3], [pages - 1, 0]])
    lens = ints([100, 50])
    for p in (0, pages - 1, pages - 3):
        k_pages[p], v_pages[p] = torch.randn((hkv, page, d), **g).bfloat16(), torch.randn((hkv, page, d), **g).bfloat16()
    x = torch.randn((2, hq + 2 * hkv, 1, d), **g).bfloat16()
    q = kd.branch_append(x[:1, :hq], x[:1, hq:hq + hkv], x[:1, hq + hkv:], k_pages, v_pages, table[:1], lens[:1])
    assert torch.equal(q, x[:1, :hq])
    assert torch.equal(k_pages[pages - 3, :, 36], x[0, hq:hq + hkv, 0]) and torch.equal(v_pages[pages - 3, :, 36], x[0, hq + hkv:, 0])
    out = kd.branch_attention(x[:, :hq], k_pages, v_pages, table, lens)
    for s, L in enumerate((100, 50)):
        own = rows_of(k_pages, table, s, L + 1), rows_of(v_pages, table, s, L + 1)
        want, bound = attention_reference(x[s, :hq], (own[0][:, :0], own[1][:, :0]), 0, own, lambda j: L + 1, d ** -0.5)
        close(out[s], want, bound, f"sequence {s}")


def continue_prompt(layout, wide, steps=5, fan=3, prompts=2, layers=2, page=8):
    """A run as a program makes it: prompts through blocks that norm and rotate, then `fan` continuations of each, token by token;
    yields (out, reference, bound) of every layer and step."""
    hq, hkv, d, N, B, T = 8, 2, 64, 64, 32, 110
    g = gen(200 + layout)
    n = prompts * fan
    cos, sin = tables(T + steps + 8, d)
    caches = [kd.KeyDiffCache(kd.KeyDiffConfig(prompts, hq, hkv, d, N, B, layout=layout)) for _ in range(layers)]
    wq = [torch.randn((d,), **g).bfloat16() for _ in range(layers)]
    wk = [torch.randn((hkv, d), **g).bfloat16() for _ in range(layers)]
    for t in range(0, T, B):
        Bt = min(B, T - t)
        x = [[torch.randn((prompts, h, Bt, d), **g).bfloat16() for h in (hq, hkv, hkv)] for _ in range(layers)]
        for l, c in enumerate(caches):   # layer by layer, evictions pending from layer to layer
            q, k = kd.norm_rope(x[l][0], x[l][1], cos, sin, pos0=t, q_weight=wq[l], k_weight=wk[l])
            c.prefill_block_deferred(q, k, x[l][2], t, carry=caches[l - 1])
    pools = [paged([0] * n, steps + 2, page, hkv, d, g, wide=wide) for _ in range(layers)]
    table, lens, pos0 = pools[0][2], torch.zeros(n, dtype=torch.int32, device="cuda"), ints([T] * n)
    for k, v, _ in pools:
        assert k.shape == pools[0][0].shape
    for step in range(steps):
        for l in range(layers):
            k_pages, v_pages, _ = pools[l]
            x = torch.randn((n, 1, hq + 2 * hkv, d), **g).bfloat16().transpose(1, 2)
            q = kd.branch_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], k_pages, v_pages, table, lens, pos0=pos0, cos=cos, sin=sin,
                                 q_weight=wq[l], k_weight=wk[l])
            out = kd.branch_attention(q, k_pages, v_pages, table, lens, prefix=caches[l])
            yield step, l, q, out, caches[l], k_pages, v_pages, table, x, wq[l], cos, sin, T
        lens += 1
    for c in caches:
        assert c.status() == 0
        c.close()


@pytest.mark.parametrize("layout", [kd.LAYOUT_FILL, kd.LAYOUT_ORDERED])
def test_continuations_of_prompts_held_by_keydiff_caches(layout, wide):
    seen = 0
    for step, l, q, out, cache, k_pages, v_pages, table, x, wq, cos, sin, T in continue_prompt(layout, wide):
        n, hq = q.shape[:2]
        assert cache.len == cache.cfg.budget_N
        want, bound = formed(x[:, :hq], wq, cos, sin, torch.full((n, 1), T + step, device="cuda"), 1e-6)
        close(q, want, bound, "queries")
        kc, vc = cache.key_rows()[:, :, :cache.len].double(), cache.value_rows()[:, :, :cache.len].double()
        for s in range(n):
            own = rows_of(k_pages, table, s, step + 1), rows_of(v_pages, table, s, step + 1)
            want, bound = attention_reference(q[s], (kc[s // 3], vc[s // 3]), cache.len, own, lambda j: step + 1, q.shape[-1] ** -0.5)
            close(out[s], want, bound, f"step {step}, layer {l}, sequence {s}")
        seen += 1
    assert seen == 10


def test_branch_attention_over_an_empty_cache_and_a_cache_of_other_heads(wide):
    hq, hkv, d = 4, 2, 64
    g = gen(81)
    cache = kd.KeyDiffCache(kd.KeyDiffConfig(1, hq, hkv, d, 64, 16, softmax_scale=0.5))
    k_pages, v_pages, table = paged([10, 0], 1, 8, hkv, d, g, wide=wide)
    for s, L in enumerate((10, 0)):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
    q = torch.randn((2, hq, 1, d), **g).bfloat16()
    out = kd.branch_attention(q, k_pages, v_pages, table, ints([10, 0]), prefix=cache)
    for s, L in enumerate((10, 0)):
        own = rows_of(k_pages, table, s, L + 1), rows_of(v_pages, table, s, L + 1)
        want, bound = attention_reference(q[s], (own[0][:, :0], own[1][:, :0]), 0, own, lambda j: L + 1, 0.5)
        close(out[s], want, bound)
    with pytest.raises(ValueError):
        kd.branch_attention(q, k_pages, v_pages, table, ints([10, 0]), prefix=cache, softmax_scale=0.3)
    other = torch.randn((2, 8, 1, d), **g).bfloat16()
    with pytest.raises(kd.KeyDiffError) as e:
        kd.branch_attention(other, k_pages, v_pages, table, ints([10, 0]), prefix=cache)
    assert e.value.code == -2
    with pytest.raises(ValueError, match="workspace"):
        kd.branch_attention(q, k_pages, v_pages, table, ints([10, 0]), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    cache.close()
    with pytest.raises(kd.KeyDiffError) as e:
        kd.branch_attention(q, k_pages, v_pages, table, ints([10, 0]), prefix=cache)
    assert e.value.code == -1


@pytest.mark.parametrize("given", [True, False])
def test_captured_steps_follow_the_lengths_they_find(given, wide):
    # append and attention captured once, replayed with lengths, tables and inputs that change, against eager calls
    hq, hkv, d, N, page, n, steps = 8, 2, 128, 200, 16, 5, 6
    g = gen(82)
    k_pages, v_pages, table = paged([90] * n, steps + 1, page, hkv, d, g, wide=wide)
    first = [0, 3, 40, -1, 90]
    for s, L in enumerate(first):
        if L > 0:
            put_rows(k_pages, table, s, torch.randn((hkv, L, d), **g).bfloat16())
            put_rows(v_pages, table, s, torch.randn((hkv, L, d), **g).bfloat16())
    kp, vp = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16()
    x = torch.randn((n, hq + 2 * hkv, 1, d), **g).bfloat16()
    lens, cos_sin = ints(first), tables(400, d)
    pos0 = ints([250] * n)
    out = torch.full((n, hq, 1, d), 3.0, dtype=torch.bfloat16, device="cuda")
    q_out = torch.zeros_like(out)
    work = torch.empty(kd.branch_workspace_bytes(n, hq, hkv, d, 1, 1), dtype=torch.uint8, device="cuda")

    def step(kpool, vpool, q_to, to, workspace):
        kd.branch_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], kpool, vpool, table, lens, pos0=pos0, cos=cos_sin[0], sin=cos_sin[1],
                         q_out=q_to)
        kd.branch_attention(q_to, kpool, vpool, table, lens, prefix=(kp, vp, N), out=to, workspace=workspace)

    # (the eager run's own pools and outputs)
    k2, v2, out2, q2 = k_pages.clone(), v_pages.clone(), out.clone(), q_out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(k_pages, v_pages, q_out, out, work if given else None)   # (None: from the graph's own pool)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(steps):
        x.copy_(torch.randn(x.shape, **g).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        step(k2, v2, q2, out2, None)
        assert torch.equal(out, out2) and torch.equal(k_pages.view(torch.int16), k2.view(torch.int16)), f"replay {i}"
        lens += (lens >= 0).to(torch.int32)
        if i == 2:
            lens[3], lens[4] = 0, -1     # a slot is given to another sequence, one is freed
        table.copy_(table)
    assert bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("layout", [kd.LAYOUT_FILL, kd.LAYOUT_ORDERED])
def test_a_captured_call_takes_no_pending_eviction_along(layout):
    hq, hkv, d, N, B = 8, 2, 64, 64, 32
    g = gen(84)
    cache = kd.KeyDiffCache(kd.KeyDiffConfig(1, hq, hkv, d, N, B, layout=layout))
    for t in range(0, 4 * B, B):
        cache.prefill_block_deferred(*(torch.randn((1, h, B, d), **g).bfloat16() for h in (hq, hkv, hkv)), t)
    k_pages, v_pages, table = paged([5, 0, 9], 1, 8, hkv, d, g)
    for s, L in enumerate((5, 0, 9)):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
    q, lens = torch.randn((3, hq, 1, d), **g).bfloat16(), ints([5, 0, 9])
    out = torch.zeros_like(q)
    work = torch.empty(kd.branch_workspace_bytes(3, hq, hkv, d, 1, 1), dtype=torch.uint8, device="cuda")

    def capture():
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        error = None
        with torch.cuda.graph(graph):
            out.mul_(0)
            try:
                kd.branch_attention(q, k_pages, v_pages, table, lens, prefix=cache, out=out, workspace=work)
            except kd.KeyDiffError as e:
                error = e
        return graph, error

    assert capture()[1].code == -3          # (the step of the last block has left its eviction pending)
    cache.finish()
    graph, error = capture()
    assert error is None
    want = kd.branch_attention(q, k_pages, v_pages, table, lens, prefix=cache)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert cache.status() == 0 and cache.len == N
    cache.close()


def test_calls_on_two_streams_with_workspaces_of_their_own():
    hq, hkv, d, N = 16, 4, 128, 3000
    g = gen(83)
    lens = [500, 60, 0, 20]
    k_pages, v_pages, table = paged(lens, 1, 32, hkv, d, g)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
    kp, vp = torch.randn((2, hkv, N, d), **g).bfloat16(), torch.randn((2, hkv, N, d), **g).bfloat16()
    qs = [torch.randn((4, hq, 1, d), **g).bfloat16() for _ in range(2)]
    L = ints(lens)
    want = [kd.branch_attention(q, k_pages, v_pages, table, L, prefix=(kp, vp, N)) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(w) for w in want]
    for _ in range(20):
        for q, s, o in zip(qs, streams, outs):   # one stream as torch's object, one as a bare handle
            kd.branch_attention(q, k_pages, v_pages, table, L, prefix=(kp, vp, N), out=o, stream=s if s is streams[0] else s.cuda_stream)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
            o.zero_()
        torch.cuda.synchronize()
    # outputs allocated by the calls belong to their stream as well
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [kd.branch_attention(q, k_pages, v_pages, table, L, prefix=(kp, vp, N), stream=s) for q, s in zip(qs, streams)]
    a = kd.norm_rope(qs[0], qs[0][:, :hkv], *tables(50, d), pos0=3, stream=streams[1].cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(got, want))
    assert all(torch.equal(x, y) for x, y in zip(a, kd.norm_rope(qs[0], qs[0][:, :hkv], *tables(50, d), pos0=3)))
    b = kd.norm_rope(qs[0], qs[0][:, :hkv], *tables(50, d), pos0=3, stream=0)   # the default stream's handle
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_return_what_is_given_and_hold_no_memory():
    g = gen(31)
    q, kv = torch.randn(3, 8, 1, 64, **g).bfloat16(), torch.randn(2, 3, 2, 1, 64, **g).bfloat16()
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    pools = torch.zeros(2, 4, 2, 16, 64, device="cuda", dtype=torch.bfloat16)
    table, lens = torch.arange(3, device="cuda", dtype=torch.int32)[:, None].contiguous(), ints([0, 3, 15])
    outs = [torch.empty_like(q), torch.empty_like(kv[0])]
    work = torch.empty(kd.branch_workspace_bytes(3, 8, 2, 64, 1, 0), device="cuda", dtype=torch.uint8)
    a, b = kd.norm_rope(q, kv[0], q_weight=w, k_weight=w, q_out=outs[0], k_out=outs[1])
    assert a is outs[0] and b is outs[1]
    assert kd.branch_append(q, kv[0], kv[1], *pools, table, lens, q_weight=w, k_weight=w, q_out=outs[0]) is outs[0]
    assert kd.branch_append(None, kv[0], kv[1], *pools, table, lens) is None
    assert kd.branch_attention(q, *pools, table, lens, out=outs[0], workspace=work) is outs[0]
    gc.collect()   # (what tests before this one left in cycles)
    held = torch.cuda.memory_allocated()
    for _ in range(20):
        x, _ = kd.norm_rope(q, kv[0], q_weight=w, k_weight=w)
        x = kd.branch_append(x, kv[0], kv[1], *pools, table, lens)
        x = kd.branch_attention(x, *pools, table, lens)
        with pytest.raises(kd.KeyDiffError):
            kd.branch_append(x, kv[0], kv[1], pools[0], pools[0], table, lens)   # the pools overlap
        with pytest.raises(ValueError, match="workspace"):
            kd.branch_attention(x, *pools, table, lens, workspace=work[:8])
    del x, _
    gc.collect()
    assert torch.cuda.memory_allocated() == held
