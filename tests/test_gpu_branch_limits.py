"""branch_append and branch_attention at the ends of what their documentation allows, against plain forms in 64 bits.  Tolerances: those of
test_gpu_branch.py, whose derivation does not depend on the sizes below."""
import pytest

import paper_2504_15364_amd as kd
from test_gpu_branch import CASES, attention_reference, close, gen, ints, paged, put_rows, rows_of, tables, wide  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ------------------------------------------------------------------------------------------------ the largest values
def rising(hkv, n, d, g):
    """n keys and values: the logits of the first two fifths are 0, the others' 15.9 (log2 units, with SCALE and queries (1, 0, ..)), a weight
    just below 2^16 of the first ones'.  Values of one sign, up to 2^100."""
    k = torch.zeros((hkv, n, d), dtype=torch.bfloat16, device="cuda")
    k[:, 2 * n // 5:, 0] = 1
    v = ((0.5 + 0.5 * torch.rand((hkv, n, d), **g)) * 2.0 ** 100).bfloat16().clamp_(max=2.0 ** 100)
    return k, v


SCALE = 15.9 / 1.4426950408889634


@pytest.mark.parametrize("prompts,fan,hq,hkv,d", [(1, 1, 32, 8, 128), (1, 16, 16, 8, 128), (1, 64, 16, 8, 64), (1, 100, 24, 8, 128), (40, 1, 8, 8, 64)])
def test_values_of_the_largest_size_over_long_prompts(prompts, fan, hq, hkv, d, wide):  # noqa: F811
    # one sign, so that sums grow with the rows: 8192 rows of weight 2^15.9 and value 2^100 would pass float's range.  (Where a prompt is cut
    # into pieces, each takes every so manieth tile: all of them meet the small logits first.)
    N, n = 32768, prompts * fan
    g = gen(7000 + n)
    k_pages, v_pages, table = paged([3] * n, 1, 16, hkv, d, g, wide=wide)
    own = torch.zeros((hkv, 4, d), dtype=torch.bfloat16, device="cuda"), rising(hkv, 4, d, g)[1]
    for s in range(n):
        put_rows(k_pages, table, s, own[0])
        put_rows(v_pages, table, s, own[1])
    prefix = [rising(hkv, N, d, g) for _ in range(prompts)]
    kp, vp = (torch.stack([x[i] for x in prefix]) for i in range(2))
    q = torch.zeros((n, hq, 1, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    out = kd.branch_attention(q, k_pages, v_pages, table, ints([3] * n), prefix=(kp, vp, N), softmax_scale=SCALE)
    for c in range(prompts):   # (the sequences of a prompt are alike)
        want, bound = attention_reference(q[c * fan], (kp[c].double(), vp[c].double()), N, (own[0].double(), own[1].double()), lambda j: 4, SCALE)
        for s in range(c * fan, (c + 1) * fan):
            close(out[s], want, bound, f"sequence {s}")


@pytest.mark.parametrize("n", [1, 600])
def test_values_of_the_largest_size_in_long_own_rows(n):
    # (600 sequences that read the same pages: a wave then sums thousands of rows by itself)
    hq, hkv, d, L = 8, 2, 64, 16383
    g = gen(7100 + n)
    k_pages, v_pages, table = paged([L], 1, 64, hkv, d, g)
    k, v = rising(hkv, L + 1, d, g)
    put_rows(k_pages, table, 0, k)
    put_rows(v_pages, table, 0, v)
    q = torch.zeros((n, hq, 1, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    out = kd.branch_attention(q, k_pages, v_pages, table.expand(n, -1).contiguous(), ints([L] * n), softmax_scale=SCALE)
    none = k[:, :0].double()
    want, bound = attention_reference(q[0], (none, none), 0, (k.double(), v.double()), lambda j: L + 1, SCALE)
    for s in range(n):
        close(out[s], want, bound, f"sequence {s}")


# ------------------------------------------------------------------------------------------------ a layer above that is broken
@pytest.mark.parametrize("fan,N", [(3, 100), (1, 9000), (64, 3000), (300, 700)])
def test_queries_that_are_nan_give_nan(fan, N, wide):  # noqa: F811
    # whatever the launches (zeros would hide it), and the other sequences' outputs stay what they are
    hq, hkv, d = 8, 2, 64
    g = gen(7200 + fan)
    lens = [(5 * i) % 40 for i in range(fan)]
    k_pages, v_pages, table = paged(lens, 1, 16, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + 1, d), **g).bfloat16())
    prefix = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16(), N
    q = torch.randn((fan, hq, 1, d), **g).bfloat16()
    want = kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=prefix)
    for bad in {0, fan // 2, fan - 1}:
        broken = q.clone()
        broken[bad, 2] = float("nan")                        # one head
        broken[bad, 5, 0, 7] = float("nan")                  # one value of another: every logit is NaN all the same
        out = kd.branch_attention(broken, k_pages, v_pages, table, ints(lens), prefix=prefix)
        assert bool(out[bad, [2, 5]].isnan().all())
        out[bad, [2, 5]] = want[bad, [2, 5]]
        assert torch.equal(out, want)


# ------------------------------------------------------------------------------------------------ where outputs may lie
@pytest.mark.parametrize("fan,N,Bt", [(3, 100, 1), (5, 60, 9), (40, 3000, 2), (1, 9000, 1)])
def test_outputs_in_the_place_of_the_queries_and_next_to_what_is_read(fan, N, Bt, wide):  # noqa: F811
    hq, hkv, d = 12, 2, 64
    g = gen(7300 + fan)
    lens = [(5 * i) % 40 for i in range(fan)]
    k_pages, v_pages, table = paged(lens, Bt, 16, hkv, d, g, wide=wide)
    for s, L in enumerate(lens):
        put_rows(k_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((hkv, L + Bt, d), **g).bfloat16())
    prefix = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16(), N
    both = torch.randn((3, fan, hq, Bt, d), **g).bfloat16()   # the queries, between two places for outputs
    q = both[1].clone()
    want = kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=prefix)
    for to in (0, 2, 1):
        out = kd.branch_attention(both[1], k_pages, v_pages, table, ints(lens), prefix=prefix, out=both[to])
        assert out.data_ptr() == both[to].data_ptr() and torch.equal(out, want)
    with pytest.raises(kd.KeyDiffError, match="overlap"):
        kd.branch_attention(both[0], k_pages, v_pages, table, ints(lens), prefix=prefix, out=both.view(-1)[d:d + q.numel()].view(q.shape))


def test_rows_behind_the_last_head_of_a_prefix_need_not_exist():
    # one head: the distance to the next one is never used, and a large one is no overlap
    import ctypes as C
    from paper_2504_15364_amd import binding
    hq, d, N, n = 4, 64, 300, 3
    g = gen(7350)
    k_pages, v_pages, table = paged([20] * n, 1, 16, 1, d, g)
    for s in range(n):
        put_rows(k_pages, table, s, torch.randn((1, 21, d), **g).bfloat16())
        put_rows(v_pages, table, s, torch.randn((1, 21, d), **g).bfloat16())
    kp, vp = torch.randn((1, 1, N, d), **g).bfloat16(), torch.randn((1, 1, N, d), **g).bfloat16()
    q, lens = torch.randn((n, hq, 1, d), **g).bfloat16(), ints([20] * n)
    want = kd.branch_attention(q, k_pages, v_pages, table, lens, prefix=(kp, vp, N))
    out, work = torch.zeros_like(q), torch.empty(kd.branch_workspace_bytes(n, hq, 1, d, 1, 1), dtype=torch.uint8, device="cuda")
    b = binding._Branches(k_pages=k_pages.data_ptr(), v_pages=v_pages.data_ptr(), table=table.data_ptr(), lens=lens.data_ptr(), n_seqs=n, n_q_heads=hq,
                          n_kv_heads=1, head_dim=d, page_rows=16, n_pages=k_pages.shape[0], table_width=table.shape[1])
    rc = binding.load_library().keydiff_branch_attention(C.byref(b), C.byref(binding._Rows(q.data_ptr(), hq * d, d, 0)), 1, kp.data_ptr(), vp.data_ptr(), 1, N,
                                                         1 << 40, 0.0, out.data_ptr(), work.data_ptr(), work.numel(),
                                                         torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(out, want)


# ------------------------------------------------------------------------------------------------ positions at the end of 64 bits
def test_blocks_whose_positions_do_not_fit_are_refused():
    hq, hkv, d, B = 4, 2, 64, 16
    g = gen(7400)
    caches = [kd.KeyDiffCache(kd.KeyDiffConfig(1, hq, hkv, d, 32, B)) for _ in range(2)]
    q, k, v = (torch.randn((1, h, B, d), **g).bfloat16() for h in (hq, hkv, hkv))
    table, w = torch.ones((100, d // 2), device="cuda"), torch.ones((d,), dtype=torch.bfloat16, device="cuda")
    for pos0 in (2 ** 63 - 1, 2 ** 63 - B, 2 ** 31 - B, -1, 85):
        calls = [lambda: caches[0].prefill_block_rope(q, k, v, pos0, table, table),
                 lambda: caches[0].prefill_block_norm_rope(q, k, v, pos0, table, table, w, w),
                 lambda: kd.prefill_block_layers(caches, [q, q], [k, k], [v, v], pos0, rope=(table, table)),
                 lambda: kd.prefill_block_layers(caches, [q, q], [k, k], [v, v], pos0, rope=(table, table), norm=([w, w], [w, w], 1e-6))]
        if pos0 != 85:   # (85: the block ends behind the tables)
            calls += [lambda: caches[0].prefill_block(q, k, v, pos0), lambda: kd.prefill_block_layers(caches, [q, q], [k, k], [v, v], pos0),
                      lambda: caches[0].prefill_block_norm_rope(q, k, v, pos0, None, None, w, w)]
        for call in calls:
            with pytest.raises(kd.KeyDiffError) as e:
                call()
            assert e.value.code == -2
    for c in caches:
        assert c.len == 0 and c.status() == 0
        c.close()


# ------------------------------------------------------------------------------------------------ tokens that are left out
@pytest.mark.parametrize("Bt", [1, 3, 70])
def test_status_tells_of_tokens_that_were_left_out(Bt):
    hq, hkv, d, page, n = 6, 2, 64, 16, 5
    g = gen(7500 + Bt)
    x = torch.randn((n, hq + 2 * hkv, Bt, d), **g).bfloat16()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    table = torch.ones((200, d // 2), device="cuda")
    status = ints([0])

    def positions(at):
        status.zero_()
        kd.norm_rope(q, k, table, table, positions=ints([[p + j for j in range(Bt)] for p in at]), status=status)
        return status.item()

    assert positions([0, 1, 2, 3, 200 - Bt]) == 0
    assert positions([0, 1, 201 - Bt, 3, 4]) == kd.LEFT_OUT_POSITION
    assert positions([-1, 1, 2, 3, 4]) == kd.LEFT_OUT_POSITION
    kd.norm_rope(q, k, table, table, status=status)
    assert status.item() == kd.LEFT_OUT_POSITION   # nothing is cleared

    k_pages, v_pages, pages = paged([100] * n, Bt, page, hkv, d, g)
    width = pages.shape[1]

    def append(lens, pos0=None, n_new=None, pages=pages, rope=True):
        status.zero_()
        kd.branch_append(q, k, v, k_pages, v_pages, pages, ints(lens), n_new=n_new, pos0=pos0, cos=table if rope else None,
                         sin=table if rope else None, status=status)
        return status.item()

    lens = [100, 0, 50, 7, 30]
    assert append(lens) == 0 and append(lens, rope=False) == 0
    assert append(lens, pos0=ints([0, 0, 0, 194 - Bt, 0])) == kd.LEFT_OUT_POSITION       # its last token at 200
    assert append(lens, pos0=ints([0, 0, 0, 193 - Bt, 0])) == 0
    assert append([100, 0, 50, -1, 30], pos0=ints([0, 0, 0, 10 ** 6, 0])) == 0                                # not in use
    assert append(lens, pos0=ints([0, 0, 0, 10 ** 6, 0]), n_new=ints([Bt, Bt, Bt, 0, Bt])) == 0               # takes none
    assert append([100, 0, width * page + 1 - Bt, 7, 30], rope=False) == kd.LEFT_OUT_ROW                       # behind the table's last row
    gone = pages.clone()
    gone[1, 0] = k_pages.shape[0]
    assert append(lens, pages=gone, rope=False) == kd.LEFT_OUT_ROW
    assert append(lens, pages=gone, pos0=ints([0, 0, 0, 10 ** 6, 0])) == kd.LEFT_OUT_ROW | kd.LEFT_OUT_POSITION


# ------------------------------------------------------------------------------------------------ pieces of many tokens
@pytest.mark.parametrize("hq,hkv,d,N,page,Bt,lens,n_new", [
    (8, 2, 128, 500, 16, 130, [0, 5, 700], [130, 7, 129]),
    (6, 2, 64, 0, 32, 300, [0, 31, 1000, 64], [300, 1, 33, 0]),
    (7, 1, 128, 3000, 64, 41, [90, 0], None),
])
def test_pieces_of_many_tokens(hq, hkv, d, N, page, Bt, lens, n_new):
    g = gen(7600 + Bt)
    n = len(lens)
    k_pages, v_pages, table = paged(lens, Bt, page, hkv, d, g)
    x = torch.randn((n, Bt, hq + 2 * hkv, d), **g).bfloat16().transpose(1, 2)
    for s, L in enumerate(lens):
        if L:
            put_rows(k_pages, table, s, torch.randn((hkv, L, d), **g).bfloat16())
            put_rows(v_pages, table, s, torch.randn((hkv, L, d), **g).bfloat16())
    taken = None if n_new is None else ints(n_new)
    kd.branch_append(None, x[:, hq:hq + hkv], x[:, hq + hkv:], k_pages, v_pages, table, ints(lens), n_new=taken)
    kp, vp = torch.randn((1, hkv, max(N, 1), d), **g).bfloat16(), torch.randn((1, hkv, max(N, 1), d), **g).bfloat16()
    out = torch.full((n, hq, Bt, d), 9.0, dtype=torch.bfloat16, device="cuda")
    kd.branch_attention(x[:, :hq], k_pages, v_pages, table, ints(lens), prefix=(kp, vp, N) if N else None, n_new=taken, out=out)
    for s, L in enumerate(lens):
        m = Bt if n_new is None else n_new[s]
        assert bool((out[s, :, m:] == 9).all())
        if m:
            own = rows_of(k_pages, table, s, L + m), rows_of(v_pages, table, s, L + m)
            want, bound = attention_reference(x[s, :hq, :m], (kp[0].double(), vp[0].double()), N, own, lambda j: L + j + 1, d ** -0.5)
            close(out[s, :, :m], want, bound, f"sequence {s}")


# ------------------------------------------------------------------------------------------------ workspaces and captured steps
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_nothing_is_written_behind_the_workspace(case, wide):  # noqa: F811
    hq, hkv, d, prompts, fan, N, page, Bt, lens, n_new = case
    n = max(prompts, 1) * fan
    g = gen(7700)
    k_pages, v_pages, table = paged(lens, Bt, page, hkv, d, g, wide=wide)
    k_pages.normal_(generator=g["generator"])
    v_pages.normal_(generator=g["generator"])
    prefix = torch.randn((max(prompts, 1), hkv, N, d), **g).bfloat16(), torch.randn((max(prompts, 1), hkv, N, d), **g).bfloat16(), N
    q = torch.randn((n, hq, Bt, d), **g).bfloat16()
    need = kd.branch_workspace_bytes(n, hq, hkv, d, Bt, prompts)
    work = torch.full((need + (1 << 22),), 0xAB, dtype=torch.uint8, device="cuda")
    kd.branch_attention(q, k_pages, v_pages, table, ints(lens), prefix=prefix if prompts else None, n_new=None if n_new is None else ints(n_new),
                        workspace=work[:need])
    assert bool((work[need:] == 0xAB).all())


def test_captured_steps_follow_rows_that_move_to_other_pages(wide):  # noqa: F811
    # between replays pages are exchanged for others, which the rows move to; the pages they leave hold NaN
    hq, hkv, d, N, page, n, Bt, steps = 8, 2, 64, 150, 16, 4, 2, 7
    g = gen(7800)
    k_pages, v_pages, table = paged([60] * n, Bt * steps, page, hkv, d, g, spare=3, wide=wide)
    first = [0, 13, 60, 31]
    for s, L in enumerate(first):
        if L:
            put_rows(k_pages, table, s, torch.randn((hkv, L, d), **g).bfloat16())
            put_rows(v_pages, table, s, torch.randn((hkv, L, d), **g).bfloat16())
    used = set(table[table >= 0].tolist())
    free = [p for p in range(k_pages.shape[0]) if p not in used]
    assert len(free) == 3
    kp, vp = torch.randn((1, hkv, N, d), **g).bfloat16(), torch.randn((1, hkv, N, d), **g).bfloat16()
    x = torch.randn((n, hq + 2 * hkv, Bt, d), **g).bfloat16()
    lens, taken, (cos, sin) = ints(first), ints([2, 2, 2, 2]), tables(400, d)
    pos0 = ints([200] * n)
    out = torch.full((n, hq, Bt, d), 3.0, dtype=torch.bfloat16, device="cuda")
    q_out = torch.full_like(out, 4.0)
    work = torch.empty(kd.branch_workspace_bytes(n, hq, hkv, d, Bt, 1), dtype=torch.uint8, device="cuda")

    def step(kpool, vpool, q_to, to, workspace):
        kd.branch_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], kpool, vpool, table, lens, n_new=taken, pos0=pos0, cos=cos, sin=sin, q_out=q_to)
        kd.branch_attention(q_to, kpool, vpool, table, lens, prefix=(kp, vp, N), n_new=taken, out=to, workspace=workspace)

    graphs, eager = (k_pages, v_pages, q_out, out), (k_pages.clone(), v_pages.clone(), q_out.clone(), out.clone())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(*graphs, work)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(steps):
        x.copy_(torch.randn(x.shape, **g).bfloat16())
        taken.copy_(ints([[2, 1, 0, 2], [1, 2, 2, 0]][i % 2]))
        graph.replay()
        torch.cuda.synchronize()
        step(*eager, None)
        for a, b, what in zip(graphs, eager, ("keys", "values", "queries", "outputs")):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), f"replay {i}: {what}"
        for s in range(n):   # ... which are those of the definition
            m, L = taken[s].item(), lens[s].item()
            if m:
                own = rows_of(k_pages, table, s, L + m), rows_of(v_pages, table, s, L + m)
                want, bound = attention_reference(q_out[s, :, :m], (kp[0].double(), vp[0].double()), N, own, lambda j: L + j + 1, d ** -0.5)
                close(out[s, :, :m], want, bound, f"replay {i}, sequence {s}")
        lens += taken
        s, c, to = i % n, (i // 2) % 3, free.pop(0)
        old = table[s, c].item()
        for pool in graphs[:2] + eager[:2]:
            pool[to] = pool[old]
            pool[old] = float("nan")
        table[s, c] = to
        free.append(old)
