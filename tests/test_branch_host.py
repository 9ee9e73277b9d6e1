"""norm_rope, branch_append and branch_attention: what they refuse, found before anything is enqueued (no GPU needed)."""
import ctypes as C
import sys

import pytest

from paper_2504_15364_amd import binding as kd

torch = pytest.importorskip("torch")
P = 4096   # stands for an aligned device pointer: every call below is refused before it would be used


def rows(data=P, seq=64 * 1024, head=1024, token=128):
    return kd._Rows(data, seq, head, token)


def form(**kw):
    f = dict(q_weight=P, k_weight=P, q_weight_stride=0, k_weight_stride=0, norm_eps=1e-6, cos_table=P, sin_table=P, table_rows=100)
    f.update(kw)
    return kd._RowForm(**f)


def branches(**kw):
    b = dict(k_pages=P, v_pages=P + (1 << 30), table=P, lens=P, n_new=None, n_seqs=4, n_q_heads=8, n_kv_heads=2, head_dim=128,
             page_rows=16, n_pages=10, table_width=4)
    b.update(kw)
    return kd._Branches(**b)


def norm_rope(q=rows(), k=rows(), batch=1, hq=8, hkv=2, d=128, Bt=4, pos0=0, positions=None, f=None, q_out=1 << 32, k_out=1 << 33):
    f = form() if f is None else f
    return kd.load_library().keydiff_norm_rope(C.byref(q), C.byref(k), batch, hq, hkv, d, Bt, pos0, positions, C.byref(f), q_out, k_out, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=rows(None)), kd.EINVAL),
    (dict(k=rows(P + 2)), kd.EINVAL),                       # not 16-byte aligned
    (dict(q=rows(token=100)), kd.ESHAPE),                   # a stride that is no multiple of 8
    (dict(k=rows(head=-128)), kd.ESHAPE),
    (dict(d=96), kd.ESHAPE),
    (dict(hq=7), kd.ESHAPE),
    (dict(Bt=0), kd.ESHAPE),
    (dict(batch=0), kd.ESHAPE),
    (dict(hq=8192, hkv=1), kd.ESHAPE),
    (dict(hq=1, hkv=1, Bt=1 << 27, batch=2), kd.ESHAPE),
    (dict(q_out=None), kd.EINVAL),
    (dict(k_out=(1 << 33) + 8), kd.EINVAL),
    (dict(q_out=P), kd.EINVAL),                             # in place
    (dict(k_out=1 << 32), kd.EINVAL),                       # both outputs in one place
    (dict(pos0=97), kd.ESHAPE),                             # the block ends behind the tables
    (dict(pos0=-1), kd.ESHAPE),
    (dict(f=form(cos_table=None)), kd.EINVAL),
    (dict(f=form(k_weight=None)), kd.EINVAL),
    (dict(f=form(q_weight=None, k_weight=None, cos_table=None, sin_table=None)), kd.EINVAL),   # nothing to do
    (dict(f=form(q_weight=P + 8)), kd.EINVAL),
    (dict(f=form(sin_table=P + 4)), kd.EINVAL),
    (dict(f=form(q_weight_stride=64)), kd.ESHAPE),          # shorter than a row
    (dict(f=form(k_weight_stride=132)), kd.ESHAPE),
    (dict(f=form(norm_eps=-1.0)), kd.EINVAL),
    (dict(f=form(norm_eps=float("nan"))), kd.EINVAL),
    (dict(f=form(table_rows=0)), kd.ESHAPE),
])
def test_norm_rope_refuses(kw, code):
    assert norm_rope(**kw) == code
    assert len(kd.load_library().keydiff_last_error()) > 8


def append(b=None, q=rows(), k=rows(), v=rows(), Bt=1, f=None, q_out=1 << 40):
    b = branches() if b is None else b
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return kd.load_library().keydiff_branch_append(ref(b), ref(q), ref(k), ref(v), Bt, None, ref(f), q_out, None)


@pytest.mark.parametrize("kw,code", [
    (dict(b=branches(k_pages=None)), kd.EINVAL),
    (dict(b=branches(table=None)), kd.EINVAL),
    (dict(b=branches(lens=None)), kd.EINVAL),
    (dict(b=branches(v_pages=(1 << 30) + 8)), kd.EINVAL),
    (dict(b=branches(page_rows=24)), kd.ESHAPE),
    (dict(b=branches(page_rows=4)), kd.ESHAPE),
    (dict(b=branches(page_rows=2048)), kd.ESHAPE),
    (dict(b=branches(n_pages=0)), kd.ESHAPE),
    (dict(b=branches(table_width=0)), kd.ESHAPE),
    (dict(b=branches(table_width=1 << 27)), kd.ESHAPE),
    (dict(b=branches(n_seqs=0)), kd.ESHAPE),
    (dict(b=branches(head_dim=80)), kd.ESHAPE),
    (dict(b=branches(n_kv_heads=3)), kd.ESHAPE),
    (dict(b=branches(v_pages=P + 256)), kd.EINVAL),         # the pools overlap
    (dict(Bt=0), kd.ESHAPE),
    (dict(q=None), kd.EINVAL),                              # q_out without q
    (dict(q_out=None), kd.EINVAL),
    (dict(q_out=(1 << 40) + 2), kd.EINVAL),
    (dict(k=None), kd.EINVAL),
    (dict(v=rows(None)), kd.EINVAL),
    (dict(v=rows(token=4)), kd.ESHAPE),
    (dict(f=form(sin_table=None)), kd.EINVAL),
    (dict(k=rows(P + 1024)), kd.EINVAL),                    # the new keys lie in the pool
])
def test_branch_append_refuses(kw, code):
    if "k" not in kw and "v" not in kw:
        kw = dict(kw, k=rows(1 << 41), v=rows(1 << 42))
        kw.setdefault("q", rows(1 << 43))
    assert append(**kw) == code
    assert len(kd.load_library().keydiff_last_error()) > 8


def attention(b=None, q=rows(), Bt=1, kp=P, vp=P, prompts=2, rows_=100, cap=100, out=P, ws=P, ws_bytes=1 << 34):
    b = branches() if b is None else b
    return kd.load_library().keydiff_branch_attention(C.byref(b), C.byref(q), Bt, kp, vp, prompts, rows_, cap, 0.0, out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(b=branches(page_rows=12)), kd.ESHAPE),
    (dict(q=rows(None)), kd.EINVAL),
    (dict(out=None), kd.EINVAL),
    (dict(ws=None), kd.EINVAL),
    (dict(ws=P + 16), kd.EINVAL),
    (dict(ws_bytes=1000), kd.ESHAPE),
    (dict(prompts=3), kd.ESHAPE),                           # four sequences do not continue three prompts
    (dict(prompts=-1), kd.ESHAPE),
    (dict(rows_=-1), kd.ESHAPE),
    (dict(cap=99), kd.ESHAPE),
    (dict(kp=None), kd.EINVAL),
    (dict(vp=P + 8), kd.EINVAL),
    (dict(b=branches(n_seqs=1 << 24, table_width=1), prompts=0), kd.ESHAPE),                                    # 2^27 query rows
    (dict(b=branches(n_seqs=1 << 20, n_q_heads=8, n_kv_heads=8, table_width=1 << 20), prompts=0), kd.ESHAPE),   # tiles do not fit int32
])
def test_branch_attention_refuses(kw, code):
    assert attention(**kw) == code
    assert len(kd.load_library().keydiff_last_error()) > 8


def test_norm_rope_steps_refuse_before_anything_is_enqueued():
    lib = kd.load_library()
    f = form()
    assert lib.keydiff_prefill_block_norm_rope(None, P, P, P, 1, 0, C.byref(f), P, None, None) == kd.EINVAL
    none2 = (C.c_void_p * 2)()
    assert lib.keydiff_prefill_block_layers_norm_rope(none2, 2, none2, none2, none2, 1, 0, None, none2, None) == kd.EINVAL
    assert lib.keydiff_cache_branch_attention(None, None, None, 1, None, None, 0, None) == kd.EINVAL


def test_workspace_covers_what_the_launch_addresses():
    # one slot of partials per workgroup (shared part) or wave (own part) and per segment: sizes grow with both
    a = kd.branch_workspace_bytes(1, 32, 8, 128, 1, 1)
    assert a >= (256 + 8) * 16 * 128 * 4
    assert kd.branch_workspace_bytes(64, 32, 8, 128, 1, 1) > kd.branch_workspace_bytes(16, 32, 8, 128, 1, 1) > a
    assert kd.branch_workspace_bytes(64, 32, 8, 128, 8, 1) > kd.branch_workspace_bytes(64, 32, 8, 128, 1, 1)
    with pytest.raises(kd.KeyDiffError):
        kd.branch_workspace_bytes(5, 32, 8, 128, 1, 2)


def test_wrapper_refuses_tensors_that_do_not_fit():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    q, k = z(2, 8, 3, 64), z(2, 2, 3, 64)
    pages, table, lens = z(5, 2, 16, 64), z(2, 4, dt=torch.int32), z(2, dt=torch.int32)
    cos = z(50, 32, dt=torch.float32)
    w = z(64)
    with pytest.raises(ValueError, match="GPU"):
        kd.norm_rope(q, k, cos, cos)                                        # host tensors
    with pytest.raises(ValueError, match="k must be"):
        kd.norm_rope(q, k[:1], cos, cos)
    with pytest.raises(ValueError, match="q must be"):
        kd.norm_rope(q.float(), k, cos, cos)
    with pytest.raises(ValueError, match="contiguous last"):
        kd.norm_rope(z(2, 8, 64, 3).transpose(2, 3), k, cos, cos)
    with pytest.raises(ValueError, match="positions"):
        kd.norm_rope(q, k, cos, cos, positions=z(2, 4, dt=torch.int32))
    with pytest.raises(ValueError, match="together"):
        kd.norm_rope(q, k, cos, None)
    with pytest.raises(ValueError, match="q_weight"):
        kd.norm_rope(q, k, cos, cos, q_weight=z(7, 64), k_weight=w)
    with pytest.raises(ValueError, match="sin"):
        kd.norm_rope(q, k, cos, z(50, 64, dt=torch.float32))
    with pytest.raises(ValueError, match="sin"):
        kd.norm_rope(q, k, cos, cos[:40].contiguous())
    with pytest.raises(ValueError, match="v_new"):
        kd.branch_append(q, k, k[:, :1], pages, pages, table, lens)
    with pytest.raises(ValueError, match="k_pages"):
        kd.branch_append(q, k, k, z(5, 3, 16, 64), pages, table, lens)
    with pytest.raises(ValueError, match="v_pages"):
        kd.branch_append(q, k, k, pages, pages[:4], table, lens)
    with pytest.raises(ValueError, match="table"):
        kd.branch_append(q, k, k, pages, pages, table[:1], lens)
    with pytest.raises(ValueError, match="lens"):
        kd.branch_append(q, k, k, pages, pages, table, lens.long())
    with pytest.raises(ValueError, match="pos0"):
        kd.branch_append(q, k, k, pages, pages, table, lens, pos0=z(3, dt=torch.int32))
    with pytest.raises(ValueError, match="without q"):
        kd.branch_append(None, k, k, pages, pages, table, lens, q_out=q)
    with pytest.raises(ValueError, match="prefix values"):
        kd.branch_attention(q, pages, pages, table, lens, prefix=(z(1, 2, 30, 64), z(1, 2, 31, 64), 30))
    with pytest.raises(ValueError, match="are to be read"):
        kd.branch_attention(q, pages, pages, table, lens, prefix=(z(1, 2, 30, 64), z(1, 2, 30, 64), 31))
    with pytest.raises(ValueError, match="out"):
        kd.branch_attention(q, pages, pages, table, lens, out=q[:1])


def test_wrapper_refuses_what_is_no_tensor_and_leaks_no_reference():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    q, pages, table, lens = z(2, 8, 3, 64), z(5, 2, 16, 64), z(2, 4, dt=torch.int32), z(2, dt=torch.int32)
    before = [sys.getrefcount(t) for t in (q, pages, table, lens)]
    for _ in range(3):
        with pytest.raises(ValueError, match="k must be a tensor"):
            kd.norm_rope(q, [1, 2])
        with pytest.raises(TypeError):
            kd.norm_rope(q, q[:, :2], q_weight=z(64), k_weight=z(64), norm_eps="small")
        with pytest.raises(TypeError):
            kd.norm_rope(q, q[:, :2], q_weight=z(64), k_weight=z(64), pos0=0.5)
        with pytest.raises(ValueError, match="four dimensions"):
            kd.branch_attention(q[0], pages, pages, table, lens)
        with pytest.raises(ValueError, match="prefix values must be a tensor"):
            kd.branch_attention(q, pages, pages, table, lens, prefix=(z(1, 2, 30, 64), None, 30))
        with pytest.raises(ValueError):
            kd.branch_attention(q, pages, pages, table, lens, prefix=(z(1, 2, 30, 64), z(1, 2, 30, 64)))
        with pytest.raises(ValueError, match="GPU"):
            kd.branch_attention(q, pages, pages, table, lens, out=q.clone())
    assert [sys.getrefcount(t) for t in (q, pages, table, lens)] == before
