"""branch_chunk_attention, branch_weights and branch_evict: what they refuse, found before anything is enqueued (no GPU needed)."""
import ctypes as C
import sys

import pytest

from paper_2504_15364_amd import binding as kd

torch = pytest.importorskip("torch")
G = 1 << 30   # pointers below stand for device memory, far apart unless a case moves one
INF, NAN = float("inf"), float("nan")


def rows(data=7 * G, seq=8 * 40 * 128, head=40 * 128, token=128):
    return kd._Rows(data, seq, head, token)


def branches(**kw):
    b = dict(k_pages=1 * G, v_pages=2 * G, table=3 * G, lens=4 * G, n_new=None, n_seqs=4, n_q_heads=8, n_kv_heads=2, head_dim=128, page_rows=16,
             n_pages=10, table_width=4)
    b.update(kw)
    return kd._Branches(**b)


def refused(rc, code, word=None):
    said = kd.load_library().keydiff_last_error()
    assert rc == code, said
    assert len(said) > 8 and (word is None or word in said), said


ROWS = 4 * 8 * 40 * 128 * 2            # bytes of q and out
LSE = 4 * 8 * 40 * 4
POOL = 10 * 2 * 16 * 128 * 2
WORDS = 10 * 2 * 16 * 4                # of the weights, and of the positions
PREFIX = 2 * 2 * 100 * 128 * 2


def chunk(b=None, q=None, Bt=40, kp=5 * G, vp=6 * G, prompts=2, prefix_len=100, cap=100, scale=0.0, out=8 * G, lse=9 * G, ws=12 * G, ws_bytes=1 << 34):
    b, q = branches() if b is None else b, rows() if q is None else q
    return kd.load_library().keydiff_branch_chunk_attention(C.byref(b), C.byref(q), Bt, kp, vp, prompts, prefix_len, cap, scale, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(b=branches(k_pages=None)), kd.EINVAL, b"null"), (dict(b=branches(v_pages=None)), kd.EINVAL, b"null"),
    (dict(b=branches(table=None)), kd.EINVAL, b"null"), (dict(b=branches(lens=None)), kd.EINVAL, b"null"),
    (dict(b=branches(v_pages=2 * G + 8)), kd.EINVAL, b"aligned"), (dict(b=branches(page_rows=24)), kd.ESHAPE, b"page_rows"),
    (dict(b=branches(page_rows=4)), kd.ESHAPE, b"page_rows"), (dict(b=branches(page_rows=2048)), kd.ESHAPE, b"page_rows"),
    (dict(b=branches(n_pages=0)), kd.ESHAPE, b"n_pages"), (dict(b=branches(table_width=1 << 27)), kd.ESHAPE, b"2^30"),
    (dict(b=branches(n_seqs=0)), kd.ESHAPE, None), (dict(b=branches(head_dim=96)), kd.ESHAPE, None), (dict(b=branches(n_kv_heads=3)), kd.ESHAPE, None),
    (dict(Bt=0), kd.ESHAPE, None), (dict(Bt=-3), kd.ESHAPE, None),
    (dict(q=rows(None)), kd.EINVAL, None), (dict(q=rows(7 * G + 2)), kd.EINVAL, b"aligned"), (dict(q=rows(token=100)), kd.ESHAPE, None),
    (dict(q=rows(head=-128)), kd.ESHAPE, None),
    (dict(out=None), kd.EINVAL, b"null"), (dict(out=8 * G + 8), kd.EINVAL, b"out must"),
    (dict(lse=None), kd.EINVAL, b"lse"), (dict(lse=9 * G + 2), kd.EINVAL, b"lse must"),
    (dict(ws=None), kd.EINVAL, b"null"), (dict(ws=12 * G + 16), kd.EINVAL, b"workspace"), (dict(ws_bytes=1000), kd.ESHAPE, b"workspace"),
    (dict(prompts=3), kd.ESHAPE, b"divide"), (dict(prompts=-1), kd.ESHAPE, b"divide"), (dict(prefix_len=-1), kd.ESHAPE, b"prefix_len"),
    (dict(prefix_len=(1 << 23) + 1, cap=1 << 24), kd.ESHAPE, b"prefix_len"), (dict(cap=99), kd.ESHAPE, None), (dict(kp=None), kd.EINVAL, None),
    (dict(vp=6 * G + 8), kd.EINVAL, None),
    (dict(scale=NAN), kd.EINVAL, b"softmax_scale"), (dict(scale=INF), kd.EINVAL, b"softmax_scale"), (dict(scale=-INF), kd.EINVAL, b"softmax_scale"),
    (dict(b=branches(n_seqs=1 << 24, table_width=1), Bt=1, prompts=0), kd.ESHAPE, b"2^26"),
    (dict(b=branches(n_seqs=1 << 22, n_q_heads=10, n_kv_heads=10, table_width=1), prompts=0), kd.ESHAPE, None),
    # 2^25 query rows, and as many as 2^21 blocks of tiles whose tables hold 2^30 rows
    (dict(b=branches(n_seqs=1 << 18, n_q_heads=2, n_kv_heads=1, page_rows=1024, table_width=(1 << 20) - 1), Bt=64, prompts=0), kd.ESHAPE, None),
])
def test_chunk_attention_refuses(kw, code, word):
    refused(chunk(**kw), code, word)


@pytest.mark.parametrize("kw", [
    dict(out=7 * G + 16), dict(out=7 * G - ROWS + 16), dict(out=7 * G, q=rows(token=8 * 128, head=128)),   # over q, shifted, or laid out token by token
    dict(out=1 * G + POOL - 16), dict(out=2 * G), dict(out=5 * G + PREFIX - 16), dict(out=6 * G), dict(out=3 * G), dict(out=4 * G),
    dict(out=11 * G, b=branches(n_new=11 * G)), dict(ws=7 * G), dict(ws=8 * G), dict(ws=8 * G + ROWS - 256), dict(ws=1 * G), dict(ws=2 * G),
    dict(ws=5 * G), dict(ws=6 * G), dict(ws=3 * G), dict(ws=4 * G), dict(ws=11 * G, b=branches(n_new=11 * G)),
    dict(lse=7 * G + ROWS - 4), dict(lse=8 * G), dict(lse=8 * G - LSE + 4), dict(lse=12 * G), dict(lse=1 * G), dict(lse=2 * G + POOL - 4), dict(lse=5 * G),
    dict(lse=6 * G), dict(lse=3 * G), dict(lse=4 * G + 12), dict(lse=11 * G, b=branches(n_new=11 * G)),
])
def test_chunk_attention_refuses_outputs_over_what_it_reads(kw):
    need = kd.branch_chunk_workspace_bytes(4, 8, 2, 128, 40, 2)
    refused(chunk(ws_bytes=need, **kw), kd.EINVAL, b"overlap")
    assert need < G


def weights(b=None, q=None, Bt=40, lse=9 * G, w=10 * G, observe=0, decay=1.0, scale=0.0, ws=12 * G, ws_bytes=1 << 34):
    b, q = branches(v_pages=None) if b is None else b, rows() if q is None else q
    return kd.load_library().keydiff_branch_weights(C.byref(b), C.byref(q), Bt, lse, w, observe, decay, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(b=branches(k_pages=None)), kd.EINVAL, b"null"), (dict(b=branches(k_pages=G + 8)), kd.EINVAL, b"aligned"),
    (dict(b=branches(page_rows=24)), kd.ESHAPE, b"page_rows"), (dict(b=branches(n_kv_heads=3)), kd.ESHAPE, None),
    (dict(b=branches(head_dim=256)), kd.ESHAPE, None), (dict(Bt=0), kd.ESHAPE, None),
    (dict(q=rows(None)), kd.EINVAL, None), (dict(q=rows(token=4)), kd.ESHAPE, None), (dict(q=rows(7 * G + 4)), kd.EINVAL, b"aligned"),
    (dict(lse=None), kd.EINVAL, b"null"), (dict(lse=9 * G + 1), kd.EINVAL, b"lse"), (dict(w=None), kd.EINVAL, b"null"),
    (dict(w=10 * G + 4), kd.EINVAL, b"aligned"), (dict(ws=None), kd.EINVAL, b"null"), (dict(ws=12 * G + 128), kd.EINVAL, b"256"),
    (dict(ws_bytes=8), kd.ESHAPE, b"workspace"), (dict(observe=-1), kd.ESHAPE, b"observe"), (dict(decay=-0.5), kd.EINVAL, b"decay"),
    (dict(decay=1.5), kd.EINVAL, b"decay"), (dict(decay=NAN), kd.EINVAL, b"decay"), (dict(scale=NAN), kd.EINVAL, b"softmax_scale"),
    (dict(scale=INF), kd.EINVAL, b"softmax_scale"), (dict(b=branches(n_seqs=1 << 24, table_width=1), Bt=1), kd.ESHAPE, b"2^26"),
])
def test_weights_refuse(kw, code, word):
    refused(weights(**kw), code, word)


@pytest.mark.parametrize("kw", [
    dict(w=7 * G), dict(w=9 * G + LSE - 16), dict(w=1 * G + POOL - 16), dict(w=3 * G), dict(w=4 * G), dict(w=12 * G),
    dict(w=11 * G, b=branches(n_new=11 * G)), dict(ws=7 * G), dict(ws=9 * G), dict(ws=10 * G), dict(ws=1 * G), dict(ws=3 * G), dict(ws=4 * G),
    dict(ws=11 * G, b=branches(n_new=11 * G)),
])
def test_weights_refuse_outputs_over_what_they_read(kw):
    refused(weights(ws_bytes=kd.branch_weights_workspace_bytes(4, 8, 2, 128, 40), **kw), kd.EINVAL, b"overlap")


def evict(b=None, Bt=3, w=10 * G, p=11 * G, pos0=13 * G, budget=20, window=4, status=14 * G, ws=12 * G, ws_bytes=1 << 34):
    b = branches(n_q_heads=2) if b is None else b
    return kd.load_library().keydiff_branch_evict(C.byref(b), Bt, w, p, pos0, budget, window, status, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(b=branches(k_pages=None)), kd.EINVAL, b"null"), (dict(b=branches(v_pages=None)), kd.EINVAL, b"null"),
    (dict(b=branches(table=None)), kd.EINVAL, b"null"), (dict(b=branches(lens=None)), kd.EINVAL, b"null"),
    (dict(b=branches(page_rows=12)), kd.ESHAPE, b"page_rows"), (dict(b=branches(n_pages=0)), kd.ESHAPE, None),
    (dict(b=branches(table_width=0)), kd.ESHAPE, None), (dict(b=branches(head_dim=32)), kd.ESHAPE, None), (dict(Bt=0), kd.ESHAPE, None),
    (dict(budget=0), kd.ESHAPE, b"budget"), (dict(budget=-7), kd.ESHAPE, b"budget"), (dict(window=-1), kd.ESHAPE, b"window"),
    (dict(window=20), kd.ESHAPE, b"window"), (dict(w=None), kd.EINVAL, b"null"), (dict(p=None), kd.EINVAL, b"null"), (dict(ws=None), kd.EINVAL, b"null"),
    (dict(w=10 * G + 8), kd.EINVAL, b"aligned"), (dict(p=11 * G + 8), kd.EINVAL, b"aligned"), (dict(status=14 * G + 2), kd.EINVAL, b"status"),
    (dict(ws=12 * G + 64), kd.EINVAL, b"256"), (dict(ws_bytes=3), kd.ESHAPE, b"workspace"),
    (dict(b=branches(n_seqs=1 << 22, n_q_heads=2, table_width=1)), kd.ESHAPE, b"2^22"),
])
def test_evict_refuses(kw, code, word):
    refused(evict(**kw), code, word)


@pytest.mark.parametrize("kw", [
    dict(b=branches(n_q_heads=2, v_pages=1 * G + POOL - 16)), dict(w=1 * G), dict(w=2 * G), dict(w=11 * G + WORDS - 16), dict(w=3 * G), dict(w=4 * G),
    dict(p=1 * G), dict(p=13 * G), dict(p=14 * G), dict(ws=1 * G), dict(ws=10 * G), dict(ws=11 * G), dict(ws=3 * G), dict(status=4 * G + 4),
    dict(status=13 * G), dict(status=3 * G), dict(status=12 * G), dict(w=15 * G, b=branches(n_q_heads=2, n_new=15 * G)),
])
def test_evict_refuses_pages_over_one_another(kw):
    refused(evict(ws_bytes=kd.branch_evict_workspace_bytes(4, 2, 64, 20), **kw), kd.EINVAL, b"overlap")


def test_calls_on_a_cache_that_is_none():
    lib, b, q = kd.load_library(), branches(), rows()
    refused(lib.keydiff_cache_branch_chunk_attention(None, C.byref(b), C.byref(q), 40, 8 * G, 9 * G, 12 * G, 1 << 34, None), kd.EINVAL)


def test_workspaces():
    lib, size = kd.load_library(), C.c_size_t()
    for call in (lib.keydiff_branch_chunk_workspace_bytes, lib.keydiff_branch_weights_workspace_bytes):
        b = branches()
        assert call(None, 40, 0, C.byref(size)) == kd.EINVAL and call(C.byref(b), 40, 0, None) == kd.EINVAL
        assert call(C.byref(b), 0, 0, C.byref(size)) == kd.ESHAPE
    assert lib.keydiff_branch_evict_workspace_bytes(None, 4, C.byref(size)) == kd.EINVAL
    # chunk attention: bounded by the device and not by the call; that of few rows is branch_attention's
    assert kd.branch_chunk_workspace_bytes(4, 8, 2, 128, 1000) == kd.branch_chunk_workspace_bytes(400, 8, 2, 128, 10000)
    assert kd.branch_chunk_workspace_bytes(64, 32, 8, 128, 8, 1) == kd.branch_workspace_bytes(64, 32, 8, 128, 8, 1)
    assert kd.branch_chunk_workspace_bytes(2, 32, 8, 128, 16, 1) == kd.branch_workspace_bytes(2, 32, 8, 128, 16, 1)
    for call in (lambda: kd.branch_chunk_workspace_bytes(5, 8, 2, 128, 40, 2), lambda: kd.branch_chunk_workspace_bytes(1 << 24, 8, 2, 128, 1),
                 lambda: kd.branch_weights_workspace_bytes(1 << 24, 8, 2, 128, 1), lambda: kd.branch_weights_workspace_bytes(4, 8, 2, 128, 1, -1),
                 lambda: kd.branch_evict_workspace_bytes(4, 2, 0, 8), lambda: kd.branch_evict_workspace_bytes(4, 2, (1 << 30) + 1, 8),
                 lambda: kd.branch_evict_workspace_bytes(4, 2, 64, 0), lambda: kd.branch_evict_workspace_bytes(1 << 23, 1, 64, 8)):
        with pytest.raises(kd.KeyDiffError) as e:
            call()
        assert e.value.code == kd.ESHAPE


def tensors(n=2, Bt=3):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    return dict(q=z(n, 8, Bt, 64), pages=z(5, 2, 16, 64), w=z(5, 2, 16, dt=torch.float32), p=z(5, 2, 16, dt=torch.int32), table=z(n, 4, dt=torch.int32),
                lens=z(n, dt=torch.int32), lse=z(n, 8, Bt, dt=torch.float32))


def test_wrapper_refuses_tensors_that_do_not_fit():
    t = tensors()
    q, pages, w, p, table, lens, lse = t.values()

    def attention(q=q, k=pages, v=pages, table=table, lens=lens, **kw):
        return kd.branch_chunk_attention(q, k, v, table, lens, **kw)

    def weigh(q=q, k=pages, w=w, table=table, lens=lens, lse=lse, **kw):
        return kd.branch_weights(q, k, w, table, lens, lse, **kw)

    def drop(k=pages, v=pages, w=w, p=p, table=table, lens=lens, budget=8, **kw):
        return kd.branch_evict(k, v, w, p, table, lens, budget, **kw)

    cases = [
        (attention, dict(), "GPU"), (attention, dict(q=q[0]), "four dimensions"), (attention, dict(q=q.float()), "q must be"),
        (attention, dict(q=q.transpose(2, 3)), "last|q must"), (attention, dict(v=pages[:4]), "v_pages"), (attention, dict(table=table[:1]), "table"),
        (attention, dict(lens=lens.long()), "lens"), (attention, dict(n_new=lens[:1]), "n_new"), (attention, dict(out=q[:1]), "out"),
        (attention, dict(lse=lse[:, :4]), "lse"), (attention, dict(lse=lse.double()), "lse"), (attention, dict(out=q.transpose(0, 1)), "out"),
        (attention, dict(prefix=(pages[:1], pages[:1, :, :3], 3)), "prefix values"), (attention, dict(prefix=(pages[:1], pages[:1], 17)), "are to be read"),
        (attention, dict(workspace=lse), "workspace|GPU"), (attention, dict(lse=3), "lse must be a tensor"),
        (weigh, dict(), "GPU"), (weigh, dict(q=q[0]), "four dimensions"), (weigh, dict(k=pages[0]), "four dimensions"), (weigh, dict(w=w[:4]), "w_pages"),
        (weigh, dict(w=w.bfloat16()), "w_pages"), (weigh, dict(w=w.transpose(1, 2)), "w_pages"), (weigh, dict(lse=lse[:, :, :2]), "lse"),
        (weigh, dict(lse=None), "lse must be a tensor"), (weigh, dict(n_new=lens.long()), "n_new"), (weigh, dict(table=table.long()), "table"),
        (drop, dict(), "GPU"), (drop, dict(k=pages[0]), "four dimensions"), (drop, dict(v=pages[:, :1]), "v_pages"), (drop, dict(w=p), "w_pages"),
        (drop, dict(p=w), "p_pages"), (drop, dict(p=p[:, :, ::2]), "p_pages"), (drop, dict(table=table[0]), "table"), (drop, dict(lens=lens[:1]), "lens"),
        (drop, dict(pos0=lens.long()), "pos0"), (drop, dict(pos0=lens[:1]), "pos0"), (drop, dict(status=lens), "status"), (drop, dict(budget=1 << 40), "budget"),
        (drop, dict(window=1 << 33), "window"), (drop, dict(Bt=-(1 << 35)), "Bt"),
    ]
    for call, kw, word in cases:
        with pytest.raises(ValueError, match=word):
            call(**kw)


def test_wrapper_refuses_what_is_no_number_and_leaks_no_reference():
    t = tensors()
    q, pages, w, p, table, lens, lse = t.values()
    before = [sys.getrefcount(x) for x in (q, pages, w, p, table, lens, lse)]
    for _ in range(3):
        for call in (lambda: kd.branch_chunk_attention(q, pages, pages, table, lens, softmax_scale="1"),
                     lambda: kd.branch_weights(q, pages, w, table, lens, lse, decay="all"),
                     lambda: kd.branch_weights(q, pages, w, table, lens, lse, observe=0.5),
                     lambda: kd.branch_evict(pages, pages, w, p, table, lens, 1.5), lambda: kd.branch_evict(pages, pages, w, p, table, lens, None)):
            with pytest.raises(TypeError):
                call()
        for call in (lambda: kd.branch_chunk_attention(q, pages, pages, table, lens, out=q.clone(), lse=lse),
                     lambda: kd.branch_weights(q, pages, w, table, lens, lse), lambda: kd.branch_evict(pages, pages, w, p, table, lens, 8)):
            with pytest.raises(ValueError, match="GPU"):
                call()
    assert [sys.getrefcount(x) for x in (q, pages, w, p, table, lens, lse)] == before


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        cuda_stream, device = 64, torch.device("cuda:1")

    q, pages, w, p, table, lens, lse = tensors().values()
    for call in (lambda: kd.branch_chunk_attention(q, pages, pages, table, lens, stream=Elsewhere()),
                 lambda: kd.branch_weights(q, pages, w, table, lens, lse, stream=Elsewhere()),
                 lambda: kd.branch_evict(pages, pages, w, p, table, lens, 8, stream=Elsewhere())):
        with pytest.raises(ValueError, match="stream belongs to cuda:1"):
            call()
