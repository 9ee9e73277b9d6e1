"""Calls of norm_rope, branch_append and branch_attention that are refused although every argument is well formed by itself (no GPU needed:
they are refused before anything is enqueued)."""
import ctypes as C

import pytest

from paper_2504_15364_amd import binding as kd

G = 1 << 30   # pointers below stand for device memory, far apart unless a case moves one


def rows(data, seq, head, token):
    return kd._Rows(data, seq, head, token)


def attention(n=4, hq=8, hkv=2, d=128, Bt=2, page_rows=16, pages=10, width=4, q=None, out=8 * G, ws=12 * G, cap=100, n_new=None,
              kp=5 * G, vp=6 * G, prompts=2, prefix_len=100, scale=0.0, **at):
    at = dict(dict(k_pages=1 * G, v_pages=2 * G, table=3 * G, lens=4 * G), **at)
    b = kd._Branches(n_new=n_new, n_seqs=n, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_rows=page_rows, n_pages=pages, table_width=width, **at)
    q = rows(7 * G, hq * Bt * d, Bt * d, d) if q is None else q
    need = kd.branch_workspace_bytes(n, hq, hkv, d, Bt, prompts)
    return kd.load_library().keydiff_branch_attention(C.byref(b), C.byref(q), Bt, kp, vp, prompts, prefix_len, cap, scale, out, ws, need, None)


ROWS = 4 * 8 * 2 * 128 * 2             # bytes of q and out above
POOL = 10 * 2 * 16 * 128 * 2
PREFIX = 2 * 2 * 100 * 128 * 2


@pytest.mark.parametrize("kw", [
    dict(out=7 * G + 16), dict(out=7 * G - ROWS + 16),                               # out over q, shifted
    dict(out=7 * G, q=rows(7 * G, 8 * 2 * 128, 128, 8 * 128)),                       # ... in its place, but q is laid out token by token
    dict(out=7 * G, q=rows(7 * G, 2 * 8 * 2 * 128, 2 * 128, 128)),                   # ... but q has gaps between sequences
    dict(out=7 * G + 8 * 2 * 128 * 2, q=rows(7 * G, 16 * 2 * 128, 2 * 128, 128)),    # ... in such a gap: within q's extent all the same
    dict(out=1 * G + POOL - 16), dict(out=2 * G), dict(out=5 * G + PREFIX - 16), dict(out=6 * G - 16), dict(out=3 * G), dict(out=4 * G),
    dict(out=9 * G, n_new=9 * G),
    dict(ws=7 * G), dict(ws=8 * G), dict(ws=1 * G), dict(ws=2 * G), dict(ws=5 * G), dict(ws=6 * G), dict(ws=3 * G), dict(ws=4 * G),
    dict(ws=8 * G + ROWS - 256), dict(ws=9 * G, n_new=9 * G),
])
def test_branch_attention_refuses_outputs_over_what_it_reads(kw):
    assert attention(**kw) == kd.EINVAL
    assert b"overlap" in kd.load_library().keydiff_last_error()


@pytest.mark.parametrize("pos0", [2 ** 63 - 1, 2 ** 63 - 4, 2 ** 31 - 4, 97])
def test_norm_rope_refuses_positions_whose_sum_with_the_tokens_does_not_fit(pos0):
    q, k = rows(1 * G, 0, 128, 128), rows(2 * G, 0, 128, 128)
    for tables in (3 * G, None):
        form = kd._RowForm(q_weight=5 * G, k_weight=5 * G, norm_eps=1e-6, cos_table=tables, sin_table=tables, table_rows=100)
        if tables is None and pos0 == 97:
            continue   # (without tables any position will do)
        rc = kd.load_library().keydiff_norm_rope(C.byref(q), C.byref(k), 1, 1, 1, 128, 4, pos0, None, C.byref(form), 6 * G, 7 * G, None)
        assert rc == kd.ESHAPE and b"position" in kd.load_library().keydiff_last_error()


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf"), 1e39])   # (1e39: infinite as a float)
def test_branch_attention_refuses_a_scale_that_is_no_number(scale):
    assert attention(scale=C.c_float(scale)) == kd.EINVAL
    assert b"softmax_scale" in kd.load_library().keydiff_last_error()


def test_no_workspace_for_calls_that_are_refused():
    # (2^27 query rows: the wrapper would allocate its gigabytes ahead of the refusal)
    assert kd.branch_workspace_bytes(1 << 23, 8, 2, 128, 1, 0) > 0
    with pytest.raises(kd.KeyDiffError) as e:
        kd.branch_workspace_bytes(1 << 24, 8, 2, 128, 1, 0)
    assert e.value.code == kd.ESHAPE


def test_a_stream_of_another_device_is_refused():
    torch = pytest.importorskip("torch")

    class Elsewhere:
        cuda_stream, device = 64, torch.device("cuda:1")

    x = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    pages, table = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16), torch.zeros((1, 1), dtype=torch.int32)
    for call in (lambda: kd.norm_rope(x, x, stream=Elsewhere()), lambda: kd.branch_append(x, x, x, pages, pages, table, table[0], stream=Elsewhere()),
                 lambda: kd.branch_attention(x, pages, pages, table, table[0], stream=Elsewhere())):
        with pytest.raises(ValueError, match="stream belongs to cuda:1"):
            call()


def test_status_words_that_do_not_fit_are_refused():
    torch = pytest.importorskip("torch")
    q, k = rows(1 * G, 0, 128, 128), rows(2 * G, 0, 128, 128)
    form = kd._RowForm(q_weight=5 * G, k_weight=5 * G, norm_eps=1e-6, status=8 * G + 2)
    assert kd.load_library().keydiff_norm_rope(C.byref(q), C.byref(k), 1, 1, 1, 128, 4, 0, None, C.byref(form), 6 * G, 7 * G, None) == kd.EINVAL
    assert b"status" in kd.load_library().keydiff_last_error()
    x = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    pages, table = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16), torch.zeros((1, 1), dtype=torch.int32)
    for status in (torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int64), torch.tensor(0, dtype=torch.int32), 3):
        with pytest.raises(ValueError, match="status"):
            kd.norm_rope(x, x, q_weight=x[0, 0, 0], k_weight=x[0, 0, 0], status=status)
        with pytest.raises(ValueError, match="status"):
            kd.branch_append(x, x, x, pages, pages, table, table[0], status=status)
