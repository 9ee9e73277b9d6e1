"""Binding of include/keydiff.h -- argument marshalling only (ctypes; the calls of a generation step through csrc/calls.cpp).

Every step of the path runs in the library's HIP kernels.  PyTorch appears only
as the owner of device memory and streams.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkeydiff.so")

OK, EINVAL, ESHAPE, ESTATE, EHIP = 0, -1, -2, -3, -4
ANCHOR_MEAN_KEY, ANCHOR_MEAN_UNIT_KEY = 0, 1
LAYOUT_ORDERED, LAYOUT_FILL = 0, 1
LEFT_OUT_POSITION, LEFT_OUT_ROW = 1, 2   # bits that norm_rope and branch_append set in `status`
KERNEL_NAMES = ("step_main", "step_score", "step_post", "compact_ordered", "aux", "event_pair", "select_alone")

EXPORTS = (
    "keydiff_workspace_bytes", "keydiff_init_cache", "keydiff_prefill_block", "keydiff_prefill_block_static",
    "keydiff_prefill_block_deferred",
    "keydiff_prefill_block_layers", "keydiff_prefill_block_rope", "keydiff_prefill_block_layers_rope", "keydiff_finish", "keydiff_decode_step",
    "keydiff_prefill_block_norm_rope", "keydiff_prefill_block_layers_norm_rope", "keydiff_norm_rope", "keydiff_branch_append",
    "keydiff_branch_workspace_bytes", "keydiff_branch_attention", "keydiff_cache_branch_attention",
    "keydiff_scores", "keydiff_cache_len", "keydiff_cache_plan", "keydiff_cache_positions", "keydiff_cache_load",
    "keydiff_cache_status", "keydiff_profile_enable", "keydiff_profile_read", "keydiff_destroy_cache",
    "keydiff_last_error", "keydiff_version",
)


class KeyDiffError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"keydiff error {code}: {message}")
        self.code = code


class _Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "budget_N", "block_B",
                                         "anchor_mode", "window_W", "layout")] + \
               [("eps", C.c_float), ("softmax_scale", C.c_float)]


class _RowForm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("q_weight_stride", C.c_int64),
                ("k_weight_stride", C.c_int64), ("norm_eps", C.c_float), ("cos_table", C.c_void_p),
                ("sin_table", C.c_void_p), ("table_rows", C.c_int64), ("status", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("seq_stride", C.c_int64), ("head_stride", C.c_int64), ("token_stride", C.c_int64)]


class _Branches(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_pages", "v_pages", "table", "lens", "n_new")] + \
               [(n, C.c_int32) for n in ("n_seqs", "n_q_heads", "n_kv_heads", "head_dim", "page_rows", "n_pages", "table_width")]


@dataclass
class KeyDiffConfig:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    budget_N: int
    block_B: int
    anchor_mode: int = ANCHOR_MEAN_KEY
    window_W: int = 0
    layout: int = LAYOUT_ORDERED
    eps: float = 0.0
    softmax_scale: float = 0.0

    def _c(self) -> _Config:
        return _Config(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.budget_N, self.block_B,
                       self.anchor_mode, self.window_W, self.layout, self.eps, self.softmax_scale)


_lib = None


def load_library() -> C.CDLL:
    """Load libkeydiff.so; there is no fallback if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = os.environ.get("KEYDIFF_LIBRARY", LIB_PATH)   # override: another build of the same ABI
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2504_15364_amd.build`")
    L = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    szp = C.POINTER(C.c_size_t)
    L.keydiff_workspace_bytes.argtypes = [C.POINTER(_Config), szp, szp, szp, szp]
    L.keydiff_init_cache.argtypes = [C.POINTER(_Config), vp, vp, vp, vp, vp, C.POINTER(vp)]
    L.keydiff_prefill_block.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp]
    L.keydiff_prefill_block_static.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp]
    L.keydiff_prefill_block_deferred.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp]
    pp = C.POINTER(vp)
    L.keydiff_prefill_block_layers.argtypes = [pp, i32, pp, pp, pp, i32, i64, pp, vp]
    L.keydiff_prefill_block_rope.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, i64, vp, vp, vp]
    L.keydiff_prefill_block_layers_rope.argtypes = [pp, i32, pp, pp, pp, i32, i64, vp, vp, i64, pp, vp]
    fp = rp = bp = vp   # keydiff_row_form_t, keydiff_rows_t, keydiff_branches_t: a structure by reference, or its bytes
    L.keydiff_prefill_block_norm_rope.argtypes = [vp, vp, vp, vp, i32, i64, fp, vp, vp, vp]
    L.keydiff_prefill_block_layers_norm_rope.argtypes = [pp, i32, pp, pp, pp, i32, i64, fp, pp, vp]
    L.keydiff_norm_rope.argtypes = [rp, rp, i32, i32, i32, i32, i32, i64, vp, fp, vp, vp, vp]
    L.keydiff_branch_append.argtypes = [bp, rp, rp, rp, i32, vp, fp, vp, vp]
    L.keydiff_branch_workspace_bytes.argtypes = [bp, i32, i32, szp]
    L.keydiff_branch_attention.argtypes = [bp, rp, i32, vp, vp, i32, i32, i64, C.c_float, vp, vp, C.c_size_t, vp]
    L.keydiff_cache_branch_attention.argtypes = [vp, bp, rp, i32, vp, vp, C.c_size_t, vp]
    L.keydiff_finish.argtypes = [vp, vp]
    L.keydiff_decode_step.argtypes = [vp, vp, vp, vp, i64, vp, vp]
    L.keydiff_scores.argtypes = [vp, vp, vp]
    L.keydiff_cache_len.argtypes = [vp, C.POINTER(i32)]
    L.keydiff_cache_plan.argtypes = [vp, C.POINTER(i32)]
    L.keydiff_cache_positions.argtypes = [vp, vp, vp]
    L.keydiff_cache_load.argtypes = [vp, vp, vp, vp, i32, vp]
    L.keydiff_cache_status.argtypes = [vp, C.POINTER(i32), vp]
    L.keydiff_profile_enable.argtypes = [vp, i32]
    L.keydiff_profile_read.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(i32)]
    L.keydiff_destroy_cache.argtypes = [vp]
    L.keydiff_destroy_cache.restype = None
    L.keydiff_last_error.argtypes = []
    L.keydiff_last_error.restype = C.c_char_p
    L.keydiff_version.argtypes = []
    for name in EXPORTS:
        if name not in ("keydiff_destroy_cache", "keydiff_last_error"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _check(rc: int):
    if rc != OK:
        raise KeyDiffError(rc, load_library().keydiff_last_error().decode())


def workspace_bytes(cfg: KeyDiffConfig):
    k, v, m, s = (C.c_size_t() for _ in range(4))
    c = cfg._c()
    _check(load_library().keydiff_workspace_bytes(C.byref(c), C.byref(k), C.byref(v), C.byref(m), C.byref(s)))
    return k.value, v.value, m.value, s.value


def _stream_ptr(stream):
    if stream is None:
        # what torch.cuda.current_stream().cuda_stream is, without the stream object around it (2.8 us a call, of 12 that
        # a block step took on the host; this way 0.2); a name of torch's own, so not to be relied on
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def check_block_shapes(cfg, q, k_new, v_new, out=None, Bt=None):
    """The tensors of one block against the cache's configuration: q (and out) [batch][Hq][Bt][d],
    k_new / v_new [batch][Hkv][Bt][d].  The C ABI takes bare pointers and cannot know how much memory
    lies behind them: a tensor smaller than the configuration says would be read past its end by the
    kernels, so the wrapper refuses it here, before anything is enqueued.  Returns Bt."""
    if Bt is None:
        Bt = int(k_new.shape[-2])
    want_q = (cfg.batch, cfg.n_q_heads, Bt, cfg.head_dim)
    want_kv = (cfg.batch, cfg.n_kv_heads, Bt, cfg.head_dim)
    # (a torch.Size is a tuple; compared as it is, the four checks take a third of the time)
    if not ((q is None or q.shape == want_q) and (k_new is None or k_new.shape == want_kv)
            and (v_new is None or v_new.shape == want_kv) and (out is None or out.shape == want_q)):
        for name, t, want in (("q", q, want_q), ("k_new", k_new, want_kv), ("v_new", v_new, want_kv), ("out", out, want_q)):
            if t is not None and tuple(t.shape) != want:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, the cache's configuration needs {want}")
    return Bt


def check_load_shapes(cfg, cap, k, v, pos):
    """Tensors handed to keydiff_cache_load: k, v [batch][Hkv][len][d] bf16, pos [batch][Hkv][len] int32."""
    import torch
    if k.dim() != 4:
        raise ValueError(f"k has shape {tuple(k.shape)}, expected [batch][Hkv][len][d]")
    ln = int(k.shape[2])
    want = (cfg.batch, cfg.n_kv_heads, ln, cfg.head_dim)
    if ln > cap:
        raise ValueError(f"{ln} rows do not fit a cache of {cap} rows per head")
    for name, t in (("k", k), ("v", v)):
        if tuple(t.shape) != want or t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bf16 tensor of shape {want}, got {tuple(t.shape)} {t.dtype}")
    if tuple(pos.shape) != want[:3] or pos.dtype != torch.int32 or not pos.is_contiguous():
        raise ValueError(f"pos must be a contiguous int32 tensor of shape {want[:3]}, got {tuple(pos.shape)} {pos.dtype}")
    return ln


def check_rope_tables(cfg, cos, sin):
    import torch
    for name, t in (("cos", cos), ("sin", sin)):
        if t.dtype != torch.float32 or not t.is_contiguous() or t.dim() != 2 or t.shape[1] != cfg.head_dim // 2:
            raise ValueError(f"{name} must be a contiguous float32 table [positions][{cfg.head_dim // 2}], got {tuple(t.shape)} {t.dtype}")
    if cos.shape != sin.shape:
        raise ValueError("cos and sin tables differ in shape")


def prefill_block_layers(caches, q, k_new, v_new, pos0: int, out=None, stream=None, rope=None, norm=None):
    """One block through the layers of a model: `caches`, `q`, `k_new`, `v_new` (and `out`) are
    sequences with one entry per layer.  Layers shaped alike share their launches; else every layer's eviction
    rides in the next layer's launch.
    rope = (cos, sin): float32 device tables [positions][head_dim / 2]; q and k_new are then rotated
    inside the call (keydiff_prefill_block_layers_rope).
    norm = (q_weights, k_weights, eps): one bf16 weight tensor per layer each, [head_dim] or [heads][head_dim]; q and k_new are
    then normed for each head inside the call, ahead of the rotation if there is one (keydiff_prefill_block_layers_norm_rope)."""
    import torch
    n = len(caches)
    assert n >= 1 and len(q) == len(k_new) == len(v_new) == n
    Bt = k_new[0].shape[-2]
    for c, tq, tk, tv in zip(caches, q, k_new, v_new):
        for t in (tq, tk, tv):
            assert t.is_contiguous() and t.dtype == torch.bfloat16 and t.device == c.device
        check_block_shapes(c.cfg, tq, tk, tv, Bt=Bt)
    if out is None:
        out = [torch.empty_like(t) for t in q]
    assert len(out) == n
    for c, to in zip(caches, out):
        assert to.is_contiguous() and to.dtype == torch.bfloat16 and to.device == c.device
        check_block_shapes(c.cfg, None, None, None, out=to, Bt=Bt)
    arr = lambda ptrs: (C.c_void_p * n)(*ptrs)
    L = caches[0]._L
    if norm is not None:
        q_weights, k_weights, eps = norm
        if not len(q_weights) == len(k_weights) == n:
            raise ValueError(f"norm needs one weight tensor per layer, got {len(q_weights)} and {len(k_weights)} for {n} layers")
        cos, sin = rope if rope is not None else (None, None)
        forms = b"".join(_native().row_form(c.cfg.n_q_heads, c.cfg.n_kv_heads, c.cfg.head_dim, cos, sin, wq, wk, eps, t)
                         for c, wq, wk, t in zip(caches, q_weights, k_weights, q))
        _check(L.keydiff_prefill_block_layers_norm_rope(arr([c._h.value for c in caches]), n,
                                                        arr([t.data_ptr() for t in q]), arr([t.data_ptr() for t in k_new]),
                                                        arr([t.data_ptr() for t in v_new]), Bt, int(pos0), forms,
                                                        arr([t.data_ptr() for t in out]), _stream_ptr(stream)))
        return out
    if rope is not None:
        cos, sin = rope
        check_rope_tables(caches[0].cfg, cos, sin)
        _check(L.keydiff_prefill_block_layers_rope(arr([c._h.value for c in caches]), n,
                                                   arr([t.data_ptr() for t in q]), arr([t.data_ptr() for t in k_new]),
                                                   arr([t.data_ptr() for t in v_new]), Bt, int(pos0), cos.data_ptr(),
                                                   sin.data_ptr(), cos.shape[0], arr([t.data_ptr() for t in out]),
                                                   _stream_ptr(stream)))
        return out
    _check(L.keydiff_prefill_block_layers(arr([c._h.value for c in caches]), n,
                                          arr([t.data_ptr() for t in q]), arr([t.data_ptr() for t in k_new]),
                                          arr([t.data_ptr() for t in v_new]), Bt, int(pos0),
                                          arr([t.data_ptr() for t in out]), _stream_ptr(stream)))
    return out


# ------------------------------------------------------------------ norms and rotation alone; continuations of a prompt
_calls = None


def _native():
    """The compiled side of these calls (csrc/calls.cpp: checks, allocation and the call of the C ABI)."""
    global _calls
    if _calls is None:
        import importlib

        from torch import _C
        L = load_library()
        try:
            m = importlib.import_module("._calls", __package__)
        except ImportError as e:
            raise ImportError(f"{e}: build it first (python -m paper_2504_15364_amd.build)") from e
        address = lambda f: C.cast(f, C.c_void_p).value  # noqa: E731
        m.bind(*(address(f) for f in (L.keydiff_norm_rope, L.keydiff_branch_append, L.keydiff_branch_workspace_bytes,
                                      L.keydiff_branch_attention, L.keydiff_cache_branch_attention)),
               _C._cuda_getCurrentRawStream)
        _calls = m
    return _calls


def _call(name, device, stream, *args):
    """The compiled function on `stream`, an object of torch's or a handle (None: torch's current stream of the tensors' device).
    Tensors that it allocates belong to that stream."""
    f = getattr(_calls or _native(), name)
    if stream is None:
        r = f(*args)
    else:
        import torch
        if hasattr(stream, "cuda_stream") and stream.device != device:   # (the call would run on the current stream of the tensors' device)
            raise ValueError(f"the stream belongs to {stream.device}, the tensors live on {device}")
        with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(stream, device=device)):
            r = f(*args)
    if type(r) is int:
        _check(r)
    return r


def norm_rope(q, k, cos=None, sin=None, pos0: int = 0, positions=None, q_weight=None, k_weight=None, norm_eps: float = 1e-6,
              q_out=None, k_out=None, stream=None, status=None):
    """Root mean square norms of the queries and keys of each head (bf16 weights [d] or [heads][d]; None: no norm) and the rotary
    position embedding (float32 tables [positions][d / 2]; None: no rotation) in one pass.
    q [batch][Hq][T][d], k [batch][Hkv][T][d] bf16, any strides with a contiguous last dimension; token j is at position pos0 + j or
    at positions[b][j] (int32 [batch][T]; a token outside the tables is left out, its rows of the outputs stay as they are).
    status: an int32 tensor of one element; LEFT_OUT_POSITION is set in it, and nothing cleared, if a token was left out.
    Returns contiguous (q_out, k_out)."""
    return _call("norm_rope", q.device, stream, q, k, cos, sin, pos0, positions, q_weight, k_weight, norm_eps, q_out, k_out, status)


def branch_append(q, k_new, v_new, k_pages, v_pages, table, lens, n_new=None, pos0=None, cos=None, sin=None, q_weight=None,
                  k_weight=None, norm_eps: float = 1e-6, q_out=None, stream=None, status=None):
    """New tokens of sequences that continue prompts: norms and rotation of q and k_new as in norm_rope, keys and values into the
    sequences' pages behind the lens[s] rows they hold, at positions pos0[s] + lens[s] + j (pos0: int32 [n_seqs], the length of the
    sequence's prompt; None: zeros).  lens is not changed.
    q [n_seqs][Hq][Bt][d] (None: keys and values only), k_new, v_new [n_seqs][Hkv][Bt][d]; k_pages, v_pages
    [pages][Hkv][page_rows][d]; table int32 [n_seqs][width]; n_new int32 [n_seqs] (None: all Bt).  Returns the contiguous queries
    for branch_attention; tokens that are not taken (behind a sequence's n_new, lens < 0) keep their rows of q_out, which
    hold anything if it is None.
    A token is left out as well where its position lies outside the tables (branch_attention counts its row all the same), its row
    outside the table or its page outside the pool.  status: an int32 tensor of one element, in which such tokens set
    LEFT_OUT_POSITION or LEFT_OUT_ROW, and nothing is cleared."""
    return _call("branch_append", k_new.device, stream, q, k_new, v_new, k_pages, v_pages, table, lens, n_new, pos0, cos, sin, q_weight,
                 k_weight, norm_eps, q_out, status)


def branch_workspace_bytes(n_seqs, n_q_heads, n_kv_heads, head_dim, Bt=1, n_prefixes=0):
    """Bytes of the workspace that branch_attention needs for calls of these sizes on the current device."""
    b = _Branches(n_seqs=n_seqs, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim)
    size = C.c_size_t()
    _check(load_library().keydiff_branch_workspace_bytes(C.byref(b), Bt, n_prefixes, C.byref(size)))
    return size.value


def branch_attention(q, k_pages, v_pages, table, lens, prefix=None, n_new=None, softmax_scale: float = 0.0, out=None, workspace=None,
                     stream=None):
    """Attention of the tokens that branch_append has appended: token j of sequence s sees all rows of its prompt and its sequence's
    own rows 0 .. lens[s] + j (lens, table, n_new, pools: as given to branch_append).
    q [n_seqs][Hq][Bt][d] bf16 (any strides with a contiguous last dimension).
    prefix: the prompts' rows, shared by the sequences that continue them: a KeyDiffCache whose batch holds the prompts, or
    (k, v, rows) with k, v bf16 [prompts][Hkv][at least rows][d]; sequence s continues prompt s / (n_seqs / prompts).  None: own rows
    alone.  (A cache with a pending eviction is finished first; ahead of a captured call, finish() it: a replay would repeat that.)
    softmax_scale <= 0: 1/sqrt(d), or the cache's.
    workspace: a uint8 tensor of at least branch_workspace_bytes that no other call in flight uses (None: allocated for the call).
    out may be q itself where q is contiguous, and must else overlap nothing that the call reads.
    Returns out [n_seqs][Hq][Bt][d]; rows behind a sequence's n_new, and those of a sequence with lens < 0, are left as they were
    (they hold anything where out is None)."""
    handle = batch = keys = values = rows = None
    if isinstance(prefix, KeyDiffCache):
        handle, batch = prefix._h.value if prefix._h else 0, prefix.cfg.batch
        if prefix.device != q.device:
            raise ValueError(f"the cache lives on {prefix.device}, the queries on {q.device}")
    elif prefix is not None:
        keys, values, rows = prefix
    return _call("branch_attention", q.device, stream, q, k_pages, v_pages, table, lens, n_new, handle, batch, keys, values, rows,
                 softmax_scale, out, workspace)


class KeyDiffCache:
    """keydiff_cache_t over torch-owned device buffers.  Method names follow the C ABI."""

    def __init__(self, cfg: KeyDiffConfig, device="cuda:0", stream=None):
        import torch
        self._L = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        kb, vb, mb, sb = workspace_bytes(cfg)
        # the library never allocates device memory: torch owns these four buffers
        self._k = torch.empty(kb, dtype=torch.uint8, device=self.device)
        self._v = torch.empty(vb, dtype=torch.uint8, device=self.device)
        self._meta = torch.empty(mb, dtype=torch.uint8, device=self.device)
        self._scratch = torch.empty(sb, dtype=torch.uint8, device=self.device)
        self._h = C.c_void_p()
        c = cfg._c()
        with torch.cuda.device(self.device):
            _check(self._L.keydiff_init_cache(C.byref(c), self._k.data_ptr(), self._v.data_ptr(),
                                              self._meta.data_ptr(), self._scratch.data_ptr(),
                                              _stream_ptr(stream), C.byref(self._h)))
        self.cap = (cfg.budget_N + cfg.block_B + 3) & ~3   # rows per head of the cache buffers (see keydiff.h)

    def close(self):
        if getattr(self, "_h", None):
            self._L.keydiff_destroy_cache(self._h)
            self._h = None

    __del__ = close

    def _block_args(self, q, k_new, v_new, out, scores_out, allocate=True):
        """Checks the tensors of one block (dtype, device, layout, shape) and returns (Bt, out)."""
        import torch
        bf16, device = torch.bfloat16, self.device
        for t in (q, k_new, v_new, out):
            if t is not None and not (t.dtype is bf16 and t.device == device and t.is_contiguous()):
                raise ValueError("block tensors must be contiguous bf16 tensors on the cache's device")
        Bt = check_block_shapes(self.cfg, q, k_new, v_new, out)
        if out is None:
            if not allocate:
                raise ValueError("this call needs the caller's `out`")
            out = torch.empty_like(q)
        if scores_out is not None:
            need = self.cfg.batch * self.cfg.n_kv_heads * (self.len + Bt)
            if not (scores_out.is_contiguous() and scores_out.dtype == torch.float32 and scores_out.device == self.device
                    and scores_out.numel() >= need):
                raise ValueError(f"scores_out must be a contiguous float32 device tensor of at least {need} elements")
        return Bt, out

    # -- the calls of the C ABI ------------------------------------------------
    def prefill_block(self, q, k_new, v_new, pos0: int, out=None, scores_out=None, stream=None):
        """q [batch][Hq][Bt][d], k_new/v_new [batch][Hkv][Bt][d] bf16 device tensors."""
        Bt, out = self._block_args(q, k_new, v_new, out, scores_out)
        _check(self._L.keydiff_prefill_block(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), Bt,
                                             int(pos0), out.data_ptr(),
                                             scores_out.data_ptr() if scores_out is not None else None,
                                             _stream_ptr(stream)))
        return out

    def prefill_block_rope(self, q, k_new, v_new, pos0: int, cos, sin, out=None, scores_out=None, stream=None):
        """prefill_block on a block whose q and k_new are not rotated yet: cos, sin float32 device
        tables [positions][head_dim / 2]."""
        Bt, out = self._block_args(q, k_new, v_new, out, scores_out)
        check_rope_tables(self.cfg, cos, sin)
        _check(self._L.keydiff_prefill_block_rope(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), Bt,
                                                  int(pos0), cos.data_ptr(), sin.data_ptr(), cos.shape[0], out.data_ptr(),
                                                  scores_out.data_ptr() if scores_out is not None else None,
                                                  _stream_ptr(stream)))
        return out

    def prefill_block_norm_rope(self, q, k_new, v_new, pos0: int, cos, sin, q_weight, k_weight, norm_eps: float = 1e-6, out=None,
                                scores_out=None, stream=None):
        """prefill_block on a block whose q and k_new are neither normed nor rotated yet: bf16 weights [head_dim] or
        [heads][head_dim] of the root mean square norm of each head's rows, tables as for prefill_block_rope.  Weights None: no
        norm; tables None: no rotation."""
        Bt, out = self._block_args(q, k_new, v_new, out, scores_out)
        cfg = self.cfg
        form = _native().row_form(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cos, sin, q_weight, k_weight, norm_eps, q)
        _check(self._L.keydiff_prefill_block_norm_rope(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), Bt,
                                                       int(pos0), form, out.data_ptr(),
                                                       scores_out.data_ptr() if scores_out is not None else None,
                                                       _stream_ptr(stream)))
        return out

    def prefill_block_static(self, q, k_new, v_new, pos0: int, out, scores_out=None, stream=None):
        """prefill_block with the step's temporaries in the library's static device array; `out` is
        the caller's (this wrapper allocates nothing either)."""
        Bt, out = self._block_args(q, k_new, v_new, out, scores_out, allocate=False)
        _check(self._L.keydiff_prefill_block_static(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), Bt,
                                                    int(pos0), out.data_ptr(),
                                                    scores_out.data_ptr() if scores_out is not None else None,
                                                    _stream_ptr(stream)))
        return out

    def prefill_block_deferred(self, q, k_new, v_new, pos0: int, out=None, carry=None, stream=None):
        """The block step with its eviction left pending; `carry` is another KeyDiffCache whose
        pending eviction this call takes along."""
        Bt, out = self._block_args(q, k_new, v_new, out, None)
        _check(self._L.keydiff_prefill_block_deferred(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), Bt,
                                                      int(pos0), out.data_ptr(),
                                                      carry._h if carry is not None else None, _stream_ptr(stream)))
        return out

    def finish(self, stream=None):
        _check(self._L.keydiff_finish(self._h, _stream_ptr(stream)))

    def decode_step(self, q, k_new, v_new, pos: int, out=None, stream=None):
        Bt, out = self._block_args(q, k_new, v_new, out, None)
        if Bt != 1:
            raise ValueError("decode_step takes one token per sequence")
        _check(self._L.keydiff_decode_step(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), int(pos),
                                           out.data_ptr(), _stream_ptr(stream)))
        return out

    def scores(self, stream=None):
        import torch
        out = torch.empty((self.cfg.batch, self.cfg.n_kv_heads, self.len), dtype=torch.float32, device=self.device)
        _check(self._L.keydiff_scores(self._h, out.data_ptr(), _stream_ptr(stream)))
        return out

    @property
    def len(self) -> int:
        n = C.c_int32()
        _check(self._L.keydiff_cache_len(self._h, C.byref(n)))
        return n.value

    def plan(self):
        """(key ranges, row tiles per head, key tiles, passengers: bit 0 a selection, bit 1 a row shift; bit 2: the step
        shared its launches with those of other layers) of the last block step."""
        out = (C.c_int32 * 4)()
        _check(self._L.keydiff_cache_plan(self._h, out))
        return tuple(out)

    def positions(self, stream=None):
        import torch
        out = torch.empty((self.cfg.batch, self.cfg.n_kv_heads, self.len), dtype=torch.int32, device=self.device)
        if self.len:
            _check(self._L.keydiff_cache_positions(self._h, out.data_ptr(), _stream_ptr(stream)))
        return out

    def load(self, k, v, pos, stream=None):
        ln = check_load_shapes(self.cfg, self.cap, k, v, pos)
        if not (k.device == v.device == pos.device == self.device):
            raise ValueError("k, v and pos must live on the cache's device")
        _check(self._L.keydiff_cache_load(self._h, k.data_ptr(), v.data_ptr(), pos.data_ptr(), ln,
                                          _stream_ptr(stream)))

    def status(self, stream=None) -> int:
        s = C.c_int32()
        _check(self._L.keydiff_cache_status(self._h, C.byref(s), _stream_ptr(stream)))
        return s.value

    def profile_enable(self, on: bool):
        _check(self._L.keydiff_profile_enable(self._h, int(on)))

    def profile_read(self):
        ms = (C.c_float * len(KERNEL_NAMES))()
        cnt = (C.c_int32 * len(KERNEL_NAMES))()
        _check(self._L.keydiff_profile_read(self._h, ms, cnt))
        return {n: (ms[i], cnt[i]) for i, n in enumerate(KERNEL_NAMES)}

    # -- views of the caller-owned buffers (tests, not the hot path) -------------
    def key_rows(self):
        """Cache keys as a [batch][Hkv][cap][d] bf16 view (rows >= len are stale)."""
        import torch
        c = self.cfg
        n = c.batch * c.n_kv_heads * self.cap * c.head_dim
        return self._k[:n * 2].view(torch.bfloat16).view(c.batch, c.n_kv_heads, self.cap, c.head_dim)

    def value_rows(self):
        import torch
        c = self.cfg
        n = c.batch * c.n_kv_heads * self.cap * c.head_dim
        return self._v[:n * 2].view(torch.bfloat16).view(c.batch, c.n_kv_heads, self.cap, c.head_dim)
