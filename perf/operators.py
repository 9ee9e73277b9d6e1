"""Timed cases of the operators around the block step: what a program that serves a model with a KeyDiff cache has them do
before the step (the norms of queries and keys and the rotation) and behind it (several continuations of a prompt, each with
rows of its own in pages, that share the prompt's cache).

Three kinds of case:

  norm_rope  norm_rope: root mean square norms of the queries and keys of each head with learned weights, and the rotary
             position embedding, in one pass over the projections' outputs
  append     branch_append: the same on new tokens of many sequences, the keys and values written into the pages of the
             sequences, the queries returned
  attention  branch_attention: attention of the new tokens of `prompts` x `fan` sequences over the N rows of their prompt's
             cache, which the `fan` sequences of a prompt share, and over the rows in the sequence's own pages

`own` false: the operators in elementary torch operations.
"""
import math

import torch

own = False

# (n_q_heads, n_kv_heads, head_dim) of the workloads in synth/configs.py and of the shapes the tests use
HEADS = {"toy": (4, 1, 64), "llama32_3b": (24, 8, 128), "llama31_8b": (32, 8, 128), "qwen25_7b": (28, 4, 128),
         "six_two": (6, 2, 128), "eight_two": (8, 2, 64)}
THETA = 500000.0
EPS = 1e-6
POSITIONS = 40960   # rows of the rotary tables


def _norm_rope(name, heads, batch, T, norm="shared", rope=True, fused=True, ragged=False):
    return {"name": name, "kind": "norm_rope", "heads": heads, "batch": batch, "T": T, "norm": norm, "rope": rope,
            "fused": fused, "ragged": ragged}


def _append(name, heads, seqs, Bt, longest, page, norm="shared", rope=True, ragged=False):
    return {"name": name, "kind": "append", "heads": heads, "seqs": seqs, "Bt": Bt, "longest": longest, "page": page,
            "norm": norm, "rope": rope, "ragged": ragged}


def _attention(name, heads, prompts, fan, N, longest, page, Bt=1):
    return {"name": name, "kind": "attention", "heads": heads, "prompts": prompts, "fan": fan, "N": N, "longest": longest,
            "page": page, "Bt": Bt}


def listed():
    return [
        # generation for one sequence: a launch and its latency
        _norm_rope("norm_rope_one_token", "qwen25_7b", 1, 1),
        # several short prompts of different lengths at once, weights of their own for every head, head_dim 64
        _norm_rope("norm_rope_ragged_64", "eight_two", 5, 1001, norm="heads", ragged=True),
        # a whole prompt of the headline workload ahead of its blocks, from the fused projection's output
        _norm_rope("norm_rope_prompt_8b", "llama31_8b", 1, 32768),
        # one token of one sequence into its page
        _append("append_one", "llama32_3b", 1, 1, 500, 16),
        # one token of each of 64 continuations of a prompt
        _append("append_decode_64", "llama31_8b", 64, 1, 2000, 64),
        # pieces of up to 300 given tokens for each of 24 sequences (a tool's answer, the next turn of a dialogue)
        _append("append_pieces_ragged", "llama32_3b", 24, 300, 700, 32, ragged=True),
        # one answer to one prompt, a few hundred tokens long: the cache dominates, latency counts
        _attention("attention_one_8b", "llama31_8b", 1, 1, 8192, 300, 64),
        # 16 samples of one prompt
        _attention("attention_16_samples_8b", "llama31_8b", 1, 16, 8192, 777, 64),
        # 64 samples with long answers: the sequences' own rows stream from HBM
        _attention("attention_64_long_8b", "llama31_8b", 1, 64, 8192, 4096, 64),
        # four prompts with eight beams each, four drafted tokens a beam checked at once, seven query heads to a KV head
        _attention("attention_beams_drafts_7b", "qwen25_7b", 4, 8, 4096, 201, 16, Bt=4),
        # 256 samples that have just begun: the shared rows are nearly all the work
        _attention("attention_256_begun_3b", "llama32_3b", 1, 256, 8192, 33, 16),
        # small heads, short caches
        _attention("attention_small_64", "eight_two", 3, 3, 250, 61, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "attention", "attention"])
    heads = rng.choice(sorted(HEADS))
    norm, rope = rng.choice(["shared", "shared", "heads", "none"]), rng.random() < 0.85
    rope = rope or norm == "none"
    if kind == "norm_rope":
        batch = _log(rng, 1, 8)
        return {"kind": kind, "heads": heads, "batch": batch, "T": max(1, _log(rng, 1, 20000) // batch), "norm": norm, "rope": rope,
                "fused": rng.random() < 0.7, "ragged": rng.random() < 0.4}
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if kind == "append":
        seqs, ragged = _log(rng, 1, 200), rng.random() < 0.5
        Bt = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 500)])
        return {"kind": kind, "heads": heads, "seqs": seqs, "Bt": max(1, min(Bt, 8000 // seqs)), "longest": _log(rng, 1, 1500), "page": page,
                "norm": norm, "rope": rope, "ragged": ragged}
    prompts = rng.choice([1, 1, 1, 2, 3, 4])
    fan = max(1, _log(rng, 1, 200) // prompts)
    N, Bt = _log(rng, 40, 12288), rng.choice([1, 1, 1, rng.randint(2, 8)])
    longest = _log(rng, 1, 4000)
    while prompts * fan * longest > 200000:
        longest //= 2
    while prompts * fan * Bt * (N + longest) > 2500000:
        Bt, N = max(1, Bt // 2), N * 3 // 4
    return {"kind": kind, "heads": heads, "prompts": prompts, "fan": fan, "N": N, "longest": longest, "page": page, "Bt": Bt}


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(count, longest):
    """Rows that `count` sequences hold, up to `longest`: spread over the range, the first as long as any, the last without one."""
    if count == 1:
        return [longest]
    return [longest] + [int(longest * ((i * 0.6180339887498949 + 0.37) % 1.0)) for i in range(1, count - 1)] + [0]


def _new_rows(case):
    """New tokens of every sequence of an append: as many of each, or up to Bt and none of some."""
    n, Bt = case["seqs"], case["Bt"]
    return [Bt if i == 0 or not case["ragged"] else int(round(Bt * ((i * 0.7548776662466927 + 0.5) % 1.0))) for i in range(n)]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    return dict(generator=g, device="cuda")


def _tables(d):
    inv = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    ang = torch.arange(POSITIONS, dtype=torch.float64, device="cuda")[:, None] * inv[None]
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def _weights(kind, heads, d, g):
    if kind == "none":
        return None
    shape = (d,) if kind == "shared" else (heads, d)
    return (1.0 + 0.3 * torch.randn(shape, **g)).bfloat16()


def _projections(batch, T, hq, hkv, d, g, fused):
    """q, k, v of T tokens as views [batch][heads][T][d]: parts of one projection's output, or tensors of their own."""
    if fused:
        x = torch.randn((batch, T, hq + 2 * hkv, d), **g).mul_(2.0).bfloat16().transpose(1, 2)
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return tuple(torch.randn((batch, h, T, d), **g).mul_(2.0).bfloat16() for h in (hq, hkv, hkv))


def _paged(lens, extra, page, g):
    """A page table for sequences of lens[i] + extra rows, pages in any order and a few unused; the number of pages."""
    need = [-(-(n + extra) // page) for n in lens]
    width, pages = max(max(need), 1), sum(need) + 3
    order = torch.randperm(pages, **g).to(torch.int32)
    table, at = torch.zeros((len(lens), width), dtype=torch.int32), 0
    order = order.cpu()
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table.cuda(), pages


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def prepare(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    g = _generator(seed)
    st = {"case": case}
    if case["kind"] == "norm_rope":
        b, T = case["batch"], case["T"]
        st["q"], st["k"], _ = _projections(b, T, hq, hkv, d, g, case["fused"])
        # ragged: every sequence goes on where it stopped; else a prompt from its first token on
        first = [(i * 911 + 37) % 4096 for i in range(b)] if case["ragged"] else [0] * b
        st["positions"] = _ints(first)[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")[None] if case["ragged"] else None
    elif case["kind"] == "append":
        n, Bt = case["seqs"], case["Bt"]
        st["q"], st["k"], st["v"] = _projections(n, Bt, hq, hkv, d, g, True)
        lens = _lengths(n, case["longest"])
        st["table"], pages = _paged(lens, Bt, case["page"], g)
        st["lens"], st["n_new"] = _ints(lens), _ints(_new_rows(case)) if case["ragged"] else None
        st["pos0"] = _ints([(i * 911 + 1000) % 32768 for i in range(n)])
        st["k_pages"] = torch.randn((pages, hkv, case["page"], d), **g).bfloat16()
        st["v_pages"] = torch.randn((pages, hkv, case["page"], d), **g).bfloat16()
        # (rows of q_out behind a sequence's new tokens are left as they are)
        st["q_out"] = torch.zeros((n, hq, Bt, d), dtype=torch.bfloat16, device="cuda")
    else:
        p, fan, N, Bt = (case[x] for x in ("prompts", "fan", "N", "Bt"))
        # keys of a head share an offset, two in a hundred are outliers (the recipe of synth/generate.py); queries lean to it
        offset = torch.randn((1, hkv, 1, d), **g) * math.sqrt(2.0)

        def keys(*shape):
            k = torch.randn(shape + (d,), **g).add_(offset)
            return k.mul_(torch.where(torch.rand(shape + (1,), **g) < 0.02, 4.0, 1.0)).bfloat16()

        st["k_prefix"], st["v_prefix"] = keys(p, hkv, N), torch.randn((p, hkv, N, d), **g).bfloat16()
        lens = _lengths(p * fan, case["longest"])
        st["table"], pages = _paged(lens, Bt, case["page"], g)
        st["lens"] = _ints(lens)
        st["k_pages"], st["v_pages"] = keys(pages, hkv, case["page"]), torch.randn((pages, hkv, case["page"], d), **g).bfloat16()
        lean = 0.5 * offset.repeat_interleave(hq // hkv, dim=1)
        st["q"] = torch.randn((p * fan, hq, Bt, d), **g).add_(lean).bfloat16()
        return st
    st["q_weight"], st["k_weight"] = _weights(case["norm"], hq, d, g), _weights(case["norm"], hkv, d, g)
    st["cos"], st["sin"] = _tables(d) if case["rope"] else (None, None)
    return st


# ------------------------------------------------------------------------------------------------ the plain forms
def _rows_plain(x, w, cos, sin):
    """Norm and rotation of x [batch][heads][T][d] in 32 bits; cos, sin [batch][T][d / 2]."""
    x = x.float()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        x = x * (w.float() if w.dim() == 1 else w.float()[:, None, :])
    if cos is not None:
        c, s, h = cos[:, None], sin[:, None], x.shape[-1] // 2
        x = torch.cat([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], dim=-1)
    return x


def _angles(st, positions):
    if st["cos"] is None:
        return None, None
    p = positions.long()
    return st["cos"][p], st["sin"][p]


def _norm_rope_plain(st):
    q, k = st["q"], st["k"]
    positions = st["positions"]
    if positions is None:
        positions = torch.arange(q.shape[2], device="cuda")[None]
    cos, sin = _angles(st, positions)
    return _rows_plain(q, st["q_weight"], cos, sin).bfloat16(), _rows_plain(k, st["k_weight"], cos, sin).bfloat16()


def _append_plain(st):
    q, k, v, page = st["q"], st["k"], st["v"], st["case"]["page"]
    Bt = q.shape[2]
    j = torch.arange(Bt, device="cuda")[None]
    row = st["lens"].long()[:, None] + j                                     # [seqs][Bt]
    cos, sin = _angles(st, st["pos0"].long()[:, None] + row)
    k = _rows_plain(k, st["k_weight"], cos, sin).bfloat16()
    q = _rows_plain(q, st["q_weight"], cos, sin).bfloat16()
    number = torch.gather(st["table"].long(), 1, row // page)
    if st["n_new"] is None:
        st["q_out"].copy_(q)
        st["k_pages"][number, :, row % page] = k.transpose(1, 2)
        st["v_pages"][number, :, row % page] = v.transpose(1, 2)
    else:
        new = j < st["n_new"][:, None]
        st["q_out"].copy_(torch.where(new[:, None, :, None], q, st["q_out"]))
        st["k_pages"][number[new], :, (row % page)[new]] = k.transpose(1, 2)[new]
        st["v_pages"][number[new], :, (row % page)[new]] = v.transpose(1, 2)[new]
    return st["q_out"], st["k_pages"], st["v_pages"]


def _attention_plain(st):
    q = st["q"]
    n, hq, Bt, d = q.shape
    p, hkv, N, _ = st["k_prefix"].shape
    G, fan = hq // hkv, n // p
    x = q.float().view(n, hkv, G * Bt, d) * (1.0 / math.sqrt(d))
    # the rows that the sequences of a prompt share: one product for all of them
    shared = x.view(p, fan, hkv, G * Bt, d).transpose(1, 2).reshape(p, hkv, fan * G * Bt, d)
    s0 = torch.matmul(shared, st["k_prefix"].float().transpose(2, 3).contiguous())
    s0 = s0.view(p, hkv, fan, G * Bt, N).transpose(1, 2).reshape(n, hkv, G * Bt, N)

    def dense(pages):   # the sequences' own rows [n][hkv][rows][d]
        return pages[st["table"].long()].transpose(1, 2).reshape(n, hkv, -1, d).float()

    k = dense(st["k_pages"])
    L = k.shape[2]
    s1 = torch.matmul(x, k.transpose(2, 3).contiguous())
    visible = st["lens"].long()[:, None] + 1 + torch.arange(Bt, device="cuda")[None]                 # [n][Bt]
    seen = torch.arange(L, device="cuda")[None, None] < visible[:, :, None]                         # [n][Bt][L]
    s1 = torch.where(seen[:, None, None], s1.view(n, hkv, G, Bt, L), float("-inf")).view(n, hkv, G * Bt, L)
    top = torch.maximum(s0.amax(-1, keepdim=True), s1.amax(-1, keepdim=True))
    e0, e1 = torch.exp(s0 - top), torch.exp(s1 - top)
    total = e0.sum(-1, keepdim=True) + e1.sum(-1, keepdim=True)
    e0 = e0.reshape(p, fan, hkv, G * Bt, N).transpose(1, 2).reshape(p, hkv, fan * G * Bt, N)
    o = torch.matmul(e0, st["v_prefix"].float())
    o = o.view(p, hkv, fan, G * Bt, d).transpose(1, 2).reshape(n, hkv, G * Bt, d)
    o = (o + torch.matmul(e1, dense(st["v_pages"]))) / total
    return o.reshape(n, hq, Bt, d).bfloat16()


def run(st):
    kind = st["case"]["kind"]
    if own:
        import paper_2504_15364_amd as kd
        if kind == "norm_rope":
            return kd.norm_rope(st["q"], st["k"], cos=st["cos"], sin=st["sin"], positions=st["positions"],
                                q_weight=st["q_weight"], k_weight=st["k_weight"], norm_eps=EPS)
        if kind == "append":
            q = kd.branch_append(st["q"], st["k"], st["v"], st["k_pages"], st["v_pages"], st["table"], st["lens"], n_new=st["n_new"],
                                 pos0=st["pos0"], cos=st["cos"], sin=st["sin"], q_weight=st["q_weight"], k_weight=st["k_weight"],
                                 norm_eps=EPS, q_out=st["q_out"])
            return q, st["k_pages"], st["v_pages"]
        return kd.branch_attention(st["q"], st["k_pages"], st["v_pages"], st["table"], st["lens"],
                                   prefix=(st["k_prefix"], st["v_prefix"], st["case"]["N"]))
    return {"norm_rope": _norm_rope_plain, "append": _append_plain, "attention": _attention_plain}[kind](st)


def work(case):
    hq, hkv, d = HEADS[case["heads"]]
    if case["kind"] == "attention":
        n, Bt, N = case["prompts"] * case["fan"], case["Bt"], case["N"]
        lens = _lengths(n, case["longest"])
        rows = case["prompts"] * N + sum(L + Bt for L in lens)
        pairs = sum(Bt * (N + L) + Bt * (Bt + 1) // 2 for L in lens)
        return {"bytes": rows * hkv * d * 4 + 2 * n * Bt * hq * d * 2, "flops": 4 * d * hq * pairs}
    if case["kind"] == "append":
        tokens, values = sum(_new_rows(case)), hkv
    else:
        tokens, values = case["batch"] * case["T"], 0
    positions = min(tokens, POSITIONS) if case["rope"] else 0
    return {"bytes": tokens * (hq + hkv + values) * d * 4 + positions * d * 4,
            "flops": tokens * (hq + hkv) * d * ((4 if case["norm"] != "none" else 0) + (3 if case["rope"] else 0))}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _turned(x, w, angle_cos, angle_sin):
    """One row's definition for all rows x [rows][heads][d] in double: y_i = x_i w_i / rms, pairs (i, i + d/2) turned by their angle."""
    x = x.double()
    if w is not None:
        x = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()
    if angle_cos is None:
        return x
    z = torch.complex(*x.chunk(2, dim=-1)) * torch.complex(angle_cos.double(), angle_sin.double())[:, None]
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    st = prepare(case, seed)
    hq, hkv, d = HEADS[case["heads"]]
    cos, sin = st.get("cos"), st.get("sin")
    at = lambda t, p: None if t is None else t[p]  # noqa: E731
    if case["kind"] == "norm_rope":
        outs = [], []
        for b in range(case["batch"]):
            p = st["positions"][b].long() if case["ragged"] else torch.arange(case["T"], device="cuda")
            for o, x, w in zip(outs, (st["q"], st["k"]), (st["q_weight"], st["k_weight"])):
                o.append(_turned(x[b].transpose(0, 1), w, at(cos, p), at(sin, p)).transpose(0, 1))
        return tuple(torch.stack(o) for o in outs)
    page = case["page"]
    if case["kind"] == "append":
        q_out, k_pages, v_pages = st["q_out"].double(), st["k_pages"].double(), st["v_pages"].double()
        for s, new in enumerate(_new_rows(case)):
            if not new:
                continue
            rows = int(st["lens"][s]) + torch.arange(new, device="cuda")
            p = int(st["pos0"][s]) + rows
            k = _turned(st["k"][s, :, :new].transpose(0, 1), st["k_weight"], at(cos, p), at(sin, p))
            number, at_row = st["table"][s, rows // page].long(), rows % page
            k_pages[number, :, at_row] = k
            v_pages[number, :, at_row] = st["v"][s, :, :new].transpose(0, 1).double()
            q_out[s, :, :new] = _turned(st["q"][s, :, :new].transpose(0, 1), st["q_weight"], at(cos, p), at(sin, p)).transpose(0, 1)
        return q_out, k_pages, v_pages
    Bt, G = case["Bt"], hq // hkv
    out = torch.empty((case["prompts"] * case["fan"], hq, Bt, d), dtype=torch.float64, device="cuda")
    for s, L in enumerate(_lengths(case["prompts"] * case["fan"], case["longest"])):
        rows = torch.arange(L + Bt, device="cuda")
        number, b = st["table"][s, rows // page].long(), s // case["fan"]
        k = torch.cat([st["k_prefix"][b], st["k_pages"][number, :, rows % page].transpose(0, 1)], dim=1).double()
        v = torch.cat([st["v_prefix"][b], st["v_pages"][number, :, rows % page].transpose(0, 1)], dim=1).double()
        for j in range(Bt):
            n = case["N"] + L + j + 1
            logits = torch.bmm(k[:, :n], st["q"][s, :, j].double().view(hkv, G, d).transpose(1, 2).contiguous()) / math.sqrt(d)
            out[s, :, j] = torch.bmm(torch.softmax(logits, dim=1).transpose(1, 2).contiguous(), v[:, :n]).view(hq, d)
    return out
