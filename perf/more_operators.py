"""Timed cases of the operators that keep the own rows of continuations, which lie in pages, within a budget: attention of pieces of many tokens,
the attention weight that every row has gathered, and the eviction of the rows that gathered least.

Three kinds of case:

  chunk    branch_chunk_attention: attention of up to `Bt` new tokens of each of `prompts` x `fan` sequences over the N rows of their
           prompt's cache and over the rows in the sequence's own pages (N 0: own rows alone), with the logarithms of the weight sums
  weights  branch_weights: for every own row and KV head the attention weight that the last `observe` new tokens give it, added to what it had
  evict    branch_evict: sequences with more than `budget` rows keep those of the largest weights; rows behind the budget that
           are kept move to the places of evicted ones, with their weights and positions

`own` false: the operators in elementary torch operations.
"""
import math

import torch

own = False

# (n_q_heads, n_kv_heads, head_dim) of the workloads in synth/configs.py and of the shapes the tests use
HEADS = {"toy": (4, 1, 64), "llama32_3b": (24, 8, 128), "llama31_8b": (32, 8, 128), "qwen25_7b": (28, 4, 128),
         "six_two": (6, 2, 128), "eight_two": (8, 2, 64)}
MOST_PAIRS = 1.0e9   # (query row, key) pairs of the largest case


def _chunk(name, heads, prompts, fan, N, Bt, longest, page, ragged=False):
    return {"name": name, "kind": "chunk", "heads": heads, "prompts": prompts, "fan": fan, "N": N, "Bt": Bt, "longest": longest, "page": page,
            "ragged": ragged}


def _weighted(name, heads, seqs, Bt, longest, page, observe=0, decay=1.0, ragged=False):
    return {"name": name, "kind": "weights", "heads": heads, "seqs": seqs, "Bt": Bt, "longest": longest, "page": page, "observe": observe,
            "decay": decay, "ragged": ragged}


def _evict(name, heads, seqs, Bt, held, budget, page, window=0, ragged=False):
    return {"name": name, "kind": "evict", "heads": heads, "seqs": seqs, "Bt": Bt, "held": held, "budget": budget, "page": page,
            "window": window, "ragged": ragged}


def listed():
    return [
        # a short turn in each of three short dialogues: latency counts; small heads
        _chunk("chunk_turn_64", "eight_two", 3, 1, 0, 33, 61, 8),
        # one block of the headline workload's size over rows in pages
        _chunk("chunk_block_8b", "llama31_8b", 1, 1, 0, 128, 8192, 64),
        # tools' answers of up to 300 tokens to 24 samples of one prompt
        _chunk("chunk_pieces_ragged_3b", "llama32_3b", 1, 24, 4096, 300, 700, 32, ragged=True),
        # four prompts from their first token on, seven query heads to a KV head
        _chunk("chunk_first_7b", "qwen25_7b", 4, 1, 0, 1000, 0, 16),
        # a long prompt in pieces of 2048 tokens, far along
        _chunk("chunk_prompt_8b", "llama31_8b", 1, 1, 0, 2048, 14336, 64),
        # a generated token in short dialogues
        _weighted("weights_token_64", "eight_two", 3, 1, 61, 8),
        # a generated token of each of 64 long answers: the keys stream from HBM
        _weighted("weights_token_8b", "llama31_8b", 64, 1, 4096, 64),
        # pieces of up to 300 tokens, older weights forgotten slowly
        _weighted("weights_pieces_ragged_3b", "llama32_3b", 8, 300, 4000, 32, decay=0.9, ragged=True),
        # a long prompt whose last 32 tokens say what to keep
        _weighted("weights_window_8b", "llama31_8b", 1, 2048, 14336, 64, observe=32),
        # short dialogues at their budget, a token each
        _evict("evict_token_64", "eight_two", 3, 1, 96, 96, 8),
        # 64 long answers at their budget, a token each
        _evict("evict_token_8b", "llama31_8b", 64, 1, 2048, 2048, 64, window=64),
        # four long prompts cut down to a budget at once, the latest tokens kept
        _evict("evict_prompt_7b", "qwen25_7b", 4, 2048, 14336, 4096, 64, window=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "weights", "evict"])
    heads = rng.choice(sorted(HEADS))
    hq, hkv, d = HEADS[heads]
    page, ragged = rng.choice([8, 16, 32, 64, 128, 256]), rng.random() < 0.5
    if kind == "chunk":
        prompts = rng.choice([1, 1, 2, 3])
        fan = max(1, _log(rng, 1, 32) // prompts)
        N = 0 if rng.random() < 0.5 else _log(rng, 40, 8192)
        Bt, longest = _log(rng, 1, 2048), rng.choice([0, _log(rng, 1, 14336), _log(rng, 1, 14336)])
        while prompts * fan * hq * Bt * (N + longest + Bt) > MOST_PAIRS or prompts * fan * (longest + Bt) > 200000:
            fan, Bt, longest, N = max(1, fan * 3 // 4), max(1, Bt * 3 // 4), longest * 3 // 4, N * 3 // 4
        return {"kind": kind, "heads": heads, "prompts": prompts, "fan": fan, "N": N, "Bt": Bt, "longest": longest, "page": page, "ragged": ragged}
    seqs = _log(rng, 1, 64)
    if kind == "weights":
        Bt, longest = rng.choice([1, 1, _log(rng, 2, 2048)]), _log(rng, 1, 14336)
        while seqs * hq * Bt * (longest + Bt) > MOST_PAIRS or seqs * (longest + Bt) > 260000:
            seqs, Bt, longest = max(1, seqs * 3 // 4), max(1, Bt * 3 // 4), longest * 3 // 4
        return {"kind": kind, "heads": heads, "seqs": seqs, "Bt": Bt, "longest": longest, "page": page, "observe": rng.choice([0, 0, 1, 32]),
                "decay": rng.choice([1.0, 1.0, 0.9, 0.0]), "ragged": ragged}
    Bt, held = rng.choice([1, rng.randint(2, 8), _log(rng, 9, 2048)]), _log(rng, 1, 14336)
    while seqs * (held + Bt) > 140000:
        seqs, held = max(1, seqs * 3 // 4), held * 3 // 4
    budget = max(1, rng.choice([held, held, int(held * rng.uniform(0.1, 1.0))]))
    return {"kind": kind, "heads": heads, "seqs": seqs, "Bt": Bt, "held": held, "budget": budget, "page": page,
            "window": rng.choice([0, budget // 8, min(64, budget - 1)]), "ragged": ragged}


# ------------------------------------------------------------------------------------------------ inputs
def _spread(i):
    return (i * 0.6180339887498949 + 0.37) % 1.0


def _lengths(case):
    """Rows that the sequences hold: chunk and weights: up to `longest`, spread over the range, the first as long as any; evict: `held`, or ragged
    anything up to it."""
    if case["kind"] == "evict":
        return [case["held"] if i == 0 or not case["ragged"] else int(case["held"] * _spread(i)) for i in range(case["seqs"])]
    n = case["prompts"] * case["fan"] if case["kind"] == "chunk" else case["seqs"]
    return [case["longest"] if i == 0 else int(case["longest"] * _spread(i)) for i in range(n)]


def _new_rows(case, n):
    """New tokens of every sequence: Bt of each, or up to Bt and none of some."""
    Bt = case["Bt"]
    return [Bt if i == 0 or not case["ragged"] else int(round(Bt * ((i * 0.7548776662466927 + 0.5) % 1.0))) for i in range(n)]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    return dict(generator=g, device="cuda")


def _paged(lens, extra, page, g):
    """A page table for sequences of lens[i] + extra rows, pages in any order and a few unused; the number of pages."""
    need = [max(1, -(-(n + extra) // page)) for n in lens]
    width, pages = max(need), sum(need) + 3
    order = torch.randperm(pages, **g).to(torch.int32).cpu()
    table, at = torch.zeros((len(lens), width), dtype=torch.int32), 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table.cuda(), pages


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def prepare(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    g = _generator(seed)
    Bt, page = case["Bt"], case["page"]
    lens = _lengths(case)
    n = len(lens)
    new = _new_rows(case, n)
    st = {"case": case, "lens": _ints(lens), "n_new": _ints(new) if case["ragged"] else None}
    st["table"], pages = _paged(lens, Bt, page, g)
    # keys of a head share an offset, two in a hundred are outliers (the recipe of synth/generate.py); queries lean to it
    offset = torch.randn((1, hkv, 1, d), **g) * math.sqrt(2.0)

    def keys(*shape):
        k = torch.randn(shape + (d,), **g).add_(offset)
        return k.mul_(torch.where(torch.rand(shape + (1,), **g) < 0.02, 4.0, 1.0)).bfloat16()

    st["k_pages"] = keys(pages, hkv, page)
    if case["kind"] != "weights":
        st["v_pages"] = torch.randn((pages, hkv, page, d), **g).bfloat16()
    if case["kind"] == "evict":
        # weights gathered so far: a few rows have most, some have none; positions of rows that earlier evictions left, in the order they left them
        first = [(i * 911 + 37) % 4096 for i in range(n)]
        first = [f + 1 if (f + m) % 7919 == 0 else f for f, m in zip(first, lens)]
        st["pos0"] = _ints(first)
        w = torch.exp(2.0 * torch.randn((pages, hkv, page), **g))
        st["w_pages"] = torch.where(torch.rand((pages, hkv, page), **g) < 0.05, 0.0, w)
        p = torch.zeros((pages, hkv, page), dtype=torch.int32, device="cuda")
        head = torch.arange(hkv, device="cuda")[:, None]
        for s, (f, m) in enumerate(zip(first, lens)):
            r = torch.arange(m, device="cuda")
            p[st["table"][s, r // page].long()[None], head, (r % page)[None]] = ((r[None] * 7919 + 131 * head) % max(f + m, 1)).to(torch.int32)
        st["p_pages"] = p
        return st
    lean = 0.5 * offset.repeat_interleave(hq // hkv, dim=1)
    st["q"] = torch.randn((n, hq, Bt, d), **g).add_(lean).bfloat16()
    if case["kind"] == "chunk":
        N = case["N"]
        st["k_prefix"] = keys(case["prompts"], hkv, N) if N else None
        st["v_prefix"] = torch.randn((case["prompts"], hkv, N, d), **g).bfloat16() if N else None
        # (rows behind a sequence's new tokens are left as they are)
        st["out"] = torch.zeros((n, hq, Bt, d), dtype=torch.bfloat16, device="cuda")
        st["lse"] = torch.zeros((n, hq, Bt), device="cuda")
    else:
        st["w_pages"] = torch.rand((pages, hkv, page), **g)
        # as attention over a prompt's rows and these leaves them: the prompt takes some part of every query's weight
        s = _own_logits(st, st["q"], torch.arange(Bt, device="cuda")[None].expand(n, -1))
        own_sum = torch.logsumexp(s, dim=-1)
        st["lse"] = torch.logaddexp(own_sum, own_sum + torch.randn(own_sum.shape, **g)).view(n, hq, Bt)
        behind = torch.arange(Bt, device="cuda")[None, None] >= torch.tensor(new, device="cuda")[:, None, None]
        st["lse"] = torch.where(behind, 0.0, st["lse"]).contiguous()
    return st


# ------------------------------------------------------------------------------------------------ the plain forms
def _dense(pages, table):
    """What sequences hold in pages [pages][hkv][page_rows]...: [n][hkv][rows]..."""
    x = pages[table.long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], x.shape[2] * x.shape[3], *x.shape[4:])


def _own_logits(st, q, j):
    """Logits of new tokens, q [n][heads][tokens][d] with their numbers j [n][tokens], against their sequences' own rows in 32 bits; minus infinity
    where a row is not seen."""
    lens = st["lens"].long()
    n, hq, T, d = q.shape
    k = _dense(st["k_pages"], st["table"]).float()
    hkv, L = k.shape[1], k.shape[2]
    G = hq // hkv
    x = q.float().view(n, hkv, G * T, d) * (1.0 / math.sqrt(d))
    s = torch.matmul(x, k.transpose(2, 3).contiguous()).view(n, hkv, G, T, L)
    seen = torch.arange(L, device="cuda")[None, None] < (lens[:, None] + 1 + j)[:, :, None]                    # [n][tokens][L]
    return torch.where(seen[:, None, None], s, float("-inf"))


def _chunk_plain(st):
    q = st["q"]
    n, hq, Bt, d = q.shape
    _, fresh, _ = _counts(st)
    j = torch.arange(Bt, device="cuda")[None].expand(n, -1)
    new = j < fresh[:, None]
    s1 = _own_logits(st, q, j)
    hkv, G, L = s1.shape[1], s1.shape[2], s1.shape[4]
    top = s1.amax(-1)
    N = st["case"]["N"]
    if N:
        p = st["case"]["prompts"]
        fan = n // p
        x = (q.float() * (1.0 / math.sqrt(d))).view(p, fan, hkv, G * Bt, d).transpose(1, 2).reshape(p, hkv, fan * G * Bt, d)
        s0 = torch.matmul(x, st["k_prefix"].float().transpose(2, 3).contiguous())
        s0 = s0.view(p, hkv, fan, G, Bt, N).transpose(1, 2).reshape(n, hkv, G, Bt, N)
        top = torch.maximum(top, s0.amax(-1))
    e1 = torch.exp(s1 - top[..., None])
    total = e1.sum(-1)
    o = torch.matmul(e1.view(n, hkv, G * Bt, L), _dense(st["v_pages"], st["table"]).float()).view(n, hkv, G, Bt, d)
    if N:
        e0 = torch.exp(s0 - top[..., None])
        total = total + e0.sum(-1)
        e0 = e0.view(p, fan, hkv, G * Bt, N).transpose(1, 2).reshape(p, hkv, fan * G * Bt, N)
        o0 = torch.matmul(e0, st["v_prefix"].float()).view(p, hkv, fan, G, Bt, d).transpose(1, 2).reshape(n, hkv, G, Bt, d)
        o = o + o0
    o = (o / total[..., None]).view(n, hq, Bt, d).bfloat16()
    lse = (top + torch.log(total)).view(n, hq, Bt)
    st["out"].copy_(torch.where(new[:, None, :, None], o, st["out"]))
    st["lse"].copy_(torch.where(new[:, None], lse, st["lse"]))
    return st["out"], st["lse"]


def _rows_of_tables(st):
    """(page, row in the page) of every row that the tables can name, [n][rows]; numbers of the rows."""
    page = st["case"]["page"]
    r = torch.arange(st["table"].shape[1] * page, device="cuda")
    return st["table"].long()[:, r // page], (r % page).expand(st["table"].shape[0], -1), r


def _counts(st):
    """Rows held, new rows, both together, [n] each."""
    lens = st["lens"].long()
    new = st["n_new"].long() if st["n_new"] is not None else torch.full_like(lens, st["case"]["Bt"])
    return lens, new, lens + new


def _weights_plain(st):
    q, lse, observe = st["q"], st["lse"], min(st["case"]["observe"] or st["case"]["Bt"], st["case"]["Bt"])
    lens, fresh, upto = _counts(st)
    j = (fresh - observe).clamp(min=0)[:, None] + torch.arange(observe, device="cuda")[None]                  # [n][observe]
    new = j < fresh[:, None]
    if observe < q.shape[2]:
        at = j.clamp(max=q.shape[2] - 1)[:, None].expand(-1, q.shape[1], -1)
        lse = torch.gather(lse, 2, at)
        q = torch.gather(q, 2, at[..., None].expand(-1, -1, -1, q.shape[3]))
    s = _own_logits(st, q, j)
    n, hkv, G = s.shape[:3]
    p = torch.exp(s - lse.reshape(n, hkv, G, observe, 1))
    gathered = torch.where(new[:, None, None, :, None], p, 0.0).sum((2, 3))                                 # [n][hkv][rows]
    page, row, r = _rows_of_tables(st)
    w = _dense(st["w_pages"], st["table"])
    w = torch.where((r[None] < lens[:, None])[:, None], st["case"]["decay"] * w, 0.0) + gathered
    put = (r[None] < upto[:, None]) & (fresh > 0)[:, None]
    st["w_pages"][page[put], :, row[put]] = w.transpose(1, 2)[put]
    return st["w_pages"]


def _evict_plain(st):
    budget, window = st["case"]["budget"], st["case"]["window"]
    lens, _, upto = _counts(st)
    page, row, r = _rows_of_tables(st)
    n, L = page.shape
    hkv = st["k_pages"].shape[1]
    pos0 = st["pos0"].long()
    # the positions of the new rows
    fresh = (r[None] >= lens[:, None]) & (r[None] < upto[:, None])
    st["p_pages"][page[fresh], :, row[fresh]] = (pos0[:, None] + r[None])[fresh].to(torch.int32)[:, None].expand(-1, hkv)
    w, p = _dense(st["w_pages"], st["table"]), _dense(st["p_pages"], st["table"]).long()
    held = (r[None] < upto[:, None])[:, None].expand(-1, hkv, -1)
    # the order in which rows are kept: the latest `window` positions, then by weight; of equal ones the lower position first
    order = torch.sort(torch.where(held, p, 1 << 40), dim=-1, stable=True).indices
    for key in (w, (p >= (pos0 + upto - window)[:, None, None]).float(), held.float()):
        order = torch.gather(order, -1, torch.sort(torch.gather(key, -1, order), dim=-1, descending=True, stable=True).indices)
    kept = torch.zeros_like(held).scatter_(-1, order, (torch.arange(L, device="cuda") < budget).expand(n, hkv, L)) & held
    movers, holes = kept & (r >= budget), ~kept & held & (r < budget)
    source = torch.sort(torch.where(movers, r, 1 << 40), dim=-1).values
    target = torch.sort(torch.where(holes, r, 1 << 40), dim=-1).values
    s, h, i = torch.nonzero(source < (1 << 40), as_tuple=True)
    a, b = source[s, h, i], target[s, h, i]
    for x in (st["k_pages"], st["v_pages"], st["w_pages"], st["p_pages"]):
        x[page[s, b], h, row[s, b]] = x[page[s, a], h, row[s, a]]
    return st["k_pages"], st["v_pages"], st["w_pages"], st["p_pages"]


def run(st):
    case = st["case"]
    if own:
        import paper_2504_15364_amd as kd
        if case["kind"] == "chunk":
            prefix = (st["k_prefix"], st["v_prefix"], case["N"]) if case["N"] else None
            return kd.branch_chunk_attention(st["q"], st["k_pages"], st["v_pages"], st["table"], st["lens"], prefix=prefix, n_new=st["n_new"],
                                             out=st["out"], lse=st["lse"])
        if case["kind"] == "weights":
            kd.branch_weights(st["q"], st["k_pages"], st["w_pages"], st["table"], st["lens"], st["lse"], n_new=st["n_new"],
                              observe=case["observe"], decay=case["decay"])
            return st["w_pages"]
        kd.branch_evict(st["k_pages"], st["v_pages"], st["w_pages"], st["p_pages"], st["table"], st["lens"], case["budget"], Bt=case["Bt"],
                        n_new=st["n_new"], pos0=st["pos0"], window=case["window"])
        return st["k_pages"], st["v_pages"], st["w_pages"], st["p_pages"]
    return {"chunk": _chunk_plain, "weights": _weights_plain, "evict": _evict_plain}[case["kind"]](st)


def work(case):
    hq, hkv, d = HEADS[case["heads"]]
    lens = _lengths(case)
    new = _new_rows(case, len(lens))
    if case["kind"] == "evict":
        size = 0
        for n, m in zip(lens, new):
            # weights and positions once; of the rows behind the budget that part is kept which the budget is of all
            # (of weights without an order: inputs as prepare gives them)
            over = max(0, n + m - case["budget"])
            size += (n + m) * 8 if over else m * 4
            if over:
                size += 2 * (4 * d + 8) * max(over * case["budget"] // (n + m), min(over, case["window"]))
        return {"bytes": size * hkv, "flops": 0}
    if case["kind"] == "chunk":
        rows = case["prompts"] * case["N"] + sum(n + m for n, m in zip(lens, new) if m)
        pairs = sum(m * (case["N"] + n) + m * (m + 1) // 2 for n, m in zip(lens, new))
        return {"bytes": rows * hkv * d * 4 + sum(new) * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}
    observe = [min(m, case["observe"]) if case["observe"] else m for m in new]
    rows = sum(n + m for n, m in zip(lens, new) if m)
    pairs = sum(o * (n + m - o) + o * (o + 1) // 2 for n, m, o in zip(lens, new, observe))
    return {"bytes": rows * hkv * (d * 2 + 8) + sum(observe) * hq * (2 * d + 4), "flops": 2 * d * hq * pairs}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _sequence_rows(pool, st, s, n):
    r = torch.arange(n, device="cuda")
    page = st["case"]["page"]
    return pool[st["table"][s, r // page].long(), :, r % page].transpose(0, 1)                              # [hkv][n]...


def _evict_exact(st):
    """Sequence by sequence and head by head: which rows stay, and where they go."""
    import numpy as np
    case = st["case"]
    budget, page = case["budget"], case["page"]
    k, v, w, p = (st[x].clone() for x in ("k_pages", "v_pages", "w_pages", "p_pages"))
    w_host, p_host, table = w.cpu().numpy(), p.cpu().numpy(), st["table"].cpu().numpy()
    pos0 = st["pos0"].tolist()
    lens = _lengths(case)
    moves = []
    for s, (held, new) in enumerate(zip(lens, _new_rows(case, len(lens)))):
        r = np.arange(held + new)
        at, row = table[s, r // page], r % page
        for h in range(w_host.shape[1]):
            p_host[at[held:], h, row[held:]] = pos0[s] + r[held:]
            if len(r) <= budget:
                continue
            weight, position = w_host[at, h, row], p_host[at, h, row]
            late = position >= pos0[s] + len(r) - case["window"]
            stays = np.zeros(len(r), dtype=bool)
            stays[np.lexsort((r, position, -weight, ~late))[:budget]] = True
            to, fro = np.flatnonzero(~stays[:budget]), budget + np.flatnonzero(stays[budget:])
            moves.append(np.stack([at[to], np.full(len(to), h), row[to], at[fro], np.full(len(to), h), row[fro]]))
    p.copy_(torch.from_numpy(p_host))
    if moves:
        m = torch.from_numpy(np.concatenate(moves, axis=1).astype(np.int64)).cuda()
        for x in (k, v, w, p):
            x[m[0], m[1], m[2]] = x[m[3], m[4], m[5]]
    return k.double(), v.double(), w.double(), p


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "evict":
        return _evict_exact(st)
    hq, hkv, d = HEADS[case["heads"]]
    G, lens = hq // hkv, _lengths(case)
    news = _new_rows(case, len(lens))
    if case["kind"] == "chunk":
        out, lse, N = st["out"].double(), st["lse"].double(), case["N"]
    else:
        weights = st["w_pages"].double()
    for s, (held, new) in enumerate(zip(lens, news)):
        if not new:
            continue
        k = _sequence_rows(st["k_pages"], st, s, held + new).double()
        if case["kind"] == "chunk":
            v = _sequence_rows(st["v_pages"], st, s, held + new).double()
            if N:
                b = s // case["fan"]
                k, v = torch.cat([st["k_prefix"][b].double(), k], 1), torch.cat([st["v_prefix"][b].double(), v], 1)
        else:
            gathered = torch.zeros(k.shape[:2], dtype=torch.float64, device="cuda")
        before = k.shape[1] - new
        for at in range(0, new, 256):                                             # 256 tokens at a time
            j = torch.arange(at, min(at + 256, new), device="cuda")
            logits = torch.matmul(st["q"][s, :, at:at + len(j)].double().view(hkv, G * len(j), d), k.transpose(1, 2).contiguous())
            logits = logits.view(hkv, G, len(j), -1) / math.sqrt(d)
            hidden = torch.arange(k.shape[1], device="cuda")[None] > (before + j)[:, None]
            logits.masked_fill_(hidden[None, None], float("-inf"))
            if case["kind"] == "chunk":
                total = torch.logsumexp(logits, -1)
                lse[s, :, at:at + len(j)] = total.view(hq, len(j))
                weight = (logits - total[..., None]).exp()
                out[s, :, at:at + len(j)] = torch.matmul(weight.view(hkv, G * len(j), -1), v).view(hq, len(j), d)
            else:
                counted = j >= new - case["observe"] if case["observe"] else j >= 0
                part = (logits - st["lse"][s, :, at:at + len(j)].double().view(hkv, G, len(j), 1)).exp()
                gathered += (part * counted[None, None, :, None]).sum((1, 2))
        if case["kind"] == "weights":
            r = torch.arange(held + new, device="cuda")
            number, row = st["table"][s, r // case["page"]].long(), r % case["page"]
            old = weights[number, :, row].t() * case["decay"]
            weights[number, :, row] = (torch.where(r[None] < held, old, 0.0) + gathered).t()
    return (out, lse) if case["kind"] == "chunk" else weights
