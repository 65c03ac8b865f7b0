"""The work that users of a cache in pages have the library do, as timed cases: attention of new tokens and of prompts over
the pages, the pages' own management, and the log probabilities of the tokens that are answered.

`run` computes a case in its plain form, elementary torch operations in 32 bits, or, where `own` is true, by the library's
calls.  Sequence lengths, numbers of rows and accepted tokens belong to the case; the values and which page holds what, to
the seed.

The cache of one case: pool [layers][2 (K, V)][pages][kv heads][page size][head dim], page_table [sequences][most pages a
sequence holds] (-1 behind its last page), lens [sequences] in tokens, refs [pages] (tables that name the page) and
free_bits [pages / 32] (bit set: free).
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _token(name, batch, ctx, heads, kv_heads, head_dim, page, window=0, sinks=0, dtype="bf16"):
    return dict(name=name, op="token", batch=batch, ctx_lo=ctx[0], ctx_hi=ctx[1], rows_lo=1, rows_hi=1, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, window=window, sinks=sinks, dtype=dtype)


def _rows(name, batch, ctx, rows, heads, kv_heads, head_dim, page, window, sinks, dtype="bf16"):
    return dict(name=name, op="rows", batch=batch, ctx_lo=ctx[0], ctx_hi=ctx[1], rows_lo=rows[0], rows_hi=rows[1], heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, page=page, window=window, sinks=sinks, dtype=dtype)


def _fork(name, layers, kv_heads, head_dim, page, parents, children, ctx, dtype="bf16"):
    return dict(name=name, op="fork", layers=layers, kv_heads=kv_heads, head_dim=head_dim, page=page, parents=parents, children=children,
                ctx_lo=ctx[0], ctx_hi=ctx[1], dtype=dtype)


def _accept(name, layers, kv_heads, head_dim, page, batch, beam_width, beam_length, ctx, dtype="bf16"):
    return dict(name=name, op="accept", layers=layers, kv_heads=kv_heads, head_dim=head_dim, page=page, batch=batch, beam_width=beam_width,
                beam_length=beam_length, ctx_lo=ctx[0], ctx_hi=ctx[1], dtype=dtype)


def _logprobs(name, rows, vocab, top, temperature=1.0, dtype="fp32"):
    return dict(name=name, op="logprobs", rows=rows, vocab=vocab, top=top, temperature=temperature, dtype=dtype)


def listed():
    return [
        # one user's chat on a model of 32 heads: the new token's K and V go into the cache, its query reads it
        _token("token_one_user", 1, (900, 900), 32, 32, 128, 16),
        # sixteen users with contexts of very different lengths
        _token("token_batch16", 16, (256, 2048), 32, 32, 128, 64),
        # a busy server with grouped heads and long contexts
        _token("token_grouped_long", 32, (100, 16384), 32, 8, 128, 64),
        # long streams of which a window and the first few tokens stay visible, 40 heads
        _token("token_window", 12, (3000, 12000), 40, 40, 128, 32, window=1024, sinks=4),
        # the fp32 configuration's heads
        _token("token_fp32", 3, (40, 250), 4, 4, 64, 16, dtype="fp32"),
        # a long prompt under a window, 32 heads
        _rows("prompt_window", 1, (4096, 4096), (4096, 4096), 32, 32, 128, 64, 1024, 4),
        # the next pieces of five users' prompts, grouped heads, odd lengths
        _rows("prompt_pieces", 5, (300, 2500), (33, 700), 32, 8, 128, 32, 512, 16),
        # beam candidates branch off their parents: a small model, then 8 layers of a model of 32 heads
        _fork("fork_small", 2, 4, 64, 16, 1, 4, (64, 90), dtype="fp32"),
        _fork("fork_beams", 8, 32, 128, 64, 4, 8, (200, 700)),
        # a verification of sixteen users' beams: rows for the packed tokens, the accepted ones move up, the rest is given back
        _accept("accept_batch16", 8, 32, 128, 32, 16, 16, 5, (100, 600)),
        # the tokens of one speculative step, and every row of a batch's verification
        _logprobs("logprobs_step", 6, 32000, 5),
        _logprobs("logprobs_rows", 1296, 32000, 20, 0.8),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["token", "token", "token", "rows", "rows", "fork", "accept", "logprobs", "logprobs"])
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    page = rng.choice([16, 32, 64, 128])
    if op == "logprobs":
        rows, vocab = _log_int(rng, 1, 1296), _log_int(rng, 500, 160000)
        rows = max(1, min(rows, 1296 * 32000 // vocab))
        return _without_name(_logprobs("", rows, vocab, rng.choice([0, 1, 5, 10, 20]), rng.choice([1.0, 0.8, 1.3]),
                                       rng.choice(["fp32", "fp32", "bf16"])))
    if op in ("fork", "accept"):
        kv_heads, head_dim = rng.choice([(4, 64), (8, 128), (32, 128), (40, 128)])
        layers = _log_int(rng, 1, 8)
        batch = _log_int(rng, 1, 16)
        hi = _log_int(rng, 20, 700)
        lo = rng.randint(max(1, hi // 8), hi)
        if op == "fork":
            children = _log_int(rng, 1, 32)
            parents = min(batch, max(1, 32 // children))
            return _without_name(_fork("", layers, kv_heads, head_dim, page, parents, children, (lo, hi), dtype))
        return _without_name(_accept("", layers, kv_heads, head_dim, page, batch, _log_int(rng, 2, 16), rng.randint(2, 5), (lo, hi), dtype))
    heads, kv_heads, head_dim = rng.choice([(32, 32, 128), (40, 40, 128), (52, 52, 128), (32, 8, 128), (32, 4, 128), (16, 1, 128), (8, 8, 64)])
    window = 0 if rng.random() < 0.4 else _log_int(rng, 64, 4096)
    sinks = rng.choice([0, 1, 4, 16, 64]) if window else 0
    if op == "token":
        batch, hi = _log_int(rng, 1, 64), _log_int(rng, 1, 16384)
        size = 2 if dtype == "bf16" else 4
        while batch > 1 and batch * hi * kv_heads * head_dim * 2 * size > 1.0e9:
            batch = max(1, batch * 3 // 4)
        hi = max(1, min(hi, int(1.0e9 / (batch * kv_heads * head_dim * 2 * size))))
        lo = hi if rng.random() < 0.3 else rng.randint(max(1, hi // 8), hi)
        return _without_name(_token("", batch, (lo, hi), heads, kv_heads, head_dim, page, window, sinks, dtype))
    batch, rows = _log_int(rng, 1, 8), _log_int(rng, 17, 4096)
    ctx = min(8192, rows + (0 if rng.random() < 0.4 else _log_int(rng, 1, 4096)))
    while batch * heads * rows * ctx > 32 * 4096 * 4096:
        batch, rows, ctx = max(1, batch - 1), max(17, rows * 3 // 4), max(17, ctx * 7 // 8)
        ctx = max(ctx, rows)
    rows_lo = rows if rng.random() < 0.3 else rng.randint(max(1, rows // 8), rows)
    if dtype == "fp32":   # the fp32 configuration is a small model
        heads, kv_heads, head_dim, rows, rows_lo = 4, 4, 64, min(rows, 256), min(rows_lo, 256)
    return _without_name(_rows("", batch, (max(rows, ctx // 2), ctx), (rows_lo, rows), heads, kv_heads, head_dim, page, window, sinks, dtype))


def _without_name(case):
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ what a case's sizes say
def _plan(case):
    """Everything that does not depend on the seed: lengths, rows, accepted rows."""
    rng = np.random.default_rng([v for k, v in sorted(case.items()) if isinstance(v, int)])
    op = case["op"]
    if op in ("token", "rows"):
        lens = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, case["batch"])
        lens[0] = case["ctx_hi"]
        rows = np.minimum(rng.integers(case["rows_lo"], case["rows_hi"] + 1, case["batch"]), lens)
        return dict(lens=lens, rows=rows)
    if op == "fork":
        lens = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, case["parents"])
        return dict(lens=lens)
    if op == "accept":
        B, BW, L = case["batch"], case["beam_width"], case["beam_length"]
        lens = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, B)
        packed = rng.integers(1 + L + (BW - 1) * L // 3, 2 + BW * L, B)
        packed = np.maximum(packed, 2 * L + 1)          # accepted rows behind the first lie past where they move to
        keep = 1 + rng.integers(0, L + 1, B)
        path = np.zeros((B, L + 1), dtype=np.int64)     # packed rows of the accepted path, the root first
        for b in range(B):
            path[b, 1:] = np.sort(rng.choice(np.arange(L + 1, packed[b]), L, replace=False))
        return dict(lens=lens, packed=packed, keep=keep, path=path)
    return {}


def _pages(tokens, page):
    return -(-tokens // page)


def _visible(case, position):
    """Keys that a query at these positions sees."""
    seen = position + 1
    return np.minimum(seen, case["window"] + np.minimum(case["sinks"], np.maximum(0, seen - case["window"]))) if case["window"] else seen


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * (12 + 8 * case["top"]), "flops": 4 * n}
    plan = _plan(case)
    hd, kv = case["head_dim"], case["kv_heads"]
    token = 2 * kv * hd * size     # a token's K and V in one layer
    if case["op"] in ("token", "rows"):
        read, scores = 0, 0
        for length, rows in zip(plan["lens"].tolist(), plan["rows"].tolist()):
            scores += int(_visible(case, np.arange(length - rows, length)).sum())
            first = max(0, length - rows - case["window"] + 1) if case["window"] else 0     # the first row's window begins here
            read += length - first + min(case["sinks"], first)
        rows = int(plan["rows"].sum())
        return {"bytes": read * token + 2 * rows * token + 2 * rows * case["heads"] * hd * size, "flops": 4 * scores * case["heads"] * hd}
    if case["op"] == "fork":
        moved = case["children"] * int((plan["lens"] % case["page"]).sum())
        tables = 8 * case["children"] * int(_pages(plan["lens"], case["page"]).sum())
    else:
        moved = int((plan["keep"] - 1).sum())
        tables = 8 * int((_pages(plan["lens"] + plan["packed"], case["page"]) - _pages(plan["lens"], case["page"])).sum())
    return {"bytes": 2 * moved * token * case["layers"] + tables, "flops": 0}


# ------------------------------------------------------------------------------------------------ inputs
def _tensor(values, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(values), dtype=dtype).to(DEVICE)


def _cache(case, rng, gen, lens, rows_of_table, layers, spare):
    """A pool filled with values and the tables of sequences of these lengths, whose pages lie anywhere in it."""
    page = case["page"]
    held = _pages(lens, page)
    n_pages = int(held.sum()) + spare
    most = int(held.max()) + 1 + (spare if case["op"] in ("fork", "accept") else 0)
    order = rng.permutation(n_pages)
    table = np.full((rows_of_table, most), -1)
    refs = np.zeros(n_pages)
    at = 0
    for s, n in enumerate(held.tolist()):
        table[s, :n] = order[at:at + n]
        at += n
    refs[order[:at]] = 1
    bits = np.zeros(-(-n_pages // 32) * 32, dtype=np.uint8)
    bits[:n_pages] = refs == 0
    free = np.packbits(bits, bitorder="little").view(np.int32)
    pool = torch.empty(layers, 2, n_pages, case["kv_heads"], page, case["head_dim"], dtype=TYPES[case["dtype"]], device=DEVICE)
    for part in pool.view(layers * 2, -1):
        part.normal_(generator=gen)
    all_lens = np.zeros(rows_of_table)
    all_lens[:len(lens)] = lens
    return dict(pool=pool, page_table=_tensor(table), lens=_tensor(all_lens), refs=_tensor(refs), free_bits=_tensor(free))


def prepare(case, seed):
    rng, gen = np.random.default_rng(seed), torch.Generator(DEVICE).manual_seed(seed)
    plan, op = _plan(case), case["op"]
    if op == "logprobs":
        # logits with a few likely tokens each and a vocabulary padded with -inf; the given tokens are mostly likely ones
        rows, vocab = case["rows"], case["vocab"]
        logits = torch.randn(rows, vocab, generator=gen, device=DEVICE).mul_(2.0)
        likely = torch.randint(0, vocab - 8, (rows, 40), generator=gen, device=DEVICE)
        logits.scatter_add_(1, likely, torch.rand(rows, 40, generator=gen, device=DEVICE) * 10)
        logits[:, vocab - 8:] = -math.inf
        tokens = torch.where(torch.rand(rows, generator=gen, device=DEVICE) < 0.8, likely[:, 0],
                             torch.randint(0, vocab - 8, (rows,), generator=gen, device=DEVICE))
        return dict(case=case, logits=logits.to(TYPES[case["dtype"]]), tokens=tokens.to(torch.int32))
    if op in ("token", "rows"):
        n, total = case["batch"], int(plan["rows"].sum())
        state = _cache(case, rng, gen, plan["lens"], n, 1, 3)
        dtype = TYPES[case["dtype"]]
        state.update(case=case, most_rows=int(plan["rows"].max()), most_len=int(plan["lens"].max()),
                     row_off=_tensor(np.concatenate([[0], np.cumsum(plan["rows"])])))
        state["q"] = torch.randn(total, case["heads"], case["head_dim"], generator=gen, device=DEVICE).to(dtype)
        state["k"], state["v"] = (torch.randn(total, case["kv_heads"], case["head_dim"], generator=gen, device=DEVICE).to(dtype) for _ in range(2))
        state["out"] = torch.empty_like(state["q"])
        return state
    if op == "fork":
        P, C = case["parents"], case["children"]
        state = _cache(case, rng, gen, plan["lens"], P + P * C, case["layers"], P * C + 5)
        state.update(case=case, src=_tensor(np.repeat(np.arange(P), C)), dst=_tensor(P + np.arange(P * C)), one=_tensor(np.ones(P * C)))
        return state
    grown = int((_pages(plan["lens"] + plan["packed"], case["page"]) - _pages(plan["lens"], case["page"])).sum())
    state = _cache(case, rng, gen, plan["lens"], case["batch"], case["layers"], grown + 3)
    state.update(case=case, packed=_tensor(plan["packed"]), keep=_tensor(plan["keep"]), path=_tensor(plan["path"]),
                 none=_tensor(np.zeros(case["batch"])))
    return state


# ------------------------------------------------------------------------------------------------ the passes
def run(state):
    case = state["case"]
    return {"token": _run_attention, "rows": _run_attention, "fork": _run_fork, "accept": _run_accept,
            "logprobs": _run_logprobs}[case["op"]](state, case)


def _handle(state, case):
    """The library's handle on the state's buffers, which a program makes once and keeps."""
    if "handle" not in state:
        from paper_2403_09919_b200 import binding
        state["handle"] = binding.PagedCache(state["pool"], state["page_table"], state["lens"], state["refs"], state["free_bits"])
    return state["handle"]


def _tables(state):
    return {k: state[k] for k in ("page_table", "lens", "refs", "free_bits", "pool")}


def _run_attention(state, case):
    """The new rows' K and V go into the cache, then their queries attend to it.  Rows are the last ones of their sequences."""
    window, sinks = case["window"], case["sinks"]
    if own:
        cache = _handle(state, case)
        several = dict(row_off=state["row_off"], max_rows=state["most_rows"]) if case["op"] == "rows" else {}
        cache.write(0, state["k"], state["v"], **several)
        out = cache.attention(0, state["q"], out=state["out"], window=window, sinks=sinks, **several)
        return {"out": out, "pool": state["pool"]}
    q, pool, table, page = state["q"], state["pool"], state["page_table"].long(), case["page"]
    total, heads, hd = q.shape
    kv, n, R, T = case["kv_heads"], case["batch"], state["most_rows"], state["most_len"]
    lens, off = state["lens"].long(), state["row_off"].long()
    count = off[1:] - off[:-1]
    row = torch.arange(total, device=DEVICE)
    seq = torch.searchsorted(off, row, right=True) - 1
    place = lens[seq] - count[seq] + row - off[seq]                     # the row's position in its sequence
    pool[0, 0][table[seq, place // page], :, place % page] = state["k"]
    pool[0, 1][table[seq, place // page], :, place % page] = state["v"]
    # keys of every sequence: all of them, or the first ones and the part that some row's window reaches
    if window and sinks + R + window - 1 < T:
        W = R + window - 1
        start = torch.clamp(lens - W, min=sinks)[:, None]
        key = torch.cat([torch.arange(sinks, device=DEVICE).expand(n, sinks), start + torch.arange(W, device=DEVICE)], 1)
    else:
        key = torch.arange(T, device=DEVICE).expand(n, T)
    there = key < lens[:, None]
    at = torch.where(there, key, 0)
    pages = torch.gather(table, 1, at // page)
    k = pool[0, 0][pages, :, at % page].float()                         # [n, keys, kv heads, head dim]
    v = pool[0, 1][pages, :, at % page].float()
    slot = torch.arange(R, device=DEVICE)
    rows = torch.clamp(off[:-1, None] + slot, max=total - 1)            # [n, R]
    position = (lens - count)[:, None] + slot
    qs = q.float()[rows].view(n, R, kv, heads // kv, hd)
    scores = torch.einsum("nrhgd,nkhd->nhgrk", qs, k) / math.sqrt(hd)
    seen = there[:, None] & (key[:, None] <= position[:, :, None])      # [n, R, keys]
    if window:
        seen &= (key[:, None] > position[:, :, None] - window) | (key[:, None] < sinks)
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = scores.sub_(torch.where(torch.isfinite(top), top, 0)).exp_()
    out = torch.einsum("nhgrk,nkhd->nrhgd", weights, v) / weights.sum(-1).permute(0, 3, 1, 2).unsqueeze(-1)
    out = out.reshape(n, R, heads, hd)[seq, row - off[seq]]
    return {"out": out.to(q.dtype), "pool": pool}


def _bits(refs):
    """The free pages' bits from the reference counts."""
    n = refs.numel()
    free = torch.zeros(-(-n // 32) * 32, dtype=torch.int64, device=refs.device)
    free[:n] = refs == 0
    words = (free.view(-1, 32) << torch.arange(32, device=refs.device)).sum(1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _extend(state, page, seqs, n_new):
    """Room for n_new more tokens of each sequence: new pages, lowest free index first, in the order of the sequences; a last
    page that is shared and not full is copied for its writer."""
    pool, table, lens, refs = state["pool"], state["page_table"], state["lens"], state["refs"]
    length = lens[seqs].long()
    held, after = -(-length // page), -(-(length + n_new) // page)
    last = table[seqs, torch.clamp(held - 1, min=0)].long()
    last = torch.where(held > 0, last, refs.argmax())                   # (a page in use, for sequences without any)
    partly = (length % page > 0) & (n_new > 0)
    earlier = torch.tril((last[:, None] == last[None, :]) & partly[None, :], -1).sum(1)
    copies = partly & (refs[last] - earlier > 1)
    need = after - held + copies
    free = torch.argsort((refs > 0).to(torch.int32), stable=True)       # free pages first, lowest index first
    first = torch.cumsum(need, 0) - need
    # copies take the first of a sequence's new pages
    new = torch.where(copies, free[torch.where(copies, first, 0)], last)
    column = torch.arange(table.shape[1], device=DEVICE)
    rank = column[None] - held[:, None]                                 # 0, 1, ... for the added columns
    added = (rank >= 0) & (column[None] < after[:, None])
    fresh = free[torch.clamp((first + copies)[:, None] + rank, 0, free.numel() - 1)].to(torch.int32)
    table[seqs] = torch.where(added, fresh, table[seqs])
    table[seqs, torch.clamp(held - 1, min=0)] = torch.where(copies, new, table[seqs, torch.clamp(held - 1, min=0)].long()).to(torch.int32)
    taken = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=DEVICE)
    taken.index_add_(0, torch.where(copies, last, refs.numel()), -torch.ones_like(lens[seqs]))
    taken.index_add_(0, torch.where(copies, new, refs.numel()), torch.ones_like(lens[seqs]))
    taken.index_add_(0, torch.where(added, fresh.long(), refs.numel()).flatten(), torch.ones(added.numel(), dtype=torch.int32, device=DEVICE))
    refs += taken[:-1]
    # the rows in front of the new tokens, into the copies
    token = torch.arange(page, device=DEVICE)
    moved = copies[:, None] & (token[None] < (length % page)[:, None])
    pool[:, :, new] = torch.where(moved[None, None, :, None, :, None], pool[:, :, last], pool[:, :, new])
    lens[seqs] = (length + n_new).to(torch.int32)


def _release(state, column_from, seqs):
    """Gives back the pages of the table's columns from column_from on."""
    table, refs = state["page_table"], state["refs"]
    gone = (torch.arange(table.shape[1], device=DEVICE)[None] >= column_from[:, None]) & (table[seqs] >= 0)
    dropped = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=DEVICE)
    dropped.index_add_(0, torch.where(gone, table[seqs].long(), refs.numel()).flatten(),
                       torch.ones(gone.numel(), dtype=torch.int32, device=DEVICE))
    refs -= dropped[:-1]
    table[seqs] = torch.where(gone, -1, table[seqs])


def _run_fork(state, case):
    """The children of the pass before are given up; every parent's new children share its pages, and each makes room for
    one token of its own."""
    if own:
        cache = _handle(state, case)
        cache.free(state["dst"])
        cache.fork(state["src"], state["dst"])
        cache.extend(state["one"], seqs=state["dst"])
        return _tables(state)
    table, lens, refs = state["page_table"], state["lens"], state["refs"]
    src, dst = state["src"].long(), state["dst"].long()
    _release(state, torch.zeros_like(dst), dst)
    lens[dst] = 0
    table[dst] = table[src]
    lens[dst] = lens[src]
    shared = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=DEVICE)
    held = table[src].long()
    shared.index_add_(0, torch.where(held >= 0, held, refs.numel()).flatten(), torch.ones(held.numel(), dtype=torch.int32, device=DEVICE))
    refs += shared[:-1]
    _extend(state, case["page"], dst, state["one"].long())
    state["free_bits"].copy_(_bits(refs))
    return _tables(state)


def _run_accept(state, case):
    """Room for the packed rows of a verification, the accepted rows move up behind the context, the rest is given back;
    then the accepted ones are taken back too, so that a pass begins where the one before did."""
    if own:
        cache = _handle(state, case)
        cache.extend(state["packed"])
        cache.compact(state["packed"], state["keep"], rows=state["path"])
        cache.compact(state["keep"], state["none"])
        return _tables(state)
    page, pool, table, lens = case["page"], state["pool"], state["page_table"], state["lens"]
    seqs = torch.arange(case["batch"], device=DEVICE)
    base = lens.long().clone()
    _extend(state, page, seqs, state["packed"].long())
    keep, path = state["keep"].long(), state["path"].long()
    j = torch.arange(path.shape[1], device=DEVICE)
    source = base[:, None] + torch.where(j[None] < keep[:, None], path, j[None])      # rows that are not kept stay
    target = base[:, None] + j[None]
    inside = target < (base + state["packed"])[:, None]
    source, target = torch.where(inside, source, base[:, None]), torch.where(inside, target, base[:, None])
    rows = pool[:, :, torch.gather(table, 1, source // page).long(), :, source % page]
    pool[:, :, torch.gather(table, 1, target // page).long(), :, target % page] = rows
    lens.copy_(base + keep)
    _release(state, -(-(base + keep) // page), seqs)
    lens.copy_(base)
    _release(state, -(-base // page), seqs)
    state["free_bits"].copy_(_bits(state["refs"]))
    return _tables(state)


def _run_logprobs(state, case):
    """Per row: the given token's log probability, the distribution's entropy, the most likely tokens with theirs."""
    top = case["top"]
    if own:
        from paper_2403_09919_b200 import binding
        return binding.token_logprobs(state["logits"], state["tokens"], top=top, temperature=case["temperature"])
    x = state["logits"].float() / case["temperature"]
    peak = x.amax(1, keepdim=True)
    e = (x - peak).exp()
    total = e.sum(1)
    lse = peak[:, 0] + total.log()
    mean = torch.where(e > 0, e * x, 0).sum(1) / total
    got = {"logprob": x.gather(1, state["tokens"].long()[:, None])[:, 0] - lse, "entropy": lse - mean}
    if top:
        index = torch.sort(state["logits"].float(), dim=1, descending=True, stable=True).indices[:, :top]
        got["top_ids"] = index.to(torch.int32)
        got["top_logprobs"] = x.gather(1, index) - lse[:, None]
    return got


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    plan = _plan(case)
    if case["op"] == "logprobs":
        x = state["logits"].double() / case["temperature"]
        logp = torch.log_softmax(x, 1)
        p = logp.exp()
        got = {"logprob": logp[torch.arange(case["rows"]), state["tokens"].long()], "entropy": -torch.special.xlogy(p, p).sum(1)}
        if case["top"]:
            got["top_ids"] = None
            got["top_logprobs"] = torch.topk(logp, case["top"], dim=1).values
        return got
    page = case["page"]
    if case["op"] in ("token", "rows"):
        return _exact_attention(state, case, plan)
    # whole numbers and moved rows: the same in any number of bits, worked through one sequence after another on the host
    pool = state["pool"]
    table = [[p for p in row if p >= 0] for row in state["page_table"].tolist()]
    lens, refs = state["lens"].tolist(), state["refs"].tolist()

    def take():
        p = refs.index(0)
        refs[p] = 1
        return p

    def grow(s, n):
        jobs = []
        if lens[s] % page and refs[table[s][-1]] > 1:
            refs[table[s][-1]] -= 1
            old, table[s][-1] = table[s][-1], take()
            jobs.append((old, table[s][-1], lens[s] % page))
        while len(table[s]) * page < lens[s] + n:
            table[s].append(take())
        lens[s] += n
        return jobs

    def shrink(s, length):
        while len(table[s]) > -(-length // page):
            refs[table[s].pop()] -= 1
        lens[s] = length

    if case["op"] == "fork":
        src, dst = state["src"].tolist(), state["dst"].tolist()
        for a, b in zip(src, dst):
            table[b], lens[b] = list(table[a]), lens[a]
            for p in table[b]:
                refs[p] += 1
        for b in dst:
            for old, new, rows in grow(b, 1):
                pool[:, :, new, :, :rows] = pool[:, :, old, :, :rows]
    else:
        for s in range(case["batch"]):
            grow(s, int(plan["packed"][s]))
        for s in range(case["batch"]):
            base = int(plan["lens"][s])
            for j in range(int(plan["keep"][s])):
                a, b = base + int(plan["path"][s, j]), base + j
                pool[:, :, table[s][b // page], :, b % page] = pool[:, :, table[s][a // page], :, a % page]
            shrink(s, base)
    width = state["page_table"].shape[1]
    words = [0] * state["free_bits"].numel()
    for p, r in enumerate(refs):
        words[p // 32] |= (r == 0) << (p % 32)
    return {"page_table": torch.tensor([row + [-1] * (width - len(row)) for row in table], dtype=torch.int32),
            "lens": torch.tensor(lens, dtype=torch.int32), "refs": torch.tensor(refs, dtype=torch.int32),
            "free_bits": torch.tensor([w - (1 << 32) if w >> 31 else w for w in words], dtype=torch.int32), "pool": pool}


def _exact_attention(state, case, plan):
    page, pool, heads, kv, hd = case["page"], state["pool"], case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty_like(state["q"], dtype=torch.float64)
    at = 0
    for s, (length, rows) in enumerate(zip(plan["lens"].tolist(), plan["rows"].tolist())):
        pages = state["page_table"][s, :_pages(length, page)].long()
        both = []
        for which, new in ((0, state["k"]), (1, state["v"])):
            x = pool[0, which][pages].transpose(1, 2).reshape(-1, kv, hd)
            x[length - rows:length] = new[at:at + rows]
            pool[0, which][pages] = x.view(-1, page, kv, hd).transpose(1, 2)
            both.append(x[:length].double())
        key = torch.arange(length, device=DEVICE)
        for lo in range(0, rows, 1024):
            hi = min(rows, lo + 1024)
            place = torch.arange(length - rows + lo, length - rows + hi, device=DEVICE)[:, None]
            hidden = key > place
            if case["window"]:
                hidden |= (key <= place - case["window"]) & (key >= case["sinks"])
            for h in range(heads):
                k, v = both[0][:, h * kv // heads], both[1][:, h * kv // heads]
                score = state["q"][at + lo:at + hi, h].double() @ k.T / math.sqrt(hd)
                out[at + lo:at + hi, h] = torch.softmax(score.masked_fill(hidden, -math.inf), 1) @ v
        at += rows
    return {"out": out, "pool": pool}
