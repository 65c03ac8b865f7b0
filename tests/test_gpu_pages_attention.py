"""Attention over a cache in pages against 64 bits: single tokens and runs of rows, windows and sinks, lengths and sizes where
tiles end, anything at all in places that a row does not see."""
import math

import numpy as np
import pytest
import torch

from helpers import dev
from pages_model import attend, tolerance
from paper_2403_09919_b200 import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def build(lens, rows, heads, kv_heads, head_dim, page, dtype, seed=0, layers=1, scale=1.0, spread=1.0):
    """A cache of sequences of these lengths whose pages lie in any order, and rows q, k, v of the last tokens (already written).
    What no token fills is NaN."""
    rng, gen = np.random.default_rng(seed), torch.Generator("cuda:0").manual_seed(seed)
    held = [-(-n // page) for n in lens]
    n_pages, S = sum(held) + 3, len(lens)
    cache = binding.PagedCache.empty(layers, kv_heads, head_dim, page, n_pages, S, max(max(held), 1) + 1, dtype)
    order = rng.permutation(n_pages)
    table, at = np.full((S, max(max(held), 1) + 1), -1), 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
    cache.page_table.copy_(dev(table))
    cache.lens.copy_(dev(np.array(lens)))
    cache.refs[torch.from_numpy(order[:at]).to("cuda:0")] = 1
    cache.pool.fill_(math.nan)
    keys, values = [], []
    for s, n in enumerate(lens):
        k, v = ((torch.randn(n, kv_heads, head_dim, generator=gen, device="cuda:0") * spread).to(DT[dtype]) for _ in range(2))
        put(cache, table, s, 0, k, v, layers - 1)
        keys.append(k)
        values.append(v)
    q = (torch.randn(sum(rows), heads, head_dim, generator=gen, device="cuda:0") * scale).to(DT[dtype])
    return cache, table, q, keys, values


def put(cache, table, s, first, k, v, layer):
    pos = torch.arange(first, first + k.shape[0], device="cuda:0")
    pages = torch.from_numpy(table[s]).to("cuda:0")[pos // cache.page_size]
    cache.pool[layer, 0][pages, :, pos % cache.page_size] = k
    cache.pool[layer, 1][pages, :, pos % cache.page_size] = v


def compare(got, lse, q, keys, values, lens, rows, window, sinks, scale=None):
    at = 0
    for n, m, k, v in zip(lens, rows, keys, values):
        part = slice(at, at + m)
        at += m
        if not m:
            continue
        ref, ref_lse, absv, absqk = attend(q[part], k, v, np.arange(n - m, n), window, sinks, scale)
        sc = scale or 1 / math.sqrt(q.shape[-1])
        err = (got[part].double() - ref).abs()
        tol = tolerance(q.dtype, ref, absv, absqk, n, sc)
        assert torch.isfinite(got[part]).all()
        assert (err <= tol).all(), (n, m, float((err / tol).max()))
        if lse is not None:
            there = torch.isfinite(ref_lse)
            assert torch.equal(there, torch.isfinite(lse[part]))
            d = (lse[part].double() - ref_lse)[there].abs()
            bound = ((q.shape[-1] + 8) * 2.0 ** -24 * absqk * sc + (n + 16) * 2.0 ** -24 + 2.0 ** -19 + ref_lse.abs() * 2.0 ** -22)[there]
            assert (d <= bound).all(), float((d / bound).max())


def run(lens, rows, heads, kv_heads, head_dim, page, dtype, window=0, sinks=0, seed=0, scale=None, spread=1.0, qscale=1.0, several=True):
    cache, table, q, keys, values = build(lens, rows, heads, kv_heads, head_dim, page, dtype, seed, scale=qscale, spread=spread)
    lse = torch.full((q.shape[0], heads), 7.0, device="cuda:0")
    kw = dict(row_off=dev(np.concatenate([[0], np.cumsum(rows)])), max_rows=max(max(rows), 1)) if several else {}
    got = cache.attention(0, q, window=window, sinks=sinks, lse=lse, scale=scale or 0.0, **kw)
    cache.poll()
    compare(got, lse, q, keys, values, lens, rows, window, sinks, scale)


HEADS = [(4, 4, 64), (32, 8, 128), (16, 1, 128), (3, 3, 128), (40, 2, 64), (24, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", HEADS)
@pytest.mark.parametrize("page,window,sinks", [(16, 0, 0), (64, 0, 0), (32, 70, 5), (128, 33, 0)])
def test_single_tokens(dtype, heads, kv_heads, head_dim, page, window, sinks):
    lens = [1, 16, 17, 64, 63, 200, 129, 513, 2, 1000, 0]
    run(lens, [1] * len(lens), heads, kv_heads, head_dim, page, dtype, window, sinks, seed=page, several=False)


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("lens", [[9000], [7, 30000, 1, 5000], [1] * 300, list(range(1, 130))])
def test_single_tokens_of_long_and_of_many_sequences(page, lens):
    run(lens, [1] * len(lens), 8, 2, 128, page, "bf16", seed=len(lens), several=False)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 200), (64, 64), (100, 3), (5000, 4), (128, 1), (129, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_windows_of_single_tokens(dtype, window, sinks):
    lens = [1, 2, 16, 63, 64, 65, 100, 128, 129, 130, 400, 1025]
    run(lens, [1] * len(lens), 4, 2, 128, 32, dtype, window, sinks, several=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 4, 128), (8, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("page,window,sinks", [(16, 0, 0), (128, 0, 0), (32, 100, 5), (64, 17, 0), (64, 130, 140)])
def test_runs_of_rows(dtype, heads, kv_heads, head_dim, page, window, sinks):
    lens, rows = [300, 128, 129, 1, 700, 40, 555], [300, 128, 1, 1, 257, 0, 33]
    run(lens, rows, heads, kv_heads, head_dim, page, dtype, window, sinks, seed=page)


@pytest.mark.parametrize("window,sinks", [(0, 0), (256, 4), (1000, 0)])
def test_a_long_run_of_rows(window, sinks):
    run([2500, 1300], [2100, 1300], 2, 1, 128, 64, "bf16", window, sinks)


@pytest.mark.parametrize("several", [False, True])
def test_scores_far_apart_and_a_scale(several):
    """Scores in the hundreds, of either sign: maxima move by large steps, weights are 0 and 1."""
    lens, rows = [700, 300], ([1, 1] if not several else [200, 150])
    run(lens, rows, 4, 2, 128, 32, "bf16", seed=3, qscale=30.0, several=several)
    run(lens, rows, 4, 2, 128, 32, "bf16", seed=4, scale=0.5, several=several)
    run(lens, rows, 4, 2, 128, 32, "bf16", window=90, sinks=2, seed=5, qscale=30.0, several=several)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 3.3e38])
@pytest.mark.parametrize("dtype,head_dim", [("bf16", 128), ("fp32", 128), ("bf16", 64)])
def test_what_a_row_does_not_see_does_not_reach_it(bad, dtype, head_dim):
    """Keys and values outside a window hold NaN, infinities or the type's largest numbers; some rows of a call see them and
    the rows behind do not."""
    window, sinks, page = 40, 3, 32
    lens, rows = [400, 150], [90, 60]
    for single in (True, False):
        r = [1, 1] if single else rows
        cache, table, q, keys, values = build(lens, r, 4, 2, head_dim, page, dtype, seed=9)
        spots = [(0, 3, 200), (1, 3, 50)] if single else [(0, 3, 230), (1, 3, 30), (0, 320, 322)]
        for s, a, b in spots:
            for x in (keys[s], values[s]):
                x[a:b] = bad
            put(cache, table, s, 0, keys[s], values[s], 0)
        kw = {} if single else dict(row_off=dev(np.array([0, 90, 150])), max_rows=90)
        got = cache.attention(0, q, window=window, sinks=sinks, **kw)
        cache.poll()
        at = 0
        for s, (n, m) in enumerate(zip(lens, r)):
            pos = np.arange(n - m, n)
            clean = np.array([not any(max(a, p - window + 1) < min(b, p + 1) for (t, a, b) in spots if t == s) for p in pos])
            assert clean.any()
            idx = torch.from_numpy(np.nonzero(clean)[0]).to("cuda:0")
            qs = q[at:at + m][idx]
            ref, _, absv, absqk = attend(qs, keys[s], values[s], pos[clean], window, sinks)
            err = (got[at:at + m][idx].double() - ref).abs()
            assert (err <= tolerance(q.dtype, ref, absv, absqk, n, 1 / math.sqrt(head_dim))).all()
            if not np.isfinite(bad) and not clean.all():      # and where it is seen it does
                dirty = torch.from_numpy(np.nonzero(~clean)[0]).to("cuda:0")
                assert not torch.isfinite(got[at:at + m][dirty]).all()
            at += m


def test_rows_behind_the_last_sequence_stay():
    for dtype, hd in (("bf16", 128), ("fp32", 64)):
        cache, table, q, keys, values = build([200, 90], [60, 50], 4, 2, hd, 16, dtype)
        q = torch.cat([q, torch.full((40, 4, hd), math.nan, device="cuda:0", dtype=q.dtype)])
        out, lse = torch.full_like(q, 5.0), torch.full((150, 4), 5.0, device="cuda:0")
        cache.attention(0, q, out=out, lse=lse, row_off=dev(np.array([0, 60, 110])), max_rows=60)
        cache.poll()
        assert (out[110:] == 5).all() and (lse[110:] == 5).all()
        compare(out, lse, q, keys, values, [200, 90], [60, 50], 0, 0)


def test_strides_layers_lists_and_in_one_buffer():
    """Rows of q, k and v as parts of one projection's output, a list of sequences in any order (one of them twice), the last of
    several layers."""
    heads, kv, hd, page = 8, 2, 128, 16
    lens = [70, 33, 200]
    for rows in ([1, 1, 1, 1], [3, 20, 50, 1]):
        cache, table, _, keys, values = build(lens, [1, 1, 1], heads, kv, hd, page, "bf16", layers=3)
        seqs = [2, 0, 1, 2]
        total = sum(rows)
        fused = torch.randn(total, heads + 2 * kv, hd, device="cuda:0").to(torch.bfloat16)
        q = fused[:, :heads]
        out = torch.zeros(total, heads + 3, hd, device="cuda:0", dtype=torch.bfloat16)
        kw = dict(seqs=dev(np.array(seqs)))
        if total > 4:
            kw.update(row_off=dev(np.concatenate([[0], np.cumsum(rows)])), max_rows=max(rows))
        cache.attention(2, q, out=out[:, 2:2 + heads], **kw)
        cache.poll()
        at = 0
        for s, m in zip(seqs, rows):
            compare(out[at:at + m, 2:2 + heads], None, q[at:at + m], [keys[s]], [values[s]], [lens[s]], [m], 0, 0)
            at += m
        assert (out[:, :2] == 0).all() and (out[:, 2 + heads:] == 0).all()


def test_pages_out_of_the_pool_and_trimmed_ones():
    for rows in ([1, 1], [80, 80]):
        cache, table, q, keys, values = build([400, 400], rows, 4, 2, 128, 16, "bf16")
        kw = dict(row_off=dev(np.array([0, rows[0], sum(rows)])), max_rows=max(rows)) if rows[0] > 1 else {}
        want = cache.attention(0, q, window=50, sinks=3, **kw)
        cache.poll()
        cache.page_table[:, 1:(400 - rows[0] - 50) // 16] = -1          # what the window has left behind
        again = cache.attention(0, q, window=50, sinks=3, **kw)
        cache.poll()
        assert torch.equal(want, again)
        cache.page_table[0, 24] = 1 << 30                               # a key that is seen lies nowhere: reported
        got = cache.attention(0, q, window=50, sinks=3, **kw)
        with pytest.raises(binding.RdError) as e:
            cache.poll()
        assert e.value.code == 1
        assert torch.equal(got[rows[0]:], want[rows[0]:])               # and the other sequence is as it was


def test_a_sequence_outside_the_table_and_more_rows_than_announced():
    cache, table, q, keys, values = build([100, 50], [1, 1], 4, 2, 128, 16, "bf16")
    out = cache.attention(0, q, seqs=dev(np.array([9, 1])))
    with pytest.raises(binding.RdError):
        cache.poll()
    assert (out[0] == 0).all()
    compare(out[1:], None, q[1:], keys[1:], values[1:], [50], [1], 0, 0)
    q3 = torch.cat([q, q])
    for limit in (1, 2):
        out = torch.full_like(q3, 3.0)
        cache.attention(0, q3, out=out, row_off=dev(np.array([0, 3, 4])), max_rows=limit)
        with pytest.raises(binding.RdError):
            cache.poll()
        assert (out[:3] == 3).all()
        compare(out[3:], None, q3[3:], keys[1:], values[1:], [50], [1], 0, 0)


def test_more_rows_than_tokens():
    """Rows that would lie before a sequence's first token have no keys."""
    cache, table, q, keys, values = build([5], [9], 4, 2, 128, 16, "bf16")
    lse = torch.zeros(9, 4, device="cuda:0")
    out = cache.attention(0, q, row_off=dev(np.array([0, 9])), max_rows=9, lse=lse)
    cache.poll()
    assert (out[:4] == 0).all() and (lse[:4] == -math.inf).all()
    compare(out[4:], lse[4:], q[4:], keys, values, [5], [5], 0, 0)


def test_in_graphs_and_repeated():
    """Captured calls of two sizes share the handle's workspace in one stream; every replay gives the same bits."""
    lens = [3000, 50, 700]
    cache, table, q, keys, values = build(lens, [1, 1, 1], 8, 2, 128, 32, "bf16")
    rows = [100, 50, 300]
    q2 = torch.randn(450, 8, 128, device="cuda:0").to(torch.bfloat16)
    off = dev(np.concatenate([[0], np.cumsum(rows)]))
    want = cache.attention(0, q).clone(), cache.attention(0, q2, row_off=off, max_rows=300, window=64, sinks=2).clone()
    o1, o2 = torch.empty_like(q), torch.empty_like(q2)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        cache.attention(0, q, out=o1)
    with torch.cuda.graph(g2):
        cache.attention(0, q2, out=o2, row_off=off, max_rows=300, window=64, sinks=2)
        cache.attention(0, q, out=o1)
    for _ in range(3):
        o1.zero_(), o2.zero_()
        g1.replay()
        assert torch.equal(o1, want[0])
        o1.zero_()
        g2.replay()
        g1.replay()
        assert torch.equal(o1, want[0]) and torch.equal(o2, want[1])
    cache.poll()


def test_refusals():
    cache, table, q, keys, values = build([50], [1], 4, 2, 128, 16, "bf16")

    def refused(code, **kw):
        with pytest.raises(binding.RdError) as e:
            cache.attention(kw.pop("layer", 0), kw.pop("q", q), **kw)
        assert e.value.code == code

    refused(1, layer=1)
    refused(1, layer=-1)
    refused(1, window=-1)
    refused(1, sinks=-1)
    refused(1, scale=-1.0)
    refused(1, scale=math.nan)
    refused(2, q=torch.cat([q, q[:, :1]], 1))                      # five heads on two
    buf = torch.zeros(4 * 128 + 8, device="cuda:0", dtype=torch.bfloat16)
    refused(2, q=buf[1:513].view(1, 4, 128))                       # not on a 16-byte boundary
    with pytest.raises(ValueError):
        cache.attention(0, q.float())
    with pytest.raises(ValueError):
        cache.attention(0, q.transpose(1, 2))
    with pytest.raises(ValueError):
        cache.attention(0, q, out=q[:, :2])
    with pytest.raises(ValueError):
        cache.attention(0, q, row_off=torch.zeros(2, dtype=torch.int64, device="cuda:0"))
    with pytest.raises(ValueError):
        cache.attention(0, q, lse=torch.zeros(1, 4, device="cuda:0", dtype=torch.float64))
    assert cache.attention(0, q[:0]).shape == (0, 4, 128)
    n = cache.launch_count()
    with pytest.raises(binding.RdError):
        cache.write(1, keys[0][:1], values[0][:1])
    assert cache.launch_count() == n
    cache.poll()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[1, 1, 1], [300, 40, 700]])
def test_the_widest_window_is_no_window(dtype, rows):
    """Positions before the first token less a window of 2^31 - 1 (a sequence of fewer tokens than rows) leave 32 bits."""
    lens = [5, 40, 700]
    cache, table, q, keys, values = build(lens, [min(m, n) for m, n in zip(rows, lens)], 4, 2, 128, 16, dtype)
    q = torch.randn(sum(rows), 4, 128, device="cuda:0").to(DT[dtype])
    kw = dict(row_off=dev(np.concatenate([[0], np.cumsum(rows)])), max_rows=max(rows)) if max(rows) > 1 else {}
    want = cache.attention(0, q, **kw)
    for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 30, 7), (701, 0)):
        assert torch.equal(cache.attention(0, q, window=window, sinks=sinks, **kw), want)
    cache.poll()
    compare(want[-rows[2]:], None, q[-rows[2]:], keys[2:], values[2:], lens[2:], rows[2:], 0, 0)


def test_a_missing_page_of_the_fp32_configuration():
    """A page that the table does not name, where a token looks: reported; what the copy's slot held before is not read."""
    cache, table, q, keys, values = build([400, 400], [1, 1], 4, 2, 128, 16, "fp32")
    want = cache.attention(0, q)
    cache.poll()
    cache.pool[0, :, torch.from_numpy(table[1, :25].copy()).to("cuda:0")] = 1e30      # (sequence 1, which the same CTAs may have read)
    cache.page_table[0, 3] = -1
    got = cache.attention(0, q)
    with pytest.raises(binding.RdError) as e:
        cache.poll()
    assert e.value.code == 1
    assert got[0].abs().max() < 100
    cache.page_table[0, 3] = int(table[0, 3])
    assert torch.equal(cache.attention(0, q)[0], want[0])
    cache.poll()


def test_refused_heads():
    cache, table, q, keys, values = build([20], [1], 2, 1, 64, 16, "bf16")
    for heads in (1025, 5000):
        with pytest.raises(binding.RdError) as e:
            cache.attention(0, torch.zeros(1, heads, 64, dtype=torch.bfloat16, device="cuda:0"))
        assert e.value.code == 2
    wide = torch.randn(1, 1024, 64, device="cuda:0").bfloat16()
    compare(cache.attention(0, wide), None, wide, keys, values, [20], [1], 0, 0)


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 2, 128), (16, 1, 128), (3, 3, 64), (40, 8, 128)])
@pytest.mark.parametrize("lens,rows", [([9000], [17]), ([5000], [256]), ([4099], [130]), ([3000, 40, 6001, 1, 0], [33, 40, 256, 1, 0])])
def test_few_rows_over_long_contexts(heads, kv_heads, head_dim, lens, rows):
    """Several CTAs share the keys of a query head's rows; some of the sequences are too short for that."""
    run(lens, rows, heads, kv_heads, head_dim, 64, "bf16", seed=heads + len(lens))


@pytest.mark.parametrize("window,sinks,page", [(2000, 0, 16), (2000, 70, 64), (1100, 5, 128), (4999, 300, 32)])
def test_few_rows_of_long_windows(window, sinks, page):
    run([7000, 2500], [200, 90], 6, 2, 128, page, "bf16", window=window, sinks=sinks)


@pytest.mark.parametrize("bad", [math.nan, math.inf, 3.3e38])
def test_few_rows_over_long_contexts_with_anything_in_hidden_places(bad):
    """Keys and values behind a row's place and before its window hold anything; a value that some rows see reaches them alone."""
    lens, rows, window = [5000], [150], 3000
    cache, table, q, keys, values = build(lens, rows, 4, 2, 128, 64, "bf16")
    kw = dict(row_off=dev(np.array([0, 150])), max_rows=150, window=window)
    want = cache.attention(0, q, **kw)
    compare(want, None, q, keys, values, lens, rows, window, 0)
    for x in (keys[0], values[0]):
        x[:5000 - 150 - window] = bad           # before every row's window
    put(cache, table, 0, 0, keys[0], values[0], 0)
    assert torch.equal(cache.attention(0, q, **kw), want)
    values[0][4900] = bad                       # position 4900: rows 50 .. 149 see it, 0 .. 49 do not
    put(cache, table, 0, 4900, keys[0][4900:4901], values[0][4900:4901], 0)
    lse = torch.zeros(150, 4, device="cuda:0")
    got = cache.attention(0, q, lse=lse, **kw)
    cache.poll()
    if not math.isfinite(bad):
        assert not torch.isfinite(got[50:]).any() and torch.isfinite(lse).all()
    v = torch.where(torch.isfinite(values[0].float()), values[0].float(), 0.0)
    v[:5000 - 150 - window] = 0
    k = keys[0].clone()
    k[:5000 - 150 - window] = 0
    ref, _, absv, absqk = attend(q[:50], k, v.to(torch.bfloat16), np.arange(4850, 4900), window, 0, None)
    tol = tolerance(q.dtype, ref, absv, absqk, 5000, 1 / math.sqrt(128))
    assert ((got[:50].double() - ref).abs() <= tol).all()


def test_few_rows_of_many_sequences_in_a_graph():
    """The parts of one call are joined before the next one's are left; the same again in a replay."""
    lens, rows = [2600, 1800, 3000], [20, 33, 7]
    cache, table, q, keys, values = build(lens, rows, 8, 2, 128, 32, "bf16")
    kw = dict(row_off=dev(np.array([0, 20, 53, 60])), max_rows=33)
    outs = [torch.empty_like(q) for _ in range(3)]
    want = cache.attention(0, q, **kw).clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for i, o in enumerate(outs):
            cache.attention(0, q if i != 1 else -q, out=o, **kw)
    for _ in range(3):
        for o in outs:
            o.fill_(7)
        g.replay()
        assert torch.equal(outs[0], want) and torch.equal(outs[2], want)
        compare(outs[1], None, -q, keys, values, lens, rows, 0, 0)
    cache.poll()


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(8, 2, 128), (32, 1, 128), (6, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("rows,window,sinks", [([6, 1, 8, 0, 3], 0, 0), ([8, 8, 8, 8, 8], 500, 5), ([7, 2, 5, 1, 1], 130, 0)])
@pytest.mark.parametrize("page", [16, 128])
def test_few_rows_of_grouped_heads(heads, kv_heads, head_dim, rows, window, sinks, page):
    """The query heads of a key and value head share a tile; contexts that are shared out and such that are not."""
    run([3000, 1, 1400, 0, 257] if rows[0] != 8 else [3000, 8, 1400, 9, 257], rows, heads, kv_heads, head_dim, page, "bf16", window=window, sinks=sinks)


@pytest.mark.parametrize("rows", [33, 64, 65])
def test_rows_of_grouped_heads_in_one_tile_and_two(rows):
    """Four heads of 33 to 64 rows fill both tiles of an item; those of 65 rows do not fit one."""
    run([700, 1500], [rows, rows - 1], 8, 2, 128, 64, "bf16")
    run([700, 1500], [rows, rows - 1], 8, 2, 128, 64, "bf16", window=90, sinks=2)


def test_few_rows_of_grouped_heads_beside_what_they_must_not_touch():
    """Strided rows, rows behind the last sequence, NaN in values that some rows do not see."""
    lens, rows = [2000, 300], [5, 4]
    cache, table, q, keys, values = build(lens, rows, 8, 2, 128, 32, "bf16")
    values[1][298] = math.nan            # position 298: the last two rows of sequence 1
    put(cache, table, 1, 0, keys[1], values[1], 0)
    wide = torch.full((12, 24, 128), 5.0, device="cuda:0", dtype=torch.bfloat16)
    wide[:9, :8] = q
    out = torch.full((12, 24, 128), 3.0, device="cuda:0", dtype=torch.bfloat16)
    cache.attention(0, wide[:, :8], out=out[:, 8:16], row_off=dev(np.array([0, 5, 9])), max_rows=5)
    cache.poll()
    assert (out[9:] == 3).all() and (out[:, :8] == 3).all() and (out[:, 16:] == 3).all()
    assert torch.isnan(out[7:9, 8:16]).all()
    compare(out[:5, 8:16], None, q[:5], keys[:1], values[:1], lens[:1], [5], 0, 0)
    compare(out[5:7, 8:16], None, q[5:7], [keys[1][:298]], [values[1][:298]], [298], [2], 0, 0)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 0), (200, 9), (33, 200)])
def test_rows_of_the_fp32_configuration(head_dim, page, window, sinks):
    """Tiles of 32 rows that end inside an entry, entries of no rows, clusters that share chunks and tiles of a single one."""
    run([1000, 40, 7, 0, 333], [70, 40, 3, 0, 32], 4, 2, head_dim, page, "fp32", window=window, sinks=sinks)
    run([2100], [33], 2, 1, head_dim, page, "fp32", window=window, sinks=sinks)
    run([600] * 20, [65] * 20, 8, 8, head_dim, page, "fp32", window=window, sinks=sinks)


def test_a_page_that_is_missing_for_rows_of_the_fp32_configuration():
    cache, table, q, keys, values = build([400, 400], [50, 50], 4, 2, 64, 16, "fp32")
    kw = dict(row_off=dev(np.array([0, 50, 100])), max_rows=50)
    want = cache.attention(0, q, **kw)
    cache.poll()
    cache.page_table[0, 3] = 1 << 20
    got = cache.attention(0, q, **kw)
    with pytest.raises(binding.RdError) as e:
        cache.poll()
    assert e.value.code == 1
    assert torch.equal(got[50:], want[50:])


def test_handles_on_streams_of_their_own_at_once():
    """Each handle's parts lie in its own workspace: calls on two streams do not meet."""
    off = dev(np.array([0, 20, 21, 30]))
    made = [build([3000, 1, 900], [20, 1, 9], 16, 4, 128, 32, dtype, seed=k) for k, dtype in enumerate(("bf16", "bf16", "fp32"))]
    calls = [lambda c=c, q=q: (c.attention(0, q[:3]), c.attention(0, q, row_off=off, max_rows=20)) for c, _, q, _, _ in made]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(10):
        got = []
        for stream, call in zip(streams, calls):
            with torch.cuda.stream(stream):
                got.append(call())
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for c, *_ in made:
        c.poll()


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 4, 128), (32, 8, 128), (16, 1, 128), (40, 2, 64)])
@pytest.mark.parametrize("window,sinks,qscale", [(0, 0, 1.0), (70, 5, 1.0), (0, 0, 4.0)])
def test_single_tokens_weights_to_sixteen_bits(heads, kv_heads, head_dim, window, sinks, qscale):
    """bf16: the weights that multiply V come in two parts, itself rounded to bf16 (off by 2^-8 of it at most) and what that left,
    rounded again (2^-8 of that): 2^-16 of sum p |v| in place of 2^-8."""
    lens = [1, 16, 17, 64, 63, 200, 129, 513, 2, 1000, 4000]
    cache, table, q, keys, values = build(lens, [1] * len(lens), heads, kv_heads, head_dim, 32, "bf16", seed=heads, scale=qscale)
    got = cache.attention(0, q, window=window, sinks=sinks)
    cache.poll()
    for i, n in enumerate(lens):
        ref, _, absv, absqk = attend(q[i:i + 1], keys[i], values[i], np.array([n - 1]), window, sinks)
        tol = tolerance(q.dtype, ref, absv, absqk, n, 1 / math.sqrt(head_dim)) - (2.0 ** -8 - 2.0 ** -16) * absv * (1 + 2.0 ** -8)
        err = (got[i:i + 1].double() - ref).abs()
        assert (err <= tol).all(), (n, float((err / tol).max()))


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (16, 1)])
def test_infinite_values_that_a_single_token_sees(heads, kv_heads):
    """Weights of exactly one, of a few bits and of many: an infinity times any of them is infinite, in its own dimension alone."""
    lens = [1, 2, 700]
    cache, table, q, keys, values = build(lens, [1] * 3, heads, kv_heads, 128, 32, "bf16", seed=2)
    keys[1][1] = keys[1][0]                       # two weights of one half
    for s in range(3):
        values[s][lens[s] // 2, :, 3], values[s][0, :, 9] = math.inf, -math.inf
        put(cache, table, s, 0, keys[s], values[s], 0)
    got = cache.attention(0, q)
    cache.poll()
    assert (got[:, :, 3] == math.inf).all() and (got[:, :, 9] == -math.inf).all()
    rest = [d for d in range(128) if d not in (3, 9)]
    for s in range(3):
        v = values[s].clone()
        v[:, :, [3, 9]] = 0
        ref, _, absv, absqk = attend(q[s:s + 1], keys[s], v, np.array([lens[s] - 1]))
        assert ((got[s:s + 1].double() - ref).abs() <= tolerance(q.dtype, ref, absv, absqk, lens[s], 128 ** -0.5))[:, :, rest].all()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n,m", [(1, 128), (20, 256), (40, 400), (127, 255)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_many_rows_before_the_first_token(page, n, m, window, sinks):
    """Rows up to 255 places before a sequence's first token, in tiles that other rows of the item fill with keys."""
    cache, table, _, keys, values = build([n], [1], 4, 2, 128, page, "bf16")
    q = torch.randn(m, 4, 128, device="cuda:0").to(torch.bfloat16)
    lse = torch.zeros(m, 4, device="cuda:0")
    out = cache.attention(0, q, row_off=dev(np.array([0, m])), max_rows=m, lse=lse, window=window, sinks=sinks)
    cache.poll()
    assert (out[:m - n] == 0).all() and (lse[:m - n] == -math.inf).all()
    compare(out[m - n:], lse[m - n:], q[m - n:], keys, values, [n], [n], window, sinks)


def test_more_sequences_and_heads_than_a_grid_takes():
    """Refused on the host, before anything is looked at."""
    for dtype in ("fp32", "bf16"):
        cache, table, q, keys, values = build([20], [1], 64, 1, 64, 16, dtype)
        n = cache.launch_count()
        for entries in (2 ** 25, 2 ** 31 - 1):
            rc = cache.L.redrafter_pages_attention(cache.h, 0, None, cache.lens.data_ptr(), entries, 1, 2, 64, q.data_ptr(), 64 * 64, q.data_ptr(), 64 * 64, None,
                                                   0.0, 0, 0, None)
            assert rc == 2
        assert cache.launch_count() == n
