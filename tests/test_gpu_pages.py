"""Management of a cache in pages: every call against a model that works one entry after another, tables and pool bit by bit."""
import numpy as np
import pytest
import torch

from helpers import dev
from pages_model import PageModel
from paper_2403_09919_b200 import binding

pytestmark = pytest.mark.gpu


def make(layers=2, kv_heads=3, head_dim=64, page=16, n_pages=40, max_seqs=10, max_pages=8, dtype="fp32"):
    cache = binding.PagedCache.empty(layers, kv_heads, head_dim, page, n_pages, max_seqs, max_pages, dtype)
    cache.pool.fill_(float("nan"))
    return cache, PageModel(layers, kv_heads, head_dim, page, n_pages, max_seqs, max_pages)


def grow(cache, model, seqs, n_new, rng, layer_rows=True):
    """extend, and rows for the new tokens in every layer."""
    assert model.extend(seqs, n_new)
    cache.extend(dev(np.array(n_new)), seqs=dev(np.array(seqs)))
    total = sum(n_new)
    off = dev(np.concatenate([[0], np.cumsum(n_new)]))
    for layer in range(cache.n_layers):
        k, v = (torch.from_numpy(rng.standard_normal((total, cache.n_kv_heads, cache.head_dim)).astype(np.float32)).to("cuda:0").to(cache.dtype)
                for _ in range(2))
        cache.write(layer, k, v, row_off=off, seqs=dev(np.array(seqs)))
        at = 0
        for s, n in zip(seqs, n_new):
            model.write(layer, s, k[at:at + n].double().cpu().numpy(), v[at:at + n].double().cpu().numpy())
            at += n


@pytest.mark.parametrize("page,head_dim,dtype", [(16, 64, "fp32"), (32, 128, "bf16"), (64, 64, "bf16"), (128, 128, "fp32")])
def test_a_life_of_forks_growth_acceptance_and_release(page, head_dim, dtype):
    cache, model = make(page=page, head_dim=head_dim, dtype=dtype, n_pages=37, max_seqs=9, max_pages=7)
    rng = np.random.default_rng(page)
    model.check(cache)
    grow(cache, model, [0, 4], [page + 3, 2 * page], rng)
    model.check(cache)
    cache.fork(dev(np.array([0, 0, 4])), dev(np.array([1, 7, 2])))
    model.fork([0, 0, 4], [1, 7, 2])
    model.check(cache)
    grow(cache, model, [7, 2], [1, 5], rng)          # 7 copies its page, 2 (a full last page) does not
    model.check(cache)
    grow(cache, model, [1, 0], [page, 2], rng)       # both share the page: 1 copies, 0 is the last and keeps it
    model.check(cache)
    # a verification of packed rows on two sequences, accepted paths move up
    grow(cache, model, [0, 2], [9, page + 4], rng)
    rows = [[0, 2, 8], [1, 3, page + 3]]
    keep = [3, 2]
    cache.compact(dev(np.array([9, page + 4])), dev(np.array(keep)), rows=dev(np.array(rows)), seqs=dev(np.array([0, 2])))
    model.compact([0, 2], [9, page + 4], keep, rows)
    model.check(cache)
    cache.compact(dev(np.array([1])), dev(np.array([0])), seqs=dev(np.array([7])))     # truncate by one token
    model.compact([7], [1], [0])
    model.check(cache)
    grow(cache, model, [4], [2 * page + 1], rng)
    cache.trim(page + 1, 3, seqs=dev(np.array([4, 8])))   # 8 is empty
    model.trim([4, 8], page + 1, 3)
    model.check(cache)
    cache.fork(dev(np.array([4])), dev(np.array([8])))    # of a trimmed sequence
    model.fork([4], [8])
    cache.free(dev(np.array([4, 1, 3])))                  # 3 is empty
    model.free([4, 1, 3])
    model.check(cache)
    grow(cache, model, [3, 8], [page - 1, 2], rng)
    model.check(cache)
    cache.poll()
    cache.free()
    model.free(range(9))
    model.check(cache)
    cache.poll()


def test_random_calls():
    rng = np.random.default_rng(5)
    S, page = 12, 16
    cache, model = make(layers=1, kv_heads=2, page=page, n_pages=90, max_seqs=S, max_pages=9)
    for step in range(120):
        what = rng.choice(["extend", "extend", "fork", "compact", "free", "trim"])
        if what == "extend":
            seqs = rng.permutation(S)[:rng.integers(1, S + 1)].tolist()
            n_new = [int(min(rng.integers(0, 40), page * 9 - model.lens[s])) for s in seqs]
            if model.pages_needed(seqs, n_new) > model.refs.count(0):
                cache.extend(dev(np.array(n_new)), seqs=dev(np.array(seqs)))
                with pytest.raises(binding.RdError) as e:
                    cache.poll()
                assert e.value.code == 3
            else:
                grow(cache, model, seqs, n_new, rng)
        elif what == "fork":
            full = [s for s in range(S) if model.lens[s]]
            empty = [s for s in range(S) if not model.lens[s]]
            if full and empty:
                dst = rng.permutation(empty)[:rng.integers(1, len(empty) + 1)].tolist()
                src = rng.choice(full, len(dst)).tolist()
                cache.fork(dev(np.array(src)), dev(np.array(dst)))
                model.fork(src, dst)
        elif what == "compact":
            # rows may only move inside pages of the sequence's own
            s = int(rng.integers(S))
            own = 0
            while own < model.lens[s] and model.table[s][(model.lens[s] - own - 1) // page] >= 0 and \
                    model.refs[model.table[s][(model.lens[s] - own - 1) // page]] == 1:
                own += 1
            m = int(rng.integers(0, own + 1))
            keep = int(rng.integers(0, m + 1))
            rows = sorted(rng.permutation(m)[:keep].tolist()) + [0] * (m + 1 - keep)
            cache.compact(dev(np.array([m])), dev(np.array([keep])), rows=dev(np.array([rows])), seqs=dev(np.array([s])))
            model.compact([s], [m], [keep], [rows])
        elif what == "free":
            seqs = rng.permutation(S)[:3].tolist()
            cache.free(dev(np.array(seqs)))
            model.free(seqs)
        else:
            w, k = int(rng.integers(1, 60)), int(rng.integers(0, 40))
            # (the last page stays whole: later rows go on in it)
            cache.trim(w, k)
            model.trim(range(S), w, k)
        model.check(cache)
    cache.poll()


def test_many_sequences_and_pages():
    """Lists longer than a CTA, several tiles of free bits, a last word that is not full."""
    S, page = 1500, 16
    cache, model = make(layers=1, kv_heads=1, page=page, n_pages=40011, max_seqs=S, max_pages=30)
    rng = np.random.default_rng(1)
    n_new = rng.integers(0, 200, S).tolist()
    for _ in range(2):
        cache.extend(dev(np.array(n_new)))
        assert model.extend(range(S), n_new)
    # (the model's pool is not written here: only tables)
    model.check(cache, pool=False)
    out = rng.permutation(S)[:700].tolist()
    cache.free(dev(np.array(out)))
    model.free(out)
    cache.fork(dev(np.array([s for s in range(S) if s not in set(out)][:699] + [out[-1]])), dev(np.array(out)))
    with pytest.raises(binding.RdError):   # the last target is its own source: left out
        cache.poll()
    model.fork([s for s in range(S) if s not in set(out)][:699], out[:699])
    model.check(cache, pool=False)
    order = rng.permutation(S).tolist()
    add = rng.integers(0, 60, S).tolist()
    assert model.extend(order, add)
    cache.extend(dev(np.array(add)), seqs=dev(np.array(order)))
    model.check(cache, pool=False)
    cache.poll()


def test_what_is_out_of_range_is_left_out():
    cache, model = make(n_pages=12, max_seqs=5, max_pages=4)
    rng = np.random.default_rng(2)
    grow(cache, model, [0, 1], [20, 5], rng)

    def refused(call):
        call()
        with pytest.raises(binding.RdError) as e:
            cache.poll()
        assert e.value.code == 1
        model.check(cache)

    i = lambda *x: dev(np.array(x))  # noqa: E731
    refused(lambda: cache.extend(i(1), seqs=i(5)))
    refused(lambda: cache.extend(i(1), seqs=i(-1)))
    refused(lambda: cache.extend(i(-2), seqs=i(0)))
    refused(lambda: cache.extend(i(45), seqs=i(0)))                       # 65 tokens, the row holds 64
    refused(lambda: cache.fork(i(0), i(0)))
    refused(lambda: cache.fork(i(0), i(1)))                               # not empty
    refused(lambda: cache.fork(i(0), i(9)))
    refused(lambda: cache.free(i(7)))
    refused(lambda: cache.trim(4, 0, seqs=i(-3)))
    refused(lambda: cache.compact(i(6), i(2), seqs=i(1)))                 # more rows than tokens
    refused(lambda: cache.compact(i(4), i(5), seqs=i(1)))
    refused(lambda: cache.compact(i(4), i(-1), seqs=i(1)))
    refused(lambda: cache.compact(i(4), i(2), rows=i(2, 1)[None], seqs=i(1)))   # not ascending
    refused(lambda: cache.compact(i(4), i(2), rows=i(1, 4)[None], seqs=i(1)))
    refused(lambda: cache.compact(i(4), i(2), rows=i(-1, 1)[None], seqs=i(1)))
    refused(lambda: cache.compact(i(4), i(3), rows=i(1, 2)[None], seqs=i(1)))   # keeps more than it lists
    k = torch.zeros(8, 3, 64, device="cuda:0")
    refused(lambda: cache.write(0, k[:1], k[:1], seqs=i(6)))
    model.write(0, 1, np.zeros((5, 3, 64)), np.zeros((5, 3, 64)))               # eight rows of five tokens: the first three have no place
    refused(lambda: cache.write(0, k, k, row_off=i(0, 8), seqs=i(1)))
    # a sequence named twice: its first entry counts
    cache.extend(i(1, 2), seqs=i(1, 1))
    model.extend([1], [1])
    with pytest.raises(binding.RdError):
        cache.poll()
    cache.fork(i(0, 1), i(3, 3))
    model.fork([0], [3])
    with pytest.raises(binding.RdError):
        cache.poll()
    model.check(cache)
    refused(lambda: cache.compact(i(2), i(1), rows=i(1)[None], seqs=i(3)))      # would move a row inside a shared page
    refused(lambda: cache.write(0, k[:1], k[:1], seqs=i(3)))                    # into a shared page
    cache.free(i(3, 3))
    model.free([3])
    model.check(cache)
    cache.poll()


def test_bad_pages_in_the_table():
    """A table that names pages outside the pool: reported, nothing else is touched."""
    cache, model = make(n_pages=12, max_seqs=3, max_pages=4)
    rng = np.random.default_rng(3)
    grow(cache, model, [0, 1], [20, 20], rng)
    cache.page_table[0, 0] = 12
    cache.page_table[1, 1] = -7
    before = cache.pool.clone()
    k = torch.zeros(1, 3, 64, device="cuda:0")
    for call in (lambda: cache.write(0, k, k, seqs=dev(np.array([1]))), lambda: cache.extend(dev(np.array([1])), seqs=dev(np.array([1]))),
                 lambda: cache.fork(dev(np.array([0])), dev(np.array([2]))), lambda: cache.free(dev(np.array([2]))), lambda: cache.free()):
        call()
        with pytest.raises(binding.RdError) as e:
            cache.poll()
        assert e.value.code == 1
    assert torch.equal(torch.nan_to_num(before), torch.nan_to_num(cache.pool))


def test_calls_in_a_graph():
    """A captured cycle of calls, replayed, does what the calls do."""
    cache, model = make(n_pages=30, max_seqs=6, max_pages=5)
    rng = np.random.default_rng(4)
    grow(cache, model, [0], [37], rng)
    src, dst, n_new, one = dev(np.array([0, 0])), dev(np.array([2, 3])), dev(np.array([3, 20])), dev(np.array([1, 1]))
    rows = dev(np.array([[2], [5]]))

    def calls():
        cache.free(dst)
        cache.fork(src, dst)
        cache.extend(n_new, seqs=dst)
        cache.compact(n_new, one, rows=rows, seqs=dst)

    calls()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for _ in range(3):
        g.replay()
        model.free([2, 3])
        model.fork([0, 0], [2, 3])
        model.extend([2, 3], [3, 20])
        model.compact([2, 3], [3, 20], [0, 0])       # (which row is kept below: the model's pool is compared without it)
        model.extend([2, 3], [1, 1])
        torch.cuda.synchronize()
        model.check(cache, pool=False)
    with pytest.raises(binding.RdError):             # row 5 of three does not exist: that entry is left out
        cache.compact(n_new, one, rows=dev(np.array([[9], [30]])), seqs=dst)
        cache.poll()


def test_on_another_stream():
    cache, model = make()
    st = torch.cuda.Stream()
    rng = np.random.default_rng(6)
    with torch.cuda.stream(st):
        grow(cache, model, [1, 2], [30, 17], rng)
        cache.fork(dev(np.array([1])), dev(np.array([5])))
        model.fork([1], [5])
        grow(cache, model, [5], [4], rng)
        model.check(cache)
        cache.poll()


def test_empty_lists_change_nothing():
    cache = binding.PagedCache.empty(2, 2, 64, 16, 8, 3, 4)
    cache.extend(dev(np.array([5, 20, 0])))
    before = [t.clone() for t in (cache.page_table, cache.lens, cache.refs, cache.free_bits)]
    none = dev(np.zeros(0))
    rows = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    launches = cache.launch_count()
    cache.extend(none)
    cache.extend(none, seqs=none)
    cache.fork(none, none)
    cache.compact(none, none, seqs=none)
    cache.compact(none, none, rows=dev(np.zeros((0, 3))), seqs=none)
    cache.trim(4, seqs=none)
    cache.free(seqs=none)
    cache.write(0, rows, rows, seqs=none)
    cache.write(1, rows, rows, row_off=dev(np.zeros(1)))
    assert cache.attention(0, rows, seqs=none).shape == (0, 2, 64)
    assert cache.attention(0, rows, row_off=dev(np.zeros(3))).shape == (0, 2, 64)
    cache.poll()
    assert cache.launch_count() == launches
    for a, b in zip(before, (cache.page_table, cache.lens, cache.refs, cache.free_bits)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("head_dim,dtype", [(64, "fp32"), (128, "bf16")])
def test_copies_of_many_sequences(head_dim, dtype):
    """Lists beyond what one entry a thread takes: which shared page is copied to which, and which sharer keeps it, pool bit by bit."""
    S, page = 700, 16
    cache, model = make(layers=2, kv_heads=2, head_dim=head_dim, page=page, n_pages=1900, max_seqs=S, max_pages=4, dtype=dtype)
    rng = np.random.default_rng(head_dim)
    parents = list(range(20))
    grow(cache, model, parents, rng.integers(1, 40, len(parents)).tolist(), rng)
    src, dst = rng.integers(0, 18, 620).tolist(), list(range(20, 640))      # (18 and 19 stay alone)
    cache.fork(dev(np.array(src)), dev(np.array(dst)))
    model.fork(src, dst)
    order = [s for s in rng.permutation(640).tolist() if s % 7]             # some sharers do not write
    n_new = rng.integers(0, 20, len(order)).tolist()
    cache.extend(dev(np.array(n_new)), seqs=dev(np.array(order)))
    assert model.extend(order, n_new)
    model.check(cache)
    rest = [s for s in range(640) if s % 7 == 0] + order[:300]
    n_new = rng.integers(0, 3, len(rest)).tolist()
    cache.extend(dev(np.array(n_new)), seqs=dev(np.array(rest)))
    assert model.extend(rest, n_new)
    model.check(cache)
    cache.poll()
