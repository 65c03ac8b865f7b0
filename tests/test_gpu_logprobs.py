"""Log probabilities of given tokens, entropy and most likely tokens against 64 bits."""
import math

import numpy as np
import pytest
import torch

from helpers import dev
from paper_2403_09919_b200 import binding

pytestmark = pytest.mark.gpu


def reference(logits, tokens, top, temperature):
    x = logits.double()
    y = x / temperature
    logp = torch.log_softmax(y, 1)
    p = logp.exp()
    ids = torch.sort(logits.float(), dim=1, descending=True, stable=True).indices[:, :top]
    return logp.gather(1, tokens.long()[:, None])[:, 0], -torch.special.xlogy(p, p).sum(1), ids, logp.gather(1, ids)


def check(logits, tokens, top, temperature=1.0, got=None):
    got = binding.token_logprobs(logits, tokens, top=top, temperature=temperature) if got is None else got
    lp, ent, ids, tlp = reference(logits, tokens, top, temperature)
    # y is formed from x and a rounded factor (2^-23 |y|), the sum's terms are off by their exponents' rounding (2^-23 |y - max|, at
    # weights e^(y - max): 2^-22 together) and by the exponential (2^-21); sums of up to V terms in a tree over 512 threads and a
    # thread's V / 2048 steps (2^-24 a step)
    y = (logits.double() / temperature).abs()
    y = torch.where(torch.isfinite(y), y, 0.0)
    sums = 2.0 ** -20 + (logits.shape[1] / 2048 + 20) * 2.0 ** -24
    scale = y.amax(1)
    tol = 2.0 ** -21 * scale + sums
    assert ((got["logprob"].double() - lp).abs() <= tol + 2.0 ** -22 * lp.abs()).all()
    # the entropy's second part is a mean of y - max
    assert ((got["entropy"].double() - ent).abs() <= 2 * tol + (2 * sums) * (1 + ent.abs() + scale)).all()
    if top:
        assert torch.equal(got["top_ids"].long(), ids)
        assert ((got["top_logprobs"].double() - tlp).abs() <= (tol + 2.0 ** -22 * scale)[:, None] + 2.0 ** -22 * tlp.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(1, 32000, 5), (7, 32000, 20), (400, 32000, 64), (3, 1000, 64), (5, 64, 64), (2, 1, 1), (9, 17, 3),
                                            (1, 151937, 20), (33, 50257, 10), (600, 5003, 0), (2, 8191, 1), (150, 257, 40)])
def test_against_64_bits(dtype, rows, vocab, top):
    gen = torch.Generator("cuda:0").manual_seed(vocab + rows)
    logits = (torch.randn(rows, vocab, generator=gen, device="cuda:0") * 3).to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda:0").to(torch.int32)
    check(logits, tokens, top)
    check(logits, tokens, top, 0.7)


@pytest.mark.parametrize("vocab", [500, 32000, 131072])
@pytest.mark.parametrize("rows", [2, 300])
def test_equal_logits_come_lowest_id_first(rows, vocab):
    """All equal; a few values only; sorted up and down (one thread group holds what is largest); -0 and 0."""
    top = 50
    tokens = dev(np.arange(rows) % vocab)
    check(torch.full((rows, vocab), 2.5, device="cuda:0"), tokens, top)
    gen = torch.Generator("cuda:0").manual_seed(1)
    check(torch.randint(0, 3, (rows, vocab), generator=gen, device="cuda:0").float(), tokens, top)
    ramp = torch.arange(vocab, device="cuda:0").float().expand(rows, vocab) / vocab * 10
    check(ramp.contiguous(), tokens, top)
    check((-ramp).contiguous(), tokens, top)
    zeros = torch.zeros(rows, vocab, device="cuda:0")
    zeros[:, ::2] = -0.0
    check(zeros, tokens, top)
    # the largest ones lie together in one thread's pieces
    x = torch.randn(rows, vocab, generator=gen, device="cuda:0")
    step = 4 * 512
    for a in range(0, vocab, step):
        x[:, a:a + 4] += 20
    check(x, tokens, top)


def test_masked_and_far_logits():
    V = 32000
    gen = torch.Generator("cuda:0").manual_seed(3)
    x = torch.randn(6, V, generator=gen, device="cuda:0")
    x[0, 10:] = -math.inf                     # ten tokens left
    x[1, :] = -math.inf
    x[1, 777] = -3.0                          # one token left: entropy 0
    x[2] = x[2] * 1000                        # one token takes all
    x[3] = torch.finfo(torch.float32).min     # the type's lowest value everywhere but in two places
    x[3, 5], x[3, 31999] = 1.0, 1.0
    x[4] -= 1e4
    x[5, ::2] = -math.inf
    tokens = dev(np.array([3, 777, 9, 5, 100, 1]))
    check(x[[0, 2, 4, 5]].contiguous(), tokens[[0, 2, 4, 5]].contiguous(), 10)
    got = binding.token_logprobs(x, tokens, top=2)
    assert got["logprob"][1] == 0 and got["entropy"][1] == 0 and got["top_ids"][1].tolist() == [777, 0]
    assert got["top_logprobs"][1].tolist() == [0, -math.inf]
    assert abs(float(got["logprob"][3]) + math.log(2)) < 1e-6 and abs(float(got["entropy"][3]) - math.log(2)) < 1e-6
    assert got["top_ids"][3].tolist() == [5, 31999]
    # a given token of probability 0
    got = binding.token_logprobs(x[:1].contiguous(), dev(np.array([20])))
    assert got["logprob"][0] == -math.inf


def test_rows_without_a_distribution():
    V = 5000
    x = torch.randn(4, V, device="cuda:0")
    x[0, 40], x[0, 41] = math.nan, 9.0
    x[1, 7], x[1, 3000] = math.inf, 50.0
    x[2] = -math.inf
    got = binding.token_logprobs(x, dev(np.array([1, 1, 1, V])), top=3)
    assert torch.isnan(got["logprob"]).all()                      # (the last: a token outside the vocabulary)
    assert torch.isnan(got["entropy"][:3]).all() and torch.isfinite(got["entropy"][3])
    assert got["top_ids"][0, :2].tolist() == [40, 41] and got["top_ids"][1, :2].tolist() == [7, 3000]
    assert got["top_ids"][2].tolist() == [0, 1, 2]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_offsets_and_row_lists(dtype):
    """Rows that begin anywhere, and rows picked from the logits in any order, some of them not there."""
    gen = torch.Generator("cuda:0").manual_seed(8)
    buf = torch.randn(13, 7003, generator=gen, device="cuda:0").to(dtype)
    for off in (0, 1, 3, 6):
        x = buf[:, off:off + 6990]
        tokens = torch.randint(0, 6990, (13,), generator=gen, device="cuda:0").to(torch.int32)
        check(x, tokens, 9)
    x = buf[:, 1:6990]
    pick = [4, 0, 12, 4, -1, 13]
    tokens = dev(np.array([5, 6, 7, 8, 9, 10]))
    got = binding.token_logprobs(x, tokens, top=4, rows=dev(np.array(pick)))
    check(x[[4, 0, 12, 4]], tokens[:4].contiguous(), 4, got={k: v[:4] for k, v in got.items()})
    for k in ("logprob", "entropy", "top_logprobs"):
        assert torch.isnan(got[k][4:]).all()
    assert (got["top_ids"][4:] == -1).all()


def test_in_a_graph_and_on_another_stream():
    x = torch.randn(20, 32000, device="cuda:0")
    tokens = dev(np.arange(20))
    want = binding.token_logprobs(x, tokens, top=5)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = binding.token_logprobs(x, tokens, top=5)
    for _ in range(2):
        for v in got.values():
            v.zero_()
        g.replay()
        for k in want:
            assert torch.equal(want[k], got[k])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = binding.token_logprobs(x, tokens, top=5)
        st.synchronize()
    for k in want:
        assert torch.equal(want[k], got[k])


def test_refusals():
    x = torch.randn(4, 100, device="cuda:0")
    t = dev(np.arange(4))
    for kw in (dict(top=65), dict(top=101), dict(top=-1), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf)):
        with pytest.raises(binding.RdError) as e:
            binding.token_logprobs(x, t, **kw)
        assert e.value.code in (1, 2)
    with pytest.raises(ValueError):
        binding.token_logprobs(x.half(), t)
    with pytest.raises(ValueError):
        binding.token_logprobs(x.T, dev(np.arange(100)))
    with pytest.raises(ValueError):
        binding.token_logprobs(x, t.long())
    with pytest.raises(ValueError):
        binding.token_logprobs(x, t[:3])
    with pytest.raises(RuntimeError):
        binding.token_logprobs(x.cpu(), t)
    assert binding.token_logprobs(x[:0], t[:0], top=3)["top_ids"].shape == (0, 3)


def test_calls_on_two_streams_at_once():
    logits = [torch.randn(300, 40000, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(k)) for k in range(2)]
    want = [binding.token_logprobs(x, top=8) for x in logits]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in logits]
    for _ in range(5):
        got = []
        for stream, x in zip(streams, logits):
            with torch.cuda.stream(stream):
                got.append(binding.token_logprobs(x, top=8))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(a[k], b[k]) for k in b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [9, 5000, 32000, 131072])
def test_nan_in_the_first_place_and_everywhere(dtype, vocab):
    """NaN stands above all, lowest id first, the first id among them too; all ids are ids of the vocabulary."""
    top = min(vocab, 12)
    x = torch.randn(5, vocab, generator=torch.Generator("cuda:0").manual_seed(vocab), device="cuda:0").to(dtype)
    x[0, 0] = math.nan
    x[1] = math.nan
    x[2, 0], x[2, vocab - 1], x[2, 3] = math.nan, math.nan, math.inf
    x[3, 0], x[3, 1:] = math.nan, -math.inf
    x[4, 0] = math.inf
    got = binding.token_logprobs(x, dev(np.zeros(5)), top=top)
    want = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(got["top_ids"].long(), want)
    for k in ("logprob", "entropy", "top_logprobs"):
        assert torch.isnan(got[k]).all()
