"""Prompts and autoregressive steps of the engine on a cache in pages, and the log probabilities of what its calls emit: the
operators as a server runs them together (a shared prompt, sequences that branch off it, a window that gives pages back)."""
import numpy as np
import pytest
import torch

from helpers import Rig, dev
from paper_2403_09919_b200 import binding, synth
from oracle import redrafter_oracle as ora

pytestmark = pytest.mark.gpu

# 128 dimensions a head, odd tile counts everywhere; and 64 dimensions a head
CFG = dict(synth.CONFIGS["tiny"], dtype="bf16", d_model=512, n_heads=4, d_ffn=1376, vocab=1000, d_rnn=512, max_batch=4, max_ctx=400,
           beam_width=4, beam_length=4)
CFG64 = dict(CFG, n_heads=8)


def rel_err(got, ref):
    return float((np.abs(got - ref) / np.abs(ref).max(axis=-1, keepdims=True)).max())


def pages_for(cfg, page=16, n_pages=120, max_seqs=8, max_pages=40):
    hd = cfg["d_model"] // cfg["n_heads"]
    cache = binding.PagedCache.empty(cfg["n_layers"], cfg["n_heads"], hd, page, n_pages, max_seqs, max_pages)
    cache.pool.fill_(float("nan"))
    return cache


def visible(n, window, sinks):
    j, p = np.arange(n)[None], np.arange(n)[:, None]
    seen = j <= p
    return seen & ((j > p - window) | (j < sinks)) if window else seen


def oracle_logits(r, tokens, window=0, sinks=0):
    """Logits after every token of a sequence, from one pass over all of them with the window as its mask."""
    cfg = dict(r.cfg, max_ctx=len(tokens))
    kv = ora.KVCache(cfg["n_layers"], len(tokens), cfg["n_heads"], r.hd, r.odt)
    return ora.llm_forward(r.W, cfg, np.asarray(tokens), np.arange(len(tokens)), visible(len(tokens), window, sinks), kv, 0, r.odt)[1]


@pytest.mark.parametrize("cfg,page,window,sinks", [(CFG, 16, 0, 0), (CFG, 64, 0, 0), (CFG, 32, 40, 3), (CFG, 16, 100, 0), (CFG64, 16, 0, 0), (CFG64, 64, 24, 2)])
def test_prompts_and_steps_on_pages_against_the_oracle(cfg, page, window, sinks):
    r = Rig(cfg=cfg)
    cache = pages_for(cfg, page)
    rng = np.random.default_rng(page + window)
    lens = [70, 33, 1, 130]
    prompts = [rng.integers(0, cfg["vocab"], size=n) for n in lens]
    forced = rng.integers(0, cfg["vocab"], size=(4, 6))
    seqs = dev(np.array([5, 0, 7, 2]))
    r.eng.use_pages(cache, seqs, window, sinks)
    r.eng.prefill(prompts)
    after_prompt = r.eng.last_logits(4).cpu().numpy()
    steps = []
    for t in range(forced.shape[1]):
        r.eng.set_state(None, dev(forced[:, t]), None)
        r.eng.ar_step()
        steps.append(r.eng.last_logits(4).cpu().numpy())
    r.eng.poll()
    cache.poll()
    assert r.eng.route_counts()["att_pages"] == cfg["n_layers"] * (1 + forced.shape[1])
    assert cache.lens.tolist() == [39, 0, 136, 0, 0, 76, 0, 7]
    for b in range(4):
        ref = oracle_logits(r, np.concatenate([prompts[b], forced[b]]), window, sinks)
        assert rel_err(after_prompt[b], ref[lens[b] - 1]) < 3e-2
        for t in range(forced.shape[1]):
            assert rel_err(steps[t][b], ref[lens[b] + t]) < 3e-2


def test_a_prompt_of_several_passes_on_pages():
    """Rows of a later pass attend to pages that earlier passes filled; the contiguous cache gives the same logits."""
    cfg = dict(CFG, max_batch=2, max_ctx=2700)
    r = Rig(cfg=cfg)
    prompts = [np.random.default_rng(1).integers(0, cfg["vocab"], size=n) for n in (2600, 300)]
    r.eng.prefill(prompts)
    want = r.eng.last_logits(2).cpu().numpy()
    cache = pages_for(cfg, 64, n_pages=50, max_seqs=2, max_pages=45)
    r.eng.use_pages(cache)
    r.eng.prefill(prompts)
    got = r.eng.last_logits(2).cpu().numpy()
    r.eng.poll()
    cache.poll()
    assert cache.lens.tolist() == [2600, 300]
    assert rel_err(got, want) < 3e-2      # two kernels of the same arithmetic: two layers' storage noise
    r.eng.use_pages(None)
    r.eng.prefill(prompts)
    assert np.array_equal(r.eng.last_logits(2).cpu().numpy(), want)


def test_sequences_branch_off_a_shared_prompt():
    """One prompt is run once; three sequences share its pages, go on with different tokens, one is given up and its place taken
    by a branch of another."""
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16)
    rng = np.random.default_rng(3)
    prompt = rng.integers(0, CFG["vocab"], size=53)
    r.eng.use_pages(cache)
    r.eng.prefill([prompt])
    used = int((cache.refs > 0).sum())
    cache.fork(dev(np.array([0, 0])), dev(np.array([1, 2])))
    assert int((cache.refs > 0).sum()) == used
    forced = rng.integers(0, CFG["vocab"], size=(3, 8))
    r.eng.set_state(dev(np.full(3, 53)), dev(forced[:, 0]), None, batch=3, ctx_bound=53)
    hist = [list(prompt) for _ in range(3)]
    for t in range(8):
        if t == 4:     # sequence 2 is given up; its place is taken by a branch of sequence 1
            cache.free(dev(np.array([2])))
            cache.fork(dev(np.array([1])), dev(np.array([2])))
            hist[2] = list(hist[1])
        r.eng.set_state(None, dev(forced[:, t]), None, batch=3)
        r.eng.ar_step()
        for b in range(3):
            hist[b].append(forced[b, t])
    got = r.eng.last_logits(3).cpu().numpy()
    r.eng.poll()
    cache.poll()
    for b in range(3):
        assert rel_err(got[b], oracle_logits(r, hist[b])[-1]) < 3e-2
    cache.free()
    assert int(cache.refs.sum()) == 0


def test_trimmed_pages_change_nothing():
    """With a window, pages behind it can be given back after every step: same logits, and the pool stays small."""
    window, sinks = 30, 2
    rng = np.random.default_rng(5)
    prompt, forced = rng.integers(0, CFG["vocab"], size=100), rng.integers(0, CFG["vocab"], size=(1, 60))
    runs = []
    for trim in (False, True):
        r = Rig(cfg=dict(CFG, max_batch=1))
        cache = pages_for(CFG, 16, n_pages=12)
        r.eng.use_pages(cache, None, window, sinks)
        r.eng.prefill([prompt])
        logits, most = [], 0
        for t in range(60):
            if trim:
                cache.trim(window, sinks)
            r.eng.set_state(None, dev(forced[:, t]), None)
            r.eng.ar_step()
            logits.append(r.eng.last_logits(1))
            most = int((cache.refs > 0).sum())
        r.eng.poll()
        cache.poll()
        runs.append(torch.cat(logits))
        assert most <= (5 if trim else 10)
    assert torch.equal(*runs)


def test_a_captured_step_on_pages():
    """A graph of autoregressive steps makes room, writes and attends; its replays continue where the one before ended."""
    cfg = dict(CFG, max_batch=2)
    prompts = [np.random.default_rng(7).integers(0, cfg["vocab"], size=n) for n in (40, 61)]
    ends = []
    for graph in (False, True):
        r = Rig(cfg=cfg)
        cache = pages_for(cfg, 16)
        r.eng.use_pages(cache)
        r.eng.prefill(prompts)
        r.eng.ar_step()
        torch.cuda.synchronize()
        tokens = torch.zeros(2, dtype=torch.int32, device="cuda:0")
        if graph:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                r.eng.ar_step(tokens)
            for _ in range(20):
                g.replay()
            r.eng.set_ctx_bound(82)
        else:
            for _ in range(20):
                r.eng.ar_step(tokens)
        r.eng.poll()
        cache.poll()
        ends.append((tokens.clone(), cache.lens.tolist(), r.eng.get_state()[0].tolist(), r.eng.last_logits(2)))
    assert torch.equal(ends[0][0], ends[1][0]) and ends[0][1:3] == ends[1][1:3]
    assert ends[0][2] == [61, 82] and torch.equal(ends[0][3], ends[1][3])


def test_refusals_and_reports():
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16, n_pages=6, max_seqs=3, max_pages=4)

    def refused(code, call):
        with pytest.raises(binding.RdError) as e:
            call()
        assert e.value.code == code

    refused(1, lambda: r.eng.use_pages(cache, None, -1))
    refused(2, lambda: r.eng.use_pages(pages_for(CFG64, 16)))
    refused(2, lambda: r.eng.use_pages(pages_for(dict(CFG, n_layers=3), 16)))
    refused(7, lambda: Rig().eng.use_pages(cache))                                    # the fp32 configuration
    refused(7, lambda: Rig(cfg=CFG, flags=binding.RD_FLAG_FORCE_SIMT).eng.use_pages(cache))
    r.eng.use_pages(cache)
    refused(3, lambda: r.eng.prefill([np.zeros(10, int)] * 4))                        # four sequences, a table of three
    refused(3, lambda: r.eng.prefill([np.zeros(65, int)]))                            # a row of the table holds 64
    r.eng.prefill([np.zeros(60, int)])
    refused(4, lambda: r.eng.step())
    refused(4, lambda: r.eng.draft())
    for _ in range(4):
        r.eng.ar_step()
    refused(3, lambda: r.eng.ar_step())                                               # 64 tokens
    r.eng.poll()
    cache.poll()
    # pages that do not hold a sequence's context
    cache.free()
    r.eng.set_state(dev(np.array([20])), dev(np.array([1])), None, batch=1, ctx_bound=20)
    r.eng.ar_step()
    refused(1, r.eng.poll)
    # too few free pages
    cache.free()
    r.eng.prefill([np.zeros(64, int), np.zeros(60, int)])
    refused(3, cache.poll)
    r.eng.use_pages(None)
    r.eng.prefill([np.zeros(10, int)])
    r.eng.step()
    try:
        r.eng.poll()
    except binding.RdError:      # (what the call without room left behind is cleared by the first poll)
        r.eng.poll()


def test_log_probabilities_of_what_a_call_emitted():
    """fp32: verification and autoregressive logits are the same, so every emitted token of a speculative step has the log
    probability that an autoregressive engine gives it at its position."""
    cfg = dict(synth.CONFIGS["tiny"], max_batch=2)
    spec, ar = Rig(cfg=cfg), Rig(cfg=cfg)
    rng = np.random.default_rng(11)
    prompts = [rng.integers(0, 1024, size=n) for n in (30, 44)]
    spec.eng.prefill(prompts)
    ar.eng.prefill(prompts)
    L = cfg["beam_length"]
    first = ar.eng.last_logprobs(top=4)
    a, b = spec.eng.last_logprobs(top=4), binding.token_logprobs(ar.eng.last_logits(2), ar.eng.get_state()[1], top=4)
    for k in first:
        assert torch.equal(first[k][:, 0], a[k][:, 0]) and torch.equal(first[k][:, 0], b[k])
        assert ((first[k][:, 1:] == -1) if k == "top_ids" else torch.isnan(first[k][:, 1:])).all()
    # what an autoregressive engine emits next, with its log probabilities
    tokens, ref = [], []
    for _ in range(3 * (L + 1)):
        t = torch.zeros(2, dtype=torch.int32, device="cuda:0")
        ar.eng.ar_step(t)
        got = ar.eng.last_logprobs(top=4, temperature=0.9)
        tokens.append(t)
        ref.append({k: v[:, 0].clone() for k, v in got.items()})
    at = [0, 0]
    for step in range(2):
        beams = np.stack([synth.plant_beams([int(tokens[at[s] + j][s]) for j in range(L)], cfg["beam_width"], L, 1024, rng, p=0.3) for s in range(2)])
        out = binding.AcceptOut(2, L, "cuda:0")
        spec.eng.step(dev(beams), out)
        got = spec.eng.last_logprobs(top=4, temperature=0.9)
        spec.eng.poll()
        for s in range(2):
            n = int(out.n_accept[s])
            for j in range(n + 1):
                want = ref[at[s] + j]
                assert int(out.tokens[s, j]) == int(tokens[at[s] + j][s]) == int(got["top_ids"][s, j, 0])
                for k in want:
                    assert torch.equal(got[k][s, j], want[k][s]), (k, s, j)
            for k in got:
                rest = got[k][s, n + 1:]
                assert ((rest == -1) if k == "top_ids" else torch.isnan(rest)).all()
            at[s] += n + 1
    assert max(at) > 2                                   # something was accepted
    # refused when the logits are of nothing that was emitted
    spec.eng.verify(spec.eng.pack(dev(beams)))
    with pytest.raises(binding.RdError) as e:
        spec.eng.last_logprobs()
    assert e.value.code == 4
    with pytest.raises(binding.RdError):
        ar.eng.last_logprobs(top=65)
    with pytest.raises(binding.RdError):
        ar.eng.last_logprobs(temperature=0.0)


def test_a_step_without_room_leaves_shared_pages_alone():
    """Two sequences share a partly filled page and no page is free: the one that would have to copy it first is not written."""
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16, n_pages=2, max_seqs=2, max_pages=4)
    prompt = np.random.default_rng(5).integers(0, CFG["vocab"], size=20)
    r.eng.use_pages(cache, dev(np.array([0, 1, 1, 1])))
    r.eng.prefill([prompt])
    cache.fork(dev(np.array([0])), dev(np.array([1])))
    cache.compact(dev(np.array([2])), dev(np.array([0])), seqs=dev(np.array([1])))      # 18 of the 20 tokens
    r.eng.poll()
    cache.poll()
    assert cache.lens.tolist() == [20, 18] and cache.refs.tolist() == [2, 2]
    before = cache.pool.clone()
    r.eng.use_pages(cache, dev(np.array([1, 0, 0, 0])))
    r.eng.set_state(dev(np.array([18])), dev(np.array([7])), None, batch=1, ctx_bound=18)
    r.eng.ar_step()
    with pytest.raises(binding.RdError):
        cache.poll()
    with pytest.raises(binding.RdError):
        r.eng.poll()
    assert torch.equal(cache.pool.view(torch.int16), before.view(torch.int16))
    assert cache.lens.tolist() == [20, 18]


def same(a, b):
    return all(torch.equal(torch.nan_to_num(a[k].float(), nan=7e9), torch.nan_to_num(b[k].float(), nan=7e9)) for k in a)


@pytest.mark.parametrize("kind", ["step", "ar_step"])
def test_log_probabilities_after_replays(kind):
    """What a replayed graph emitted, whatever the host's last call was: a prompt, a verification."""
    cfg = dict(synth.CONFIGS["tiny"], max_batch=2)
    eager, rig = Rig(cfg=cfg), Rig(cfg=cfg)
    rng = np.random.default_rng(12)
    old, new = ([rng.integers(0, 1024, size=n) for n in lens] for lens in ((20, 31), (40, 9)))
    out = [binding.AcceptOut(2, cfg["beam_length"], "cuda:0") for _ in range(2)]
    token = [torch.zeros(2, dtype=torch.int32, device="cuda:0") for _ in range(2)]

    def call(r, i):
        r.eng.step(out=out[i]) if kind == "step" else r.eng.ar_step(token[i])

    rig.eng.prefill(old)
    call(rig, 0)
    torch.cuda.synchronize()
    before = rig.eng.last_logprobs(top=3)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(rig, 0)
    assert same(before, rig.eng.last_logprobs(top=3))      # capturing has emitted nothing
    rig.eng.prefill(new)
    eager.eng.prefill(new)
    assert same(rig.eng.last_logprobs(top=3), eager.eng.last_logprobs(top=3))
    for _ in range(2):
        g.replay()
        call(eager, 1)
        assert same(rig.eng.last_logprobs(top=3, temperature=0.9), eager.eng.last_logprobs(top=3, temperature=0.9))
    rig.eng.set_ctx_bound(60)
    beams, _ = rig.eng.draft()
    rig.eng.verify(rig.eng.pack(beams))
    nothing = rig.eng.last_logprobs(top=3)                 # (the host cannot know; the device does)
    assert torch.isnan(nothing["logprob"]).all() and (nothing["top_ids"] == -1).all()
    torch.cuda.synchronize()
    del g


def test_log_probabilities_of_a_graph_that_has_not_run():
    """A captured step fills nothing."""
    cfg = dict(synth.CONFIGS["tiny"], max_batch=2)
    r = Rig(cfg=cfg)
    r.eng.prefill([np.arange(20), np.arange(9)])
    beams, _ = r.eng.draft()
    r.eng.verify(r.eng.pack(beams))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.eng.step()
    got = r.eng.last_logprobs(top=2)
    assert torch.isnan(got["logprob"]).all() and torch.isnan(got["entropy"]).all() and (got["top_ids"] == -1).all()
    torch.cuda.synchronize()
    del g


@pytest.mark.parametrize("accept", ["accept", "accept_static"])
def test_log_probabilities_after_an_acceptance_of_the_callers(accept):
    """The acceptance of rows that the caller verified leaves another root, and of accepted tokens the handle's logits know nothing."""
    r = Rig(cfg=dict(synth.CONFIGS["tiny"], max_batch=2))
    prompts = [np.arange(20), np.arange(9)]
    r.eng.prefill(prompts)
    beams, _ = r.eng.draft()
    packed = r.eng.pack(beams)
    argmax, hidden, _ = r.eng.verify(packed)
    for before in (lambda: r.eng.prefill(prompts), r.eng.step, r.eng.ar_step):
        before()
        r.eng.last_logprobs()
        getattr(r.eng, accept)(beams, packed, argmax, hidden)
        with pytest.raises(binding.RdError) as e:
            r.eng.last_logprobs()
        assert e.value.code == 4


def test_pages_of_another_length_are_not_written():
    """A prompt into a sequence that is not empty, a context shorter than its pages: reported, and the pages stay as they are; the
    other sequences of the pass go on."""
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16)
    rng = np.random.default_rng(9)
    r.eng.use_pages(cache, dev(np.array([1, 2, 3, 4])))
    r.eng.prefill([rng.integers(0, CFG["vocab"], size=n) for n in (50, 23)])
    r.eng.poll()
    before = [t.clone() for t in (cache.pool.view(torch.int16), cache.page_table, cache.refs)]

    def unchanged(lens):
        with pytest.raises(binding.RdError) as e:
            r.eng.poll()
        assert e.value.code == 1
        cache.poll()
        assert cache.lens.tolist() == lens
        table = cache.page_table.tolist()
        held = [p for s in (1, 2) for p in table[s] if p >= 0]
        assert [t[:5] for t in table[1:3]] == [t[:5] for t in before[1].tolist()[1:3]]
        assert torch.equal(cache.pool.view(torch.int16)[:, :, held], before[0][:, :, held])

    r.eng.prefill([rng.integers(0, CFG["vocab"], size=n) for n in (20, 64, 30)])       # sequences 1 and 2 are not empty, 3 is
    unchanged([0, 50, 23, 30, 0, 0, 0, 0])
    r.eng.set_state(dev(np.array([30, 22, 30])), dev(np.array([1, 2, 3])), None, batch=3, ctx_bound=50)
    r.eng.ar_step()
    unchanged([0, 50, 23, 31, 0, 0, 0, 0])


def test_a_later_pass_of_a_prompt_that_was_left_out():
    """A prompt of several passes into a sequence that holds as many tokens as the first pass takes: all of it is left out."""
    cfg = dict(CFG, max_batch=1, max_ctx=2700)
    r = Rig(cfg=cfg)
    cache = pages_for(cfg, 64, n_pages=50, max_seqs=2, max_pages=45)
    rng = np.random.default_rng(10)
    r.eng.use_pages(cache)
    r.eng.prefill([rng.integers(0, cfg["vocab"], size=1024)])
    r.eng.poll()
    before = cache.pool.clone()
    r.eng.prefill([rng.integers(0, cfg["vocab"], size=1500)])
    with pytest.raises(binding.RdError):
        r.eng.poll()
    cache.poll()
    assert cache.lens.tolist() == [1024, 0]
    assert torch.equal(cache.pool.view(torch.int16), before.view(torch.int16))


def test_contexts_that_lie_in_pages_are_not_taken_for_the_handles_own():
    """Back on the handle's own cache, which holds nothing of what ran on pages: refused until a prompt or a state says otherwise."""
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16)
    prompt = np.arange(40)

    def refused(call):
        with pytest.raises(binding.RdError) as e:
            call()
        assert e.value.code == 4

    r.eng.prefill([prompt])
    own = r.eng.get_state()
    r.eng.use_pages(cache)
    r.eng.prefill([prompt])
    r.eng.use_pages(None)
    for call in (r.eng.step, r.eng.ar_step, r.eng.draft):
        refused(call)
    r.eng.use_pages(cache)
    r.eng.ar_step()                                   # the pages still hold it
    r.eng.use_pages(None)
    refused(r.eng.step)
    r.eng.set_state(None, own[1], None)               # (no contexts: those of the pages)
    refused(r.eng.step)
    r.eng.set_state(*own, ctx_bound=40)               # what the handle's own cache held before
    r.eng.step()
    r.eng.poll()
    cache.poll()
    r.eng.prefill([prompt])
    r.eng.use_pages(cache)                            # pages in use and not yet run on change nothing
    r.eng.use_pages(None)
    r.eng.step()
    r.eng.poll()


def test_a_closed_cache_is_refused():
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16)
    r.eng.use_pages(cache)
    r.eng.prefill([np.arange(10)])
    torch.cuda.synchronize()
    cache.close()
    for call in (lambda: r.eng.prefill([np.arange(10)]), r.eng.ar_step, lambda: r.eng.use_pages(cache)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(binding.RdError):
        cache.reset()
    r.eng.use_pages(None)
    r.eng.prefill([np.arange(10)])
    r.eng.step()
    r.eng.poll()


def test_contexts_set_while_pages_are_in_use_are_those_of_the_pages():
    """A branch's state belongs to the pages, though nothing has run on them since."""
    r = Rig(cfg=CFG)
    cache = pages_for(CFG, 16)
    r.eng.use_pages(cache)
    r.eng.prefill([np.arange(40)])
    cache.fork(dev(np.array([0])), dev(np.array([1])))
    r.eng.set_state(dev(np.array([40, 40])), dev(np.array([1, 2])), None, batch=2, ctx_bound=40)
    r.eng.use_pages(None)
    for call in (r.eng.step, r.eng.ar_step):
        with pytest.raises(binding.RdError) as e:
            call()
        assert e.value.code == 4
    r.eng.use_pages(cache)
    r.eng.ar_step()
    r.eng.poll()
    cache.poll()
    assert cache.lens.tolist()[:2] == [41, 41]
