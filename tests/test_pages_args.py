"""Checks of the paged cache's and the log probabilities' arguments that need no GPU."""
import ctypes as C

import pytest
import torch

from paper_2403_09919_b200 import binding


def cache(**over):
    f = dict(n_layers=2, n_kv_heads=4, head_dim=128, dtype=1, page_size=64, n_pages=10, max_seqs=3, max_seq_pages=5)
    f.update(over)
    return binding.RdPageCache(struct_bytes=f.pop("struct_bytes", C.sizeof(binding.RdPageCache)), **f)


def test_sizes():
    L = binding.lib()
    assert L.redrafter_pages_pool_bytes(C.byref(cache())) == 2 * 2 * 10 * 4 * 64 * 128 * 2
    assert L.redrafter_pages_pool_bytes(C.byref(cache(dtype=0))) == 2 * 2 * 10 * 4 * 64 * 128 * 4
    assert L.redrafter_pages_workspace_bytes(C.byref(cache())) > 0
    for bad in (dict(struct_bytes=8), dict(n_layers=0), dict(n_kv_heads=-1), dict(head_dim=96), dict(dtype=2), dict(page_size=8), dict(page_size=48),
                dict(page_size=256), dict(n_pages=0), dict(max_seqs=0), dict(max_seq_pages=0), dict(n_pages=1 << 22)):
        assert L.redrafter_pages_pool_bytes(C.byref(cache(**bad))) == 0, bad
        assert L.redrafter_pages_workspace_bytes(C.byref(cache(**bad))) == 0, bad


def test_null_and_bad_arguments():
    L = binding.lib()
    h = C.c_void_p()
    buf = C.create_string_buffer(1024)
    at = (C.addressof(buf) + 255) // 256 * 256
    assert L.redrafter_pages_init(None, None, 0, None) == 1
    assert L.redrafter_pages_init(C.byref(cache()), at, 256, C.byref(h)) == 1           # null buffers
    full = dict(pool=at, page_table=at, lens=at, refs=at, free_bits=at)
    assert L.redrafter_pages_init(C.byref(cache(**full, head_dim=80)), at, 256, C.byref(h)) == 2
    assert L.redrafter_pages_init(C.byref(cache(**full)), at + 16, 1 << 20, C.byref(h)) == 1
    assert L.redrafter_pages_init(C.byref(cache(**full)), at, 100, C.byref(h)) == 3      # workspace too small
    assert b"workspace" in L.redrafter_pages_last_error(None)
    assert not h
    assert L.redrafter_pages_destroy(None) == 1
    for rc in (L.redrafter_pages_reset(None, None), L.redrafter_pages_extend(None, None, None, 0, None), L.redrafter_pages_fork(None, None, None, 0, None),
               L.redrafter_pages_compact(None, None, None, None, None, 0, 0, None), L.redrafter_pages_trim(None, None, 1, 0, 0, None),
               L.redrafter_pages_free(None, None, 0, None), L.redrafter_pages_write(None, 0, None, None, 0, 0, None, 0, None, 0, None),
               L.redrafter_pages_attention(None, 0, None, None, 0, 0, 0, 1, None, 0, None, 0, None, 0.0, 0, 0, None), L.redrafter_pages_poll(None, None)):
        assert rc == 1
    assert L.redrafter_pages_launch_count(None) == 0


def test_log_probabilities():
    L = binding.lib()
    assert L.redrafter_token_logprobs(None, None) == 1
    ok = dict(struct_bytes=C.sizeof(binding.RdLogprobs), dtype=0, rows=2, n_logit_rows=2, vocab=100, top=0, temperature=1.0, row_stride=100, logits=4096)
    for bad, code in ((dict(struct_bytes=4), 1), (dict(dtype=5), 1), (dict(vocab=0), 1), (dict(rows=-1), 1), (dict(rows=3), 1), (dict(top=65), 2), (dict(top=-1), 2),
                      (dict(vocab=10, row_stride=10, top=11), 2), (dict(temperature=0.0), 1), (dict(temperature=1e-40), 1), (dict(row_stride=99), 2), (dict(logits=None), 1), (dict(logits=4097), 1),
                      (dict(logprob=4096), 1), (dict(top=1), 1)):
        assert L.redrafter_token_logprobs(C.byref(binding.RdLogprobs(**dict(ok, **bad))), None) == code, bad
    assert L.redrafter_token_logprobs(C.byref(binding.RdLogprobs(**dict(ok, rows=0))), None) == 0


def test_there_is_no_cpu_path():
    t = torch.zeros(4, 10)
    with pytest.raises(RuntimeError):
        binding.token_logprobs(t)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        binding.PagedCache(torch.zeros(1, 2, 1, 1, 16, 64), i, i[0], i[0], i[0])


def test_sizes_that_do_not_fit_what_the_kernels_count_in():
    """Entries of the table, and a sequence's tokens times its heads (two at least), below 2^31."""
    L = binding.lib()
    for bad, good in ((dict(max_seqs=1 << 16, max_seq_pages=1 << 15), dict(max_seqs=(1 << 16) - 1, max_seq_pages=1 << 15, page_size=16)),
                      (dict(max_seq_pages=1 << 23), dict(max_seq_pages=(1 << 23) - 1)),                          # 2^29 tokens of 4 heads
                      (dict(n_kv_heads=1, max_seq_pages=1 << 24), dict(n_kv_heads=1, max_seq_pages=(1 << 24) - 1))):   # 2^30 tokens
        assert L.redrafter_pages_workspace_bytes(C.byref(cache(**bad))) == 0, bad
        assert L.redrafter_pages_workspace_bytes(C.byref(cache(**good))) > 0, good


def test_a_temperature_whose_reciprocal_in_base_two_is_no_number():
    L = binding.lib()
    a = binding.RdLogprobs(struct_bytes=C.sizeof(binding.RdLogprobs), dtype=0, rows=1, n_logit_rows=1, vocab=8, temperature=3.2e-39, row_stride=8, logits=4096)
    assert L.redrafter_token_logprobs(C.byref(a), None) == 1
