"""A Batch shared by calls of different sizes that overlap in time (threads
with a context each): every call keeps the description that it was given.
And calls of more queries than their numbering holds (fake device addresses;
skipped where a GPU is present)."""
import ctypes as C
import threading

import pytest
import torch

from paper_2609_31938_amd import c3c, tokens

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer argument tests run on CPU-only hosts")
lib = c3c.lib


def shared():
    b = tokens.Batch.__new__(tokens.Batch)
    b._d = tokens._BatchDesc(1 << 20, 2 << 20, 3 << 20, 4, 5, 0, 7, 8)
    return b


def fields(ref):
    d = ref._obj
    return d.table, d.cu, d.len, d.B, d.cols, d.T, d.max_new, d.max_len


def test_a_call_keeps_its_rows():
    b = shared()
    calls = [(T, b._of(T)) for T in (3, 9, 9, 0, 3)]
    for T, ref in calls:
        assert fields(ref) == (1 << 20, 2 << 20, 3 << 20, 4, 5, T, 7, 8)


def test_threads_that_share_a_batch():
    b, wrong, start = shared(), [], threading.Barrier(4)

    def work(T):
        start.wait()
        for _ in range(20000):
            if fields(b._of(T))[5] != T:
                wrong.append(T)

    threads = [threading.Thread(target=work, args=(T,)) for T in (1, 2, 3, 4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@no_gpu
def test_columns_past_32_bits_are_refused():
    ctx = c3c.Context()
    for T, qh in (((1 << 30), 4), ((1 << 31) - 1, 2), ((1 << 29) - 512, 8)):
        b = tokens._BatchDesc(1 << 20, 2 << 20, 3 << 20, 1, 1, T, 1, 1)
        c = tokens._CacheDesc(4 << 20, 5 << 20, 6 << 20, 7 << 20, 1, 2, 16, 16)
        st = lib.c3c_paged_attention(ctx._h, C.byref(c), C.byref(b), 1, qh, 1 << 40, qh * 16, 0.1, 1, 0, 1 << 50, None, None)
        assert st == c3c.E_INVAL and "2^31" in ctx.last_error, (T, qh, ctx.last_error)
