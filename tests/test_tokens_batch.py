"""A Batch shared by calls of different sizes that overlap in time (threads
with a context each): every call keeps the description that it was given."""
import threading

from paper_2609_31938_amd import tokens


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
