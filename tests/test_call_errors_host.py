"""Messages of failing calls without a context, across threads.  No GPU is needed: every call here is refused."""
import threading

from paper_2204_04179_amd import gram


def in_thread(f):
    out = []
    t = threading.Thread(target=lambda: out.append(f()))
    t.start()
    t.join()
    return out[0]


def test_a_thread_without_an_error_of_its_own_reads_the_last_of_all_threads():
    lib = gram.load()
    read = lambda: lib.gram_last_error(None)
    assert in_thread(lambda: lib.gram_create(None, None)) == gram.ERR_ARG
    assert in_thread(read) == b"gram_create: out is NULL"

    def mine_then_anothers():
        lib.gram_layer_norm(None, 0, None, None, None, -1, 8, 0.0, None, 0, None, None)
        in_thread(lambda: lib.gram_create(None, None))
        return read()

    assert in_thread(mine_then_anothers) == b"gram_layer_norm: m < 0"
    assert in_thread(read) == b"gram_create: out is NULL"
