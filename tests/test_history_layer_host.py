"""The collaborative filter's layer without a GPU: buckets of distances, work sizes, and refusals.  No kernel is launched:
every call here is refused, or has nothing to do."""
import ctypes as C

import pytest

import layer_oracle as lo
from paper_2204_04179_amd import gram


@pytest.mark.parametrize("buckets,far,both", [(32, 128, False), (32, 128, True), (1, 1, False), (2, 2, False), (2, 5, True),
                                              (3, 9, False), (64, 1 << 20, False), (64, 1 << 30, True), (12, 40, False), (16, 64, True),
                                              (7, 4, False), (64, 33, False)])
def test_buckets_of_distances(buckets, far, both):
    plan = gram.HistoryAttention(1, 1, 8, buckets=buckets, max_distance=far, two_sided=both)
    top = min(4 * far, 5000)
    side = lo.bucket_list(top, buckets, far, both)
    for n in range(top + 1):
        assert plan.bucket(n) == side[n], n
        after = side[n] + buckets // 2 if both else 0
        if n:
            assert plan.bucket(-n) == after, -n
    if far > 5000:                                            # around each border, decided in whole numbers
        h = buckets // 2 if both else buckets
        e = h // 2
        for b in range(1, h - e):
            lo_n, hi_n = e, 1 << 31
            while lo_n < hi_n:                                # the smallest n with (n / e)^(h - e) >= (far / e)^b
                mid = (lo_n + hi_n) // 2
                if mid ** (h - e) * e ** b >= far ** b * e ** (h - e):
                    hi_n = mid
                else:
                    lo_n = mid + 1
            assert (plan.bucket(lo_n - 1), plan.bucket(lo_n)) == (e + b - 1, e + b)
    assert gram.HistoryAttention(1, 1, 8).bucket(3) == -1


@pytest.mark.parametrize("change", [dict(heads=0), dict(heads=3, kv_heads=2), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=129),
                                    dict(dtype=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0),
                                    dict(cap=float("nan")), dict(buckets=-1), dict(buckets=65, max_distance=500), dict(buckets=8),
                                    dict(buckets=8, max_distance=4), dict(buckets=7, max_distance=50, two_sided=True),
                                    dict(buckets=8, max_distance=(1 << 30) + 1), dict(heads=65536, kv_heads=1)])
def test_settings_that_are_refused(change):
    with pytest.raises(gram.GramError) as e:
        gram.HistoryAttention(**{**dict(heads=2, kv_heads=2, head_dim=8), **change})
    assert e.value.status == gram.ERR_ARG and "gram_attention" in str(e.value)


def test_sizes_and_pointers_that_are_refused():
    lib = gram.load()
    plan = gram.HistoryAttention(2, 2, 8, buckets=4, max_distance=8)
    cfg = C.byref(plan.cfg)
    assert lib.gram_attention(None, 1, 1, None, None, None, None, None, None, None, None, None) == gram.ERR_ARG
    # sizes: a null work size, and a refusal that says why
    for batch, length in ((-1, 4), (1, -1), (1, 262145), (1 << 22, 128)):
        assert plan.backward_bytes(batch, length) == 0
        assert lib.gram_attention(cfg, batch, length, None, None, None, None, None, None, None, None, None) == gram.ERR_ARG
        assert b"gram_attention: " in lib.gram_last_error(None)
    assert plan.backward_bytes(0, 0) > 0 and plan.backward_bytes(3, 100) >= 3 * 2 * (100 + 2 * 4) * 4
    assert plan.step_bytes(1, 0) == 0 and plan.step_bytes(-1, 5) == 0 and plan.step_bytes(4, 8192) > plan.step_bytes(4, 64) > 0
    some = 1 << 20                                            # never dereferenced: each call is refused before a launch
    rows = lambda **k: C.byref(gram.GramRows(**{**dict(data=some, batch_stride=64, row_stride=16, head_stride=8), **k}))
    good = rows()

    def forward(q=good, k=good, v=good, o=good, prefix=None, table=some, plan=plan):
        return lib.gram_attention(C.byref(plan.cfg), 1, 4, q, k, v, o, None, prefix, table, None, None)

    assert forward(q=None) == forward(o=None) == forward(table=None) == forward(k=rows(data=None)) == gram.ERR_ARG
    assert b"NULL" in lib.gram_last_error(None)
    assert forward(q=rows(data=some + 1)) == gram.ERR_ARG and b"aligned" in lib.gram_last_error(None)
    assert forward(v=rows(row_stride=-16)) == forward(v=rows(row_stride=1 << 25)) == gram.ERR_ARG
    assert b"64 MiB" in lib.gram_last_error(None)
    both_ways = gram.HistoryAttention(2, 2, 8, causal=False)
    assert forward(prefix=some, table=None, plan=both_ways) == gram.ERR_ARG and b"prefix" in lib.gram_last_error(None)

    def backward(lse=some, work=some, dtable=None, table=some, plan=plan, dq=good):
        return lib.gram_attention_backward(C.byref(plan.cfg), 1, 4, good, good, good, good, lse, good, dq, good, good, None, None,
                                           table, dtable, work, None)

    assert backward(lse=None) == backward(work=None) == backward(work=some + 8) == backward(dq=None) == gram.ERR_ARG
    assert backward(dtable=some, table=None, plan=both_ways) == gram.ERR_ARG and b"buckets" in lib.gram_last_error(None)

    def step(lengths=some, work=some, capacity=8192, q=good, table=some):
        return lib.gram_attention_step(cfg, 1, capacity, q, good, good, good, good, lengths, None, table, good, work, None)

    assert step(lengths=None) == step(work=None) == step(work=some + 4) == step(capacity=0) == step(q=None) == gram.ERR_ARG
    assert lib.gram_attention_step(cfg, 0, 16, None, None, None, None, None, None, None, None, None, None, None) == gram.OK


def test_operands_whose_written_rows_overlap_are_refused():
    lib = gram.load()
    plan = gram.HistoryAttention(2, 2, 8)
    cfg, some = C.byref(plan.cfg), 1 << 20                    # never dereferenced
    rows = lambda b=64, r=16, h=8: C.byref(gram.GramRows(some, b, r, h))
    good, null = rows(), None
    for bad in (rows(b=0), rows(r=0), rows(h=0), rows(h=7), rows(b=4)):
        assert lib.gram_attention(cfg, 2, 4, good, good, good, bad, null, null, null, null, null) == gram.ERR_ARG
        assert b"overlap" in lib.gram_last_error(None)
        for at in range(3):
            out = [good] * 3
            out[at] = bad
            assert lib.gram_attention_backward(cfg, 2, 4, good, good, good, good, some, good, *out, null, null, null, null, some,
                                               null) == gram.ERR_ARG
            assert b"overlap" in lib.gram_last_error(None)
    for bad in (rows(b=0), rows(r=0), rows(h=0)):
        for caches in ((good, bad), (bad, good)):
            assert lib.gram_attention_step(cfg, 2, 4, good, good, good, *caches, some, null, null, good, some, null) == gram.ERR_ARG
            assert b"overlap" in lib.gram_last_error(None)
    # the stride of something that there is one of means nothing: only the missing pointer is to blame
    assert lib.gram_attention(cfg, 1, 4, good, good, null, rows(b=-5), null, null, null, null, null) == gram.ERR_ARG
    assert b"NULL" in lib.gram_last_error(None)
    # row numbers of a cache stay below 2^30
    assert plan.step_bytes(1, 1 << 30) > 0 and plan.step_bytes(1, (1 << 30) + 1) == 0
    assert lib.gram_attention_step(cfg, 1, 2147483647, good, good, good, good, good, some, null, null, good, some, null) == gram.ERR_ARG
    assert b"2^30" in lib.gram_last_error(None)


def test_layer_norm_refusals():
    lib = gram.load()
    some = 1 << 20

    def norm(x=some, xt=0, w=some, m=3, d=8, eps=1e-5, y=some, yt=1):
        return lib.gram_layer_norm(x, xt, w, some, None, m, d, eps, y, yt, None, None)

    for bad in (dict(m=-1), dict(d=0), dict(d=8193), dict(xt=2), dict(yt=-1), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(x=None), dict(w=None), dict(y=None)):
        assert norm(**bad) == gram.ERR_ARG, bad
        assert b"gram_layer_norm: " in lib.gram_last_error(None)
    assert norm(m=0, x=None) == gram.OK

    def back(stats=some, dw=some, work=some, d=8, m=3):
        return lib.gram_layer_norm_backward(some, 0, some, stats, some, 1, None, None, m, d, some, dw, some, work, None)

    assert back(stats=None) == back(dw=None) == back(work=None) == back(work=some + 2) == back(d=9000) == back(m=-2) == gram.ERR_ARG
    assert gram.layer_norm_work_bytes(-1, 8) == 0 and gram.layer_norm_work_bytes(5, 8193) == 0
    assert gram.layer_norm_work_bytes(0, 8) > 0 and gram.layer_norm_work_bytes(1 << 40, 8192) == 1024 * 2 * 8192 * 4


def test_tensors_that_are_refused_by_the_binding():
    import torch
    plan = gram.HistoryAttention(2, 1, 8, dtype=gram.F32)
    q, k = torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 1, 8)
    with pytest.raises(gram.GramError, match="current device"):
        plan.forward(q, k, k, q)                              # host memory
    for bad in (torch.zeros(1, 4, 1, 8), torch.zeros(1, 4, 2, 16)[..., ::2], q.bfloat16(), torch.zeros(4, 2, 8)):
        with pytest.raises(gram.GramError, match="forward: q|length, heads"):
            plan.forward(bad, k, k, q)
    with pytest.raises(gram.GramError, match="expected"):
        gram.layer_norm(torch.zeros(3, 8)[:, ::2], torch.zeros(4), torch.zeros(4), torch.zeros(3, 4))
    with pytest.raises(gram.GramError, match="q .batch, heads"):
        plan.step(q, k, k, k, k, None, q, None)


def test_each_thread_has_its_own_message():
    import threading
    lib = gram.load()
    lib.gram_layer_norm(None, 0, None, None, None, -1, 8, 0.0, None, 0, None, None)
    seen = []

    def other():
        lib.gram_attention(None, 1, 1, None, None, None, None, None, None, None, None, None)
        seen.append(lib.gram_last_error(None))

    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert b"cfg is NULL" in seen[0] and b"gram_layer_norm: m < 0" in lib.gram_last_error(None)
