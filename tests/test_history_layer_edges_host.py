"""Edges of the collaborative filter's layer that need no GPU: numbers that do not fit the library's, refused by the binding."""
import pytest

from paper_2204_04179_amd import gram

WIDE = 1 << 32                 # what a 32-bit field would take for zero


@pytest.mark.parametrize("change", [dict(heads=WIDE + 2), dict(kv_heads=WIDE + 2), dict(head_dim=WIDE + 8), dict(dtype=WIDE + 1),
                                    dict(buckets=WIDE), dict(buckets=WIDE + 8, max_distance=50), dict(buckets=8, max_distance=WIDE + 50),
                                    dict(heads=-WIDE + 2)])
def test_settings_beyond_32_bits_are_refused_not_wrapped(change):
    with pytest.raises(gram.GramError) as e:
        gram.HistoryAttention(**{**dict(heads=2, kv_heads=2, head_dim=8), **change})
    assert e.value.status == gram.ERR_ARG and "32 bits" in str(e.value)


def test_distances_beyond_32_bits_have_the_bucket_of_far_ones():
    plan = gram.HistoryAttention(1, 1, 8, buckets=16, max_distance=64, two_sided=True)
    assert plan.bucket(WIDE + 1) == plan.bucket((1 << 31) - 1) == 7 and plan.bucket(-WIDE - 1) == plan.bucket(-(1 << 31)) == 15


@pytest.mark.parametrize("sizes", [(WIDE + 1, 4), (1, WIDE + 4)])
def test_sizes_beyond_32_bits_have_no_work_buffer(sizes):
    plan = gram.HistoryAttention(1, 1, 8)
    assert plan.backward_bytes(*sizes) == 0 and plan.step_bytes(*sizes) == 0
    assert gram.layer_norm_work_bytes(4, sizes[1]) == (0 if sizes[1] > WIDE else gram.layer_norm_work_bytes(4, 4))


def test_tensors_of_more_rows_than_32_bits_hold_are_refused():
    import torch
    plan = gram.HistoryAttention(1, 1, 1, dtype=gram.F32)
    for shape in ((WIDE + 1, 1, 1, 1), (1, WIDE + 1, 1, 1)):
        q = torch.empty(shape, device="meta")
        for call in (lambda: plan.forward(q, q, q, q), lambda: plan.backward(q, q, q, q, None, q, q, q, q, None),
                     lambda: plan.step(q[:, 0], q[:, 0], q[:, 0], q, q, None, q[:, 0], None)):
            with pytest.raises(gram.GramError, match="32 bits"):
                call()
