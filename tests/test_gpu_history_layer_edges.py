"""Edges of the collaborative filter's layer on the GPU, against the definitions in 64 bits (tests/layer_oracle.py): rows past
the end of a history, values that are not finite, biases far from zero, many heads on one key head."""
import pytest

import layer_oracle as lo
import test_gpu_history_layer as base
from test_gpu_history_layer import case, draw, inputs, name_of, oracle_of, placed, plan_of, run_gpu

pytestmark = pytest.mark.gpu


# ---- rows past the end of a history -----------------------------------------------------------------------

PAST = [
    case("f32", 1, 70, 2, 1, 16, buckets=8, far=40), case("bf16", 2, 200, 2, 2, 64, causal=False, buckets=16, far=64, both=True),
    case("bf16", 66, 70, 2, 2, 20, buckets=8, far=40), case("f32", 1, 130, 2, 2, 128, cap=4.0, buckets=8, far=20),
    case("bf16", 1, 257, 4, 1, 128, buckets=32, far=128),
]


@pytest.mark.parametrize("c", PAST, ids=name_of)
def test_rows_past_the_end_have_no_weight_whatever_the_table_holds(c):
    """The last tile of a history without segments holds rows that are not there; exp of some entries overflows float32."""
    import torch
    from paper_2204_04179_amd import gram
    *data, table = inputs(torch, c, seed=31)
    table[:, ::2] += 100.0
    want = oracle_of(c, *data, table)
    got = run_gpu(torch, gram, c, *data, table)
    for n in got:
        lo.assert_within(got[n], want[n], n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_entry_of_the_table_that_no_pair_reaches_changes_nothing(dtype):
    import torch
    from paper_2204_04179_amd import gram
    c = case(dtype, 1, 200, 2, 2, 64, buckets=64, far=256)
    assert lo.bucket_list(255, 64, 256, False)[199] < 63 == lo.bucket_list(255, 64, 256, False)[255]
    *data, table = inputs(torch, c, seed=32)
    table[:, 63] = float("inf")
    want = oracle_of(c, *data, table)
    got = run_gpu(torch, gram, c, *data, table)
    for n in got:
        lo.assert_within(got[n], want[n], n)
