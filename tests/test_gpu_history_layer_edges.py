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


# ---- values that are not finite ---------------------------------------------------------------------------


def check_spoilt(c, at, what, odd, prefix=None, segments=None):
    """Position `at` of every history holds the value `odd` in the operand `what` (or in all).  Rows that have nothing to do
    with it are what the definition has for them; every gradient that it enters is not finite in any head."""
    import torch
    from paper_2204_04179_amd import gram
    q, k, v, do, _, _, table = inputs(torch, c, seed=100)
    B, L = c["B"], c["L"]
    pre = None if prefix is None else torch.tensor([prefix[b % len(prefix)] for b in range(B)], dtype=torch.int32)
    seg = None if segments is None else torch.full((B, L), segments, dtype=torch.int32)
    clean = [t.clone() for t in (q, k, v, do)]
    for n, t, z in zip(("q", "k", "v", "do"), (q, k, v, do), clean):
        if what in (n, "all"):
            t[:, at], z[:, at] = odd, 0.0
    bad = torch.zeros(B, L, dtype=torch.bool)
    bad[:, at] = True
    want = oracle_of(c, *clean, seg, pre, table)
    got = {n: t.cpu() for n, t in run_gpu(torch, gram, c, q, k, v, do, seg, pre, table).items()}
    see = lo.visible(L, seg, c["causal"], pre, B)[:, 0].expand(B, L, L)               # [B, query, key]
    held = bad if what in ("k", "v", "all") else torch.zeros_like(bad)
    row = (see & held[:, None, :]).any(2) | (bad if what in ("q", "all") else False)   # queries without a result
    grow = row | (bad if what == "do" else False)                                     # and without gradients
    gkey = (see & grow[:, :, None]).any(1)                                            # keys that those see
    for n, spoilt in (("o", row), ("dq", grow), ("dk", gkey), ("dv", gkey)):
        value, bound = want[n]
        lo.assert_within(got[n][~spoilt], (value[~spoilt], bound[~spoilt]), f"{n} of the others")
        if (n, what) != ("dv", "v"):                       # dv is made of weights and do: a value has no part in it
            finite = torch.isfinite(got[n][spoilt].float()).all(-1)
            assert not bool(finite.any()), f"{n}: {int(finite.sum())} of {finite.numel()} rows and heads are finite"
    if table is not None:
        i = torch.arange(L)
        of = lo.buckets_of(i[:, None] - i[None, :], c["buckets"], c["far"], c["both"])
        reached = torch.zeros(c["buckets"], dtype=torch.bool)
        reached[of[(see & grow[:, :, None]).any(0)]] = True
        assert not bool(torch.isfinite(got["dtable"][:, reached]).any()), "dtable"


# A prefix that ends within a tile: some waves of a block see all of a tile and others do not.
INSIDE = [
    (case("bf16", 1, 200, 2, 1, 64, prefix=True), (40,), 20), (case("bf16", 1, 200, 2, 1, 64, prefix=True), (40,), 50),
    (case("f32", 2, 200, 2, 2, 20, prefix=True, buckets=8, far=30, both=True), (100, 40), 33),
    (case("bf16", 70, 130, 2, 2, 128, prefix=True), (100, 40, 127), 70),
    (case("f32", 1, 300, 4, 2, 128, prefix=True, cap=5.0), (100,), 110),
]


@pytest.mark.parametrize("what", ["k", "v", "q", "do", "all"])
@pytest.mark.parametrize("c,prefix,at", INSIDE, ids=lambda p: name_of(p) if isinstance(p, dict) else str(p))
def test_non_finite_values_where_a_prefix_ends_within_a_tile(c, prefix, at, what):
    check_spoilt(c, at, what, float("nan"), prefix=prefix)
    if what in ("do", "v"):
        check_spoilt(c, at, what, float("inf"), prefix=prefix)


# One whole tile, all of it visible: no padding, one session or none, every position within the prefix.
WHOLE = [
    (case("bf16", 2, 64, 2, 1, 64, causal=False, buckets=8, far=30, both=True), None, 0),
    (case("f32", 2, 64, 2, 2, 20, causal=False), None, 7), (case("bf16", 3, 64, 2, 2, 128, prefix=True, buckets=8, far=30), (64, 90), None),
    (case("f32", 1, 64, 4, 2, 64, prefix=True, cap=5.0), (64,), 2), (case("bf16", 2, 64, 2, 2, 32, prefix=True), (64, 63, 20), 1),
]


@pytest.mark.parametrize("what", ["k", "v", "q", "do", "all"])
@pytest.mark.parametrize("c,prefix,segments", WHOLE, ids=lambda p: name_of(p) if isinstance(p, dict) else str(p))
def test_non_finite_values_in_a_history_of_one_whole_tile(c, prefix, segments, what):
    check_spoilt(c, 10, what, float("nan"), prefix=prefix, segments=segments)
    if what in ("do", "v"):
        check_spoilt(c, 10, what, float("inf"), prefix=prefix, segments=segments)


# ---- scores of minus infinity, biases far from zero -------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_whose_scores_are_all_minus_infinity_yields_zeros(dtype):
    """As in the forward pass.  Caches of one part and of several; histories that see other rows too are not touched by it."""
    import torch
    from paper_2204_04179_amd import gram
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    for rows, lens in ((7, [0, 3, -1, 6]), (1500, [0, 1499, 1500, 700])):
        lens = torch.tensor(lens, dtype=torch.int32)
        q, kn, vn = draw(torch, (4, 2, 16), 1, dt), draw(torch, (4, 1, 16), 2, dt), draw(torch, (4, 1, 16), 3, dt)
        kc, vc = draw(torch, (4, rows, 1, 16), 4, dt), draw(torch, (4, rows, 1, 16), 5, dt)
        for hidden in (1, 8):                              # the new item alone; everything
            table = draw(torch, (2, 8), 6, torch.float32)
            table[:, :hidden] = -float("inf")
            seen = table.clone()
            seen[:, :hidden] = -200.0                      # exp(-200) is nothing beside the others
            o, bound, _, _ = lo.step(q, kn, vn, kc, vc, lens, scale=0.25, table=seen, far=20)
            nothing = torch.tensor([n == 0 or hidden == 8 for n in lens.tolist()])
            o[nothing], bound[nothing] = 0.0, 0.0
            plan = gram.HistoryAttention(2, 1, 16, dtype=gram.F32 if dtype == "f32" else gram.BF16, buckets=8, max_distance=20)
            O = torch.full((4, 2, 16), float("nan"), dtype=dt, device="cuda")
            work = torch.empty(plan.step_bytes(4, rows), dtype=torch.uint8, device="cuda")
            plan.step(q.cuda(), kn.cuda(), vn.cuda(), kc.cuda(), vc.cuda(), lens.cuda(), O, work, table=table.cuda())
            lo.assert_within(O, (o, bound), f"o of {rows}, {hidden} hidden")


def gradients(torch, gram, c, q, k, v, do, seg, prefix, table, table_gradient):
    """As run_gpu, with or without the table's gradient."""
    plan = plan_of(gram, c)
    B, L, H = c["B"], c["L"], c["H"]
    Q, K, V, DO = (placed(torch, t, c["layout"]) for t in (q, k, v, do))
    O, DQ, DK, DV = (placed(torch, torch.full_like(t, float("nan")), c["layout"]) for t in (q, q, k, v))
    seg, prefix, table = (None if t is None else t.cuda() for t in (seg, prefix, table))
    lse = torch.full((B, H, L), float("nan"), device="cuda")
    plan.forward(Q, K, V, O, lse=lse, segments=seg, prefix=prefix, table=table)
    work = torch.full((plan.backward_bytes(B, L),), 255, dtype=torch.uint8, device="cuda")      # NaN wherever it is read as floats
    dtable = torch.full((H, c["buckets"]), float("nan"), device="cuda") if table_gradient else None
    plan.backward(Q, K, V, O, lse, DO, DQ, DK, DV, work, segments=seg, prefix=prefix, table=table, dtable=dtable)
    out = dict(o=O, lse=lse, dq=DQ, dk=DK, dv=DV)
    return {**out, "dtable": dtable} if table_gradient else out


FAR = [
    case("f32", 2, 70, 2, 1, 16, buckets=8, far=40), case("bf16", 1, 200, 2, 2, 64, pad="holes", buckets=16, far=64),
    case("bf16", 66, 70, 2, 2, 20, buckets=8, far=40), case("f32", 3, 40, 4, 2, 24, docs=True, buckets=8, far=40),
    case("bf16", 3, 50, 2, 2, 20, pad="tail", prefix=True, buckets=8, far=40, both=True), case("f32", 1, 150, 2, 2, 128, causal=False, buckets=8, far=40, both=True),
    case("bf16", 33, 260, 4, 2, 36, cap=5.0, buckets=8, far=40), case("bf16", 1, 300, 2, 1, 128, docs=True, prefix=True, buckets=32, far=128, both=True),
    case("bf16", 50, 200, 2, 2, 128, docs=True, buckets=8, far=40), case("f32", 1, 64, 2, 2, 64, cap=5.0, buckets=1, far=2),
    case("f32", 1, 129, 1, 1, 127, layout="odd", buckets=8, far=40),
]


@pytest.mark.parametrize("table_gradient", [True, False])
@pytest.mark.parametrize("bias", [300.0, -70000.0, -1e9])
@pytest.mark.parametrize("c", FAR, ids=name_of)
def test_a_bias_that_all_pairs_share_changes_no_weight(c, bias, table_gradient):
    """However far from zero it is, where the sum of a row's weights is lost beside it.  The products are too small to count
    (q is 2^-60 of what it would be), so all weights of a row are the same."""
    import torch
    from paper_2204_04179_amd import gram
    q, k, v, do, seg, prefix, table = inputs(torch, c, seed=41)
    q = q * 2.0 ** -60
    want = oracle_of(c, q, k, v, do, seg, prefix, torch.zeros_like(table) if table_gradient else None)
    got = gradients(torch, gram, c, q, k, v, do, seg, prefix, torch.full_like(table, bias), table_gradient)
    for n in got:
        if n == "lse":
            value, bound = want[n]
            lo.assert_within(got[n], (value + bias, bound + 8 * lo.U * abs(bias)), n)
        else:
            lo.assert_within(got[n], want[n], n)


@pytest.mark.parametrize("table_gradient", [True, False])
@pytest.mark.parametrize("bias", [-1e9, -1.23e7, -3.3e10])
@pytest.mark.parametrize("c", FAR, ids=name_of)
def test_a_bias_that_hides_each_position_from_itself(c, bias, table_gradient):
    """At distance 0, as programs mask: the first position of a session sees nothing else and has weight one."""
    import torch
    from paper_2204_04179_amd import gram
    *data, table = inputs(torch, c, seed=42)
    mild = table.clone()
    table[:, 0], mild[:, 0] = bias, -100.0             # exp(-90) is nothing beside the others
    if c["buckets"] == 1:
        mild[:] = 0.0
        data[0] = data[0] * 2.0 ** -60
    want = oracle_of(c, *data, mild)
    got = gradients(torch, gram, c, *data, table, table_gradient)
    for n in got:
        if n != "lse":
            lo.assert_within(got[n], want[n], n)


@pytest.mark.parametrize("table_gradient", [True, False])
@pytest.mark.parametrize("bias", ["lowest", "highest", -2.5e38])
@pytest.mark.parametrize("c", FAR, ids=name_of)
def test_a_bias_at_the_end_of_its_type(c, bias, table_gradient):
    """The lowest finite number is no minus infinity: where all that a row sees has it, the row is the mean of its values."""
    import torch
    from paper_2204_04179_amd import gram
    big = torch.finfo(torch.float32).max
    entry = {"lowest": -big, "highest": big}.get(bias, bias)
    q, k, v, do, seg, prefix, table = inputs(torch, c, seed=43)
    q = q * 2.0 ** -60
    want = oracle_of(c, q, k, v, do, seg, prefix, torch.zeros_like(table) if table_gradient else None)
    got = gradients(torch, gram, c, q, k, v, do, seg, prefix, torch.full_like(table, entry), table_gradient)
    for n in got:
        if n != "lse":
            lo.assert_within(got[n], want[n], n)
    lse = got["lse"].cpu()
    nothing = torch.isinf(want["lse"][0])
    assert bool((lse[~nothing] == (big if entry > 0 else -big)).all()) and bool((lse[nothing] == -float("inf")).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [40, 1500])
def test_a_step_with_a_bias_at_the_end_of_its_type(dtype, rows):
    import torch
    from paper_2204_04179_amd import gram
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    lens = torch.tensor([0, rows - 1, rows // 2], dtype=torch.int32)
    q, kn, vn = draw(torch, (3, 4, 16), 1, dt) * 2.0 ** -60, draw(torch, (3, 2, 16), 2, dt), draw(torch, (3, 2, 16), 3, dt)
    kc, vc = draw(torch, (3, rows, 2, 16), 4, dt), draw(torch, (3, rows, 2, 16), 5, dt)
    plan = gram.HistoryAttention(4, 2, 16, dtype=gram.F32 if dtype == "f32" else gram.BF16, buckets=8, max_distance=20)
    o, bound, _, _ = lo.step(q, kn, vn, kc, vc, lens, scale=0.25, table=torch.zeros(4, 8), far=20)
    for sign in (-1.0, 1.0):
        table = torch.full((4, 8), sign * torch.finfo(torch.float32).max)
        O = torch.full((3, 4, 16), float("nan"), dtype=dt, device="cuda")
        work = torch.empty(plan.step_bytes(3, rows), dtype=torch.uint8, device="cuda")
        plan.step(q.cuda(), kn.cuda(), vn.cuda(), kc.cuda(), vc.cuda(), lens.cuda(), O, work, table=table.cuda())
        lo.assert_within(O, (o, bound), "o")


# ---- many heads on one key head ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,rows,H,KV,D,cap,buckets,far,first,layout", [
    (3, 70, 17, 1, 64, 0.0, 8, 20, False, "rows"), (2, 1500, 40, 1, 36, 30.0, 32, 128, True, "odd"), (4, 600, 34, 2, 128, 0.0, 16, 64, False, "heads"),
    (2, 33, 32, 1, 20, 4.0, 0, 0, False, "rows"), (3, 1030, 50, 2, 128, 0.0, 64, 300, False, "rows")])
def test_a_step_of_more_heads_than_a_block_takes(dtype, B, rows, H, KV, D, cap, buckets, far, first, layout):
    """Sixteen query heads of a key head go to one block, the next sixteen to another."""
    base.test_cached_step(dtype, B, rows, H, KV, D, cap, buckets, far, False, first, layout)


# ---- more histories of one tile than there are CUs, heads of more than 64 -----------------------------------

ONE_TILE = [
    case("bf16", 70, 20, 4, 4, 100, pad="tail", buckets=8, far=12), case("bf16", 90, 32, 3, 3, 128, docs=True), case("bf16", 130, 50, 4, 2, 72, prefix=True, buckets=32, far=40, both=True),
    case("bf16", 130, 50, 4, 2, 128, pad="holes", cap=5.0), case("bf16", 66, 60, 4, 4, 128, buckets=8, far=12), case("bf16", 300, 1, 1, 1, 65, buckets=2, far=3),
]


@pytest.mark.parametrize("c", ONE_TILE, ids=name_of)
def test_many_histories_of_one_tile_and_wide_heads(c):
    base.test_attention_and_its_backward(c)


@pytest.mark.parametrize("c", [ONE_TILE[0], ONE_TILE[4]], ids=name_of)
def test_biases_far_from_zero_among_many_histories_of_one_tile(c):
    for table_gradient in (True, False):
        test_a_bias_that_all_pairs_share_changes_no_weight(c, -1e9, table_gradient)
        test_a_bias_at_the_end_of_its_type(c, "lowest", table_gradient)


# ---- finite values whose products overflow where they are masked ------------------------------------------

LOUD = [
    case("bf16", 1, 200, 2, 1, 64, docs=True, buckets=8, far=30), case("f32", 2, 70, 2, 2, 20, docs=True, cap=5.0), case("bf16", 1, 130, 2, 2, 128),
    case("bf16", 50, 200, 2, 2, 128, buckets=8, far=30), case("f32", 40, 130, 4, 2, 64, cap=5.0, buckets=8, far=30), case("bf16", 3, 50, 2, 2, 20, docs=True, cap=5.0, buckets=8, far=30),
    case("f32", 1, 300, 2, 2, 128, docs=True), case("bf16", 70, 150, 4, 2, 64, docs=True, cap=5.0),
]


@pytest.mark.parametrize("c", LOUD, ids=name_of)
def test_products_that_overflow_where_they_are_masked_reach_no_one(c):
    """The first 20 positions hold a very large dout and q, the others, which those do not see, very large values and keys that cancel
    in no order: the products of the two are infinite or no number, and have no part in the first positions' gradients."""
    import torch
    from paper_2204_04179_amd import gram
    q, k, v, do, _, _, table = inputs(torch, c, seed=51)
    B, L, n = c["B"], c["L"], 20
    seg = torch.where(torch.arange(L) < n, 3, 4).int().expand(B, L).contiguous() if c["docs"] else None
    do[:, :n] *= 2.0 ** 60
    v[:, n:] *= 2.0 ** 80
    q[:, :n] = q[:, :n].sign() * 2.0 ** 30
    k[:, :n] *= 2.0 ** -30
    k[:, n:] = k[:, n:].sign() * 2.0 ** 120
    part = [t[:, :n] for t in (q, k, v, do)]
    want = oracle_of({**c, "L": n}, *part, None, None, table)
    got = run_gpu(torch, gram, c, q, k, v, do, seg, None, table)
    for name in ("o", "dq"):
        lo.assert_within(got[name][:, :n], want[name], name)
    if c["docs"]:
        for name in ("dk", "dv"):
            lo.assert_within(got[name][:, :n], want[name], name)


@pytest.mark.parametrize("c", [LOUD[0], LOUD[3], LOUD[4], LOUD[5], case("bf16", 3, 64, 2, 2, 64, causal=False)], ids=name_of)
def test_a_query_without_a_gradient_that_sees_a_nan_has_one(c):
    """Its dout is zero, and zero times the NaN of its weights is NaN."""
    import torch
    from paper_2204_04179_amd import gram
    q, k, v, do, _, _, table = inputs(torch, c, seed=52)
    k[:, 5], do[:] = float("nan"), 0.0
    got = run_gpu(torch, gram, c, q, k, v, do, None, None, table)
    assert not bool(torch.isfinite(got["dq"][:, 5:].float()).any()) and not bool(torch.isfinite(got["dv"].float()).any())
    if c["causal"]:
        assert bool((got["dq"][:, :5] == 0).all())
