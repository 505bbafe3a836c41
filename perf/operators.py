"""Performance cases of the collaborative filter's layer: layer norm of the positions' representations and attention
over item histories, from the smallest batch a test would use to long histories and large caches.

The kinds:

  norm        layer norm of [M, d] rows (an inference pass)
  norm_train  the same with its backward pass: input gradient, on top of the gradient that comes past the layer, and
              the gradients of weight and bias
  attend      attention over [B, L] histories (an inference pass): capped scores, a learned bias by distance, padding,
              documents, causal and prefix masks
  train       the same with its backward pass, down to the gradient of the learned bias
  step        one new item per history, appended to a cache of keys and values and attended from

With `own` false an operator is computed in its plain form, elementary tensor operations in 32 bits; with `own` true by
the calls of `paper_2204_04179_amd.gram`.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"
_DTYPE = {BF16: torch.bfloat16, F32: torch.float32}
_DEVICE = "cuda"


def _norm(name, M, d, x, y, train, pad="none"):
    case = dict(kind="norm_train" if train else "norm", M=M, d=d, x=x, y=y, pad=pad)
    if name:
        case["name"] = name
    return case


def _attend(name, kind, dtype, B, L, heads, kv, D, causal=True, prefix=0, docs=1, pad="none", cap=0.0, buckets=0, far=0,
            both=False):
    case = dict(kind=kind, dtype=dtype, B=B, L=L, heads=heads, kv=kv, D=D, causal=causal, prefix=prefix, docs=docs, pad=pad,
                cap=cap, buckets=buckets, far=far, both=both)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the smallest layer norm: a handful of short histories in float32 (a unit test, a tutorial)
        _norm("norm_tiny_f32", 64, 32, F32, F32, False),
        # the positions of the large batch on their way into bf16 projections
        _norm("norm_large", 204_800, 1024, F32, BF16, False),
        # one training step of a news recommender, width no power of two, padded positions
        _norm("norm_train_news", 7_040, 400, F32, BF16, True, "last3"),
        # one training step on the large batch, positions kept in bf16
        _norm("norm_train_large", 204_800, 1024, BF16, BF16, True),
        # the smallest attention: four histories of 16 in float32, the last three positions padding
        _attend("attend_tiny_f32", "attend", F32, 4, 16, 2, 2, 16, pad="last3"),
        # a long prompt of packed sessions: shared key heads, capped scores, bias by distance
        _attend("attend_long_sessions", "attend", BF16, 1, 8192, 8, 2, 128, docs=8, cap=30.0, buckets=32, far=128),
        # training on the knowledge-tracing shape: causal, padded histories, bias by distance
        _attend("train_kt", "train", BF16, 64, 100, 4, 4, 64, pad="uniform20", buckets=32, far=128),
        # training on the news shape: 20 heads of width 20, clicked items visible to all, bias on both sides
        _attend("train_news", "train", BF16, 128, 55, 20, 20, 20, prefix=50, buckets=32, far=64, both=True),
        # training on the large batch
        _attend("train_large", "train", BF16, 1024, 200, 8, 8, 128, buckets=32, far=128),
        # float32 training on long ragged histories, every position visible within its session
        _attend("train_long_f32", "train", F32, 2, 1003, 4, 2, 64, causal=False, docs=2, pad="uniform20", cap=20.0, buckets=32,
                far=256, both=True),
        # serving: the next item of 64 short histories
        _attend("step_kt", "step", BF16, 64, 200, 4, 4, 64, pad="uniform20", buckets=32, far=128),
        # serving: the next item of 64 long histories, shared key heads
        _attend("step_long", "step", BF16, 64, 8192, 8, 2, 128, pad="uniform20", cap=30.0, buckets=32, far=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["norm", "norm_train", "attend", "attend", "train", "train", "train", "step", "step"])
    if kind in ("norm", "norm_train"):
        d = rng.choice([8 * _log(rng, 4, 512), 4 * _log(rng, 2, 256), _log(rng, 1, 1500)])
        M = min(_log(rng, 1, 204_800), 200_000_000 // d)
        return _norm(None, M, d, rng.choice([F32, BF16]), rng.choice([F32, BF16]), kind == "norm_train",
                     rng.choice(["none", "last3"]))
    dtype = rng.choice([BF16, BF16, F32])
    D = rng.choice([8 * rng.randint(2, 16), 64, 128, rng.choice([20, 36, 100]), rng.randint(1, 128)])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4, 5])
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    buckets, far = rng.choice([(0, 0), (32, 128), (16, 64), (64, 512), (12, 40)])
    pad = rng.choice(["none", "last3", "uniform20"])
    if kind == "step":
        cap_rows = _log(rng, 1, 8192)
        B = max(1, min(_log(rng, 1, 512), 250_000_000 // (cap_rows * kv * D), 60_000_000 // (cap_rows * heads)))
        return _attend(None, kind, dtype, B, cap_rows, heads, kv, D, pad=pad, cap=cap, buckets=buckets, far=far)
    L = min(_log(rng, 1, 3000), int(math.sqrt(200_000_000 / heads)))
    B = max(1, min(_log(rng, 1, 1024), 200_000_000 // (heads * L * L), 100_000_000 // (L * heads * D)))
    causal = rng.random() < 0.7
    prefix = rng.randint(0, L) if causal and rng.random() < 0.3 else 0
    both = buckets > 0 and (not causal or prefix > 0)
    return _attend(None, kind, dtype, B, L, heads, kv, D, causal, prefix, rng.choice([1, 1, 3]), pad, cap, buckets, far, both)


# ---- inputs -----------------------------------------------------------------------------------------------


def _segments(B, L, pad, docs, rng):
    """int32 [B, L]: the session each position belongs to, -1 at padding."""
    seg = np.zeros((B, L), dtype=np.int32)
    if docs > 1:
        seg = np.cumsum(rng.random((B, L)) < docs / L, axis=1).astype(np.int32)
    if pad == "last3":
        seg[:, max(0, L - 3):] = -1
    elif pad == "uniform20":
        lens = rng.integers(min(20, L), L + 1, size=B)
        seg[np.arange(L)[None, :] >= lens[:, None]] = -1
    return seg


def prepare(case, seed):
    dev = _DEVICE
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = np.random.default_rng(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device=dev).mul_(scale).add_(mean).to(dtype)

    st = dict(case)
    if case["kind"] in ("norm", "norm_train"):
        M, d = case["M"], case["d"]
        xt, yt = _DTYPE[case["x"]], _DTYPE[case["y"]]
        st.update(x=normal(M, d, dtype=xt, scale=1.5, mean=0.3), w=normal(d, scale=0.2, mean=1.0), b=normal(d, scale=0.2),
                  y=torch.empty(M, d, dtype=yt, device=dev), segments=None)
        if case["pad"] == "last3":
            st["segments"] = torch.from_numpy(np.where(np.arange(M) % 55 >= 52, -1, 0).astype(np.int32)).to(dev)
        if case["kind"] == "norm_train":
            st.update(dy=normal(M, d, dtype=yt), past=normal(M, d), dx=torch.empty(M, d, device=dev),
                      dw=torch.empty(d, device=dev), db=torch.empty(d, device=dev), stats=torch.empty(M, 2, device=dev))
        return st
    B, L, H, KV, D, dt = case["B"], case["L"], case["heads"], case["kv"], case["D"], _DTYPE[case["dtype"]]
    st["table"] = normal(H, case["buckets"], scale=0.5) if case["buckets"] else None
    if case["kind"] == "step":
        lens = np.full(B, L - 1, dtype=np.int32)
        if case["pad"] == "uniform20":
            lens = rng.integers(0, L, size=B).astype(np.int32)
        elif case["pad"] == "last3":
            lens[: B // 3] = -1                                     # histories that ask for nothing this time
        st.update(q=normal(B, H, D, dtype=dt), k_new=normal(B, KV, D, dtype=dt), v_new=normal(B, KV, D, dtype=dt),
                  k_cache=normal(B, L, KV, D, dtype=dt), v_cache=normal(B, L, KV, D, dtype=dt),
                  lengths=torch.from_numpy(lens).to(dev), o=torch.empty(B, H, D, dtype=dt, device=dev))
        return st
    qkv = normal(B, L, H + 2 * KV, D, dtype=dt)                     # as one projection leaves it
    st.update(q=qkv[:, :, :H], k=qkv[:, :, H:H + KV], v=qkv[:, :, H + KV:], o=torch.empty(B, L, H, D, dtype=dt, device=dev),
              segments=None, prefix=None)
    if case["docs"] > 1 or case["pad"] != "none":
        st["segments"] = torch.from_numpy(_segments(B, L, case["pad"], case["docs"], rng)).to(dev)
    if case["prefix"]:
        st["prefix"] = torch.from_numpy(rng.integers(0, case["prefix"] + 1, size=B).astype(np.int32)).to(dev)
    if case["kind"] == "train":
        dqkv = torch.empty_like(qkv)
        st.update(do=normal(B, L, H, D, dtype=dt), lse=torch.empty(B, H, L, device=dev), dq=dqkv[:, :, :H],
                  dk=dqkv[:, :, H:H + KV], dv=dqkv[:, :, H + KV:],
                  dtable=torch.empty(H, case["buckets"], device=dev) if case["buckets"] else None)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------


def run(st):
    if st["kind"] in ("norm", "norm_train"):
        return _own_norm(st) if own else _plain_norm(st)
    if st["kind"] == "step":
        return _own_step(st) if own else _plain_step(st)
    return _own_attend(st) if own else _plain_attend(st)


def _own_norm(st):
    from paper_2204_04179_amd import gram

    if st["kind"] == "norm":
        gram.layer_norm(st["x"], st["w"], st["b"], st["y"], segments=st["segments"])
        return st["y"]
    if "work" not in st:
        st["work"] = torch.empty(gram.layer_norm_work_bytes(st["M"], st["d"]), dtype=torch.uint8, device=_DEVICE)
    gram.layer_norm(st["x"], st["w"], st["b"], st["y"], stats=st["stats"], segments=st["segments"])
    gram.layer_norm_backward(st["x"], st["w"], st["stats"], st["dy"], st["dx"], st["dw"], st["db"], st["work"],
                             segments=st["segments"], add=st["past"])
    return st["y"], st["dx"], st["dw"], st["db"]


def _plan(st):
    """The layer's plan and workspace, which a program keeps with the layer."""
    from paper_2204_04179_amd import gram

    if "plan" not in st:
        st["plan"] = plan = gram.HistoryAttention(st["heads"], st["kv"], st["D"],
                                                  dtype=gram.BF16 if st["dtype"] == BF16 else gram.F32, cap=st["cap"],
                                                  causal=st["causal"], buckets=st["buckets"], max_distance=st["far"],
                                                  two_sided=st["both"])
        size = plan.step_bytes(st["B"], st["L"]) if st["kind"] == "step" else plan.backward_bytes(st["B"], st["L"])
        st["work"] = torch.empty(size, dtype=torch.uint8, device=_DEVICE)
    return st["plan"]


def _own_attend(st):
    plan = _plan(st)
    if st["kind"] == "attend":
        plan.forward(st["q"], st["k"], st["v"], st["o"], segments=st["segments"], prefix=st["prefix"], table=st["table"])
        return st["o"]
    plan.forward(st["q"], st["k"], st["v"], st["o"], lse=st["lse"], segments=st["segments"], prefix=st["prefix"],
                 table=st["table"])
    plan.backward(st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"], st["dq"], st["dk"], st["dv"], st["work"],
                  segments=st["segments"], prefix=st["prefix"], table=st["table"], dtable=st["dtable"])
    out = (st["o"], st["dq"], st["dk"], st["dv"])
    return out + (st["dtable"],) if st["dtable"] is not None else out


def _own_step(st):
    _plan(st).step(st["q"], st["k_new"], st["v_new"], st["k_cache"], st["v_cache"], st["lengths"], st["o"], st["work"],
                   table=st["table"])
    return st["o"], st["k_cache"], st["v_cache"]


# ---- plain forms ------------------------------------------------------------------------------------------


def _plain_norm(st):
    x, w = st["x"].float(), st["w"]
    keep = None if st["segments"] is None else (st["segments"] >= 0)[:, None]
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = ((xc * xc).mean(1, keepdim=True) + 1e-5).rsqrt()
    xh = xc * rstd
    y = xh * w + st["b"]
    if keep is not None:
        y = torch.where(keep, y, torch.zeros_like(y))
    y = y.to(st["y"].dtype)
    if st["kind"] == "norm":
        return y
    dy = st["dy"].float()
    if keep is not None:
        dy = torch.where(keep, dy, torch.zeros_like(dy))
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) + st["past"]
    if keep is not None:
        dx = torch.where(keep, dx, torch.zeros_like(dx))
    return y, dx, (dy * xh).sum(0), dy.sum(0)


def _bucket(n, top, buckets, far, both):
    """Bucket of the distances n (query minus key, whole numbers of at most `top`): one each for near ones, then ever
    wider."""
    h = buckets // 2 if both else buckets
    e = h // 2
    size = torch.arange(top + 1, dtype=torch.float64, device=n.device)
    near = torch.arange(top + 1, device=n.device)
    if h > 1:
        # the bucket of a distance m >= e is e + floor((h - e) ln(m / e) / ln(far / e)); a value within 1e-11 of a whole
        # number is that number
        steps = (h - e) * torch.log(size.clamp(min=e) / e) / math.log(far / e)
        wide = (e + torch.floor(steps + 1e-11)).clamp(max=h - 1).long()
        of = torch.where(near < e, near, wide)
    else:
        of = torch.zeros_like(near)
    after = of[(-n).clamp(min=0)] + h if both else torch.zeros_like(n)
    return torch.where(n >= 0, of[n.clamp(min=0)], after)


def _visible(st):
    B, L, dev = st["B"], st["L"], st["q"].device
    i = torch.arange(L, device=dev)
    vis = torch.ones(1, L, L, dtype=torch.bool, device=dev)
    if st["causal"]:
        vis = (i[None, :] <= i[:, None])[None]
        if st["prefix"] is not None:
            vis = vis | (i[None, None, :] < st["prefix"][:, None, None])
    if st["segments"] is not None:
        seg = st["segments"]
        vis = vis & (seg[:, :, None] == seg[:, None, :]) & (seg >= 0)[:, :, None]
    return vis[:, None]


def _plain_attend(st):
    H, KV, D, cap = st["heads"], st["kv"], st["D"], st["cap"]
    B, L, dt = st["B"], st["L"], st["o"].dtype
    scale = D ** -0.5
    q = st["q"].float().permute(0, 2, 1, 3).contiguous()
    k = st["k"].float().permute(0, 2, 1, 3).repeat_interleave(H // KV, 1).contiguous()
    v = st["v"].float().permute(0, 2, 1, 3).repeat_interleave(H // KV, 1).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    slope = None
    if cap:
        th = torch.tanh(s / cap)
        s = cap * th
        slope = 1 - th * th if st["kind"] == "train" else None
        del th
    if st["table"] is not None:
        i = torch.arange(L, device=q.device)
        of = _bucket(i[:, None] - i[None, :], L, st["buckets"], st["far"], st["both"])
        s += st["table"][:, of]
    vis = _visible(st)
    s = s.masked_fill(~vis, -math.inf)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    del s
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, v)

    def rows(t, like):
        return t.permute(0, 2, 1, 3).to(like.dtype)

    if st["kind"] == "attend":
        return rows(o, st["o"])
    do = st["do"].float().permute(0, 2, 1, 3).contiguous()
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(3, keepdim=True))
    del dp
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    del p
    dz = ds * slope * scale if slope is not None else ds * scale
    dq = torch.matmul(dz, k)
    dk = torch.matmul(dz.transpose(2, 3).contiguous(), q)
    del dz
    dk, dv = (t.view(B, KV, H // KV, L, D).sum(2) for t in (dk, dv))
    out = (rows(o, st["o"]), rows(dq, st["o"]), rows(dk, st["o"]), rows(dv, st["o"]))
    if st["table"] is None:
        return out
    # sums over all pairs of a bucket, in 64 bits: first over those of one distance, which a row length of 2 L - 1 brings
    # into one column each, then over the distances of a bucket
    skewed = torch.zeros(H, L, 2 * L, dtype=torch.float64, device=q.device)
    skewed[:, :, :L] = ds.sum(0, dtype=torch.float64).flip(2)
    by_distance = skewed.view(H, -1)[:, : L * (2 * L - 1)].view(H, L, 2 * L - 1).sum(1)
    far = _bucket(torch.arange(2 * L - 1, device=q.device) - (L - 1), L, st["buckets"], st["far"], st["both"])
    one_hot = (far[:, None] == torch.arange(st["buckets"], device=q.device)).double()
    dtable = torch.matmul(by_distance, one_hot).float()
    return out + (dtable,)


def _plain_step(st):
    H, KV, D, cap = st["heads"], st["kv"], st["D"], st["cap"]
    B, L, lens = st["B"], st["L"], st["lengths"].long()
    live = (lens >= 0) & (lens < L)
    b = torch.arange(B, device=lens.device)
    at = lens.clamp(0, L - 1)
    st["k_cache"][b, at] = torch.where(live[:, None, None], st["k_new"], st["k_cache"][b, at])
    st["v_cache"][b, at] = torch.where(live[:, None, None], st["v_new"], st["v_cache"][b, at])
    q = st["q"].float().view(B, KV, H // KV, D)
    k = st["k_cache"].float().permute(0, 2, 3, 1).contiguous()
    s = torch.matmul(q, k) * D ** -0.5
    del k
    if cap:
        s = cap * torch.tanh(s / cap)
    j = torch.arange(L, device=lens.device)
    if st["table"] is not None:
        of = _bucket((lens[:, None] - j[None, :]).clamp(min=0), L, st["buckets"], st["far"], st["both"])
        s = s + st["table"][:, of].permute(1, 0, 2).reshape(B, KV, H // KV, L)
    s = s.masked_fill((j[None, :] > lens[:, None])[:, None, None], -math.inf)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    p = torch.where(live[:, None, None, None], p, torch.zeros_like(p))
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, st["v_cache"].float().permute(0, 2, 1, 3).contiguous())
    return o.reshape(B, H, D).to(st["o"].dtype), st["k_cache"], st["v_cache"]


# ---- what a pass cannot do without ------------------------------------------------------------------------


def _pairs(case):
    """Visible pairs of a batch, for the lengths that the masks have on average."""
    L, B = case["L"], case["B"]
    n = {"none": L, "last3": max(0, L - 3), "uniform20": (min(20, L) + L) / 2}[case["pad"]]
    run_, docs = n / case["docs"], case["docs"]
    pairs = docs * (run_ * (run_ + 1) / 2 if case["causal"] else run_ * run_)
    if case["prefix"]:
        pairs += (min(case["prefix"], n) / 2) ** 2 / 2
    return B * pairs


def work(case):
    size = {BF16: 2, F32: 4}
    if case["kind"] in ("norm", "norm_train"):
        M, d, x, y = case["M"], case["d"], size[case["x"]], size[case["y"]]
        if case["kind"] == "norm":
            return {"bytes": M * d * (x + y) + 8 * d, "flops": 8 * M * d}
        return {"bytes": M * d * (x + y + y + 4 + 4) + 16 * d, "flops": 22 * M * d}
    B, L, H, KV, D, e = case["B"], case["L"], case["heads"], case["kv"], case["D"], size[case["dtype"]]
    if case["kind"] == "step":
        rows = {"none": L, "last3": L * (B - B // 3) / B, "uniform20": (L + 1) / 2}[case["pad"]] * B
        return {"bytes": e * D * (2 * KV * rows + B * (2 * H + 2 * KV)), "flops": 4 * D * H * rows}
    pairs = _pairs(case) * H
    if case["kind"] == "attend":
        return {"bytes": e * D * B * L * 2 * (H + KV), "flops": 4 * D * pairs}
    return {"bytes": e * D * B * L * (4 * H + 4 * KV), "flops": 14 * D * pairs}


# ---- the definition in 64 bits ----------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("norm", "norm_train"):
        return _exact_norm(st)
    if case["kind"] == "step":
        return _exact_step(st)
    parts = [_exact_histories(st, a, c) for a, c in _chunks(st)]
    out = [torch.cat([p[t] for p in parts]) for t in range(len(parts[0]) - 1)]
    if case["kind"] == "attend":
        return out[0]
    return tuple(out) if st["table"] is None else tuple(out) + (sum(p[-1] for p in parts),)


def _exact_norm(st):
    x, w, b = (st[t].double().requires_grad_() for t in ("x", "w", "b"))
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    y = (x - mean) / torch.sqrt(var + 1e-5) * w + b
    keep = torch.ones(len(x), 1, dtype=torch.float64, device=x.device)
    if st["segments"] is not None:
        keep = (st["segments"] >= 0).double()[:, None]
    y = y * keep
    if st["kind"] == "norm":
        return y.detach()
    dx, dw, db = torch.autograd.grad(y, (x, w, b), st["dy"].double())
    return y.detach(), dx + st["past"].double() * keep, dw, db


def _bucket_list(top, buckets, far, both):
    """Buckets of the distances 0..top on one side, each decided in whole numbers of any length."""
    h = buckets // 2 if both else buckets
    e, of, b = h // 2, [], 0
    for n in range(top + 1):
        if n < e or h == 1:
            b = min(n, h - 1) if h > 1 else 0
        else:
            b = max(b, e)
            while b + 1 < h and n ** (h - e) * e ** (b + 1 - e) >= far ** (b + 1 - e) * e ** (h - e):
                b += 1
        of.append(b)
    return of


def _distance_table(st, device):
    """[heads, 2 L + 1] in 64 bits: the bias at distance -L..L."""
    L, h = st["L"], st["buckets"] // 2 if st["both"] else st["buckets"]
    of = _bucket_list(L, st["buckets"], st["far"], st["both"])
    row = [(of[-n] + h if st["both"] else 0) if n < 0 else of[n] for n in range(-L, L + 1)]
    return torch.tensor(row, device=device)


def _chunks(st):
    each = max(1, int(2.0e8 // (st["heads"] * st["L"] ** 2)))
    return [(a, min(a + each, st["B"])) for a in range(0, st["B"], each)]


def _exact_histories(st, a, c):
    train, H, KV, L = st["kind"] == "train", st["heads"], st["kv"], st["L"]
    dev = st["q"].device
    leaves = [st[t][a:c].double().requires_grad_(train) for t in ("q", "k", "v")]
    table = None if st["table"] is None else st["table"].double().requires_grad_(train)
    q, k, v = (t.transpose(1, 2).contiguous() for t in leaves)
    k, v = ((t[:, :, None] * torch.ones(1, 1, H // KV, 1, 1, dtype=t.dtype, device=dev)).reshape(c - a, H, L, -1) for t in (k, v))
    s = q @ k.transpose(2, 3).contiguous() / math.sqrt(st["D"])
    if st["cap"]:
        s = st["cap"] * torch.tanh(s / st["cap"])
    i = torch.arange(L, device=dev)
    if table is not None:
        by_distance = table[:, _distance_table(st, dev)]
        s = s + by_distance[:, i[:, None] - i[None, :] + L]
    see = torch.ones(c - a, L, L, dtype=torch.bool, device=dev)
    if st["causal"]:
        see &= i[:, None] >= i
        if st["prefix"] is not None:
            see |= (i < st["prefix"][a:c, None])[:, None, :]
    if st["segments"] is not None:
        seg = st["segments"][a:c]
        see &= (seg[:, :, None] == seg[:, None, :]) & (seg[:, None, :] != -1)
    p = torch.softmax(s.masked_fill(~see[:, None], -1e300), 3) * see[:, None]
    o = (p @ v).transpose(1, 2)
    if not train:
        return [o.detach(), None]
    grads = torch.autograd.grad(o, leaves + ([table] if table is not None else []), st["do"][a:c].double())
    return [o.detach(), *grads[:3], grads[3] if table is not None else None]


def _exact_step(st):
    B, L, H, KV = st["B"], st["L"], st["heads"], st["kv"]
    lens, dev = st["lengths"].tolist(), st["q"].device
    of = _bucket_list(L, st["buckets"], st["far"], st["both"]) if st["table"] is not None else None
    of = None if of is None else torch.tensor(of, device=dev)
    o = torch.zeros(st["o"].shape, dtype=torch.float64, device=dev)
    kc, vc = st["k_cache"].clone(), st["v_cache"].clone()
    for b, n in enumerate(lens):
        if n < 0:
            continue
        kc[b, n], vc[b, n] = st["k_new"][b], st["v_new"][b]
        q = st["q"][b].double().view(KV, H // KV, -1)
        s = torch.einsum("hgd,nhd->hgn", q, kc[b, : n + 1].double()) / math.sqrt(st["D"])
        if st["cap"]:
            s = st["cap"] * torch.tanh(s / st["cap"])
        if of is not None:
            s = s + st["table"].double()[:, of[n - torch.arange(n + 1, device=dev)]].view(KV, H // KV, n + 1)
        o[b] = torch.einsum("hgn,nhd->hgd", torch.softmax(s, 2), vc[b, : n + 1].double()).reshape(H, -1)
    return o, kc.double(), vc.double()
