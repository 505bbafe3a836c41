"""64-bit definitions of the collaborative filter's layer (layer norm, attention over histories, one cached step) for the
tests, with a bound on the rounding of an implementation beside every value.

Rounding: an operation in float32 is off by at most U = 2**-24 of its result, a rounding to bf16 by at most HB = 2**-8.
A sum of n products in float32 is off by at most n U times the sum of their magnitudes, whatever the order."""
import torch

U, HB = 2.0 ** -24, 2.0 ** -8
F64 = torch.float64


def half_step(dtype):
    return HB if dtype == torch.bfloat16 else U


def bucket_list(top, buckets, far, both):
    """Buckets of the distances 0..top of one side, decided in whole numbers of any length."""
    h = buckets // 2 if both else buckets
    e, out, b = h // 2, [], 0
    for n in range(top + 1):
        if h == 1:
            b = 0
        elif n < e:
            b = n
        else:
            b = max(b, e)
            while b + 1 < h and n ** (h - e) * e ** (b + 1 - e) >= far ** (b + 1 - e) * e ** (h - e):
                b += 1
        out.append(b)
    return out


def buckets_of(distance, buckets, far, both):
    """Bucket of each entry of a whole-number tensor of distances (query minus key)."""
    side = torch.tensor(bucket_list(int(distance.abs().max()) if distance.numel() else 0, buckets, far, both))
    after = side[(-distance).clamp(min=0)] + buckets // 2 if both else torch.zeros_like(distance)
    return torch.where(distance >= 0, side[distance.clamp(min=0)], after)


def visible(L, segments, causal, prefix, B):
    i = torch.arange(L)
    see = torch.ones(B, L, L, dtype=torch.bool)
    if causal:
        see = see & (i[None, :] <= i[:, None])[None]
        if prefix is not None:
            see = see | (i[None, None, :] < prefix[:, None, None])
    if segments is not None:
        see = see & (segments[:, :, None] == segments[:, None, :]) & (segments >= 0)[:, :, None]
    return see[:, None]


def attention(q, k, v, *, scale, cap=0.0, causal=True, segments=None, prefix=None, table=None, far=0, both=False, do=None):
    """q [B,L,H,D], k, v [B,L,KV,D] on the CPU, any float type.  Returns {name: (value, bound)} in 64 bits for o, lse and,
    with do, dq, dk, dv and dtable; the bound is for operands of q's type."""
    low = q.dtype == torch.bfloat16
    B, L, H, D = q.shape
    KV = k.shape[2]
    g = H // KV
    Q, K, V = (t.to(F64).permute(0, 2, 1, 3) for t in (q, k, v))
    K, V = (t.repeat_interleave(g, 1) for t in (K, V))
    z = Q @ K.transpose(2, 3) * scale
    size = Q.abs() @ K.abs().transpose(2, 3) * abs(scale)
    slope = torch.ones_like(z)
    s = z
    if cap:
        th = torch.tanh(z / cap)
        slope, s = 1 - th * th, cap * th
    of = None
    if table is not None:
        i = torch.arange(L)
        of = buckets_of(i[:, None] - i[None, :], table.shape[1], far, both)
        bias = table.to(F64)[:, of]
        s, size = s + bias, size + bias.abs()
    see = visible(L, segments, causal, prefix, B)
    any_ = see.any(3, keepdim=True)
    top = torch.where(see, s, torch.full_like(s, -torch.inf)).amax(3, keepdim=True)
    top = torch.where(any_, top, torch.zeros_like(top))
    e = torch.where(see, torch.exp(s - top), torch.zeros_like(s))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(any_, total, torch.ones_like(total))
    o = p @ V
    # a score is off by (D + 8) U of its terms (cap: a tanh off by 4 U of itself, so of |s| too), which moves a weight by
    # that times itself, and its row's sum by at most as much again; sums over L keys and D columns follow
    rel = (2 * (D + 8) * float((size * see).detach().max() if see.any() else 0.0) + L + D + 64) * U
    wround = HB if low else U                       # a weight as it enters the second product
    out = dict(o=(o, (wround + rel) * (p @ V.abs()) + half_step(q.dtype) * o.abs()))
    lse = torch.where(any_, top + torch.log(torch.where(any_, total, torch.ones_like(total))), torch.full_like(top, -torch.inf))[..., 0]
    out["lse"] = (lse, rel + 4 * U * torch.where(torch.isinf(lse), torch.zeros_like(lse), lse).abs())
    if do is not None:
        G = do.to(F64).permute(0, 2, 1, 3)
        dp = G @ V.transpose(2, 3)
        dp_size = G.abs() @ V.abs().transpose(2, 3)
        delta = (p * dp).sum(3, keepdim=True)
        delta_size = (p * dp_size).sum(3, keepdim=True)
        ds = p * (dp - delta)
        ds_size = p * (dp_size + delta_size)
        # delta from the stored o: off by the rounding of o and of the weights in it.  With a table it is summed in float32
        delta_err = (2 * HB * delta_size) if low and table is None else 0.0 * delta_size
        ds_err = 3 * rel * ds_size + p * delta_err
        dz, dz_err = ds * slope, ds_err * slope + 16 * U * ds.abs()
        grow = wround * dz.abs() + dz_err
        fold = lambda t: t.view(B, KV, g, L, D).sum(2)
        last = (L + 64) * U
        sc = abs(scale)
        out["dq"] = (dz @ K * scale, sc * (grow @ K.abs() + last * (dz.abs() @ K.abs())))
        out["dk"] = (fold(dz.transpose(2, 3) @ Q) * scale,
                     sc * fold(grow.transpose(2, 3) @ Q.abs() + g * last * (dz.abs().transpose(2, 3) @ Q.abs())))
        pT = p.transpose(2, 3)
        out["dv"] = (fold(pT @ G), fold((wround + rel + g * last) * (pT @ G.abs())))
        for n in ("dq", "dk", "dv"):
            out[n] = (out[n][0], out[n][1] + half_step(q.dtype) * out[n][0].abs())
        if table is not None:
            one = torch.nn.functional.one_hot(of.reshape(-1), table.shape[1]).to(F64)
            add = lambda t: t.sum(0).reshape(H, -1) @ one
            # partial sums of a block run over at most 64 L terms
            out["dtable"] = (add(ds), add(ds_err) + 64 * L * U * add(ds.abs()))
    rows = lambda t: t.permute(0, 2, 1, 3)
    return {n: (t, b) if n in ("lse", "dtable") else (rows(t), rows(b)) for n, (t, b) in out.items()}


def layer_norm(x, w, b, y_dtype, segments=None, eps=1e-5, dy=None, add=None):
    """{name: (value, bound)} for y and, with dy, dx, dw, db."""
    M, d = x.shape
    X, w, b = x.to(F64), w.to(F64), b.to(F64)
    keep = torch.ones(M, 1, dtype=F64) if segments is None else (segments >= 0).to(F64)[:, None]
    X = torch.where(keep > 0, X, torch.zeros_like(X))
    mean = X.mean(1, keepdim=True)
    c = X - mean
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    xh = c * r
    # mean: d + 2 roundings of mean |x|; a centred value carries that and its own; var, root and product a few each
    c_err = (d + 4) * U * X.abs().mean(1, keepdim=True) + U * X.abs()
    xh_err = r * c_err + xh.abs() * ((d + 8) * U + r * r * (c.abs() * c_err).mean(1, keepdim=True) * 2)
    y = xh * w + b
    out = dict(y=(y * keep, keep * (xh_err * w.abs() + 4 * U * ((xh * w).abs() + b.abs())) + half_step(y_dtype) * (y * keep).abs()))
    if dy is not None:
        G = torch.where(keep > 0, dy.to(F64), torch.zeros(M, d, dtype=F64))
        g = G * w
        m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        dx = r * (g - m1 - xh * m2)
        a1, a2 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
        r_rel = (d + 8) * U + r * r * (c.abs() * c_err).mean(1, keepdim=True) * 2
        err = r * ((d + 16) * U * (g.abs() + a1 + xh.abs() * a2) + xh_err * m2.abs() +
                   xh.abs() * (g.abs() * xh_err).mean(1, keepdim=True)) + dx.abs() * r_rel
        A = torch.zeros(M, d, dtype=F64) if add is None else torch.where(keep > 0, add.to(F64), torch.zeros(M, d, dtype=F64))
        out["dx"] = (keep * dx + A, keep * (err + 2 * U * (A.abs() + dx.abs())))
        out["dw"] = ((G * xh).sum(0), (G.abs() * xh_err).sum(0) + (M + 4) * U * (G * xh).abs().sum(0))
        out["db"] = (G.sum(0), (M + 4) * U * G.abs().sum(0))
    return out


def step(q, k_new, v_new, k_cache, v_cache, lengths, *, scale, cap=0.0, first=None, table=None, far=0, both=False):
    """(o, bound, k_cache, v_cache) of one cached step, o in 64 bits."""
    B, H, D = q.shape
    capacity, KV = k_cache.shape[1], k_cache.shape[2]
    kc, vc = k_cache.clone(), v_cache.clone()
    o, bound = torch.zeros(B, H, D, dtype=F64), torch.zeros(B, H, D, dtype=F64)
    for b, n in enumerate(lengths.tolist()):
        if not 0 <= n < capacity:
            continue
        kc[b, n], vc[b, n] = k_new[b], v_new[b]
        lo = 0 if first is None else min(max(int(first[b]), 0), n)
        K, V = (t[b, lo:n + 1].to(F64).repeat_interleave(H // KV, 1).transpose(0, 1) for t in (kc, vc))
        Q = q[b].to(F64)[:, :, None]
        s, size = (K @ Q)[..., 0] * scale, (K.abs() @ Q.abs())[..., 0] * abs(scale)
        if cap:
            s = cap * torch.tanh(s / cap)
        if table is not None:
            bias = table.to(F64)[:, buckets_of(n - torch.arange(lo, n + 1), table.shape[1], far, both)]
            s, size = s + bias, size + bias.abs()
        p = torch.softmax(s, 1)[:, None]
        rel = (2 * (D + 8) * float(size.max()) + (n + 1 - lo) + D + 64) * U
        o[b] = (p @ V)[:, 0]
        bound[b] = rel * (p @ V.abs())[:, 0] + half_step(q.dtype) * o[b].abs()
    return o, bound, kc, vc


def assert_within(got, want, what):
    """Every entry within its bound; infinities and NaN where the definition has them."""
    value, bound = want
    got = got.detach().cpu().to(F64)
    assert got.shape == value.shape, f"{what}: shape {tuple(got.shape)} against {tuple(value.shape)}"
    if not value.numel():
        return
    odd = ~torch.isfinite(value)
    assert bool((torch.isfinite(got) == ~odd).all()), f"{what}: {int((torch.isfinite(got) == odd).sum())} entries (not) finite"
    off = torch.where(odd, torch.zeros_like(value), (got - value).abs())
    # the smallest numbers of a type are rounded to a multiple of its smallest
    room = bound + 2.0 ** -125
    worst = int((off / room).argmax())
    assert bool((off <= room).all()), (f"{what}: entry {worst} is {float(got.reshape(-1)[worst]):.9g}, "
                                       f"{float(value.reshape(-1)[worst]):.9g} expected within {float(room.reshape(-1)[worst]):.3g}")
