"""Attention with modified scores in float64 on the CPU, written out as matrices, with
bounds of the rounding errors that kernels of a given input type may make.

The bounds count, per element, with u the half step of the type (finfo.eps / 2) and e = 2^-24:
  scores    a float32 dot product of d terms (d + 8 roundings of the sum of magnitudes),
            the cap, bias and exponent arithmetic on values as large as the score, the cap, the
            bias and the log-sum-exp (8 roundings each)
  weights   relative error of a weight: the score's error; rounded to the type for the products
  D_i       from o and its residual, which carry twice the type's bits
  sums      one rounding per term, and the output's own rounding.
Nothing is fitted: a wrong index, mask or factor is far outside them.
"""
import math

import torch

E32 = 2.0 ** -24


def bucket_of(distance, buckets, max_distance, two_sided):
    """By the definition, with exact powers: the largest b whose lower end is at most the distance."""
    n = buckets // 2 if two_sided else buckets
    h = n // 2

    def side(x):
        if x < h:
            return x
        b = h
        while b + 1 < n and x ** (n - h) >= max_distance ** (b + 1 - h) * h ** (n - b - 1):
            b += 1
        return b

    if two_sided:
        return side(abs(distance)) + (n if distance > 0 else 0)
    return side(max(-distance, 0))


def bucket_index(pos, n_k, buckets, max_distance, two_sided):
    """[n_q, n_k] bucket of every pair for the positions ``pos`` of the queries."""
    lo, hi = -max(pos), n_k - 1 - min(pos)
    table = torch.tensor([bucket_of(x, buckets, max_distance, two_sided) for x in range(lo, hi + 1)])
    return table[torch.arange(n_k)[None, :] - torch.tensor(pos)[:, None] - lo]


def visible(B, n_q, n_k, causal, kv_len, docs, prefix_len, q_pos):
    j = torch.arange(n_k)
    seen = torch.ones(B, n_q, n_k, dtype=torch.bool)
    for b in range(B):
        pos = torch.arange(n_q) + (max(0, q_pos[b]) if q_pos is not None else 0)
        if causal:
            seen[b] = j[None, :] <= pos[:, None]
            if prefix_len is not None:
                seen[b] |= (j < prefix_len[b])[None, :]
        if kv_len is not None:
            seen[b] &= (j < kv_len[b])[None, :]
        if docs is not None:
            a, c = docs[0][b], docs[1][b]
            seen[b] &= (a[:, None] == c[None, :]) & (a[:, None] >= 0)
    return seen


def reference(q, k, v, do=None, *, dtype, causal=False, scale=None, kv_len=None, softcap=None, slopes=None, bias=None,
              max_distance=128, two_sided=False, docs=None, prefix_len=None, q_pos=None):
    """{name: (value, bound)} of o, lse and, with do, dq, dk, dv, dbias; CPU tensors in, float64 out."""
    B, H, n_q, d = q.shape
    n_k, G = k.shape[2], H // k.shape[1]
    u = torch.finfo(dtype).eps / 2
    u2 = max(u * u, E32)  # o with its residual
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    seen = visible(B, n_q, n_k, causal, kv_len, docs, prefix_len, q_pos)[:, None]
    # What masks hide does not count, whatever it holds.
    alive_q, alive_k = seen.any(-1)[..., None], seen.any(-2)[..., None]
    q = torch.where(alive_q, q.double(), 0.0)
    k, v = (torch.where(alive_k, t.double(), 0.0).repeat_interleave(G, 1) for t in (k, v))
    x = q @ k.transpose(2, 3) * scale
    mag = q.abs() @ k.abs().transpose(2, 3) * scale  # of the products
    es = (d + 8) * E32 * mag
    y, slope = x, torch.ones_like(x)
    if softcap is not None:
        t = torch.tanh(x / softcap)
        y, slope = softcap * t, 1 - t * t
        es = es + 8 * E32 * softcap
    s = y
    if slopes is not None or bias is not None:
        add = torch.zeros(B, H, n_q, n_k, dtype=torch.float64)
        index = []
        for b in range(B):
            pos = [i + (max(0, q_pos[b]) if q_pos is not None else 0) for i in range(n_q)]
            if slopes is not None:
                far = (torch.arange(n_k)[None, :] - torch.tensor(pos)[:, None]).abs().double()
                add[b] -= slopes.double()[:, None, None] * far
            if bias is not None:
                index.append(bucket_index(pos, n_k, bias.shape[0], max_distance, two_sided))
                add[b] += bias.double().t()[:, index[b]]
        s = s + add
        es = es + 8 * E32 * add.abs()
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    w = torch.exp(s - m)
    l = w.sum(-1, keepdim=True)
    lse = torch.where(l > 0, m + torch.log(l), -math.inf)
    p = w / torch.where(l > 0, l, 1.0)
    big = torch.where(lse.isinf(), 0.0, lse.abs())
    es = torch.where(seen, es + 8 * E32 * (torch.where(seen, s, 0.0).abs() + big + 1), 0.0)
    o = p @ v
    pv = p @ v.abs()
    ep = p * es                                  # error of the weights before their rounding
    norm = ep.sum(-1, keepdim=True)              # and of their sum
    eo = ep @ v.abs() + norm * pv + (u + n_k * E32) * pv
    out = {"o": (o, 1.01 * (eo + u * o.abs())), "lse": (lse[..., 0], 1.01 * (norm + 8 * E32 * (big + 1))[..., 0])}
    if do is None:
        return out
    g = torch.where(alive_q, do.double(), 0.0)
    D = (g * o).sum(-1, keepdim=True)
    gm = g.abs() @ v.abs().transpose(2, 3)       # magnitudes of dP's products
    go = (g.abs() * o.abs()).sum(-1, keepdim=True)
    # o before its rounding has the forward's error; its two parts leave u2 of it.
    eD = (g.abs() * (eo + u2 * o.abs())).sum(-1, keepdim=True) + (d + 8) * E32 * go
    dp = g @ v.transpose(2, 3) - D
    eps_p = es + norm                            # weights from the log-sum-exp
    ds = p * dp
    eds = p * ((d + 8) * E32 * (gm + go) + eD + eps_p * dp.abs()) + 4 * E32 * ds.abs()

    def shared(t):  # sum over the heads of a key head
        return t.view(B, H // G, G, n_k, d).sum(2)

    n = n_q * G
    dv = shared(p.transpose(2, 3) @ g)
    edv = shared((p * eps_p).transpose(2, 3) @ g.abs() + (u + n * E32) * (p.transpose(2, 3) @ g.abs()))
    dx = ds * slope
    edx = eds * slope + ds.abs() * 16 * E32 + (u + n * E32) * dx.abs()
    dq = scale * (dx @ k)
    edq = scale * ((edx + n_k * E32 * dx.abs()) @ k.abs())
    dk = scale * shared(dx.transpose(2, 3) @ q)
    edk = scale * shared(edx.transpose(2, 3) @ q.abs())
    for name, val, err in (("dq", dq, edq), ("dk", dk, edk), ("dv", dv, edv)):
        out[name] = (val, 1.01 * (err + u * val.abs()))
    if bias is not None:
        db, eb = (torch.zeros(bias.shape, dtype=torch.float64) for _ in range(2))
        for b in range(B):
            flat = index[b].flatten()
            db.index_add_(0, flat, ds[b].reshape(H, -1).t())
            eb.index_add_(0, flat, (eds + (n_q + n_k) * E32 * ds.abs())[b].reshape(H, -1).t())
        ub = torch.finfo(bias.dtype).eps / 2
        out["dbias"] = (db, 1.01 * (eb + ub * db.abs()))
    return out


def assert_within(name, got, want):
    """``got`` is within the bound of ``want`` everywhere (and infinite where it is)."""
    value, bound = want
    got = got.detach().double().cpu()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    inf = value.isinf()
    assert torch.equal(got[inf], value[inf]), name
    off = (got - value)[~inf].abs()
    limit = (bound + 2.0 ** -126)[~inf]
    assert torch.isfinite(off).all(), name + " is not finite"
    worst = (off / limit).max().item() if off.numel() else 0.0
    print("  %-5s at most %.3g of its bound" % (name, worst), flush=True)
    assert worst <= 1.0, (name, worst)
