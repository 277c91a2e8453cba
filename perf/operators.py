"""Attention with modified scores, a learned relative position bias and attention over a
shared prefix: the workloads whose speed is measured, their plain form in elementary torch
operations, the work they cannot do without, and float64 results to compare with.

A case's ``kind`` names the entry point it goes through:

* ``train``  -- ``attention_scored`` under autograd, forward and backward;
* ``fwd``    -- ``attention_scored_fwd`` for inference: prefill, and decode against a cache;
* ``shared`` -- ``attention_shared_prefix``: a decode step of a batch that shares a prefix.

``own`` says whether ``run`` makes the framework's calls or computes the plain form.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def _case(kind, dtype, B, H, H_kv, n_q, n_k, d, **more):
    """``gain``: standard deviation of the scores before a cap (queries are that much
    larger than N(0, 1)).  ``cap``, ``slopes``, ``docs`` (documents in a row of tokens,
    the last few tokens padding) and ``prefix`` (tokens every query sees) modify the
    scores; ``buckets`` with ``span`` (the distance of the last bucket) and ``two_sided``
    give the learned bias.  ``kv_min``: 0 for no key padding, else the valid key lengths
    run evenly from kv_min to n_k.  ``at_end``: the queries are the last valid
    positions, else the first.  ``n_p``: keys of the shared prefix."""
    c = {"kind": kind, "dtype": dtype, "B": B, "H": H, "H_kv": H_kv, "n_q": n_q, "n_k": n_k, "d": d,
         "causal": False, "gain": 1.0, "cap": 0.0, "slopes": False, "docs": 0, "prefix": 0, "buckets": 0, "span": 128,
         "two_sided": False, "kv_min": 0, "at_end": False, "n_p": 0}
    assert set(more) <= set(c) | {"name"}
    return {**c, **more}


def listed():
    return [
        # Training a language model with capped scores and grouped key heads.
        _case("train", "bf16", 2, 16, 4, 4096, 4096, 128, causal=True, cap=50.0, gain=4.0, name="train_bf16_cap_gqa_n4096_d128"),
        # Training with a distance bias instead of positions, an odd length.
        _case("train", "bf16", 4, 12, 12, 1999, 1999, 64, causal=True, slopes=True, name="train_bf16_slopes_n1999"),
        # Pretraining on documents packed into rows of tokens.
        _case("train", "fp16", 2, 16, 16, 8192, 8192, 64, causal=True, docs=14, name="train_fp16_docs_n8192"),
        # A prefix language model at full precision.
        _case("train", "fp32", 2, 8, 4, 700, 700, 64, causal=True, prefix=201, name="train_fp32_prefix_n700"),
        # Prefill of one prompt through capped scores and shared key heads.
        _case("fwd", "bf16", 1, 32, 8, 2047, 2047, 128, causal=True, cap=30.0, gain=4.0, name="prefill_bf16_cap_gqa_n2047_d128"),
        # Decode: one token for each of a batch of sequences with caches of different lengths.
        _case("fwd", "bf16", 16, 32, 8, 1, 32768, 128, causal=True, cap=50.0, gain=4.0, kv_min=9000, at_end=True,
              name="decode_bf16_cap_gqa_nk32768_d128"),
        # The smallest training call, where latency and launches count.
        _case("train", "fp32", 1, 4, 4, 64, 64, 64, buckets=32, two_sided=True, name="train_fp32_buckets_n64"),
        # An encoder's padded batch with a learned bias in both directions.
        _case("train", "bf16", 16, 12, 12, 512, 512, 64, buckets=32, two_sided=True, kv_min=100,
              name="train_bf16_buckets_padded_n512"),
        # A long decoder with a learned bias.
        _case("train", "bf16", 4, 16, 16, 4096, 4096, 64, causal=True, buckets=32, name="train_bf16_buckets_causal_n4096"),
        # Decode of a few tokens at once with a learned bias.
        _case("fwd", "fp16", 8, 16, 16, 3, 4097, 64, causal=True, buckets=32, kv_min=700, at_end=True,
              name="decode_fp16_buckets_nk4097"),
        # A decode step of 64 answers to one long prompt.
        _case("shared", "bf16", 64, 32, 8, 1, 640, 128, n_p=16384, kv_min=5, at_end=True, name="shared_bf16_b64_np16384_d128"),
        # A few speculative tokens of a few sequences after a short common prompt.
        _case("shared", "fp16", 5, 8, 8, 4, 77, 64, causal=True, n_p=1000, kv_min=30, at_end=True, name="shared_fp16_b5_np1000"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["train", "train", "train", "prefill", "decode", "decode", "shared", "shared"])
    d, H_kv = rng.choice([64, 128]), _log_uniform(rng, 1, 16)
    G = rng.choice([1, 1, 2, 3, 4, 8])
    B = _log_uniform(rng, 1, 16)
    if kind == "shared":
        n_q = rng.choice([1, 1, 1, rng.randint(2, 8)])
        B, n_k = _log_uniform(rng, 2, 128), _log_uniform(rng, max(8, n_q), 2048)
        c = _case("shared", rng.choice(["bf16", "bf16", "fp16", "fp32"]), B, H_kv * G, H_kv, n_q, n_k, d, at_end=True,
                  causal=n_q > 1, n_p=_log_uniform(rng, 100, 32768), kv_min=max(n_q, n_k // rng.randint(2, 9)))
    else:
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        if kind == "decode":
            n_q, n = rng.choice([1, 1, rng.randint(2, 16)]), _log_uniform(rng, 200, 65536)
            c = _case("fwd", dtype, B, H_kv * G, H_kv, n_q, n, d, causal=True, at_end=True)
        elif kind == "prefill":
            n = _log_uniform(rng, 65, 8192)
            c = _case("fwd", dtype, min(B, 4), H_kv * G, H_kv, n, n, d, causal=True)
        else:
            n = _log_uniform(rng, 50, 8192)
            c = _case("train", dtype, B, H_kv * G, H_kv, n, n, d, causal=rng.random() < 0.7)
        mods = rng.choice(["cap", "slopes", "buckets", "buckets", "docs", "prefix", "cap buckets"])
        if "cap" in mods:
            c["cap"], c["gain"] = rng.choice([20.0, 30.0, 50.0]), 4.0
        if "slopes" in mods:
            c["slopes"] = True
        if "buckets" in mods:
            c["buckets"], c["span"] = rng.choice([8, 32, 32, 64]), rng.choice([64, 128, 128, 300])
            c["two_sided"] = not c["causal"]
        if mods == "docs" and kind != "decode":
            c["docs"] = rng.randint(2, max(2, min(40, n // 16)))
        if mods == "prefix" and c["causal"]:
            c["prefix"] = rng.randint(1, n)
        if B > 1 and not c["docs"] and rng.random() < 0.4:
            c["kv_min"] = max(c["n_q"] if c["at_end"] else 1, n // rng.randint(2, 8))
    # No dearer than the largest listed case, in work (float32 products take six times the
    # 16-bit ones' time) and in the plain form's score matrices.
    while (work(c)["flops"] > (8e10 if c["dtype"] == "fp32" else 4.7e11) or work(c)["bytes"] > 1.3e9
           or c["B"] * c["H"] * c["n_q"] * (c["n_k"] + c["n_p"]) > 1.05e9):
        if c["B"] > 2:
            c["B"] = c["B"] * 2 // 3
        else:
            c["n_q"], c["n_k"] = max(1, c["n_q"] * 2 // 3), max(16, c["n_k"] * 2 // 3)
            c["kv_min"], c["prefix"] = min(c["kv_min"], c["n_k"]), min(c["prefix"], c["n_k"])
            c["docs"] = min(c["docs"], c["n_k"] // 8)
            if c["kv_min"]:
                c["kv_min"] = max(c["kv_min"], c["n_q"] if c["at_end"] else 1)
    if c["B"] == 1:
        c["kv_min"] = 0
    return c


def _kv_lens(case):
    B, n, lo = case["B"], case["n_k"], case["kv_min"]
    return [n] * B if not lo else [lo + (n - lo) * b // max(1, B - 1) for b in range(B)]


def _doc_lens(case):
    """Lengths of a row's documents (their order comes from the seed); what is left is padding."""
    m, n = case["docs"], case["n_k"] - case["n_k"] // 50
    weights = [1 + (7 * i + 3) % 11 for i in range(m)]
    return [max(1, n * w // sum(weights)) for w in weights]


def _pairs(case):
    """Query-key pairs that contribute to a pass; for a shared prefix those of the own keys."""
    n_q, total = case["n_q"], 0
    if case["docs"]:
        one = sum(m * (m + 1) // 2 if case["causal"] else m * m for m in _doc_lens(case))
        return one * case["B"] * case["H"]
    for n in _kv_lens(case):
        if not case["causal"]:
            total += n_q * n
            continue
        p0 = n - n_q if case["at_end"] else 0
        total += sum(min(n, max(p0 + i + 1, case["prefix"])) for i in range(n_q))
    return total * case["H"]


def work(case):
    B, H, H_kv, n_q, n_k, n_p, d = (case[x] for x in ("B", "H", "H_kv", "n_q", "n_k", "n_p", "d"))
    e, P = BYTES[case["dtype"]], _pairs(case)
    keys = sum(_kv_lens(case)) * H_kv
    q, kv = e * B * H * n_q * d, e * 2 * keys * d
    if case["kind"] == "shared":
        return {"bytes": 2 * q + kv + e * 2 * H_kv * n_p * d, "flops": 4 * d * (P + B * H * n_q * n_p)}
    if case["kind"] == "fwd":
        return {"bytes": 2 * q + kv, "flops": 4 * d * P}
    # forward S, O; backward S again (the score matrix is never stored), dP, dV, dK, dQ
    return {"bytes": 4 * q + kv + e * 2 * B * H_kv * n_k * d, "flops": 14 * d * P}


def _int32(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, H, H_kv, n_q, n_k, d = (case[x] for x in ("B", "H", "H_kv", "n_q", "n_k", "d"))
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dt)

    s = {"case": case, "kv_len": None, "q_pos": None, "docs": None, "prefix_len": None, "slopes": None, "table": None}
    s["q"], s["k"], s["v"] = normal(B, H, n_q, d, std=case["gain"]), normal(B, H_kv, n_k, d), normal(B, H_kv, n_k, d)
    lens = _int32(_kv_lens(case))[torch.randperm(B, generator=g, device="cuda")].contiguous()
    if case["kv_min"]:
        s["kv_len"] = lens
    if case["at_end"]:
        s["q_pos"] = lens - n_q
    if case["docs"]:
        rows = []
        for _ in range(B):
            order = torch.randperm(case["docs"], generator=g, device="cuda")
            size = _int32(_doc_lens(case))[order].long()
            row = torch.arange(case["docs"], device="cuda", dtype=torch.int32).repeat_interleave(size)[:n_k]
            rows.append(torch.nn.functional.pad(row, (0, n_k - row.numel()), value=-1))
        s["docs"] = torch.stack(rows)
    if case["prefix"]:
        s["prefix_len"] = _int32([case["prefix"]] * B)
    if case["slopes"]:
        s["slopes"] = torch.exp2(-8.0 / H * torch.arange(1, H + 1, device="cuda", dtype=torch.float32))
    if case["buckets"]:
        s["table"] = normal(case["buckets"], H)
    if case["kind"] == "shared":
        s["k_prefix"], s["v_prefix"] = normal(H_kv, case["n_p"], d), normal(H_kv, case["n_p"], d)
    if case["kind"] == "train":
        s["do"] = normal(B, H, n_q, d)
        for x in ("q", "k", "v", "table"):
            if s[x] is not None:
                s[x].requires_grad_()
    return s


def run(state):
    if not own:
        with torch.no_grad():
            return _plain_shared(state) if state["case"]["kind"] == "shared" else _plain(state)
    from paper_2112_05682_amd import attention_scored, attention_scored_fwd, attention_shared_prefix

    case, q, k, v = state["case"], state["q"], state["k"], state["v"]
    if case["kind"] == "shared":
        return {"o": attention_shared_prefix(q, state["k_prefix"], state["v_prefix"], k, v, causal=case["causal"],
                                             kv_len=state["kv_len"], q_pos=state["q_pos"])}
    mods = {"causal": case["causal"], "softcap": case["cap"] or None, "slopes": state["slopes"], "bias": state["table"],
            "max_distance": case["span"], "bidirectional": case["two_sided"], "docs": state["docs"],
            "prefix_len": state["prefix_len"], "kv_len": state["kv_len"], "q_pos": state["q_pos"]}
    if case["kind"] == "fwd":
        o, _ = attention_scored_fwd(q, k, v, need_lse=False, **mods)
        return {"o": o}
    o = attention_scored(q, k, v, **mods)
    leaves = {"dq": q, "dk": k, "dv": v}
    if state["table"] is not None:
        leaves["dtable"] = state["table"]
    return {"o": o, **dict(zip(leaves, torch.autograd.grad(o, tuple(leaves.values()), state["do"])))}


# ---- the plain form: float32 matrices of scores, weights and their gradients.

def _edges(n, span):
    """Smallest distance of each of a side's n buckets: one bucket a distance up to
    n // 2, then bucket b starts at h (span / h)^((b - h) / (n - h)), h = n // 2."""
    h = n // 2
    edges = list(range(h))
    for b in range(h, n):
        x = h
        while x ** (n - h) < span ** (b - h) * h ** (n - b):
            x += 1
        edges.append(x)
    return edges


def _bucket(case, distance):
    """Bucket of each distance j - position."""
    n = case["buckets"] // 2 if case["two_sided"] else case["buckets"]
    edges = torch.tensor(_edges(n, case["span"]), device=distance.device)
    far = distance.abs() if case["two_sided"] else (-distance).clamp(min=0)
    side = n * (distance > 0).long() if case["two_sided"] else 0
    return torch.searchsorted(edges, far, right=True) - 1 + side


def _visible(state):
    """Positions j - pos_i, [B, 1, n_q, n_k], and which pairs are visible."""
    case, dev = state["case"], state["q"].device
    n_q, n_k = case["n_q"], case["n_k"]
    j = torch.arange(n_k, device=dev)
    pos = torch.arange(n_q, device=dev)[None]
    if state["q_pos"] is not None:
        pos = pos + state["q_pos"].long()[:, None]
    distance = (j[None, None, :] - pos[:, :, None])[:, None]
    seen = torch.ones_like(distance, dtype=torch.bool)
    if case["causal"]:
        seen = distance <= 0
        if state["prefix_len"] is not None:
            seen = seen | (j < state["prefix_len"].long()[:, None])[:, None, None, :]
    if state["kv_len"] is not None:
        seen = seen & (j < state["kv_len"].long()[:, None])[:, None, None, :]
    if state["docs"] is not None:
        a, b = state["docs"][:, None, :n_q, None], state["docs"][:, None, None, :]
        seen = seen & (a == b) & (a >= 0)
    return distance, seen


def _softmax_parts(s):
    """exp(s - max) of each row and its sum, 0 and 1 for a row of -inf."""
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    l = e.sum(-1, keepdim=True)
    return e, torch.where(l == 0, 1.0, l)


def _plain(state):
    case, dt = state["case"], state["q"].dtype
    B, H, H_kv, n_q, n_k, d = (case[x] for x in ("B", "H", "H_kv", "n_q", "n_k", "d"))
    rows = (B, H_kv, H // H_kv * n_q)  # the queries of a group of heads, one under the other
    q, k, v = state["q"].float().view(*rows, d), state["k"].float(), state["v"].float()
    scale = 1.0 / math.sqrt(d)
    kt = k.transpose(2, 3).contiguous()
    s = (torch.matmul(q, kt) * scale).view(B, H, n_q, n_k)
    t = None
    if case["cap"]:
        t = torch.tanh(s / case["cap"])
        s = case["cap"] * t
    distance, seen = _visible(state)
    if state["slopes"] is not None:
        s = s - state["slopes"][:, None, None] * distance.abs().float()
    if state["table"] is not None:
        s = s + state["table"].float()[_bucket(case, distance[:, 0])].permute(0, 3, 1, 2)
    p, l = _softmax_parts(torch.where(seen, s, -math.inf))
    p = p / l
    o = torch.matmul(p.view(*rows, n_k), v).view(B, H, n_q, d)
    if case["kind"] == "fwd":
        return {"o": o.to(dt)}
    do = state["do"].float()
    g = do.view(*rows, d)
    dv = torch.matmul(p.view(*rows, n_k).transpose(2, 3).contiguous(), g)
    ds = torch.matmul(g, v.transpose(2, 3).contiguous()).view(B, H, n_q, n_k)
    ds = p * (ds - (do * o).sum(-1, keepdim=True))
    out = {"o": o.to(dt), "dv": dv.to(dt)}
    if state["table"] is not None:
        # Sums of the diagonals: rows flipped and shifted by one place each.
        x = torch.nn.functional.pad(ds.sum(0).flip(1), (0, n_q)).view(H, -1)[:, : n_q * (n_k + n_q - 1)]
        x = x.view(H, n_q, n_k + n_q - 1).sum(1, dtype=torch.float64)
        at = _bucket(case, torch.arange(1 - n_q, n_k, device=q.device))
        one = torch.nn.functional.one_hot(at, case["buckets"]).double()
        out["dtable"] = torch.matmul(x, one).t().contiguous().to(dt)
    if t is not None:
        ds = ds * (1 - t * t)
    ds = (ds * scale).view(*rows, n_k)
    out["dq"] = torch.matmul(ds, k).view(B, H, n_q, d).to(dt)
    out["dk"] = torch.matmul(ds.transpose(2, 3).contiguous(), q).to(dt)
    return out


def _plain_shared(state):
    case, dt = state["case"], state["q"].dtype
    B, H, H_kv, n_q, n_k, n_p, d = (case[x] for x in ("B", "H", "H_kv", "n_q", "n_k", "n_p", "d"))
    G, scale = H // H_kv, 1.0 / math.sqrt(d)
    q = state["q"].float().view(B, H_kv, G * n_q, d)
    # Every sequence's queries against the prefix, once for each key head.
    qp = q.transpose(0, 1).reshape(H_kv, B * G * n_q, d)
    sp = torch.matmul(qp, state["k_prefix"].float().transpose(1, 2).contiguous()) * scale
    sp = sp.view(H_kv, B, G * n_q, n_p).transpose(0, 1).reshape(B, H, n_q, n_p)
    so = (torch.matmul(q, state["k"].float().transpose(2, 3).contiguous()) * scale).view(B, H, n_q, n_k)
    so = torch.where(_visible(state)[1], so, -math.inf)
    e, l = _softmax_parts(torch.cat([sp, so], dim=-1))
    p = (e / l).view(B, H_kv, G * n_q, n_p + n_k)
    pp = p[..., :n_p].transpose(0, 1).reshape(H_kv, B * G * n_q, n_p)
    o = torch.matmul(pp, state["v_prefix"].float()).view(H_kv, B, G * n_q, d).transpose(0, 1)
    o = o + torch.matmul(p[..., n_p:].contiguous(), state["v"].float())
    return {"o": o.reshape(B, H, n_q, d).to(dt)}


# ---- float64, one (batch, head) at a time, from the definition.

def _exact_bias(case, state, b, h, j0, j1):
    """Bias and visibility of queries j0 .. j1 - 1 of batch b, head h, against every key."""
    n_k, dev = case["n_k"], state["q"].device
    start = 0 if state["q_pos"] is None else int(state["q_pos"][b])
    key = torch.arange(n_k, device=dev)
    pos = torch.arange(start + j0, start + j1, device=dev)
    ahead = key[None, :] - pos[:, None]
    bias = torch.zeros(ahead.shape, dtype=torch.float64, device=dev)
    ok = (key < (n_k if state["kv_len"] is None else int(state["kv_len"][b])))[None, :].expand(ahead.shape)
    if case["causal"]:
        reach = 0 if state["prefix_len"] is None else int(state["prefix_len"][b])
        ok = ok & ((ahead <= 0) | (key < reach)[None, :])
    if state["docs"] is not None:
        ids = state["docs"][b]
        ok = ok & (ids[j0:j1, None] == ids[None, :]) & (ids[j0:j1, None] >= 0)
    if state["slopes"] is not None:
        bias -= state["slopes"][h].double() * ahead.abs()
    index = None
    if state["table"] is not None:
        n = case["buckets"] // (2 if case["two_sided"] else 1)
        far = ahead.abs() if case["two_sided"] else (-ahead).clamp(min=0)
        index = torch.zeros_like(ahead)
        for edge in _edges(n, case["span"])[1:]:
            index += far >= edge
        if case["two_sided"]:
            index += n * (ahead > 0)
        bias += state["table"].detach()[:, h].double()[index]
    return bias, ok, index


def exact(case, seed):
    s = prepare(case, seed)
    B, H, H_kv, n_q, d = (case[x] for x in ("B", "H", "H_kv", "n_q", "d"))
    n_k, scale, train = case["n_k"], 1.0 / math.sqrt(d), case["kind"] == "train"
    with torch.no_grad():
        q, k, v = (s[x].detach() for x in ("q", "k", "v"))
        o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        if train:
            dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device=q.device) for x in (q, k, v))
            table = torch.zeros(max(1, case["buckets"]), H, dtype=torch.float64, device=q.device)
        step = max(1, (1 << 26) // (n_k + case["n_p"]))
        for b in range(B):
            for h in range(H):
                c = h // (H // H_kv)
                kt, vt = k[b, c].double(), v[b, c].double()
                if case["kind"] == "shared":
                    kt = torch.cat([s["k_prefix"][c].double(), kt])
                    vt = torch.cat([s["v_prefix"][c].double(), vt])
                for i in range(0, n_q, step):
                    e = min(n_q, i + step)
                    qi = q[b, h, i:e].double()
                    x = torch.mm(qi, kt.t()) * scale
                    slope = None
                    if case["cap"]:
                        y = torch.tanh(x / case["cap"])
                        x, slope = case["cap"] * y, 1 - y * y
                    bias, ok, index = _exact_bias(case, s, b, h, i, e)
                    if case["kind"] == "shared":
                        bias = torch.nn.functional.pad(bias, (case["n_p"], 0))
                        ok = torch.nn.functional.pad(ok, (case["n_p"], 0), value=True)
                    x = (x + bias).masked_fill(~ok, -math.inf)
                    p = torch.nan_to_num(torch.softmax(x, dim=1), nan=0.0)
                    o[b, h, i:e] = torch.mm(p, vt)
                    if not train:
                        continue
                    g = s["do"][b, h, i:e].double()
                    dv[b, c] += torch.mm(p.t(), g)
                    w = torch.mm(g, vt.t())
                    w = p * (w - (w * p).sum(1, keepdim=True))
                    if index is not None:
                        table[:, h] += torch.bincount(index.flatten(), weights=w.flatten(), minlength=case["buckets"])
                    if slope is not None:
                        w = w * slope
                    dq[b, h, i:e] = torch.mm(w, kt) * scale
                    dk[b, c] += torch.mm(w.t(), qi) * scale
        if not train:
            return {"o": o}
        out = {"o": o, "dq": dq, "dk": dk, "dv": dv}
        if case["buckets"]:
            out["dtable"] = table
        return out
