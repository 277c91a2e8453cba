"""Attention with modified scores on the GPU against float64 (scored_ref.py, whose bounds
count roundings): caps, distance biases, learned biases with their gradient, documents,
prefixes, grouped key heads, positions against a cache, every kernel variant."""
import pytest
import torch

from paper_2112_05682_amd import attention_scored, attention_scored_bwd, attention_scored_fwd
from scored_ref import assert_within, reference

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def inputs(dtype, B, H, Hkv, nq, nk, d, seed=0, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    q, do = (torch.randn(B, H, nq, d, generator=g) for _ in range(2))
    k, v = (torch.randn(B, Hkv, nk, d, generator=g) for _ in range(2))
    return [t.to(DT[dtype]) for t in (q * gain, k, v, do)]


def alibi(H):
    return torch.exp2(-8.0 / H * torch.arange(1, H + 1, dtype=torch.float32))


def table(buckets, H, dtype, seed=5):
    return torch.randn(buckets, H, generator=torch.Generator().manual_seed(seed)).to(dtype)


def packed(B, n, lens, pad):
    """Documents of the given lengths in turn, the last ``pad`` tokens without one."""
    ids = torch.arange(len(lens), dtype=torch.int32).repeat_interleave(torch.tensor(lens))
    ids = ids.repeat(n // ids.numel() + 1)[:n].clone()
    ids = torch.stack([ids.roll(7 * b) for b in range(B)])
    if pad:
        ids[:, n - pad:] = -1
    return ids


def to_gpu(mods):
    r = {}
    for key, x in mods.items():
        if key in ("kv_len", "prefix_len", "q_pos") and x is not None:
            r[key] = torch.tensor(x, dtype=torch.int32, device="cuda")
        elif key == "docs" and x is not None:
            r[key] = tuple(t.cuda() for t in x)
        elif key == "two_sided":
            r["bidirectional"] = x
        else:
            r[key] = x.cuda() if isinstance(x, torch.Tensor) else x
    return r


def check(dtype, q, k, v, do, mods, train=True):
    ref = reference(q, k, v, do if train else None, dtype=DT[dtype], **mods)
    m = to_gpu(mods)
    qg, kg, vg, dog = (t.cuda() for t in (q, k, v, do))
    o, lse, o_lo = attention_scored_fwd(qg, kg, vg, residual=True, **m)
    torch.cuda.synchronize()
    assert_within("o", o, ref["o"])
    assert_within("lse", lse, ref["lse"])
    if not train:
        return
    got = dict(zip(("dq", "dk", "dv", "dbias"), attention_scored_bwd(qg, kg, vg, o, lse, dog, o_lo=o_lo, **m)))
    torch.cuda.synchronize()
    for name in ("dq", "dk", "dv") + (("dbias",) if mods.get("bias") is not None else ()):
        assert_within(name, got[name], ref[name])


MODS = {
    "plain": lambda H, nq, nk, dt: {},
    "causal": lambda H, nq, nk, dt: {"causal": True},
    "cap": lambda H, nq, nk, dt: {"causal": True, "softcap": 5.0},
    "slopes": lambda H, nq, nk, dt: {"slopes": alibi(H)},
    "slopes_causal": lambda H, nq, nk, dt: {"slopes": alibi(H), "causal": True},
    "buckets": lambda H, nq, nk, dt: {"bias": table(32, H, dt), "two_sided": True},
    "buckets_causal": lambda H, nq, nk, dt: {"bias": table(8, H, dt), "causal": True, "max_distance": 40},
    "buckets_ahead": lambda H, nq, nk, dt: {"bias": table(16, H, torch.float32), "two_sided": False, "max_distance": 20},
    "all": lambda H, nq, nk, dt: {"bias": table(12, H, dt), "causal": True, "softcap": 3.0, "slopes": alibi(H),
                                  "prefix_len": [nk // 3, 0], "kv_len": [nk, max(1, nk - 5)], "max_distance": 50},
    "prefix": lambda H, nq, nk, dt: {"causal": True, "prefix_len": [nk // 2 + 1, 1]},
    "docs": lambda H, nq, nk, dt: {"causal": True, "docs": (packed(2, nq, [5, 40, 1, 70, 33], 3), packed(2, nk, [5, 40, 1, 70, 33], 3))},
    "docs_far": lambda H, nq, nk, dt: {"docs": (packed(2, nq, [130, 3, 90], 0), packed(2, nk, [90, 130, 3], 11))},
    "padded": lambda H, nq, nk, dt: {"kv_len": [nk // 2, 0], "softcap": 20.0, "bias": table(8, H, dt), "two_sided": True},
}
SHAPES = [("bf16", 4, 2, 150, 150, 64), ("fp16", 3, 1, 100, 217, 128), ("fp32", 2, 2, 97, 130, 64), ("bf16", 6, 2, 300, 300, 128),
          ("fp32", 4, 1, 70, 70, 128), ("fp16", 2, 1, 1, 1, 64)]


@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_forward_and_backward(shape, mod):
    dtype, H, Hkv, nq, nk, d = shape
    print("scored", shape, mod, flush=True)
    q, k, v, do = inputs(dtype, 2, H, Hkv, nq, nk, d, gain=2.0)
    check(dtype, q, k, v, do, MODS[mod](H, nq, nk, DT[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("BH,n,d", [(135, 70, 64), (270, 100, 64), (270, 100, 128), (40, 65, 128)])
def test_row_waves(dtype, BH, n, d):
    """Grids on which 1, 2 or 4 waves of a workgroup have rows of their own."""
    print("rows", dtype, BH, n, d, flush=True)
    q, k, v, do = inputs(dtype, BH, 1, 1, n, n, d)
    check(dtype, q, k, v, do, {"causal": True, "softcap": 8.0, "bias": table(16, 1, DT[dtype]), "max_distance": 30},
          train=BH < 140)


DECODE = [  # dtype, B, H, Hkv, nq, nk, d, kv_len
    ("bf16", 2, 8, 2, 1, 3000, 128, [3000, 1]), ("fp16", 3, 4, 4, 3, 1500, 64, [1500, 700, 3]),
    ("fp32", 2, 6, 2, 1, 900, 64, [900, 33]), ("bf16", 1, 12, 1, 5, 777, 64, [777]), ("bf16", 2, 3, 1, 16, 260, 128, [260, 16]),
    ("fp32", 2, 4, 4, 2, 2100, 128, [2100, 2]), ("bf16", 1, 1, 1, 1, 1, 64, [1]), ("fp16", 2, 40, 1, 1, 400, 128, [400, 399]),
    ("bf16", 1, 130, 1, 1, 500, 64, [500]), ("fp32", 1, 71, 1, 3, 150, 64, [150]), ("fp16", 2, 24, 2, 30, 333, 64, [333, 40]),
]


@pytest.mark.parametrize("mod", ["none", "cap", "slopes", "buckets", "prefix", "docs", "empty"])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(map(str, c[:7])))
def test_decode(case, mod):
    """The last positions of caches of different lengths; garbage behind them is not seen."""
    dtype, B, H, Hkv, nq, nk, d, lens = case
    print("decode", case, mod, flush=True)
    q, k, v, do = inputs(dtype, B, H, Hkv, nq, nk, d, gain=2.0)
    lens = [0] * B if mod == "empty" else lens
    for b in range(B):
        k[b, :, lens[b]:] = float("nan")
        v[b, :, lens[b]:] = float("inf")
    mods = {"causal": True, "kv_len": lens, "q_pos": [n - nq for n in lens]}
    mods.update({"none": {}, "empty": {}, "cap": {"softcap": 4.0}, "slopes": {"slopes": alibi(H)},
                 "buckets": {"bias": table(32, H, DT[dtype]), "softcap": 30.0}, "prefix": {"prefix_len": [5] * B},
                 "docs": {"docs": (torch.ones(B, nq, dtype=torch.int32), (torch.arange(nk, dtype=torch.int32) // 60 % 3 - 1).repeat(B, 1))}}[mod])
    check(dtype, q, k, v, do, mods, train=False)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_what_masks_hide_may_hold_anything(dtype, d):
    """NaN and infinities behind kv_len, and in tokens without a document, reach no result."""
    B, H, Hkv, n = 2, 4, 2, 200
    q, k, v, do = inputs(dtype, B, H, Hkv, n, n, d)
    lens = [150, 64]
    for b in range(B):
        k[b, :, lens[b]:], v[b, :, lens[b]:] = float("nan"), float("inf")
    check(dtype, q, k, v, do, {"kv_len": lens})
    q, k, v, do = inputs(dtype, B, H, Hkv, n, n, d)
    ids = packed(B, n, [30, 50, 9], 20)
    ids[:, 40:55] = -3
    for b in range(B):
        for t in (q, k, v, do):
            t[b][:, ids[b] < 0] = float("nan")
    check(dtype, q, k, v, do, {"docs": (ids, ids), "causal": True, "bias": table(8, H, DT[dtype])})
    check(dtype, q, k, v, do, {"docs": (ids, ids), "softcap": 10.0})


def test_long_documents_are_skipped_to():
    """Rows and keys whose documents lie many tiles apart (windows of 64 tiles each)."""
    n = 9000
    q, k, v, do = inputs("bf16", 1, 1, 1, 130, n, 64)
    kd = (torch.arange(n, dtype=torch.int32) // 100)[None].contiguous()
    qd = torch.tensor([[0] * 30 + [89] * 40 + [44] * 60], dtype=torch.int32)
    check("bf16", q, k, v, do, {"docs": (qd, kd)})
    q, k, v, do = inputs("bf16", 1, 1, 1, n, 130, 64)
    check("bf16", q, k, v, do, {"docs": (kd, qd)})


@pytest.mark.parametrize("layout", ["bnhd", "sliced", "shared"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides(layout, dtype):
    B, H, n, d = 2, 4, 90, 64
    g = torch.Generator().manual_seed(1)

    def make(heads):
        if layout == "bnhd":
            return torch.randn(B, n, heads, d, generator=g).to(DT[dtype]).cuda().transpose(1, 2)
        if layout == "sliced":
            return torch.randn(B, heads, n, d + 32, generator=g).to(DT[dtype]).cuda()[..., 16:16 + d]
        return torch.randn(B, 1, n, d, generator=g).to(DT[dtype]).cuda().expand(B, heads, n, d)

    q, k, v = make(H), make(2), make(2)
    do = torch.randn(B, n, H, d, generator=g).to(DT[dtype]).cuda().transpose(1, 2)
    mods = {"causal": True, "slopes": alibi(H), "softcap": 10.0}
    ref = reference(*(t.cpu() for t in (q, k, v, do)), dtype=DT[dtype], **mods)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    o = attention_scored(*leaves, **to_gpu(mods))
    grads = torch.autograd.grad(o, leaves, do)
    for name, x in zip(("o", "dq", "dk", "dv"), (o, *grads)):
        assert_within(name, x, ref[name])
    out = torch.empty(B, n, H, d, dtype=DT[dtype], device="cuda").transpose(1, 2)
    assert attention_scored_fwd(q, k, v, out=out, need_lse=False, **to_gpu(mods))[0] is out
    assert torch.equal(out, o)


def test_gradients_against_differences():
    """Central differences of sum(o do) in float64 arithmetic of the reference, and the
    kernels' float32 gradients along the same directions."""
    B, H, n, d = 1, 2, 40, 64
    q, k, v, do = inputs("fp32", B, H, 1, n, n, d)
    mods = {"causal": True, "softcap": 2.0, "bias": table(8, H, torch.float32), "max_distance": 20, "slopes": alibi(H)}
    m = to_gpu(mods)
    leaves = [t.cuda().requires_grad_() for t in (q, k, v, mods["bias"])]
    m.pop("bias")
    grads = torch.autograd.grad(attention_scored(*leaves[:3], bias=leaves[3], **m), leaves, do.cuda())
    g = torch.Generator().manual_seed(3)
    x = [t.double() for t in (q, k, v, mods["bias"])]
    rest = {key: val for key, val in mods.items() if key != "bias"}

    def loss(y):
        return (reference(*y[:3], dtype=torch.float32, bias=y[3], **rest)["o"][0] * do.double()).sum()

    for i, name in enumerate(("dq", "dk", "dv", "dbias")):
        r = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        up, down = ([t + s * h * r if j == i else t for j, t in enumerate(x)] for s in (1, -1))
        want = ((loss(up) - loss(down)) / (2 * h)).item()
        got = (grads[i].double().cpu() * r).sum().item()
        # h^2 of the third derivative and 1e-16 / h of the loss; the kernels' float32.
        size = (grads[i].double().cpu().abs() * r.abs()).sum().item()
        assert abs(got - want) <= 1e-5 * size + 1e-7, (name, got, want)


def test_same_results_every_time():
    q, k, v, do = (t.cuda() for t in inputs("bf16", 2, 6, 2, 300, 300, 64))
    m = to_gpu({"causal": True, "bias": table(32, 6, torch.float32), "softcap": 10.0})
    first = None
    for _ in range(4):
        o, lse, o_lo = attention_scored_fwd(q, k, v, residual=True, **m)
        r = (o, lse, *attention_scored_bwd(q, k, v, o, lse, do, o_lo=o_lo, **m))
        first = first or r
        assert all(torch.equal(a, b) for a, b in zip(first, r))


def test_parts_of_the_gradient():
    """Skipped gradients are None and the others the same."""
    q, k, v, do = (t.cuda() for t in inputs("fp16", 1, 2, 1, 80, 80, 64))
    m = to_gpu({"bias": table(8, 2, torch.float16), "two_sided": True})
    o, lse, o_lo = attention_scored_fwd(q, k, v, residual=True, **m)
    full = attention_scored_bwd(q, k, v, o, lse, do, o_lo=o_lo, **m)
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, True, False)):
        part = attention_scored_bwd(q, k, v, o, lse, do, need_dq=need[0], need_dkdv=need[1], need_dbias=need[2], o_lo=o_lo, **m)
        for x, y, n in zip(part, full, (need[0], need[1], need[1], need[2])):
            assert (torch.equal(x, y) if n else x is None)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_a_bias_of_minus_infinity_hides(dtype, d):
    """A window: far keys' bucket is -inf, also of the first tiles that a row meets.  The same
    bits as with -10^4, whose weights are 0 (2^-14000 of the nearest key's)."""
    B, H, Hkv, n = 2, 4, 2, 700
    q, k, v, do = inputs(dtype, B, H, Hkv, n, n, d, seed=3)
    t = table(32, H, DT[dtype])
    t[31] = -1e4
    hidden = t.clone()
    hidden[31] = float("-inf")
    ref = reference(q, k, v, do, dtype=DT[dtype], causal=True, bias=t, max_distance=40)
    dev = [x.cuda() for x in (q, k, v)]
    got = []
    for bias in (t.cuda(), hidden.cuda()):
        kw = dict(causal=True, bias=bias, max_distance=40)
        o, lse, o_lo = attention_scored_fwd(*dev, residual=True, **kw)
        grads = attention_scored_bwd(*dev, o, lse, do.cuda(), o_lo=o_lo, **kw)
        last = attention_scored_fwd(dev[0][:, :, -2:], *dev[1:], q_pos=torch.full((B,), n - 2, dtype=torch.int32, device="cuda"),
                                    **kw)
        got.append((o, lse, *grads, *last))
    torch.cuda.synchronize()
    for name, x in zip(("o", "lse", "dq", "dk", "dv", "dbias"), got[0]):
        assert_within(name, x, ref[name])
    for a, b in zip(*got):
        assert torch.equal(a, b)
    # Every bucket: rows that see nothing.
    kw = dict(causal=True, bias=torch.full_like(t, float("-inf")).cuda(), max_distance=40)
    o, lse, o_lo = attention_scored_fwd(*dev, residual=True, **kw)
    for x in (o, *attention_scored_bwd(*dev, o, lse, do.cuda(), o_lo=o_lo, **kw)):
        assert not x.any()
    assert (lse == float("-inf")).all()


@pytest.mark.parametrize("mod", ["none", "cap", "slopes", "buckets", "prefix", "empty"])
@pytest.mark.parametrize("case", [("fp32", 3, 8, 1, 1, 1300, 64, [1300, 65, 1]), ("fp32", 2, 6, 2, 2, 700, 128, [700, 31]),
                                  ("fp32", 1, 5, 5, 1, 3000, 128, [3000]), ("fp32", 2, 2, 2, 8, 500, 64, [500, 8]),
                                  ("fp32", 300, 4, 1, 1, 40, 64, None)], ids=lambda c: "-".join(map(str, c[:7])))
def test_few_float32_rows(case, mod):
    """1 to 8 rows of a key head, in one range and in several."""
    test_decode(case[:7] + (case[7] or [1 + i % 40 for i in range(case[1])],), mod)


@pytest.mark.parametrize("d", [64, 128])
def test_few_float32_rows_of_a_strided_cache(d):
    B, H, Hkv, n = 2, 4, 2, 600
    q, k, v, _ = (t.cuda() for t in inputs("fp32", B, H, Hkv, 1, n, d))
    want = attention_scored_fwd(q, k, v, softcap=3.0)
    rows = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v)]
    wide = [torch.cat([t, t], 3)[..., :d] for t in (k, v)]
    out = torch.full((B, 1, H, d), 7.0, device="cuda").transpose(1, 2)
    for x in (rows, wide):
        for a, b in zip(attention_scored_fwd(q, *x, softcap=3.0, out=out), want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,B,H,Hkv,n,d,mod", [
    ("bf16", 1, 8, 4, 3000, 64, "buckets"), ("fp16", 1, 4, 1, 6100, 64, "cap"), ("bf16", 1, 2, 1, 4100, 128, "slopes"),
    ("bf16", 3, 4, 4, 3000, 64, "prefix"), ("bf16", 2, 8, 8, 2000, 128, "none"), ("fp32", 1, 4, 2, 1700, 64, "buckets"),
    ("fp32", 2, 6, 6, 900, 128, "prefix")])
def test_key_ranges_of_many_rows(dtype, B, H, Hkv, n, d, mod):
    """Long heads whose row tiles are split over keys; the first rows, some in the middle, and
    the last ones against the reference of those rows."""
    q, k, v, _ = inputs(dtype, B, H, Hkv, n, n, d, seed=11, gain=2.0)
    mods = {"kv_len": [n - 333 * b for b in range(B)]}
    mods.update({"none": {}, "cap": {"softcap": 4.0}, "slopes": {"slopes": alibi(H)}, "prefix": {"prefix_len": [n // 3] * B},
                 "buckets": {"bias": table(32, H, DT[dtype]), "softcap": 30.0}}[mod])
    o, lse, _ = attention_scored_fwd(q.cuda(), k.cuda(), v.cuda(), causal=True, residual=True, **to_gpu(mods))
    torch.cuda.synchronize()
    for start in (0, n // 2 - 7, n - 40):
        rows = slice(start, start + 40)
        ref = reference(q[:, :, rows], k, v, dtype=DT[dtype], causal=True, q_pos=[start] * B, **mods)
        assert_within("o", o[:, :, rows], ref["o"])
        assert_within("lse", lse[:, :, rows], ref["lse"])
