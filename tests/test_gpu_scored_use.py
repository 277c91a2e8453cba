"""Scored and shared-prefix attention as programs use them: training and serving steps
that agree with each other, graphs, streams, the native calls against the general path,
caches beyond 2^31 elements."""
import math

import pytest
import torch

from paper_2112_05682_amd import (_lib, attention, attention_scored, attention_scored_bwd, attention_scored_fwd,
                                  attention_shared_prefix)
from scored_ref import assert_within, reference

pytestmark = pytest.mark.gpu


def randn(*shape, dtype=torch.bfloat16, seed=0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def int32(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def rows_of(want, rows):
    """The same (value, bound) for some of the queries."""
    return tuple(t[:, :, rows] for t in want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_without_modifications_it_is_plain_attention(dtype):
    q, k, v, do = (randn(2, 3, 200, 64, dtype=dtype, seed=i) for i in range(4))
    for causal in (False, True):
        want = reference(*(t.cpu() for t in (q, k, v, do)), dtype=dtype, causal=causal)
        for f in (attention, attention_scored):  # both within the bounds of the same rounding
            x = [t.detach().requires_grad_() for t in (q, k, v)]
            o = f(*x, causal=causal)
            for name, t in zip(("o", "dq", "dk", "dv"), (o, *torch.autograd.grad(o, x, do))):
                assert_within(name, t, want[name])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prefill_decode_and_shared_prefix_agree(dtype):
    """One pass over whole sequences that begin alike; the same rows as decode steps against
    each sequence's cache; and against the shared prefix and the own keys."""
    B, H, Hkv, n_p, n_o, d = 3, 6, 2, 150, 40, 64
    kp, vp = (randn(Hkv, n_p, d, dtype=dtype, seed=s) for s in (1, 2))
    ko, vo = (randn(B, Hkv, n_o, d, dtype=dtype, seed=s) for s in (3, 4))
    q = randn(B, H, n_p + n_o, d, dtype=dtype, seed=5)
    k, v = (torch.cat([p[None].expand(B, -1, -1, -1), o], 2) for p, o in ((kp, ko), (vp, vo)))
    bias = randn(32, H, dtype=dtype, seed=6)
    host = [t.cpu() for t in (q, k, v)]
    for mods in ({}, {"softcap": 20.0}, {"bias": bias}, {"prefix_len": [7, 0, 180]}):
        m_ = {key: int32(*x) if isinstance(x, list) else x for key, x in mods.items()}
        want = reference(*host, dtype=dtype, causal=True, **{key: x.cpu() if isinstance(x, torch.Tensor) else x for key, x in mods.items()})
        full, lse = attention_scored_fwd(q, k, v, causal=True, **m_)
        assert_within("o", full, want["o"])
        assert_within("lse", lse, want["lse"])
        for n, m in ((n_p + 1, 1), (n_p + 25, 4), (n_p + n_o, 7)):  # m tokens that end at n
            rows = slice(n - m, n)
            o, l = attention_scored_fwd(q[:, :, rows], k, v, causal=True, kv_len=int32(*[n] * B), q_pos=int32(*[n - m] * B), **m_)
            if "prefix_len" not in mods or n == n_p + n_o:  # (a prefix of 180 reaches beyond a shorter cache)
                assert_within("o", o, rows_of(want["o"], rows))
                assert_within("lse", l, rows_of(want["lse"], rows))
            if not mods:
                s, l = attention_shared_prefix(q[:, :, rows], kp, vp, ko, vo, causal=True, kv_len=int32(*[n - n_p] * B),
                                               q_pos=int32(*[n - m - n_p] * B), need_lse=True)
                assert_within("o", s, rows_of(want["o"], rows))
                assert_within("lse", l, rows_of(want["lse"], rows))


def test_a_language_model_step_trains_its_bias():
    """A layer with packed documents, capped scores and a learned bias: gradients of every
    parameter against the same layer with attention in float64."""
    torch.manual_seed(0)
    B, n, H, Hkv, d = 2, 120, 4, 2, 64
    E = H * d
    docs = torch.arange(n, dtype=torch.int32).div(50, rounding_mode="floor").int().repeat(B, 1)
    docs[:, -6:] = -1
    x = torch.randn(B, n, E)
    w = [torch.randn(o, E) * E ** -0.5 for o in (E, Hkv * d, Hkv * d, E)]
    table = torch.randn(16, H)
    mods = {"causal": True, "softcap": 10.0, "max_distance": 40}

    def layer(x, w, table, attend):
        q, k, v = (torch.nn.functional.linear(x, a).view(B, n, -1, d).transpose(1, 2) for a in w[:3])
        return torch.nn.functional.linear(attend(q, k, v, table).transpose(1, 2).reshape(B, n, E), w[3])

    def plain(q, k, v, table):
        from scored_ref import bucket_index, visible
        k, v = (t.repeat_interleave(H // Hkv, 1) for t in (k, v))
        s = 10.0 * torch.tanh(q @ k.transpose(2, 3) / math.sqrt(d) / 10.0)
        s = s + table[bucket_index(list(range(n)), n, 16, 40, False)].permute(2, 0, 1)
        seen = visible(B, n, n, True, None, (docs, docs), None, None)[:, None]
        s = s.masked_fill(~seen, -math.inf)
        p = torch.where(seen.any(-1, keepdim=True), torch.softmax(torch.where(seen.any(-1, keepdim=True), s, 0.0), -1), 0.0)
        return p @ v

    dev = [t.cuda().requires_grad_() for t in (x, *w, table)]
    y = layer(dev[0], dev[1:5], dev[5], lambda q, k, v, t: attention_scored(q, k, v, bias=t, docs=docs.cuda(), **mods))
    g = torch.randn(B, n, E)
    got = torch.autograd.grad(y, dev, g.cuda())
    ref = [t.double().requires_grad_() for t in (x, *w, table)]
    z = layer(ref[0], ref[1:5], ref[5], plain)
    want = torch.autograd.grad(z, ref, g.double())
    for a, b in zip((y, *got), (z, *want)):
        # float32 products of up to E = 256 terms and sums over B n = 240 rows.
        assert (a.double().cpu() - b).abs().max() <= 600 * 2.0 ** -24 * b.abs().max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_graph_replays(dtype):
    """Forward and backward captured together, a decode step and a shared-prefix step: every
    replay on new inputs gives the eager results, with eager work in between."""
    B, H, Hkv, n, d = 2, 4, 2, 150, 64
    q, k, v, do = (randn(B, h, n, d, dtype=dtype, seed=i) for i, h in enumerate((H, Hkv, Hkv, H)))
    bias = randn(8, H, dtype=dtype, seed=9)
    docs = torch.arange(n, dtype=torch.int32, device="cuda").div(60, rounding_mode="floor").int().repeat(B, 1)
    lens, pos = int32(n, 70), int32(n - 1, 69)

    def work():
        m = {"causal": True, "bias": bias, "max_distance": 30, "docs": docs, "softcap": 10.0}
        o, lse, o_lo = attention_scored_fwd(q, k, v, residual=True, **m)
        grads = attention_scored_bwd(q, k, v, o, lse, do, o_lo=o_lo, **m)
        step, _ = attention_scored_fwd(q[:, :, :1], k, v, causal=True, kv_len=lens, q_pos=pos, bias=bias)
        return (o, lse, *grads, step, attention_shared_prefix(q[:, :, :1], k[0], v[0], k, v, kv_len=lens))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    with torch.cuda.graph(second, pool=graph.pool()):
        other = work()
    for i in range(4):
        for j, t in enumerate((q, k, v, do)):
            t.copy_(randn(*t.shape, dtype=dtype, seed=100 + 10 * i + j))
        lens.copy_(int32(n - 3 * i, 20 + i))
        pos.copy_(lens - 1)
        eager = work()
        torch.cuda.synchronize()
        (graph if i % 2 else second).replay()
        torch.cuda.synchronize()
        for a, b in zip(captured if i % 2 else other, eager):
            assert torch.equal(a, b)


def test_streams():
    """Calls on two streams at once give the results of calls one after the other."""
    xs = [[randn(2, h, 300, 64, seed=10 * s + i) for i, h in enumerate((4, 2, 2, 4))] for s in range(2)]
    m = {"causal": True, "softcap": 5.0}

    def one(q, k, v, do):
        o, lse, o_lo = attention_scored_fwd(q, k, v, residual=True, **m)
        return (o, lse, *attention_scored_bwd(q, k, v, o, lse, do, o_lo=o_lo, **m)[:3],
                attention_shared_prefix(q[:, :, :2], k[0], v[0], k, v))

    want = [one(*x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(one(*x))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(s, t) for s, t in zip(a, b))


class _Off:
    """Native calls that accept nothing."""

    scored_fwd = scored_bwd = scored_apply = prefix_fwd = staticmethod(lambda *a: None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_native_calls_match_the_general_path(dtype, monkeypatch):
    B, H, Hkv, n, d = 2, 4, 2, 70, 64
    q, do = (randn(B, n, H, d, dtype=dtype, seed=s).transpose(1, 2) for s in (0, 3))
    k, v = (randn(B, Hkv, n, d + 8, dtype=dtype, seed=s)[..., :d] for s in (1, 2))
    lens = int32(70, 12)
    docs = torch.zeros(B, n, dtype=torch.int32, device="cuda")
    for m in ({}, {"causal": True, "softcap": 3, "slopes": torch.ones(H, device="cuda") / 8, "q_pos": int32(2, 0)},
              {"bias": randn(8, H, dtype=torch.float32), "bidirectional": True, "kv_len": lens, "scale": 0.2},
              {"causal": True, "docs": docs, "prefix_len": lens}, {"docs": (docs, docs)}):
        def both():
            o, lse, o_lo = attention_scored_fwd(q, k, v, residual=True, **m)
            x = [t.detach().requires_grad_() for t in (q, k, v)]
            y = attention_scored(*x, **m)
            p = attention_shared_prefix(q, k[0], v[0], k, v, kv_len=lens)
            return (o, lse, *attention_scored_bwd(q, k, v, o, lse, do, o_lo=o_lo, **m), y, *torch.autograd.grad(y, x, do), p)

        assert _lib.native().scored_fwd is not _Off.scored_fwd
        a = both()
        with monkeypatch.context() as mp:
            mp.setattr(_lib, "_native", _Off)
            b = both()
        for s, t in zip(a, b):
            assert (s is None) == (t is None) and (s is None or (torch.equal(s, t) and s.stride() == t.stride()))


def test_inputs_that_are_refused_on_the_gpu():
    q, k, v = randn(2, 4, 10, 64), randn(2, 2, 10, 64), randn(2, 2, 10, 64)
    bad = [dict(softcap=0.0), dict(softcap=-1.0), dict(softcap="x"), dict(slopes=torch.ones(4)), dict(slopes=torch.ones(3, device="cuda")),
           dict(slopes=torch.ones(4, device="cuda").half()), dict(bias=torch.zeros(8, 3, device="cuda")), dict(bias=torch.zeros(8, 4)),
           dict(bias=torch.zeros(7, 4, device="cuda")), dict(bias=torch.zeros(8, 4, device="cuda").half()),
           dict(bias=torch.zeros(4, 8, device="cuda").t()), dict(docs=torch.zeros(2, 10, device="cuda")), dict(docs=int32(1)),
           dict(docs=torch.zeros(2, 9, dtype=torch.int32, device="cuda")), dict(docs=(torch.zeros(2, 10, dtype=torch.int32, device="cuda"),)),
           dict(prefix_len=int32(1, 2)), dict(causal=True, prefix_len=int32(1)), dict(q_pos=3), dict(q_pos=torch.zeros(2, device="cuda")),
           dict(kv_len=int32(1, 2, 3)), dict(out=torch.empty(2, 4, 10, 64, device="cuda"))]
    for m in bad:
        with pytest.raises((ValueError, TypeError)):
            attention_scored_fwd(q, k, v, **m)
    for args in ((q, k[:, :, :9], v), (q, k.float(), v), (q[..., :32], k[..., :32], v[..., :32]), (q.transpose(2, 3), k, v)):
        with pytest.raises((ValueError, TypeError, _lib.MeaError)):
            attention_scored_fwd(*args)
    with pytest.raises(ValueError):
        attention_shared_prefix(q, k, v, k, v)
    with pytest.raises(ValueError):
        attention_shared_prefix(q, k[0, :1], v[0, :1], k, v)
    with pytest.raises((ValueError, TypeError)):
        attention_shared_prefix(q, k[0].float(), v[0].float(), k, v)
    with pytest.raises(ValueError):
        attention_scored_bwd(q, k, v, q, torch.zeros(2, 4, 10, device="cuda"), q, need_dq=False, need_dkdv=False)


def test_no_second_derivative():
    q, k, v = (randn(1, 2, 20, 64, dtype=torch.float32, seed=i).requires_grad_() for i in range(3))
    g, = torch.autograd.grad(attention_scored(q, k, v).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("n_q", [1, 100])
def test_offsets_beyond_32_bits(n_q):
    """Keys and values whose last batch lies past 2^31 elements, and (decode) a row of keys that
    passes 2^32 bytes."""
    H, Hkv, n, d = 4, 2, 260, 64
    far = (1 << 31) + 4096
    buf = torch.empty(2 * far + Hkv * n * d, dtype=torch.bfloat16, device="cuda")
    q, do = randn(2, H, n_q, d, seed=1), randn(2, H, n_q, d, seed=2)
    k0, v0 = randn(2, Hkv, n, d, seed=3), randn(2, Hkv, n, d, seed=4)
    # K and V share the buffer: K's batches at 0 and far, V's at far + 2^20 and 2 far.
    k = buf.as_strided((2, Hkv, n, d), (far, n * d, d, 1))
    v = buf.as_strided((2, Hkv, n, d), (far - (1 << 20), n * d, d, 1), storage_offset=far + (1 << 20))
    k.copy_(k0)
    v.copy_(v0)
    mods = {"causal": True, "q_pos": [n - n_q, 30 - min(30, n_q)], "kv_len": [n, max(30, n_q)]}
    ref = reference(*(t.cpu() for t in (q, k0, v0, do)), dtype=torch.bfloat16, **mods)
    m = {"causal": True, "q_pos": int32(*mods["q_pos"]), "kv_len": int32(*mods["kv_len"])}
    o, lse, o_lo = attention_scored_fwd(q, k, v, residual=True, **m)
    assert_within("o", o, ref["o"])
    for name, x in zip(("dq", "dk", "dv"), attention_scored_bwd(q, k, v, o, lse, do, o_lo=o_lo, **m)):
        assert_within(name, x, ref[name])
    if n_q == 1:
        # One head of 2^25 + 11 keys of 64 features: all zero but the last three, so that every
        # other weight is 1 and its value 0.
        rows = (1 << 25) + 11
        long = buf[:rows * d].view(1, 1, rows, d)
        long.zero_()
        tail = randn(3, d, seed=8, std=2.0)
        long[0, 0, -3:] = tail
        qq = randn(1, 2, 1, d, seed=9, std=2.0)
        s = torch.exp((qq[0, :, 0].double() @ tail.double().t()) / 8)
        want = (s / (s.sum(1, keepdim=True) + rows - 3)) @ tail.double()
        got, _ = attention_scored_fwd(qq, long, long, causal=True, q_pos=int32(rows - 1))
        # The weights' and the output's rounding, and the float32 sum of 2^25 ones in parts.
        size = (s / (s.sum(1, keepdim=True) + rows - 3)) @ tail.double().abs()
        assert ((got[0, :, 0].double() - want).abs() <= 2.0 ** -7 * size + 1e-12).all()
        pre = attention_shared_prefix(qq, long[0], long[0], tail[None, None].contiguous(), tail[None, None].contiguous())
        want = (2 * s / (2 * s.sum(1, keepdim=True) + rows - 3)) @ tail.double()
        assert ((pre[0, :, 0].double() - want).abs() <= 2.0 ** -7 * 2 * size + 1e-12).all()


@pytest.mark.parametrize("dtype,d,n_q", [(torch.bfloat16, 64, 1), (torch.float16, 128, 3), (torch.float32, 64, 2)])
def test_many_ranges(dtype, d, n_q):
    """Few rows on a long cache: ranges up to the most there are, the short sequence's mostly
    empty and the empty one's all; the same against a shared prefix of that length."""
    B, H, n_k = 3, 4, 40000
    q, k, v = randn(B, H, n_q, d, dtype=dtype, seed=1, std=3.0), *(randn(B, 1, n_k, d, dtype=dtype, seed=s) for s in (2, 3))
    lens = [n_k, 700, 0]
    want = reference(*(t.cpu() for t in (q, k, v)), dtype=dtype, kv_len=lens)
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = float("nan"), float("nan")
    o, lse, o_lo = attention_scored_fwd(q, k, v, kv_len=int32(*lens), residual=True)
    assert_within("o", o, want["o"])
    assert_within("lse", lse, want["lse"])
    for b, n in enumerate(lens[:2]):
        one = [t[b:b + 1, :, :n] for t in (k, v)]
        want = reference(q[b:b + 1].cpu(), *(t.cpu() for t in one), dtype=dtype)
        o, lse = attention_shared_prefix(q[b:b + 1], *(t[0, :, 5:] for t in one), *(t[:, :, :5] for t in one), need_lse=True)
        assert_within("o", o, want["o"])
        assert_within("lse", lse, want["lse"])


def test_a_captured_gradient_beside_an_eager_graph():
    """Refused while an eager graph of the same leaves lives (before anything is recorded);
    captured and replayed once it is gone."""
    B, H, n, d = 2, 4, 130, 64
    leaves = [randn(B, H, n, d, seed=i).requires_grad_() for i in range(3)] + [randn(16, H, seed=4).requires_grad_()]
    do, buf = randn(B, H, n, d, seed=5), torch.ones(4, device="cuda")

    def step():
        o = attention_scored(*leaves[:3], causal=True, bias=leaves[3], max_distance=50)
        return (o.detach(), *torch.autograd.grad(o, leaves, do))

    alive = attention_scored(*leaves[:3], causal=True, bias=leaves[3], max_distance=50)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        buf.zero_()
        with pytest.raises(RuntimeError, match="still lives"):
            step()
    del alive, graph
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        with torch.no_grad():
            for j, t in enumerate(leaves):
                t.copy_(randn(*t.shape, seed=100 + 10 * i + j))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)
