"""Attention with modified scores and over a shared prefix, without a GPU: buckets against
their definition, and what the C entry points and the Python functions refuse (before
anything is launched: the addresses are not real)."""
import ctypes

import pytest
import torch

from paper_2112_05682_amd import (_lib, attention_scored, attention_scored_bwd, attention_scored_fwd,
                                  attention_shared_prefix, bucket_edges)
from scored_ref import bucket_of

FAKE = 0x10000
INVALID, UNSUPPORTED, WORKSPACE = _lib.MEA_ERR_INVALID_ARG, _lib.MEA_ERR_UNSUPPORTED, _lib.MEA_ERR_WORKSPACE


@pytest.mark.parametrize("buckets,max_distance", [(2, 2), (2, 100), (3, 9), (8, 5), (8, 40), (16, 128), (32, 128), (31, 300),
                                                  (64, 500), (32, 1000000)])
def test_bucket_edges(buckets, max_distance):
    edges = bucket_edges(buckets, max_distance)
    assert len(edges) == buckets and edges[0] == 0 and list(edges) == sorted(edges)
    for x in [*range(0, 1200), *(e + d for e in edges for d in (-1, 0, 1) if e + d >= 0)]:
        got = sum(e <= x for e in edges) - 1
        assert got == bucket_of(-x, buckets, max_distance, False), x
    # Exact at powers, where the logarithm's rounding would decide: 16 * 2^((b - 16) / 8) is whole for b = 16, 24.
    assert bucket_edges(32, 64)[24] == 32 and bucket_edges(16, 128)[10] == 16


@pytest.mark.parametrize("buckets,max_distance", [(1, 10), (0, 10), (8, 4), (8, 0)])
def test_bucket_edges_refuse(buckets, max_distance):
    with pytest.raises(ValueError):
        bucket_edges(buckets, max_distance)


def problem(**kw):
    base = dict(batch=2, heads=8, n_q=100, n_k=120, d=64, dtype=_lib.MEA_BF16, causal=True, scale=0.125)
    base.update(kw)
    return _lib.problem(**base)


def score(edges=None, **kw):
    s = _lib.MeaScore()
    if edges is not None:
        a = (ctypes.c_int32 * len(edges))(*edges)
        s.edges, s.n_edges, s.table = a, len(edges), FAKE
    for key, x in kw.items():
        setattr(s, key, x)
    return s


def statuses(p, s):
    """Of every scored entry point, which agree."""
    lib, out = _lib.load(), ctypes.c_size_t(0)
    r = {lib.mea_scored_attention_fwd_workspace_size(ctypes.byref(p), ctypes.byref(s), ctypes.byref(out)),
         lib.mea_scored_attention_bwd_workspace_size(ctypes.byref(p), ctypes.byref(s), ctypes.byref(out)),
         _lib.scored_bwd(p, s, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 0, None)}
    return r


@pytest.mark.parametrize("kw,status", [
    (dict(kv_heads=3), INVALID), (dict(kv_heads=-1), INVALID), (dict(kv_heads=16), INVALID),
    (dict(softcap=-1.0), INVALID), (dict(softcap=float("nan")), INVALID), (dict(softcap=float("inf")), INVALID),
    (dict(softcap=1e-44), INVALID),
    (dict(q_doc=FAKE), INVALID), (dict(k_doc=FAKE), INVALID), (dict(q_doc=FAKE + 2, k_doc=FAKE), INVALID),
    (dict(slopes=FAKE + 1), INVALID), (dict(q_pos=FAKE + 2), INVALID), (dict(prefix_len=FAKE + 2), INVALID),
    (dict(edges=[0]), INVALID), (dict(edges=[1, 2]), INVALID), (dict(edges=[0, 5, 4]), INVALID), (dict(edges=[0, 0]), INVALID),
    (dict(edges=[0, 513]), UNSUPPORTED), (dict(edges=list(range(65))), UNSUPPORTED), (dict(edges=[0, 1], two_sided=2), INVALID),
    (dict(edges=[0, 1], table_dtype=5), UNSUPPORTED), (dict(edges=[0, 1], table=FAKE + 2, table_dtype=0), INVALID),
    (dict(table=FAKE), INVALID),
])
def test_scores_that_are_refused(kw, status):
    kw = dict(kw)
    assert statuses(problem(), score(**kw)) == {status}


@pytest.mark.parametrize("kw,status", [
    (dict(d=32), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(n_q=0), INVALID), (dict(n_k=0), INVALID),
    (dict(scale=0.0), INVALID), (dict(out_f32=True), UNSUPPORTED), (dict(d_v=128), UNSUPPORTED), (dict(heads=0), INVALID),
])
def test_problems_that_are_refused(kw, status):
    assert statuses(problem(**kw), score()) == {status}
    x = _lib.MeaSharedPrefix()
    x.n_p, x.k, x.v = 10, FAKE, FAKE
    out = ctypes.c_size_t(0)
    p = problem(**kw)
    assert _lib.load().mea_prefix_attention_fwd_workspace_size(ctypes.byref(p), ctypes.byref(x), ctypes.byref(out)) == status


def test_prefix_mask_needs_causal():
    assert statuses(problem(causal=False), score(prefix_len=FAKE)) == {INVALID}
    assert _lib.scored_fwd_workspace_size(problem(), score(prefix_len=FAKE)) >= 0


def test_pointers_and_workspaces_that_are_refused():
    p, s = problem(n_q=1, heads=8, n_k=100000), score()
    need = _lib.scored_fwd_workspace_size(p, s)
    assert need > 0  # the keys are split
    fwd = lambda q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=None, lo=None, ws=FAKE, n=need: _lib.scored_fwd(  # noqa: E731
        p, s, q, k, v, o, lse, lo, ws, n, None)
    for bad in (None, FAKE + 8):
        for name in "qkvo":
            assert fwd(**{name: bad}) == INVALID
    assert fwd(lse=FAKE + 4) == INVALID and fwd(lo=FAKE + 2) == INVALID
    assert fwd(n=need - 1) == WORKSPACE and fwd(ws=None) == WORKSPACE
    f32 = problem(dtype=_lib.MEA_F32)
    assert _lib.scored_fwd(f32, s, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, 1 << 40, None) == INVALID
    p = problem()
    need = _lib.scored_bwd_workspace_size(p, s)
    names = ("q", "k", "v", "o", "o_lo", "d_o", "lse", "dq", "dk", "dv", "d_table")

    def bwd(n=need, ws=FAKE, **kw):
        given = {**dict.fromkeys(names, FAKE), "o_lo": None, "d_table": None, **kw}
        return _lib.scored_bwd(p, s, *(given[x] for x in names), ws, n, None)

    for name in ("q", "k", "v", "o", "d_o", "lse"):
        assert bwd(**{name: None}) == INVALID and bwd(**{name: FAKE + 4}) == INVALID
    assert bwd(dk=None) == INVALID and bwd(dv=None) == INVALID and bwd(dq=None, dk=None, dv=None) == INVALID
    assert bwd(dq=FAKE + 2) == INVALID and bwd(o_lo=FAKE + 2) == INVALID
    assert bwd(d_table=FAKE) == INVALID  # no table
    assert bwd(n=need - 1) == WORKSPACE and bwd(ws=None) == WORKSPACE


def test_strides_are_over_the_key_heads():
    B, H, kv, nq, nk, d = 2, 8, 2, 100, 120, 64
    ok = {"q": (H * nq * d, nq * d, d), "k": (kv * nk * d, nk * d, d), "v": (kv * nk * d, nk * d, d), "o": (H * nq * d, nq * d, d)}
    for bad in ({"k": (kv * nk * d, 60, d)}, {"v": (kv * nk * d, nk * d, 32)}, {"o": (H * nq * d, 0, d)}, {"q": (-8, nq * d, d)}):
        p = _lib.problem(B, H, nq, nk, d, _lib.MEA_BF16, False, 0.125, strides={**ok, **bad})
        assert _lib.scored_fwd(p, score(kv_heads=kv), FAKE, FAKE, FAKE, FAKE, None, None, FAKE, 1 << 40, None) == INVALID


def test_shared_prefixes_that_are_refused():
    def status(p=None, **kw):
        x = _lib.MeaSharedPrefix()
        x.n_p, x.k, x.v, x.kv_heads = 10, FAKE, FAKE, 2
        for key, val in kw.items():
            setattr(x, key, val)
        p = p or problem(n_q=1, causal=False)
        return _lib.prefix_fwd(p, x, FAKE, FAKE, FAKE, FAKE, None, FAKE, 0, None)

    assert status() == WORKSPACE
    for kw in (dict(n_p=0), dict(n_p=1 << 31), dict(kv_heads=3), dict(k=None), dict(v=FAKE + 8), dict(q_pos=FAKE + 1)):
        assert status(**kw) == INVALID, kw
    lib, out = _lib.load(), ctypes.c_size_t(0)
    p, x = problem(n_q=1), _lib.MeaSharedPrefix()
    assert lib.mea_prefix_attention_fwd_workspace_size(ctypes.byref(p), None, ctypes.byref(out)) == INVALID
    x.n_p = 5
    assert lib.mea_prefix_attention_fwd_workspace_size(ctypes.byref(p), ctypes.byref(x), None) == INVALID
    assert lib.mea_scored_attention_fwd_workspace_size(ctypes.byref(p), None, ctypes.byref(out)) == INVALID
    assert lib.mea_scored_attention_bwd_workspace_size(None, ctypes.byref(score()), ctypes.byref(out)) == INVALID


def test_struct_layouts_match_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    if not shutil.which("gcc") or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("needs gcc and the ROCm headers")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    mirrors = {"mea_score": _lib.MeaScore, "mea_shared_prefix": _lib.MeaSharedPrefix}
    parts = ["sizeof(%s)" % n for n in mirrors] + ["offsetof(%s, %s)" % (n, f) for n, m in mirrors.items() for f, _ in m._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mea.h"\nint main(void) {\n%s\nreturn 0; }\n'
                   % "\n".join('printf("%%zu\\n", %s);' % x for x in parts))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(root, "include"), "-I/opt/rocm/include", str(src),
                    "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(m) for m in mirrors.values()] + [getattr(m, f).offset for m in mirrors.values()
                                                                  for f, _ in m._fields_]
    text = open(os.path.join(root, "include", "mea.h")).read()
    assert "#define MEA_MAX_SIDE_BUCKETS %d " % _lib.MAX_SIDE_BUCKETS in text
    assert "#define MEA_MAX_BIAS_SPAN %d " % _lib.MAX_BIAS_SPAN in text


def test_host_tensors_are_refused():
    q, k = torch.zeros(1, 4, 5, 64), torch.zeros(1, 2, 5, 64)
    for f in (lambda: attention_scored(q, k, k), lambda: attention_scored_fwd(q, k, k),
              lambda: attention_scored_bwd(q, k, k, q, torch.zeros(1, 4, 5), q),
              lambda: attention_shared_prefix(q, k[0], k[0], k, k)):
        with pytest.raises(ValueError, match="GPU"):
            f()
    with pytest.raises(ValueError):
        attention_scored_fwd(q, torch.zeros(1, 3, 5, 64), torch.zeros(1, 3, 5, 64))  # 4 heads over 3
    with pytest.raises(ValueError):
        attention_scored_fwd(q[0], k[0], k[0])
    with pytest.raises(TypeError):
        attention_scored_fwd(q.double(), k.double(), k.double())
    with pytest.raises(ValueError, match="gradient"):
        attention_scored(q, k, k, slopes=torch.ones(4, requires_grad=True))
    with pytest.raises(ValueError, match="no_grad"):
        attention_shared_prefix(q.requires_grad_(), k[0], k[0], k, k)
    with pytest.raises(ValueError):
        attention_scored_fwd(k, k, k, bias=torch.zeros(7, 2), bidirectional=True)  # an odd number on two sides
    with pytest.raises(ValueError):
        attention_scored_fwd(k, k, k, bias=torch.zeros(300, 2), max_distance=10000)


def test_host_code_under_address_and_undefined_sanitizers(tmp_path):
    """scored_api.hip with recorders for its launchers (tests/native/scored_check.cpp): the
    buffers of every launch lie in the workspace that was asked for."""
    import os
    import subprocess
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("needs hipcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    common = ["-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", *san, "-I" + os.path.join(root, "include")]
    api, drv, exe = (str(tmp_path / n) for n in ("api.o", "drv.o", "check"))
    for cmd in (
            [hipcc, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *common, "-c",
             os.path.join(root, "paper_2112_05682_amd", "csrc", "scored_api.hip"), "-o", api],
            [hipcc, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-x", "hip", *common,
             "-c", os.path.join(root, "tests", "native", "scored_check.cpp"), "-o", drv],
            [hipcc, "--offload-arch=gfx950", *san, api, drv, "-o", exe],
            [exe]):
        r = subprocess.run(cmd, capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"), timeout=300)
        assert r.returncode == 0, "%s\n%s\n%s" % (" ".join(cmd), r.stdout[-2000:], r.stderr[-3000:])
    assert "scored_check ok" in r.stdout
    print(r.stdout)


def test_strides_of_a_prefix():
    """A row stride of 0 would mean contiguous rows to the library."""
    from paper_2112_05682_amd.scored import _prefix_strides
    one = torch.zeros(64).expand(3, 1, 64)  # one key for all heads
    s = _prefix_strides("k_prefix", one)
    assert (s.head, s.row) == (0, 64)
    s = _prefix_strides("k_prefix", torch.zeros(5, 3, 64).transpose(0, 1))
    assert (s.head, s.row) == (64, 192)
    for t in (torch.zeros(3, 1, 64).expand(3, 7, 64), torch.zeros(500).as_strided((3, 4, 64), (64, 32, 1))):
        with pytest.raises(ValueError, match="overlap"):
            _prefix_strides("k_prefix", t)
