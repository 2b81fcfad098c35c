"""Host-side checks of the calls on a paged cache and of the scores of given tokens: every entry point
that include/ts_cache.h declares is there, and bad arguments return the documented codes before the
device is touched (no compute call is made here); the float64 reference of the GPU tests."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

import cache_ref as R
from paper_2002_00876_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000          # 256-aligned, never dereferenced: every call below fails validation
NULL_ARG, BAD_DIM, WORKSPACE, BAD_ARG = -1, -2, -3, -7


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def test_library_exports_every_declared_symbol(L):
    for header, some in (("ts_cache.h", {"ts_cache_append", "ts_cache_attend"}),
                         ("ts_token.h", {"ts_token_score", "ts_token_score_grad"})):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names = set(re.findall(r"\b(ts_[a-z_]+)\s*\(", text))
        assert some <= names
        for name in names:
            assert ctypes.cast(getattr(L, name), ctypes.c_void_p).value


def layout(P=9, S=16, Hk=2, D=64, sp=2048, st=128, sh=64):
    return binding.CacheLayout(P, S, Hk, D, sp, st, sh)


def strides(n, value=64):
    return (ctypes.c_int64 * n)(*[value] * n)


def append(L, k=FAKE, v=FAKE, q=FAKE, s=None, dt=1, f=FAKE, R=64, kc=FAKE, vc=FAKE, lay=None, pages=FAKE,
           M=4, starts=FAKE, B=2, N=3, Hq=4, out=FAKE, **c):
    return L.ts_cache_append(k, v, q, strides(9) if s is None else s, dt, f, R, 0, None, kc, vc,
                             layout(**c) if lay is None else lay, pages, M, starts, None, B, N, Hq, out,
                             None)


def attend(L, q=FAKE, s=None, dt=1, kc=FAKE, vc=FAKE, lay=None, pages=FAKE, M=4, starts=FAKE, B=2, N=3,
           Hq=4, scale=0.1, out=FAKE, ws=FAKE, nb=1 << 40, **c):
    return L.ts_cache_attend(q, strides(3) if s is None else s, dt, kc, vc,
                             layout(**c) if lay is None else lay, pages, M, starts, None, None, B, N, Hq,
                             scale, out, None, ws, nb, None)


def score(L, p=FAKE, dt=0, sb=0, sn=0, z=FAKE, B=2, N=3, V=10, K=4, T=1.0, lp=FAKE, e=FAKE, alt=FAKE,
          alp=FAKE, ws=None, nb=0):
    return L.ts_token_score(p, dt, sb, sn, z, None, B, N, V, K, T, lp, e, alt, alp, ws, nb, None)


def score_grad(L, p=FAKE, dt=0, sb=0, sn=0, z=FAKE, B=2, N=3, V=10, T=1.0, g=FAKE, ws=None, nb=0):
    return L.ts_token_score_grad(p, dt, sb, sn, z, None, None, None, B, N, V, T, None, None, g, ws, nb,
                                 None)


def test_bad_dimensions_are_rejected(L):
    assert L.ts_cache_max_head() == 256 and L.ts_cache_max_nodes() == 256
    for f in (append, attend):
        for bad in (dict(B=0), dict(N=0), dict(B=-1), dict(Hq=0), dict(Hq=3), dict(Hq=1026), dict(Hk=0),
                    dict(Hk=-2), dict(D=0), dict(D=12), dict(D=264), dict(P=0), dict(P=1 << 31),
                    dict(S=0), dict(M=0), dict(M=1 << 27), dict(M=1 << 62), dict(S=1 << 62),
                    dict(B=1 << 28, N=2), dict(B=1 << 62, N=4)):
            assert f(L, **bad) == BAD_DIM, (f.__name__, bad)
    for bad in (dict(R=-16), dict(R=8), dict(R=72), dict(R=80), dict(R=(1 << 63) - 16)):
        assert append(L, **bad) == BAD_DIM, bad
    assert attend(L, N=257) == BAD_DIM
    assert attend(L, B=1 << 23, Hk=2, Hq=2, N=1) == BAD_DIM
    assert attend(L, B=256, Hk=600, Hq=600, N=1, S=1 << 15, M=1 << 15) == BAD_DIM   # 2^33 units a stretch
    assert attend(L, B=256, Hk=1, Hq=1, N=1, S=1 << 15, M=1 << 15, nb=0) == WORKSPACE
    assert "ts_cache_attend" in L.ts_last_error().decode()
    most_v = L.ts_token_max_vocab()
    for f in (score, score_grad):
        for bad in (dict(B=0), dict(N=0), dict(V=0), dict(V=most_v + 1), dict(B=1 << 20, N=1 << 10)):
            assert f(L, **bad) == BAD_DIM, (f.__name__, bad)
    for bad in (dict(K=-1), dict(K=11), dict(V=1000, K=257)):
        assert score(L, **bad) == BAD_DIM, bad


def test_bad_types_strides_and_alignment_are_rejected(L):
    for f in (append, attend):
        for bad in (dict(dt=0), dict(dt=3), dict(dt=-1), dict(kc=FAKE + 8), dict(vc=FAKE + 2), dict(sp=-8),
                    dict(st=4), dict(sh=7), dict(sp=1 << 41), dict(q=FAKE + 4), dict(out=FAKE + 8)):
            assert f(L, **bad) == BAD_ARG, (f.__name__, bad)
        for value in (-8, 4, 1 << 41):
            assert f(L, s=strides(9, value)) == BAD_ARG
    for bad in (dict(k=FAKE + 8), dict(v=FAKE + 8)):
        assert append(L, **bad) == BAD_ARG
    for scale in (0.0, -1.0, math.nan, math.inf, 1e7, 1e-7):
        assert attend(L, scale=scale) == BAD_ARG
    for f in (score, score_grad):
        for bad in (dict(dt=3), dict(sb=-1), dict(sn=1 << 41), dict(T=0.0), dict(T=math.nan)):
            assert f(L, **bad) == BAD_ARG, (f.__name__, bad)


def test_null_pointers_are_rejected(L):
    null = ctypes.POINTER(binding.CacheLayout)()
    for bad in (dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(kc=None), dict(vc=None),
                dict(pages=None), dict(starts=None), dict(lay=null),
                dict(s=ctypes.POINTER(ctypes.c_int64)())):
        assert append(L, **bad) == NULL_ARG, bad
    for bad in (dict(q=None), dict(out=None), dict(kc=None), dict(vc=None), dict(pages=None),
                dict(starts=None), dict(ws=None), dict(lay=null),
                dict(s=ctypes.POINTER(ctypes.c_int64)())):
        assert attend(L, **bad) == NULL_ARG, bad
    for bad in ("p", "z", "lp", "e", "alt", "alp"):
        assert score(L, **{bad: None}) == NULL_ARG, bad
    for bad in ("p", "z", "g"):
        assert score_grad(L, **{bad: None}) == NULL_ARG, bad


def test_workspaces(L):
    ws = binding.tree_workspace_bytes
    for bad in ((0, 3, 4, 2, 64), (2, 257, 4, 2, 64), (2, 3, 3, 2, 64), (2, 3, 4, 2, 65),
                (2, 3, 4, 2, 264), (1 << 62, 4, 4, 2, 64)):
        assert ws(*bad) == 0
    need = ws(2, 3, 4, 2, 64)
    assert need > 0 and need % 256 == 0 and ws(2, 60, 4, 2, 64) > need
    assert attend(L, nb=need - 1) == WORKSPACE
    assert attend(L, ws=FAKE + 8) == WORKSPACE
    ws = binding.token_workspace_bytes
    score_op, grad_op = binding.TOKEN_SCORE, binding.TOKEN_SCORE_GRAD
    assert ws(score_op, 2, 3, 10, 11) == 0 and ws(score_op, 2, 3, 0, 0) == 0
    assert ws(score_op, 2, 3, 100000, 8) == ws(binding.TOKEN_TOP, 2, 3, 100000, 8)
    need = ws(grad_op, 2, 3, 100000)
    assert need > 0 and need == ws(score_op, 2, 3, 100000, 0)
    assert score_grad(L, V=100000, ws=FAKE, nb=need - 1) == WORKSPACE
    assert score(L, V=100000, K=0, ws=FAKE, nb=need - 1) == WORKSPACE
    assert score(L, V=100000, K=3) == NULL_ARG


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16)
    c = torch.zeros((9, 16, 4, 64), dtype=torch.bfloat16)
    i = torch.zeros((2, 3), dtype=torch.int32)
    for call in (lambda: binding.cache_append(x, x, c, c, i, i[:, 0]),
                 lambda: binding.tree_attention(x, c, c, i, i[:, 0]),
                 lambda: binding.score(x[:, :, 0].float(), i), lambda: binding.score_grad(x[:, :, 0], i)):
        with pytest.raises(ValueError):
            call()


# ---- the float64 reference itself ----

def test_reference_attention_of_a_path_is_causal():
    rng = np.random.default_rng(0)
    n, start, D = 3, 4, 8
    k, v = rng.normal(size=(4, 2, 1, D)), rng.normal(size=(4, 2, 1, D))
    q = rng.normal(size=(1, n, 1, D))
    pages = np.array([[2, 0, 3, 1]])
    out, lse, _, _ = R.attend(q, k, v, pages, [start], [n], None, 0.5, "bfloat16")
    row = lambda x, j: x[pages[0, j // 2], j % 2, 0]  # noqa: E731
    for i in range(n):
        s = [0.5 * row(k, j) @ q[0, i, 0] for j in range(start + i + 1)]
        w = np.exp(s)
        assert np.allclose(out[0, i, 0], sum(a * row(v, j) for j, a in enumerate(w)) / w.sum())
        assert np.isclose(lse[0, i, 0], math.log(w.sum()))
    path = R.attend(q, k, v, pages, [start], [n], np.array([[-1, 0, 1]]), 0.5, "bfloat16")
    assert np.array_equal(path[0], out)
    assert R.sees(3, 2, 5, [-1, 0, 0, 1, 2]) == [0, 1, 2, 3, 5]


def test_reference_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(1)
    freqs = np.array([1.0, 0.1, 0.01, 0.001], dtype=np.float32)
    x, y = rng.normal(size=(2, 1, 12))
    for neighbours in (False, True):
        turn = lambda z, at: R.rotate(z[None, None], np.array([[at]]), freqs, neighbours,  # noqa: E731
                                      "float16")[0][0, 0]
        assert np.isclose(np.linalg.norm(turn(x, 77)), np.linalg.norm(x))
        assert np.allclose(turn(x, 77)[:, 8:], x[:, 8:])
        assert np.isclose((turn(x, 9) * turn(y, 4)).sum(), (turn(x, 105) * turn(y, 100)).sum())
