"""Softmax attention without a GPU: the library exports what its header declares and rejects bad
arguments before it enqueues anything (fake device addresses, never dereferenced), and the binding
refuses bad tensors (CPU tensors: every check below comes before the device check)."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2609_04910_amd import attention as at
from paper_2609_04910_amd import gauss_sum as gs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "gs_attention.h")).read()
NAMES = set(re.findall(r"\b(gs_attention_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)))


def test_exports_every_declared_symbol():
    lib = at.load()
    assert NAMES == set(at.EXPORTED)
    out = subprocess.run(["nm", "-D", "--defined-only", at.LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert NAMES <= set(re.findall(r"\bT (\w+)", out))
    assert all(hasattr(lib, n) for n in NAMES)


def test_structures_match_the_header(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#define __HIP_PLATFORM_AMD__\n#include "gs_attention.h"\n#include <stdio.h>\nint main(void) {'
                   'printf("%zu %zu %zu %zu %zu %d %d", sizeof(gs_attention_problem), sizeof(gs_attention_array), '
                   'sizeof(gs_attention_cache), offsetof(gs_attention_problem, scale), offsetof(gs_attention_cache, lens), '
                   'GS_ATTENTION_REST_OUT, GS_ATTENTION_REST_LSE); return 0; }')
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(at.Problem), ctypes.sizeof(at.Array), ctypes.sizeof(at.Cache), at.Problem.scale.offset,
                   at.Cache.lens.offset, at.REST_OUT, at.REST_LSE]


FAKE = 1 << 32
STEP = 1 << 24


def problem(B=2, M=8, N=10, Hq=4, Hkv=2, D=64, C=32, window=0, dtype=gs.GS_F16, packed=0, causal=0, rest=0, scale=0.1):
    return at.Problem(B, M, N, Hq, Hkv, D, C, window, dtype, packed, causal, rest, scale)


def array(i, rows, heads, width, data=None, batch=None, row=None, head=None):
    return at.Array(FAKE + i * STEP if data is None else data, rows * heads * width if batch is None else batch,
                    heads * width if row is None else row, width if head is None else head)


def fwd(p, /, **kw):
    q, k, v = array(0, p.M, p.Hq, p.D), array(1, p.N, p.Hkv, p.D), array(2, p.N, p.Hkv, p.C)
    o = array(3, p.M, p.Hq, p.C)
    a = dict(p=p, q=q, k=k, v=v, qi=None, ki=None, out=o, low=None, lse=FAKE + 4 * STEP)
    a.update(kw)
    r = at._ref
    return at.load().gs_attention_fwd(r(a["p"]), r(a["q"]), r(a["k"]), r(a["v"]), a["qi"], a["ki"], r(a["out"]),
                                      r(a["low"]), a["lse"], None, 0, None)


BIG = 1 << 31


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), 2), (dict(B=(1 << 20) + 1), 2), (dict(M=-1), 2), (dict(N=BIG), 2), (dict(M=BIG), 2), (dict(Hq=3), 2),
    (dict(Hq=0), 2), (dict(Hkv=0), 2), (dict(Hq=1 << 15), 2), (dict(D=0), 2), (dict(D=257), 2), (dict(C=0), 2),
    (dict(C=257), 2), (dict(window=-1), 2), (dict(window=3), 2), (dict(window=BIG, causal=1), 2),
    (dict(dtype=gs.GS_F32), 4), (dict(dtype=9), 4), (dict(scale=float("nan")), 3), (dict(scale=float("inf")), 3),
    (dict(scale=3e38), 3), (dict(scale=-3e38), 3), (dict(B=0), 0), (dict(M=0), 0),
    (dict(packed=1), 1),                                      # no offsets
    (dict(B=1 << 20, M=1 << 30, Hq=1, Hkv=1), 2),             # more tiles than a grid holds
])
def test_problems_that_are_refused(kw, status):
    assert fwd(problem(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(p=None), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(out=None), 1),
    (dict(q=array(0, 8, 4, 64, data=0)), 1), (dict(q=array(0, 8, 4, 64, data=FAKE + 1)), 5),
    (dict(lse=FAKE + 4 * STEP + 2), 5), (dict(qi=FAKE + 5 * STEP + 1), 5),
    (dict(k=array(1, 10, 2, 64, row=-128)), 2), (dict(k=array(1, 10, 2, 64, batch=1 << 50)), 2),
    (dict(out=array(3, 8, 4, 32, head=0)), 9), (dict(out=array(3, 8, 4, 32, row=64)), 9),   # elements that are not distinct
    (dict(out=array(3, 8, 4, 32, batch=0)), 9), (dict(out=array(0, 8, 4, 32)), 9),
    (dict(out=array(3, 8, 4, 32, data=FAKE + STEP - 64)), 9),
    (dict(lse=FAKE + 3 * STEP + 128), 9), (dict(low=array(3, 8, 4, 32)), 9), (dict(qi=FAKE + 3 * STEP), 9),
])
def test_arrays_that_are_refused(kw, status):
    assert fwd(problem(), **kw) == status


def bwd(p, ws=FAKE + 20 * STEP, wsb=None, **kw):
    a = dict(q=array(0, p.M, p.Hq, p.D), k=array(1, p.N, p.Hkv, p.D), v=array(2, p.N, p.Hkv, p.C),
             out=array(3, p.M, p.Hq, p.C), low=None, lse=FAKE + 4 * STEP, dout=array(5, p.M, p.Hq, p.C),
             dq=array(6, p.M, p.Hq, p.D), dk=array(7, p.N, p.Hkv, p.D), dv=array(8, p.N, p.Hkv, p.C))
    a.update(kw)
    r = at._ref
    if wsb is None:
        wsb = at.load().gs_attention_bwd_workspace_size(r(p), 1, 1, 1)
    return at.load().gs_attention_bwd(r(p), r(a["q"]), r(a["k"]), r(a["v"]), None, None, r(a["out"]), r(a["low"]), a["lse"],
                                      r(a["dout"]), r(a["dq"]), r(a["dk"]), r(a["dv"]), ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dq=None, dk=None, dv=None), 1), (dict(lse=None), 1), (dict(dout=None), 1), (dict(out=None), 1),
    (dict(ws=None), 6), (dict(wsb=64), 6), (dict(ws=FAKE + 20 * STEP + 64), 5), (dict(ws=FAKE + 6 * STEP), 9),
    (dict(dq=array(0, 8, 4, 64)), 9), (dict(dk=array(8, 10, 2, 64)), 9), (dict(dv=array(8, 10, 2, 32, head=16)), 9),
    (dict(dq=array(6, 8, 4, 64, data=FAKE + 6 * STEP + 1)), 5), (dict(low=array(7, 8, 4, 32)), 9),
])
def test_backward_refusals(kw, status):
    assert bwd(problem(), **kw) == status


def test_workspace_sizes():
    f = at.load().gs_attention_bwd_workspace_size
    assert f(at._ref(problem()), 1, 1, 1) >= 2 * 4 * 8 * 4
    assert f(at._ref(problem()), 0, 0, 0) == 0 and f(at._ref(problem(D=0)), 1, 1, 1) == 0 and f(None, 1, 1, 1) == 0
    assert at.load().gs_attention_paged_workspace_size(None, None) == 0
    assert at.load().gs_attention_fwd_workspace_size(None) == 0
    long = problem(B=1, M=1, N=100000)
    need = at.load().gs_attention_fwd_workspace_size(at._ref(long))
    assert need >= 2 * 4 * (32 + 2) * 4 and need < 1 << 24
    assert fwd(long) == 6                                     # the parts of its rows need a workspace


def cache(pages=6, size=16, width=3, k=None, v=None, table=FAKE + 12 * STEP, lens=FAKE + 13 * STEP, C=32):
    return at.Cache(k or array(10, size, 2, 64), v or array(11, size, 2, C), pages, size, width, table, lens)


def paged(p=None, c=None, qi=None, ws=FAKE + 20 * STEP, wsb=1 << 40, out=None, lse=FAKE + 4 * STEP):
    p = p or problem(causal=1)
    r = at._ref
    return at.load().gs_attention_paged(r(p), r(array(0, p.M, p.Hq, p.D)), r(c) if c is not False else None, qi,
                                        r(out or array(3, p.M, p.Hq, p.C)), lse, ws, wsb, None)


def append(p=None, c=None, qi=None, k=None):
    p = p or problem()
    r = at._ref
    return at.load().gs_attention_append(r(p), r(k or array(0, p.M, p.Hkv, p.D)), r(array(2, p.M, p.Hkv, p.C)), r(c), qi, None)


@pytest.mark.parametrize("make,status", [
    (dict(pages=-1), 2), (dict(size=0), 2), (dict(width=-1), 2), (dict(size=1 << 20, width=1 << 20), 2), (dict(table=None), 1),
    (dict(lens=None), 1), (dict(table=FAKE + 2), 5), (dict(k=array(10, 16, 2, 64, data=0)), 1),
    (dict(v=array(11, 16, 2, 32, data=FAKE + 11 * STEP + 1)), 5),
])
def test_caches_that_are_refused(make, status):
    assert paged(c=cache(**make)) == status
    assert append(c=cache(**make)) == status


def test_paged_refusals():
    assert paged(c=False) == 1
    assert paged(problem(), cache()) == 4                     # not causal
    assert paged(problem(causal=1, packed=1), cache()) == 1   # no offsets
    assert paged(problem(causal=1), cache(), qi=FAKE + 14 * STEP) == 4
    assert paged(c=cache(), out=array(10, 8, 4, 32)) == 9
    assert paged(c=cache(), out=array(12, 8, 4, 32)) == 9     # over the table
    assert append(c=cache(), k=array(10, 8, 2, 64)) == 9
    assert append(c=cache(k=array(10, 16, 2, 64, head=0))) == 9
    assert append(problem(M=0), cache()) == 0 and append(problem(B=0), cache()) == 0
    assert append(c=cache(width=0, table=None)) == 0 and append(c=cache(pages=0)) == 0
    assert append(c=cache(v=array(10, 16, 2, 32))) == 9       # keys and values in one place


H, BF = torch.float16, torch.bfloat16


def z(*shape, dtype=H):
    return torch.zeros(shape, dtype=dtype)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


@pytest.mark.parametrize("args,kw,error,text", [
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), {}, ValueError, "GPU tensor"),          # fine but for the device
    ((z(5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), {}, ValueError, "4 dimensions"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 9), z(1, 6, 2, 4)), {}, ValueError, "k must be"),
    ((z(1, 5, 2, 8), z(1, 7, 2, 8), z(1, 6, 2, 4)), {}, ValueError, "k must be"),
    ((z(1, 5, 3, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), {}, ValueError, "multiple"),
    ((z(2, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), {}, ValueError, "sequences"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8, dtype=BF), z(1, 6, 2, 4)), {}, TypeError, "share a dtype"),
    ((z(1, 5, 2, 8, dtype=torch.float32), z(1, 6, 2, 8), z(1, 6, 2, 4)), {}, TypeError, "float16 or bfloat16"),
    ((z(1, 8, 2, 5).transpose(1, 3), z(1, 6, 2, 8), z(1, 6, 2, 4)), {}, ValueError, "contiguous"),
    ((z(1, 5, 2, 0), z(1, 6, 2, 0), z(1, 6, 2, 4)), {}, ValueError, "D and C"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 257)), {}, ValueError, "D and C"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), dict(window=3), ValueError, "window"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), dict(window=-3, causal=True), ValueError, "window"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), dict(k_lens=torch.tensor([3])), TypeError, "int32"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), dict(k_lens=i32(3, 4)), ValueError, "k_lens"),
    ((z(1, 5, 2, 8), z(1, 6, 2, 8), z(1, 6, 2, 4)), dict(k_offsets=i32(0, 6)), ValueError, "needs q_offsets"),
    ((z(5, 2, 8), z(6, 2, 8), z(6, 2, 4)), dict(q_offsets=i32(0, 5), k_lens=i32(3)), ValueError, "packed"),
    ((z(5, 2, 8), z(6, 2, 8), z(6, 2, 4)), dict(q_offsets=i32(0, 5), k_offsets=i32(0, 3, 6)), ValueError, "k_offsets"),
    ((z(5, 2, 8), z(6, 2, 8), z(6, 2, 4)), dict(q_offsets=i32()), ValueError, "q_offsets"),
])
def test_binding_refuses(args, kw, error, text):
    with pytest.raises(error, match=text):
        at.attention_fwd(*args, **kw)
    with pytest.raises(error, match=text):
        at.attention(*args, **kw)
    with pytest.raises(error, match=text):
        at.attention_bwd(*args, z(1, 5, 2, 4), torch.zeros(1, 2, 5), z(1, 5, 2, 4), **kw)


PAGES = (z(4, 16, 2, 8), z(4, 16, 2, 4), torch.zeros(2, 3, dtype=torch.int32), i32(5, 6))


@pytest.mark.parametrize("change,error,text", [
    ({}, ValueError, "GPU tensor"),
    ({0: z(4, 16, 2, 9)}, ValueError, "k_pages"), ({1: z(4, 15, 2, 4)}, ValueError, "k_pages"),
    ({0: z(4, 0, 2, 8), 1: z(4, 0, 2, 4)}, ValueError, "at least one row"), ({1: z(16, 2, 4)}, ValueError, "4 dimensions"),
    ({0: z(4, 16, 2, 8, dtype=BF)}, TypeError, "share a dtype"), ({2: torch.zeros(2, 3)}, TypeError, "page_table"),
    ({2: torch.zeros(3, 2, dtype=torch.int32).t()}, ValueError, "page_table"), ({3: i32(5)}, ValueError, "seq_lens"),
    ({3: torch.tensor([5, 6])}, TypeError, "seq_lens"), ({4: i32(0, 4)}, ValueError, "q_offsets"),
    ({2: torch.zeros(3, 3, dtype=torch.int32), 3: i32(1, 2, 3)}, ValueError, "give q_offsets"),
])
def test_binding_refuses_caches(change, error, text):
    args = list(PAGES) + [None]
    for i, t in change.items():
        args[i] = t
    with pytest.raises(error, match=text):
        at.attention_paged(z(4, 4, 8), *args)
    with pytest.raises(error, match=text):
        at.attention_append(z(4, 2, 8), z(4, 2, 4), *args)


def test_binding_refuses_other_heads_in_the_pages():
    with pytest.raises(ValueError, match="heads"):
        at.attention_append(z(4, 4, 8), z(4, 4, 4), *PAGES)
    with pytest.raises(ValueError, match="share rows"):
        at.attention_append(z(4, 2, 8), z(3, 2, 4), *PAGES)
    with pytest.raises(ValueError, match="multiple"):
        at.attention_paged(z(4, 3, 8), *PAGES)
    with pytest.raises(ValueError, match="negative"):
        at.attention_paged(z(4, 4, 8), *PAGES, window=-1)
