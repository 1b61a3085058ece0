"""The large tiles of the attention kernels, which calls of many sequences and heads take, against 64 bits:
second tiles of a sequence, waves without rows, borders of causal and window masks, ragged lengths,
unaligned rows, query heads shared by workgroups.  A few sequences and key heads of every call are
compared; which kernels ran is read from a trace."""
import math

import pytest
import torch

import attention_ref as ref
from paper_2609_04910_amd import attention as at

pytestmark = pytest.mark.gpu

# name: B, M, N, Hq, Hkv, causal, window, layout, and whether the query heads of a key head are shared
CASES = {
    "causal": (16, 200, 200, 32, 32, True, 0, "dense", False),
    "window": (16, 300, 300, 32, 32, True, 70, "dense", False),
    "no mask": (16, 140, 290, 32, 32, False, 0, "dense", False),
    "more rows than keys": (16, 300, 140, 32, 32, True, 0, "dense", False),
    "padded": (16, 257, 257, 32, 32, True, 0, "padded", False),
    "shared heads": (16, 150, 300, 32, 8, False, 0, "padded", True),
    "shared heads, causal": (16, 300, 300, 64, 16, True, 0, "dense", True),
    "packed": (20, 300, 300, 32, 32, True, 0, "packed", False),
    "packed, window": (20, 300, 300, 32, 16, True, 33, "packed", False),
}
WIDTHS = [(64, 64, True), (64, 64, False), (40, 56, True), (128, 128, True), (128, 128, False), (96, 128, True), (128, 100, True)]


def odd(t):
    """The same numbers with rows at odd 16-bit addresses."""
    buf = torch.empty(t.numel() // t.shape[-1] * (t.shape[-1] + 1) + 1, dtype=t.dtype, device="cuda")
    w = buf[1:].view(t.shape[:-1] + (t.shape[-1] + 1,))[..., :t.shape[-1]]
    w.copy_(t)
    return w


def inputs(case, D, C, aligned, dtype):
    """(tensors, keyword arguments, rows, keys): all sequences' lengths."""
    B, M, N, Hq, Hkv, causal, window, layout, _ = CASES[case]
    gen = torch.Generator(device="cuda").manual_seed(M + N + D)
    gap = torch.Generator().manual_seed(M)
    rows, keys = [M] * B, [N] * B
    if layout != "dense":
        rows = torch.randint(0, M + 1, (B,), generator=gap).tolist()
        keys = list(rows) if M == N else torch.randint(0, N + 1, (B,), generator=gap).tolist()
        rows[0], keys[0], rows[-1], keys[-1], rows[3], keys[5] = M, N, 129, min(N, 131), 0, 0
    lead = [(sum(rows),), (sum(keys),)] if layout == "packed" else [(B, M), (B, N)]
    t = [torch.randn(lead[s] + (h, w), generator=gen, device="cuda").to(dtype)
         for s, h, w in ((0, Hq, D), (1, Hkv, D), (1, Hkv, C), (0, Hq, C))]
    t[3] *= 0.1
    if not aligned:
        t = [odd(x) for x in t]
    kw = dict(causal=causal, window=window)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    if layout == "padded":
        kw.update(q_lens=i32(rows), k_lens=i32(keys))
    if layout == "packed":
        kw.update(q_offsets=i32([sum(rows[:b]) for b in range(B + 1)]), k_offsets=i32([sum(keys[:b]) for b in range(B + 1)]))
    return t, kw, rows, keys


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,C,aligned", WIDTHS)
@pytest.mark.parametrize("case", CASES)
def test_against_64_bits(case, D, C, aligned, dtype):
    (q, k, v, g), kw, rows, keys = inputs(case, D, C, aligned, dtype)
    out, lse = at.attention_fwd(q, k, v, **kw)
    dq, dk, dv = at.attention_bwd(q, k, v, out, lse, g, **kw)
    packed, Hq, Hkv = "q_offsets" in kw, q.shape[-2], k.shape[-2]
    G, B = Hq // Hkv, len(rows)
    for b, h in ((0, 0), (B - 1, Hkv - 1), (7, Hkv // 2), (3, 1), (5, 2)):
        heads = slice(h * G, (h + 1) * G)
        if packed:
            i, j = slice(sum(rows[:b]), sum(rows[:b + 1])), slice(sum(keys[:b]), sum(keys[:b + 1]))
            on_q, on_k, stat = (i, heads), (j, slice(h, h + 1)), lse[heads, i]
        else:
            on_q, on_k = (b, slice(0, rows[b]), heads), (b, slice(0, keys[b]), slice(h, h + 1))
            stat = lse[b, heads, :rows[b]]
        r = ref.one(q[on_q], k[on_k], v[on_k], D ** -0.5, kw["causal"], kw["window"], dout=g[on_q])
        for name, t in (("out", out[on_q]), ("lse", stat), ("dq", dq[on_q]), ("dk", dk[on_k]), ("dv", dv[on_k])):
            ref.check("%s of sequence %d, key head %d" % (name, b, h), t, *r[name])
    if "q_lens" in kw:
        for b in range(B):
            assert not out[b, rows[b]:].any() and (lse[b, :, rows[b]:] == -math.inf).all()
            assert not dq[b, rows[b]:].any() and not dk[b, keys[b]:].any() and not dv[b, keys[b]:].any()


def kernels_of(call):
    from torch.profiler import ProfilerActivity, profile
    with profile(activities=[ProfilerActivity.CUDA]) as trace:
        call()
        torch.cuda.synchronize()
    return [e.key for e in trace.key_averages() if "k_attn" in e.key]


@pytest.mark.filterwarnings("ignore:.*Profiler clears events")
@pytest.mark.parametrize("D,C,aligned", WIDTHS)
@pytest.mark.parametrize("case", CASES)
def test_these_calls_take_the_large_tiles(case, D, C, aligned):
    """So that a changed threshold does not leave them untested."""
    (q, k, v, g), kw, _, _ = inputs(case, D, C, aligned, torch.float16)
    out, lse = at.attention_fwd(q, k, v, **kw)
    names = kernels_of(lambda: (at.attention_fwd(q, k, v, **kw), at.attention_bwd(q, k, v, out, lse, g, **kw)))
    if not names:
        pytest.skip("no kernel trace on this machine")
    wide = "true" if aligned and C % 8 == 0 else "false"
    width, rows = (64, 2) if max(D, C) <= 64 else (128, 3)
    if width == 128 and CASES[case][1] <= 192:
        rows = 2                               # 512 tiles of 192 rows: below the 1024 from which they are taken
    for kernel in ("k_attn_fwd<gs::F16, %d, %d, 4, false, %s>" % (width, rows, wide),
                   "k_attn_bwd<gs::F16, %d, 2, 4, false, %s>" % (width, wide),
                   "k_attn_bwd<gs::F16, %d, 2, 4, true, %s>" % (width, wide)):
        assert any(kernel in n for n in names), (kernel, names)
    assert any("k_attn_sum" in n for n in names) == CASES[case][8]
