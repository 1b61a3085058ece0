"""Softmax attention and its gradients on the GPU against 64 bits (attention_ref.one), at the sizes,
layouts and masks where the kernels take other paths: tails of tiles, padded widths, unaligned
rows, rows that see nothing, empty sequences, shared heads."""
import math

import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def at():
    from paper_2609_04910_amd import attention
    attention.load()
    return attention


def normal(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(dtype).cuda()


def make(seed, B, M, N, Hq, Hkv, D, C, dtype, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (normal(gen, (B, M, Hq, D), dtype, std), normal(gen, (B, N, Hkv, D), dtype),
            normal(gen, (B, N, Hkv, C), dtype), normal(gen, (B, M, Hq, C), dtype, 0.1))


def check_dense(at, q, k, v, g, scale=None, rows=None, keys=None, **kw):
    """Every sequence against the reference; rows of no sequence are 0 and -inf."""
    out, lse = at.attention_fwd(q, k, v, scale=scale, **kw)
    grads = at.attention_bwd(q, k, v, out, lse, g, scale=scale, **kw)
    B, M, N = q.shape[0], q.shape[1], k.shape[1]
    sc = q.shape[-1] ** -0.5 if scale is None else scale
    mask = {n: kw[n] for n in ("causal", "window") if n in kw}
    for b in range(B):
        m, n = (M if rows is None else rows[b]), (N if keys is None else keys[b])
        r = ref.one(q[b, :m], k[b, :n], v[b, :n], sc, dout=g[b, :m], **mask)
        got = {"out": out[b, :m], "lse": lse[b, :, :m], "dq": grads[0][b, :m], "dk": grads[1][b, :n],
               "dv": grads[2][b, :n]}
        for name, t in got.items():
            ref.check("%s of sequence %d" % (name, b), t, *r[name])
        for t in (out[b, m:], grads[0][b, m:], grads[1][b, n:], grads[2][b, n:]):
            assert not t.any()
        assert (lse[b, :, m:] == -math.inf).all()


SHAPES = [  # B, M, N, Hq, Hkv, D, C, causal, window
    (1, 1, 1, 1, 1, 64, 64, True, 0),
    (1, 1, 70, 2, 1, 64, 64, False, 0),
    (2, 3, 2, 1, 1, 8, 8, True, 0),          # a row that sees nothing
    (1, 37, 37, 4, 4, 64, 64, True, 0),
    (2, 130, 130, 4, 2, 128, 128, True, 0),
    (1, 129, 65, 2, 2, 128, 128, True, 0),   # 64 rows that see nothing
    (1, 200, 333, 6, 2, 128, 128, True, 50),
    (1, 300, 300, 2, 1, 64, 64, True, 1),
    (1, 150, 90, 2, 1, 64, 64, True, 7),
    (2, 257, 191, 3, 1, 80, 48, False, 0),
    (1, 64, 128, 2, 2, 96, 128, False, 0),
    (1, 100, 77, 2, 2, 33, 17, False, 0),    # rows of no whole 16 bytes
    (1, 65, 65, 1, 1, 1, 1, True, 0),
    (1, 140, 140, 2, 1, 256, 256, True, 0),
    (1, 70, 40, 2, 1, 200, 129, False, 0),
    (1, 90, 600, 8, 1, 128, 64, True, 0),
    (4, 1100, 1100, 1, 1, 128, 128, False, 0),
    (130, 130, 130, 4, 4, 128, 128, False, 0),  # enough workgroups for whole tiles
    # few rows, or few workgroups: the keys are cut into parts
    (1, 1, 5000, 8, 2, 128, 128, False, 0),
    (2, 3, 3000, 4, 4, 64, 64, True, 0),
    (1, 20, 4000, 2, 1, 64, 48, True, 900),
    (1, 5, 2000, 3, 1, 33, 17, False, 0),
    (1, 2, 1500, 2, 1, 256, 256, False, 0),
    (1, 200, 3000, 1, 1, 128, 100, True, 0),
    (1, 3000, 1100, 1, 1, 64, 64, True, 0),  # most rows see nothing
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_dense_against_64_bits(at, shape, dtype):
    B, M, N, Hq, Hkv, D, C, causal, window = shape
    q, k, v, g = make(M + N + D, B, M, N, Hq, Hkv, D, C, dtype)
    check_dense(at, q, k, v, g, causal=causal, window=window)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0, 1e-3])
def test_scales(at, scale):
    q, k, v, g = make(5, 1, 75, 140, 2, 1, 64, 64, torch.bfloat16)
    check_dense(at, q, k, v, g, scale=scale)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_peaked_scores(at, dtype):
    """Scores far apart, the largest late: the running offset grows many times."""
    q, k, v, g = make(6, 1, 70, 400, 2, 1, 64, 64, dtype, std=4.0)
    k = k * (1 + torch.arange(400, device="cuda").view(1, 400, 1, 1) / 80).to(dtype)
    check_dense(at, q, k, v, g)


@pytest.mark.parametrize("dout_std", [1e-6, 300.0])
def test_small_and_large_upstream_gradients(at, dout_std):
    """fp16: dS far below and above its range unless it is scaled."""
    q, k, v, g = make(8, 1, 70, 2000, 2, 1, 64, 64, torch.float16, std=0.2)
    g = (g.float() * (dout_std * 10)).half()
    check_dense(at, q, k, v, g)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_padded_lengths(at, dtype):
    rows, keys = [33, 0, 100, 1, 64], [70, 20, 0, 130, 64]
    q, k, v, g = make(9, 5, 100, 130, 4, 2, 64, 64, dtype)
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (rows, keys)]
    for t, n in ((q, rows), (k, keys), (v, keys), (g, rows)):
        for b in range(5):
            t[b, n[b]:] = float("nan")   # never looked at
    for causal in (False, True):
        check_dense(at, q, k, v, g, rows=rows, keys=keys, q_lens=lens[0], k_lens=lens[1], causal=causal)


def test_only_key_lengths(at):
    q, k, v, g = make(10, 3, 40, 90, 2, 2, 64, 64, torch.bfloat16)
    check_dense(at, q, k, v, g, keys=[90, 1, 37], k_lens=torch.tensor([90, 1, 37], dtype=torch.int32, device="cuda"))


def test_lengths_out_of_range_are_brought_into_it(at):
    q, k, v, g = make(11, 2, 40, 50, 2, 2, 64, 64, torch.bfloat16)
    check_dense(at, q, k, v, g, rows=[40, 0], keys=[0, 50], q_lens=torch.tensor([1000, -3], dtype=torch.int32, device="cuda"),
                k_lens=torch.tensor([-9, 51], dtype=torch.int32, device="cuda"))


PACKED = [
    ([37], [37], True, 0, 0),
    ([1, 200, 0, 64, 65, 0], [1, 200, 0, 64, 65, 0], True, 0, 5),
    ([130, 3, 128], [10, 300, 128], True, 40, 3),
    ([5, 0, 70], [0, 9, 200], False, 0, 1),
    ([0, 0], [0, 0], True, 0, 7),
    ([3] * 150, [5] * 150, True, 0, 2),       # more sequences than a wave has lanes
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", PACKED, ids=lambda c: "%d-%d" % (len(c[0]), sum(c[0])))
def test_packed_against_64_bits(at, case, dtype):
    rows, keys, causal, window, rest = case
    T, S = sum(rows) + rest, sum(keys) + rest
    gen = torch.Generator().manual_seed(T)
    q, g = normal(gen, (T, 4, 64), dtype), normal(gen, (T, 4, 48), dtype)
    k, v = normal(gen, (S, 2, 64), dtype), normal(gen, (S, 2, 48), dtype)
    for t, n in ((q, sum(rows)), (g, sum(rows)), (k, sum(keys)), (v, sum(keys))):
        t[n:] = float("nan")
    offs = [torch.tensor([sum(x[:i]) for i in range(len(x) + 1)], dtype=torch.int32, device="cuda") for x in (rows, keys)]
    kw = dict(q_offsets=offs[0], k_offsets=offs[1], causal=causal, window=window)
    out, lse = at.attention_fwd(q, k, v, **kw)
    dq, dk, dv = at.attention_bwd(q, k, v, out, lse, g, **kw)
    for b in range(len(rows)):
        i, j = slice(sum(rows[:b]), sum(rows[:b + 1])), slice(sum(keys[:b]), sum(keys[:b + 1]))
        r = ref.one(q[i], k[j], v[j], 0.125, causal, window, dout=g[i])
        for name, t in (("out", out[i]), ("lse", lse[:, i]), ("dq", dq[i]), ("dk", dk[j]), ("dv", dv[j])):
            ref.check("%s of sequence %d" % (name, b), t, *r[name])
    assert not out[sum(rows):].any() and not dq[sum(rows):].any()
    assert not dk[sum(keys):].any() and not dv[sum(keys):].any()
    assert (lse[:, sum(rows):] == -math.inf).all()


@pytest.mark.parametrize("M,N", [(6, 3000), (150, 3000)])
def test_lengths_where_keys_are_cut_into_parts(at, M, N):
    rows, keys = [M, 1, 0, 3], [N, 700, 900, 0]
    q, k, v, g = make(22, 4, M, N, 2, 1, 64, 64, torch.bfloat16)
    for t, n in ((q, rows), (k, keys), (v, keys)):
        for b in range(4):
            t[b, n[b]:] = float("nan")
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (rows, keys)]
    assert at.attention_fwd_workspace_size(4, M, N, 2, 1, 64, 64) > 0
    kw = dict(q_lens=lens[0], k_lens=lens[1], causal=True)
    check_dense(at, q, k, v, g, rows=rows, keys=keys, **kw)
    out, lse, low = torch.full_like(q, 7.0), torch.full((4, 2, M), 7.0, device="cuda"), torch.full_like(q, 7.0)
    at.attention_fwd(q, k, v, out=out, lse=lse, low=low, **kw)
    fresh, _ = at.attention_fwd(q, k, v, **kw)
    for b in range(4):
        assert (out[b, rows[b]:] == 7).all() and (low[b, rows[b]:] == 7).all() and (lse[b, :, rows[b]:] == 7).all()
        assert torch.equal(out[b, :rows[b]], fresh[b, :rows[b]])
        exact = ref.one(q[b, :rows[b]], k[b, :keys[b]], v[b, :keys[b]], 0.125, True)["out"][0]
        assert (out[b, :rows[b]].cpu().double() - exact).norm() + 1e-9 >= \
            (out[b, :rows[b]].cpu().double() + low[b, :rows[b]].cpu().double() - exact).norm()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hkv,D,C", [(6, 1, 128, 128), (8, 2, 64, 48), (4, 1, 256, 199), (12, 1, 100, 33)])
def test_shared_key_heads(at, Hq, Hkv, D, C, dtype):
    """The query heads of a key head shared by workgroups, their sums joined: padded, packed, causal."""
    rows, keys = [130, 0, 77], [60, 140, 0]
    q, k, v, g = make(24, 3, 130, 140, Hq, Hkv, D, C, dtype)
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (rows, keys)]
    for causal in (False, True):
        check_dense(at, q, k, v, g, rows=rows, keys=keys, q_lens=lens[0], k_lens=lens[1], causal=causal)
    offs = [torch.tensor([0, 130, 130, 207], dtype=torch.int32, device="cuda"), torch.tensor([0, 60, 200, 200], dtype=torch.int32, device="cuda")]
    pk = [torch.cat([t[b, :n[b]] for b in range(3)] + [t[0, :4] * math.nan]) for t, n in ((q, rows), (k, keys), (v, keys), (g, rows))]
    out, lse = at.attention_fwd(*pk[:3], q_offsets=offs[0], k_offsets=offs[1])
    grads = at.attention_bwd(*pk[:3], out, lse, pk[3], q_offsets=offs[0], k_offsets=offs[1])
    for b, (i, j) in enumerate(zip((slice(0, 130), slice(0, 0), slice(130, 207)), (slice(0, 60), slice(60, 200), slice(200, 200)))):
        r = ref.one(pk[0][i], pk[1][j], pk[2][j], D ** -0.5, dout=pk[3][i])
        for name, t in (("dq", grads[0][i]), ("dk", grads[1][j]), ("dv", grads[2][j])):
            ref.check("%s of sequence %d" % (name, b), t, *r[name])
    assert not grads[1][200:].any() and not grads[2][200:].any()
    only = at.attention_bwd(*pk[:3], out, lse, pk[3], q_offsets=offs[0], k_offsets=offs[1], want=(False, False, True))
    assert torch.equal(only[2], grads[2])


def test_packed_rows_of_few_keys_and_many(at):
    gen = torch.Generator().manual_seed(23)
    rows, keys = [3, 1, 0, 2], [4000, 9, 500, 1700]
    q = normal(gen, (sum(rows) + 2, 4, 64), torch.float16)
    k, v = (normal(gen, (sum(keys), 2, 64), torch.float16) for _ in range(2))
    offs = [torch.tensor([sum(x[:i]) for i in range(5)], dtype=torch.int32, device="cuda") for x in (rows, keys)]
    assert at.attention_fwd_workspace_size(4, 8, sum(keys), 4, 2, 64, 64, packed=True) > 0
    kw = dict(q_offsets=offs[0], k_offsets=offs[1])
    out, lse = at.attention_fwd(q, k, v, **kw)
    mine = torch.full_like(out, 7.0)
    at.attention_fwd(q, k, v, out=mine, **kw)
    for b in range(4):
        i, j = slice(sum(rows[:b]), sum(rows[:b + 1])), slice(sum(keys[:b]), sum(keys[:b + 1]))
        r = ref.one(q[i], k[j], v[j], 0.125)
        ref.check("out", out[i], *r["out"])
        ref.check("lse", lse[:, i], *r["lse"])
        assert torch.equal(mine[i], out[i])
    assert not out[6:].any() and (lse[:, 6:] == -math.inf).all() and (mine[6:] == 7).all()


def test_rows_of_no_sequence_in_the_callers_arrays_are_left(at):
    gen = torch.Generator().manual_seed(1)
    q, k, v = (normal(gen, (50, 2, 64), torch.bfloat16) for _ in range(3))
    offs = torch.tensor([0, 20, 33], dtype=torch.int32, device="cuda")
    out = torch.full((50, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2, 50), 7.0, device="cuda")
    at.attention_fwd(q, k, v, q_offsets=offs, out=out, lse=lse)
    assert (out[33:] == 7).all() and (lse[:, 33:] == 7).all() and not (out[:33] == 7).all()
    q2, k2, v2 = (t[None].contiguous() for t in (q, k, v))
    out2, lse2 = torch.full_like(q2, 7.0), torch.full((1, 2, 50), 7.0, device="cuda")
    lens = torch.tensor([33], dtype=torch.int32, device="cuda")
    at.attention_fwd(q2, k2, v2, q_lens=lens, out=out2, lse=lse2)
    assert (out2[:, 33:] == 7).all() and (lse2[..., 33:] == 7).all() and not (out2[:, :33] == 7).all()


def test_strides(at):
    """Heads before rows, one fused array, unaligned rows, broadcast keys; gradients of a broadcast
    input through autograd are those of its one row set."""
    gen = torch.Generator().manual_seed(2)
    B, M, H, D = 2, 75, 2, 64
    fused = normal(gen, (B, M, 3, H, D), torch.bfloat16)
    q, k, v = fused.unbind(2)
    g = normal(gen, (B, M, H, D), torch.bfloat16)
    check_dense(at, q, k, v, g, causal=True)
    heads_first = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, g)]
    check_dense(at, *heads_first, causal=True)
    odd = []
    for t in (q, k, v, g):
        buf = torch.zeros(B * M * H * (D + 1) + 1, dtype=t.dtype, device="cuda")
        w = buf[1:].view(B, M, H, D + 1)[..., :D]
        w.copy_(t)
        odd.append(w)
    check_dense(at, *odd, causal=True)
    one = [t[:1].expand(B, -1, -1, -1) for t in (k, v)]
    check_dense(at, q, one[0], one[1], g)
    leaf = [t[:1].clone().requires_grad_(True) for t in (k, v)]
    o = at.attention(q, leaf[0].expand(B, -1, -1, -1), leaf[1].expand(B, -1, -1, -1))
    gk, gv = torch.autograd.grad(o, leaf, g)
    low = torch.empty_like(g)
    out, lse = at.attention_fwd(q, one[0], one[1], low=low)
    _, dk, dv = at.attention_bwd(q, one[0], one[1], out, lse, g, low=low)   # the same call as autograd's
    torch.testing.assert_close(gk.float(), dk.float().sum(0, keepdim=True), rtol=2 ** -7, atol=1e-4)
    torch.testing.assert_close(gv.float(), dv.float().sum(0, keepdim=True), rtol=2 ** -7, atol=1e-4)
    buf = torch.full((B * M * H * (D + 1) + 1,), 7.0, dtype=torch.bfloat16, device="cuda")
    odd_out = buf[1:].view(B, M, H, D + 1)[..., :D]
    at.attention_fwd(q, k, v, out=odd_out)
    assert torch.equal(odd_out, at.attention_fwd(q, k, v)[0]) and (buf[1:].view(B, M, H, D + 1)[..., D] == 7).all() and buf[0] == 7
    wide = torch.zeros(B, M, 2 * H, D, dtype=torch.bfloat16, device="cuda")
    at.attention_fwd(q, k, v, out=wide[:, :, ::2])
    assert torch.equal(wide[:, :, ::2], at.attention_fwd(q, k, v)[0]) and not wide[:, :, 1::2].any()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
def test_hidden_infinities_reach_no_row(at, where, bad, dtype):
    """A key or value that is not finite reaches the rows that see it and no other (causal and
    window borders run through its tile)."""
    M = 130
    q, k, v, _ = make(12, 1, M, M, 2, 1, 64, 64, dtype)
    {"k": k, "v": v}[where][0, 70, 0, 5] = bad
    out, lse = at.attention_fwd(q, k, v, causal=True, window=40)
    clean = {"k": k.clone(), "v": v.clone()}
    clean[where][0, 70, 0, 5] = 0
    out0, lse0 = at.attention_fwd(q, clean["k"], clean["v"], causal=True, window=40)
    see = torch.zeros(M, dtype=torch.bool, device="cuda")
    see[70:110] = True
    assert torch.equal(out[0, ~see], out0[0, ~see]) and torch.equal(lse[0][:, ~see], lse0[0][:, ~see])
    if where == "v":
        want = out0.clone()
        want[0, see, :, 5] = bad
        assert torch.equal(out.isnan(), want.isnan())
        assert torch.equal(out[0, see][..., 5].nan_to_num(1, 2, 3), want[0, see][..., 5].nan_to_num(1, 2, 3))
        assert torch.equal(lse, lse0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_hidden_infinities_reach_no_gradient(at, dtype):
    M = 130
    q, k, v, g = make(13, 1, M, M, 2, 1, 64, 64, dtype)
    kw = dict(causal=True, window=40)
    out, lse = at.attention_fwd(q, k, v, **kw)
    base = at.attention_bwd(q, k, v, out, lse, g, **kw)
    # a row of dout that is not finite: its own dq, and the dk, dv of the keys 31 .. 70 that it sees
    g2 = g.clone()
    g2[0, 70, :, 3] = math.inf
    dq, dk, dv = at.attention_bwd(q, k, v, out, lse, g2, **kw)
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[70] = False
    keys = torch.ones(M, dtype=torch.bool, device="cuda")
    keys[31:71] = False
    if dtype == torch.bfloat16:  # fp16 gradients carry a common power of two, which an infinity sets aside
        assert torch.equal(dq[0, rows], base[0][0, rows])
        assert torch.equal(dk[0, keys], base[1][0, keys])
    assert dq[0, rows].isfinite().all() and dk[0, keys].isfinite().all() and dv[0, keys].isfinite().all()
    assert torch.equal(dv[0, keys], base[2][0, keys])
    assert not dq[0, 70].isfinite().any() and not dv[0, 31:71, :, 3].isfinite().any()
    # a key: its rows' gradients, and no other's
    k2 = k.clone()
    k2[0, 70] = math.nan
    out2, lse2 = at.attention_fwd(q, k2, v, **kw)
    dq, dk, dv = at.attention_bwd(q, k2, v, out2, lse2, g, **kw)
    rows[:] = True
    rows[70:110] = False
    assert torch.equal(dq[0, rows], base[0][0, rows])
    assert dq[0, 70:110].isnan().all()
    assert dk[0, :31].isfinite().all() and dv[0, 110:].isfinite().all()


def test_second_derivatives_are_refused(at):
    """create_graph: the first gradients as ever, and an error, not a wrong value, for the second."""
    q, k, v, g = make(25, 1, 20, 20, 2, 1, 64, 64, torch.float16)
    q.requires_grad_(True)
    plain, = torch.autograd.grad(at.attention(q, k, v), q, g)
    dq, = torch.autograd.grad(at.attention(q, k, v), q, g, create_graph=True)
    assert torch.equal(plain, dq)
    with pytest.raises(RuntimeError, match="once_differentiable|does not require grad"):
        torch.autograd.grad(dq.float().square().sum(), q)


def test_gradients_against_differences(at):
    """Directional differences of L = <dout, out>, in 64 bits around the 16-bit point, and the gradients'
    inner products with the direction: to 2 % of the sum of |terms|' root (rounding to 16 bits)."""
    q, k, v, g = make(14, 1, 40, 60, 4, 2, 64, 64, torch.float16, std=0.5)
    out, lse = at.attention_fwd(q, k, v, causal=True)
    grads = at.attention_bwd(q, k, v, out, lse, g, causal=True)
    gen = torch.Generator().manual_seed(3)
    x = [t.cpu().double() for t in (q, k, v)]

    def loss(y):
        s = (y[0][0].transpose(0, 1) @ y[1][0].repeat_interleave(2, 1).transpose(0, 1).transpose(1, 2)) * 0.125
        s = s.masked_fill(~ref.visible(40, 60, True, 0), -math.inf)
        o = torch.softmax(s, -1) @ y[2][0].repeat_interleave(2, 1).transpose(0, 1)
        return (o.transpose(0, 1) * g[0].cpu().double()).sum()

    for n in range(3):
        d = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)
        step = 1e-4
        y, z = list(x), list(x)
        y[n], z[n] = x[n] + step * d, x[n] - step * d
        want = (loss(y) - loss(z)) / (2 * step)
        got = (grads[n].cpu().double() * d).sum()
        size = (grads[n].cpu().double() * d).norm()
        assert abs(got - want) <= 0.02 * size, (n, got, want, size)


def test_autograd_only_wanted_gradients(at):
    q, k, v, g = make(15, 1, 50, 50, 2, 1, 64, 64, torch.bfloat16)
    out, lse = at.attention_fwd(q, k, v)
    full = at.attention_bwd(q, k, v, out, lse, g)
    for want in ((True, False, False), (False, True, False), (False, False, True)):
        part = at.attention_bwd(q, k, v, out, lse, g, want=want)
        for w, p, f in zip(want, part, full):
            assert (p is None) != w and (p is None or torch.equal(p, f))
    q.requires_grad_(True)
    o = at.attention(q, k, v)
    assert torch.equal(o, out)
    low = torch.empty_like(out)
    at.attention_fwd(q.detach(), k, v, low=low)
    dq, = torch.autograd.grad(o, q, g)
    assert torch.equal(dq, at.attention_bwd(q.detach(), k, v, out, lse, g, low=low)[0])
    dq2, = torch.autograd.grad(at.attention(q, k, v).sum(), q)   # an upstream gradient of stride 0
    dq3 = at.attention_bwd(q.detach(), k, v, out, lse, torch.ones_like(out), low=low)[0]
    assert torch.equal(dq2, dq3)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_rounding_leaves(at, dtype):
    """low: out + low is out to twice the digits, so <dout, out> in the backward pass is too, and with it
    the gradients of rows of few keys, where it does not cancel."""
    q, k, v, g = make(21, 1, 20, 20, 2, 1, 64, 64, dtype, std=0.3)
    low = torch.empty_like(g)
    out, lse = at.attention_fwd(q, k, v, causal=True, low=low)
    r = ref.one(q[0], k[0], v[0], 0.125, True, dout=g[0])
    plain, _ = at.attention_fwd(q, k, v, causal=True)
    assert torch.equal(out, plain)
    u = ref.half_step(dtype)
    assert (low.float().abs() <= u * (1 + u) * out.float().abs() + 2.0 ** -25).all()
    with_low, without = at.attention_bwd(q, k, v, out, lse, g, causal=True, low=low), at.attention_bwd(q, k, v, out, lse, g, causal=True)
    for name, a, b in zip(("dq", "dk", "dv"), with_low, without):
        ref.check(name, a[0], *r[name])
        err = [(t[0].cpu().double() - r[name][0]).norm() for t in (a, b)]
        assert err[0] <= err[1] * 1.02, (name, err)
    assert torch.equal(with_low[2], without[2])


def test_results_repeat_bit_for_bit(at):
    q, k, v, g = make(16, 2, 500, 500, 8, 2, 128, 128, torch.float16)
    first = None
    for _ in range(3):
        out, lse = at.attention_fwd(q, k, v, causal=True)
        res = (out, lse) + at.attention_bwd(q, k, v, out, lse, g, causal=True)
        first = first or res
        for a, b in zip(first, res):
            assert torch.equal(a, b)


def test_no_rows_or_no_keys(at):
    for M, N in ((0, 5), (5, 0), (0, 0)):
        q, k, v, g = make(17, 2, M, N, 2, 1, 64, 64, torch.float16)
        out, lse = at.attention_fwd(q, k, v)
        dq, dk, dv = at.attention_bwd(q, k, v, out, lse, g)
        assert not out.any() and (lse == -math.inf).all()
        for t, like in ((dq, q), (dk, k), (dv, v)):
            assert t.shape == like.shape and not t.any()


def test_packed_rows_before_the_first_sequence(at):
    """Offsets that do not start at 0: the rows before them belong to no sequence."""
    gen = torch.Generator().manual_seed(28)
    q, k, v, g = (normal(gen, (60, 2, 64), torch.bfloat16) for _ in range(4))
    for t in (q, k, v, g):
        t[:7] = float("nan")
    offs = torch.tensor([7, 30, 50], dtype=torch.int32, device="cuda")
    out, lse = at.attention_fwd(q, k, v, q_offsets=offs, causal=True)
    grads = at.attention_bwd(q, k, v, out, lse, g, q_offsets=offs, causal=True)
    for i in (slice(7, 30), slice(30, 50)):
        r = ref.one(q[i], k[i], v[i], 0.125, True, dout=g[i])
        for name, t in (("out", out[i]), ("lse", lse[:, i]), ("dq", grads[0][i]), ("dk", grads[1][i]), ("dv", grads[2][i])):
            ref.check(name, t, *r[name])
    for t in (out,) + grads:
        assert not t[:7].any() and not t[50:].any()
    assert (lse[:, :7] == -math.inf).all() and (lse[:, 50:] == -math.inf).all()


def test_packed_without_sequences(at):
    """One offset, no sequence: every row is one of none."""
    gen = torch.Generator().manual_seed(26)
    q, k, v = (normal(gen, (n, 2, 64), torch.float16) for n in (40, 3000, 3000))
    offs = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = at.attention_fwd(q, k, v, q_offsets=offs)
    assert not out.any() and (lse == -math.inf).all()
    for t in at.attention_bwd(q, k, v, out, lse, torch.ones_like(out), q_offsets=offs):
        assert not t.any()


def test_captured_autograd_step_replays(at):
    """The step through autograd, captured with leaves of its own (a leaf that an eager graph holds would
    bring that graph's stream into the capture)."""
    q, k, v, g = make(27, 2, 70, 70, 4, 2, 64, 64, torch.bfloat16)

    def step(leaves):
        out = at.attention(*leaves, causal=True)
        return (out.detach(),) + torch.autograd.grad(out, leaves, g)

    eager = [t.clone() for t in step([t.clone().requires_grad_(True) for t in (q, k, v)])]
    mine = [t.clone().requires_grad_(True) for t in (q, k, v)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(mine)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(mine)
    for _ in range(3):
        for t in held:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a, b)


def test_threads(at):
    """Calls from several host threads at once, each on a stream of its own."""
    import threading
    sets = [make(30 + i, 1, 100 + i, 150, 2, 1, 64, 64, torch.float16) for i in range(4)]
    want = [at.attention_fwd(q, k, v)[0] for q, k, v, _ in sets]
    torch.cuda.synchronize()
    got, streams = [None] * 4, [torch.cuda.Stream() for _ in range(4)]

    def work(i):
        q, k, v, _ = sets[i]
        for _ in range(50):
            got[i] = at.attention_fwd(q, k, v, stream=streams[i])[0]

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_captured_step_replays(at):
    """Forward and backward captured into a graph: every replay equals the eager call, with other
    eager calls between the replays."""
    q, k, v, g = make(18, 2, 150, 150, 4, 2, 64, 64, torch.float16)

    def step():
        out, lse = at.attention_fwd(q, k, v, causal=True)
        return (out, lse) + at.attention_bwd(q, k, v, out, lse, g, causal=True)

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    other = make(19, 1, 90, 300, 4, 2, 64, 64, torch.float16)
    for _ in range(3):
        for t in held:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a, b)
        out, lse = at.attention_fwd(*other[:3])
        at.attention_bwd(*other[:3], out, lse, other[3])
        torch.cuda.synchronize()


def test_calls_on_two_streams(at):
    """Two calls in flight on streams of their own, results allocated by the calls."""
    sets = [make(20 + i, 1, 300, 300, 4, 2, 64, 64, torch.float16) for i in range(2)]
    want = []
    for q, k, v, g in sets:
        out, lse = at.attention_fwd(q, k, v, causal=True)
        want.append((out, lse) + at.attention_bwd(q, k, v, out, lse, g, causal=True))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = []
        for (q, k, v, g), st in zip(sets, streams):
            out, lse = at.attention_fwd(q, k, v, causal=True, stream=st)
            got.append((out, lse) + at.attention_bwd(q, k, v, out, lse, g, causal=True, stream=st))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y)
