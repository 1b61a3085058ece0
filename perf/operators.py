"""The attention operators whose speed is tracked, over the range in which they are used.

A case names one operator (``call``) and its sizes:
  fwd      attention_fwd: the softmax-weighted sum and its log-sum-exp
  step     attention under autograd: the sum, then the gradients of q, k and v
  append   attention_append: the keys and values of new tokens into the pages of a cache
  paged    attention_paged: a chunk of new tokens, or one new token, of every sequence over its pages

Layouts: ``dense`` (B x M x H x D, every sequence whole), ``padded`` (the same
with the number of rows of every sequence in use) and ``packed`` (rows of all
sequences one behind the other, with offsets).  Where ``own`` is false the
operators are computed in their plain form in 32 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _case(call, B=1, M=1, N=0, Hq=8, Hkv=8, D=64, C=0, dtype="bf16", layout="dense", causal=True, window=0,
          page=16, lens=0, name=None):
    """M: (most) query rows or new tokens of a sequence; N: (most) keys of a sequence, new ones
    included (0: M).  lens: seed of the sequences' own lengths."""
    case = dict(call=call, B=B, M=M, N=N or M, Hq=Hq, Hkv=Hkv, D=D, C=C or D, dtype=dtype, layout=layout,
                causal=causal, window=window, page=page, lens=lens)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # a short prompt of a small model, or attention pooling of a small set: latency
        _case("fwd", M=37, Hq=4, Hkv=4, dtype="f16", name="fwd_small"),
        # a mixed prefill batch: ten ragged sequences packed, four query heads to a key head
        _case("fwd", B=10, M=1200, Hq=16, Hkv=4, D=128, layout="packed", lens=3, name="fwd_packed"),
        # a long prompt: bound by the matrix cores
        _case("fwd", M=16384, Hq=16, Hkv=4, D=128, name="fwd_long"),
        # a training step of a small model in half precision
        _case("step", B=4, M=512, Hq=8, Hkv=8, dtype="f16", name="step_small"),
        # cross attention over padded sets (normalised kernel regression): odd sizes,
        # other widths for keys and values, no causal mask, some sets empty
        _case("step", B=6, M=501, N=1403, Hq=6, Hkv=6, D=80, C=48, dtype="f16", layout="padded", causal=False, lens=5,
              name="step_cross"),
        # a training step over packed documents with a sliding window
        _case("step", B=6, M=2047, Hq=16, Hkv=4, D=128, layout="packed", window=1000, lens=7, name="step_window"),
        # a training step at wide heads
        _case("step", B=2, M=2048, Hq=8, Hkv=8, D=256, name="step_d256"),
        # a large training step
        _case("step", M=8192, Hq=32, Hkv=8, D=128, name="step_large"),
        # new tokens of a decode batch into the cache: latency
        _case("append", B=8, M=1, N=900, Hkv=8, D=128, lens=1, name="append_token"),
        # a prefill chunk into the cache
        _case("append", B=8, M=2048, N=4096, Hkv=8, D=128, page=64, lens=2, name="append_chunk"),
        # one new token of every sequence of a large decode batch
        _case("paged", B=64, M=1, N=8192, Hq=32, Hkv=8, D=128, lens=4, name="paged_token"),
        # chunks of long prompts over what is cached of them
        _case("paged", B=4, M=512, N=12000, Hq=32, Hkv=8, D=128, page=64, lens=6, name="paged_chunk"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["fwd", "fwd", "step", "step", "step", "append", "paged", "paged", "paged"])
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 8])
    D = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 256])
    dtype, lens = rng.choice(["bf16", "bf16", "f16"]), rng.randrange(1 << 20)
    kind = dict(Hq=Hkv * G, Hkv=Hkv, D=D, dtype=dtype, lens=lens)
    if call in ("append", "paged"):
        page = rng.choice([16, 16, 32, 64, 128, 20])
        M, B = (1, _log_int(rng, 1, 64)) if rng.random() < 0.5 else (_log_int(rng, 2, 512), _log_int(rng, 1, 6))
        N = max(M, _log_int(rng, 64, 8192))
        return _case(call, B=B, M=M, N=N, page=page, window=rng.choice([0, 0, 0, 700]), **kind)
    layout = rng.choice(["dense", "padded", "packed"])
    M = _log_int(rng, 16, 6000)
    B = max(1, min(_log_int(rng, 1, 16), 8000 // M))
    causal = rng.random() < 0.7
    N, C = M, D
    if not causal:
        N = max(1, _log_int(rng, 16, 6000))
        B = max(1, min(B, 8000 // N))
        C = rng.choice([D, D, 48, 64])
    while B * M * N * kind["Hq"] * (D + C) > (1 << 37):  # at most a sixth of the largest listed case's products
        M, N = M * 3 // 4, N * 3 // 4
    window = rng.choice([0, 0, max(1, M // 3)]) if causal else 0
    return _case(call, B=B, M=M, N=N, C=C, layout=layout, causal=causal, window=window, **kind)


def _lengths(case):
    """(rows, keys) of every sequence, as lists: what a data loader or scheduler knows."""
    B, M, N = case["B"], case["M"], case["N"]
    rng = random.Random(case["lens"] * 7919 + 13)
    if case["call"] in ("append", "paged"):
        rows = [M if M == 1 else rng.randint(max(1, M // 2), M) for _ in range(B)]
        keys = [max(r, rng.randint(max(1, N // 4), N)) for r in rows]
        keys[rng.randrange(B)] = N
        return rows, keys
    if case["layout"] == "dense":
        return [M] * B, [N] * B
    rows = [rng.randint(M // 4, M) for _ in range(B)]
    rows[rng.randrange(B)] = M
    keys = list(rows) if case["causal"] else [rng.randint(N // 4, N) for _ in range(B)]
    if B > 3 and not case["causal"]:
        keys[rng.randrange(B)] = 0  # an empty set
    return rows, keys


def _offsets(lens, dev):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    rows, keys = _lengths(case)
    B, M, N, Hq, Hkv, D, C = (case[n] for n in ("B", "M", "N", "Hq", "Hkv", "D", "C"))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).mul_(std).to(dt)

    state = dict(case, rows=rows, keys=keys, scale=D ** -0.5)
    if case["call"] in ("append", "paged"):
        page = case["page"]
        width = -(-N // page)
        used = [-(-n // page) for n in keys]
        pages = sum(used) + 3
        order = torch.randperm(pages, generator=gen, device=dev).tolist()
        table = torch.full((B, width), -1, dtype=torch.int32)
        for b in range(B):
            table[b, :used[b]] = torch.tensor([order.pop() for _ in range(used[b])], dtype=torch.int32)
        T = sum(rows)
        state.update(k_pages=normal(pages, page, Hkv, D), v_pages=normal(pages, page, Hkv, C), page_table=table.to(dev),
                     seq_lens=torch.tensor(keys, dtype=torch.int32, device=dev),
                     q_offsets=None if M == 1 else _offsets(rows, dev))
        if case["call"] == "append":
            state.update(k=normal(T, Hkv, D), v=normal(T, Hkv, C))
        else:
            state.update(q=normal(T, Hq, D))
        return state
    if case["layout"] == "packed":
        state.update(q=normal(sum(rows), Hq, D), k=normal(sum(keys), Hkv, D), v=normal(sum(keys), Hkv, C),
                     lengths=dict(q_offsets=_offsets(rows, dev), k_offsets=_offsets(keys, dev)))
    else:
        state.update(q=normal(B, M, Hq, D), k=normal(B, N, Hkv, D), v=normal(B, N, Hkv, C), lengths={})
        if case["layout"] == "padded":
            state["lengths"] = dict(q_lens=torch.tensor(rows, dtype=torch.int32, device=dev),
                                    k_lens=torch.tensor(keys, dtype=torch.int32, device=dev))
    if case["call"] == "step":
        state["dout"] = normal(*state["q"].shape[:-1], C, std=0.02)
        for n in ("q", "k", "v"):
            state[n].requires_grad_(True)
    return state


def run(state):
    if own:
        return _run_own(state)
    with torch.no_grad():
        return _run_plain(state)


def _run_own(s):
    from paper_2609_04910_amd import attention as at
    if s["call"] == "fwd":
        return at.attention_fwd(s["q"], s["k"], s["v"], causal=s["causal"], window=s["window"], **s["lengths"])
    if s["call"] == "step":
        out = at.attention(s["q"], s["k"], s["v"], causal=s["causal"], window=s["window"], **s["lengths"])
        return (out.detach(),) + torch.autograd.grad(out, (s["q"], s["k"], s["v"]), s["dout"])
    if s["call"] == "append":
        at.attention_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["page_table"], s["seq_lens"],
                            q_offsets=s["q_offsets"])
        return s["k_pages"], s["v_pages"]
    return at.attention_paged(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["seq_lens"],
                              q_offsets=s["q_offsets"], window=s["window"])


def _sequence_of(offsets, total):
    """Sequence and row within it of each of `total` packed rows."""
    row = torch.arange(total, device=offsets.device)
    seq = torch.searchsorted(offsets[1:].contiguous(), row.to(torch.int32), right=True)
    return seq, row - offsets[seq]


def _visible(place, key, window, causal):
    """place: position of the row among its keys."""
    see = torch.ones(torch.broadcast_shapes(place.shape, key.shape), dtype=torch.bool, device=place.device)
    if causal:
        see = see & (key <= place)
    if window:
        see = see & (key > place - window)
    return see


def _attend(q, k, v, see, scale):
    """q: B x Hkv x G x M x D, k, v: B x Hkv x 1 x N x (D, C), see: B x 1 x 1 x M x N;
    (probabilities, out, lse) in 32 bits; rows that see nothing: 0 and -inf."""
    s = (q @ k.transpose(-1, -2)).mul_(scale).masked_fill_(~see, -math.inf)
    m = s.amax(-1, keepdim=True) if s.shape[-1] else s.new_full(s.shape[:-1] + (1,), -math.inf)
    p = s.sub_(m.masked_fill(m == -math.inf, 0.0)).exp_()
    z = p.sum(-1, keepdim=True)
    p = p.div_(z.masked_fill(z == 0.0, 1.0))
    return p, p @ v, (m + z.log()).squeeze(-1)


def _heads(x, Hkv):
    """B x M x H x D -> B x Hkv x (H / Hkv) x M x D in 32 bits."""
    B, M, H, D = x.shape
    return x.float().view(B, M, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).contiguous()


def _rows(x):
    """B x Hkv x G x M x D -> B x M x H x D."""
    B, Hkv, G, M, D = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(B, M, Hkv * G, D)


def _run_plain(s):
    dt, dev, Hkv, window, causal = DTYPES[s["dtype"]], s["v_pages" if "v_pages" in s else "v"].device, s["Hkv"], s["window"], s["causal"]
    if s["call"] in ("append", "paged"):
        x = s["k"] if s["call"] == "append" else s["q"]
        offsets = s["q_offsets"]
        if offsets is None:
            offsets = torch.arange(x.shape[0] + 1, device=dev, dtype=torch.int32)
        seq, at = _sequence_of(offsets, x.shape[0])
        first = s["seq_lens"] - (offsets[1:] - offsets[:-1])
        place = first[seq] + at
        if s["call"] == "append":
            slot = (s["page_table"][seq, place // s["page"]].long(), (place % s["page"]).long())
            s["k_pages"][slot] = s["k"]
            s["v_pages"][slot] = s["v"]
            return s["k_pages"], s["v_pages"]
        B, width = s["page_table"].shape
        table = s["page_table"].clamp(min=0).long()
        k = s["k_pages"][table].reshape(B, width * s["page"], Hkv, s["D"])
        v = s["v_pages"][table].reshape(B, width * s["page"], Hkv, s["C"])
        q = torch.zeros((B, s["M"]) + x.shape[1:], dtype=torch.float32, device=dev)
        q[seq, at] = x.float()
        key = torch.arange(width * s["page"], device=dev)
        where = first[:, None] + torch.arange(s["M"], device=dev)
        see = _visible(where[:, :, None], key, window, True) & (key < s["seq_lens"][:, None, None])
        out = _attend(_heads(q, Hkv), _heads(k, Hkv), _heads(v, Hkv), see[:, None, None], s["scale"])[1]
        return _rows(out)[seq, at].to(dt)
    q, k, v = s["q"], s["k"], s["v"]
    if s["layout"] == "packed":
        qo, ko = s["lengths"]["q_offsets"], s["lengths"]["k_offsets"]
        qs, qi = _sequence_of(qo, q.shape[0])
        ks, ki = _sequence_of(ko, k.shape[0])
        ahead = (ko[1:] - ko[:-1]) - (qo[1:] - qo[:-1])
        see = ((qs[:, None] == ks) & _visible((qi + ahead[qs])[:, None], ki, window, causal))[None]
        q, k, v = q[None], k[None], v[None]
    else:
        row, key = torch.arange(s["M"], device=dev), torch.arange(s["N"], device=dev)
        nq = s["lengths"]["q_lens"] if s["lengths"] else torch.full((s["B"],), s["M"], device=dev)
        nk = s["lengths"]["k_lens"] if s["lengths"] else torch.full((s["B"],), s["N"], device=dev)
        see = _visible((row + (nk - nq)[:, None])[:, :, None], key, window, causal)
        see = see & (key < nk[:, None, None]) & (row[:, None] < nq[:, None, None])
    see = see[:, None, None]
    qf, kf, vf = _heads(q, Hkv), _heads(k, Hkv), _heads(v, Hkv)
    p, out, lse = _attend(qf, kf, vf, see, s["scale"])
    packed = s["layout"] == "packed"
    whole = (lambda t: _rows(t).to(dt)[0] if packed else _rows(t).to(dt))
    if s["call"] == "fwd":
        lse = lse.flatten(1, 2)
        return whole(out), lse[0] if packed else lse
    g = s["dout"]
    gf = _heads(g[None] if packed else g, Hkv)
    dv = (p.transpose(-1, -2) @ gf).sum(2, keepdim=True)
    ds = gf @ vf.transpose(-1, -2)
    ds = ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p)
    dq = (ds @ kf).mul_(s["scale"])
    dk = (ds.transpose(-1, -2) @ qf).sum(2, keepdim=True).mul_(s["scale"])
    return whole(out), whole(dq), whole(dk), whole(dv)


def _pairs(case):
    """(visible pairs of all sequences, keys that some row sees)."""
    pairs = seen = 0
    rows, keys = _lengths(case)
    causal = case["causal"] or case["call"] == "paged"
    for m, n in zip(rows, keys):
        if not causal:
            pairs, seen = pairs + m * n, seen + (n if m else 0)
            continue
        low = n
        for i in range(m):
            end = min(n, n - m + i + 1)
            start = max(0, end - case["window"]) if case["window"] else 0
            if end > start:
                pairs, low = pairs + end - start, min(low, start)
        seen += n - low
    return pairs, seen


def work(case):
    """Inputs read once and outputs written once; per visible pair and query head 2 D + 2 C flops for
    the sum, and 4 D + 4 C for the gradients (dS, dV, dQ and dK; probabilities are not counted twice)."""
    rows, keys = _lengths(case)
    Hq, Hkv, D, C = case["Hq"], case["Hkv"], case["D"], case["C"]
    if case["call"] == "append":
        return {"bytes": 2 * sum(rows) * Hkv * (D + C) * 2, "flops": 0}
    pairs, seen = _pairs(case)
    flops = pairs * Hq * (2 * D + 2 * C)
    if case["call"] == "paged":
        return {"bytes": 2 * (sum(rows) * Hq * (D + C) + seen * Hkv * (D + C)), "flops": flops}
    m, n = (case["B"] * case["M"], case["B"] * case["N"]) if case["layout"] == "padded" else (sum(rows), sum(keys))
    if case["call"] == "fwd":
        return {"bytes": 2 * (sum(rows) * Hq * D + m * Hq * C + seen * Hkv * (D + C)) + 4 * m * Hq, "flops": flops}
    return {"bytes": 2 * (sum(rows) * Hq * (D + C) + seen * Hkv * (D + C) + m * Hq * (C + D) + n * Hkv * (D + C)),
            "flops": 3 * flops}


def _exact_one(q, k, v, scale, causal, window, dout=None):
    """One sequence, in 64 bits: q: m x Hq x D, k, v: n x Hkv x (D, C).  Head by head, from the
    definition: out = sum w v / sum w with w = exp(scale q.k) over the keys that a row sees."""
    m, Hq, n, Hkv = q.shape[0], q.shape[1], k.shape[0], k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out = q.new_zeros(m, Hq, v.shape[2])
    lse = q.new_full((Hq, m), -math.inf)
    grads = None if dout is None else (torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v))
    if m == 0 or n == 0:
        return out, lse, grads
    i = torch.arange(m, device=q.device).unsqueeze(1) + (n - m)
    j = torch.arange(n, device=q.device).unsqueeze(0)
    hidden = torch.zeros(m, n, dtype=torch.bool, device=q.device)
    if causal:
        hidden |= j > i
        if window:
            hidden |= j <= i - window
    for h in range(Hq):
        kh, vh = k[:, h * Hkv // Hq], v[:, h * Hkv // Hq]
        x = torch.mm(q[:, h], kh.t()) * scale
        x[hidden] = -math.inf
        lse[h] = torch.logsumexp(x, 1)
        w = torch.exp(x - torch.where(torch.isinf(lse[h]), torch.zeros_like(lse[h]), lse[h])[:, None])
        out[:, h] = torch.mm(w, vh)
        if dout is None:
            continue
        g = dout[:, h].double()
        e = w * (torch.mm(g, vh.t()) - (g * out[:, h]).sum(1, keepdim=True))
        grads[0][:, h] = scale * torch.mm(e, kh)
        grads[1][:, h * Hkv // Hq] += scale * torch.mm(e.t(), q[:, h])
        grads[2][:, h * Hkv // Hq] += torch.mm(w.t(), g)
    return out, lse, grads


def exact(case, seed):
    s = prepare(case, seed)
    rows, keys = _lengths(case)
    qs = [sum(rows[:b]) for b in range(case["B"])]
    if case["call"] in ("append", "paged"):
        page, table = case["page"], s["page_table"].tolist()
        if case["call"] == "append":
            k, v = s["k_pages"].clone(), s["v_pages"].clone()
            for b, (m, n) in enumerate(zip(rows, keys)):
                where = torch.arange(n - m, n, device=k.device)
                pages = torch.tensor(table[b], device=k.device)[torch.div(where, page, rounding_mode="floor")]
                k[pages, where % page] = s["k"][qs[b]:qs[b] + m]
                v[pages, where % page] = s["v"][qs[b]:qs[b] + m]
            return k.double(), v.double()
        out = []
        for b, (m, n) in enumerate(zip(rows, keys)):
            pages = table[b][:-(-n // page)]
            k = torch.cat([s["k_pages"][p] for p in pages])[:n]
            v = torch.cat([s["v_pages"][p] for p in pages])[:n]
            out.append(_exact_one(s["q"][qs[b]:qs[b] + m], k, v, s["scale"], True, case["window"])[0])
        return torch.cat(out)
    ks = [sum(keys[:b]) for b in range(case["B"])]
    q, k, v = (s[n].detach() for n in ("q", "k", "v"))
    g = s.get("dout")
    packed = case["layout"] == "packed"
    out = torch.zeros(q.shape[:-1] + (case["C"],), dtype=torch.float64, device=q.device)
    lse = torch.full(((case["Hq"],) if packed else (case["B"], case["Hq"])) + (sum(rows) if packed else case["M"],),
                     -math.inf, dtype=torch.float64, device=q.device)
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device=q.device) for t in (q, k, v))
    for b, (m, n) in enumerate(zip(rows, keys)):
        at = (slice(qs[b], qs[b] + m),) if packed else (b, slice(0, m))
        on = (slice(ks[b], ks[b] + n),) if packed else (b, slice(0, n))
        o, z, grads = _exact_one(q[at], k[on], v[on], s["scale"], case["causal"], case["window"],
                                 None if g is None else g[at])
        out[at] = o
        lse[(slice(None),) + at if packed else (b, slice(None), slice(0, m))] = z
        if grads is not None:
            dq[at], dk[on], dv[on] = grads
    return (out, lse) if case["call"] == "fwd" else (out, dq, dk, dv)
