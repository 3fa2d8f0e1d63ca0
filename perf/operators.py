"""The operators on caches in pages as a user of this library calls them, as cases that can be timed and compared.

  attention  rs_paged_attention: new tokens of several sequences, one each (decode) or a span each (a chunk of a prompt, a
             catch-up), attend to their sequence's positions in a cache of pages, causally, in a sliding window if asked
  append     rs_paged_append: the rows of a QKV projection: q rotated to its position, k rotated into the pages, v into the pages
  rope       rs_rope_rows: heads rotated to their positions; pairs half a head apart or side by side, part of the head, scaled

`run` computes the plain form, elementary torch operations in 32 bits on all sequences at once, or, with `own`, makes the
library's calls.  K pages are [page][KV head][position][channel], V pages [page][KV head][channel][position], bf16; q, k and v
are fp32 (what this library's models compute with) or bf16.
Head layouts are those of the package's models (1.5B: 12 query and 2 KV heads of 128 channels, 7B: 28 / 4, 14B and 32B: 40 / 8,
the tiny pair: 32 channels) and one of 64 channels.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = {"s15": (12, 2, 128), "m7": (28, 4, 128), "m14": (40, 8, 128), "h64": (16, 4, 64), "tiny": (8, 2, 32)}
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
THETA = 1e6


def _attention(name, heads, dtype, seqs, rows, pos_lo, pos_hi, page, window=0):
    """rows new tokens of seqs sequences that hold pos_lo .. pos_hi positions before them."""
    c = {"kind": "attention", "heads": heads, "dtype": dtype, "seqs": seqs, "rows": rows, "pos_lo": pos_lo, "pos_hi": pos_hi, "page": page, "window": window}
    return c if name is None else dict(c, name=name)


def _append(name, heads, dtype, seqs, rows, pos_lo, pos_hi, page, rot, interleaved=False, factor=1.0):
    c = {"kind": "append", "heads": heads, "dtype": dtype, "seqs": seqs, "rows": rows, "pos_lo": pos_lo, "pos_hi": pos_hi, "page": page, "rot": rot,
         "interleaved": interleaved, "factor": factor}
    return c if name is None else dict(c, name=name)


def _rope(name, heads, dtype, rows, pos_hi, rot, interleaved=False, factor=1.0, inverse=False):
    c = {"kind": "rope", "heads": heads, "dtype": dtype, "rows": rows, "pos_hi": pos_hi, "rot": rot, "interleaved": interleaved, "factor": factor, "inverse": inverse}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a decode step of the small model early in a reply: latency only
        _attention("attention_s15_decode_1_short", "s15", "fp32", 1, 1, 200, 200, 64),
        # the large model's step of the stitched loop at batch 1, late in its context
        _attention("attention_m7_decode_1", "m7", "fp32", 1, 1, 4561, 4561, 64),
        # the largest batch of the package's workloads, contexts of all lengths
        _attention("attention_m7_decode_128", "m7", "bf16", 128, 128, 512, 4607, 64),
        # a catch-up of the large model late in a long context, an odd number of rows
        _attention("attention_m14_catchup_61", "m14", "fp32", 1, 61, 9001, 9001, 128),
        # small pages, a sliding window, spans of all lengths
        _attention("attention_h64_window_33", "h64", "bf16", 33, 701, 0, 6000, 16, window=1000),
        # chunks of four long prompts: the matrix cores' case
        _attention("attention_m14_chunks_8192", "m14", "bf16", 4, 8192, 0, 14000, 64),
        # the new token of one sequence; the new tokens of the largest batch
        _append("append_s15_decode_1", "s15", "fp32", 1, 1, 4570, 4570, 64, 128),
        _append("append_m7_decode_128", "m7", "bf16", 128, 128, 512, 4607, 64, 128),
        # part of the head rotated, neighbours paired, small pages, ragged spans
        _append("append_m7_partial_517", "m7", "fp32", 9, 517, 0, 5000, 16, 64, interleaved=True),
        # chunks of four long prompts of a model stretched to four times its context
        _append("append_m14_chunks_8192", "m14", "bf16", 4, 8192, 0, 100000, 64, 128, factor=4.0),
        # queries of a batch of spans; queries of a long prompt
        _rope("rope_m7_128", "m7", "fp32", 128, 4608, 128),
        _rope("rope_m14_16384", "m14", "bf16", 16384, 131072, 128, interleaved=True, factor=4.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    u = rng.random()
    heads, dtype = rng.choice(["s15", "m7", "m7", "m14", "m14", "h64", "tiny"]), rng.choice(["fp32", "bf16", "bf16"])
    nq, nkv, hd = HEADS[heads]
    page = rng.choice([16, 32, 64, 128, 256])
    rot = rng.choice([hd, hd, hd, hd // 2, hd // 4 * 3])
    inter, factor = rng.random() < 0.3, rng.choice([1.0, 1.0, 2.0, 4.0, 7.5])
    if u < 0.2:
        return _rope(None, heads, dtype, _log_int(rng, 1, 16000), _log_int(rng, 100, 131072), rot, inter, factor, rng.random() < 0.4)
    if rng.random() < 0.4:
        seqs = rows = _log_int(rng, 1, 128)
    else:
        rows = _log_int(rng, 2, 8192)
        seqs = min(_log_int(rng, 1, 64), rows)
    # a batch's caches together are at most about a gigabyte a tensor; prompts in long chunks cost at most what the largest listed ones do
    most = min((500 << 20) // (seqs * nkv * hd), 16000, 8192 * 40 * 9000 // (rows * nq) if rows > seqs else 1 << 30)
    if dtype == "fp32":
        most = min(most, max(64, 1200 * 40 * 9000 // (rows * nq)))
    hi = _log_int(rng, 16, max(32, most))
    lo = rng.randint(0, hi) if seqs > 1 else hi
    if u < 0.5:
        return _append(None, heads, dtype, seqs, rows, lo, hi, page, rot, inter, factor)
    return _attention(None, heads, dtype, seqs, rows, lo, hi, page, window=_log_int(rng, 1, 8192) if rng.random() < 0.3 else 0)


# ------------------------------------------------------------------ what a case stands for, from the case alone
def _spans(c):
    """(new rows, positions held before) of every sequence: uneven, the rows between half and one and a half of their mean."""
    n, rows = c["seqs"], c["rows"]
    weight = [1.0 + 0.5 * math.sin(2.4 * i + 0.7) for i in range(n)] if rows > n else [1.0] * n
    span = [max(1, int(rows * w / sum(weight))) for w in weight]
    i = 0
    while sum(span) != rows:
        step = 1 if sum(span) < rows else -1
        if span[i % n] + step >= 1:
            span[i % n] += step
        i += 1
    lo, hi = c["pos_lo"], c["pos_hi"]
    return span, [lo + (i * 7919 + 13 * i * i) % (hi - lo + 1) if n > 1 else hi for i in range(n)]


def _frequencies(rot, factor):
    """theta^(-2i/rot); with a factor, by parts (arXiv 2309.00071): wavelengths of which 32 and more fit the original context of 32768
    positions stay, those of which at most one fits are stretched, those between are blended.  And the amplitude 0.1 ln(factor) + 1."""
    f = THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if factor == 1.0:
        return f, 1.0
    keep = ((32768 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0, 1)
    return f * (keep + (1 - keep) / factor), 0.1 * math.log(factor) + 1.0


def work(c):
    nq, nkv, hd = HEADS[c["heads"]]
    size = 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "rope":
        return {"bytes": c["rows"] * (2 * nq * hd * size + 4), "flops": c["rows"] * nq * c["rot"] * 3}
    span, pos0 = _spans(c)
    if c["kind"] == "append":
        return {"bytes": c["rows"] * hd * ((2 * nq + 2 * nkv) * size + 2 * nkv * 2), "flops": c["rows"] * (nq + nkv) * c["rot"] * 3}
    w = c["window"] or 1 << 40
    seen = sum(p + m - max(0, p - w + 1) for m, p in zip(span, pos0))             # positions that some row of the sequence sees
    pairs = 0
    for m, p in zip(span, pos0):
        short = min(m, max(0, w - 1 - p))                                         # rows that see all from position 0 on
        pairs += short * (p + 1) + short * (short - 1) // 2
        pairs += (m - short) * w if c["window"] else (m - short) * (p + short + 1) + (m - short) * (m - short - 1) // 2
    return {"bytes": c["rows"] * nq * (2 * hd * size + 4) + seen * nkv * hd * 2 * 2, "flops": 4 * hd * nq * pairs}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _inputs(c, seed):
    """Everything the operator reads; the same for prepare() and exact()."""
    nq, nkv, hd = HEADS[c["heads"]]
    dt, g, rows = DTYPES[c["dtype"]], _gen(seed), c["rows"]
    s = {"case": c}
    if c["kind"] != "attention":
        f, s["amplitude"] = _frequencies(c["rot"], c["factor"])
        s["freq"] = f.cuda()
    if c["kind"] == "rope":
        s["pos"] = torch.randint(0, c["pos_hi"], (rows,), device="cuda", generator=g).to(torch.int32)
        s["x"] = _normal(g, (rows, nq, hd), dt)
        return s
    span, pos0 = _spans(c)
    n, page = c["seqs"], c["page"]
    need = [(p + m + page - 1) // page for p, m in zip(pos0, span)]
    total = sum(need)
    order = torch.randperm(total, device="cuda", generator=g).to(torch.int32).tolist()
    table, at, longest = [], 0, max(need)
    for k in need:                                               # the pages of a sequence lie anywhere; what it has not got is -1
        table.append(order[at:at + k] + [-1] * (longest - k))
        at += k
    slot = torch.randperm(n, device="cuda", generator=g).to(torch.int32)
    s["table"] = torch.empty(n, longest, dtype=torch.int32, device="cuda")
    s["table"][slot.long()] = _int(table)
    off = [0]
    for m in span:
        off.append(off[-1] + m)
    s.update(slot=slot, off=_int(off), pos0=_int(pos0), n=n, rows=rows, longest=max(span), last=max(p + m for p, m in zip(pos0, span)))
    s["k_pages"] = _normal(g, (total, nkv, page, hd), torch.bfloat16)
    s["v_pages"] = _normal(g, (total, nkv, hd, page), torch.bfloat16)
    if c["kind"] == "attention":
        s["q"] = _normal(g, (rows, nq, hd), dt)
    else:
        s["qkv"] = _normal(g, (rows, nq + 2 * nkv, hd), dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2507_17307_amd as P
        s["P"] = P
        if case["kind"] != "attention":
            s["rope"] = P.Rope(s["freq"], interleaved=case["interleaved"], amplitude=s["amplitude"])
        if case["kind"] == "rope":
            s["out"] = torch.empty_like(s["x"])
            return s
        s["cache"] = P.PagedCache(s["k_pages"], s["v_pages"], s["table"])
        if case["kind"] == "append":
            nq, nkv, hd = HEADS[case["heads"]]
            s["q"], s["k"], s["v"] = s["qkv"].split([nq, nkv, nkv], 1)
            s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        else:
            s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
            s["scratch"] = torch.empty(P.rs_paged_attention_scratch_bytes(s["cache"], s["n"], s["rows"], s["q"].shape[1]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def _rotate(x, pos, freq, amplitude, interleaved, inverse=False):
    """x [rows, heads, channels] in 32 bits; angles in 64."""
    rot = 2 * freq.numel()
    angle = pos.double()[:, None] * freq[None]
    cos, sin = (angle.cos() * amplitude).float()[:, None], (angle.sin() * (-amplitude if inverse else amplitude)).float()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _row_places(s):
    """(sequence, position) of every row."""
    r = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(s["off"].long(), r, right=True) - 1
    return seq, s["pos0"].long()[seq] + r - s["off"].long()[seq]


def _plain_append(s):
    c = s["case"]
    nq, nkv, hd = HEADS[c["heads"]]
    seq, pos = _row_places(s)
    page, place = s["table"][s["slot"].long()[seq], pos // c["page"]].long(), pos % c["page"]
    q, k, v = s["qkv"].float().split([nq, nkv, nkv], 1)
    s["k_pages"][page, :, place, :] = _rotate(k, pos, s["freq"], s["amplitude"], c["interleaved"]).to(torch.bfloat16)
    s["v_pages"][page, :, :, place] = v.to(torch.bfloat16)
    return _rotate(q, pos, s["freq"], s["amplitude"], c["interleaved"]).to(s["qkv"].dtype)


def _plain_attention(s):
    c = s["case"]
    nq, nkv, hd = HEADS[c["heads"]]
    n, m, g, length = s["n"], s["longest"], nq // nkv, s["last"]
    pages = s["table"].long()[s["slot"].long()].clamp(min=0)
    k = s["k_pages"][pages].transpose(1, 2).reshape(n, nkv, -1, hd)[:, :, :length].float()
    v = s["v_pages"][pages].permute(0, 2, 1, 4, 3).reshape(n, nkv, -1, hd)[:, :, :length].float()
    # rows of every sequence, as many as the longest span has
    off, i = s["off"].long(), torch.arange(m, device="cuda")
    row = (off[:-1, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"].float()[row].view(n, m, nkv, g, hd).permute(0, 2, 1, 3, 4).reshape(n, nkv, m * g, hd)
    at = s["pos0"].long()[:, None] + i
    j = torch.arange(length, device="cuda")
    seen = j <= at[..., None]
    if c["window"]:
        seen = seen & (j > at[..., None] - c["window"])
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(hd ** -0.5).view(n, nkv, m, g, length)
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(n, nkv, m * g, length), v).view(n, nkv, m, g, hd) / total
    lse = (top + total.log())[..., 0]
    seq, pos = _row_places(s)
    i = pos - s["pos0"].long()[seq]
    return out.permute(0, 2, 1, 3, 4)[seq, i].reshape(s["rows"], nq, hd).to(s["q"].dtype), lse.permute(0, 2, 1, 3)[seq, i].reshape(s["rows"], nq)


def run(s):
    c = s["case"]
    if c["kind"] == "rope":
        if own:
            s["P"].rs_rope_rows(s["rope"], s["pos"], s["x"], s["out"], inverse=c["inverse"])
            return s["out"]
        return _rotate(s["x"].float(), s["pos"], s["freq"], s["amplitude"], c["interleaved"], c["inverse"]).to(s["x"].dtype)
    if c["kind"] == "append":
        if own:
            s["P"].rs_paged_append(s["cache"], s["n"], s["rows"], s["slot"], s["off"], s["pos0"], s["rope"], s["q"], s["k"], s["v"], s["out"])
            q = s["out"]
        else:
            q = _plain_append(s)
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if own:
        s["P"].rs_paged_attention(s["cache"], s["n"], s["rows"], s["slot"], s["off"], s["pos0"], s["q"], HEADS[c["heads"]][2] ** -0.5, c["window"],
                                  s["out"], s["lse"], s["scratch"])
        out, lse = s["out"], s["lse"]
    else:
        out, lse = _plain_attention(s)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_turn(x, pos, freq, amplitude, interleaved, inverse):
    """Pairs as complex numbers, multiplied by amplitude e^(i angle)."""
    rot = 2 * freq.numel()
    x = x.double()
    angle = torch.outer(pos.double(), freq) * (-1.0 if inverse else 1.0)
    turn = torch.polar(torch.full_like(angle, amplitude), angle)[:, None]
    y = x.clone()
    re, im = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., re].contiguous(), x[..., im].contiguous()) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    nq, nkv, hd = HEADS[case["heads"]]
    if case["kind"] == "rope":
        return _exact_turn(s["x"], s["pos"], s["freq"], s["amplitude"], case["interleaved"], case["inverse"])
    page, table = case["page"], s["table"].tolist()
    span, pos0 = _spans(case)
    slot, off = s["slot"].tolist(), s["off"].tolist()
    if case["kind"] == "append":
        q, k, v = s["qkv"][:, :nq], s["qkv"][:, nq:nq + nkv], s["qkv"][:, nq + nkv:]
        pos = torch.cat([torch.arange(p, p + m) for m, p in zip(span, pos0)]).cuda()
        turned = _exact_turn(k, pos, s["freq"], s["amplitude"], case["interleaved"], False)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        for b in range(len(span)):
            for first in range(pos0[b] // page * page, pos0[b] + span[b], page):              # page by page
                lo, hi = max(first, pos0[b]), min(first + page, pos0[b] + span[b])
                to, r = table[slot[b]][first // page], off[b] + lo - pos0[b]
                kp[to, :, lo - first:hi - first] = turned[r:r + hi - lo].transpose(0, 1)
                vp[to, :, :, lo - first:hi - first] = v[r:r + hi - lo].double().permute(1, 2, 0)
        return {"q": _exact_turn(q, pos, s["freq"], s["amplitude"], case["interleaved"], False), "k_pages": kp, "v_pages": vp}
    out, lse = torch.empty(case["rows"], nq, hd, dtype=torch.float64, device="cuda"), torch.empty(case["rows"], nq, dtype=torch.float64, device="cuda")
    for b in range(len(span)):
        held = pos0[b] + span[b]
        mine = torch.tensor(table[slot[b]][:(held + page - 1) // page], device="cuda")
        kk = s["k_pages"][mine].double().permute(1, 0, 2, 3).reshape(nkv, -1, hd)[:, :held]
        vv = s["v_pages"][mine].double().permute(1, 0, 3, 2).reshape(nkv, -1, hd)[:, :held]
        for r in range(0, span[b], 512):                                                      # a few rows at a time: scores of 64 bits are large
            rows = slice(off[b] + r, off[b] + min(r + 512, span[b]))
            p = torch.arange(pos0[b] + r, pos0[b] + min(r + 512, span[b]), device="cuda")[:, None]
            j = torch.arange(held, device="cuda")[None]
            hide = (j > p) | (j <= p - (case["window"] or 1 << 40))
            for h in range(nq):
                x = s["q"][rows, h].double() @ kk[h // (nq // nkv)].T * hd ** -0.5
                x[hide] = -math.inf
                z = torch.logsumexp(x, -1)
                lse[rows, h] = z
                out[rows, h] = torch.exp(x - z[:, None]) @ vv[h // (nq // nkv)]
    return {"out": out, "lse": lse}
