"""Caches in pages in 64 bits: what the GPU tests compare with, and how far fp32 arithmetic may be from it (not a test module)."""
import math

import torch

F32, BF16 = 2.0 ** -24, 2.0 ** -8                # half a step, relative to the value


def half_step(dtype):
    return F32 if dtype == torch.float32 else BF16


def turned(x, pos, freq, amplitude=1.0, interleaved=False, inverse=False):
    """x [rows, heads, channels] rotated to pos, in 64 bits, and a bound on an fp32 rotation's error.  Error: the reduced angle is rounded to fp32 and
    sine and cosine are good to 2 ulp of at most 1 (3 x 2^-23 in all, and 2^-24 for the amplitude's product), each of the two products and their sum are rounded."""
    rot = 2 * freq.numel()
    x = x.double()
    a = pos.double()[:, None, None] * freq
    c, s = a.cos() * amplitude, a.sin() * (-amplitude if inverse else amplitude)
    p, q = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, err = x.clone(), torch.zeros_like(x)
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., first], y[..., second] = p * c - q * s, q * c + p * s
    err[..., first] = err[..., second] = (p.abs() + q.abs()) * abs(amplitude) * (3 * 2.0 ** -23 + 3 * F32)
    return y, err


def close(got, want, err, what=""):
    """got, rounded once to its type, against want, whose fp32 computation may be err off."""
    h = half_step(got.dtype)
    off = (got.double() - want).abs() - (err * (1 + h) + want.abs() * h + 1e-37)
    assert bool((off <= 0).all()), f"{what}: {float(off.max())} beyond the bound, at {off.argmax().item()} of {tuple(off.shape)}"


class Pages:
    """A cache in pages, its page table and the spans of a call, made from a seed on the CPU and moved to the GPU."""

    def __init__(self, spans, pos0, n_kv, hd, page, seed=0, spare_pages=2, spare_slots=1, fill=None):
        g = torch.Generator().manual_seed(seed)
        n = len(spans)
        need = [(p + m + page - 1) // page for m, p in zip(spans, pos0)]
        total, longest = sum(need) + spare_pages, max(max(need), 1)
        order = torch.randperm(total, generator=g).tolist()
        self.slot = torch.randperm(n + spare_slots, generator=g)[:n].to(torch.int32)
        table = torch.full((n + spare_slots, longest), -1, dtype=torch.int32)
        at = 0
        for b in range(n):
            table[self.slot[b], :need[b]] = torch.tensor(order[at:at + need[b]], dtype=torch.int32)
            at += need[b]
        self.spans, self.pos0, self.page, self.n_kv, self.hd, self.n = spans, pos0, page, n_kv, hd, n
        self.k = torch.randn(total, n_kv, page, hd, generator=g).to(torch.bfloat16)
        self.v = torch.randn(total, n_kv, hd, page, generator=g).to(torch.bfloat16)
        if fill is not None:                                             # whatever no sequence holds
            held = torch.zeros(total, page, dtype=torch.bool)
            for b in range(n):
                for j in range(pos0[b] + spans[b]):
                    held[table[self.slot[b], j // page], j % page] = True
            self.k.masked_fill_(~held[:, None, :, None], fill)
            self.v.masked_fill_(~held[:, None, None, :], fill)
        self.table = table
        off = [0]
        for m in spans:
            off.append(off[-1] + m)
        self.off = torch.tensor(off, dtype=torch.int32)
        self.rows = off[-1]
        self.gen = g

    def gpu(self):
        import paper_2507_17307_amd as P
        self.dk, self.dv, self.dtable = self.k.cuda(), self.v.cuda(), self.table.cuda()
        self.dslot, self.doff, self.dpos = self.slot.cuda(), self.off.cuda(), torch.tensor(self.pos0, dtype=torch.int32).cuda()
        self.cache = P.PagedCache(self.dk, self.dv, self.dtable)
        return self

    def held(self, b, k=None, v=None):
        """(K [positions, KV heads, channels], V likewise) of sequence b."""
        k, v = self.k if k is None else k, self.v if v is None else v
        end = self.pos0[b] + self.spans[b]
        pages = self.table[self.slot[b].long(), :(end + self.page - 1) // self.page].long()
        return (k[pages].permute(0, 2, 1, 3).reshape(-1, self.n_kv, self.hd)[:end], v[pages].permute(0, 3, 1, 2).reshape(-1, self.n_kv, self.hd)[:end])


def attention(pg, q, scale, window=0):
    """(out, lse, bound on out's error, bound on lse's) in 64 bits: q [rows, query heads, channels].
    A score is a sum of hd products in fp32, hd + 4 roundings of at most sum |q k|, and its place in the exponent is rounded twice; a probability
    has that error times e and 2^-22 of the hardware's exponential and, where q is bf16, a rounding to bf16; sums of n add n roundings, the products with v the same."""
    nq, hd = q.shape[1], q.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse, e_out, e_lse = torch.zeros(q.shape[:2], dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    r = 0
    for b, (m, p0) in enumerate(zip(pg.spans, pg.pos0)):
        if m == 0:
            continue
        k, v = (t.double().repeat_interleave(nq // pg.n_kv, 1).transpose(0, 1) for t in pg.held(b))           # [heads, positions, channels]
        x = q[r:r + m].double().transpose(0, 1)                                                                # [heads, rows, channels]
        j, p = torch.arange(p0 + m), torch.arange(p0, p0 + m)[:, None]
        hide = (j > p) | (j <= p - (window if window else 1 << 40))
        # (a NaN that a row does not see must not reach it in this computation either)
        kc, vc = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
        s = (x @ kc.transpose(1, 2)) * scale
        mag = (x.abs() @ kc.abs().transpose(1, 2)) * scale
        seen_bad = ((~torch.isfinite(k)).any(2)[:, None, :] & ~hide).any(2)
        s = s.masked_fill(hide, -math.inf)
        z = torch.logsumexp(s, -1)
        w = torch.exp(s - z[..., None])
        o = w @ vc
        ds = ((hd + 4) * F32 * mag + 4 * F32 * (s.abs() + z[..., None].abs())).masked_fill(hide, 0).amax(-1)
        n = torch.full_like(ds, 1) * (~hide).sum(-1)
        rel = 2.1 * ds + 2 * n * F32 + 2.0 ** -20 + (BF16 if q.dtype == torch.bfloat16 else 0.0)
        eo = rel[..., None] * (w @ vc.abs())
        for sign in (math.inf, -math.inf, math.nan):                                                           # what a row does see reaches it
            has = torch.isnan(v) if math.isnan(sign) else v == sign
            hit = (~hide).double() @ has.double()
            o = torch.where(hit > 0, o + sign, o)
        o = torch.where(seen_bad[..., None], math.nan, o)
        out[r:r + m], lse[r:r + m] = o.transpose(0, 1), torch.where(seen_bad, math.nan, z).transpose(0, 1)
        e_out[r:r + m], e_lse[r:r + m] = eo.transpose(0, 1), (2.1 * ds + 2 * n * F32 + 2.0 ** -20).transpose(0, 1)
        r += m
    return out, lse, e_out, e_lse
