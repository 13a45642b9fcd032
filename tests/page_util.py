"""The paged cache in plain form, in 64 bits on the CPU, from its definition in include/gear.h: layout, quantizer, attention, and how
far an implementation in the declared precisions may be off."""
import math

import torch

D = 128
DTYPES = (torch.float16, torch.bfloat16)


def to_type(x, dtype):
    """float64 values rounded to the type, once: through fp32 only where that is exact or rounds to the same side (torch's own way goes
    through fp32: a value within half an fp32 step of a tie would be rounded twice)."""
    y = x.to(torch.float32)
    # round to odd: an inexact fp32 value gets its last bit set, so that the second rounding sees on which side it was
    bits = y.view(torch.int32)
    inexact = y.double() != x
    toward = (y.double().abs() > x.abs()) & inexact               # rounded away: the truncated neighbour
    bits = torch.where(toward, bits - 1, bits)
    bits = torch.where(inexact & torch.isfinite(y), bits | 1, bits)
    return bits.view(torch.float32).to(dtype)


def quantise(x, bits, group, dtype):
    """(codes, scale, zero) of rows [..., 128] (any float type): codes [..., 128] int64, the others [..., 128 / group] of the type."""
    x = x.double().unflatten(-1, (D // group, group))
    zero, top = x.amin(-1), x.amax(-1)
    # the scale is defined through fp32: a difference and a quotient, each rounded
    scale = ((top - zero).float() / torch.tensor(float(2 ** bits - 1))).to(dtype)
    s = scale.double()
    code = torch.where(s[..., None] > 0, (x - zero[..., None]) / torch.where(s > 0, s, 1.0)[..., None], 0.0).round().clamp(0, 2 ** bits - 1)
    return code.flatten(-2).long(), scale, zero.to(dtype)


def stored_values(code, scale, zero, group, dtype):
    s, z = (t.double().repeat_interleave(group, -1) for t in (scale, zero))
    return to_type(code.double() * s + z, dtype)


def expected(x, bits, group, dtype):
    """What rows read back as."""
    return x if bits == 16 else stored_values(*quantise(x, bits, group, dtype), group, dtype)


def block_bytes(bits, group, page):
    return page * (D * bits // 8 + (0 if bits == 16 else 4 * D // group))


def pack(x, bits, group, dtype):
    """Block bytes [..., bytes] of rows [..., page, 128]."""
    page = x.shape[-2]
    if bits == 16:
        return x.contiguous().view(torch.uint8).reshape(*x.shape[:-2], -1)
    code, scale, zero = quantise(x, bits, group, dtype)
    if bits == 8:
        rows = code.to(torch.uint8)
    else:
        word = sum(code[..., e::8] << (4 * (e // 2) + 16 * (e % 2)) for e in range(8))            # [..., page, 16]
        rows = torch.stack([(word >> (8 * k)) & 255 for k in range(4)], -1).to(torch.uint8)
    words = torch.stack((scale, zero), -1).transpose(-3, -2).contiguous().view(torch.uint8)        # [..., G, page, 4]
    lead = x.shape[:-2]
    return torch.cat((rows.reshape(*lead, -1), words.reshape(*lead, -1)), -1)


def unpack(blocks, bits, group, dtype, page):
    """Rows [..., page, 128] that blocks [..., bytes] hold, as values of the type."""
    rb = D * bits // 8
    rows = blocks[..., :page * rb].reshape(*blocks.shape[:-1], page, rb).contiguous()
    if bits == 16:
        return rows.view(dtype)
    if bits == 4:
        by = rows.long()
        word = by[..., 0::4] | by[..., 1::4] << 8 | by[..., 2::4] << 16 | by[..., 3::4] << 24
        rows = torch.stack([(word >> (4 * (e // 2) + 16 * (e % 2))) & 15 for e in range(8)], -1).flatten(-2)
    words = blocks[..., page * rb:].contiguous().view(dtype).reshape(*blocks.shape[:-1], D // group, page, 2).transpose(-3, -2)
    return stored_values(rows.long(), words[..., 0], words[..., 1], group, dtype)


def attend(q, K, V, q_start, kv_len, table, scale, causal):
    """(out, bound) in 64 bits: q [T, H_q, 128]; K, V [pages, H, page, 128] the pool's values; lists of ints.  Rows outside every sequence
    are NaN in both.  bound: how far an output of the declared precisions may be from out."""
    T, Hq, _ = q.shape
    n_pages, H, page, _ = K.shape
    gq, dtype = Hq // H, q.dtype
    eps = torch.finfo(dtype).eps / 2
    out = torch.full((T, Hq, D), math.nan, dtype=torch.float64)
    bound = torch.full((T, Hq, D), math.nan, dtype=torch.float64)
    for s in range(len(kv_len)):
        q0, q1 = q_start[s], q_start[s + 1]
        n, kv = q1 - q0, max(0, min(kv_len[s], len(table[s]) * page))
        if n <= 0:
            continue
        pos = torch.arange(kv)
        pages = torch.tensor([table[s][p // page] for p in range(kv)], dtype=torch.long)
        there = (pages >= 0) & (pages < n_pages)
        at = torch.where(there, pages, 0)
        k, v = (torch.where(there[:, None, None], X[at, :, pos % page].double(), 0.0) for X in (K, V))   # [kv, H, 128]
        last = torch.full((n,), kv) if not causal else (kv - n + 1 + torch.arange(n))
        ban = ~there[None, :] | (pos[None, :] >= last[:, None])                                          # [n, kv]
        for j in range(Hq):
            qq, kk, vv = q[q0:q1, j].double(), k[:, j // gq], v[:, j // gq]
            # (what no row sees may be anything)
            kk, vv = (torch.where(ban.all(0)[:, None], 0.0, t) for t in (kk, vv))
            sc = (qq @ kk.t() * scale).masked_fill(ban, -math.inf)
            top = sc.amax(-1, keepdim=True) if kv else torch.full((n, 1), -math.inf, dtype=torch.float64)
            w = torch.where(ban, 0.0, torch.exp(sc - torch.where(torch.isfinite(top), top, 0.0)))
            l = w.sum(-1, keepdim=True)
            p = torch.where(l > 0, w / torch.where(l > 0, l, 1.0), 0.0)
            o, A = p @ vv, p @ vv.abs()
            # scores: 128 products summed in fp32, times the scale (two roundings), and the exponent's argument; a score off by x changes a weight
            # and the sum by x each
            ds = (abs(scale) * (qq.abs() @ kk.abs().t()) * 136 * 2.0 ** -24).masked_fill(ban, 0.0).amax(-1, keepdim=True) if kv else 0.0
            # weights: rounded to the type for the product (relative eps; half the last subnormal step of fp16, against a sum of at least 1),
            # exp2 and the sums of kv terms in fp32
            rel = eps + 2 * ds + (kv + 64) * 2.0 ** -23
            tiny = (kv * 2.0 ** -25 if dtype == torch.float16 else 0.0) * (vv.abs().amax(0) if kv else 0.0)
            b = A * rel + tiny
            out[q0:q1, j], bound[q0:q1, j] = o, b + eps * (o.abs() + b) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    return out, bound


def sink_and_tail(K, V, q, table, kv, page):
    """In place: the first 256 of kv tokens hold a Key in every 32nd (one for each wave of a block) whose weight is 2^26 times that of all others, and
    no Value; the others' Values are about 1.  Returns the scale."""
    K[:], q[:] = 0.0, 1.0
    V[:] = 0.5 + V.abs().clamp(max=1.0)
    for i in range(0, 256, 32):
        p, r = int(table[i // page]), i % page
        K[p, :, r], V[p, :, r] = 1.0, 0.0
    assert kv > 256
    return 26 * math.log(2.0) / 128


def tail_bound(q, K, V, table, kv, q0, q1, scale, page):
    """(out, bound) of one sequence and head in fp16.  A weight is rounded to fp16, half a step 2^-11 of it or, of a subnormal number, 2^-25; the numbers
    are weights times a power of two that brings a row's greatest to 2^7 at least, so that is 2^-32 of the greatest: of less than the sum."""
    at = torch.arange(kv)
    k, v = (X[torch.tensor(table)[at // page].long(), 0, at % page].double() for X in (K, V))
    sc = q[q0:q1, 0].double() @ k.t() * scale
    sc = sc.masked_fill(at[None] >= (kv - (q1 - q0) + 1 + torch.arange(q1 - q0))[:, None], -math.inf)
    p = torch.softmax(sc, -1)
    o = p @ v
    # fp32: a score of at most 18 (its products are exact), the exponent's argument and exp2, sums of kv terms
    b = o * (2.0 ** -11 + (kv + 64 + 18) * 2.0 ** -23) + kv * 2.0 ** -32 * v.amax()
    return o, b + (o + b) * 2.0 ** -11 + 2.0 ** -25


def quantise_fp32(x, bits, group, dtype):
    """(codes, scale, zero) as include/gear.h states them, in its own arithmetic: the difference and the quotient in fp32.  (Against quantise above: where the
    difference is not exact in fp32 and rounds to a half of the scale.)"""
    x = x.float().unflatten(-1, (D // group, group))
    zero, top = x.amin(-1), x.amax(-1)
    scale = ((top - zero) / torch.tensor(float(2 ** bits - 1))).to(dtype).float()
    code = torch.where(scale[..., None] > 0, (x - zero[..., None]) / torch.where(scale > 0, scale, 1.0)[..., None], 0.0).round().clamp(0, 2 ** bits - 1)
    return code.flatten(-2).long(), scale.to(dtype), zero.to(dtype)


def values_fp32(code, scale, zero, group, dtype):
    """What codes stand for as include/gear.h states it: rounded once in fp16, to fp32 first in bf16."""
    if dtype == torch.float16:
        return stored_values(code, scale, zero, group, dtype)
    s, z = (t.float().repeat_interleave(group, -1) for t in (scale, zero))
    return (code.float() * s + z).to(dtype)                  # (the product is exact)


def block_of_codes(code, scale, zero, bits):
    """Block bytes [..., bytes] of codes [..., page, 128] and their words."""
    if bits == 8:
        rows = code.to(torch.uint8)
    else:
        word = sum(code[..., e::8] << (4 * (e // 2) + 16 * (e % 2)) for e in range(8))
        rows = torch.stack([(word >> (8 * k)) & 255 for k in range(4)], -1).to(torch.uint8)
    words = torch.stack((scale, zero), -1).transpose(-3, -2).contiguous().view(torch.uint8)
    lead = code.shape[:-2]
    return torch.cat((rows.reshape(*lead, -1), words.reshape(*lead, -1)), -1)


def rows_at_ties(bits, dtype):
    """Rows [n, 128] (every group of 32 alike) whose differences from their least value are halves of the scale but for less than fp32 holds, and the codes that the
    difference rounded to fp32 gives them; the exact ones differ."""
    levels, tiny = 2 ** bits - 1, 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -40
    rows, codes = [], []
    for s in (1.0, 0.5, 2.0):
        # the least value next to nothing: (k + 1/2) s above or below a half, which go to the even side alike
        for sign in (-1, 1):
            for k in range(2, 12):
                if (k % 2 == 0) == (sign < 0):               # rounded to even is the other side
                    rows.append([sign * tiny, levels * s, (k + 0.5) * s] + [s] * 29)
                    codes.append((k if k % 2 == 0 else k + 1, k + 1 if k % 2 == 0 else k))
        # a value next to nothing, the least one halves of the scale
        if bits == 4 or dtype == torch.float16:              # (a bf16 number has eight bits: levels - k - 1/2 needs nine)
            for k in (2, 4):
                rows.append([-(k + 0.5) * s, (levels - k - 0.5) * s, tiny] + [s * 0.5] * 29)
                codes.append((k, k + 1))
    x = torch.tensor(rows, dtype=torch.float64).repeat(1, 4).to(dtype)
    return x, codes
