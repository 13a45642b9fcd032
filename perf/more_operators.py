"""What surrounds the paged cache's reads and writes in a server's step, as timed cases.

Six kinds of pass:

  append   a step's or a prompt's queries and Keys turned by their positions; the Keys and Values put into their slots
  rotate   rows of a tensor turned back by their positions (Keys that are to stand somewhere else)
  step     slots for the next tokens of a list of sequences, taken from the free pages, and the tokens dropped again
  fork     rows of the page table that share a prompt, their next tokens (a shared, partly filled page is copied), and the rows freed
  compact  the pages in use moved to the front of the pool
  attn     the queries of a batch whose sequences share their first pages in groups

A pool's page holds, per KV head, the Key rows, their (scale, zero) words, the Value rows, their words.  A row of b-bit codes holds
128 b / 8 bytes (8 bits: channel c in byte c; 4 bits: channel 8 w + e in word w at bits 4 (e / 2) + 16 (e % 2)); the words lie as
[128 / group][page], scale in the low half.  16 bits: the rows alone.  A page table has a row of page numbers per sequence, -1 where
there is none; refs counts the entries that name a page.
"""
import math
import random

import torch

own = False

D = 128
DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _named(name, c):
    return dict(c, name=name) if name else c


def _append(name, dtype, bits, group, page, H_kv, gq, seqs, n, rot, interleaved, scaled, pos_hi, fused, salt=0):
    """n new tokens of each sequence, behind up to pos_hi others; rot of the 128 channels turn."""
    return _named(name, dict(kind="append", dtype=dtype, bits=bits, group=group, page=page, H_kv=H_kv, gq=gq, seqs=seqs, n=n, rot=rot,
                             interleaved=interleaved, scaled=scaled, pos_hi=pos_hi, fused=fused, salt=salt))


def _rotate(name, dtype, heads, seqs, n, rot, interleaved, scaled, pos_hi, heads_first, salt=0):
    return _named(name, dict(kind="rotate", dtype=dtype, heads=heads, seqs=seqs, n=n, rot=rot, interleaved=interleaved, scaled=scaled,
                             pos_hi=pos_hi, heads_first=heads_first, salt=salt))


def _step(name, page, seqs, n, kv_lo, kv_hi, others, free, salt=0):
    """seqs sequences of kv_lo..kv_hi tokens get n more, beside `others` of 500..1000 that get none; there are `free` times the needed pages, and those."""
    return _named(name, dict(kind="step", page=page, seqs=seqs, n=n, kv_lo=kv_lo, kv_hi=kv_hi, others=others, free=free, salt=salt))


def _fork(name, dtype, page, H_kv, prompts, rows, n, kv_lo, kv_hi, pools, salt=0):
    """rows copies of prompts of kv_lo..kv_hi tokens, n new tokens each, in the pools of `pools` layers."""
    return _named(name, dict(kind="fork", dtype=dtype, page=page, H_kv=H_kv, prompts=prompts, rows=rows, n=n, kv_lo=kv_lo, kv_hi=kv_hi, pools=pools, salt=salt))


def _compact(name, dtype, page, H_kv, seqs, kv_lo, kv_hi, live, salt=0):
    """Pages of seqs sequences scattered over a pool, `live` of whose pages are in use."""
    return _named(name, dict(kind="compact", dtype=dtype, page=page, H_kv=H_kv, seqs=seqs, kv_lo=kv_lo, kv_hi=kv_hi, live=live, salt=salt))


def _attn(name, dtype, bits, group, page, H_kv, gq, groups, seqs, pre_lo, pre_hi, own_lo, own_hi, q_lo, q_hi, salt=0):
    """seqs sequences in groups that share their first pre_lo..pre_hi tokens and have own_lo..own_hi more, q_lo..q_hi new ones among them."""
    return _named(name, dict(kind="attn", dtype=dtype, bits=bits, group=group, page=page, H_kv=H_kv, gq=gq, groups=groups, seqs=seqs, pre_lo=pre_lo,
                             pre_hi=pre_hi, own_lo=own_lo, own_hi=own_hi, q_lo=q_lo, q_hi=q_hi, salt=salt))


def listed():
    return [
        # one token of each of 16 sequences on a LLaMA-2-7B layer, out of the fused projection's output: latency counts
        _append("append_step_7b_b16", "f16", 16, 128, 16, 32, 1, 16, 1, 128, False, False, 4096, True),
        # four prompts of 8192 tokens on a Llama-3-8B layer, frequencies scaled for long contexts: the largest write
        _append("append_gqa_b4_8k", "bf16", 16, 128, 64, 8, 4, 4, 8192, 128, False, True, 0, True),
        # an odd batch of odd length, half of the channels in neighbouring pairs, 8-bit pages, far positions
        _append("append_part_b7_1777_8bit", "f16", 8, 64, 32, 40, 1, 7, 1777, 64, True, False, 1 << 20, False),
        # the Keys of 16 sequences of 4096 tokens on a 32-head layer, brought back head by head, to be put at other positions
        _rotate("rotate_back_7b_b16_4k", "f16", 32, 16, 4096, 128, False, False, 4096, True),
        # a decode step's bookkeeping for 64 sequences of about 8192 tokens
        _step("step_b64_8k", 16, 64, 1, 7000, 8192, 0, 1.0),
        # 32 prompts come in at once beside 100 sequences that are being decoded
        _step("step_prompts_b32_8k", 16, 32, 8192, 0, 0, 100, 2.0),
        # 16 samples of one prompt of 4097 tokens and more, four layers whose pools lie one behind the other
        _fork("fork_b16_4k", "f16", 16, 32, 1, 16, 1, 4097, 4097, 4),
        # a pool of a grouped-query layer, half of whose pages are free, in no order
        _compact("compact_gqa_b64", "bf16", 64, 8, 64, 2000, 8192, 0.5),
        # one token of each of 16 samples of one prompt on a LLaMA-2-7B layer: the smallest read
        _attn("shared_7b_b16_2k", "f16", 16, 128, 16, 32, 1, 1, 16, 2077, 2077, 1, 64, 1, 1),
        # a Llama-3-8B layer, 64 sequences behind one system prompt of 8192 tokens
        _attn("shared_gqa_b64_8k", "bf16", 16, 128, 64, 8, 4, 1, 64, 8192, 8192, 100, 1000, 1, 1),
        # five groups of unequal size and length, 8-bit pages
        _attn("shared_groups5_b48_8bit", "f16", 8, 64, 16, 8, 4, 5, 48, 1500, 6001, 33, 700, 1, 1),
        # questions of 20 to 60 tokens about one document
        _attn("questions_gqa_b16_6k", "bf16", 16, 128, 64, 8, 4, 1, 16, 6100, 6100, 20, 60, 20, 60),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "append", "rotate", "step", "fork", "compact", "attn", "attn", "attn", "attn"))
    dtype = rng.choice(("f16", "bf16"))
    page = rng.choice((16, 16, 32, 64, 128))
    H_kv, gq = rng.choice(((32, 1), (40, 1), (8, 4), (8, 4), (8, 8), (4, 8), (16, 2), (7, 2)))
    rot, interleaved, scaled = rng.choice((128, 128, 128, 64, 96, 50)), rng.random() < 0.4, rng.random() < 0.4
    salt = rng.randrange(1 << 20)
    if kind in ("append", "rotate"):
        n = _log(rng, 1, 8192)
        seqs = _log(rng, 1, max(1, min(64, 1200000 // (H_kv * (gq + 2) * n))))
        pos_hi = _log(rng, 1, 1 << 22)
        if kind == "rotate":
            return _rotate(None, dtype, H_kv * gq, seqs, n, rot, interleaved, scaled, pos_hi, rng.random() < 0.5, salt)
        bits, group = rng.choice(((16, 128), (16, 128), (8, 128), (8, 64), (8, 32)))
        return _append(None, dtype, bits, group, page, H_kv, gq, seqs, n, rot, interleaved, scaled, pos_hi, rng.random() < 0.5, salt)
    if kind == "step":
        seqs = _log(rng, 1, 1000)
        n = 1 if rng.random() < 0.5 else _log(rng, 1, max(1, min(8192, 260000 // seqs)))
        kv = _log(rng, 1, max(1, min(8192, 1000000 // seqs)))
        return _step(None, page, seqs, n, kv // 2, kv, rng.randint(20, 100), rng.choice((1.0, 2.0, 20.0)), salt)
    if kind == "fork":
        rows = _log(rng, 1, 64)
        H_kv, prompts = rng.choice((8, 32, 7)), rng.randint(1, max(1, rows // 3))
        kv = _log(rng, 1, max(1, min(8192, 400000 // (H_kv * prompts))))
        return _fork(None, dtype, page, H_kv, prompts, rows, rng.choice((1, 1, 5, 100)), max(1, kv // 2), kv, rng.randint(1, 4), salt)
    if kind == "compact":
        seqs = _log(rng, 1, 64)
        kv = _log(rng, 20, max(20, min(8192, 300000 // seqs)))
        return _compact(None, dtype, page, 8, seqs, kv // 2, kv, rng.uniform(0.3, 0.95), salt)
    bits, group = rng.choice(((16, 128), (16, 128), (8, 128), (8, 64), (8, 32), (4, 64), (4, 32)))
    seqs = _log(rng, 2, 64)
    # at most 64 sequences of 9000 tokens of 8 KV heads and 256 columns each
    pre = _log(rng, 100, max(100, min(16384, 4000000 // (H_kv * seqs))))
    rest = _log(rng, 1, 1000)
    form = rng.choice(("one", "one", "few", "question"))
    q = 1 if form == "one" else rng.randint(2, 8) if form == "few" else _log(rng, 9, 64)
    q = max(1, min(q, 120000000 // (H_kv * gq * seqs * pre)))   # (the operations of the listed questions)
    return _attn(None, dtype, bits, group, page, H_kv, gq, rng.randint(1, max(1, min(6, seqs // 2))), seqs, int(pre * rng.uniform(0.3, 1.0)), pre,
                 max(q, rest // 3), max(q, rest), 1 if form == "one" else max(1, q // 2), q, salt)


# ---- what a case fixes, so that every seed is the same work
def _starts(c):
    """The position of every sequence's first new token."""
    r = random.Random(c["salt"])
    return [r.randint(0, c["pos_hi"]) for _ in range(c["seqs"])]


def _frequencies(c):
    """Radians per position of each pair: base 10000 (500000 where they are scaled for eight times the trained length of 8192: the pairs
    that turn less than once there by an eighth of their angle, those that turn more than four times by all of it)."""
    f = (500000.0 if c["scaled"] else 10000.0) ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
    if c["scaled"]:
        keep = ((8192 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / 8.0)
    return f


def _lengths(c, lo, hi, count):
    r = random.Random(c["salt"] + 1)
    return [r.randint(lo, hi) for _ in range(count)]


def _groups(c):
    """(first sequence of every group and the end, shared tokens of every group, tokens, new tokens of every sequence)."""
    r = random.Random(c["salt"])
    cuts = sorted(r.sample(range(1, c["seqs"]), c["groups"] - 1)) if c["groups"] > 1 else []
    first = [0] + cuts + [c["seqs"]]
    prefix = [r.randint(c["pre_lo"], c["pre_hi"]) for _ in range(c["groups"])]
    kv, q = [], []
    for g in range(c["groups"]):
        for _ in range(first[g], first[g + 1]):
            q.append(r.randint(c["q_lo"], c["q_hi"]))
            kv.append(prefix[g] + max(q[-1], r.randint(c["own_lo"], c["own_hi"])))
    return first, prefix, kv, q


# ---- the pool's formats
def _row_bytes(c):
    return D * c["bits"] // 8


def _block_bytes(c):
    return c["page"] * (_row_bytes(c) + (0 if c["bits"] == 16 else 4 * D // c["group"]))


def _quantise(c, x):
    """Codes and (scale, zero) of rows [..., 128]: the decisions in 64 bits."""
    dt, g = TYPES[c["dtype"]], c["group"]
    x = x.double().unflatten(-1, (D // g, g))
    zero, most = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((most - zero) / (2 ** c["bits"] - 1)).to(dt).double()
    code = ((x - zero) / torch.where(scale > 0, scale, 1.0)).round().clamp(0, 2 ** c["bits"] - 1)
    return torch.where(scale > 0, code, 0.0), scale, zero


def _values(c, code, scale, zero):
    """What codes [..., 128 / g, g] stand for: scale * code + zero, rounded to the cache's type."""
    return (code.float() * scale.float() + zero.float()).to(TYPES[c["dtype"]]).flatten(-2)


def _pack(c, x):
    """Blocks of pages [n, bytes] from rows [n, page, 128]."""
    if c["bits"] == 16:
        return x.contiguous().view(torch.uint8).flatten(1)
    code, scale, zero = _quantise(c, x)
    code = code.flatten(-2)
    if c["bits"] == 8:
        rows = code.to(torch.uint8)
    else:
        shifts = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], dtype=torch.int32, device=DEVICE)
        rows = (code.to(torch.int32).unflatten(-1, (D // 8, 8)) << shifts).sum(-1).to(torch.int32).view(torch.uint8)
    words = torch.cat((scale, zero), -1).to(TYPES[c["dtype"]])                    # [n, page, 128 / g, 2]
    words = words.transpose(1, 2).contiguous().view(torch.uint8)
    return torch.cat((rows.reshape(x.shape[0], -1), words.reshape(x.shape[0], -1)), 1)


def _unpack(c, blocks):
    """Rows [..., page, 128] in 32 bits from blocks of pages [..., bytes]."""
    dt, rb, page = TYPES[c["dtype"]], _row_bytes(c), c["page"]
    rows = blocks[..., :page * rb].unflatten(-1, (page, rb)).contiguous()
    if c["bits"] == 16:
        return rows.view(dt).float()
    if c["bits"] == 4:
        shifts = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], dtype=torch.int32, device=DEVICE)
        rows = ((rows.view(torch.int32).unsqueeze(-1) >> shifts) & 15).flatten(-2)
    words = blocks[..., page * rb:].contiguous().view(dt).unflatten(-1, (D // c["group"], page, 2)).transpose(-3, -2)
    return _values(c, rows.unflatten(-1, (D // c["group"], c["group"])), words[..., :1], words[..., 1:]).float()


# ---- inputs
def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _rows(gen, shape, dt, few_large):
    """N(0, 1) rows [..., heads, 128], with a few channels of large magnitude per head (Keys) or heavy-tailed ones (Values)."""
    x = torch.randn(shape, generator=gen, device=DEVICE)
    if few_large:
        sig = torch.ones(shape[-2], D, device=DEVICE)
        at = torch.rand(shape[-2], D, generator=gen, device=DEVICE).argsort(dim=1)[:, :4]
        x = x * sig.scatter_(1, at, 10.0 + 10.0 * torch.rand(shape[-2], 4, generator=gen, device=DEVICE))
    else:
        x = x * (0.5 + x.abs() * 0.3)
    return x.to(dt)


def _prepare_append(c, gen):
    dt, S, n, H, gq, page = TYPES[c["dtype"]], c["seqs"], c["n"], c["H_kv"], c["gq"], c["page"]
    start = torch.tensor(_starts(c), device=DEVICE)
    s = {"case": c, "positions": start[:, None] + torch.arange(n, device=DEVICE), "freq": _frequencies(c).to(DEVICE)}
    width = -(-(n + page - 1) // page)
    s["n_pages"] = S * width + 3
    table = torch.randperm(s["n_pages"], generator=gen, device=DEVICE)[:S * width].view(S, width)
    at = (start % page)[:, None] + torch.arange(n, device=DEVICE)
    s["slots"] = (table.gather(1, at // page) * page + at % page).contiguous()
    s["pool"] = torch.zeros(s["n_pages"] * H * 2 * _block_bytes(c), dtype=torch.uint8, device=DEVICE)
    qkv = torch.empty(S, n, H * (gq + 2), D, dtype=dt, device=DEVICE)      # the projection's rows: query heads, Keys, Values
    s["q"], s["K"], s["V"] = qkv[:, :, :H * gq], qkv[:, :, H * gq:H * (gq + 1)], qkv[:, :, H * (gq + 1):]
    if not c["fused"]:
        s["q"], s["K"], s["V"] = (x.contiguous() for x in (s["q"], s["K"], s["V"]))
    for i in range(S):
        s["q"][i] = torch.randn(n, H * gq, D, generator=gen, device=DEVICE).to(dt)
        s["K"][i], s["V"][i] = _rows(gen, (n, H, D), dt, True), _rows(gen, (n, H, D), dt, False)
    return s


def _prepare_rotate(c, gen):
    dt, S, n, H = TYPES[c["dtype"]], c["seqs"], c["n"], c["heads"]
    s = {"case": c, "positions": torch.tensor(_starts(c), device=DEVICE)[:, None] + torch.arange(n, device=DEVICE), "freq": _frequencies(c).to(DEVICE)}
    x = torch.empty((S, H, n, D) if c["heads_first"] else (S, n, H, D), dtype=dt, device=DEVICE)
    s["x"] = x.transpose(1, 2) if c["heads_first"] else x                  # [S, n, heads, 128]
    for i in range(S):
        s["x"][i] = _rows(gen, (n, H, D), dt, True)
    return s


def _table(c, gen, lengths, n_rows, width, n_pages):
    """A page table whose first rows hold pages for so many tokens, drawn without order."""
    page = c["page"]
    pages = -(-torch.tensor(lengths) // page)
    entry = torch.arange(width)
    held = entry[None, :] < torch.cat((pages, torch.zeros(n_rows - len(lengths), dtype=torch.long)))[:, None]
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    rank = (held.flatten().cumsum(0) - 1).clamp(min=0).to(DEVICE)
    table = torch.where(held.flatten().to(DEVICE), order[rank], -1).view(n_rows, width).contiguous()
    kv_len = _int(list(lengths) + [0] * (n_rows - len(lengths)))
    return {"case": c, "table": table, "kv_len": kv_len, "refs": _count(table, n_pages), "n_pages": n_pages}


def _count(table, n_pages):
    named = torch.where(table >= 0, table, n_pages).flatten().long()
    return torch.zeros(n_pages + 1, dtype=torch.int32, device=DEVICE).scatter_add_(0, named, torch.ones_like(named, dtype=torch.int32))[:n_pages].contiguous()


def _pool(c, gen, shape):
    """Pages [*shape, words] of 16-bit rows as numbers of the pool's type."""
    x = torch.empty(*shape, c["H_kv"] * 2 * c["page"] * D, dtype=TYPES[c["dtype"]], device=DEVICE)
    return x.normal_(generator=gen)


def _prepare_step(c, gen):
    page, S, n = c["page"], c["seqs"], c["n"]
    kv, others = _lengths(c, c["kv_lo"], c["kv_hi"], S), _lengths(c, 500, 1000, c["others"])
    used, needed = sum(-(-k // page) for k in kv + others), sum(-(-(k + n) // page) - -(-k // page) for k in kv)
    s = _table(c, gen, kv + others, S + c["others"], max(-(-(k + n) // page) for k in kv + others) + 1, used + int(c["free"] * max(needed, used // 8)) + needed)
    s["rows"] = torch.randperm(S, generator=gen, device=DEVICE).to(torch.int32)
    s["counts"] = torch.full((S,), n, dtype=torch.int32, device=DEVICE)
    s["keep"] = s["kv_len"][s["rows"].long()].contiguous()
    return s


def _prepare_fork(c, gen):
    page, P, R, n = c["page"], c["prompts"], c["rows"], c["n"]
    kv = _lengths(c, c["kv_lo"], c["kv_hi"], P)
    used = sum(-(-k // page) for k in kv)
    s = _table(c, gen, kv, P + R, -(-(max(kv) + n) // page) + 1, used + R * (-(-n // page) + 2) + 5)
    s["src"], s["dst"] = _int([i % P for i in range(R)]), _int([P + i for i in range(R)])
    s["counts"], s["keep"] = _int([n] * R), _int([0] * R)
    s["pool"] = _pool(c, gen, (c["pools"], s["n_pages"]))
    return s


def _prepare_compact(c, gen):
    kv = _lengths(c, max(1, c["kv_lo"]), c["kv_hi"], c["seqs"])
    used = sum(-(-k // c["page"]) for k in kv)
    s = _table(c, gen, kv, c["seqs"], -(-max(kv) // c["page"]), int(used / c["live"]) + 1)
    # every second sequence shares the first quarter of its pages with the one before
    t = s["table"]
    both = torch.arange(t.shape[1], device=DEVICE) < (torch.minimum(s["kv_len"][0:-1:2], s["kv_len"][1::2]) // c["page"] // 4)[:, None]
    t[1::2] = torch.where(both, t[0:-1:2], t[1::2])
    s["refs"] = _count(t, s["n_pages"])
    s["pool"] = _pool(c, gen, (s["n_pages"],))
    s["max_moves"] = s["n_pages"] // 2
    return s


def _prepare_attn(c, gen):
    page, H, S = c["page"], c["H_kv"], c["seqs"]
    first, prefix, kv, q = _groups(c)
    width = -(-max(kv) // page)
    table = torch.full((S, width), -1, dtype=torch.long)
    used, copies = 0, []
    for g in range(c["groups"]):
        whole, part = prefix[g] // page, prefix[g] % page
        for i in range(first[g], first[g + 1]):
            mine = -(-kv[i] // page)
            if i == first[g]:
                fresh, table[i, :whole] = used + whole, torch.arange(used, used + whole)
                used = fresh
            else:
                table[i, :whole] = table[first[g], :whole]
            table[i, whole:mine] = torch.arange(used, used + mine - whole)
            if part and i > first[g]:   # (the page in which the sequences part is each one's own, with the shared rows in it)
                copies.append((first[g], i, whole))
            used += mine - whole
    n_pages = used + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE)
    table = table.to(DEVICE)
    table = torch.where(table >= 0, order[table.clamp(min=0)], -1).to(torch.int32).contiguous()
    s = {"case": c, "n_pages": n_pages, "table": table, "kv_len": _int(kv), "q_start": _int([sum(q[:i]) for i in range(S + 1)]), "tokens": sum(q),
         "max_q": max(q), "max_kv": max(kv), "group_start": _int(first), "prefix": _int(prefix), "max_prefix": max(prefix),
         "max_group": max(sum(q[first[g]:first[g + 1]]) for g in range(c["groups"]))}
    s["pool"] = torch.empty(n_pages * H * 2 * _block_bytes(c), dtype=torch.uint8, device=DEVICE)
    blocks = s["pool"].view(n_pages, H, 2, -1)
    step = max(1, (1 << 25) // (H * page * D))
    for p in range(0, n_pages, step):
        m = min(step, n_pages - p)
        for which in (0, 1):
            x = _rows(gen, (m, page, H, D), TYPES[c["dtype"]], which == 0).transpose(1, 2).reshape(m * H, page, D)
            blocks[p:p + m, :, which] = _pack(c, x).view(m, H, -1)
    if copies:
        a, b, w = torch.tensor(copies, device=DEVICE).unbind(1)
        blocks[table[b, w].long()] = blocks[table[a, w].long()]
    s["q"] = torch.randn(s["tokens"], H * c["gq"], D, generator=gen, device=DEVICE).to(TYPES[c["dtype"]])
    s["workspace"] = torch.empty(512 << 20, dtype=torch.uint8, device=DEVICE)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return {"append": _prepare_append, "rotate": _prepare_rotate, "step": _prepare_step, "fork": _prepare_fork, "compact": _prepare_compact,
            "attn": _prepare_attn}[case["kind"]](case, gen)


# ---- the framework's calls
def _empty(*shape, dtype=torch.int32):
    return torch.empty(shape, dtype=dtype, device=DEVICE)


def _run_own(s):
    from paper_2403_05527_amd import binding as gb
    c = s["case"]
    kind = c["kind"]
    if kind == "append":
        cfg = gb.make_page_config(s["n_pages"], c["page"], c["H_kv"], c["bits"], c["group"], TYPES[c["dtype"]])
        rope = gb.make_rope(s["freq"], interleaved=c["interleaved"])
        q = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        gb.gear_page_write_rope(cfg, s["pool"], rope, s["K"], s["V"], s["slots"], s["positions"], s["q"], q)
        if c["bits"] == 16:
            return q, s["pool"].view(TYPES[c["dtype"]])
        K, V = (_empty(*s["K"].shape, dtype=q.dtype) for _ in range(2))
        gb.gear_page_read(cfg, s["pool"], K, V, s["slots"])
        return q, K, V
    if kind == "rotate":
        out = torch.empty_like(s["x"])
        gb.gear_rotate(gb.make_rope(s["freq"], interleaved=c["interleaved"], inverse=True), s["x"], out, s["positions"])
        return out
    if kind == "attn":
        cfg = gb.make_page_config(s["n_pages"], c["page"], c["H_kv"], c["bits"], c["group"], TYPES[c["dtype"]])
        batch = gb.make_page_batch(s["q_start"], s["kv_len"], s["table"], s["tokens"], s["max_q"], s["max_kv"])
        groups = gb.make_page_groups(s["group_start"], s["prefix"], s["max_group"], s["max_prefix"])
        out = torch.empty_like(s["q"])
        gb.gear_page_attn_shared(cfg, s["pool"], batch, groups, s["q"], out, D ** -0.5, s["workspace"])
        return out
    if kind == "step":
        t = gb.make_page_table(s["table"], s["kv_len"], s["refs"], c["page"])
        n = c["seqs"]
        slots, copies, refused = _empty(n, c["n"], dtype=torch.int64), _empty(n, 2), _empty(n)
        gb.gear_page_extend(t, s["rows"], s["counts"], slots, copies, refused)
        gb.gear_page_truncate(t, s["rows"], s["keep"])
        return slots, copies, refused, s["table"], s["kv_len"], s["refs"]
    cfg = gb.make_page_config(s["n_pages"], c["page"], c["H_kv"], 16, D, TYPES[c["dtype"]])
    if kind == "fork":
        t = gb.make_page_table(s["table"], s["kv_len"], s["refs"], c["page"])
        n = c["rows"]
        slots, copies, refused = _empty(n, c["n"], dtype=torch.int64), _empty(n, 2), _empty(n)
        gb.gear_page_fork(t, s["src"], s["dst"])
        gb.gear_page_extend(t, s["dst"], s["counts"], slots, copies, refused)
        gb.gear_page_move(cfg, s["pool"].view(torch.uint8).view(c["pools"], -1), copies)
        table = s["table"].clone()
        gb.gear_page_truncate(t, s["dst"], s["keep"])
        return slots, copies, refused, table, s["table"], s["kv_len"], s["refs"], s["pool"]
    table, kv_len, refs = s["table"].clone(), s["kv_len"].clone(), s["refs"].clone()
    moves, counts = _empty(s["max_moves"], 2), _empty(2)
    gb.gear_page_compact(gb.make_page_table(table, kv_len, refs, c["page"]), moves, counts)
    gb.gear_page_move(cfg, s["pool"].view(torch.uint8).flatten(), moves)
    return moves, counts, table, refs, s["pool"]


# ---- the same in plain form
def _turned(c, x, cos, sin):
    """Rows [S, n, heads, 128] in 32 bits; cos, sin [S, n, 1, rot / 2]."""
    r, x = c["rot"], x.float()
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((y, x[..., r:]), -1).to(TYPES[c["dtype"]])


def _angles(s):
    """(cos, sin) [S, n, 1, rot / 2], from angles in 64 bits: far positions."""
    t = s["positions"].double()[..., None, None] * s["freq"]
    return torch.cos(t).float(), torch.sin(t).float()


def _plain_append(s):
    c = s["case"]
    cos, sin = _angles(s)
    q, K, V = _turned(c, s["q"], cos, sin), _turned(c, s["K"], cos, sin), s["V"].contiguous()
    if c["bits"] < 16:
        return (q,) + tuple(_values(c, *_quantise(c, x)) for x in (K, V))
    pool = s["pool"].view(TYPES[c["dtype"]]).view(s["n_pages"], c["H_kv"], 2, c["page"], D)
    page, row = s["slots"] // c["page"], s["slots"] % c["page"]
    pool[page, :, 0, row], pool[page, :, 1, row] = K, V
    return q, s["pool"].view(TYPES[c["dtype"]])


def _plain_rotate(s):
    cos, sin = _angles(s)
    y = _turned(s["case"], s["x"], cos, -sin)
    return y.transpose(1, 2).contiguous().transpose(1, 2) if s["case"]["heads_first"] else y


def _drop(s, rows, keep):
    """Rows of the table keep their first tokens, in place."""
    page, t, n_pages = s["case"]["page"], s["table"], s["n_pages"]
    rows = rows.long()
    mine = t[rows]
    gone = (torch.arange(t.shape[1], device=DEVICE) >= ((keep + page - 1) // page)[:, None]) & (mine >= 0)
    at = torch.where(gone, mine, n_pages).flatten().long()
    s["refs"].add_(torch.zeros(n_pages + 1, dtype=torch.int32, device=DEVICE).scatter_add_(0, at, -torch.ones_like(at, dtype=torch.int32))[:n_pages])
    t[rows] = torch.where(gone, -1, mine)
    s["kv_len"][rows] = torch.minimum(s["kv_len"][rows], keep)


def _grow(s, rows, counts, most):
    """Room for new tokens, in place: (slots, copies, refused)."""
    page, t, refs, n_pages = s["case"]["page"], s["table"], s["refs"], s["n_pages"]
    rows, counts, width = rows.long(), counts.long(), t.shape[1]
    kv = s["kv_len"][rows].long()
    first = kv // page
    held = t[rows].gather(1, first[:, None].clamp(max=width - 1))[:, 0].long()
    partly = (kv % page > 0) & (counts > 0)
    mine = torch.where(partly, held, n_pages)
    named = torch.cat((refs, torch.zeros(1, dtype=torch.int32, device=DEVICE)))[mine]
    shared = partly & (named > 1)
    # of the sequences that are about to write into one page, the last may keep it, if nobody else has it
    before = ((mine[:, None] == mine[None, :]) & shared[None, :]).tril(-1).sum(1)
    copy = shared & (named - before > 1)
    keeps = (partly & ~copy).long()
    need = torch.where(counts > 0, (kv + counts - 1) // page - first + 1 - keeps, 0)
    free = refs == 0
    refused = (need > 0) & (need.cumsum(0) > free.sum())
    base = need.cumsum(0) - need
    rank = torch.where(free, free.long().cumsum(0) - 1, n_pages)
    order = torch.full((n_pages + 1,), -1, dtype=torch.long, device=DEVICE).scatter_(0, rank, torch.arange(n_pages, device=DEVICE))
    j = torch.arange(most // page + 2, device=DEVICE)
    entry, k = first[:, None] + j, j - keeps[:, None]
    new = (k >= 0) & (k < need[:, None]) & ~refused[:, None]
    page_of = torch.where(new, order[(base[:, None] + k).clamp(0, n_pages)], n_pages)
    flat = torch.cat((t.flatten(), torch.zeros(1, dtype=torch.int32, device=DEVICE)))
    flat.scatter_(0, torch.where(new, rows[:, None] * width + entry, t.numel()).flatten(), page_of.to(torch.int32).flatten())
    t.copy_(flat[:-1].view_as(t))
    copy = copy & ~refused
    change = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEVICE)
    change.scatter_add_(0, page_of.flatten(), torch.ones(page_of.numel(), dtype=torch.int32, device=DEVICE))
    change.scatter_add_(0, torch.where(copy, mine, n_pages), -torch.ones_like(rows, dtype=torch.int32))
    refs.add_(change[:n_pages])
    pos = kv[:, None] + torch.arange(most, device=DEVICE)
    slots = t[rows].gather(1, (pos // page).clamp(max=width - 1)).long() * page + pos % page
    slots = torch.where((torch.arange(most, device=DEVICE) < counts[:, None]) & ~refused[:, None], slots, -1)
    copies = torch.where(copy[:, None], torch.stack((mine, page_of[:, 0]), 1), -1).to(torch.int32)
    s["kv_len"][rows] = torch.where(refused, kv, kv + counts).to(torch.int32)
    return slots, copies, torch.where(refused, 2, 0).to(torch.int32)


def _plain_step(s):
    got = _grow(s, s["rows"], s["counts"], s["case"]["n"])
    _drop(s, s["rows"], s["keep"])
    return got + (s["table"], s["kv_len"], s["refs"])


def _plain_fork(s):
    src, dst, n_pages = s["src"].long(), s["dst"].long(), s["n_pages"]
    s["table"][dst] = s["table"][src]
    s["kv_len"][dst] = s["kv_len"][src]
    s["refs"].add_(_count(s["table"][dst], n_pages))
    slots, copies, refused = _grow(s, s["dst"], s["counts"], s["case"]["n"])
    a, b = copies.long().unbind(1)
    # (no copy: the last page onto itself)
    a, b = torch.where(a >= 0, a, n_pages - 1), torch.where(b >= 0, b, n_pages - 1)
    s["pool"][:, b] = s["pool"][:, a]
    table = s["table"].clone()
    _drop(s, s["dst"], s["keep"])
    return slots, copies, refused, table, s["table"], s["kv_len"], s["refs"], s["pool"]


def _plain_compact(s):
    table, refs, n_pages, most = s["table"].clone(), s["refs"].clone(), s["n_pages"], s["max_moves"]
    page = torch.arange(n_pages, device=DEVICE)
    live = refs > 0
    n_live = live.sum()
    to, of = ~live & (page < n_live), live & (page >= n_live)
    count = to.sum().clamp(max=most)
    k_to, k_of = to.long().cumsum(0) - 1, of.flip(0).long().cumsum(0).flip(0) - 1
    to, of = to & (k_to < count), of & (k_of < count)
    moves = torch.full((2, n_pages + 1), -1, dtype=torch.int32, device=DEVICE)
    moves[0].scatter_(0, torch.where(of, k_of, n_pages), page.to(torch.int32))
    moves[1].scatter_(0, torch.where(to, k_to, n_pages), page.to(torch.int32))
    moves = moves[:, :most].t().contiguous()
    goes = torch.where(of, moves[:, 1][k_of.clamp(0, most - 1)].long(), page)
    table = torch.where(table >= 0, goes[table.clamp(min=0).long()].to(torch.int32), table)
    after = torch.zeros(n_pages, dtype=torch.int32, device=DEVICE).scatter_add_(0, goes, refs)
    a, b = moves.long().unbind(1)
    a, b = torch.where(a >= 0, a, n_pages - 1), torch.where(b >= 0, b, n_pages - 1)
    s["pool"][b] = s["pool"][a]   # (where there are fewer moves: the last page onto itself)
    return moves, torch.stack((n_live, count)).to(torch.int32), table, after, s["pool"]


def _plain_attn(s):
    c = s["case"]
    table = s["table"].clamp(min=0).long()
    blocks = s["pool"].view(s["n_pages"], c["H_kv"], 2, -1)
    # [S, width, H, page, 128] -> [S, H, tokens, 128]
    K, V = (_unpack(c, blocks[:, :, which][table]).transpose(1, 2).flatten(2, 3) for which in (0, 1))
    S, H, gq, max_q = c["seqs"], c["H_kv"], c["gq"], s["max_q"]
    start, kv_len = s["q_start"].long(), s["kv_len"].long()
    q_len = start[1:] - start[:-1]
    row = torch.arange(max_q, device=DEVICE)
    at = (start[:-1, None] + row).clamp(max=s["tokens"] - 1)                        # [S, max_q]
    q = s["q"][at].float().view(S, max_q, H, gq, D).permute(0, 2, 3, 1, 4).reshape(S, H, gq * max_q, D)
    score = torch.matmul(q, K.transpose(2, 3).contiguous()).view(S, H, gq, max_q, -1).mul_(D ** -0.5)
    sees = torch.minimum((kv_len - q_len)[:, None] + row + 1, kv_len[:, None])      # [S, max_q]
    hidden = torch.arange(score.shape[-1], device=DEVICE) >= sees[:, :, None]       # [S, max_q, tokens]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    p = score.sub_(score.amax(-1, keepdim=True)).exp_()
    V = V * (torch.arange(V.shape[2], device=DEVICE)[None, :] < kv_len[:, None])[:, None, :, None]
    o = torch.matmul(p.view(S, H, gq * max_q, -1), V).view(S, H, gq, max_q, D) / p.sum(-1, keepdim=True)
    out = torch.empty(s["tokens"], H * gq, D, dtype=TYPES[c["dtype"]], device=DEVICE)
    live = row < q_len[:, None]
    out[at[live]] = o.permute(0, 3, 1, 2, 4).reshape(S, max_q, H * gq, D)[live].to(out.dtype)
    return out


def _run_plain(s):
    return {"append": _plain_append, "rotate": _plain_rotate, "step": _plain_step, "fork": _plain_fork, "compact": _plain_compact,
            "attn": _plain_attn}[s["case"]["kind"]](s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- from the definitions, in 64 bits
def _exact_turn(c, x, positions, sign):
    """Pair by pair; x [S, n, heads, 128]."""
    y = x.double()
    freq = [_frequencies(c)[p].item() for p in range(c["rot"] // 2)]
    got = y.clone()
    for p, f in enumerate(freq):
        i, j = (2 * p, 2 * p + 1) if c["interleaved"] else (p, p + c["rot"] // 2)
        t = sign * positions.double()[..., None] * f
        got[..., i] = y[..., i] * t.cos() - y[..., j] * t.sin()
        got[..., j] = y[..., i] * t.sin() + y[..., j] * t.cos()
    return got


def exact(case, seed):
    c = case
    if c["kind"] in ("step", "fork", "compact"):
        return None   # whole numbers, and bytes that are moved
    s = prepare(c, seed)
    dt = TYPES[c["dtype"]]
    if c["kind"] == "rotate":
        return _exact_turn(c, s["x"], s["positions"], -1.0)
    if c["kind"] == "append":
        q, K, V = _exact_turn(c, s["q"], s["positions"], 1.0), _exact_turn(c, s["K"], s["positions"], 1.0), s["V"].double()
        if c["bits"] == 16:
            pool = torch.zeros(s["n_pages"], c["H_kv"], 2, c["page"], D, dtype=torch.float64, device=DEVICE)
            for i in range(c["seqs"]):
                at = s["slots"][i]
                pool[at // c["page"], :, 0, at % c["page"]] = K[i]
                pool[at // c["page"], :, 1, at % c["page"]] = V[i]
            return q, pool.flatten()
        back = []
        for x in (K.to(dt).double(), V):   # (what is quantized is the turned row in the cache's type)
            v = x.reshape(-1, c["group"])
            low = v.min(1, keepdim=True).values
            gap = ((v.max(1, keepdim=True).values - low) / 255).to(dt).double()
            k = torch.clamp(torch.round((v - low) / gap), max=255)
            back.append(torch.where(gap > 0, low + torch.nan_to_num(k) * gap, low).view(x.shape))
        return (q,) + tuple(back)
    G, page, H = D // c["group"], c["page"], c["H_kv"]
    pool = s["pool"].view(s["n_pages"], H, 2, -1)

    def stored(which, pages, h):
        """[tokens, 128] of one sequence's pages and one head."""
        b = pool[pages, h, which]
        at = page * D * c["bits"] // 8
        if c["bits"] == 16:
            return b.contiguous().view(dt).reshape(-1, D).double()
        by = b[:, :at].reshape(-1, D * c["bits"] // 8).long()
        if c["bits"] == 4:   # word w: bytes 4 w .. 4 w + 3
            word = by[:, 0::4] + (by[:, 1::4] << 8) + (by[:, 2::4] << 16) + (by[:, 3::4] << 24)
            by = torch.stack([word >> (4 * (e // 2) + 16 * (e % 2)) & 15 for e in range(8)], -1).reshape(-1, D)
        w = b[:, at:].contiguous().view(dt).view(-1, G, page, 2).double()
        scale, zero = (w[..., k].permute(0, 2, 1).reshape(-1, G).repeat_interleave(c["group"], 1) for k in (0, 1))
        return (scale * by.double() + zero).to(dt).double()   # (a code stands for a value of the cache's type)

    _, _, kv_len, q_len = _groups(c)
    out = torch.empty(s["tokens"], H * c["gq"], D, dtype=torch.float64, device=DEVICE)
    begin = 0
    for i, (n, total) in enumerate(zip(q_len, kv_len)):
        pages = s["table"][i, :-(-total // page)].long()
        ban = torch.arange(total, device=DEVICE)[None, :] > torch.arange(total - n, total, device=DEVICE)[:, None]
        for h in range(H):
            K, V = (stored(w, pages, h)[:total] for w in (0, 1))
            for g in range(h * c["gq"], (h + 1) * c["gq"]):
                score = (s["q"][begin:begin + n, g].double() @ K.t() / math.sqrt(D)).masked_fill(ban, -math.inf)
                out[begin:begin + n, g] = torch.softmax(score, -1) @ V
        begin += n
    return out


def work(case):
    c = case
    kind = c["kind"]
    if kind == "append":   # q, K and V in; q out; the pages written, and read where they are codes
        rows = c["seqs"] * c["n"]
        stored = 2 * c["H_kv"] * _block_bytes(c) // c["page"]
        back = 0 if c["bits"] == 16 else stored + 4 * c["H_kv"] * D
        return {"bytes": rows * (2 * D * c["H_kv"] * (2 * c["gq"] + 2) + stored + back + 16) + 4 * c["rot"],
                "flops": rows * (3 * c["rot"] * c["H_kv"] * (c["gq"] + 1) + (0 if c["bits"] == 16 else 2 * c["H_kv"] * D * 10))}
    if kind == "rotate":
        rows = c["seqs"] * c["n"]
        return {"bytes": rows * (4 * D * c["heads"] + 8), "flops": rows * 3 * c["rot"] * c["heads"]}
    page = c["page"]
    if kind in ("step", "fork"):   # refs read once, slots written, the entries that come and go, lengths and counts
        seqs = c["seqs"] if kind == "step" else c["rows"]
        kv = _lengths(c, c["kv_lo"], c["kv_hi"], c["seqs"] if kind == "step" else c["prompts"])
        used = sum(-(-k // page) for k in kv + _lengths(c, 500, 1000, c.get("others", 0)))
        entries = sum(-(-(kv[i % len(kv)] + c["n"]) // page) - (-(-kv[i % len(kv)] // page) if kind == "step" else 0) for i in range(seqs))
        moved = 0
        if kind == "fork":   # (the last of a prompt's copies has to copy, too: the prompt itself has the page)
            moved = sum(1 for i in range(seqs) if kv[i % len(kv)] % page)
        return {"bytes": 4 * (used + entries) + 8 * seqs * c["n"] + 8 * entries + 24 * seqs + moved * c.get("pools", 0) * 2 * 4 * D * page * c.get("H_kv", 0),
                "flops": 4 * (used + seqs * c["n"])}
    if kind == "compact":   # the pages that move, read and written; table and refs read and written
        kv = _lengths(c, max(1, c["kv_lo"]), c["kv_hi"], c["seqs"])
        used = sum(-(-k // page) for k in kv)
        live = used - sum(min(kv[i], kv[i + 1]) // page // 4 for i in range(0, c["seqs"] - 1, 2))
        n_pages = int(used / c["live"]) + 1
        moved = live * (n_pages - live) // n_pages
        return {"bytes": moved * 2 * 4 * D * page * c["H_kv"] + 8 * n_pages + 8 * used, "flops": 4 * (n_pages + used)}
    first, prefix, kv_len, q_len = _groups(c)
    row = 2 * c["H_kv"] * _block_bytes(c) // page                               # a token's bytes in the pool, Keys and Values
    tokens = sum(prefix) + sum(kv_len[i] - prefix[g] for g in range(c["groups"]) for i in range(first[g], first[g + 1]))
    seen = sum(n * (total - n) + n * (n + 1) // 2 for n, total in zip(q_len, kv_len))
    return {"bytes": tokens * row + 4 * sum(q_len) * c["H_kv"] * c["gq"] * D, "flops": 4 * D * c["H_kv"] * c["gq"] * seen}
