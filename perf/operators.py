"""The operators of a serving instance's decode step, by which their speed is
followed: the 8-bit token cache (append, attention, eviction) and products with
4-bit weights.  ``own`` chooses between the package's kernels and the plain
form of the same definitions.

A case says which operator runs (``op``) and on what:

  append   new tokens into the cache: block scales, codes held requantised
  attend   attention of each sequence's new tokens over its cached tokens, with
           the attention weights accumulated per slot where ``weights`` is set
  evict    sequences over the budget give up the slots of least weight
  w4       rows times a matrix of 4-bit codes with group scales

The cache is a pool of blocks of 64 slots.  Keys are held as [block, kv head,
slot, dim], values as [block, kv head, 4, dim, 16]: slot t of a block stands in
group (t / 4) % 4, there at place (t / 16) * 4 + t % 4.  One power-of-two scale
for a block and head; code times scale is the value.  A sequence is a row of the
block table (blocks in any order) and a length.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 64
TOP = {"e4m3": 448.0, "int8": 127.0}      # largest code
LEAST = -100                              # least exponent of a scale
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TYPE = {"bf16": torch.bfloat16, "f16": torch.float16}
# where a value's slot stands inside its block: group * 16 + place
PLACE = [((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3) for t in range(BLOCK)]


# -- cases --------------------------------------------------------------------

def _cache(op, seqs, heads, kv_heads, dim, length, **more):
    c = {"op": op, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "length": length,      # slots of the longest sequence, new ones included
         "new": 1,              # new tokens of a sequence (the most of any)
         "ragged": True,        # lengths (and new tokens) between none and the most
         "format": "e4m3", "type": "bf16",
         "weights": False,      # attend: accumulate the weights
         "budget": 0, "recent": 0}
    c.update(more)
    return c


def _w4(rows, outs, ins, group, **more):
    return {"op": "w4", "rows": rows, "outs": outs, "ins": ins, "group": group, "type": "bf16",
            **more}


def listed():
    cases = {
        # one decode step of a batch writes one token a sequence
        "append_token": _cache("append", 64, 0, 8, 128, 2048),
        # ragged prompts written whole, 8-bit integers, narrow heads
        "append_prompt": _cache("append", 6, 0, 8, 64, 2500, new=2100, format="int8", type="f16"),
        # one request alone, a short answer so far: the smallest call, all latency
        "attend_one": _cache("attend", 1, 32, 8, 128, 700, ragged=False),
        # the everyday decode step: a ragged batch that keeps its weights for evictions
        "attend_batch": _cache("attend", 48, 32, 8, 128, 4096, weights=True),
        # a few drafted tokens checked at once, odd heads and an odd width
        "attend_odd": _cache("attend", 7, 20, 4, 80, 1500, new=3, format="int8", type="f16",
                             weights=True),
        # two mega prompts in decode: few rows over a very long axis
        "attend_long": _cache("attend", 2, 64, 8, 128, 150000),
        # a full instance: the largest batch, several GB of cache
        "attend_large": _cache("attend", 192, 64, 8, 128, 16000, format="int8", type="f16"),
        # prompts over the context of earlier turns, weights begun
        "attend_prompt": _cache("attend", 5, 32, 8, 128, 2600, new=2000, weights=True),
        # a batch in steady decode gives a block back every 64 tokens
        "evict_step": _cache("evict", 64, 0, 8, 128, 1024 + 64, ragged=False, budget=1024,
                             recent=128),
        # long ragged prompts cut to the budget
        "evict_prompt": _cache("evict", 12, 0, 8, 128, 16000, budget=2048, recent=256,
                               format="int8", type="f16"),
        # one token through a square projection
        "w4_token": _w4(1, 4096, 4096, 128),
        # a decode batch through a wide one with an odd number of outputs
        "w4_batch": _w4(48, 20001, 8192, 32, type="f16"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "evict", "w4", "w4"])
    kind = rng.choice(["bf16", "f16"])
    if op == "w4":
        group = rng.choice([32, 64, 128])
        rows = _log(rng, 1, 64)
        return _w4(rows, _log(rng, 300, 20001), group * _log(rng, max(1, 512 // group), 8192 // group),
                   group, type=kind)
    kv = rng.choice([1, 2, 4, 8])
    dim = rng.choice([64, 80, 96, 128, 128])
    fmt = rng.choice(["e4m3", "int8"])
    if op == "append":
        new = rng.choice([1, 1, _log(rng, 2, 2100)])
        seqs = _log(rng, 1, 128) if new == 1 else _log(rng, 1, 6)
        return _cache("append", seqs, 0, kv, dim, new + _log(rng, 1, 2000), new=new, format=fmt,
                      type=kind)
    if op == "evict":
        budget = BLOCK * _log(rng, 2, 32)
        return _cache("evict", _log(rng, 1, 32), 0, kv, dim, budget + _log(rng, 1, 14000),
                      budget=budget, recent=rng.randrange(0, budget // 2), format=fmt, type=kind)
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    weights = rng.random() < 0.5
    shape = rng.choice(["token", "token", "draft", "prompt"])
    if shape == "prompt":
        new = _log(rng, 17, 1500)
        return _cache("attend", _log(rng, 1, 4), kv * group, kv, dim, new + _log(rng, 1, 1000),
                      new=new, format=fmt, type=kind, weights=weights)
    length = _log(rng, 8, 60000)
    seqs = _log(rng, 1, max(1, min(192, 1500000 // length)))
    return _cache("attend", seqs, kv * group, kv, dim, length,
                  new=1 if shape == "token" else min(length, rng.randrange(2, 8)), format=fmt,
                  type=kind, weights=weights)


def _share(k):
    """A number in (0, 1) for sequence k, spread evenly."""
    return ((k + 1) * 0.6180339887498949) % 1.0


def _lengths(c):
    """(length, new tokens) of each sequence: the first the longest, in a batch
    of four or more the second without a token."""
    most = [(c["length"], c["new"])] * c["seqs"]
    if not c["ragged"]:
        return most
    out = []
    for k, (length, new) in enumerate(most):
        u = 1.0 if k == 0 else _share(k)
        m = max(1, int(new * u))
        out.append((max(m, int(length * u)), m))
    if c["seqs"] >= 4:
        out[1] = (0, 1 if c["new"] == 1 else 0)
    return out


def _pairs(c):
    """(row, slot) pairs that see each other, over all sequences."""
    return sum(max(0, length - new + t + 1) for length, new in _lengths(c) for t in range(new))


def work(case):
    c = case
    if c["op"] == "w4":
        m, n, k = c["rows"], c["outs"], c["ins"]
        return {"bytes": n * k / 2 + n * k / c["group"] * 2.5 + 2 * m * (n + k),
                "flops": 2 * m * n * k}
    d, kv = c["dim"], c["kv_heads"]
    rows = sum(n for _, n in _lengths(c))
    slots = sum(length for length, _ in _lengths(c))
    if c["op"] == "append":
        return {"bytes": rows * kv * (2 * d * 2 + 2 * d + 8), "flops": rows * kv * d * 6}
    if c["op"] == "attend":
        return {"bytes": slots * kv * (2 * d + 0.125 + (8 if c["weights"] else 0)) +
                rows * c["heads"] * d * 4, "flops": 4 * d * c["heads"] * _pairs(c)}
    bytes_, flops = 0, 0
    for length, _ in _lengths(c):
        if length <= c["budget"]:
            continue
        tail = length - c["budget"]
        kept = min(c["recent"], tail)
        kept += (tail - kept) * (c["budget"] - c["recent"]) / max(1, length - c["recent"])
        bytes_ += kv * (8 * length + kept * 2 * (2 * d + 8))
        flops += kv * length * 4
    return {"bytes": bytes_ + 1, "flops": flops}


# -- inputs -------------------------------------------------------------------

def _by_slot(x):
    """Values held as [.., 4, dim, 16], slot by slot: [.., 64, dim]."""
    at = torch.tensor(PLACE, device=x.device)
    return x.transpose(-1, -2).flatten(-3, -2)[..., at, :]


def _as_held(x):
    """Values slot by slot, as they are held."""
    at = torch.argsort(torch.tensor(PLACE, device=x.device))
    return x[..., at, :].unflatten(-2, (4, 16)).transpose(-1, -2)


def _codes(x, fmt):
    """Block scales and codes of values [block, head, 64, dim]."""
    a = x.abs().amax(dim=(2, 3))
    scale = _power(a, fmt)
    y = x / scale[:, :, None, None]
    return scale, (y.to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().to(torch.int8))


def prepare(case, seed):
    c = case
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    rnd = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    dt = TYPE[c["type"]]
    if c["op"] == "w4":
        m, n, k, g = c["rows"], c["outs"], c["ins"], c["group"]
        s = {"case": c, "x": rnd(m, k).to(dt),
             "codes": torch.randint(0, 16, (n, k), generator=gen, device=dev, dtype=torch.uint8),
             "scale": (0.01 * (0.5 + torch.rand((n, k // g), generator=gen, device=dev))).half(),
             "zero": torch.randint(5, 11, (n, k // g), generator=gen, device=dev,
                                   dtype=torch.uint8)}
        if own:
            from paper_2407_00047_amd import qlm
            s["w4"] = qlm.w4_pack(s["codes"], s["scale"], s["zero"])
            s["ws"] = qlm.w4_workspace(s["w4"], m)
        return s
    kv, d, seqs, fmt = c["kv_heads"], c["dim"], c["seqs"], c["format"]
    both = _lengths(c)
    blocks = [-(-length // BLOCK) for length, _ in both]
    width = max(1, max(blocks))
    if c["op"] == "evict":
        width = max(width, c["budget"] // BLOCK)
    total = sum(blocks)
    # the pool's blocks in any order; the last one belongs to nobody
    order = torch.randperm(total, generator=gen, device=dev).cpu().tolist()
    table = [[total] * width for _ in range(seqs)]
    at = 0
    for b, n in enumerate(blocks):
        table[b][:n] = order[at:at + n]
        at += n
    n_blocks = total + 1
    channel = torch.exp(0.7 * rnd(kv, 1, d))
    k_codes = torch.empty((n_blocks, kv, BLOCK, d), dtype=CODE[fmt], device=dev)
    v_codes = torch.empty((n_blocks, kv, 4, d, 16), dtype=CODE[fmt], device=dev)
    k_scale = torch.empty((n_blocks, kv), device=dev)
    v_scale = torch.empty((n_blocks, kv), device=dev)
    step = max(1, (1 << 28) // (kv * BLOCK * d))
    for b in range(0, n_blocks, step):
        e = min(n_blocks, b + step)
        k_scale[b:e], k_codes[b:e] = _codes(rnd(e - b, kv, BLOCK, d) * channel, fmt)
        v_scale[b:e], q = _codes(rnd(e - b, kv, BLOCK, d), fmt)
        v_codes.view(torch.uint8)[b:e] = _as_held(q.view(torch.uint8))
    lengths = torch.tensor([x for x, _ in both], dtype=torch.int32, device=dev)
    start = np.concatenate([[0], np.cumsum([n for _, n in both])]).astype(np.int32)
    table = torch.tensor(table, dtype=torch.int32, device=dev)
    slots = torch.arange(BLOCK, device=dev, dtype=torch.int32)
    position = torch.zeros((n_blocks, kv, BLOCK), dtype=torch.int32, device=dev)
    where = (torch.arange(width, device=dev, dtype=torch.int32)[None, :, None, None] * BLOCK +
             slots).expand(seqs, width, kv, BLOCK)
    position[table.long()] = where
    position[total] = 0
    weight = torch.exp(2.0 * rnd(n_blocks, kv, BLOCK))
    # slots that no token stands in hold whatever was there: not-a-numbers too
    if fmt == "e4m3":
        for b, (length, _) in enumerate(both):
            if length % BLOCK:
                last, used = int(table[b, length // BLOCK]), length % BLOCK
                k_codes.view(torch.uint8)[last, :, used:] = 0x7f
                held = _by_slot(v_codes.view(torch.uint8)[last])
                held[:, used:] = 0x7f
                v_codes.view(torch.uint8)[last] = _as_held(held)
    s = {"case": c, "k_codes": k_codes, "v_codes": v_codes, "k_scale": k_scale,
         "v_scale": v_scale, "position": position, "weight": weight, "table": table,
         "lengths": lengths, "n_rows": int(start[-1]), "max_new": max(n for _, n in both),
         "max_length": max(x for x, _ in both),
         "row_start": torch.from_numpy(start).to(dev)}
    if c["op"] == "append":
        s["k"] = (rnd(s["n_rows"], kv, d) * channel[None, :, 0]).to(dt)
        s["v"] = rnd(s["n_rows"], kv, d).to(dt)
        s["first"] = lengths - (s["row_start"][1:] - s["row_start"][:-1])
    if c["op"] == "attend":
        s["q"] = (rnd(s["n_rows"], c["heads"], d) * 1.5).to(dt)
        s["weight0"] = weight.clone()
    if c["op"] == "evict":
        s["weight0"], s["position0"] = weight.clone(), position.clone()
        s["out_lengths"] = torch.empty_like(lengths)
    if own:
        from paper_2407_00047_amd import qlm
        s["cache"] = qlm.DeviceKvCache(k_codes, v_codes, k_scale, v_scale, position, weight)
        s["batch"] = qlm.KvBatch(table, lengths, s["row_start"], s["n_rows"], s["max_new"],
                                 s["max_length"])
        if c["op"] == "attend":
            s["ws"] = qlm.kv_attention_workspace(s["cache"], s["batch"], c["heads"], c["weights"])
        if c["op"] == "evict":
            s["ws"] = qlm.kv_evict_workspace(s["cache"], s["batch"], c["budget"])
    return s


# -- one pass -----------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    return (_own if own else _plain)[op](s)


def _cache_out(s):
    return {n: s[n] for n in ("k_codes", "v_codes", "k_scale", "v_scale", "position", "weight")}


def _own_append(s):
    from paper_2407_00047_amd import qlm
    qlm.kv_append(s["cache"], s["batch"], s["k"], s["v"], s["first"])
    return _cache_out(s)


def _own_attend(s):
    from paper_2407_00047_amd import qlm
    if not s["case"]["weights"]:
        return {"out": qlm.kv_attention(s["cache"], s["batch"], s["q"], ws=s["ws"])}
    s["weight"].copy_(s["weight0"])       # a step adds to the weights of the steps before
    out = qlm.kv_attention(s["cache"], s["batch"], s["q"], weight_decay=1.0, ws=s["ws"])
    return {"out": out, "weight": s["weight"]}


def _own_evict(s):
    from paper_2407_00047_amd import qlm
    s["weight"].copy_(s["weight0"])
    s["position"].copy_(s["position0"])
    qlm.kv_evict(s["cache"], s["batch"], s["case"]["budget"], s["case"]["recent"],
                 out=s["out_lengths"], ws=s["ws"])
    return dict(_cache_out(s), lengths=s["out_lengths"])


def _own_w4(s):
    from paper_2407_00047_amd import qlm
    return qlm.w4_matmul(s["x"], s["w4"], ws=s["ws"])


def _power(a, fmt):
    """The least power of two that holds magnitude a in a code, 2^LEAST at least."""
    m, e = torch.frexp(a)
    top_m, top_e = math.frexp(TOP[fmt])
    e = torch.where(a > 0, e - top_e + (m > top_m).to(e.dtype), torch.full_like(e, LEAST))
    return torch.ldexp(torch.ones_like(a), e.clamp(min=LEAST))


def _encode(y, fmt):
    """Codes (as bytes) of values over their scale."""
    y = y.clamp(-TOP[fmt], TOP[fmt])
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(y.isnan(), 0.0, y).round().to(torch.int8).view(torch.uint8)


def _write(x, codes, scale, fmt, blk, off, first_blk, held):
    """New values x [row, head, dim] into the keys' or the values' codes."""
    xf = x.float()
    a = torch.where(xf.isfinite(), xf.abs(), 0.0).amax(-1)
    need = torch.zeros_like(scale).scatter_reduce(0, blk[:, None].expand_as(a), a, "amax")
    hit = torch.zeros_like(scale[:, 0])
    hit = hit.scatter_reduce(0, blk, torch.ones_like(hit[blk]), "amax") > 0
    fresh = torch.zeros_like(scale[:, 0])
    fresh = fresh.scatter_reduce(0, blk, (off == 0).float(), "amax") > 0
    old = torch.where(fresh[:, None], 0.0, scale)
    grown = torch.where(hit[:, None], torch.maximum(old, _power(need, fmt)), scale)
    # the codes held by a block whose scale grows (only a sequence's first block holds any)
    ratio = torch.where(held[:, None], scale[first_blk] / grown[first_blk], 1.0)
    raw = codes.view(torch.uint8)
    held = codes[first_blk].float()
    raw[first_blk] = _encode(held * ratio.view(ratio.shape + (1,) * (held.ndim - 2)), fmt)
    scale.copy_(grown)
    y = _encode(xf / scale[blk][:, :, None], fmt)
    heads = torch.arange(scale.shape[1], device=x.device)
    if raw.ndim == 4:
        raw[blk[:, None], heads, off[:, None]] = y
    else:
        at = torch.tensor(PLACE, device=x.device)[off]
        raw.view(*raw.shape[:2], 4, -1, 16)[blk[:, None], heads, at[:, None] // 16, :,
                                            at[:, None] % 16] = y


def _rows(s):
    """(sequence, place among the sequence's rows) of each row."""
    n = (s["row_start"][1:] - s["row_start"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=n.device), n,
                                  output_size=s["n_rows"])
    return n, seq, torch.arange(s["n_rows"], device=n.device) - s["row_start"].long()[seq]


def _plain_append(s):
    fmt = s["case"]["format"]
    n, seq, i = _rows(s)
    start = s["lengths"].long() - n
    slot = start[seq] + i
    keep = slot >= 0                      # a row of a sequence without slots has none
    seq, slot, i = seq[keep], slot[keep], i[keep]
    table = s["table"].long()
    blk, off = table[seq, slot // BLOCK], slot % BLOCK
    first = start.clamp(min=0) // BLOCK
    held = (n > 0) & (start > 0) & (start % BLOCK != 0)
    first_blk = table.gather(1, first.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    _write(s["k"][keep], s["k_codes"], s["k_scale"], fmt, blk, off, first_blk, held)
    _write(s["v"][keep], s["v_codes"], s["v_scale"], fmt, blk, off, first_blk, held)
    heads = torch.arange(s["position"].shape[1], device=blk.device)
    pos = (s["first"][seq] + i).int()
    s["position"][blk[:, None], heads, off[:, None]] = pos[:, None]
    s["weight"][blk[:, None], heads, off[:, None]] = 0.0
    return _cache_out(s)


def _values(s, table, name):
    """Cached values of every sequence's slots in single precision [seq, head, slot, dim]."""
    x = s[name + "_codes"][table].float()
    if name == "v":
        x = _by_slot(x)
    x = x * s[name + "_scale"][table][..., None, None]
    b, nb, h, _, d = x.shape
    return x.transpose(1, 2).reshape(b, h, nb * BLOCK, d)


def _plain_attend(s):
    c = s["case"]
    q, table = s["q"], s["table"].long()
    n, seq, i = _rows(s)
    seqs, kv, d, t = c["seqs"], c["kv_heads"], c["dim"], s["max_new"]
    g = c["heads"] // kv
    qp = torch.zeros((seqs, t, kv, g, d), device=q.device)
    qp[seq, i] = q.float().view(-1, kv, g, d)
    qp = qp.permute(0, 2, 3, 1, 4).reshape(seqs, kv, g * t, d)
    slots = torch.arange(table.shape[1] * BLOCK, device=q.device)
    used = slots < s["lengths"][:, None]                                   # [seq, slot]
    last = (s["lengths"].long() - n)[:, None] + torch.arange(t, device=q.device)
    seen = (slots <= last[:, :, None]) & used[:, None] & \
        (torch.arange(t, device=q.device) < n[:, None])[:, :, None]       # [seq, t, slot]
    seen = seen[:, None, None].expand(-1, -1, g, -1, -1).reshape(seqs, 1, g * t, -1)
    sc = torch.matmul(qp, _values(s, table, "k").transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    sc.masked_fill_(~seen, -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = sc.sub_(torch.where(m.isfinite(), m, 0.0)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp(min=1e-30))
    v = _values(s, table, "v").masked_fill_(~used[:, None, :, None], 0.0)
    o = torch.matmul(p, v).view(seqs, kv, g, t, d).permute(0, 3, 1, 2, 4)
    out = o[seq, i].reshape(-1, c["heads"], d).to(q.dtype)
    if not c["weights"]:
        return {"out": out}
    got = p.sum(2).view(seqs, kv, -1, BLOCK).transpose(1, 2)               # [seq, block, head, 64]
    s["weight"].copy_(s["weight0"])
    was = s["weight"][table]
    s["weight"][table] = torch.where(used.view(seqs, -1, 1, BLOCK), was + got, was)
    return {"out": out, "weight": s["weight"]}


def _refill(s, name, table, src, hole, fmt):
    """The blocks of `table` [seq, nb] with the values of slots src [seq, head,
    slot] in their holes."""
    every = s["table"].long()
    seqs, nb = table.shape
    kv = src.shape[1]
    codes, scale = s[name + "_codes"], s[name + "_scale"]
    heads = torch.arange(kv, device=src.device)[None, :, None]
    blk = every.gather(1, (src // BLOCK).view(seqs, -1)).view_as(src)
    raw = codes.view(torch.uint8)
    if name == "k":
        got = raw[blk, heads, src % BLOCK]
    else:
        at = torch.tensor(PLACE, device=src.device)[src % BLOCK]
        got = raw[blk, heads, at // 16, :, at % 16]
    x = got.view(codes.dtype).float() * scale[blk, heads][..., None]
    x = torch.where(hole[..., None], x, 0.0)
    a = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1).view(seqs, kv, nb, BLOCK).amax(-1)
    old = scale[table].transpose(1, 2)                                      # [seq, head, nb]
    any_hole = hole.view(seqs, kv, nb, BLOCK).any(-1)
    grown = torch.where(any_hole, torch.maximum(old, _power(a, fmt)), old)
    held = codes[table].float()
    if name == "v":
        held = _by_slot(held)
    held = held.transpose(1, 2) * (old / grown)[..., None, None]            # [seq, head, nb, 64, d]
    y = torch.where(hole.view(seqs, kv, nb, BLOCK, 1),
                    x.view(seqs, kv, nb, BLOCK, -1) / grown[..., None, None], held)
    y = _encode(y, fmt).transpose(1, 2)
    if name == "v":
        y = _as_held(y)
    raw[table] = y
    scale[table] = grown.transpose(1, 2)


def _plain_evict(s):
    c = s["case"]
    fmt, budget, recent = c["format"], c["budget"], c["recent"]
    s["weight"].copy_(s["weight0"])
    s["position"].copy_(s["position0"])
    table = s["table"].long()
    seqs, width = table.shape
    kv = c["kv_heads"]
    flat = lambda x: x[table].transpose(1, 2).reshape(seqs, kv, -1)  # noqa: E731
    w, pos = flat(s["weight"]).double(), flat(s["position"]).long()
    slots = torch.arange(width * BLOCK, device=table.device)
    used = (slots < s["lengths"][:, None])[:, None].expand(-1, kv, -1)
    newest = torch.where(used, pos, -1).amax(-1, keepdim=True)
    key = torch.where(w.isnan(), -1e300, w.clamp(-1e299, 1e299))
    key = torch.where(pos > newest - recent, 2e300, key)
    key = torch.where(used, key, -math.inf)
    order = torch.argsort(key, dim=-1, descending=True, stable=True)
    over = (s["lengths"] > budget)[:, None, None]
    keep = torch.zeros_like(used).scatter(2, order[:, :, :budget], True)
    hole = over & ~keep & (slots < budget)
    moved = over & keep & (slots >= budget)
    # the i-th hole takes the i-th kept slot past the budget
    rank_hole, rank_moved = hole.cumsum(-1) - 1, moved.cumsum(-1) - 1
    n = width * BLOCK
    lists = torch.zeros((seqs, kv, n + 1), dtype=torch.long, device=table.device)
    lists.scatter_(2, torch.where(moved, rank_moved, n), slots.expand_as(moved).contiguous())
    src = torch.where(hole, lists.gather(2, rank_hole.clamp(min=0)), slots)[:, :, :budget]
    hole = hole[:, :, :budget]
    front = table[:, :budget // BLOCK]
    _refill(s, "k", front, src, hole, fmt)
    _refill(s, "v", front, src, hole, fmt)
    pick = lambda x: x.gather(2, src).view(seqs, kv, -1, BLOCK).transpose(1, 2)  # noqa: E731
    s["weight"][front] = pick(flat(s["weight"]))
    s["position"][front] = pick(flat(s["position"]))
    s["out_lengths"].copy_(s["lengths"].clamp(max=budget))
    return dict(_cache_out(s), lengths=s["out_lengths"])


def _plain_w4(s):
    g = s["case"]["group"]
    n, k = s["codes"].shape
    w = (s["codes"].float().view(n, k // g, g) - s["zero"].float()[:, :, None]) * \
        s["scale"].float()[:, :, None]
    return torch.matmul(s["x"].float(), w.view(n, k).t()).to(s["x"].dtype)


_own = {"append": _own_append, "attend": _own_attend, "evict": _own_evict, "w4": _own_w4}
_plain = {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict,
          "w4": _plain_w4}


# -- the definitions in 64 bits -------------------------------------------------

def _exact_scale(a, fmt):
    if not a > 0:
        return 2.0 ** LEAST
    e = LEAST
    for e in range(max(LEAST, int(math.floor(math.log2(a / TOP[fmt]))) - 1), 200):
        if a <= TOP[fmt] * 2.0 ** e:
            break
    return 2.0 ** e


def _exact_code(y, fmt):
    """The nearest code's value, ties to even."""
    if fmt == "int8":
        return np.rint(np.clip(np.nan_to_num(y, nan=0.0, posinf=127, neginf=-127), -127, 127))
    y = np.clip(y, -448.0, 448.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(y))), -6.0)
    step = np.exp2(np.where(np.isfinite(e), e, -6.0) - 3.0)
    return np.rint(y / step) * step


class _Host:
    """The cache in host memory, in 64 bits, slot by slot."""

    def __init__(self, s):
        self.fmt = s["case"]["format"]
        f64 = lambda x: x.float().cpu().numpy().astype(np.float64)  # noqa: E731
        self.k = f64(s["k_codes"])
        v = f64(s["v_codes"])
        v = v.transpose(0, 1, 2, 4, 3).reshape(v.shape[0], v.shape[1], BLOCK, -1)
        self.v = v[:, :, PLACE]
        self.ks, self.vs = f64(s["k_scale"]), f64(s["v_scale"])
        self.pos, self.weight = s["position"].cpu().numpy().copy(), f64(s["weight"])
        self.table = s["table"].cpu().numpy()
        self.lengths = s["lengths"].cpu().numpy()

    def put(self, codes, scale, blk, h, offs, x, fresh):
        """Values x [n, dim] into the slots offs of one block and head."""
        a = np.abs(x[np.isfinite(x)])
        need = _exact_scale(a.max() if a.size else 0.0, self.fmt)
        old = scale[blk, h]
        new = need if fresh else max(old, need)
        if not fresh and new > old:
            codes[blk, h] = _exact_code(codes[blk, h] * (old / new), self.fmt)
        codes[blk, h, offs] = _exact_code(x / new, self.fmt)
        scale[blk, h] = new

    def out(self):
        v = self.v[:, :, np.argsort(PLACE)]
        v = v.reshape(v.shape[0], v.shape[1], 4, 16, -1).transpose(0, 1, 2, 4, 3)
        return {"k_codes": self.k, "v_codes": v, "k_scale": self.ks, "v_scale": self.vs,
                "position": self.pos, "weight": self.weight}


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict,
            "w4": _exact_w4}[c["op"]](c, s)


def _exact_append(c, s):
    if s["k_codes"].numel() > 1 << 28:
        return None
    host = _Host(s)
    k, v = s["k"].double().cpu().numpy(), s["v"].double().cpu().numpy()
    start, first = s["row_start"].cpu().numpy(), s["first"].cpu().numpy()
    for b in range(c["seqs"]):
        n = start[b + 1] - start[b]
        begin = host.lengths[b] - n
        for j in range(max(begin, 0) // BLOCK, -(-host.lengths[b] // BLOCK)):
            lo, hi = max(begin, j * BLOCK), min(host.lengths[b], (j + 1) * BLOCK)
            rows = np.arange(lo, hi) - begin
            offs = np.arange(lo, hi) - j * BLOCK
            blk = host.table[b, j]
            for h in range(c["kv_heads"]):
                host.put(host.k, host.ks, blk, h, offs, k[start[b] + rows, h], lo == j * BLOCK)
                host.put(host.v, host.vs, blk, h, offs, v[start[b] + rows, h], lo == j * BLOCK)
                host.pos[blk, h, offs] = first[b] + rows
                host.weight[blk, h, offs] = 0.0
    return host.out()


def _exact_attend(c, s):
    kv, d = c["kv_heads"], c["dim"]
    g = c["heads"] // kv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    weight = s["weight"].double()
    start = s["row_start"].cpu().tolist()
    at = torch.tensor(PLACE, device="cuda")
    for b, (length, n) in enumerate(_lengths(c)):
        if length == 0 or n == 0:
            continue
        ids = s["table"][b, :-(-length // BLOCK)].long()
        for h in range(kv):
            key = s["k_codes"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]
            val = s["v_codes"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None, None]
            key = key.reshape(-1, d)[:length]
            val = val.transpose(2, 3).reshape(-1, BLOCK, d)[:, at].reshape(-1, d)[:length]
            q = s["q"][start[b]:start[b + 1], h * g:(h + 1) * g].double().reshape(n * g, d)
            sc = (q @ key.t().contiguous()) / math.sqrt(d)
            last = length - n + torch.arange(n, device="cuda").repeat_interleave(g)
            sc[torch.arange(length, device="cuda")[None] > last[:, None]] = -math.inf
            p = torch.softmax(sc, -1)
            out[start[b]:start[b + 1], h * g:(h + 1) * g] = (p @ val).view(n, g, d)
            w = torch.zeros(ids.numel() * BLOCK, dtype=torch.float64, device="cuda")
            w[:length] = p.sum(0)
            weight[ids, h] += w.view(-1, BLOCK)
    return {"out": out, "weight": weight} if c["weights"] else {"out": out}


def _exact_evict(c, s):
    if s["k_codes"].numel() > 1 << 29:
        return None
    host = _Host(s)
    budget, recent = c["budget"], c["recent"]
    for b in range(c["seqs"]):
        length = int(host.lengths[b])
        if length <= budget:
            continue
        ids = host.table[b]
        for h in range(c["kv_heads"]):
            w = host.weight[ids, h].reshape(-1)[:length]
            pos = host.pos[ids, h].reshape(-1)[:length]
            safe = pos > pos.max() - recent
            # by protection, then weight, then the lowest slot
            order = np.lexsort((np.arange(length), -w, ~safe))
            keep = np.zeros(length, bool)
            keep[order[:budget]] = True
            holes = np.flatnonzero(~keep[:budget])
            moved = budget + np.flatnonzero(keep[budget:])
            took = {n: getattr(host, n)[ids[moved // BLOCK], h, moved % BLOCK].copy()
                    for n in ("k", "v", "pos", "weight")}
            kx = took["k"] * host.ks[ids[moved // BLOCK], h][:, None]
            vx = took["v"] * host.vs[ids[moved // BLOCK], h][:, None]
            for j in np.unique(holes // BLOCK):
                mine = np.flatnonzero(holes // BLOCK == j)
                offs = holes[mine] % BLOCK
                host.put(host.k, host.ks, ids[j], h, offs, kx[mine], False)
                host.put(host.v, host.vs, ids[j], h, offs, vx[mine], False)
                host.pos[ids[j], h, offs] = took["pos"][mine]
                host.weight[ids[j], h, offs] = took["weight"][mine]
    return dict(host.out(), lengths=np.minimum(host.lengths, budget))


def _exact_w4(c, s):
    g = c["group"]
    out = torch.empty((c["rows"], c["outs"]), dtype=torch.float64, device="cuda")
    x = s["x"].double()
    for b in range(0, c["outs"], 4096):
        e = min(c["outs"], b + 4096)
        z = s["zero"][b:e].double().repeat_interleave(g, 1)
        f = s["scale"][b:e].double().repeat_interleave(g, 1)
        out[:, b:e] = x @ ((s["codes"][b:e].double() - z) * f).t().contiguous()
    return out
