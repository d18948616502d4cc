"""The operators of a serving instance that checks drafted tokens, by which their
speed is followed: appends that turn keys and queries by their positions on the
way into the 8-bit token cache, rows coded in 8-bit floating point, products of
such rows with 8-bit weights, and the verification of drafted tokens.  ``own``
chooses between the package's kernels and the plain form of the same definitions.

A case says which operator runs (``op``) and on what:

  rotate   new tokens into the cache, keys and queries turned by their positions
           (on one axis, or on three: time, height and width)
  rows     rows of 16 bits as e4m3 codes with a scale for 128 inputs
  product  coded rows times a matrix of e4m3 codes with a scale for 128 x 128
  verify   drafted tokens against the target's probabilities

The cache is a pool of blocks of 64 slots: keys as [block, kv head, slot, dim],
values as [block, kv head, 4, dim, 16], slot t of a block in group (t / 4) % 4,
there at place (t / 16) * 4 + t % 4; one power-of-two scale for a block and head.
Coded rows and weights are held in tiles of 16 rows and 128 inputs, [tile, input
block, 8, 16, 16]: input k of row r of a tile at [k / 16, r, k % 16].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 64                                # slots of a cache block
WIDE = 128                                # inputs under one scale
TILE = 16                                 # rows of a tile
TOP = {"e4m3": 448.0, "int8": 127.0}      # largest code
LEAST = -100                              # least exponent of a scale
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# where a value's slot stands inside its block: group * 16 + place
PLACE = [((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3) for t in range(BLOCK)]


# -- cases --------------------------------------------------------------------

def _rotate(seqs, heads, kv_heads, dim, length, **more):
    c = {"op": "rotate", "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "length": length,        # slots of the longest sequence, new ones included
         "new": 1,                # new tokens of a sequence (the most of any)
         "turned": dim,           # dims that turn
         "pairs": "halves",       # dim i with i + turned / 2, or "neighbours" 2i with 2i + 1
         "axes": 1, "format": "e4m3", "type": "bf16"}
    return dict(c, **more)


def _verify(seqs, drafts, words, **more):
    return dict({"op": "verify", "seqs": seqs,
                 "drafts": drafts,        # drafted tokens of a sequence (the most of any)
                 "words": words, "type": "f32",
                 "drawn": True},          # drafts drawn from probabilities that are given
                **more)


def _rows8(rows, ins, kind="bf16"):
    return {"op": "rows", "rows": rows, "ins": ins, "type": kind}


def _product(rows, outs, ins, kind="bf16"):
    return {"op": "product", "rows": rows, "outs": outs, "ins": ins, "type": kind}


def listed():
    cases = {
        # one decode step of a batch: a token a sequence
        "rotate_token": _rotate(64, 32, 8, 128, 2048),
        # a few drafted tokens each, odd heads, an odd width of which half turns
        "rotate_drafts": _rotate(7, 20, 4, 80, 1500, new=3, turned=40, pairs="neighbours",
                                 format="int8", type="f16"),
        # ragged prompts with pictures: three positions a token
        "rotate_prompt": _rotate(6, 32, 8, 128, 2500, new=2100, axes=3),
        # the inputs of one token's projection: all latency
        "rows_token": _rows8(1, 4096),
        # a long prompt's inner activations
        "rows_prompt": _rows8(8000, 16384),
        # one token through a square projection
        "product_token": _product(1, 4096, 4096),
        # a decode batch with drafts through a wide projection
        "product_drafts": _product(96, 16384, 4096),
        # odd sizes: a ragged batch of short prompts onto an odd vocabulary
        "product_odd": _product(777, 20001, 5000, "f16"),
        # a long prompt through the wide projection
        "product_prompt": _product(8192, 16384, 4096),
        # one request alone with four drafts
        "verify_one": _verify(1, 4, 32000),
        # a batch whose drafts were looked up, not drawn; 16-bit probabilities, odd vocabulary
        "verify_lookup": _verify(48, 7, 50001, type="bf16", drawn=False),
        # a full instance, a large vocabulary
        "verify_batch": _verify(256, 4, 131072),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["rotate", "rotate", "rows", "product", "product", "product", "verify",
                     "verify"])
    kind = rng.choice(["bf16", "f16"])
    if op == "rows":
        return _rows8(_log(rng, 1, 8000), _log(rng, 200, 16384), kind)
    if op == "product":
        rows = _log(rng, 1, 8192)
        few = rows < 1000
        return _product(rows, _log(rng, 300, 20001 if few else 16384),
                        _log(rng, 500, 16384 if few else 4096), kind)
    if op == "verify":
        drafts = rng.randrange(0, 8)
        return _verify(_log(rng, 1, 256 if drafts < 5 else 150), drafts, _log(rng, 1000, 131072),
                       type=rng.choice(["f32", "f32", "bf16", "f16"]), drawn=rng.random() < 0.7)
    kv, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 128])
    new = rng.choice([1, rng.randrange(2, 8), _log(rng, 9, 2100)])
    return _rotate(_log(rng, 1, 128 if new < 9 else 6), kv * rng.choice([1, 2, 4, 5]), kv, dim,
                   new + _log(rng, 1, 2000), new=new,
                   turned=rng.choice([dim, dim, dim // 2, 2 * rng.randrange(1, dim // 2)]),
                   pairs=rng.choice(["halves", "neighbours"]), axes=rng.choice([1, 1, 3]),
                   format=rng.choice(["e4m3", "int8"]), type=kind)


def _share(k):
    """A number in (0, 1) for sequence k, spread evenly."""
    return ((k + 1) * 0.6180339887498949) % 1.0


def _lengths(c):
    """(length, new tokens) of each sequence: the first the longest, in a batch
    of four or more the second without a token."""
    most = c["drafts"] + 1 if c["op"] == "verify" else c["new"]
    longest = 1000 if c["op"] == "verify" else c["length"]
    out = []
    for k in range(c["seqs"]):
        u = 1.0 if k == 0 else _share(k)
        n = max(1, int(round(most * u)))
        out.append((max(n, int(longest * u)), n))
    if c["seqs"] >= 4:
        out[1] = (0, 0)
    return out


def work(case):
    c = case
    if c["op"] == "rows":
        m, k = c["rows"], c["ins"]
        return {"bytes": m * (3 * k + 4 * -(-k // WIDE)), "flops": 3 * m * k}
    if c["op"] == "product":
        m, n, k = c["rows"], c["outs"], c["ins"]
        blocks = -(-k // WIDE)
        return {"bytes": m * k + n * k + 4 * blocks * (m + -(-n // WIDE)) + 2 * m * n,
                "flops": 2 * m * n * k}
    rows = sum(n for _, n in _lengths(c))
    if c["op"] == "verify":
        # one row of the target's of each sequence, and one of the draft's where a token is
        # refused (counted for three sequences of four)
        size = 4 if c["type"] == "f32" else 2
        live = sum(n > 0 for _, n in _lengths(c))
        refused = 0.75 if c["drafts"] and c["drawn"] else 0.0
        return {"bytes": live * c["words"] * size * (1 + refused) + rows * (8 + 2 * size),
                "flops": live * c["words"] * 3}
    d, kv, h = c["dim"], c["kv_heads"], c["heads"]
    return {"bytes": rows * (4 * h * d + kv * (6 * d + 8) + 4 * c["turned"] + 4 * c["axes"]),
            "flops": rows * (3 * (h + kv) * c["turned"] + 6 * kv * d)}


# -- inputs -------------------------------------------------------------------

def _as_held(x):
    """Values slot by slot [.., 64, dim], as they are held [.., 4, dim, 16]."""
    at = torch.argsort(torch.tensor(PLACE, device=x.device))
    return x[..., at, :].unflatten(-2, (4, 16)).transpose(-1, -2)


def _power(a, fmt):
    """The least power of two that holds magnitude a in a code, 2^LEAST at least."""
    m, e = torch.frexp(a)
    top_m, top_e = math.frexp(TOP[fmt])
    e = torch.where(a > 0, e - top_e + (m > top_m).to(e.dtype), torch.full_like(e, LEAST))
    return ((e.clamp(min=LEAST) + 127).int() << 23).view(torch.float32)


def _encode(y, fmt):
    """Codes (as bytes) of values over their scale."""
    y = y.clamp(-TOP[fmt], TOP[fmt])
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(y.isnan(), 0.0, y).round().to(torch.int8).view(torch.uint8)


def _tiles(codes):
    """Codes [rows, ins] (bytes) as tiles, zeros past the last row and input."""
    rows, ins = codes.shape
    r, b = -(-rows // TILE), -(-ins // WIDE)
    codes = torch.nn.functional.pad(codes, (0, b * WIDE - ins, 0, r * TILE - rows))
    return codes.view(r, TILE, b, 8, 16).permute(0, 2, 3, 1, 4).contiguous()


def _coded(x):
    """Rows as codes in tiles and scales [input block, row]."""
    rows, ins = x.shape
    r, b = -(-rows // TILE) * TILE, -(-ins // WIDE)
    x = torch.nn.functional.pad(x.float(), (0, b * WIDE - ins, 0, r - rows)).view(r, b, WIDE)
    scale = _power(torch.where(x.isfinite(), x.abs(), 0.0).amax(-1), "e4m3")
    codes = _encode(x / scale[..., None], "e4m3").view(r, b * WIDE)
    return _tiles(codes).view(torch.float8_e4m3fn), scale.t().contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"rotate": _prepare_rotate, "rows": _prepare_rows, "product": _prepare_product,
            "verify": _prepare_verify}[case["op"]](case, gen)


def _activations(gen, rows, ins, kind):
    """Rows whose channels differ in size, some by far."""
    channel = torch.exp(0.8 * torch.randn((1, ins), generator=gen, device="cuda"))
    return (torch.randn((rows, ins), generator=gen, device="cuda") * channel).to(TYPE[kind])


def _prepare_rows(c, gen):
    return {"case": c, "x": _activations(gen, c["rows"], c["ins"], c["type"])}


def _prepare_product(c, gen):
    m, n, k = c["rows"], c["outs"], c["ins"]
    codes, scale = _coded(_activations(gen, m, k, c["type"]))
    weight = torch.randn((n, k), generator=gen, device="cuda").mul_(110.0).clamp_(-448.0, 448.0)
    w = {"codes": weight.to(torch.float8_e4m3fn),
         "scale": 4e-4 * (0.5 + torch.rand((-(-n // WIDE), -(-k // WIDE)), generator=gen,
                                           device="cuda"))}
    s = {"case": c, "codes": codes, "scale": scale, "w": w}
    if own:
        from paper_2407_00047_amd import qlm
        s["rows"] = qlm.F8Rows(codes, scale, m, k)
        s["weight"] = qlm.f8_pack(w["codes"], w["scale"])
        s["ws"] = qlm.f8_workspace(s["weight"], m)
    return s


def _batch(c):
    """Rows' starts, lengths, the most rows and the most slots of a sequence."""
    both = _lengths(c)
    start = torch.tensor(np.concatenate([[0], np.cumsum([n for _, n in both])]).astype(np.int32))
    return {"row_start": start.to("cuda"), "n_rows": int(start[-1]),
            "lengths": torch.tensor([x for x, _ in both], dtype=torch.int32, device="cuda"),
            "max_new": max(n for _, n in both), "max_length": max(x for x, _ in both)}


def _prepare_verify(c, gen):
    s = dict(_batch(c), case=c)
    rows, words = s["n_rows"], c["words"]
    logits = 2.5 * torch.randn((rows, words), generator=gen, device="cuda")
    # a draft model that is a little off the target
    near = logits + 0.7 * torch.randn((rows, words), generator=gen, device="cuda")
    s["target"] = torch.softmax(logits, -1).to(TYPE[c["type"]])
    near = torch.softmax(near, -1)
    s["draft"] = near.to(TYPE[c["type"]]) if c["drawn"] else None
    # (the token of row r + 1 was drawn by the draft model behind row r)
    noise = torch.rand((rows, words), generator=gen, device="cuda").clamp_(min=1e-12)
    s["tokens"] = torch.roll((near / -noise.log_()).argmax(-1), 1).int()
    s["uniform"] = torch.rand(rows, generator=gen, device="cuda")
    if own:
        from paper_2407_00047_amd import qlm
        table = torch.zeros((c["seqs"], -(-s["max_length"] // BLOCK)), dtype=torch.int32,
                            device="cuda")
        s["batch"] = qlm.KvBatch(table, s["lengths"], s["row_start"], rows, s["max_new"],
                                 s["max_length"])
        s["ws"] = qlm.draft_verify_workspace(s["batch"], words)
    return s


def _prepare_rotate(c, gen):
    dev = "cuda"
    rnd = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    kv, d, fmt, seqs = c["kv_heads"], c["dim"], c["format"], c["seqs"]
    s = dict(_batch(c), case=c)
    blocks = (-(-s["lengths"].cpu().long() // BLOCK)).tolist()
    width, total = max(1, max(blocks)), sum(blocks)
    # the pool's blocks in any order; the last one belongs to nobody
    order = torch.randperm(total, generator=gen, device=dev).cpu()
    table = torch.full((seqs, width), total, dtype=torch.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = table.to(dev)
    n_blocks = total + 1
    channel = torch.exp(0.7 * rnd(kv, 1, d))
    for name, x in (("k", rnd(n_blocks, kv, BLOCK, d) * channel), ("v", rnd(n_blocks, kv, BLOCK, d))):
        scale = _power(x.abs().amax(dim=(2, 3)), fmt)
        codes = _encode(x / scale[:, :, None, None], fmt)
        codes = codes if name == "k" else _as_held(codes).contiguous()
        s[name + "_codes"], s[name + "_scale"] = codes.view(CODE[fmt]), scale
    s["position"] = torch.randint(0, 1000, (n_blocks, kv, BLOCK), generator=gen, device=dev,
                                  dtype=torch.int32)
    s["weight"] = torch.exp(2.0 * rnd(n_blocks, kv, BLOCK))
    rows = s["n_rows"]
    dt = TYPE[c["type"]]
    # one product's outputs: queries, keys and values beside each other
    qkv = torch.cat([rnd(rows, c["heads"], d), rnd(rows, kv, d) * channel[None, :, 0],
                     rnd(rows, kv, d)], 1).to(dt)
    s["q"], s["k"], s["v"] = qkv.split([c["heads"], kv, kv], 1)
    # positions run ahead of slots where tokens were given up
    n = s["row_start"][1:] - s["row_start"][:-1]
    ahead = torch.randint(0, 4000, (seqs,), generator=gen, device=dev, dtype=torch.int32)
    s["first"] = s["lengths"] - n + ahead
    seq = torch.repeat_interleave(torch.arange(seqs, device=dev), n.long(), output_size=rows)
    i = torch.arange(rows, device=dev, dtype=torch.int32) - s["row_start"][seq]
    one = s["first"][seq] + i
    # pictures of 24 x 24 tokens among the text: one time, its rows and columns
    picture = (i // 576) % 2 == 1
    base = s["first"][seq] + i // 576 * 576
    grid = torch.stack([base, base + i % 576 // 24, base + i % 24])
    s["where"] = (torch.where(picture, grid, one) if c["axes"] == 3 else one[None]).contiguous()
    # 16384 positions, angles in 64 bits
    half = c["turned"] // 2
    freq = 10000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
    angle = torch.arange(16384, device=dev, dtype=torch.float64)[:, None] * freq
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    s["axis"] = None
    if c["axes"] == 3:           # a quarter of the pairs for the time, the others by turns
        share = torch.arange(half, device=dev) * 8 // half
        s["axis"] = torch.where(share < 2, 0, torch.where(share < 5, 1, 2)).int()
    if own:
        from paper_2407_00047_amd import qlm
        s["cache"] = qlm.DeviceKvCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"],
                                       s["position"], s["weight"])
        s["batch"] = qlm.KvBatch(s["table"], s["lengths"], s["row_start"], rows, s["max_new"],
                                 s["max_length"])
        s["rotary"] = qlm.Rotary(s["cos"], s["sin"], interleaved=c["pairs"] == "neighbours",
                                 axis=s["axis"])
    return s


# -- one pass -----------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    return (_own if own else _plain)[op](s)


def _cache_out(s, q):
    return dict({n: s[n] for n in ("k_codes", "v_codes", "k_scale", "v_scale", "position",
                                   "weight")}, q=q)


def _own_rotate(s):
    from paper_2407_00047_amd import qlm
    q = qlm.kv_append_rotated(s["cache"], s["batch"], s["k"], s["v"], s["q"], s["rotary"],
                              position=s["where"], first_position=s["first"])
    return _cache_out(s, q)


def _own_rows(s):
    from paper_2407_00047_amd import qlm
    got = qlm.f8_rows(s["x"])
    return {"codes": got.codes, "scale": got.scale}


def _own_product(s):
    from paper_2407_00047_amd import qlm
    return qlm.f8_matmul(s["rows"], s["weight"], dtype=TYPE[s["case"]["type"]], ws=s["ws"])


def _own_verify(s):
    from paper_2407_00047_amd import qlm
    tokens, count, lengths = qlm.draft_verify(s["batch"], s["tokens"], s["target"], s["draft"],
                                              s["uniform"], ws=s["ws"])
    return {"tokens": tokens, "count": count, "lengths": lengths}


def _write(x, codes, scale, fmt, blk, off, first_blk, held):
    """New values x [row, head, dim] into the keys' or the values' codes."""
    a = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    need = torch.zeros_like(scale).scatter_reduce(0, blk[:, None].expand_as(a), a, "amax")
    none = torch.zeros_like(scale[:, 0])
    hit = none.scatter_reduce(0, blk, torch.ones_like(none[blk]), "amax") > 0
    fresh = none.scatter_reduce(0, blk, (off == 0).float(), "amax") > 0
    old = torch.where(fresh[:, None], 0.0, scale)
    grown = torch.where(hit[:, None], torch.maximum(old, _power(need, fmt)), scale)
    # the codes held by a block whose scale grows (only a sequence's first block holds any)
    ratio = torch.where(held[:, None], scale[first_blk] / grown[first_blk], 1.0)
    raw = codes.view(torch.uint8)
    was = codes[first_blk].float()
    raw[first_blk] = _encode(was * ratio.view(ratio.shape + (1,) * (was.ndim - 2)), fmt)
    scale.copy_(grown)
    y = _encode(x / scale[blk][:, :, None], fmt)
    heads = torch.arange(scale.shape[1], device=x.device)
    if raw.ndim == 4:
        raw[blk[:, None], heads, off[:, None]] = y
    else:
        at = torch.tensor(PLACE, device=x.device)[off]
        raw.view(*raw.shape[:2], 4, -1, 16)[blk[:, None], heads, at[:, None] // 16, :,
                                            at[:, None] % 16] = y


def _turn(x, cos, sin, pairs):
    """x [row, head, dim] turned by angles [row, pair], in single precision."""
    x = x.float()
    half = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    if pairs == "halves":
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _plain_rotate(s):
    c = s["case"]
    fmt, dev = c["format"], s["q"].device
    half = c["turned"] // 2
    pair = torch.arange(half, device=dev)
    at = s["where"].long()[s["axis"].long() if s["axis"] is not None else 0 * pair]
    at = at.clamp(0, s["cos"].shape[0] - 1).t()                        # [row, pair]
    cos, sin = s["cos"][at, pair], s["sin"][at, pair]
    q = _turn(s["q"], cos, sin, c["pairs"]).to(s["q"].dtype)
    k, v = _turn(s["k"], cos, sin, c["pairs"]), s["v"].float()
    n = (s["row_start"][1:] - s["row_start"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=dev), n, output_size=s["n_rows"])
    i = torch.arange(s["n_rows"], device=dev) - s["row_start"].long()[seq]
    start = s["lengths"].long() - n
    slot = start[seq] + i
    table = s["table"].long()
    blk, off = table[seq, slot // BLOCK], slot % BLOCK
    held = (n > 0) & (start > 0) & (start % BLOCK != 0)
    first_blk = table.gather(1, (start // BLOCK).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    _write(k, s["k_codes"], s["k_scale"], fmt, blk, off, first_blk, held)
    _write(v, s["v_codes"], s["v_scale"], fmt, blk, off, first_blk, held)
    heads = torch.arange(c["kv_heads"], device=dev)
    s["position"][blk[:, None], heads, off[:, None]] = (s["first"][seq] + i).int()[:, None]
    s["weight"][blk[:, None], heads, off[:, None]] = 0.0
    return _cache_out(s, q)


def _plain_rows(s):
    codes, scale = _coded(s["x"])
    return {"codes": codes, "scale": scale}


def _plain_product(s):
    m, n, k = (s["case"][x] for x in ("rows", "outs", "ins"))
    x = s["codes"].float() * s["scale"].view(s["scale"].shape[0], -1, TILE).permute(
        1, 0, 2)[:, :, None, :, None]
    x = x.permute(0, 3, 1, 2, 4).reshape(-1, s["scale"].shape[0] * WIDE)[:m, :k]
    scale = s["w"]["scale"].repeat_interleave(WIDE, 0)[:n].repeat_interleave(WIDE, 1)[:, :k]
    return torch.matmul(x, (s["w"]["codes"].float() * scale).t()).to(TYPE[s["case"]["type"]])


def _plain_verify(s):
    # (64 bits: which word a number falls on is decided next to a border of long sums)
    start, tokens = s["row_start"].long(), s["tokens"]
    n = start[1:] - start[:-1]
    place = torch.arange(s["max_new"], device=n.device)
    rows = (start[:-1, None] + place).clamp(max=s["n_rows"] - 1)         # [sequence, place]
    after = tokens[(rows + 1).clamp(max=s["n_rows"] - 1)].long()
    p = s["target"][rows, after].double()
    q = s["draft"][rows, after].double() if s["draft"] is not None else torch.ones_like(p)
    good = (s["uniform"][rows].double() * q < p) & (place < n[:, None] - 1)
    kept = good.long().cumprod(-1).sum(-1)                               # accepted drafts
    row = (start[:-1] + kept).clamp(max=s["n_rows"] - 1)
    p = s["target"][row].double()
    refused = (kept < n - 1)[:, None]
    if s["draft"] is not None:
        q = s["draft"][row].double()
    else:
        token = tokens[(row + 1).clamp(max=s["n_rows"] - 1)].long()
        q = torch.zeros_like(p).scatter_(1, token[:, None], 1.0)
    left = torch.where(refused, (p - q).clamp(min=0.0), p)
    left = torch.where(left.sum(-1, keepdim=True) > 0, left, p)
    below = left.cumsum(-1)
    u = s["uniform"][(start[1:] - 1).clamp(min=0)].double()
    word = (below <= (u * below[:, -1])[:, None]).sum(-1)
    count = torch.where(n > 0, kept + 1, 0)
    out = torch.where(place < kept[:, None], after, -1)
    out = torch.where(place == kept[:, None], word[:, None], out)
    out = torch.where(n[:, None] > 0, out, -1)
    return {"tokens": out.int(), "count": count.int(),
            "lengths": (s["lengths"] - (n - count).int()).clamp(min=0)}


_own = {"rotate": _own_rotate, "rows": _own_rows, "product": _own_product, "verify": _own_verify}
_plain = {"rotate": _plain_rotate, "rows": _plain_rows, "product": _plain_product,
          "verify": _plain_verify}


# -- the definitions in 64 bits -----------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "rows": _exact_rows, "product": _exact_product,
            "verify": _exact_verify}[case["op"]](case, s)


def _two_to(e):
    """2^e in 64 bits, from the bits (a power function may round)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_scale(a, fmt):
    """2^e of the least e >= LEAST with a <= top 2^e."""
    e = torch.ceil(torch.log2((a / TOP[fmt]).clamp(min=1e-300)))
    e = torch.where(a > TOP[fmt] * _two_to(e), e + 1, e)          # (log2 rounds)
    e = torch.where(a <= TOP[fmt] * _two_to(e - 1), e - 1, e)
    return _two_to(e.clamp(min=LEAST))


def _exact_e4m3(y):
    """The value of the nearest code, ties to even: steps of an eighth of y's power of two,
    of 2^-9 below 2^-6."""
    y = y.clamp(-448.0, 448.0)
    step = _two_to(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _exact_rows(c, s):
    m, k = c["rows"], c["ins"]
    x = s["x"].double()
    tiles, blocks = -(-m // TILE), -(-k // WIDE)
    codes = torch.zeros((tiles, blocks, 8, TILE, 16), dtype=torch.float64, device=x.device)
    scale = torch.full((blocks, tiles * TILE), 2.0 ** LEAST, dtype=torch.float64, device=x.device)
    for b in range(blocks):
        part = x[:, b * WIDE:(b + 1) * WIDE]
        by = _exact_scale(part.abs().amax(-1), "e4m3")
        scale[b, :m] = by
        got = torch.zeros((tiles * TILE, WIDE), dtype=torch.float64, device=x.device)
        got[:m, :part.shape[1]] = _exact_e4m3(part / by[:, None])
        codes[:, b] = got.view(tiles, TILE, 8, 16).transpose(1, 2)
    return {"codes": codes, "scale": scale}


def _exact_product(c, s):
    m, n, k = c["rows"], c["outs"], c["ins"]
    out = torch.zeros((m, n), dtype=torch.float64, device=s["codes"].device)
    for b in range(-(-k // WIDE)):
        x = s["codes"][:, b].double().permute(0, 2, 1, 3).reshape(-1, WIDE)[:m]
        w = s["w"]["codes"][:, b * WIDE:(b + 1) * WIDE].double()
        by = s["w"]["scale"][:, b].double().repeat_interleave(WIDE)[:n]
        out += (x[:, :w.shape[1]] * s["scale"][b, :m, None].double()) @ (w * by[:, None]).t()
    return out


def _exact_rotate(c, s):
    """Queries and scales; the codes in e4m3 (of 8-bit integers, whole numbers, none)."""
    where = s["where"].cpu().numpy().clip(0, s["cos"].shape[0] - 1)
    cos, sin = s["cos"].cpu().numpy().astype(np.float64), s["sin"].cpu().numpy().astype(np.float64)
    half = c["turned"] // 2
    axis = np.zeros(half, np.int64) if s["axis"] is None else s["axis"].cpu().numpy()

    def turn(x):
        x = x.double().cpu().numpy()
        y = x.copy()
        for i in range(half):
            a, b = (i, i + half) if c["pairs"] == "halves" else (2 * i, 2 * i + 1)
            p = where[axis[i]]
            z = (x[..., a] + 1j * x[..., b]) * (cos[p, i] + 1j * sin[p, i])[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        return torch.from_numpy(y).cuda()

    got = {"q": turn(s["q"]), "position": None, "weight": None}
    fmt = c["format"]
    for name, x in (("k", turn(s["k"])), ("v", s["v"].double())):
        codes, scale = s[name + "_codes"].double(), s[name + "_scale"].double()
        at = torch.argsort(torch.tensor(PLACE, device=x.device))
        if name == "v":                     # slot by slot
            codes = codes.transpose(-1, -2).flatten(-3, -2)[..., torch.argsort(at), :]
        row = 0
        for b, (length, n) in enumerate(_lengths(c)):
            for j in range((length - n) // BLOCK, -(-length // BLOCK) if n else 0):
                lo, hi = max(length - n, j * BLOCK), min(length, (j + 1) * BLOCK)
                blk, o = int(s["table"][b, j]), lo % BLOCK
                new = x[row + lo - (length - n):row + hi - (length - n)].transpose(0, 1)
                need = _exact_scale(new.abs().amax(dim=(1, 2)), fmt)
                if o:
                    now = torch.maximum(scale[blk], need)
                    if fmt == "e4m3":
                        codes[blk] = _exact_e4m3(codes[blk] * (scale[blk] / now)[:, None, None])
                    need = now
                scale[blk] = need
                if fmt == "e4m3":
                    codes[blk, :, o:o + hi - lo] = _exact_e4m3(new / need[:, None, None])
            row += n
        if name == "v":
            codes = codes[..., at, :].unflatten(-2, (4, 16)).transpose(-1, -2)
        got[name + "_codes"] = codes if fmt == "e4m3" else None
        got[name + "_scale"] = scale
    return got


def _exact_verify(c, s):
    both = _lengths(c)
    most = s["max_new"]
    tokens = np.full((c["seqs"], most), -1, np.int32)
    count, lengths = np.zeros(c["seqs"], np.int32), np.zeros(c["seqs"], np.int32)
    given, uniform = s["tokens"].cpu().numpy(), s["uniform"].cpu().numpy().astype(np.float64)
    row = 0
    for b, (length, n) in enumerate(both):
        lengths[b] = length
        if n == 0:
            continue
        kept = 0
        while kept < n - 1:
            t = int(given[row + kept + 1])
            q = float(s["draft"][row + kept, t]) if s["draft"] is not None else 1.0
            if not uniform[row + kept] * q < float(s["target"][row + kept, t]):
                break
            tokens[b, kept] = t
            kept += 1
        left = s["target"][row + kept].double().cpu().numpy()
        if kept < n - 1:
            q = np.zeros_like(left)
            if s["draft"] is not None:
                q = s["draft"][row + kept].double().cpu().numpy()
            else:
                q[given[row + kept + 1]] = 1.0
            rest = np.maximum(left - q, 0.0)
            left = rest if rest.sum() > 0 else left
        below = np.cumsum(left)
        tokens[b, kept] = np.searchsorted(below, uniform[row + n - 1] * below[-1], side="right")
        count[b], lengths[b] = kept + 1, length - (n - kept - 1)
        row += n
    return {"tokens": tokens, "count": count, "lengths": lengths}
