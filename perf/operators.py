"""What is measured of the key/value cache operators: appending to a paged cache (4-bit or 16-bit),
selecting blocks of it by a cheap score, and attending over the whole cache or over the selected
blocks.  Each case is a dict of plain values; `run` is one pass in plain torch operations (32 bits,
rounded once at the end) or, where `own` is set, through the library's entry points.

Cache formats.  16-bit: keys and values [pages, kv heads, page, d] (any strides).  4-bit: per 16 tokens
of a page and kv head one record of 18 d bytes; a token's d elements are in groups of 64, a group holds
16-bit (scale s, offset z) and codes u = 0..15 that stand for s u + z.  Record (planes p of
D = min(d, 128) elements, D / 64 groups each):
  keys     [p][token 16][c 4][group][h 2][nibble 8]: element 64 group + 16 c + 8 h + nibble of the plane
  values   [p][octet 2][r 8][c 4][parity 2][nibble D / 8]: token 8 octet + 2 c + parity, element D/8 r + nibble
  key parameters    [token 16][group of d][s, z]
  value parameters  [octet 2][group of d][c 4][s of parity 0, s of parity 1, z of parity 0, z of parity 1]
Two codes per byte, the lower nibble first.

Block bounds: for each full page and kv head the largest and the smallest key value of every channel,
in 8 bits with one scale (largest magnitude / 127).
"""

import math

import torch

own = False

HELD = {"bf16": torch.bfloat16, "fp16": torch.float16}
GOLDEN = 0.6180339887498949


# ---- cases -------------------------------------------------------------------------------------

def _case(name, op, **kw):
    c = dict(name=name, op=op, fmt="int4", dtype="bf16", d=128, hkv=8, group=4, page=64, nreq=1, len_lo=1024, len_hi=1024,
             new_lo=1, new_hi=1, nsel=0, sink=1, local=2, empty=False, layout="hnd")
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of a few conversations: one token each, latency counts
        _case("append_step", "append", nreq=7, len_lo=64, len_hi=5000, empty=True),
        # a batch of prompts of odd lengths, written to the 4-bit cache in one call
        _case("append_prompts", "append", nreq=9, len_lo=1500, len_hi=4099, new_lo=700, new_hi=4099),
        # further turns of running conversations, 16-bit cache with the head axis inside the token's
        _case("append_turns_16bit", "append", fmt="fp16", dtype="fp16", d=64, hkv=5, page=32, nreq=12, len_lo=600, len_hi=3001,
              new_lo=33, new_hi=600, layout="nhd"),
        # one long conversation, one new token: blocks chosen among two thousand
        _case("select_one_long", "select", len_lo=131050, len_hi=131050, nsel=64),
        # a decode batch of ragged lengths, small pages
        _case("select_batch", "select", d=128, page=32, nreq=64, len_lo=900, len_hi=32000, nsel=48, group=8, empty=True),
        # a chunk of a long prompt: every token chooses its own blocks
        _case("select_prompt", "select", fmt="bf16", nreq=1, len_lo=32768, len_hi=32768, new_lo=2048, new_hi=2048, nsel=16),
        # the whole 4-bit cache, one short conversation: latency counts
        _case("full4_short", "attend", nreq=1, len_lo=333, len_hi=333),
        # the whole 4-bit cache of one long conversation
        _case("full4_one_long", "attend", nreq=1, len_lo=100003, len_hi=100003, group=8),
        # a full decode batch of ragged lengths
        _case("full4_batch", "attend", nreq=64, len_lo=500, len_hi=16000, group=8, empty=True),
        # several drafted tokens per request, checked in one call; narrow heads
        _case("full4_drafts", "attend", dtype="fp16", d=64, hkv=4, group=7, page=16, nreq=17, len_lo=100, len_hi=9001, new_lo=2, new_hi=6),
        # a decode batch over selected blocks of a 16-bit cache
        _case("sparse_batch", "attend", fmt="bf16", nreq=48, len_lo=3000, len_hi=20000, nsel=40, empty=True),
        # a chunk of a prompt, every token over its own selected blocks
        _case("sparse_prompt", "attend", fmt="bf16", nreq=1, len_lo=8192, len_hi=8192, new_lo=2048, new_hi=2048, nsel=16, group=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw(rng)
        if _cost(c) <= _cost(listed()[-1]) and _plain_cells(c) <= 2 ** 30 and work(c)["bytes"] <= 3e9:
            return c


def _draw(rng):
    kind = rng.choice(["append", "append", "select", "select", "full", "full", "full", "sparse", "sparse", "sparse"])
    fmt = "int4" if kind == "full" else rng.choice(["int4", "int4", "bf16", "fp16"])
    dtype = fmt if fmt != "int4" else rng.choice(["bf16", "fp16"])
    c = _case("", "attend" if kind in ("full", "sparse") else kind, fmt=fmt, dtype=dtype, d=rng.choice([64, 128, 128, 256]), hkv=rng.choice([1, 2, 4, 5, 8]),
              group=rng.choice([1, 3, 4, 7, 8, 16]), page=rng.choice([16, 32, 64, 64, 128]), layout=rng.choice(["hnd", "nhd"]) if fmt != "int4" else "hnd")
    many = rng.random() < 0.25            # a prompt or a further turn rather than single tokens
    c["nreq"] = _log(rng, 1, 6) if many else _log(rng, 1, 96)
    c["len_hi"] = _log(rng, 65, 9000) if many else _log(rng, 30, 60000)
    c["len_lo"] = rng.randint(max(1, c["len_hi"] // 8), c["len_hi"])
    if kind == "append":
        c["new_hi"] = min(c["len_lo"], _log(rng, 2, 4000)) if many else 1
    elif kind == "full":
        c["new_hi"] = min(c["len_lo"], _log(rng, 1, 12))
    else:
        c["new_hi"] = min(c["len_lo"], _log(rng, 2, 2500)) if many else 1
    c["new_lo"] = rng.randint(max(1, c["new_hi"] // 3), c["new_hi"])
    if kind in ("select", "sparse"):
        c["nsel"], c["sink"], c["local"] = _log(rng, 4, 96), rng.randint(0, 2), rng.randint(1, 2)
    c["empty"] = c["nreq"] > 2 and rng.random() < 0.3
    del c["name"]
    return c


def _lengths(c):
    """Tokens held by each request after the call, and how many of them are new: spread evenly over the case's ranges."""
    held, new = [], []
    for i in range(c["nreq"]):
        a, b = (i * GOLDEN) % 1.0, (i * GOLDEN * GOLDEN + 0.25 * (i > 0)) % 1.0
        held.append(int(round(c["len_hi"] - a * (c["len_hi"] - c["len_lo"]))))
        new.append(min(held[-1], int(round(c["new_hi"] - b * (c["new_hi"] - c["new_lo"])))))
    if c["empty"]:                        # an unused slot of a batch of fixed size: a token that sees nothing
        held[-1], new[-1] = 0, 1
    return held, new


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _plain_cells(c):
    """Values of the largest array that the plain form makes."""
    held, new = _lengths(c)
    wide = -(-max(held) // c["page"]) * c["page"]
    if c["op"] == "append":
        return sum(new) * c["hkv"] * c["d"]
    if c["op"] == "select":
        return c["nreq"] * c["hkv"] * max(max(new) * c["group"] * (wide // c["page"]), wide * c["d"] // 4)
    return c["nreq"] * c["hkv"] * max(max(new) * c["group"] * wide, wide * c["d"])


def work(c):
    held, new = _lengths(c)
    ntok, d, hkv, page = sum(new), c["d"], c["hkv"], c["page"]
    hq = hkv * c["group"]
    token = hkv * (18 * d / 16 if c["fmt"] == "int4" else 4 * d)      # a token's keys and values as held
    if c["op"] == "append":
        done = sum(h // page - (h - n) // page for h, n in zip(held, new) if h)
        # the new tokens are read and written as held, then what is held is read and written as values; bounds of full pages
        part = sum(((h - n) % page) * (h // page > (h - n) // page) for h, n in zip(held, new) if h)
        return {"bytes": ntok * hkv * d * 8 + 2 * ntok * token + part * token / 2 + done * hkv * (4 * d + 8) + _npages(c)[1] * hkv * d * 8, "flops": 0}
    if c["op"] == "select":
        blocks = pairs = 0
        for h, n in zip(held, new):
            blocks += h // page
            pairs += sum((h - n + j + 1) // page for j in range(n) if h)
        return {"bytes": blocks * hkv * (2 * d + 4) + ntok * hq * d * 2 + ntok * hkv * c["nsel"] * 4, "flops": pairs * hq * 4 * d}
    keys = read = 0
    for h, n in zip(held, new):
        if c["nsel"]:
            seen = [min(h - n + j + 1, c["nsel"] * page) for j in range(n) if h]
            keys += sum(seen)
            read += min(h, sum(seen))
        else:
            keys += sum(h - n + j + 1 for j in range(n) if h)
            read += h
    return {"bytes": read * token + ntok * hq * (4 * d + 4) + ntok * hkv * c["nsel"] * 4, "flops": keys * hq * 4 * d}


# ---- inputs ------------------------------------------------------------------------------------

def _npages(c):
    """Columns of the block table, and pages that the new tokens lie in."""
    held, new = _lengths(c)
    cols = max(1, -(-max(held) // c["page"]))
    touched = sum((h - 1) // c["page"] - (h - n) // c["page"] + 1 for h, n in zip(held, new) if h)
    return cols, max(1, touched)


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(seed)
    dev, dt = "cuda", HELD[c["dtype"]]
    held, new = _lengths(c)
    d, hkv, page, nreq = c["d"], c["hkv"], c["page"], c["nreq"]
    ntok, hq = sum(new), hkv * c["group"]
    cols, _ = _npages(c)
    blocks = [-(-h // page) for h in held]
    npages = sum(blocks) + 3
    s = {"c": c, "held": held, "new": new}
    s["seq_len"] = torch.tensor(held, dtype=torch.int32, device=dev)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s["q_start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["req"] = torch.repeat_interleave(torch.arange(nreq, device=dev), torch.tensor(new, device=dev))
    s["pos"] = torch.tensor([h - n + j if h else -1 for h, n in zip(held, new) for j in range(n)], device=dev)
    perm = torch.randperm(npages, generator=g, device=dev)
    table, at = torch.full((nreq, cols), -1, dtype=torch.int32, device=dev), 0
    for i, b in enumerate(blocks):
        table[i, :b] = perm[at:at + b]
        at += b
    s["table"] = table
    channel = 0.6 + 2.0 * torch.rand(hkv, 1, d, generator=g, device=dev) ** 6      # a few wide channels

    def keys(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    if c["op"] == "append":
        s["k"] = (keys(ntok, hkv, d) * channel[:, 0] + 0.3).to(dt)
        s["v"] = (0.7 * keys(ntok, hkv, d)).to(dt)
        s["touched"] = torch.tensor([[i, b] for i, (h, n) in enumerate(zip(held, new)) if h for b in range((h - n) // page, (h - 1) // page + 1)]
                                    or [[0, 0]], device=dev)
        s["touched"] = table[s["touched"][:, 0], s["touched"][:, 1]].clamp(min=0)
    if c["op"] != "select":
        # what is held: block drifts besides the channels, as neighbouring tokens have
        k, v = keys(npages, hkv, page, d), keys(npages, hkv, page, d)
        k = k.mul_(channel).add_(0.5 * keys(npages, hkv, 1, d))
        v = v.mul_(0.7)
        if c["fmt"] == "int4":
            s["records"] = _pack(k.to(dt).float(), v.to(dt).float())
        else:
            for name, x in (("ck", k), ("cv", v)):
                x = x.to(dt)
                s[name] = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if c["layout"] == "nhd" else x
        del k, v
    else:
        if c["fmt"] == "int4":
            s["records"] = torch.zeros(npages, hkv, page // 16, 18 * d, dtype=torch.uint8, device=dev)
        else:
            s["ck"] = torch.zeros(npages, hkv, page, d, dtype=dt, device=dev)
            s["cv"] = s["ck"]
    if c["op"] == "select":
        mid = keys(npages, hkv, d) * channel[:, 0]
        half = (0.8 + keys(npages, hkv, d).abs()) * channel[:, 0]
        s["bounds"], s["bounds_scale"] = _codes(mid + half, mid - half)
    else:
        s["bounds"] = torch.zeros(npages, hkv, 2, d, dtype=torch.int8, device=dev)
        s["bounds_scale"] = torch.zeros(npages, hkv, dtype=torch.float32, device=dev)
    if c["op"] != "append":
        s["q"] = (0.8 * keys(ntok, hq, d)).to(dt)
    if c["op"] == "attend" and c["nsel"]:
        # lists as a selection leaves them: the first and the last blocks, the others alike for neighbouring tokens
        s["blocks"] = torch.full((ntok, hkv, c["nsel"]), -1, dtype=torch.int32, device=dev)
        order = torch.rand(nreq, hkv, cols, generator=g, device=dev)[s["req"]]
        order += 0.5 * torch.rand(ntok // 16 + 1, hkv, cols, generator=g, device=dev)[torch.arange(ntok, device=dev) // 16]
        order += 0.3 * torch.rand(ntok, hkv, cols, generator=g, device=dev)
        b, last = torch.arange(cols, device=dev), (s["pos"] // page)[:, None, None]
        order = order + 9.0 * (b < c["sink"]) + 9.0 * (b > last - c["local"])
        order = torch.where(b <= torch.where(s["pos"][:, None, None] < 0, -1, last), order, torch.tensor(-1.0, device=dev))
        top, at = order.topk(min(c["nsel"], cols), dim=2)
        at = torch.where(top < 0, cols, at).sort(dim=2).values
        s["blocks"][:, :, :at.shape[2]] = torch.where(at == cols, -1, at).to(torch.int32)
    s["out"] = torch.empty(ntok, hq, d, dtype=dt, device=dev)
    s["lse"] = torch.empty(ntok, hq, dtype=torch.float32, device=dev)
    if own:
        import paper_2312_01712_b200 as lib
        s["lib"] = lib
        bounds = dict(bounds=s["bounds"], bounds_scale=s["bounds_scale"])
        s["cache"] = lib.KvCacheHandle(records=s["records"], **bounds) if c["fmt"] == "int4" else lib.KvCacheHandle(k=s["ck"], v=s["cv"], **bounds)
        s["batch"] = lib.KvBatchHandle(s["table"], s["seq_len"], None if c["new_hi"] == 1 else s["q_start"])
    return s


# ---- the 4-bit format and the 8-bit bounds, in plain operations --------------------------------

def _codes(hi, lo):
    """8-bit codes and scale of the channels' bounds [..., d]."""
    top = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
    inv = torch.where(top > 0, 127.0 / top, torch.zeros_like(top))
    both = torch.stack((hi * inv, lo * inv), -2).round().clamp(-127, 127)
    return both.to(torch.int8), (top / 127.0)[..., 0].contiguous()


def _quantize(x):
    """Codes [..., d], scales and offsets [..., d / 64] of values held in 4 bits."""
    x = x.unflatten(-1, (-1, 64)).clamp(-65504, 65504)
    z = x.amin(-1, keepdim=True).half().float()
    s = ((x.amax(-1, keepdim=True) - z) / 15.0).half().float()
    u = torch.where(s > 0, ((x - z) / s).round().clamp(0, 15), torch.zeros_like(x))
    return u.flatten(-2).to(torch.uint8), s[..., 0], z[..., 0]


def _value(u, s, z):
    return (u.float().unflatten(-1, (-1, 64)) * s[..., None] + z[..., None]).flatten(-2)


def _pack(k, v):
    """Records [..., page / 16, 18 d] of keys and values [..., page, d]."""
    d = k.shape[-1]
    k, v = k.unflatten(-2, (-1, 16)), v.unflatten(-2, (-1, 16))
    D, lead = min(d, 128), k.shape[:-2]
    (uk, sk, zk), (uv, sv, zv) = _quantize(k), _quantize(v)
    uk = uk.view(*lead, 16, d // D, D // 64, 4, 2, 8)                 # token, plane, group, c, h, nibble
    uk = uk.permute(*range(len(lead)), -5, -6, -3, -4, -2, -1).flatten(len(lead))
    uv = uv.view(*lead, 2, 4, 2, d // D, 8, D // 8)                   # octet, c, parity, plane, r, nibble
    uv = uv.permute(*range(len(lead)), -3, -6, -2, -5, -4, -1).flatten(len(lead))
    kp = torch.stack((sk, zk), -1).half().flatten(len(lead))
    vp = torch.stack((sv, zv), -1).view(*lead, 2, 4, 2, d // 64, 2)   # octet, c, parity, group, (s, z)
    vp = vp.permute(*range(len(lead)), -5, -2, -4, -1, -3).half().flatten(len(lead))
    codes = torch.cat((uk, uv), -1)
    return torch.cat((codes[..., 0::2] | (codes[..., 1::2] << 4), kp.contiguous().view(torch.uint8), vp.contiguous().view(torch.uint8)), -1)


def _unpack(records, d):
    """Codes, scales and offsets of keys and of values [..., page, d] from records [..., page / 16, 18 d]."""
    lead, D, n = records.shape[:-1], min(d, 128), len(records.shape) - 1
    codes = torch.stack((records[..., :16 * d] & 15, records[..., :16 * d] >> 4), -1).flatten(-2)
    uk = codes[..., :16 * d].view(*lead, d // D, 16, 4, D // 64, 2, 8)
    uk = uk.permute(*range(n), -5, -6, -3, -4, -2, -1).reshape(*lead, 16, d).flatten(-3, -2)
    uv = codes[..., 16 * d:].view(*lead, d // D, 2, 8, 4, 2, D // 8)
    uv = uv.permute(*range(n), -5, -3, -2, -6, -4, -1).reshape(*lead, 16, d).flatten(-3, -2)
    kp = records[..., 16 * d:17 * d].contiguous().view(torch.float16).view(*lead, 16, d // 64, 2)
    vp = records[..., 17 * d:].contiguous().view(torch.float16).view(*lead, 2, d // 64, 4, 2, 2)
    vp = vp.permute(*range(n), -5, -3, -1, -4, -2).reshape(*lead, 16, d // 64, 2)
    kp, vp = kp.flatten(-4, -3).float(), vp.flatten(-4, -3).float()
    return (uk, kp[..., 0], kp[..., 1]), (uv, vp[..., 0], vp[..., 1])


def _held(s, pages):
    """Keys and values [..., kv heads, page, d] of physical pages, in 32 bits."""
    c = s["c"]
    if c["fmt"] != "int4":
        return s["ck"][pages].float(), s["cv"][pages].float()
    k, v = _unpack(s["records"][pages], c["d"])
    return _value(*k), _value(*v)


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    c = s["c"]
    if own:
        lib, cache, batch = s["lib"], s["cache"], s["batch"]
        if c["op"] == "append":
            lib.ivfpq_kv_append(cache, batch, s["k"], s["v"])
            k, v = lib.ivfpq_kv_read(cache, batch, s["k"].shape[0], dtype=s["k"].dtype)
            hi, lo = lib.ivfpq_kv_read_bounds(cache, s["touched"])
            return {"k": k, "v": v, "hi": hi, "lo": lo}
        if c["op"] == "select":
            return {"blocks": lib.ivfpq_kv_select(cache, batch, s["q"], c["nsel"], nsink=c["sink"], nlocal=c["local"])}
        lib.ivfpq_kv_attend(cache, batch, s["q"], blocks=s.get("blocks"), out=s["out"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    return {"append": _plain_append, "select": _plain_select, "attend": _plain_attend}[c["op"]](s)


def _plain_append(s):
    c, dt = s["c"], s["k"].dtype
    page, table = c["page"], s["table"].long()
    real = s["pos"] >= 0
    pos, req = s["pos"].clamp(min=0), s["req"]
    where = table[req, pos // page].clamp(min=0)
    k, v = _held(s, s["touched"].long())
    if c["fmt"] == "int4":
        k_new, v_new = _value(*_quantize(s["k"].float())), _value(*_quantize(s["v"].float()))
    else:
        k_new, v_new = s["k"].float(), s["v"].float()
    # the pages that the tokens lie in, with the tokens in their places
    n = s["touched"].shape[0]
    slot = torch.zeros(s["bounds"].shape[0], dtype=torch.long, device=k.device)
    slot[s["touched"].long()] = torch.arange(n, device=k.device)
    spot = torch.where(real, slot[where] * page + pos % page, n * page)
    k, v = (torch.cat((x.transpose(1, 2).flatten(0, 1), torch.zeros_like(x[:1, :, 0]))) for x in (k, v))
    k[spot], v[spot] = k_new, v_new
    if c["fmt"] == "int4":       # written back: codes of held values are the codes that they came from
        rk, rv = s["k"].float(), s["v"].float()
        _write_records(s, where, pos, real, rk, rv)
    else:
        s["ck"][where[real], :, pos[real] % page], s["cv"][where[real], :, pos[real] % page] = s["k"][real], s["v"][real]
    # bounds of the pages that became full
    hi, lo = (f(k[:-1].unflatten(0, (n, page)), 1) for f in (torch.amax, torch.amin))
    codes, scale = _codes(hi, lo)
    last = (pos % page == page - 1) & real
    full = slot[where[last]]
    s["bounds"][where[last]], s["bounds_scale"][where[last]] = codes[full], scale[full]
    b = s["bounds"][s["touched"].long()].float() * s["bounds_scale"][s["touched"].long()][..., None, None]
    out = [torch.where(real[:, None, None], x[spot], torch.zeros_like(x[spot])).to(dt) for x in (k, v)]
    return {"k": out[0], "v": out[1], "hi": b[:, :, 0].contiguous(), "lo": b[:, :, 1].contiguous()}


def _write_records(s, where, pos, real, k, v):
    """Tokens' codes and parameters into their records: a record full of the token is made, and the bytes taken that are the token's own."""
    d = s["c"]["d"]
    t = pos % 16
    owned = _owned_bytes(d, k.device)
    new = _pack(*(x[:, :, None].expand(-1, -1, 16, -1) for x in (k, v)))[:, :, 0]
    keep = real.nonzero()[:, 0]
    at = owned[t[keep]]
    s["records"][where[keep][:, None], :, (pos[keep] % s["c"]["page"] // 16)[:, None], at] = new[keep[:, None], :, at]


def _owned_bytes(d, dev):
    """Offsets in a record of the bytes that belong to each of its 16 tokens: [16, 18 d / 16]."""
    D = min(d, 128)
    at = torch.arange(18 * d, device=dev)
    key = at % (16 * D // 2) // (D // 2)
    w = D // 16                                            # bytes of a token in one value word group
    val = (at - 8 * d) % (16 * D // 2)
    val = val // (8 * D // 2) * 8 + val // (2 * w) % 4 * 2 + val // w % 2
    kp = (at - 16 * d) // (d // 16)
    vp = at - 17 * d
    vp = vp // (d // 2) * 8 + vp // 8 % 4 * 2 + vp // 2 % 2
    token = torch.where(at < 8 * d, key, torch.where(at < 16 * d, val, torch.where(at < 17 * d, kp, vp)))
    return token.sort(stable=True).indices.view(16, -1)


def _padded(s, x):
    """Rows of the tokens, by request: [requests, most tokens, ...]."""
    j = torch.arange(x.shape[0], device=x.device) - s["q_start"].long()[s["req"]]
    y = torch.zeros(s["c"]["nreq"], max(s["new"]), *x.shape[1:], dtype=x.dtype, device=x.device)
    y[s["req"], j] = x
    return y, j


def _plain_select(s):
    c = s["c"]
    hkv, G, page, n = c["hkv"], c["group"], c["page"], c["nsel"]
    table = s["table"].long().clamp(min=0)
    q = s["q"].float().unflatten(1, (hkv, G))
    top = q.abs().amax((2, 3), keepdim=True)
    q = (q * torch.where(top > 0, 127.0 / top, torch.zeros_like(top))).round()
    q, j = _padded(s, q)                                                      # [r, t, hkv, G, d]
    b = s["bounds"][table].float()                                            # [r, b, hkv, 2, d]
    q = torch.cat((q.clamp(min=0), q.clamp(max=0)), -1).permute(0, 2, 1, 3, 4).flatten(2, 3)
    hits = q @ b.flatten(3).permute(0, 2, 3, 1)                               # whole numbers below 2^24
    hits = hits.unflatten(2, (-1, G)).amax(3)                                 # [r, hkv, t, b]
    score = (hits * s["bounds_scale"][table].permute(0, 2, 1)[:, :, None])[s["req"], :, j]   # [tok, hkv, b]
    cols = table.shape[1]
    at = torch.arange(cols, device=q.device)
    seen = ((s["pos"] + page) // page)[:, None, None]                         # blocks that the token sees
    score = score + 0.0
    inf = torch.tensor(float("inf"), device=q.device)
    score = torch.where((at < c["sink"]) | (at >= seen - c["local"]), inf, score)
    score = torch.where(at < seen, score, -inf)
    order = score.sort(dim=2, descending=True, stable=True).indices[:, :, :n]
    order = torch.where(order < seen, order, cols).sort(dim=2).values
    out = torch.full((order.shape[0], hkv, n), -1, dtype=torch.int32, device=q.device)
    out[:, :, :order.shape[2]] = torch.where(order == cols, -1, order).to(torch.int32)
    return {"blocks": out}


def _plain_attend(s):
    c = s["c"]
    hkv, G, page, d, nreq = c["hkv"], c["group"], c["page"], c["d"], c["nreq"]
    table = s["table"].long()
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in _held(s, table.clamp(min=0)))        # [r, hkv, L, d]
    q, j = _padded(s, s["q"].float().unflatten(1, (hkv, G)))
    t = q.shape[1]
    logit = q.permute(0, 2, 1, 3, 4).flatten(2, 3) @ k.transpose(2, 3)                    # [r, hkv, t G, L]
    logit = logit.mul_(1.0 / math.sqrt(d)).unflatten(2, (t, G))
    at = torch.arange(k.shape[2], device=k.device)
    pos = torch.full((nreq, t), -1, device=k.device)
    pos[s["req"], j] = s["pos"]
    seen = (at <= pos[:, :, None])[:, None]                                               # [r, 1, t, L]
    if "blocks" in s:
        cols = table.shape[1]
        chosen = torch.zeros(q.shape[0], t, hkv, cols + 1, dtype=torch.bool, device=k.device)
        b = s["blocks"].long()
        chosen[s["req"][:, None, None], j[:, None, None], torch.arange(hkv, device=k.device)[:, None], torch.where(b < 0, cols, b)] = True
        seen = seen & chosen[..., :cols].permute(0, 2, 1, 3).repeat_interleave(page, 3)
    logit = logit.masked_fill_(~seen[:, :, :, None], float("-inf"))
    m = logit.amax(-1, keepdim=True)
    p = logit.sub_(m.clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ v).unflatten(2, (t, G)) / total.clamp(min=1e-30)
    lse = (m + total.log())[..., 0]
    out, lse = (x.transpose(1, 2).flatten(2, 3)[s["req"], j] for x in (out, lse))
    s["out"].copy_(out)
    s["lse"].copy_(lse)
    return {"out": s["out"], "lse": s["lse"]}


# ---- 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "select":
        return None                      # whole numbers
    s = prepare(case, seed)
    return _exact_append(s) if c["op"] == "append" else _exact_attend(s)


def _exact_values(x):
    """What 64-element groups of x stand for once held in 4 bits."""
    y = x.double().reshape(*x.shape[:-1], -1, 64)
    z = y.min(-1, keepdim=True)[0].to(torch.float16).double()
    step = ((y.max(-1, keepdim=True)[0] - z) / 15).to(torch.float16).double()
    u = torch.round((y - z) / step).clamp(0, 15)
    return torch.where(step > 0, u * step + z, z).reshape(x.shape)


def _exact_record(rec, d):
    """Keys and values [16, d] of records [n, 18 d], element by element from the format's definition."""
    D, dev = min(d, 128), rec.device
    t, e = torch.arange(16, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    p, o = e // D, e % D
    nib = p * 16 * D + t * D + (o % 64 // 16) * (D // 4) + (o // 64) * 16 + o % 16
    ku = (rec[:, nib // 2] >> (4 * (nib % 2)).to(torch.uint8)) & 15
    w = D // 8
    nib = p * 16 * D + (t // 8) * 8 * D + (o // w) * 8 * w + (t % 8) * w + o % w
    vu = (rec[:, 8 * d + nib // 2] >> (4 * (nib % 2)).to(torch.uint8)) & 15
    kp = rec[:, 16 * d:17 * d].contiguous().view(torch.float16).double()
    vp = rec[:, 17 * d:].contiguous().view(torch.float16).double()
    at = (t * (d // 64) + e // 64) * 2
    k = ku.double() * kp[:, at] + kp[:, at + 1]
    at = ((t // 8) * (d // 64) + e // 64) * 16 + (t % 8) // 2 * 4 + t % 2
    v = vu.double() * vp[:, at] + vp[:, at + 2]
    return k, v


def _exact_pages(s, pages, h):
    """Keys and values [tokens, d] of one kv head over a list of pages, in 64 bits."""
    if "records" in s:
        k, v = _exact_record(s["records"][pages, h].reshape(-1, 18 * s["c"]["d"]), s["c"]["d"])
    else:
        k, v = s["ck"][pages, h].double(), s["cv"][pages, h].double()
    return k.reshape(-1, s["c"]["d"]), v.reshape(-1, s["c"]["d"])


def _exact_append(s):
    c, page, hkv, d = s["c"], s["c"]["page"], s["c"]["hkv"], s["c"]["d"]
    held = (lambda x: _exact_values(x)) if c["fmt"] == "int4" else (lambda x: x.double())
    k, v = held(s["k"]), held(s["v"])
    hi = torch.zeros(s["touched"].shape[0], hkv, d, dtype=torch.float64, device=k.device)
    lo = torch.zeros_like(hi)
    i, tok = 0, 0
    for r, (h, n) in enumerate(zip(s["held"], s["new"])):
        if h:
            for b in range((h - n) // page, (h - 1) // page + 1):
                if (b + 1) * page <= h:
                    old = max(0, h - n - b * page)
                    for g in range(hkv):
                        kk = k[tok + b * page + old - (h - n):tok + (b + 1) * page - (h - n), g]
                        if old:
                            kk = torch.cat((_exact_pages(s, s["touched"][i:i + 1].long(), g)[0][:old], kk))
                        top = kk.abs().max()
                        hi[i, g] = torch.round(kk.max(0)[0] * 127 / top) * top / 127
                        lo[i, g] = torch.round(kk.min(0)[0] * 127 / top) * top / 127
                i += 1
        else:
            k[tok:tok + n], v[tok:tok + n] = 0, 0
        tok += n
    return {"k": k, "v": v, "hi": hi, "lo": lo}


def _exact_attend(s):
    c, page, hkv, G, d = s["c"], s["c"]["page"], s["c"]["hkv"], s["c"]["group"], s["c"]["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=s["q"].device)
    tok = 0
    for r, (h, n) in enumerate(zip(s["held"], s["new"])):
        for g in range(hkv if h else 0):
            k, v = _exact_pages(s, s["table"][r, :-(-h // page)].long(), g)
            key = torch.arange(k.shape[0], device=k.device)
            for a in range(0, n, 256):
                b = min(n, a + 256)
                x = torch.einsum("tgd,kd->tgk", s["q"][tok + a:tok + b, g * G:(g + 1) * G].double(), k) / math.sqrt(d)
                see = key[None] <= torch.arange(h - n + a, h - n + b, device=k.device)[:, None]
                if "blocks" in s:
                    picked = (torch.arange(k.shape[0] // page, device=k.device)[None, :, None] == s["blocks"][tok + a:tok + b, g][:, None, :]).any(2)
                    see &= picked.repeat_interleave(page, 1)
                x = torch.where(see[:, None], x, -math.inf)
                lse[tok + a:tok + b, g * G:(g + 1) * G] = torch.logsumexp(x, -1)
                out[tok + a:tok + b, g * G:(g + 1) * G] = torch.softmax(x, -1) @ v
        tok += n
    return {"out": out, "lse": lse}
