"""Plain 64-bit reference of the key/value cache operators, straight from the definitions in
include/ivfpq.h (formats, quantizer, block scores, attention).  Test infrastructure; shares nothing with the CUDA path."""

import math

import numpy as np
import torch


def code_positions(d):
    """Nibble index of every (token, element) of a record: keys, values (counted from the value codes)."""
    D = min(d, 128)
    key, val = np.zeros((16, d), np.int64), np.zeros((16, d), np.int64)
    for t in range(16):
        for e in range(d):
            p, o = divmod(e, D)
            g, r = divmod(o, 64)
            c, r = divmod(r, 16)
            half, nib = divmod(r, 8)
            key[t, e] = (((((p * 16 + t) * 4 + c) * (D // 64) + g) * 2 + half) * 8) + nib
            chunk, nib = divmod(o, D // 8)
            octet, tt = divmod(t, 8)
            cc, parity = divmod(tt, 2)
            val[t, e] = (((((p * 2 + octet) * 8 + chunk) * 4 + cc) * 2 + parity) * (D // 8)) + nib
    return key, val


def decode_records(rec, d):
    """(codes, scale, offset) of keys and of values, [..., 16, d], from uint8 records [..., 18 d] (numpy)."""
    rec = np.ascontiguousarray(rec)
    key, val = code_positions(d)
    G = d // 64

    def nibbles(at, base):
        b = rec[..., base + at // 2]
        return np.where(at % 2 == 0, b & 15, b >> 4).astype(np.int64)

    kp = np.ascontiguousarray(rec[..., 16 * d:17 * d]).view(np.float16).reshape(*rec.shape[:-1], 16, G, 2).astype(np.float64)
    vp = np.ascontiguousarray(rec[..., 17 * d:]).view(np.float16).reshape(*rec.shape[:-1], 2, G, 4, 4).astype(np.float64)
    vs, vz = np.zeros_like(kp[..., 0]), np.zeros_like(kp[..., 0])
    for t in range(16):
        vs[..., t, :] = vp[..., t // 8, :, t % 8 // 2, t % 2]
        vz[..., t, :] = vp[..., t // 8, :, t % 8 // 2, 2 + t % 2]
    rep = lambda x: np.repeat(x, 64, axis=-1)  # noqa: E731
    return (nibbles(key, 0), rep(kp[..., 0]), rep(kp[..., 1])), (nibbles(val, 8 * d), rep(vs), rep(vz))


def held_values(rec, d):
    """Keys and values [pages, heads, page, d] in 64 bits of records [pages, heads, page / 16, 18 d]."""
    k, v = decode_records(rec, d)
    out = [u * s + z for u, s, z in (k, v)]
    return [x.reshape(x.shape[0], x.shape[1], -1, d) for x in out]


def encode_records(k, v):
    """Records of keys and values [pages, heads, page, d] (float64 numpy): a test's way to fill a 4-bit cache."""
    P, H, page, d = k.shape
    key, val = code_positions(d)
    rec = np.zeros((P, H, page // 16, 18 * d), np.uint8)
    nib = np.zeros((P, H, page // 16, 32 * d), np.uint8)
    for x, pos, base, which in ((k, key, 0, 0), (v, val, 16 * d, 1)):
        g = x.reshape(P, H, page // 16, 16, d // 64, 64)
        z = g.min(-1).astype(np.float16).astype(np.float64)
        s = ((g.max(-1) - z) / 15).astype(np.float16).astype(np.float64)
        with np.errstate(divide="ignore", invalid="ignore"):
            u = np.where(s[..., None] > 0, np.clip(np.rint((g - z[..., None]) / s[..., None]), 0, 15), 0)
        u = u.reshape(P, H, page // 16, 16, d).astype(np.uint8)
        nib[..., base + pos] = u
        par = np.zeros((P, H, page // 16, d // 2), np.float16)
        for t in range(16):
            for q in range(d // 64):
                if which == 0:
                    at = (t * (d // 64) + q) * 2
                    par[..., at], par[..., at + 1] = s[..., t, q], z[..., t, q]
                else:
                    at = ((t // 8 * (d // 64) + q) * 4 + t % 8 // 2) * 4 + t % 2
                    par[..., at], par[..., at + 2] = s[..., t, q], z[..., t, q]
        lo = 16 * d + which * d
        rec[..., lo:lo + d] = np.ascontiguousarray(par).view(np.uint8)
    rec[..., :16 * d] = nib[..., 0::2] | (nib[..., 1::2] << 4)
    return rec


def positions(seq_len, q_start):
    """(request, position) of every token."""
    out = []
    for r, n in enumerate(seq_len):
        f, e = (r, r + 1) if q_start is None else (q_start[r], q_start[r + 1])
        out += [(r, n - (e - f) + j) for j in range(e - f)]
    return out


def select(bounds, scale, table, seq_len, q_start, q, page, nselect, nsink, nlocal):
    """Block lists [tokens, kv heads, nselect]: bounds int8 [pages, heads, 2, d], q fp32 [tokens, query heads, d] (numpy)."""
    hkv, hq = bounds.shape[1], q.shape[1]
    G = hq // hkv
    out = np.full((q.shape[0], hkv, nselect), -1, np.int32)
    for t, (r, pos) in enumerate(positions(seq_len, q_start)):
        nb = pos // page + 1 if pos >= 0 else 0
        for h in range(hkv):
            if nb <= nselect:
                out[t, h, :nb] = np.arange(nb)
                continue
            x = q[t, h * G:(h + 1) * G].astype(np.float32)
            top = np.float32(np.abs(x).max())
            f = np.float32(np.float32(1) / top) * np.float32(127) if top > 0 else np.float32(0)
            q8 = np.rint(x * f).astype(np.int64)
            b = bounds[table[r, :nb], h].astype(np.int64)                       # [nb, 2, d]
            dots = np.maximum(q8[:, None] * b[None, :, 0], q8[:, None] * b[None, :, 1]).sum(-1).max(0)
            score = dots.astype(np.float32) * scale[table[r, :nb], h]
            forced = (np.arange(nb) < nsink) | (np.arange(nb) >= nb - nlocal)
            rest = [b for b in np.argsort(-score.astype(np.float64), kind="stable") if not forced[b]]
            pick = list(np.nonzero(forced)[0]) + rest[:nselect - int(forced.sum())]
            out[t, h] = np.sort(pick)
    return out


def attend(k, v, table, seq_len, q_start, q, page, scale=None, blocks=None):
    """out, lse, and what error bounds need: sum p |v|, largest sum |q k| scale.  k, v [pages, heads, page, d] float64 torch."""
    hkv, hq, d = k.shape[1], q.shape[1], q.shape[2]
    G = hq // hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    q = q.double()
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    big = torch.zeros_like(lse)
    for t, (r, pos) in enumerate(positions(seq_len, q_start)):
        if pos < 0:
            continue
        for h in range(hkv):
            nb = pos // page + 1
            use = range(nb) if blocks is None else [b for b in blocks[t, h].tolist() if 0 <= b < nb]
            at = [(int(table[r, b]), i) for b in use for i in range(min(page, pos + 1 - b * page))]
            if not at:
                continue
            pg, sl = torch.tensor(at, device=q.device).T
            kk, vv = k[pg, h, sl], v[pg, h, sl]
            x = q[t, h * G:(h + 1) * G] @ kk.T * scale
            p = torch.softmax(x, -1)
            out[t, h * G:(h + 1) * G] = p @ vv
            mag[t, h * G:(h + 1) * G] = p @ vv.abs()
            lse[t, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
            big[t, h * G:(h + 1) * G] = (q[t, h * G:(h + 1) * G].abs() @ kk.abs().T).amax(-1) * abs(scale)
    return out, lse, mag, big
