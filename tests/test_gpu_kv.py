"""Key/value cache operators on the GPU against the plain 64-bit reference (kv_reference.py)."""

import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2312_01712_b200 as lib

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # unit roundoff


class Setup:
    """A filled cache, a batch on it and its reference form."""

    def __init__(self, fmt="int4", dtype="bf16", d=128, hkv=2, G=4, page=64, lens=(100,), news=None, layout="hnd", seed=0, spare=2,
                 span=1.0, poison=True):
        rng = np.random.default_rng(seed)
        self.fmt, self.dt, self.d, self.hkv, self.G, self.page = fmt, DT[dtype], d, hkv, G, page
        self.lens, self.q_start = list(lens), None
        n = len(lens)
        news = [1] * n if news is None else list(news)
        if any(x != 1 for x in news):
            self.q_start = [0] + np.cumsum(news).tolist()
        self.ntok = sum(news)
        nblk = [max(0, -(-x // page)) for x in lens]
        self.cols = max(1, max(nblk)) + 1
        P = sum(nblk) + spare
        perm = rng.permutation(P)
        self.table = np.full((n, self.cols), -1, np.int32)
        at = 0
        for r, b in enumerate(nblk):
            self.table[r, :b] = perm[at:at + b]
            at += b
        k = rng.standard_normal((P, hkv, page, d)) * span + 0.3 * rng.standard_normal((P, hkv, 1, d))
        v = rng.standard_normal((P, hkv, page, d)) * span
        r16 = lambda x: torch.from_numpy(x).to(self.dt)  # noqa: E731
        # slots that no request holds: whatever an earlier owner left, not-a-number among it
        unheld = np.ones((P, page), bool)
        for r, x in enumerate(lens):
            for b in range(nblk[r]):
                unheld[self.table[r, b], :max(0, min(page, x - b * page))] = False
        if fmt == "int4":
            rec = ref.encode_records(r16(k).double().numpy(), r16(v).double().numpy())
            self.kref, self.vref = [torch.from_numpy(x).cuda() for x in ref.held_values(rec, d)]
            if poison:
                for p in range(P):
                    for t in np.nonzero(unheld[p])[0]:
                        part = rec[p, :, t // 16]
                        tt, g = t % 16, d // 64
                        part[:, 16 * d:17 * d].view(np.uint16).reshape(hkv, 16, g, 2)[:, tt] = 0x7e00     # NaN
                        part[:, 17 * d:].view(np.uint16).reshape(hkv, 2, g, 4, 4)[:, tt // 8, :, tt % 8 // 2, tt % 2::2] = 0xfc00
            self.tensors = dict(records=torch.from_numpy(rec).cuda())
        else:
            kt, vt = r16(k), r16(v)
            self.kref, self.vref = kt.double().cuda(), vt.double().cuda()
            if poison:
                m = torch.from_numpy(unheld)[:, None, :, None].expand(kt.shape)
                kt, vt = kt.masked_fill(m, float("nan")), vt.masked_fill(m, float("inf"))
            if layout == "nhd":
                kt, vt = (x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for x in (kt, vt))
            elif layout == "joint":                    # keys and values side by side in one buffer, rows padded
                both = torch.zeros(P, hkv, page, 2, d + 8, dtype=self.dt, device="cuda")
                both[..., 0, :d], both[..., 1, :d] = kt.cuda(), vt.cuda()
                kt, vt = both[..., 0, :d], both[..., 1, :d]
            self.tensors = dict(k=kt.cuda(), v=vt.cuda())
        self.tensors["bounds"] = torch.zeros(P, hkv, 2, d, dtype=torch.int8, device="cuda")
        self.tensors["bounds_scale"] = torch.zeros(P, hkv, dtype=torch.float32, device="cuda")
        self.cache = lib.KvCacheHandle(**self.tensors)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.batch = lib.KvBatchHandle(i32(self.table), i32(self.lens), None if self.q_start is None else i32(self.q_start))
        qkv = torch.from_numpy(rng.standard_normal((self.ntok, hkv * G + 3, d))).to(self.dt).cuda()
        self.q = qkv[:, 1:1 + hkv * G]                  # a slice of a wider projection
        self.pos = ref.positions(self.lens, self.q_start)

    def check(self, blocks=None, scale=None, q=None, table=None):
        q = self.q if q is None else q
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        out = lib.ivfpq_kv_attend(self.cache, self.batch, q, blocks=blocks, scale=scale, lse=lse)
        assert lib.ivfpq_kv_status(self.cache) == lib.IVFPQ_OK
        eo, el, mag, big = ref.attend(self.kref, self.vref, self.table if table is None else table, self.lens, self.q_start, q, self.page,
                                      scale, blocks)
        n = max(1, max(self.lens))
        u = ROUND[q.dtype]
        held = ROUND[torch.float16] if self.fmt == "int4" else u
        logit = (big * (self.d + 16) * 2.0 ** -24 + 2.0 ** -20)[..., None]       # error of a logit, and of exp
        tol = u * eo.abs() + mag * (2 * held * 1.05 + 2 * logit) + n * 2.0 ** -25 * float(self.vref.abs().max()) + 2.0 ** -24
        bad = (out.double() - eo).abs() > tol
        assert not bad.any(), (int(bad.sum()), float((out.double() - eo).abs().max()))
        assert torch.equal(torch.isinf(lse), torch.isinf(el)) and not torch.isnan(out).any()
        f = torch.isfinite(el)
        assert bool(((lse.double() - el).abs()[f] <= (logit[..., 0] + 2.0 ** -22 * el.abs() + 2.0 ** -20)[f]).all())
        return out, lse


FORMATS = [("int4", "bf16"), ("int4", "fp16"), ("bf16", "bf16"), ("fp16", "fp16")]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32), (128, 128)])
def test_attend_whole_cache_of_every_length(fmt, dtype, d, page):
    lens = (1, 0, 2, page - 1, page, page + 1, 15, 16, 17, 31, 33, 3 * page + 5, 0, 700)
    Setup(fmt, dtype, d=d, page=page, lens=lens, seed=d + page).check()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("G,hkv", [(1, 3), (2, 2), (3, 1), (7, 2), (8, 1), (9, 1), (16, 2), (20, 1), (40, 1)])
def test_attend_groups_of_heads(fmt, dtype, G, hkv):
    Setup(fmt, dtype, G=G, hkv=hkv, lens=(130, 5, 64, 300), seed=G).check()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("G", [1, 4, 7, 16])
def test_attend_several_tokens_per_request(fmt, dtype, G):
    # drafted tokens, a whole prompt, a request without new tokens, more new tokens than are held
    Setup(fmt, dtype, G=G, page=32, lens=(70, 33, 200, 0, 3, 90, 1), news=(5, 33, 0, 1, 5, 70, 1), seed=G).check()


@pytest.mark.parametrize("layout", ["nhd", "joint"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_attend_strided_caches(layout, d):
    Setup("bf16", "bf16", d=d, layout=layout, hkv=3, G=2, lens=(100, 257), seed=5).check()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("d,page,G", [(128, 64, 8), (64, 16, 3), (256, 128, 16), (128, 32, 1)])
def test_attend_listed_blocks(fmt, dtype, d, page, G):
    s = Setup(fmt, dtype, d=d, page=page, G=G, lens=(9 * page + 3, 4 * page, 5, 0, 6 * page + 1), news=(3, 1, 1, 1, 20), seed=7)
    rng = np.random.default_rng(1)
    n = 6
    blocks = np.full((s.ntok, s.hkv, n), -1, np.int32)
    for t, (r, pos) in enumerate(s.pos):
        for h in range(s.hkv):
            pick = rng.permutation(max(1, pos // page + 1))[:rng.integers(0, n + 1)] if pos >= 0 else []
            at = np.sort(rng.permutation(n)[:len(pick)])
            blocks[t, h, at] = pick                      # any order, gaps of -1
    blocks[0, 0] = -1                                    # a row that sees nothing
    blocks[1, 1, :2] = (pos_blocks(s, 1, page) + 3, 1 << 20)   # beyond the token's position: passed over
    s.check(torch.from_numpy(blocks).cuda())


def pos_blocks(s, t, page):
    return s.pos[t][1] // page + 1


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_attend_long_prompt_over_listed_blocks(fmt, dtype):
    s = Setup(fmt, dtype, page=16, G=4, lens=(400, 77), news=(301, 77), seed=11)
    rng = np.random.default_rng(2)
    blocks = np.full((s.ntok, s.hkv, 5), -1, np.int32)
    for t, (r, pos) in enumerate(s.pos):
        for h in range(s.hkv):
            own, rest = pos // 16, rng.permutation(pos // 16 + 1)
            pick = np.unique(np.concatenate(([own, 0], rest[:3])))
            blocks[t, h, :len(pick)] = pick
    s.check(torch.from_numpy(blocks).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("page,G", [(16, 4), (64, 8), (128, 3), (32, 1)])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, page, G):
    # held infinities and not-a-numbers in a block, and in tokens of the prompt's own end: a token that did not list the
    # block, or comes before the token, must not notice
    n = 6 * page + 40
    s = Setup(dtype, dtype, page=page, G=G, lens=(n, 3 * page), news=(100, 2 * page), seed=page)
    bad_block, bad_pos = 2, n - 30
    for name in ("k", "v"):
        x = s.tensors[name]
        x[int(s.table[0, bad_block]), :, 5] = float("nan") if name == "k" else float("inf")
        x[int(s.table[0, bad_pos // page]), :, bad_pos % page] = float("nan")
    rng = np.random.default_rng(3)
    blocks = np.full((s.ntok, s.hkv, 4), -1, np.int32)
    touched = np.zeros((s.ntok, s.hkv), bool)
    for t, (r, pos) in enumerate(s.pos):
        for h in range(s.hkv):
            pick = np.unique(np.concatenate((rng.permutation(pos // page + 1)[:3], [pos // page])))
            blocks[t, h, :len(pick)] = pick
            touched[t, h] = r == 0 and ((bad_block in pick and pos >= bad_block * page + 5) or (pos >= bad_pos and bad_pos // page in pick))
    bt = torch.from_numpy(blocks).cuda()
    out = lib.ivfpq_kv_attend(s.cache, s.batch, s.q, blocks=bt)
    clean, _, mag, big = ref.attend(s.kref, s.vref, s.table, s.lens, s.q_start, s.q, page, None, bt)
    free = torch.from_numpy(~touched).cuda().repeat_interleave(G, 1)
    assert bool(free.any()) and bool((~free).any())
    tol = ROUND[s.dt] * clean.abs() + mag * (2 * ROUND[s.dt] * 1.05 + 2 * (big * 144 * 2.0 ** -24 + 2.0 ** -20)[..., None]) + 1e-4
    assert bool(((out.double() - clean).abs() <= tol)[free].all())
    assert bool(torch.isnan(out)[~free].any(-1).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("G", [1, 3, 8, 16])
def test_tokens_do_not_notice_later_ones_that_are_not_finite(dtype, G):
    # drafted tokens over the whole cache: the last token's key and value are not finite
    s = Setup(dtype, dtype, G=G, lens=(150, 37, 64), news=(5, 4, 6), seed=G)
    for r, n in enumerate(s.lens):
        for name in ("k", "v"):
            s.tensors[name][int(s.table[r, (n - 1) // s.page]), :, (n - 1) % s.page] = float("nan") if r else float("inf")
    out = lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
    clean, _, mag, big = ref.attend(s.kref, s.vref, s.table, s.lens, s.q_start, s.q, s.page)
    last = torch.tensor([pos == s.lens[r] - 1 for r, pos in s.pos], device="cuda")
    tol = ROUND[s.dt] * clean.abs() + mag * (2 * ROUND[s.dt] * 1.05 + 2 * (big * 144 * 2.0 ** -24 + 2.0 ** -20)[..., None]) + 1e-4
    assert bool(((out.double() - clean).abs() <= tol)[~last].all())
    assert bool(torch.isnan(out)[last].any(-1).all())


def test_attend_scales_and_wide_logits():
    for fmt, dtype in (("int4", "fp16"), ("bf16", "bf16")):
        s = Setup(fmt, dtype, lens=(300, 40), seed=3)
        for scale in (0.0, 1.0, -0.3, 1e-4):
            s.check(scale=scale)
        s.check(q=s.q * 30)                               # logits of hundreds: a few keys take all
        s.check(q=s.q * 2.0 ** -18, scale=2.0 ** 15)      # tiny queries


@pytest.mark.parametrize("span", [1e-3, 50.0])
def test_attend_ranges_of_held_values(span):
    for fmt, dtype in FORMATS:
        Setup(fmt, dtype, lens=(200,), span=span, seed=4).check(scale=0.1 / span ** 1)


def test_attend_long_cache_split_over_the_gpu_is_deterministic():
    for fmt, dtype in (("int4", "bf16"), ("fp16", "fp16")):
        s = Setup(fmt, dtype, hkv=1, G=4, page=128, lens=(30011, 17, 6000), seed=9)
        a = s.check()
        for _ in range(3):
            lse = torch.empty(s.q.shape[:2], dtype=torch.float32, device="cuda")
            out = lib.ivfpq_kv_attend(s.cache, s.batch, s.q, lse=lse)
            assert torch.equal(out, a[0]) and torch.equal(lse, a[1])


def test_attend_offsets_past_32_bits():
    # a cache of 2^31 + elements; the request lives in its last pages
    P, hkv, page, d = 17000, 16, 64, 128
    assert P * hkv * page * d > 2 ** 31
    k = torch.zeros(P, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    k[-4:] = torch.randn(4, hkv, page, d, generator=g, device="cuda").to(torch.bfloat16)
    cache = lib.KvCacheHandle(k=k, v=k)
    table = torch.tensor([[P - 1, P - 3, P - 4, P - 2]], dtype=torch.int32, device="cuda")
    batch = lib.KvBatchHandle(table, torch.tensor([250], dtype=torch.int32, device="cuda"))
    q = torch.randn(1, hkv, d, generator=g, device="cuda").to(torch.bfloat16)
    out = lib.ivfpq_kv_attend(cache, batch, q)
    held = k[-4:].double()
    want, _, mag, _ = ref.attend(held, held, np.array([[3, 1, 0, 2]]), [250], None, q, page)
    assert bool(((out.double() - want).abs() <= mag * 3.2 * 2.0 ** -8 + 1e-4).all())


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32)])
def test_append_then_read(fmt, dtype, d, page):
    s = Setup(fmt, dtype, d=d, page=page, hkv=3, lens=(2 * page + 5, page, 0, 40, 3, 200), news=(page + 9, 1, 1, 40, 5, 0), seed=d)
    rng = np.random.default_rng(8)
    wide = torch.from_numpy(rng.standard_normal((s.ntok, 9, d))).to(s.dt).cuda()
    k, v = wide[:, 1:4], wide[:, 5:8]
    k[0, 0, :64] = 1.5                                    # a constant group
    before = {n: x.clone() for n, x in s.tensors.items()}
    lib.ivfpq_kv_append(s.cache, s.batch, k, v)
    assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_OK
    got = lib.ivfpq_kv_read(s.cache, s.batch, s.ntok, dtype=s.dt)
    where = [(t, s.table[r, pos // page], pos % page) for t, (r, pos) in enumerate(s.pos) if pos >= 0]
    t, p, o = (np.array(x) for x in zip(*where))
    gone = np.ones(s.ntok, bool)
    gone[t] = False
    for x, y in zip(got, (k, v)):
        assert not x[torch.from_numpy(gone).cuda()].any()
    if fmt == "int4":
        rec, old = s.tensors["records"].cpu().numpy(), before["records"].cpu().numpy()
        (ku, ks, kz), (vu, vs, vz) = ref.decode_records(rec, d)
        for (u, sc, z), x, y in (((ku, ks, kz), k, got[0]), ((vu, vs, vz), v, got[1])):
            u, sc, z = (a.reshape(a.shape[0], 3, page, d)[p, :, o] for a in (u, sc, z))
            x = x.double().cpu().numpy()[t]
            g = x.reshape(len(t), 3, d // 64, 64)
            rep = lambda a: np.repeat(a, 64, -1)  # noqa: E731
            assert np.array_equal(z, rep(g.min(-1).astype(np.float16).astype(np.float64)))
            want = rep((g.max(-1) - z[..., ::64]) / 15)
            assert np.all(np.abs(sc - want) <= 2.0 ** -11 * 1.01 * want + 2.0 ** -24)
            held = u * sc + z
            inside = (x >= z) & (x <= z + 15 * sc)
            assert np.all(np.abs(held - x)[inside] <= (0.5 + 1e-5) * sc[inside])
            assert np.all(np.abs(held - x) <= 0.51 * sc + 15 * sc * 2.0 ** -11 + np.abs(z) * 2.0 ** -11 + 2.0 ** -24)
            assert np.all(np.abs(y.double().cpu().numpy()[t] - held) <= ROUND[s.dt] * np.abs(held) * 1.001 + 2.0 ** -24)
        # nothing but the tokens' own codes and parameters changed
        key, val = ref.code_positions(d)
        mine = np.zeros(rec.shape, bool)
        for pp, oo in zip(p, o):
            tt, G = oo % 16, d // 64
            r = mine[pp, :, oo // 16]
            r[:, key[tt] // 2] = True
            r[:, 8 * d + val[tt] // 2] = True
            r[:, 16 * d:17 * d].reshape(3, 16, G * 4)[:, tt] = True
            r[:, 17 * d:].reshape(3, 2, G, 4, 4, 2)[:, tt // 8, :, tt % 8 // 2, tt % 2::2] = True
        assert np.array_equal(rec[~mine], old[~mine])
    else:
        for name, x, y in (("k", k, got[0]), ("v", v, got[1])):
            held = s.tensors[name]
            tt, pp, oo = (torch.from_numpy(a.astype(np.int64)).cuda() for a in (t, p, o))
            assert torch.equal(held[pp, :, oo], x[tt]) and torch.equal(y[tt], x[tt])
            same = torch.ones(held.shape[0], page, dtype=torch.bool, device="cuda")
            same[pp, oo] = False
            a, b = held.permute(0, 2, 1, 3)[same], before[name].permute(0, 2, 1, 3)[same]
            assert torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32), (128, 128)])
def test_bounds_hold_the_keys_and_do_not_depend_on_the_steps(fmt, dtype, d, page):
    n = 2 * page + 7
    rng = np.random.default_rng(d)
    x = torch.from_numpy(rng.standard_normal((2, n, 2, d)) * np.array([1.0, 8.0])[rng.integers(0, 2, d)]).to(DT[dtype]).cuda()
    made = []
    for steps in ([n], [1] * n, [page - 1, 2, page, 6]):
        s = Setup(fmt, dtype, d=d, page=page, lens=(n,), news=(n,), seed=1, poison=False)
        at = 0
        for m in steps:
            i32 = lambda y: torch.tensor(y, dtype=torch.int32, device="cuda")  # noqa: E731
            b = lib.KvBatchHandle(i32(s.table), i32([at + m]), i32([0, m]) if m != 1 else None)
            lib.ivfpq_kv_append(s.cache, b, x[0, at:at + m], x[1, at:at + m])
            at += m
        made.append(s)
    pages = torch.from_numpy(made[0].table[0, :2].astype(np.int32)).cuda()
    for s in made[1:]:
        for name in s.tensors:
            a, b = (z.contiguous().view(torch.uint8) for z in (s.tensors[name], made[0].tensors[name]))
            assert torch.equal(a, b), name
    s = made[0]
    k = torch.from_numpy(ref.held_values(s.tensors["records"].cpu().numpy(), d)[0]).cuda() if fmt == "int4" else s.tensors["k"].double()
    hi, lo = lib.ivfpq_kv_read_bounds(s.cache, pages)
    kk = k[pages.long()]
    scale = s.tensors["bounds_scale"][pages.long()].double()[..., None]
    assert bool(((kk.abs().amax((2, 3)) / 127 - scale[..., 0]).abs() <= 2.0 ** -22 * scale[..., 0]).all())
    assert bool(((hi - kk.amax(2)).abs() <= 0.5001 * scale).all()) and bool(((lo - kk.amin(2)).abs() <= 0.5001 * scale).all())
    unfinished = int(s.table[0, 2])
    assert not s.tensors["bounds"][unfinished].any() and not s.tensors["bounds_scale"][unfinished].any()


def test_append_of_infinities_keeps_the_cache_finite():
    s = Setup("int4", "bf16", lens=(20,), news=(20,), poison=False)
    x = torch.randn(20, 2, 128, device="cuda").to(torch.bfloat16)
    x[3, 0, 5], x[4, 1, 70], x[5, 0, 1] = float("inf"), float("-inf"), 3e38
    lib.ivfpq_kv_append(s.cache, s.batch, x, x)
    k, v = lib.ivfpq_kv_read(s.cache, s.batch, 20, dtype=torch.float16)
    assert torch.isfinite(k).all() and torch.isfinite(v).all() and k[3, 0, 5] > 6e4 and k[4, 1, 70] < -6e4


def bounded(s, seed, tie=False):
    """Random bounds for the whole cache."""
    rng = np.random.default_rng(seed)
    P = s.tensors["bounds"].shape[0]
    a = rng.integers(-127, 128, (P, s.hkv, 2, s.d)).astype(np.int8)
    b = np.stack((a.max(2), a.min(2)), 2)
    scale = (0.01 + rng.random((P, s.hkv))).astype(np.float32)
    if tie:
        b[:], scale[:] = b[:1], 0.5
    s.tensors["bounds"].copy_(torch.from_numpy(b))
    s.tensors["bounds_scale"].copy_(torch.from_numpy(scale))
    return b, scale


@pytest.mark.parametrize("d,page,G,hkv", [(128, 64, 4, 2), (64, 16, 1, 3), (256, 32, 7, 1), (128, 16, 8, 2), (64, 32, 16, 1), (128, 32, 20, 1),
                                          (128, 16, 3, 2), (128, 128, 64, 1)])
@pytest.mark.parametrize("nselect,nsink,nlocal", [(1, 0, 1), (9, 1, 2), (40, 2, 2)])
def test_select_equals_the_reference(d, page, G, hkv, nselect, nsink, nlocal):
    for dtype in ("bf16", "fp16"):
        s = Setup("int4", dtype, d=d, page=page, G=G, hkv=hkv, lens=(0, 1, page, nselect * page, nselect * page + 1, 90 * page + 3, 60 * page),
                  news=(1, 1, 1, 1, 1, 1, 1), seed=d + G, poison=False)
        b, sc = bounded(s, G)
        got = lib.ivfpq_kv_select(s.cache, s.batch, s.q, nselect, nsink=nsink, nlocal=nlocal)
        assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_OK
        want = ref.select(b, sc, s.table, s.lens, s.q_start, s.q.float().cpu().numpy(), page, nselect, nsink, nlocal)
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("G,hkv", [(1, 2), (3, 1), (4, 2), (8, 1), (12, 1)])
def test_select_several_tokens_per_request(G, hkv):
    s = Setup("int4", "bf16", G=G, hkv=hkv, page=16, lens=(500, 33, 0, 300, 2), news=(41, 33, 1, 1, 4), seed=G, poison=False)
    b, sc = bounded(s, 3)
    got = lib.ivfpq_kv_select(s.cache, s.batch, s.q, 7, nsink=1, nlocal=1)
    want = ref.select(b, sc, s.table, s.lens, s.q_start, s.q.float().cpu().numpy(), 16, 7, 1, 1)
    assert np.array_equal(got.cpu().numpy(), want)


def test_select_ties_go_to_the_first_blocks_and_zero_queries_are_ties():
    s = Setup("int4", "bf16", page=16, lens=(1600, 900), seed=1, poison=False)
    b, sc = bounded(s, 5, tie=True)
    for q in (s.q, torch.zeros_like(s.q)):
        got = lib.ivfpq_kv_select(s.cache, s.batch, q, 10, nsink=1, nlocal=2).cpu().numpy()
        assert np.array_equal(got, ref.select(b, sc, s.table, s.lens, None, q.float().cpu().numpy(), 16, 10, 1, 2))
        assert got[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, 98, 99]


def test_select_of_scores_that_are_not_finite():
    s = Setup("int4", "bf16", page=16, lens=(800,), seed=1, poison=False)
    b, sc = bounded(s, 5)
    page7, page9 = int(s.table[0, 7]), int(s.table[0, 9])
    s.tensors["bounds_scale"][page7] = float("nan")       # ranks last
    s.tensors["bounds_scale"][page9] = float("inf")
    s.tensors["bounds"][page9, :, 0] = 127
    s.tensors["bounds"][page9, :, 1] = -127
    got = lib.ivfpq_kv_select(s.cache, s.batch, s.q, 49, nsink=0, nlocal=1).cpu().numpy()
    assert all(7 not in row and 9 in row for row in got.reshape(-1, 49).tolist())


@pytest.mark.parametrize("nblk,nselect", [(20000, 64), (32768, 1024), (5000, 1000), (2049, 3)])
def test_select_among_many_blocks(nblk, nselect):
    d, hkv, page = 64, 2, 16
    g = torch.Generator("cuda").manual_seed(nblk)
    P = 300
    rng = np.random.default_rng(nblk)
    table = rng.integers(0, P, (2, nblk)).astype(np.int32)      # pages shared: many ties
    lens = [nblk * page - 3, nblk * page // 2]
    cache = lib.KvCacheHandle.empty(P, hkv, page, d)
    a = rng.integers(-127, 128, (P, hkv, 2, d)).astype(np.int8)
    b, sc = np.stack((a.max(2), a.min(2)), 2), rng.random((P, hkv)).astype(np.float32)
    cache.bounds.copy_(torch.from_numpy(b))
    cache.bounds_scale.copy_(torch.from_numpy(sc))
    batch = lib.KvBatchHandle(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = torch.randn(2, hkv * 4, d, generator=g, device="cuda").to(torch.bfloat16)
    got = lib.ivfpq_kv_select(cache, batch, q, nselect, nsink=1, nlocal=1)
    assert np.array_equal(got.cpu().numpy(), ref.select(b, sc, table, lens, None, q.float().cpu().numpy(), page, nselect, 1, 1))


def test_pages_outside_the_cache_are_skipped_and_flagged():
    s = Setup("int4", "bf16", lens=(300, 100), seed=2)
    good = s.batch.block_table.clone()
    for bad in (1 << 30, -5, s.cache.npages):
        s.batch.block_table.copy_(good)
        s.batch.block_table[0, 2] = bad
        out = lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
        assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_ERR_DEVICE_FLAG
        assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_OK      # reported once
        assert not torch.isnan(out).any()
        blocks = torch.tensor([[[0, 1, 3, 4, -1]] * 2, [[0, 1, -1, -1, -1]] * 2], dtype=torch.int32, device="cuda")
        s.batch.block_table.copy_(good)
        assert torch.allclose(out.float(), lib.ivfpq_kv_attend(s.cache, s.batch, s.q, blocks=blocks).float(), atol=2e-2)
    s.batch.block_table[0, 4] = 1 << 30
    x = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    lib.ivfpq_kv_append(s.cache, s.batch, x, x)
    assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_ERR_DEVICE_FLAG
    lib.ivfpq_kv_read_bounds(s.cache, torch.tensor([0, s.cache.npages], dtype=torch.int32, device="cuda"))
    assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_ERR_DEVICE_FLAG


def test_lengths_beyond_the_table_and_wild_starts_are_flagged():
    s = Setup("int4", "bf16", lens=(300, 100), news=(3, 2), seed=2)
    s.batch.seq_len[0] = 1 << 30
    lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
    assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_ERR_DEVICE_FLAG
    s.batch.seq_len[0] = 300
    for wild in ([0, 3, 1 << 30], [0, 4, 2], [-7, 3, 5]):
        s.batch.q_start.copy_(torch.tensor(wild, dtype=torch.int32))
        x = torch.zeros(5, 2, 128, dtype=torch.bfloat16, device="cuda")
        lib.ivfpq_kv_append(s.cache, s.batch, x, x)
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
        lib.ivfpq_kv_select(s.cache, s.batch, s.q, 2)
        lib.ivfpq_kv_read(s.cache, s.batch, 5)
        assert lib.ivfpq_kv_status(s.cache) == lib.IVFPQ_ERR_DEVICE_FLAG


def test_calls_on_two_streams_and_in_a_graph():
    s = Setup("int4", "bf16", hkv=2, lens=(9000, 40, 2500), seed=6, page=128)
    want = lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
    q2 = (s.q * 0.5).contiguous()
    want2 = lib.ivfpq_kv_attend(s.cache, s.batch, q2)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(a):
            x = lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
        with torch.cuda.stream(b):
            y = lib.ivfpq_kv_attend(s.cache, s.batch, q2)
        torch.cuda.synchronize()
        assert torch.equal(x, want) and torch.equal(y, want2)
    out = torch.empty_like(want)
    q = s.q.contiguous()
    with torch.cuda.stream(a):
        lib.ivfpq_kv_attend(s.cache, s.batch, q, out=out)      # the stream's workspace exists before the capture
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=a):
            lib.ivfpq_kv_attend(s.cache, s.batch, q, out=out)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    s.batch.seq_len.copy_(torch.tensor([500, 39, 2499], dtype=torch.int32))      # lengths are read when the graph runs
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, lib.ivfpq_kv_attend(s.cache, s.batch, q))


def test_a_first_call_on_a_stream_may_be_captured():
    s = Setup("int4", "bf16", hkv=2, lens=(9000, 40, 2500), seed=8, page=128)
    want = lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
    q = s.q.contiguous()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, graphs = [torch.zeros_like(want), torch.zeros_like(want)], [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    for out, g in zip(outs, graphs):                           # two graphs of one stream that had no call before
        with torch.cuda.graph(g, stream=streams[0]):
            lib.ivfpq_kv_attend(s.cache, s.batch, q, out=out)
    assert not s.cache._ws[streams[0].cuda_stream][:lib.IVFPQ_KV_WORKSPACE_ZERO].any()      # zeroed before any replay
    with torch.cuda.stream(streams[0]):                        # a plain call, then the graphs in the other order
        plain = lib.ivfpq_kv_attend(s.cache, s.batch, q)
    torch.cuda.synchronize()
    graphs[1].replay()
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(plain, want) and torch.equal(outs[0], want) and torch.equal(outs[1], want)
    g = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="before capturing"):
        with torch.cuda.graph(g, stream=streams[1]):
            lib.ivfpq_kv_attend(s.cache, s.batch, q, out=outs[0])
    with torch.cuda.stream(streams[1]):
        assert torch.equal(lib.ivfpq_kv_attend(s.cache, s.batch, q), want)


def test_the_binding_checks_tensors_and_the_first_use_of_select_needs_bounds():
    s = Setup("bf16", "bf16", lens=(100, 50))
    with pytest.raises(ValueError):
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q.float())
    with pytest.raises(ValueError):
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q[..., ::2])
    with pytest.raises(ValueError):
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q, out=torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q, blocks=torch.zeros(2, 2, 3, dtype=torch.int64, device="cuda"))
    with pytest.raises(lib.IvfpqError) as e:
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q.half())      # another type than the cache's
    assert e.value.code == lib.IVFPQ_ERR_UNSUPPORTED
    with pytest.raises(lib.IvfpqError) as e:
        lib.ivfpq_kv_attend(s.cache, s.batch, s.q[:1])         # one token for two requests
    assert e.value.code == lib.IVFPQ_ERR_INVALID_ARGUMENT
    bare = lib.KvCacheHandle(k=s.tensors["k"], v=s.tensors["v"])
    with pytest.raises(lib.IvfpqError) as e:
        lib.ivfpq_kv_select(bare, s.batch, s.q, 4)
    assert e.value.code == lib.IVFPQ_ERR_INVALID_ARGUMENT


def test_selecting_every_block_is_the_whole_cache():
    for fmt, dtype in FORMATS:
        s = Setup(fmt, dtype, page=16, lens=(300, 20, 0), seed=8)
        whole = lib.ivfpq_kv_attend(s.cache, s.batch, s.q)
        blocks = lib.ivfpq_kv_select(s.cache, s.batch, s.q, 32)
        assert torch.allclose(lib.ivfpq_kv_attend(s.cache, s.batch, s.q, blocks=blocks).float(), whole.float(), atol=2e-2, rtol=2e-2)


@pytest.mark.parametrize("bits", [4, 16])
def test_the_curve_of_kept_attention(bits):
    from paper_2312_01712_b200 import kv_curve
    rows = kv_curve.curve([4, 12, 40], context=2400, nreq=3, hkv=2, page=64, bits=bits)
    kept, error = [r["kept_attention"] for r in rows], [r["rel_error"] for r in rows]
    assert kept == sorted(kept) and kept[0] > 0.02 and abs(kept[-1] - 1) < 1e-3      # 38 blocks: the last row lists them all
    assert error[0] > error[1] > error[2] and error[2] < 1e-2
