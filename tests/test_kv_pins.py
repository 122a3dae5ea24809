"""The key/value cache operators without a GPU: the record layout, the reference's own consistency, and the
arguments that every entry point refuses before it touches the device."""

import ctypes

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2312_01712_b200 as lib
from paper_2312_01712_b200 import build as libbuild


@pytest.fixture(scope="module")
def L():
    libbuild.build()
    from paper_2312_01712_b200 import kv
    return kv._load()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_record_layout_is_a_permutation_and_round_trips(d):
    key, val = ref.code_positions(d)
    assert sorted(key.ravel()) == list(range(16 * d)) and sorted(val.ravel()) == list(range(16 * d))
    rng = np.random.default_rng(d)
    k, v = rng.standard_normal((2, 3, 2, 32, d))
    v[0, 0, 3] = 0.25                                  # a constant group: scale 0
    rec = ref.encode_records(k, v)
    for x, y, (u, s, z) in zip((k, v), ref.held_values(rec, d), ref.decode_records(rec, d)):
        s = s.reshape(x.shape)
        assert u.min() >= 0 and u.max() == 15
        # half a step, and what rounding the scale and the offset to 11 bits leaves out at the ends of the range
        assert np.all(np.abs(x - y) <= 0.5 * s + 16 * s * 2.0 ** -11 + np.abs(x) * 2.0 ** -10 + 1e-6)
    assert np.array_equal(ref.held_values(rec, d)[1][0, 0, 3], np.full(d, 0.25))


def cache(L, **kw):
    base = dict(format=lib.IVFPQ_KV_INT4, d=128, nheads=2, page=64, npages=10, records=1 << 20, bounds=1 << 21, bounds_scale=1 << 22,
                k=None, v=None)
    base.update(kw)
    c = lib.ivfpq_kv_cache_t()
    for n, x in base.items():
        if n in ("k_stride", "v_stride"):
            getattr(c, n)[:] = x
        else:
            setattr(c, n, x)
    return c


def batch(**kw):
    base = dict(nreq=3, max_blocks=8, table_stride=8, block_table=1 << 16, seq_len=1 << 16, q_start=None)
    base.update(kw)
    b = lib.ivfpq_kv_batch_t()
    for n, x in base.items():
        setattr(b, n, x)
    return b


def calls(L, c, b, ntok=3, dtype=lib.IVFPQ_KV_BF16, p=1 << 24, ts=256, hs=128, nq=4, nsel=4, sink=1, local=1, blocks=None, att_sel=0,
          scale=0.1, out=1 << 24, ws=1 << 23, wsb=None):
    wsb = L.ivfpq_kv_workspace_bytes(128) if wsb is None else wsb
    rc, rb = (ctypes.byref(c) if c is not None else None), (ctypes.byref(b) if b is not None else None)
    return dict(
        append=L.ivfpq_kv_append(rc, rb, ntok, dtype, p, ts, hs, p, ts, hs, ws, wsb, None),
        read=L.ivfpq_kv_read(rc, rb, ntok, dtype, out, out, ws, wsb, None),
        select=L.ivfpq_kv_select(rc, rb, ntok, dtype, p, ts, hs, nq, nsel, sink, local, out, ws, wsb, None),
        attend=L.ivfpq_kv_attend(rc, rb, ntok, dtype, p, ts, hs, nq, scale, blocks, att_sel, out, None, ws, wsb, None))


BAD, UNS, WS = lib.IVFPQ_ERR_INVALID_ARGUMENT, lib.IVFPQ_ERR_UNSUPPORTED, lib.IVFPQ_ERR_WORKSPACE
ALL = ("append", "read", "select", "attend")


@pytest.mark.parametrize("ckw,bkw,kw,code,which", [
    (None, {}, {}, BAD, ALL), ({}, None, {}, BAD, ALL),
    (dict(d=96), {}, {}, UNS, ALL), (dict(d=0), {}, {}, UNS, ALL), (dict(page=48), {}, {}, UNS, ALL),
    (dict(page=256), {}, {}, UNS, ALL), (dict(format=3), {}, {}, UNS, ALL), (dict(nheads=0), {}, {}, BAD, ALL),
    (dict(npages=0), {}, {}, BAD, ALL), (dict(npages=1 << 31), {}, {}, UNS, ALL), (dict(nheads=1025), {}, {}, UNS, ("append", "read")),
    (dict(records=None), {}, {}, BAD, ALL), (dict(records=(1 << 20) + 8), {}, {}, BAD, ALL),
    (dict(bounds=None), {}, {}, BAD, ALL), (dict(bounds=None, bounds_scale=None), {}, {}, BAD, ("select",)),
    (dict(format=lib.IVFPQ_KV_BF16), {}, {}, BAD, ALL),
    (dict(format=lib.IVFPQ_KV_BF16, k=1 << 20, v=1 << 20, k_stride=(4, 8, 8), v_stride=(8, 8, 8)), {}, {}, BAD, ALL),
    (dict(format=lib.IVFPQ_KV_FP16, k=1 << 20, v=1 << 20, k_stride=(8, 8, 8), v_stride=(8, 8, 8)), {}, {}, UNS, ALL),   # bf16 tokens
    ({}, dict(nreq=0), {}, BAD, ALL), ({}, dict(max_blocks=0), {}, BAD, ALL), ({}, dict(table_stride=7), {}, BAD, ALL),
    ({}, dict(block_table=None), {}, BAD, ALL), ({}, dict(seq_len=None), {}, BAD, ALL), ({}, dict(block_table=(1 << 16) + 2), {}, BAD, ALL),
    ({}, dict(max_blocks=lib.IVFPQ_KV_MAX_BLOCKS + 1, table_stride=1 << 20), {}, UNS, ("select",)),
    ({}, dict(max_blocks=(1 << 24) + 1, table_stride=1 << 30), {}, UNS, ALL),
    ({}, {}, dict(ntok=4), BAD, ALL), ({}, {}, dict(ntok=0), BAD, ALL), ({}, dict(q_start=1 << 16), dict(ntok=(1 << 20) + 1), UNS, ALL),
    ({}, {}, dict(dtype=lib.IVFPQ_KV_INT4), UNS, ALL), ({}, {}, dict(dtype=7), UNS, ALL),
    ({}, {}, dict(p=None), BAD, ("append", "select", "attend")), ({}, {}, dict(p=(1 << 24) + 2), BAD, ("append", "select", "attend")),
    ({}, {}, dict(ts=100), BAD, ("append", "select", "attend")), ({}, {}, dict(hs=12), BAD, ("append", "select", "attend")),
    ({}, {}, dict(nq=5), BAD, ("select", "attend")), ({}, {}, dict(nq=0), BAD, ("select", "attend")),
    ({}, {}, dict(nq=2 * lib.IVFPQ_KV_MAX_GROUP + 2), UNS, ("select", "attend")),
    ({}, {}, dict(out=None), BAD, ("read", "select", "attend")), ({}, {}, dict(out=(1 << 24) + 2), BAD, ("read", "select", "attend")),
    ({}, {}, dict(nsel=0), BAD, ("select",)), ({}, {}, dict(local=0), BAD, ("select",)), ({}, {}, dict(sink=-1), BAD, ("select",)),
    ({}, {}, dict(sink=3, local=2), BAD, ("select",)), ({}, {}, dict(nsel=lib.IVFPQ_KV_MAX_SELECT + 1), UNS, ("select",)),
    ({}, {}, dict(att_sel=3), BAD, ("attend",)), ({}, {}, dict(blocks=1 << 24), BAD, ("attend",)),
    ({}, {}, dict(blocks=1 << 24, att_sel=lib.IVFPQ_KV_MAX_SELECT + 1), UNS, ("attend",)),
    ({}, {}, dict(scale=float("nan")), BAD, ("attend",)), ({}, {}, dict(scale=float("inf")), BAD, ("attend",)),
    ({}, {}, dict(ws=None), BAD, ALL), ({}, {}, dict(ws=(1 << 23) + 128), WS, ALL), ({}, {}, dict(wsb=100), WS, ALL),
])
def test_refusals(L, ckw, bkw, kw, code, which):
    got = calls(L, None if ckw is None else cache(L, **ckw), None if bkw is None else batch(**bkw), **kw)
    assert {n: got[n] for n in which} == {n: code for n in which}


def test_refusals_of_read_bounds_status_and_workspace(L):
    n = L.ivfpq_kv_workspace_bytes(128)
    assert n % 256 == 0 and n >= lib.IVFPQ_KV_WORKSPACE_ZERO
    assert L.ivfpq_kv_workspace_bytes(96) == 0 and lib.ivfpq_kv_workspace_bytes(64) > 0
    p, c = 1 << 24, cache(L)
    f = lambda c=c, pages=p, k=1, u=p, lo=p, ws=p, wsb=n: L.ivfpq_kv_read_bounds(ctypes.byref(c), pages, k, u, lo, ws, wsb, None)  # noqa: E731
    assert f(c=cache(L, bounds=None, bounds_scale=None)) == BAD
    assert f(pages=None) == BAD and f(k=0) == BAD and f(u=None) == BAD and f(lo=p + 8) == BAD and f(ws=None) == BAD
    assert f(wsb=n - 1) == WS and f(k=(1 << 24) + 1) == UNS
    assert L.ivfpq_kv_status(None, None) == BAD and L.ivfpq_kv_status(p + 8, None) == WS


def test_the_binding_refuses_tensors_of_the_wrong_kind():
    with pytest.raises(ValueError):
        lib.KvCacheHandle()
    with pytest.raises(ValueError):
        lib.KvCacheHandle(records=torch.zeros(2, 2, 4, 18 * 128, dtype=torch.uint8))      # not on a device
    with pytest.raises(ValueError):
        lib.KvCacheHandle(k=torch.zeros(2, 2, 64, 128), v=torch.zeros(2, 2, 64, 128))
    with pytest.raises(ValueError):
        lib.KvBatchHandle(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
