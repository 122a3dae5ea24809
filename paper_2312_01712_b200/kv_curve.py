"""Kept attention against the number of blocks listed, the form in which the paper's discussion brings similarity search to a
language model's attention (`python -m paper_2312_01712_b200.kv_curve --context 32768 --blocks 8,16,32,64`).

Builds a paged key/value cache the way a server does (a prompt appended in chunks, then one token per request), and for every number of blocks
runs a decode step: append, select, attend over the lists.  Prints one JSON line per number with the share of the softmax mass
that the listed blocks hold, the relative error of the output against attention over the whole cache, and device times."""

from __future__ import annotations

import argparse
import json

import torch

from . import binding, kv as lib


def synthetic(nreq: int, context: int, hkv: int, group: int, d: int, dtype, seed: int, device: str):
    """Keys with a few wide channels and a drift per stretch of text; queries that look back at some of the stretches."""
    g = torch.Generator(device).manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device=device)  # noqa: E731
    stretch = 96
    topics = rnd(nreq, context // stretch + 1, hkv, d)
    wide = 0.6 + 2.0 * torch.rand(hkv, d, generator=g, device=device) ** 6
    at = torch.arange(context, device=device) // stretch
    k = (0.7 * rnd(nreq, context, hkv, d) + 1.2 * topics[:, at]) * wide
    v = 0.7 * rnd(nreq, context, hkv, d)
    pick = torch.randint(0, topics.shape[1], (nreq, 4), generator=g, device=device)
    look = topics[torch.arange(nreq, device=device)[:, None], pick].mean(1)
    q = (1.5 * look[:, :, None] + 0.6 * rnd(nreq, hkv, group, d)).flatten(1, 2)
    return k.to(dtype), v.to(dtype), q.to(dtype)


def fill(cache: "lib.KvCacheHandle", table: torch.Tensor, k: torch.Tensor, v: torch.Tensor, chunk: int = 4096) -> None:
    """Appends all requests' keys and values [requests, tokens, heads, d] in chunks of tokens, as prompts arrive."""
    nreq, n = k.shape[:2]
    for lo in range(0, n, chunk):
        hi = min(n, lo + chunk)
        lens = torch.full((nreq,), hi, dtype=torch.int32, device=k.device)
        start = torch.arange(nreq + 1, dtype=torch.int32, device=k.device) * (hi - lo)
        lib.ivfpq_kv_append(cache, lib.KvBatchHandle(table, lens, start), k[:, lo:hi].flatten(0, 1), v[:, lo:hi].flatten(0, 1))


def timed(step, iters: int = 20) -> float:
    """Median device time of `step` in microseconds, L2 flushed in between."""
    flush = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        step()
    evs = []
    for _ in range(iters):
        flush.zero_()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        step()
        b.record()
        evs.append((a, b))
    torch.cuda.synchronize()
    return sorted(a.elapsed_time(b) for a, b in evs)[iters // 2] * 1e3


def curve(blocks, context: int = 32768, nreq: int = 4, hkv: int = 8, group: int = 4, d: int = 128, page: int = 64, bits: int = 4,
          dtype=torch.bfloat16, seed: int = 0, device: str = "cuda"):
    k, v, q = synthetic(nreq, context, hkv, group, d, dtype, seed, device)
    cols = -(-context // page)
    cache = lib.KvCacheHandle.empty(nreq * cols, hkv, page, d, dtype=None if bits == 4 else dtype, device=device)
    g = torch.Generator(device).manual_seed(seed + 1)
    table = torch.randperm(nreq * cols, generator=g, device=device).to(torch.int32).view(nreq, cols)
    fill(cache, table, k[:, :-1], v[:, :-1])
    # the decode step: the last token of every request
    batch = lib.KvBatchHandle(table, torch.full((nreq,), context, dtype=torch.int32, device=device))
    last_k, last_v = k[:, -1].contiguous(), v[:, -1].contiguous()
    lse = torch.empty(nreq, hkv * group, dtype=torch.float32, device=device)

    def whole():
        lib.ivfpq_kv_append(cache, batch, last_k, last_v)
        return lib.ivfpq_kv_attend(cache, batch, q, lse=lse)

    out = whole().float()
    all_lse = lse.clone()
    us = timed(whole)
    rows = []
    for n in blocks:
        def step():
            lib.ivfpq_kv_append(cache, batch, last_k, last_v)
            lists = lib.ivfpq_kv_select(cache, batch, q, n, nsink=1, nlocal=2)
            return lib.ivfpq_kv_attend(cache, batch, q, blocks=lists, lse=lse)

        some = step().float()
        rows.append(dict(blocks=n, of=cols, kept_attention=float((lse - all_lse).exp().mean()),
                         rel_error=float((some - out).norm() / out.norm()), step_us=timed(step), whole_us=us))
    if lib.ivfpq_kv_status(cache) != binding.IVFPQ_OK:
        raise binding.IvfpqError(binding.IVFPQ_ERR_DEVICE_FLAG, "kv_curve")
    return rows


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--context", type=int, default=32768)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--blocks", default="8,16,32,64,128")
    ap.add_argument("--page", type=int, default=64)
    ap.add_argument("--bits", type=int, default=4, choices=(4, 16))
    a = ap.parse_args()
    for row in curve([int(x) for x in a.blocks.split(",")], a.context, a.requests, page=a.page, bits=a.bits):
        print(json.dumps(row), flush=True)


if __name__ == "__main__":
    main()
