"""Float64 / plain-list oracle of the serving calls: pages, rows and attention of one new token over a paged cache.

Written from the definitions in include/lightkv.h, request by request; shares no code with the library.
"""
from __future__ import annotations

import math

import numpy as np

COUNT, PAGE, NO_PAGES = 8, 16, 32


def assign_pages(held, seq_len, add, table, free_pages, n_free, page_size, n_slots=0, slot_stride=0):
    """Lists in, a dict out: seq_len_out, table, free_pages, n_free, slot_map, slot_start, status.  One request after the other."""
    table, memory = [list(r) for r in table], list(free_pages)
    batch, width, n_pages, status = len(seq_len), len(table[0]), len(memory), 0
    room = width * page_size

    def pages(n):
        return -(-n // page_size)

    h, w = [], []
    for b in range(batch):
        n = max(held[b], 0) if held is not None else 0
        if n > room:
            n, status = room, status | COUNT
        h.append(n)
        w.append(0 if seq_len[b] < 0 else seq_len[b] + add)
    if not 0 <= n_free <= n_pages:
        n_free, status = min(max(n_free, 0), n_pages), status | COUNT
    stack = memory[:n_free]
    for b in range(batch):
        if w[b] < h[b]:
            stack += table[b][pages(w[b]):pages(h[b])]
    height, asked, length, served = len(stack), 0, [], []
    for b in range(batch):
        more = pages(w[b]) - pages(h[b])
        ok = w[b] <= room
        if not ok:
            status |= COUNT
        elif more > 0:
            asked += more
            ok = asked <= height
            if not ok:
                status |= NO_PAGES
        if ok and more > 0:
            for j in range(more):
                table[b][pages(h[b]) + j] = stack.pop()
        served.append(ok)
        length.append(seq_len[b] if seq_len[b] < 0 else w[b] if ok else h[b])
    if len(stack) > n_pages:
        stack, status = stack[:n_pages], status | COUNT
    memory[n_free:len(stack)] = stack[n_free:]
    slots, start = [-1] * n_slots, [0]
    for b in range(batch):
        fresh = max(w[b] - h[b], 0)
        for i in range(fresh):
            at = start[-1] + i if not slot_stride else b * slot_stride + i if i < slot_stride else n_slots
            if at >= n_slots:
                status |= COUNT if n_slots else 0
                break
            if served[b]:
                p = h[b] + i
                page = table[b][p // page_size]
                if 0 <= page < n_pages:
                    slots[at] = page * page_size + p % page_size
                else:
                    status |= PAGE
        start.append(start[-1] + fresh)
    return dict(seq_len_out=length, table=table, free_pages=memory, n_free=len(stack), slot_map=slots,
                slot_start=[min(v, 2 ** 31 - 1) for v in start], status=status)


def append_kv(k_new, v_new, k_cache, v_cache, slot_map):
    """[T, Hkv, dh] rows into copies of [pages, Hkv, page_size, dh] caches; returns (k, v, status)."""
    k, v, status = k_cache.copy(), v_cache.copy(), 0
    n_pages, page_size = k.shape[0], k.shape[2]
    for t, slot in enumerate(slot_map):
        if slot >= n_pages * page_size:
            status |= PAGE
        elif slot >= 0:
            k[slot // page_size, :, slot % page_size] = k_new[t]
            v[slot // page_size, :, slot % page_size] = v_new[t]
    return k, v, status


def cache_rows(cache, pages, n, page_size):
    """Rows 0 .. n - 1 of a request, [Hkv, n, dh], and which of them are there."""
    keys = np.arange(n)
    page = np.asarray(pages, dtype=np.int64)[keys // page_size] if n else np.zeros(0, np.int64)
    there = (page >= 0) & (page < cache.shape[0])
    rows = cache[np.where(there, page, 0), :, keys % page_size]           # [n, Hkv, dh]
    return np.moveaxis(rows, 1, 0).astype(np.float64), there


def with_new_row(k, v, k_new, v_new, slot=0):
    """A request's rows [Hkv, n, dh] with those of the new token, [Hkv, dh], as the last ones; slot < 0: there is no new token."""
    k, v = k.copy(), v.copy()
    if slot >= 0 and k.shape[1] > 0:
        k[:, -1], v[:, -1] = k_new, v_new
    return k, v


def attend(q, k, v, there, scale):
    """One request: q [H, dh], k / v [Hkv, n, dh] -> out [H, dh], lse [H], sum_j p_j |v_j| [H, dh], max_j sum_d |q_d k_jd| [H]."""
    heads, dh = q.shape
    group = heads // k.shape[0]
    out, mass, lse, span = np.zeros((heads, dh)), np.zeros((heads, dh)), np.full(heads, -math.inf), np.zeros(heads)
    if not there.any():
        return out, lse, mass, span
    for h in range(heads):
        kk, vv, x = k[h // group][there], v[h // group][there], q[h].astype(np.float64)
        s = scale * (kk @ x)
        top = s.max()
        e = np.exp(s - top)
        total = e.sum()
        out[h] = (e / total) @ vv
        mass[h] = (e / total) @ np.abs(vv)
        lse[h] = top + math.log(total)
        span[h] = scale * (np.abs(kk) @ np.abs(x)).max()
    return out, lse, mass, span
